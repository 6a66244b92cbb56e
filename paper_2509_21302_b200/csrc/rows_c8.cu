// The row operators of the rotation-free 8-bit path: quantizer, its inverse, RMS norm with the residual's addition, and the norm with its
// output in 8 bits.  Per row, all in fp32:
//   h[k] = x[k] + r[k]                             (stored, if asked for, rounded to the type; what follows uses the unrounded sum)
//   y[k] = (h[k] * rstd) * gamma[k],  rstd = 1 / sqrt(sum h^2 / K + eps)
//   amax = max(max_k |y[k]|, 1e-8),  scale = amax / 127,  q[k] = round(y[k] * (127 * (1 / amax))), half to even
// Every one of these operations is rounded to fp32 by itself, so that the codes of given y are those of the formula in plain fp32 arithmetic,
// bit for bit.  That shows where elements of 16 bits lie exactly between two codes: with the product rounded straight to the integer (one
// multiply-add) other codes came out there.
// They move K e bytes in, K (and K e) out, against a handful of operations per element: HBM bounds them from a few hundred rows on,
// and latency (one load, two reductions, one store) below.  A row therefore stays in registers between its one load and its one store.
#include "element.cuh"
#include "qvggt_internal.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace {

using element::Chunk;
using element::store8;

constexpr int WARP_ROWS = 8;               // rows of a CTA where a warp takes a row
constexpr int MAX_THREADS = 1024;

struct Rows {
    const void *x, *r;                     // r: residual or nullptr
    void *h, *y;                           // or nullptr
    signed char *q;
    float *scales;
    const float *gamma;
    long long ldx, ldr, ldh, ldy, ldq;     // in elements
    float eps;
    int M, K;
    bool wide_h, wide_y, wide_q;           // every row of it begins on a 16-byte boundary (q: 8 bytes)
};

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Sum / largest of a value per thread over the row's threads: a warp, or the CTA (every thread gets the result; `part` holds 32 words).
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float *part)
{
    v = warp_sum(v);
    if (WARP) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum((threadIdx.x & 31) < (blockDim.x >> 5) ? part[threadIdx.x & 31] : 0.0f);
}

template <bool WARP>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *part)
{
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if (WARP) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    return __reduce_max_sync(0xFFFFFFFFu, (threadIdx.x & 31) < (blockDim.x >> 5) ? part[threadIdx.x & 31] : 0u);
}

// A row's eight-element chunks t, t + threads, ... belong to thread t: CHUNKS of them in registers, or (CHUNKS = 0, rows too long for
// that) any number, read again for every pass.  WIDE: every row of x, r and gamma begins on a 16-byte boundary.
template <class T, bool NORM, bool QUANT, bool WARP, bool WIDE, int CHUNKS>
__global__ void __launch_bounds__(WARP ? WARP_ROWS * 32 : MAX_THREADS) rows_kernel(const __grid_constant__ Rows p)
{
    __shared__ float part_sum[32];
    __shared__ uint32_t part_max[32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const long long m = WARP ? (long long)blockIdx.x * WARP_ROWS + (threadIdx.x >> 5) : blockIdx.x;
    if (m >= p.M) return;                                                    // (whole warps)
    const int t = WARP ? threadIdx.x & 31 : threadIdx.x, threads = WARP ? 32 : blockDim.x;
    const int chunks = (p.K + 7) / 8;
    const T *x = static_cast<const T *>(p.x) + m * p.ldx;
    const T *r = p.r ? static_cast<const T *>(p.r) + m * p.ldr : nullptr;

    auto add = [](float (&v)[8], const float (&a)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += a[i];
    };
    auto store_sum = [&](int c, const float (&v)[8]) {
        const int k = 8 * c, n = p.K - k;
        if (NORM && p.h) store8(static_cast<T *>(p.h) + m * p.ldh + k, p.wide_h && n >= 8, n, v);
    };
    float rstd = 1.0f;
    auto normalize = [&](int c, const Chunk<float, WIDE> &gamma, float (&v)[8]) {
        float g[8];
        gamma.get(p.gamma + 8 * c, p.K - 8 * c, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (v[i] * rstd) * g[i];
    };
    float inv = 0.0f;
    bool finite = true;
    auto store_row = [&](int c, const float (&v)[8]) {
        const int k = 8 * c, n = p.K - k;
        if constexpr (!QUANT) {
            store8(static_cast<T *>(p.y) + m * p.ldy + k, p.wide_y && n >= 8, n, v);
        } else {
            uint32_t u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(__fadd_rn(__fmul_rn(v[i], inv), 12582912.0f));   // 1.5 * 2^23: the code is the low byte
            uint32_t lo = __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
            uint32_t hi = __byte_perm(__byte_perm(u[4], u[5], 0x0040), __byte_perm(u[6], u[7], 0x0040), 0x5410);
            if (!finite) lo = hi = 0;
            signed char *q = p.q + m * p.ldq + k;
            if (p.wide_q && n >= 8) {
                *reinterpret_cast<uint2 *>(q) = make_uint2(lo, hi);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n) q[i] = static_cast<signed char>((i < 4 ? lo : hi) >> (8 * (i & 3)));
            }
        }
    };
    auto square = [](const float (&v)[8]) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __fmaf_rn(v[i], v[i], s);
        return s;
    };
    auto largest = [](const float (&v)[8], uint32_t a) {                     // on the bits: NaN is the largest of all
#pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        return a;
    };
    auto finish_sum = [&](float s) { rstd = __frsqrt_rn(__fdiv_rn(row_sum<WARP>(s, part_sum), (float)p.K) + p.eps); };
    auto finish_max = [&](uint32_t a) {
        a = row_max<WARP>(a, part_max);
        finite = a < 0x7F800000u;
        const float amax = fmaxf(__uint_as_float(a), 1e-8f);
        inv = __fmul_rn(__frcp_rn(amax), 127.0f);
        if (t == 0) p.scales[m] = finite ? __fdiv_rn(amax, 127.0f) : __uint_as_float(0x7FC00000u);
    };

    if constexpr (CHUNKS > 0) {
        // Everything that is read is on its way before the first value is used (a chunk at a time, with the choice of wide and narrow
        // loads in between, each load waited for the one before it: 43 968 x 4096 bf16, norm and codes 185 us).
        Chunk<T, WIDE> cx[CHUNKS], cr[CHUNKS];
        Chunk<float, WIDE> cg[CHUNKS];
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int c = t + i * threads;
            cx[i].clear();
            if (c < chunks) cx[i].fetch(x + 8 * c, p.K - 8 * c);
        }
        if (NORM && r) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int c = t + i * threads;
                cr[i].clear();
                if (c < chunks) cr[i].fetch(r + 8 * c, p.K - 8 * c);
            }
        }
        if (NORM) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int c = t + i * threads;
                cg[i].clear();
                if (c < chunks) cg[i].fetch(p.gamma + 8 * c, p.K - 8 * c);
            }
        }
        float v[CHUNKS][8];
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) cx[i].get(x + 8 * (t + i * threads), p.K - 8 * (t + i * threads), v[i]);
        if (NORM && r) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                float a[8];
                cr[i].get(r + 8 * (t + i * threads), p.K - 8 * (t + i * threads), a);
                add(v[i], a);
            }
        }
        if (NORM) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) s += square(v[i]);
            if (p.h) {
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i)
                    if (t + i * threads < chunks) store_sum(t + i * threads, v[i]);
            }
            finish_sum(s);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) normalize(t + i * threads, cg[i], v[i]);
        }
        if (QUANT) {
            uint32_t a = 0;
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) a = largest(v[i], a);
            finish_max(a);
        }
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
            if (t + i * threads < chunks) store_row(t + i * threads, v[i]);
    } else {
        float v[8];
        auto load = [&](int c) {
            const int n = p.K - 8 * c;
            Chunk<T, WIDE> cx, cr;
            cx.fetch(x + 8 * c, n);
            if (NORM && r) cr.fetch(r + 8 * c, n);
            cx.get(x + 8 * c, n, v);
            if (NORM && r) {
                float a[8];
                cr.get(r + 8 * c, n, a);
                add(v, a);
            }
        };
        auto normalized = [&](int c) {
            if (!NORM) return;
            Chunk<float, WIDE> cg;
            cg.fetch(p.gamma + 8 * c, p.K - 8 * c);
            normalize(c, cg, v);
        };
        if (NORM) {
            float s = 0.0f;
            for (int c = t; c < chunks; c += threads) { load(c); s += square(v); }
            finish_sum(s);
        }
        if (QUANT) {
            uint32_t a = 0;
            for (int c = t; c < chunks; c += threads) { load(c); normalized(c); a = largest(v, a); }
            finish_max(a);
        }
        // the sum is stored last: it may take the place of x or r, which every pass reads
        for (int c = t; c < chunks; c += threads) { load(c); store_sum(c, v); normalized(c); store_row(c, v); }
    }
}

// v = q * scale, eight codes per thread, DEQ_ROWS rows of them at once.  A CTA is `columns` threads wide along a row, 256 / columns rows high.
constexpr int DEQ_ROWS = 4;
template <class T>
__global__ void __launch_bounds__(256) dequantize_kernel(const signed char *q, long long ldq, const float *scales, T *y, long long ldy, int M, int K, int columns, bool wide_q, bool wide_y)
{
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int high = 256 / columns, row = threadIdx.x / columns;
    const int k = 8 * (blockIdx.y * columns + threadIdx.x % columns), n = K - k;
    const long long m0 = (long long)blockIdx.x * (high * DEQ_ROWS) + row;
    if (row >= high || n <= 0) return;
    uint2 w[DEQ_ROWS];
    float s[DEQ_ROWS];
#pragma unroll
    for (int i = 0; i < DEQ_ROWS; ++i) {
        const long long m = m0 + i * high;
        w[i] = make_uint2(0, 0);
        s[i] = 0.0f;
        if (m < M) {
            const signed char *src = q + m * ldq + k;
            s[i] = scales[m];
            if (wide_q && n >= 8) w[i] = *reinterpret_cast<const uint2 *>(src);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) (j < 4 ? w[i].x : w[i].y) |= static_cast<uint32_t>(static_cast<unsigned char>(src[j])) << (8 * (j & 3));
        }
    }
#pragma unroll
    for (int i = 0; i < DEQ_ROWS; ++i) {
        const long long m = m0 + i * high;
        if (m >= M) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = static_cast<float>(static_cast<signed char>((j < 4 ? w[i].x : w[i].y) >> (8 * (j & 3)))) * s[i];
        store8(y + m * ldy + k, wide_y && n >= 8, n, v);
    }
}

template <class Kernel, class... Args>
cudaError_t launch(Kernel kernel, dim3 grid, int threads, cudaStream_t st, Args... args)
{
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <class T, bool NORM, bool QUANT, bool WIDE>
cudaError_t dispatch(const Rows &p, cudaStream_t st)
{
    const int chunks = (p.K + 7) / 8;
    if (chunks <= 64) {
        const dim3 grid((p.M - 1) / WARP_ROWS + 1);
        if (chunks <= 32) return launch(rows_kernel<T, NORM, QUANT, true, WIDE, 1>, grid, WARP_ROWS * 32, st, p);
        return launch(rows_kernel<T, NORM, QUANT, true, WIDE, 2>, grid, WARP_ROWS * 32, st, p);
    }
    if (chunks <= 2 * MAX_THREADS) return launch(rows_kernel<T, NORM, QUANT, false, WIDE, 2>, dim3(p.M), (chunks + 63) / 64 * 32, st, p);
    return launch(rows_kernel<T, NORM, QUANT, false, WIDE, 0>, dim3(p.M), MAX_THREADS, st, p);
}

template <bool NORM, bool QUANT>
cudaError_t by_type(int type, bool wide, const Rows &p, cudaStream_t st)
{
    if (type == QVGGT_BF16) return wide ? dispatch<__nv_bfloat16, NORM, QUANT, true>(p, st) : dispatch<__nv_bfloat16, NORM, QUANT, false>(p, st);
    if (type == QVGGT_FP16) return wide ? dispatch<__half, NORM, QUANT, true>(p, st) : dispatch<__half, NORM, QUANT, false>(p, st);
    return wide ? dispatch<float, NORM, QUANT, true>(p, st) : dispatch<float, NORM, QUANT, false>(p, st);
}

int bytes_of(int type) { return type == QVGGT_FP32 ? 4 : 2; }

bool rows_aligned(const void *p, long long ld, int bytes, int boundary)
{
    return (reinterpret_cast<uintptr_t>(p) % boundary) == 0 && (ld * bytes) % boundary == 0;
}

}  // namespace

cudaError_t qvggt_launch_rows(int type, const void *X, long long ldx, const void *R, long long ldr, int M, int K, const float *gamma, float eps,
                              void *H, long long ldh, void *Y, long long ldy, signed char *Xq8, long long ldq, float *scales, cudaStream_t st)
{
    const int e = bytes_of(type);
    Rows p = {};
    p.x = X; p.r = R; p.h = H; p.y = Y; p.q = Xq8; p.scales = scales; p.gamma = gamma;
    p.ldx = ldx; p.ldr = ldr; p.ldh = ldh; p.ldy = ldy; p.ldq = ldq;
    p.eps = eps; p.M = M; p.K = K;
    const bool wide = rows_aligned(X, ldx, e, 16) && (!R || rows_aligned(R, ldr, e, 16)) && rows_aligned(gamma, 0, 4, 16);
    p.wide_h = rows_aligned(H, ldh, e, 16);
    p.wide_y = rows_aligned(Y, ldy, e, 16);
    p.wide_q = rows_aligned(Xq8, ldq, 1, 8);
    if (!gamma) return by_type<false, true>(type, wide, p, st);
    return Xq8 ? by_type<true, true>(type, wide, p, st) : by_type<true, false>(type, wide, p, st);
}

cudaError_t qvggt_launch_dequantize(int type, const signed char *Xq8, long long ldq, const float *scales, int M, int K, void *Y, long long ldy, cudaStream_t st)
{
    const bool wide_q = rows_aligned(Xq8, ldq, 1, 8), wide_y = rows_aligned(Y, ldy, bytes_of(type), 16);
    const int chunks = (K + 7) / 8, wide = (chunks + 255) / 256, columns = (chunks + wide - 1) / wide, high = 256 / columns * DEQ_ROWS;
    const dim3 grid((M - 1) / high + 1, wide);
    if (type == QVGGT_BF16) return launch(dequantize_kernel<__nv_bfloat16>, grid, 256, st, Xq8, ldq, scales, static_cast<__nv_bfloat16 *>(Y), ldy, M, K, columns, wide_q, wide_y);
    if (type == QVGGT_FP16) return launch(dequantize_kernel<__half>, grid, 256, st, Xq8, ldq, scales, static_cast<__half *>(Y), ldy, M, K, columns, wide_q, wide_y);
    return launch(dequantize_kernel<float>, grid, 256, st, Xq8, ldq, scales, static_cast<float *>(Y), ldy, M, K, columns, wide_q, wide_y);
}
