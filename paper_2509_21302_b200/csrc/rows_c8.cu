// The row operators of the rotation-free 8-bit path: quantizer, its inverse, RMS norm with the residual's addition, and the norm with its
// output in 8 bits.  Per row, all in fp32:
//   h[k] = x[k] + r[k]                             (stored, if asked for, rounded to the type; what follows uses the unrounded sum)
//   y[k] = (h[k] * rstd) * gamma[k],  rstd = 1 / sqrt(sum h^2 / K + eps)
//   amax = max(max_k |y[k]|, 1e-8),  scale = amax / 127,  q[k] = round(y[k] * (127 * (1 / amax))), half to even
// In the quantizer every one of these operations is rounded to fp32 by itself, so that its codes are those of the formula in plain fp32
// arithmetic, bit for bit (behind the norm they are taken from h gamma, see Row).  That shows where elements of 16 bits lie exactly between two codes: with the product rounded straight to the
// integer (one multiply-add) other codes came out there.
// They move K e bytes in, K (and K e) out, against a handful of operations per element: HBM bounds them from a few hundred rows on,
// and latency (one load, one reduction, one store) below.  A row therefore stays in registers between its one load and its one store.
#include "element.cuh"
#include "gemm_common.cuh"
#include "qvggt_internal.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace {

using element::ALIGNED;
using element::ANY;
using element::Chunk;
using element::REGULAR;
using element::store8;
using element::store16;

constexpr int SHORT_THREADS = 256;         // of a CTA where a warp, or a part of one, takes a row
constexpr int MAX_THREADS = 1024;

struct Rows {
    const void *x, *r;                     // r: residual or nullptr
    void *h, *y;                           // or nullptr
    signed char *q;
    float *scales;
    const float *gamma;
    long long ldx, ldr, ldh, ldy, ldq;     // in elements
    float eps, one_over_k, floor_factor;   // floor_factor: 127 * (1 / 1e-8), every operation rounded
    int M, K;
    uint32_t zero;                         // 0, which the compiler cannot know (ptx::f32x2_one)
    bool wide_h, wide_y, wide_q, wide_g;   // every row of it begins on a 16-byte boundary (q: 8 bytes)
};

// Sum of s and largest of a over `lanes` neighbouring lanes (a power of two; all 32 take part).
template <bool SUM, bool MAX>
__device__ __forceinline__ void reduce_lanes(float &s, uint32_t &a, int lanes)
{
#pragma unroll
    for (int o = 16; o; o >>= 1)
        if (SUM && o < lanes) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (!MAX) return;
    if (lanes == 32) {
        a = __reduce_max_sync(0xFFFFFFFFu, a);
    } else {
#pragma unroll
        for (int o = 8; o; o >>= 1)
            if (o < lanes) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
    }
}

// The same over the row's threads: LANES of a warp, or (0) the CTA, which meets once for both (every thread gets the results; `part` holds 32
// pairs that no thread still reads from an earlier call: two meetings back is enough).
template <int LANES, bool SUM, bool MAX>
__device__ __forceinline__ void reduce_row(float &s, uint32_t &a, uint2 *part)
{
    reduce_lanes<SUM, MAX>(s, a, LANES ? LANES : 32);
    if (LANES) return;
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (lane == 0) part[threadIdx.x >> 5] = make_uint2(__float_as_uint(s), a);
    __syncthreads();
    const int lanes = warps <= 4 ? 4 : warps <= 8 ? 8 : 32, mine = lane & (lanes - 1);
    const uint2 v = mine < warps ? part[mine] : make_uint2(0, 0);
    s = __uint_as_float(v.x);
    a = v.y;
    reduce_lanes<SUM, false>(s, a, lanes);
    if (MAX) a = __reduce_max_sync(0xFFFFFFFFu, a);
}

// The same where a warp stands for two (see rows_kernel): s is the sum of the first, `more` that of the second, as many warps further on.  Where that
// makes more than 32, which no CTA holds, the two are added up before.  (The end is reduce_row's: as a function of both it moved registers in the launches
// with two chunks a thread, fp32 3000 x 2304 9.6 -> 10.2 us.)
template <bool SUM, bool MAX>
__device__ __forceinline__ void reduce_row_twofold(float &s, float more, uint32_t &a, uint2 *part)
{
    uint32_t none = 0;
    reduce_lanes<SUM, MAX>(s, a, 32);
    reduce_lanes<SUM, false>(more, none, 32);
    const int lane = threadIdx.x & 31, own = blockDim.x >> 5;
    const bool apart = SUM && own <= 16;
    if (SUM && !apart) s += more;
    if (lane == 0) {
        part[threadIdx.x >> 5] = make_uint2(__float_as_uint(s), a);
        if (apart) part[(threadIdx.x >> 5) + own] = make_uint2(__float_as_uint(more), 0);
    }
    __syncthreads();
    const int warps = apart ? 2 * own : own;
    const int lanes = warps <= 4 ? 4 : warps <= 8 ? 8 : 32, mine = lane & (lanes - 1);
    const uint2 v = mine < warps ? part[mine] : make_uint2(0, 0);
    s = __uint_as_float(v.x);
    a = v.y;
    reduce_lanes<SUM, false>(s, a, lanes);
    if (MAX) a = __reduce_max_sync(0xFFFFFFFFu, a);
}

// gamma of a chunk, n (> 0) elements from its first on.  It is aligned as good as always, whatever the rows are.
template <int LAYOUT>
__device__ __forceinline__ void load_gamma(const float *gamma, bool wide, int n, uint64_t (&g)[4])
{
    if (LAYOUT == REGULAR || wide) {
        Chunk<float, LAYOUT == ANY ? ALIGNED : LAYOUT> c;
        c.fetch(gamma, n);
        c.get(gamma, n, g);
    } else {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? __ldg(gamma + i) : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = ptx::f32x2_pack(f[2 * i], f[2 * i + 1]);
    }
}

// The arithmetic on a row's chunks of eight elements, two elements in a word; the same in both kernels below.
// With both, norm and codes, the values that go into the quantizer are w = h gamma: rstd is common to all of a row, so the codes of
// y = rstd w are those of w, and sum and maximum are taken in one pass (two passes with a meeting each: 43 968 x 4096 bf16 172 us).
template <class T, bool NORM, bool QUANT, int LAYOUT>
struct Row {
    float sum = 0.0f, sum_more = 0.0f;                   // sum_more: of the second half of a thread's chunks, where it has two halves
    uint32_t top = 0;                                    // bits of the largest magnitude: NaN is the largest of all
    uint64_t factor = 0;                                 // rstd, or what turns values into codes
    bool finite = true;

    // Takes values into sum and maximum; with codes behind the norm, v turns into w.
    __device__ __forceinline__ void take(uint64_t (&v)[4], const uint64_t (&g)[4], bool more = false)
    {
        if (NORM) {
            uint64_t s = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) s = ptx::f32x2_fma(v[i], v[i], s);
            float lo, hi;
            ptx::f32x2_unpack(s, lo, hi);
            if (more) sum_more += lo + hi;
            else sum += lo + hi;
        }
        if (QUANT) {
            float t = __uint_as_float(top);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (NORM) v[i] = ptx::f32x2_mul(v[i], g[i]);
                float lo, hi;
                ptx::f32x2_unpack(v[i], lo, hi);
                asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(t) : "f"(t), "f"(lo), "f"(hi));
            }
            top = __float_as_uint(t);
        }
    }
    // scale: where the row's goes, in one of its threads.
    __device__ __forceinline__ void end(const Rows &p, float *scale)
    {
        float rstd = 1.0f;
        if (NORM) rstd = rsqrtf(__fmaf_rn(sum, p.one_over_k, p.eps));
        if (QUANT) {
            const float t = __uint_as_float(top), amax = NORM ? __fmul_rn(t, rstd) : t;
            finite = top < 0x7F800000u && amax < __uint_as_float(0x7F800000u);       // neither infinite nor NaN
            const float f = amax >= 1e-8f ? __fmul_rn(__frcp_rn(t), 127.0f) : __fmul_rn(p.floor_factor, rstd);
            factor = ptx::f32x2_pack(f, f);
            if (scale) *scale = finite ? __fdiv_rn(fmaxf(amax, 1e-8f), 127.0f) : __uint_as_float(0x7FC00000u);
        } else {
            factor = ptx::f32x2_pack(rstd, rstd);
        }
    }
    // Results of a chunk, n elements from its first on, to y.
    __device__ __forceinline__ void store(T *y, bool wide, int n, const uint64_t (&v)[4], const uint64_t (&g)[4]) const
    {
        uint64_t z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = ptx::f32x2_mul(ptx::f32x2_mul(v[i], factor), g[i]);
        store8(y, LAYOUT == REGULAR || (wide && n >= 8), n, z);
    }
    __device__ __forceinline__ void store(signed char *q, bool wide, int n, const uint64_t (&v)[4], uint64_t one2) const
    {
        const uint64_t magic = ptx::f32x2_pack(12582912.0f, 12582912.0f);            // 1.5 * 2^23: the code is the low byte
        uint32_t u[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi;
            ptx::f32x2_unpack(ptx::f32x2_add_uncontracted(ptx::f32x2_mul(v[i], factor), magic, one2), lo, hi);
            u[2 * i] = __float_as_uint(lo);
            u[2 * i + 1] = __float_as_uint(hi);
        }
        uint32_t lo = __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
        uint32_t hi = __byte_perm(__byte_perm(u[4], u[5], 0x0040), __byte_perm(u[6], u[7], 0x0040), 0x5410);
        lo = finite ? lo : 0;
        hi = finite ? hi : 0;
        if (LAYOUT == REGULAR || (wide && n >= 8)) {
            *reinterpret_cast<uint2 *>(q) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) q[i] = static_cast<signed char>((i < 4 ? lo : hi) >> (8 * (i & 3)));
        }
    }
};

__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void async_wait(int pending)       // at most so many groups (0 or 1) still on their way
{
    if (pending <= 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else asm volatile("cp.async.wait_group 1;" ::: "memory");
}

// Rows in registers: thread t of a row's threads (LANES of a warp, or (0) the CTA) has the chunks t, t + threads, .. (CHUNKS of them).  Its
// threads take `turns` rows; while one is worked on, the next `depth` are on their way to shared memory, each warp fetching what it will
// read itself, so that no warp waits for another but in the reduction.  gamma comes from L1 for every row.
// A thread with four chunks stands for the threads t and t + threads of the `half` that a launch with two chunks a thread has (the first has its chunks
// 0 and 2; the last warp may have no second to stand for) and adds up as they would: which of the two launches takes a row, which goes by the
// number of rows, does not show in its results.
template <class T, bool NORM, bool QUANT, int LANES, int LAYOUT, int CHUNKS>
__global__ void __launch_bounds__(LANES ? SHORT_THREADS : MAX_THREADS, LANES ? (CHUNKS > 1 ? 3 : 4) : 1) rows_kernel(const __grid_constant__ Rows p, int turns, int depth)
{
    using C = Chunk<T, LAYOUT>;
    constexpr int GROUP = LANES ? LANES : 32, step = LANES ? SHORT_THREADS / GROUP : 1;      // lanes that fetch together; rows of a CTA at once
    constexpr uint32_t BLOCK = C::template GRANULES<GROUP> * 16, TENSOR = CHUNKS * BLOCK;
    extern __shared__ uint4 ring[];                                          // [group][depth][x, r][CHUNKS][granules]
    __shared__ uint2 part[2][32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int t = LANES ? threadIdx.x % GROUP : threadIdx.x, threads = LANES ? GROUP : blockDim.x, lane = threadIdx.x % GROUP;
    const bool residual = NORM && CHUNKS < 4 && p.r;                         // (with one, by_length() takes two chunks)
    const uint32_t slot_bytes = residual ? 2 * TENSOR : TENSOR, mine = ptx::smem_addr(ring) + threadIdx.x / GROUP * depth * slot_bytes;
    const long long first = (long long)blockIdx.x * turns * step, left = (p.M - first + step - 1) / step, m0 = first + (LANES ? threadIdx.x / GROUP : 0);
    const int rows = left < turns ? (int)left : turns;                       // turns of this CTA
    const int mine_rows = (int)min((long long)rows, (p.M - m0 + step - 1) / step);       // in the last, a group may have no row
    const int half = (p.K + 511) / 512 * 32, K_more = t + threads < half ? p.K : 0;      // (four chunks a thread only)
    auto length = [&](int i) { return CHUNKS == 4 && (i & 1) ? K_more : p.K; };          // of the row, as chunk i sees it
    int at[CHUNKS], n[CHUNKS];                                               // a chunk's first element, elements from there on
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        at[i] = 8 * (CHUNKS < 4 ? t + i * threads : t + (i & 1) * threads + (i >> 1) * half);
        n[i] = length(i) - at[i];
    }
    // rows of this thread's, one after the other: read, fetched ahead, written
    const T *x = static_cast<const T *>(p.x) + m0 * p.ldx, *r = static_cast<const T *>(p.r) + m0 * p.ldr, *x_ahead = x, *r_ahead = r;
    T *h = static_cast<T *>(p.h) + m0 * p.ldh, *y = static_cast<T *>(p.y) + m0 * p.ldy;
    signed char *q = p.q + m0 * p.ldq;
    float *scale = QUANT && t == 0 ? p.scales + m0 : nullptr;
    const uint64_t one2 = ptx::f32x2_one(p.zero);

    auto fetch = [&](int turn, uint32_t slot) {
        if (turn < mine_rows) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int a = at[i] - 8 * lane;                              // the group's first
                C::template fetch_async<GROUP>(slot + i * BLOCK, x_ahead + a, length(i) - a, lane);
                if (residual) C::template fetch_async<GROUP>(slot + TENSOR + i * BLOCK, r_ahead + a, length(i) - a, lane);
            }
            x_ahead += step * p.ldx;
            r_ahead += step * p.ldr;
        }
        async_commit();
    };
    for (int d = 0; d < depth; ++d) fetch(d, mine + d * slot_bytes);
    if (LAYOUT == REGULAR)                                                   // what no copy writes is read as zero
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
            for (uint32_t a = mine + i * BLOCK; n[i] <= 0 && a < mine + depth * slot_bytes; a += TENSOR)
#pragma unroll
                for (int j = 0; j < C::SPAN; ++j) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(a + (lane * C::SPAN + j) * 16), "r"(0) : "memory");
    uint32_t slot = mine;
    for (int turn = 0; turn < rows; ++turn) {
        Row<T, NORM, QUANT, LAYOUT> row;
        const bool here = turn < mine_rows;
        uint64_t v[CHUNKS][4];
        async_wait(depth - 1);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            C c;
            c.fetched(slot + i * BLOCK, lane);
            c.get(x + at[i], n[i], v[i]);
            if (residual) {
                uint64_t a[4];
                c.fetched(slot + TENSOR + i * BLOCK, lane);
                c.get(r + at[i], n[i], a);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] = ptx::f32x2_add(v[i][j], a[j]);
            }
        }
        __syncwarp();                                                        // every lane has read the slot that is fetched into now
        fetch(turn + depth, slot);
        slot = slot == mine && depth > 1 ? mine + slot_bytes : mine;
        // (of a chunk beyond the row, whose values are zeros, the row's first gammas: no choice between loads, and nothing that the row
        // does not meet anyway)
        auto gamma = [&](int i, uint64_t (&g)[4]) {
            const int a = n[i] > 0 ? at[i] : 0;
            load_gamma<LAYOUT>(p.gamma + a, p.wide_g, p.K - a, g);
        };
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            if (NORM && p.h && here && n[i] > 0) store8(h + at[i], LAYOUT == REGULAR || (p.wide_h && n[i] >= 8), n[i], v[i]);
            uint64_t g[4];
            if (NORM && QUANT) gamma(i, g);
            row.take(v[i], g, CHUNKS == 4 && (i & 1));
        }
        if constexpr (CHUNKS == 4) reduce_row_twofold<NORM, QUANT>(row.sum, row.sum_more, row.top, part[turn & 1]);
        else reduce_row<LANES, NORM, QUANT>(row.sum, row.top, part[turn & 1]);
        row.end(p, here ? scale : nullptr);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
            if (here && n[i] > 0) {
                if constexpr (QUANT) row.store(q + at[i], p.wide_q, n[i], v[i], one2);
                else {
                    uint64_t g[4];
                    gamma(i, g);
                    row.store(y + at[i], p.wide_y, n[i], v[i], g);
                }
            }
        if (LAYOUT == ANY) { x += step * p.ldx; r += step * p.ldr; }         // (only where the row begins in its granule is asked of them)
        if (NORM) h += step * p.ldh;
        if (QUANT) { q += step * p.ldq; scale = scale ? scale + step : scale; }
        else y += step * p.ldy;
    }
}

// Rows too long for that: a CTA reads its row twice.
template <class T, bool NORM, bool QUANT, int LAYOUT>
__global__ void __launch_bounds__(MAX_THREADS) long_rows_kernel(const __grid_constant__ Rows p)
{
    __shared__ uint2 part[32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const long long m = blockIdx.x;
    const T *x = static_cast<const T *>(p.x) + m * p.ldx, *r = static_cast<const T *>(p.r) + m * p.ldr;
    const bool residual = NORM && p.r;
    Row<T, NORM, QUANT, LAYOUT> row;
    uint64_t v[4], g[4];
    auto load = [&](int at) {
        const int n = p.K - at;
        Chunk<T, LAYOUT> cx, cr;
        cx.fetch(x + at, n);
        if (residual) cr.fetch(r + at, n);
        if (NORM) load_gamma<LAYOUT>(p.gamma + at, p.wide_g, n, g);
        cx.get(x + at, n, v);
        if (residual) {
            uint64_t a[4];
            cr.get(r + at, n, a);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = ptx::f32x2_add(v[i], a[i]);
        }
    };
    for (int at = 8 * threadIdx.x; at < p.K; at += 8 * MAX_THREADS) { load(at); row.take(v, g); }
    reduce_row<0, NORM, QUANT>(row.sum, row.top, part);
    row.end(p, QUANT && threadIdx.x == 0 ? p.scales + m : nullptr);
    const uint64_t one2 = ptx::f32x2_one(p.zero);
    // the sum is stored in the last pass: it may take the place of x or r, which both read
    for (int at = 8 * threadIdx.x; at < p.K; at += 8 * MAX_THREADS) {
        const int n = p.K - at;
        load(at);
        if (NORM && p.h) store8(static_cast<T *>(p.h) + m * p.ldh + at, LAYOUT == REGULAR || (p.wide_h && n >= 8), n, v);
        if constexpr (QUANT) {
            if (NORM)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = ptx::f32x2_mul(v[i], g[i]);
            row.store(p.q + m * p.ldq + at, p.wide_q, n, v, one2);
        } else {
            row.store(static_cast<T *>(p.y) + m * p.ldy + at, p.wide_y, n, v, g);
        }
    }
}

// v = q * scale: 16 bytes of results per thread, DEQ_ROWS rows of them at once.  A CTA is `columns` threads wide along a row, 256 / columns
// rows high.
constexpr int DEQ_ROWS = 4;
template <class T>
__global__ void __launch_bounds__(256) dequantize_kernel(const signed char *q, long long ldq, const float *scales, T *y, long long ldy, int M, int K, int columns, bool wide_q, bool wide_y)
{
    constexpr int E = 16 / sizeof(T);
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int high = 256 / columns, row = threadIdx.x / columns;
    const int k = E * (blockIdx.y * columns + threadIdx.x % columns), n = K - k;
    const long long m0 = (long long)blockIdx.x * (high * DEQ_ROWS) + row;
    if (row >= high || n <= 0) return;
    uint32_t w[DEQ_ROWS][E / 4];
    float s[DEQ_ROWS];
#pragma unroll
    for (int i = 0; i < DEQ_ROWS; ++i) {
        const long long m = m0 + i * high;
#pragma unroll
        for (int j = 0; j < E / 4; ++j) w[i][j] = 0;
        s[i] = 0.0f;
        if (m < M) {
            const signed char *src = q + m * ldq + k;
            s[i] = scales[m];
            if (wide_q && n >= E) {
                if constexpr (E == 8) {
                    const uint2 u = *reinterpret_cast<const uint2 *>(src);
                    w[i][0] = u.x;
                    w[i][1] = u.y;
                } else {
                    w[i][0] = *reinterpret_cast<const uint32_t *>(src);
                }
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (j < n) w[i][j / 4] |= static_cast<uint32_t>(static_cast<unsigned char>(src[j])) << (8 * (j & 3));
            }
        }
    }
#pragma unroll
    for (int i = 0; i < DEQ_ROWS; ++i) {
        const long long m = m0 + i * high;
        if (m >= M) continue;
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = static_cast<float>(static_cast<signed char>(w[i][j / 4] >> (8 * (j & 3)))) * s[i];
        store16(y + m * ldy + k, wide_y && n >= E, n, v);
    }
}

template <class Kernel, class... Args>
cudaError_t launch(Kernel kernel, dim3 grid, int threads, int smem, cudaStream_t st, Args... args)
{
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

constexpr int SM_SMEM = 220 * 1024, SM_THREADS = 1024;      // threads of an SM at 64 registers each

// Shared memory of one row ahead, for each group of lanes that fetches together.
template <class T, int LAYOUT, int GROUP>
int ring_bytes(const Rows &p, int chunks) { return (p.r ? 2 : 1) * chunks * Chunk<T, LAYOUT>::template GRANULES<GROUP> * 16; }

template <class T, bool NORM, bool QUANT, int LANES, int LAYOUT, int CHUNKS>
cudaError_t launch_rows(const Rows &p, int threads, cudaStream_t st)
{
    constexpr int GROUP = LANES ? LANES : 32;
    auto kernel = rows_kernel<T, NORM, QUANT, LANES, LAYOUT, CHUNKS>;
    static QvggtPerDevice cache;
    int sms = 0;
    cudaError_t e = qvggt_configure_kernel(kernel, threads, SM_SMEM, 1, cache, &sms);
    if (e != cudaSuccess) return e;
    const long long units = LANES ? (p.M - 1) / (SHORT_THREADS / GROUP) + 1 : p.M;        // CTAs that one row each would make
    const int slot = threads / GROUP * ring_bytes<T, LAYOUT, GROUP>(p, CHUNKS), per_sm = SM_THREADS / threads;
    // Rows per CTA: enough for the copies to run ahead, few enough for the SMs, which differ in their way to memory, to share the rows out among
    // themselves (with every CTA's share fixed, rows of the whole grid apart: 43 968 x 4096, norm with residual 263 us against 212).  About the
    // root of the CTAs that follow one another on an SM's slot; us with 1 / 2 / 4 / 8 / 16: 10 992 x 1024 norm, residual, codes 17.8 / 16.1 /
    // 17.4; 10 992 x 4096 64 / 55 / 52 / 53 / 63; 43 968 x 4096 250 / 213 / 193 / 189 / 197; fp32 10 992 x 4096 87 / 88 / 91 / 97 / 107.
    const long long queue = units / ((long long)sms * per_sm);
    const int most = sizeof(T) == 4 ? 2 : 8;
    int turns = 1;
    while (2 * turns <= most && 4LL * turns * turns <= queue) turns *= 2;
    // Two rows ahead where little is done with a row (43 968 x 4096: quantizer 98 with one, 86 with two; norm and codes 145 and 155).
    int depth = SM_SMEM / per_sm / slot, wanted = NORM && QUANT ? 1 : 2;
    if (depth > wanted) depth = wanted;
    if (depth > turns) depth = turns;
    if (depth < 1) depth = 1;
    const int ctas = (int)((units - 1) / turns + 1);
    return launch(kernel, dim3(ctas), threads, depth * slot, st, p, turns, depth);
}

template <class T, bool NORM, bool QUANT, int LAYOUT>
cudaError_t by_length(const Rows &p, cudaStream_t st)
{
    const int chunks = (p.K + 7) / 8;
    if (chunks <= 8) return launch_rows<T, NORM, QUANT, 8, LAYOUT, 1>(p, SHORT_THREADS, st);
    if (chunks <= 16) return launch_rows<T, NORM, QUANT, 16, LAYOUT, 1>(p, SHORT_THREADS, st);
    if (chunks <= 32) return launch_rows<T, NORM, QUANT, 32, LAYOUT, 1>(p, SHORT_THREADS, st);
    if (chunks <= 64) return launch_rows<T, NORM, QUANT, 32, LAYOUT, 2>(p, SHORT_THREADS, st);
    // Four chunks a thread, half the warps, where arithmetic shows beside the little that is read: every warp spends some 250 instructions
    // a row on what does not depend on its chunks.  43 968 x 4096 bf16, us with two / four: norm and codes 121 / 102, quantizer 80 / 80;
    // 10 992 x 4096 33 / 29.5 and 22.7 / 20.9; but with a residual 50 / 52, norm alone 32 / 32, one row 1.9 / 2.5.  The sum of a norm is added up
    // in the same order by both; so rows too long for two chunks always take four behind a norm (few rows by
    // long_rows_kernel / four: 1 x 32 768 5.3 / 4.9, 500 x 32 768 18.9 / 17.2, 2000 x 32 768 81 / 61, fp32 3000 x 17 000 99 / 70).
    if constexpr (QUANT)
        if (!p.r && chunks > 128 && chunks <= 4 * MAX_THREADS && (p.M >= 4096 || (NORM && chunks > 2 * MAX_THREADS))) return launch_rows<T, NORM, QUANT, 0, LAYOUT, 4>(p, (chunks + 127) / 128 * 32, st);
    if (chunks <= 2 * MAX_THREADS) return launch_rows<T, NORM, QUANT, 0, LAYOUT, 2>(p, (chunks + 63) / 64 * 32, st);
    return launch(long_rows_kernel<T, NORM, QUANT, LAYOUT>, dim3(p.M), MAX_THREADS, 0, st, p);
}

template <class T, bool NORM, bool QUANT>
cudaError_t by_layout(int layout, const Rows &p, cudaStream_t st)
{
    if (layout == element::REGULAR) return by_length<T, NORM, QUANT, element::REGULAR>(p, st);
    return layout == element::ALIGNED ? by_length<T, NORM, QUANT, element::ALIGNED>(p, st) : by_length<T, NORM, QUANT, element::ANY>(p, st);
}

template <bool NORM, bool QUANT>
cudaError_t by_type(int type, int layout, const Rows &p, cudaStream_t st)
{
    if (type == QVGGT_BF16) return by_layout<__nv_bfloat16, NORM, QUANT>(layout, p, st);
    return type == QVGGT_FP16 ? by_layout<__half, NORM, QUANT>(layout, p, st) : by_layout<float, NORM, QUANT>(layout, p, st);
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
    p.one_over_k = 1.0f / (float)K;
    p.floor_factor = (1.0f / 1e-8f) * 127.0f;
    p.wide_h = rows_aligned(H, ldh, e, 16);
    p.wide_y = rows_aligned(Y, ldy, e, 16);
    p.wide_q = rows_aligned(Xq8, ldq, 1, 8);
    p.wide_g = rows_aligned(gamma, 0, 4, 16);
    const bool aligned = rows_aligned(X, ldx, e, 16) && (!R || rows_aligned(R, ldr, e, 16));
    const int layout = !aligned ? element::ANY : K % 8 == 0 && p.wide_g && (!H || p.wide_h) && (!Y || p.wide_y) && (!Xq8 || p.wide_q) ? element::REGULAR : element::ALIGNED;
    if (!gamma) return by_type<false, true>(type, layout, p, st);
    return Xq8 ? by_type<true, true>(type, layout, p, st) : by_type<true, false>(type, layout, p, st);
}

cudaError_t qvggt_launch_dequantize(int type, const signed char *Xq8, long long ldq, const float *scales, int M, int K, void *Y, long long ldy, cudaStream_t st)
{
    const bool wide_q = rows_aligned(Xq8, ldq, 1, 8), wide_y = rows_aligned(Y, ldy, bytes_of(type), 16);
    const int chunks = (K * bytes_of(type) - 1) / 16 + 1, wide = (chunks + 255) / 256, columns = (chunks + wide - 1) / wide, high = 256 / columns * DEQ_ROWS;
    const dim3 grid((M - 1) / high + 1, wide);
    if (type == QVGGT_BF16) return launch(dequantize_kernel<__nv_bfloat16>, grid, 256, 0, st, Xq8, ldq, scales, static_cast<__nv_bfloat16 *>(Y), ldy, M, K, columns, wide_q, wide_y);
    if (type == QVGGT_FP16) return launch(dequantize_kernel<__half>, grid, 256, 0, st, Xq8, ldq, scales, static_cast<__half *>(Y), ldy, M, K, columns, wide_q, wide_y);
    return launch(dequantize_kernel<float>, grid, 256, 0, st, Xq8, ldq, scales, static_cast<float *>(Y), ldy, M, K, columns, wide_q, wide_y);
}
