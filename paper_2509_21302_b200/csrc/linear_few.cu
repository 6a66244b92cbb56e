// Integer product of 8-bit codes for few token rows, any K and N:
//   Y[m][n] = float(acc) * (a_scale[m] * w_scale[n]) + bias[n]   (one rounding for the product of the scales, one for the multiply-add),
//   acc[m][n] = sum_k Xq[m][k] Wq[n][k] in int32.
// With a handful of rows the N K bytes of the weights are all there is.  A CTA owns 16 channels, its warps share K, and a lane's 16
// consecutive bytes of a row stand for whichever k the fragment of mma.sync asks for: the same permutation of K for both operands, which
// an integer sum does not see.  The warps' partial sums meet in shared memory.
#include "element.cuh"
#include "linear_plan.cuh"
#include "qvggt_internal.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace {

constexpr int CH = 16;          // channels per CTA: the rows of one MMA
constexpr int WARPS = 16;
constexpr int BLOCKS = 2;       // blocks of 128 codes that a warp has in flight

__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A lane's 32 of 128 consecutive codes of a row: 2 x 16 bytes, 64 apart.  Pieces beyond K are zero; the piece that K ends in is read
// whole (rows are 16 bytes apart or a multiple of that) and, with TAIL, cleared behind K: zero in one of two operands is enough.
struct Piece {
    uint4 v[2];
    template <bool TAIL>
    __device__ __forceinline__ void load(const signed char *row, bool ok, int k0, int K, int t)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = k0 + 16 * t + 64 * i, left = K - k;
            v[i] = make_uint4(0, 0, 0, 0);
            if (ok && left > 0) {
                v[i] = __ldcg(reinterpret_cast<const uint4 *>(row + k));
                if (TAIL && left < 16) {
                    auto keep = [&](uint32_t w, int b) { return left >= b + 4 ? w : left <= b ? 0u : w & ((1u << (8 * (left - b))) - 1u); };
                    v[i] = make_uint4(keep(v[i].x, 0), keep(v[i].y, 4), keep(v[i].z, 8), keep(v[i].w, 12));
                }
            }
        }
    }
    __device__ __forceinline__ uint32_t word(int i) const
    {
        const uint4 &q = v[i >> 2];
        const int j = i & 3;
        return j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w;
    }
};

// NT: tiles of 8 token rows per CTA.
template <class T, int NT>
__global__ void __launch_bounds__(WARPS * 32)
linear_few_kernel(const signed char *__restrict__ Xq, long long ldx, const float *__restrict__ a_scale, const signed char *__restrict__ Wq, long long ldw,
                  const float *__restrict__ w_scale, const T *__restrict__ bias, T *__restrict__ Y, long long ldy, int M, int N, int K)
{
    constexpr int TOK = 8 * NT, PITCH = CH + 4;
    __shared__ int part[WARPS * TOK * PITCH];               // [warp][token][channel]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * CH;
    const long long m0 = (blockIdx.y + (long long)gridDim.y * blockIdx.z) * TOK;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (m0 >= M) return;
    const signed char *w0 = Wq + (long long)(n0 + g) * ldw, *w1 = w0 + 8 * ldw;
    const bool ok0 = n0 + g < N, ok1 = n0 + g + 8 < N;
    int acc[NT][4] = {};
    for (int k = warp * 128; k < K; k += WARPS * BLOCKS * 128) {
        Piece wa[BLOCKS], wb[BLOCKS];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            wa[i].template load<true>(w0, ok0, k + WARPS * 128 * i, K, t);
            wb[i].template load<true>(w1, ok1, k + WARPS * 128 * i, K, t);
        }
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const long long m = m0 + 8 * j + g;
                Piece x;
                x.template load<false>(Xq + m * ldx, m < M, k + WARPS * 128 * i, K, t);
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    mma_s8(acc[j], wa[i].word(2 * s), wb[i].word(2 * s), wa[i].word(2 * s + 1), wb[i].word(2 * s + 1), x.word(2 * s), x.word(2 * s + 1));
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {                          // fragment: channels g and g + 8, tokens 2 t and 2 t + 1
        int *d = part + (warp * TOK + 8 * j + 2 * t) * PITCH + g;
        d[0] = acc[j][0]; d[PITCH] = acc[j][1]; d[8] = acc[j][2]; d[PITCH + 8] = acc[j][3];
    }
    __syncthreads();
    for (int o = threadIdx.x; o < TOK * CH; o += WARPS * 32) {
        const int tok = o / CH, c = o % CH, n = n0 + c;
        const long long m = m0 + tok;
        if (m >= M || n >= N) continue;
        int s = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += part[(w * TOK + tok) * PITCH + c];
        const float b = bias ? element::to_float(bias[n]) : 0.0f;
        Y[m * ldy + n] = element::from_float<T>(__fmaf_rn(static_cast<float>(s), __fmul_rn(a_scale[m], w_scale[n]), b));
    }
}

template <class T, int NT>
cudaError_t launch(const QvggtLinear &p, cudaStream_t st)
{
    const long long tiles = ((long long)p.M + 8 * NT - 1) / (8 * NT);
    const unsigned gy = tiles < 32768 ? tiles : 32768;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((p.N - 1) / CH + 1, gy, (tiles - 1) / gy + 1);
    cfg.blockDim = dim3(WARPS * 32);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, linear_few_kernel<T, NT>, p.Xq8, p.ldx, p.a_scale, p.Wq8, p.ldw, p.w_scale, static_cast<const T *>(p.bias),
                              static_cast<T *>(p.Y), p.ldy, p.M, p.N, p.K);
}

// Up to eight rows as linear_plan::choose() sends them; more where the tiles kernel, which would take them, does not count so far (N beyond some
// tens of millions).
template <class T>
cudaError_t by_rows(const QvggtLinear &p, cudaStream_t st)
{
    return p.M <= 8 ? launch<T, 1>(p, st) : launch<T, 4>(p, st);
}

}  // namespace

cudaError_t qvggt_launch_linear_few(const QvggtLinear &p, cudaStream_t st)
{
    return p.type == QVGGT_BF16 ? by_rows<__nv_bfloat16>(p, st) : p.type == QVGGT_FP16 ? by_rows<__half>(p, st) : by_rows<float>(p, st);
}

cudaError_t qvggt_launch_linear(const QvggtLinear &p, cudaStream_t st)
{
    const int sms = qvggt_sm_count();
    if (sms < 1) return cudaErrorInvalidDevice;
    linear_plan::Split split = {};
    const linear_plan::Kernel kernel = linear_plan::choose(p.M, p.N, p.K, sms, &split);
    cudaError_t e = cudaErrorNotSupported;
    if (kernel == linear_plan::TOKEN) e = qvggt_launch_linear_token(p, st);
    else if (kernel == linear_plan::SPLIT) e = qvggt_launch_linear_split(p, split, st);
    else if (kernel == linear_plan::TILES) e = qvggt_launch_linear_tiles(p, st);
    return e == cudaErrorNotSupported ? qvggt_launch_linear_few(p, st) : e;       // also for sizes beyond what the others count with
}
