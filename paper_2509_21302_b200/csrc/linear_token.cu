// Integer product of 8-bit codes for one to four token rows, any K and N (the same sums and epilogue as linear_split.cu):
//   Y[m][n] = fma(float(acc), a_scale[m] * w_scale[n], bias[n]),  acc[m][n] = sum_k Xq[m][k] Wq[n][k] in int32.
// One token is the N K bytes of the weights and the latency of one launch.  A warp takes two or four channels and reads their rows as they lie,
// 512 consecutive bytes a load, sixteen bytes a lane; the products are dp4a, the lanes' sums meet in one instruction, and nothing goes through
// shared memory unless several warps share a long row.  What is under way hides the memory's latency best as many warps with few loads each
// (one row, N = K = 1024 / 4096, us, four warps a CTA: two pieces in flight 1.5 / 4.3, four 1.6 / 3.8; eight warps with four 1.7 / 4.6, with eight 2.2 /
// 6.1; one channel with eight 2.0 / 4.9).  Before the previous kernel of the stream has ended the rows are already on their way to L2 (a
// prefetch neither sees nor changes what that may still write).
#include "element.cuh"
#include "linear_plan.cuh"
#include "qvggt_internal.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace {

constexpr int WARPS = 4, PIECE = 512;             // warps of a CTA that nothing else decides; codes of a row that a warp reads with one load
// Most warps that share a row.  Four rows: bounds for 16 warps make it 92 registers instead of 72 (N = K = 4096: 6.0 us instead of 4.4).
__host__ __device__ constexpr int most_warps(int tok) { return tok < 4 ? 16 : WARPS; }

// TOK: token rows, those from M on not read.  CHANNELS: of a warp.  FLIGHT: pieces of each row on their way at once.  `share` warps (1, 2,
// .. most_warps) share the pieces of a row.
template <class T, int TOK, int CHANNELS, int FLIGHT>
__global__ void __launch_bounds__(most_warps(TOK) * 32)
linear_token_kernel(const signed char *__restrict__ Xq, long long ldx, const float *__restrict__ a_scale, const signed char *__restrict__ Wq, long long ldw,
                    const float *__restrict__ w_scale, const T *__restrict__ bias, T *__restrict__ Y, long long ldy, int M, int N, int K, int share)
{
    __shared__ int parts[most_warps(TOK)][TOK * CHANNELS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % share;
    const long long n0 = ((long long)blockIdx.x * ((blockDim.x >> 5) / share) + warp / share) * CHANNELS;
    const signed char *w[CHANNELS];
#pragma unroll
    for (int c = 0; c < CHANNELS; ++c) w[c] = Wq + min(n0 + c, (long long)N - 1) * ldw;     // a channel beyond N computes the last one's sums
    ptx::grid_launch_dependents();
#pragma unroll
    for (int c = 0; c < CHANNELS; ++c)
        for (int k = PIECE * part + 128 * (lane & 3) + PIECE * share * (lane >> 2); k < K; k += 8 * PIECE * share)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(w[c] + k));
    ptx::grid_dependency_wait();
    int acc[TOK][CHANNELS] = {};
    for (int k0 = PIECE * part; k0 < K; k0 += FLIGHT * PIECE * share) {
        uint4 b[CHANNELS][FLIGHT], a[TOK][FLIGHT];
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            const int k = k0 + i * PIECE * share + 16 * lane;
#pragma unroll
            for (int c = 0; c < CHANNELS; ++c) {
                b[c][i] = make_uint4(0, 0, 0, 0);
                if (k < K) b[c][i] = __ldcg(reinterpret_cast<const uint4 *>(w[c] + k));
            }
#pragma unroll
            for (int m = 0; m < TOK; ++m) {
                a[m][i] = make_uint4(0, 0, 0, 0);
                if (k < K && m < M) a[m][i] = __ldca(reinterpret_cast<const uint4 *>(Xq + m * ldx + k));
            }
        }
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            const int left = K - (k0 + i * PIECE * share + 16 * lane);
#pragma unroll
            for (int m = 0; m < TOK; ++m) {
                uint4 x = a[m][i];
                if (left > 0 && left < 16) {                          // zeros behind K, in one of the two operands
                    auto keep = [&](uint32_t v, int at) { return left >= at + 4 ? v : left <= at ? 0u : v & ((1u << (8 * (left - at))) - 1u); };
                    x = make_uint4(keep(x.x, 0), keep(x.y, 4), keep(x.z, 8), keep(x.w, 12));
                }
#pragma unroll
                for (int c = 0; c < CHANNELS; ++c) {
                    acc[m][c] = __dp4a((int)x.x, (int)b[c][i].x, acc[m][c]);
                    acc[m][c] = __dp4a((int)x.y, (int)b[c][i].y, acc[m][c]);
                    acc[m][c] = __dp4a((int)x.z, (int)b[c][i].z, acc[m][c]);
                    acc[m][c] = __dp4a((int)x.w, (int)b[c][i].w, acc[m][c]);
                }
            }
        }
    }
    // lane m CHANNELS + c keeps the sum of token m and channel c
    int mine = 0;
#pragma unroll
    for (int m = 0; m < TOK; ++m)
#pragma unroll
        for (int c = 0; c < CHANNELS; ++c) {
            const int s = __reduce_add_sync(0xFFFFFFFFu, acc[m][c]);
            if (lane == m * CHANNELS + c) mine = s;
        }
    if (share > 1) {
        if (lane < TOK * CHANNELS) parts[warp][lane] = mine;
        __syncthreads();
        if (part != 0) return;
        mine = 0;
        if (lane < TOK * CHANNELS)
            for (int i = 0; i < share; ++i) mine += parts[warp + i][lane];
    }
    const int m = lane / CHANNELS;
    const long long n = n0 + lane % CHANNELS;
    if (m >= TOK || m >= M || n >= N) return;
    const float b = bias ? element::to_float(bias[n]) : 0.0f;
    Y[m * ldy + n] = element::from_float<T>(__fmaf_rn(static_cast<float>(mine), __fmul_rn(a_scale[m], w_scale[n]), b));
}

// Warps enough to have a good part of the weights on their way, while each still has two pieces or more (half or twice as many warps: up to
// 20 % slower somewhere; one row, N = 64, K = 16384: 2.0 us, four warps a row 2.3).
int warps_of_a_row(const QvggtLinear &p, int channels, int most)
{
    const long long groups = (p.N - 1LL) / channels + 1;
    int share = 1;
    while (share < most && groups * share < 16LL * qvggt_sm_count() && p.K > 2 * share * PIECE) share *= 2;
    return share;
}

template <class T, int TOK, int CHANNELS, int FLIGHT>
cudaError_t launch(const QvggtLinear &p, int share, cudaStream_t st)
{
    const int warps = share > WARPS ? share : WARPS;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.N - 1LL) / (CHANNELS * (warps / share)) + 1));
    cfg.blockDim = dim3(warps * 32);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, linear_token_kernel<T, TOK, CHANNELS, FLIGHT>, p.Xq8, p.ldx, p.a_scale, p.Wq8, p.ldw, p.w_scale, static_cast<const T *>(p.bias),
                              static_cast<T *>(p.Y), p.ldy, p.M, p.N, p.K, share);
}

// One row: four pieces in flight where a warp has more than two (N = 5003, K = 2011: 2.65 us, two 3.2; N = 8192, K = 1024, two each: 2.5 / 2.2).  Two rows:
// two (N = K = 4096 4.0, four 5.5).  Three and four: four channels, whose codes of X are read half as often, and one piece (4.4; two channels and two
// pieces 6.9).
template <class T>
cudaError_t by_rows(const QvggtLinear &p, cudaStream_t st)
{
    if (p.M > 2) return launch<T, 4, 4, 1>(p, warps_of_a_row(p, 4, most_warps(4)), st);
    const int share = warps_of_a_row(p, 2, most_warps(2));
    if (p.M == 2) return launch<T, 2, 2, 2>(p, share, st);
    return p.K > 2 * share * PIECE ? launch<T, 1, 2, 4>(p, share, st) : launch<T, 1, 2, 2>(p, share, st);
}

}  // namespace

cudaError_t qvggt_launch_linear_token(const QvggtLinear &p, cudaStream_t st)
{
    if (p.M > 4) return cudaErrorNotSupported;
    return p.type == QVGGT_BF16 ? by_rows<__nv_bfloat16>(p, st) : p.type == QVGGT_FP16 ? by_rows<__half>(p, st) : by_rows<float>(p, st);
}
