// Integer product of 8-bit codes for a batch of up to some hundred token rows, any K and N:
//   Y[m][n] = fma(float(acc), a_scale[m] * w_scale[n], bias[n]),  acc[m][n] = sum_k Xq[m][k] Wq[n][k] in int32.
// Such a product is the N K bytes of its weights: the tensor core is hardly used, but the bytes have to be asked for all at once, from all
// SMs.  So the channels are the rows of the MMA (128 a tile) and the tokens its columns (16 .. 256, as many as there are), and the K-blocks of a
// tile are shared by the CTAs of a cluster, each of which streams its part through a ring of TMA stages as deep as shared memory is large.
// The partial sums, integers, meet in distributed shared memory: every CTA adds up and finishes its share of the tokens.  No workspace, no
// atomics, one launch.
//   warp 0: one thread issues the TMA loads;  warp 1: one thread issues tcgen05.mma;  all eight warps: sums to shared memory, epilogue
// Every wait is bounded; on expiry the kernel records a code in the status word and leaves through the common exit (what its cluster stores
// is then not the product).
#include <cuda.h>

#include "element.cuh"
#include "gemm_common.cuh"
#include "linear_plan.cuh"
#include "qvggt_internal.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace {

using linear_plan::BK;                 // codes along K per stage = one 128-byte swizzled row
using linear_plan::CH;                 // channels of a tile: rows of the MMA, TMEM lanes
using linear_plan::MAX_TOK;            // tokens of a tile: columns of the MMA
constexpr int WARPS = 8;
constexpr int MAX_STAGES = 12;
constexpr int AHEAD = 16;              // blocks brought into L2 before the previous kernel ends.  One row, us with 0 / 8 / 16 / 32 / all: N = K = 4096 5.8 /
                                       // 5.4 / 5.4 / 5.4 / 5.4, N = 16 384, K = 4096 13.5 / 12.6 / 12.2 / 13.5 / 13.5, N = K = 7183 12.9 / 12.6 / 12.2 / 13.1 / 13.2,
                                       // N = K = 16 384 43.8 / 42.7 / 42.9 / 44.5 / 52.6 (what comes too early is displaced again)
static_assert(CH == 128 && BK == 128 && MAX_TOK == 256, "what the instruction descriptor and tensor memory take");
constexpr int W_BYTES = CH * BK;
constexpr int OFF_FULL = 0, OFF_EMPTY = OFF_FULL + 8 * MAX_STAGES, OFF_DONE = OFF_EMPTY + 8 * MAX_STAGES, OFF_TMEM = OFF_DONE + 8, OFF_ABORT = OFF_TMEM + 4;
constexpr int OFF_OPS = 1024;          // stages; then the partial sums [token][channel]

__device__ int split_status;           // see qvggt_linear_status

__device__ __forceinline__ uint4 ld_cluster(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// wait_limit: bound of every device-side wait, in cycles; any but the usual one starves the kernel: nothing is loaded, so that the first wait for
// operands runs out (used only to exercise that path; no asynchronous operation is in flight).
// One tile of CH channels x tok tokens per cluster of SPLIT CTAs; blockIdx.x = tile * SPLIT + rank, blockIdx.y = tile of tokens.
template <class T, int SPLIT>
__global__ void __launch_bounds__(WARPS * 32)
linear_split_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const float *__restrict__ a_scale, const float *__restrict__ w_scale,
                    const T *__restrict__ bias, T *__restrict__ Y, long long ldy, int M, int N, int K, int tok, int stages, int tmem_cols, long long wait_limit)
{
    int *status = &split_status;
    const bool starved = wait_limit != ptx::kWaitLimitCycles;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sbase = ptx::smem_addr(smem), ops = sbase + OFF_OPS;
    const uint32_t bar_full = sbase + OFF_FULL, bar_empty = sbase + OFF_EMPTY, bar_done = sbase + OFF_DONE;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + OFF_TMEM);
    volatile int *s_abort = reinterpret_cast<volatile int *>(smem + OFF_ABORT);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = SPLIT > 1 ? (int)ptx::cluster_ctarank() : 0;
    const int n0 = (int)(blockIdx.x / SPLIT) * CH;
    const int m0 = blockIdx.y * tok, rows = min(tok, M - m0);
    const int KB = (K + BK - 1) / BK, first = KB * rank / SPLIT, blocks = KB * (rank + 1) / SPLIT - first;
    const int stage_bytes = W_BYTES + tok * BK;

    if (threadIdx.x == 0) {
        gemmc::init_barriers(bar_full, stages, 1);
        gemmc::init_barriers(bar_empty, stages, 1);
        ptx::mbar_init(bar_done, 1);
        ptx::fence_mbar_init();
        *s_abort = 0;
    }
    if (warp == 1) { ptx::tmem_alloc(ptx::smem_addr(s_tmem), tmem_cols); ptx::tmem_relinquish(); }
    if (warp == 0 && lane == 0) { ptx::prefetch_tensormap(&map_w); ptx::prefetch_tensormap(&map_x); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *s_tmem;
    // The next kernel of the stream may set itself up, and the first weights may be on their way to L2, while the previous one ends: a
    // prefetch neither sees nor changes what that may still write.
    ptx::grid_launch_dependents();
    if (warp == 0 && !starved && ptx::elect_one())
        for (int i = 0; i < min(blocks, AHEAD); ++i) ptx::tma_prefetch_2d(&map_w, (first + i) * BK, n0);
    __syncwarp();
    ptx::grid_dependency_wait();

    if (warp == 0) {
        if (!starved && ptx::elect_one()) {
            gemmc::Ring r;
            int i = 0;
            for (; i < blocks; ++i) {
                if (i >= stages && !ptx::mbar_wait(bar_empty + 8 * r.s, r.ph ^ 1, s_abort, status, QVGGT_DEV_TIMEOUT_EMPTY, 0, wait_limit)) break;
                const uint32_t stage = ops + r.s * stage_bytes;
                ptx::mbar_arrive_expect_tx(bar_full + 8 * r.s, stage_bytes);
                ptx::tma_load_2d(&map_w, bar_full + 8 * r.s, stage, (first + i) * BK, n0);
                ptx::tma_load_2d(&map_x, bar_full + 8 * r.s, stage + W_BYTES, (first + i) * BK, m0);
                r.advance(stages);
            }
            if (!ptx::mbar_wait(bar_done, 0, s_abort, status, QVGGT_DEV_TIMEOUT_ACCUM, 20, wait_limit))       // the copies in flight end before the CTA does
                for (int j = max(0, i - stages); j < i; ++j)
                    for (int n = 0; n < 100000 && !ptx::mbar_try_wait(bar_full + 8 * (j % stages), (j / stages) & 1); ++n) {}
        }
        __syncwarp();
    } else if (warp == 1) {
        if (ptx::elect_one()) {
            const uint32_t idesc = ptx::idesc_i8(CH, tok);
            gemmc::Ring r;
            for (int i = 0; i < blocks; ++i) {
                if (!ptx::mbar_wait(bar_full + 8 * r.s, r.ph, s_abort, status, QVGGT_DEV_TIMEOUT_FULL, 0, wait_limit)) break;
                ptx::tc_fence_after_sync();
                const uint32_t stage = ops + r.s * stage_bytes;
                gemmc::mma_kblock_i8<false>(tmem, stage, stage + W_BYTES, idesc, i == 0);
                if (i + stages < blocks) ptx::mma_commit(bar_empty + 8 * r.s);
                if (i == blocks - 1) ptx::mma_commit(bar_done);
                r.advance(stages);
            }
        }
        __syncwarp();
    }

    // Partial sums to shared memory, over the operands: behind the last MMA nothing reads them, and every load has been consumed by one.
    int *part = reinterpret_cast<int *>(smem + OFF_OPS);
    bool alive = ptx::mbar_wait(bar_done, 0, s_abort, status, QVGGT_DEV_TIMEOUT_ACCUM, 20, wait_limit);
    alive = __all_sync(0xFFFFFFFFu, alive);
    ptx::tc_fence_after_sync();
    if (alive) {
        const int quarter = warp & 3;
        for (int c = (warp >> 2) * 16; c < rows; c += 64) {
            uint32_t raw[2][16];
            const uint32_t at = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + c;
            const bool more = c + 32 < rows;
            ptx::tmem_ld_32x16(at, raw[0]);
            if (more) ptx::tmem_ld_32x16(at + 32, raw[1]);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) part[(c + j) * CH + quarter * 32 + lane] = static_cast<int>(raw[0][j]);
            if (more)
#pragma unroll
                for (int j = 0; j < 16; ++j) part[(c + 32 + j) * CH + quarter * 32 + lane] = static_cast<int>(raw[1][j]);
        }
    }
    ptx::tc_fence_before_sync();
    if (SPLIT > 1) ptx::cluster_sync();
    else __syncthreads();

    // A warp finishes a token at a time, four channels a lane; the cluster's CTAs take turns.
    const int c = 4 * lane, n = n0 + c;
    if (alive && n < N) {
        float ws[4], bs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ws[i] = n + i < N ? __ldg(w_scale + n + i) : 0.0f;
            bs[i] = bias && n + i < N ? element::to_float(bias[n + i]) : 0.0f;
        }
        constexpr int AT_ONCE = SPLIT == 8 ? 2 : 4, STEP = WARPS * SPLIT;          // tokens whose sums are on their way together
        for (int r0 = warp * SPLIT + rank; r0 < rows; r0 += AT_ONCE * STEP) {
            uint4 v[AT_ONCE][SPLIT];
            float as[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const int r = r0 + j * STEP;
                if (r >= rows) break;
                as[j] = __ldg(a_scale + m0 + r);
#pragma unroll
                for (int k = 0; k < SPLIT; ++k) v[j][k] = ld_cluster(ptx::map_to_cta(ops + (r * CH + c) * 4, k));
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const int r = r0 + j * STEP;
                if (r >= rows) break;
                int s[4] = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < SPLIT; ++k) { s[0] += v[j][k].x; s[1] += v[j][k].y; s[2] += v[j][k].z; s[3] += v[j][k].w; }
                float z[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = __fmaf_rn(static_cast<float>(s[i]), __fmul_rn(as[j], ws[i]), bs[i]);
                T *y = Y + (long long)(m0 + r) * ldy + n;
                if (linear_plan::four_channels(n, N) && (reinterpret_cast<uintptr_t>(y) & (4 * sizeof(T) - 1)) == 0) {
                    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(y) = make_float4(z[0], z[1], z[2], z[3]);
                    else *reinterpret_cast<uint2 *>(y) = make_uint2(element::pack2<T>(z[0], z[1]), element::pack2<T>(z[2], z[3]));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (n + i < N) y[i] = element::from_float<T>(z[i]);
                }
            }
        }
    }
    if (SPLIT > 1) ptx::cluster_sync_relaxed();        // a CTA's sums stay until its peers have read them
    else __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, tmem_cols);
    }
}

constexpr int SMEM_FULL = 232448 - 2048;      // stages of a CTA that has its SM to itself, and of one that shares it
constexpr int SMEM_HALF = 232448 / 2 - 4096;

template <class T, int SPLIT>
cudaError_t launch(const QvggtLinear &p, const linear_plan::Split &plan, long long wait_limit, cudaStream_t st)
{
    static QvggtPerDevice cache;
    int sms = 0;
    cudaError_t e = qvggt_configure_kernel(linear_split_kernel<T, SPLIT>, WARPS * 32, OFF_OPS + SMEM_FULL + 1024, 1, cache, &sms);
    if (e != cudaSuccess) return e;
    const int row_tiles = plan.row_tiles, tok = plan.tok, tiles = (int)plan.tiles, KB = (p.K - 1) / BK + 1;
    if (KB < SPLIT || row_tiles > 65535) return cudaErrorNotSupported;
    const int stage_bytes = W_BYTES + tok * BK;
    const int blocks = (KB + SPLIT - 1) / SPLIT;
    // Half of the SM, so that the next kernel's CTAs, or this one's, set themselves up beside it -- where five stages fit (three: N = K = 4096, 128
    // rows 10.2 us instead of 8.1), and no long stream would do with fewer than the whole SM holds (N = 16 384, K = 4096 18.8 instead of 13.4).
    const int limit = (blocks < 5 ? blocks : 5) * stage_bytes <= SMEM_HALF && ((long long)tiles * row_tiles * SPLIT > sms || blocks <= 12) ? SMEM_HALF : SMEM_FULL;
    int stages = limit / stage_bytes;
    if (stages > MAX_STAGES) stages = MAX_STAGES;
    if (stages > blocks) stages = blocks;
    int ops = stages * stage_bytes;
    if (ops < tok * CH * 4) ops = tok * CH * 4;
    int tmem_cols = 32;
    while (tmem_cols < tok) tmem_cols *= 2;
    CUtensorMap map_w, map_x;
    if (!qvggt_make_map(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, p.Wq8, p.K, p.N, p.ldw, BK, CH, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !qvggt_make_map(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, p.Xq8, p.K, p.M, p.ldx, BK, tok, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = SPLIT; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * SPLIT, row_tiles);
    cfg.blockDim = dim3(WARPS * 32);
    cfg.dynamicSmemBytes = OFF_OPS + ops + 1024;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, linear_split_kernel<T, SPLIT>, map_w, map_x, p.a_scale, p.w_scale, static_cast<const T *>(p.bias), static_cast<T *>(p.Y), p.ldy,
                              p.M, p.N, p.K, tok, stages, tmem_cols, wait_limit);
}

template <class T>
cudaError_t by_split(const QvggtLinear &p, const linear_plan::Split &s, long long limit, cudaStream_t st)
{
    return s.split == 8 ? launch<T, 8>(p, s, limit, st) : s.split == 4 ? launch<T, 4>(p, s, limit, st) : s.split == 2 ? launch<T, 2>(p, s, limit, st) : launch<T, 1>(p, s, limit, st);
}

}  // namespace

cudaError_t qvggt_launch_linear_split(const QvggtLinear &p, const linear_plan::Split &plan, cudaStream_t st)
{
    if (p.type == QVGGT_BF16) return by_split<__nv_bfloat16>(p, plan, ptx::kWaitLimitCycles, st);
    return p.type == QVGGT_FP16 ? by_split<__half>(p, plan, ptx::kWaitLimitCycles, st) : by_split<float>(p, plan, ptx::kWaitLimitCycles, st);
}

cudaError_t qvggt_launch_linear_starved(const QvggtLinear &p, long long wait_limit_cycles, cudaStream_t st)
{
    const int sms = qvggt_sm_count();
    return sms < 1 ? cudaErrorInvalidDevice : by_split<__nv_bfloat16>(p, linear_plan::best_split(p.M, p.N, p.K, sms), wait_limit_cycles, st);
}

cudaError_t qvggt_read_split_status(int *code) { return cudaMemcpyFromSymbol(code, split_status, sizeof(int)); }
