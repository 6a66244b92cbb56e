// Which kernel takes a product of 8-bit codes, and how the split kernel (linear_split.cu) cuts it up: plain arithmetic, with no CUDA header, so
// that it can be compiled and checked by itself.
#pragma once
#ifndef __CUDACC__
#define __host__
#define __device__
#define __forceinline__ inline
#endif

namespace linear_plan {

constexpr int CH = 128;                // channels of a tile of the split kernel
constexpr int BK = 128;                // codes along K of a block
constexpr int MAX_TOK = 256;           // tokens of a tile, a multiple of 16
constexpr int FEW_ROWS = 48;           // row tiles are not made smaller than this

// Whether the four channels from n on (0 <= n < N) exist.  N goes up to 2^31 - 1, so n + 4 need not be an int.
__host__ __device__ __forceinline__ bool four_channels(int n, int N) { return n <= N - 4; }

struct Split {
    int split;                         // CTAs that share the K of a tile
    int tok, row_tiles;                // tokens of a tile, tiles along the tokens
    long long tiles;                   // along the channels
    float us;                          // what it is expected to take, beyond what every launch does
};

// What a round of `ctas` CTAs takes: their blocks at 140 KB per us each, half of it at 9 GB per ms in all where that is more, and what the sums cost in distributed shared
// memory, by the token.  Measured (us at 64 / 128 rows, N = 1024, K = 4096, one row tile): 1 CTA a tile 8.0 / 9.6, 2 5.9 / 7.2, 4 4.8 / 6.2, 8 4.7 / 6.0;
// with row tiles of 64 instead of 256 rows at 256 rows 16.2 / 11.0 / 9.6 -> 8.1 / 6.1 / 5.8 (1, 2, 4); N = K = 5418, 192 rows, 1 CTA, row tiles of 64,
// where the total shows: 20.8.
inline float split_us(int split, int tok, int KB, long long ctas)
{
    const float sums = split == 1 ? 0.3f + 0.012f * tok : split == 2 ? 0.8f + 0.012f * tok : split == 4 ? 0.6f + 0.0165f * tok : 1.0f + 0.0175f * tok;
    const float kb = ((KB + split - 1) / split) * (16.0f + tok / 8.0f), each = kb / 140.0f, all = kb * (float)ctas / 9000.0f;
    return 0.5f * (each + (each > all ? each : all)) + sums;
}

// For `split` CTAs a tile: as many row tiles as leave one round of CTAs.
inline Split make_split(int M, int N, int K, int split, int sms)
{
    Split s = {};
    s.split = split;
    s.tiles = (N - 1LL) / CH + 1;
    const int most = (M - 1) / FEW_ROWS + 1, least = (M - 1) / MAX_TOK + 1;
    long long rows = sms / (split * s.tiles);
    rows = rows < least ? least : rows > most ? most : rows;
    s.tok = (((M - 1) / (int)rows + 1) + 15) / 16 * 16;
    s.row_tiles = (M - 1) / s.tok + 1;
    const long long ctas = s.tiles * s.row_tiles * split;
    const long long rounds = (ctas + sms - 1) / sms;
    s.us = split_us(split, s.tok, (K - 1) / BK + 1, ctas / rounds) * (float)rounds;
    return s;
}

// The best of them.  Clusters of eight that have their SMs to themselves find room for a few only (16 of them: 11.3 us instead of 6.9 for
// N = 2048, K = 8192, 64 rows); clusters that share their SMs may be some more than one round.
inline Split best_split(int M, int N, int K, int sms)
{
    const int KB = (K - 1) / BK + 1;
    Split best = make_split(M, N, K, 1, sms);
    for (int split = 2; split <= 8; split *= 2) {
        Split s = make_split(M, N, K, split, sms);
        const long long ctas = s.tiles * s.row_tiles * split;
        if (KB < 2 * split || ctas > (split == 8 ? sms / 2 : M <= 32 ? sms + sms / 4 : sms)) continue;
        if (ctas > sms) s.us = split_us(split, s.tok, KB, ctas);
        if (s.us < best.us) best = s;
    }
    return best;
}

enum Kernel { TOKEN, FEW, SPLIT, TILES };

// The kernel for one to four rows (linear_token.cu) reads the weights with ordinary loads and multiplies without the tensor core: it starts fastest,
// and is the slower one where its arithmetic shows.  us, token / the best of the others (weights from memory):
//   1 row    N = K = 1024 1.5 / 2.7    K = 4096 2.1 / 3.4    N = K = 4096 3.8 / 5.4    7183 11.0 / 12.3    N = 16384, K = 4096 12.0 / 12.4
//            N = K = 16384 53 / 44     N = 64, K = 16384 2.0 / 4.8
//   2 rows   N = K = 1024 1.6 / 2.7    4096 4.0 / 5.4         5792 9.7 / 9.5    N = 16384, K = 4096 14.0 / 12.4
//   4 rows   N = K = 1024 2.1 / 2.7    4096 4.4 / 5.4         5792 10.2 / 9.5   N = 64, K = 16384 4.8 / 4.8    N = 128, K = 131056 55 / 27
// Many short rows leave its lanes idle: 1 row, K = 64, N = 8192 2.1 / 2.8, 16384 3.4 / 2.9; K = 512, N = 32768 6.1 / 5.7; K = 1024 6.7 / 7.5.
inline bool token_wins(int M, int N, int K)
{
    if (M > 4 || (long long)N * K > (M == 1 ? 1 << 26 : 1 << 24) || (M > 2 && K > 16384)) return false;
    return N <= 8192 || K >= 1024;
}

// The kernel for few rows (linear_few.cu) starts faster than the two on the tensor core's fifth generation, but its loads wait for registers, and
// K is shared by 16 warps only (8 rows, N = 256: K = 2048 2.8, split 2.9; 4096 3.6, 3.2): it has the smallest products.  The tiles kernel
// (gemm_c8.cu) takes about 0.2 us per K-block and round of its 256 x 256 tiles, hardly less for fewer rows, and half of the weights' way from
// memory on top; the split kernel is for batches.  us,
// few / split / tiles (weights from memory):
//   N = K = 1024          1 row 2.7 / 2.9 / 4.2    16 3.3 / 3.2 / 3.9    32 3.8 / 3.5 / 3.8    64 3.9 / 4.2 / 3.9    128 7.0 / 5.3 / 4.0
//   N = 1000, K = 520     1 row 2.6 / 3.0 / 3.6    32 3.7 / 3.5 / 3.5    64 3.7 / 4.5 / 3.6
//   N = K = 4096          1 row 10.7 / 5.4 / 14.3  64 23.8 / 6.7 / 9.3   128 39.5 / 8.1 / 9.4    256 72 / 9.5 / 9.5
//   N = 8192, K = 1024    1 row 9.0 / 4.1 / 6.7    64 24.6 / 4.8 / 5.6   128 47.7 / 6.0 / 5.2
//   N = 5003, K = 2011    1 row 7.4 / 4.3 / 10.5   64 20.6 / 5.8 / 8.0   96 - / 6.7 / 6.7        128 36.6 / 7.5 / 6.9
//   N = 16384, K = 4096   1 row 35 / 13.7 / 20.9   64 84 / 14.9 / 16.2   128 154 / 17.1 / 16.4
//   N = 1024, K = 4096    1 row 3.6 / 3.4 / 9.3    64 5.6 / 4.7 / 7.8    256 - / 5.8 / 7.9       512 - / 7.6 / 8.3
//   N = 2048, K = 8192    1 row 10.2 / 5.5 / 16.3  64 22.3 / 6.9 / 14.5  256 64 / 10.0 / 14.6    512 - / 14.2 / 14.4
inline Kernel choose(int M, int N, int K, int sms, Split *s)
{
    if (token_wins(M, N, K)) return TOKEN;
    if (M <= 8 && (long long)N * K <= 1 << 21 && K <= 2048) return FEW;
    if (M > 512) return TILES;
    *s = best_split(M, N, K, sms);
    const int KB = (K - 1) / BK + 1, pairs = sms > 1 ? sms / 2 : 1;
    const long long tiles = ((M - 1LL) / 256 + 1) * ((N - 1LL) / 256 + 1), rounds = (tiles + pairs - 1) / pairs;
    return M <= 32 || s->us < 0.1f + 0.2f * KB * rounds + (float)N * K / 13e6f ? SPLIT : TILES;
}

}  // namespace linear_plan
