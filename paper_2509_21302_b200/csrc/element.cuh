// The element types of the rotation-free path (activations, residual, results, bias): bf16, fp16, fp32.  Everything is computed in fp32;
// conversions to 16 bits round to nearest even, once, where a result is stored.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "sm100_ptx.cuh"

namespace element {

__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(float v) { return v; }

template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }

// Two neighbouring 16-bit elements in one word, the first in the low half.
template <class T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w)
{
    __half2 h;
    memcpy(&h, &w, 4);
    return __half22float2(h);
}

template <class T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}

// How the rows of a call lie.  REGULAR: all of them, inputs and outputs, begin on 16-byte boundaries (codes: 8) and hold whole chunks of
// eight elements.  ALIGNED: the inputs begin on 16-byte boundaries.  ANY.
enum Layout { REGULAR, ALIGNED, ANY };

// Eight consecutive elements of a row as they lie in memory: the 16-byte granules that hold them (a granule is read only where one of the n
// elements that exist lies in it).  fetch() only loads, so that many chunks can be on their way before the first is used.  With ANY the
// elements are shifted out of one granule more.
template <class T, int LAYOUT>
struct Chunk {
    static constexpr int SPAN = sizeof(T) / 2;                        // granules of eight elements
    static constexpr int WORDS = 4 * (SPAN + (LAYOUT == ANY ? 1 : 0));
    uint32_t w[WORDS];
    __device__ __forceinline__ void fetch(const T *p, int n)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = LAYOUT != ANY ? at : at & ~uintptr_t(15), end = at + min(n, 8) * sizeof(T);
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (LAYOUT == REGULAR || i == 0 || base + 16 * i < end) v = *reinterpret_cast<const uint4 *>(base + 16 * i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    }
    // The granules of LANES chunks in a row, for so many lanes: asynchronous copies of neighbouring granules by neighbouring lanes (a granule
    // of its own chunk's each would fetch every 32-byte sector of fp32, and of misaligned rows, twice).  p: lane 0's first element, n:
    // elements of the row from there on, those behind the last lane's chunk included.  Lanes then read their own, behind a wait of every
    // lane for its copies and a __syncwarp().
    template <int LANES> static constexpr int GRANULES = LANES * SPAN + (LAYOUT == ANY ? 1 : 0);
    template <int LANES>
    __device__ __forceinline__ static void fetch_async(uint32_t smem, const T *p, int n, int lane)
    {
        if constexpr (LAYOUT != ANY) {
            constexpr int E = 16 / sizeof(T);                            // elements of a granule
#pragma unroll
            for (int i = 0; i < SPAN; ++i)
                if (n > E * (lane + LANES * i)) async_copy16(smem + (lane + LANES * i) * 16, p + E * (lane + LANES * i));
        } else {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = at & ~uintptr_t(15);
            const int granules = n > 0 ? static_cast<int>((at & 15) + static_cast<uint32_t>(n) * sizeof(T) + 15) / 16 : 0;
#pragma unroll
            for (int i = 0; i < (GRANULES<LANES> + LANES - 1) / LANES; ++i)
                if (lane + LANES * i < min(granules, GRANULES<LANES>)) async_copy16(smem + (lane + LANES * i) * 16, reinterpret_cast<const void *>(base + 16 * (lane + LANES * i)));
        }
    }
    __device__ __forceinline__ static void async_copy16(uint32_t smem, const void *p) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(p) : "memory"); }
    __device__ __forceinline__ void fetched(uint32_t smem, int lane)
    {
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3]) : "r"(smem + (lane * SPAN + i) * 16) : "memory");
    }
    // The values, two in a word; those behind the first n are zero (also those of granules that were never fetched; REGULAR: n <= 0 gives
    // anything).  p: as for fetch().
    __device__ __forceinline__ void get(const T *p, int n, uint64_t (&v)[4]) const
    {
        uint32_t u[WORDS];
#pragma unroll
        for (int i = 0; i < WORDS; ++i) u[i] = w[i];
        if constexpr (LAYOUT == ANY) {
            const uint32_t byte = reinterpret_cast<uintptr_t>(p) & 15;
#pragma unroll
            for (int i = 0; i + 2 < WORDS; ++i) u[i] = byte & 8 ? u[i + 2] : u[i];
#pragma unroll
            for (int i = 0; i + 1 < WORDS; ++i) u[i] = byte & 4 ? u[i + 1] : u[i];
            if constexpr (sizeof(T) == 2)
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = __funnelshift_r(u[i], u[i + 1], 8 * (byte & 2));
        }
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            if constexpr (sizeof(T) == 2) {
                const float2 two = unpack2<T>(u[i / 2]);
                f[i] = two.x;
                f[i + 1] = two.y;
            } else {
                f[i] = __uint_as_float(u[i]);
                f[i + 1] = __uint_as_float(u[i + 1]);
            }
        }
        if (LAYOUT != REGULAR && n < 8)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = i < n ? f[i] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ptx::f32x2_pack(f[2 * i], f[2 * i + 1]);
    }
};

// Stores 16 bytes of elements: `wide`: p is on a 16-byte boundary and all of them exist; otherwise the first n, one by one.
template <class T, int E>
__device__ __forceinline__ void store16(T *p, bool wide, int n, const float (&v)[E])
{
    static_assert(E * sizeof(T) == 16, "16 bytes");
    if (wide) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
        else *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < n) p[i] = from_float<T>(v[i]);
    }
}

// Eight elements, two in a word.
template <class T>
__device__ __forceinline__ void store8(T *p, bool wide, int n, const uint64_t (&v)[4])
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) ptx::f32x2_unpack(v[i], f[2 * i], f[2 * i + 1]);
    if constexpr (sizeof(T) == 2) {
        store16(p, wide, n, f);
    } else {
        const float a[4] = {f[0], f[1], f[2], f[3]}, b[4] = {f[4], f[5], f[6], f[7]};
        store16(p, wide, n, a);
        store16(p + 4, wide, n - 4, b);
    }
}

}  // namespace element
