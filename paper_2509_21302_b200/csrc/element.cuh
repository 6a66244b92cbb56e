// The element types of the rotation-free path (activations, residual, results, bias): bf16, fp16, fp32.  Everything is computed in fp32;
// conversions to 16 bits round to nearest even, once, where a result is stored.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

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

// Eight consecutive elements of a row as they lie in memory: the 16-byte granules that hold them (a granule is read only where one of the n
// elements, 1 .. 8, that exist lies in it).  fetch() only loads, so that many chunks can be on their way before the first is used.  With
// WIDE every row begins on a 16-byte boundary; otherwise get() shifts the elements out of one granule more.
template <class T, bool WIDE>
struct Chunk {
    static constexpr int SPAN = sizeof(T) / 2;                        // granules of eight elements
    static constexpr int WORDS = 4 * (SPAN + (WIDE ? 0 : 1));
    uint32_t w[WORDS];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void fetch(const T *p, int n)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = WIDE ? at : at & ~uintptr_t(15), end = at + min(n, 8) * sizeof(T);
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (i == 0 || base + 16 * i < end) v = *reinterpret_cast<const uint4 *>(base + 16 * i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    }
    // The values; those behind the first n are zero.
    __device__ __forceinline__ void get(const T *p, int n, float (&v)[8]) const
    {
        uint32_t u[WORDS];
#pragma unroll
        for (int i = 0; i < WORDS; ++i) u[i] = w[i];
        if constexpr (!WIDE) {
            const uint32_t byte = reinterpret_cast<uintptr_t>(p) & 15;
#pragma unroll
            for (int i = 0; i + 2 < WORDS; ++i) u[i] = byte & 8 ? u[i + 2] : u[i];
#pragma unroll
            for (int i = 0; i + 1 < WORDS; ++i) u[i] = byte & 4 ? u[i + 1] : u[i];
            if constexpr (sizeof(T) == 2)
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = __funnelshift_r(u[i], u[i + 1], 8 * (byte & 2));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (sizeof(T) == 2) {
                const float2 f = unpack2<T>(u[i / 2]);
                v[i] = i & 1 ? f.y : f.x;
            } else {
                v[i] = __uint_as_float(u[i]);
            }
        }
        if (n < 8)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.0f;
    }
};

// Stores eight elements: `wide`: p is on a 16-byte boundary and all eight exist; otherwise the first n of them, one by one.
template <class T>
__device__ __forceinline__ void store8(T *p, bool wide, int n, const float (&v)[8])
{
    if (wide) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
        } else {
            reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = from_float<T>(v[i]);
    }
}

}  // namespace element
