// Eight elements of a row per thread and step, bf16 or fp32, as they lie in memory: the access shared by the memory-bound operators of a
// training step (norm, embedding, clip).  kVec: eight consecutive elements at a 16-byte aligned address.  Otherwise any alignment and any
// width: elements `step` apart, so that the threads of a group still read and write next to each other.
#pragma once
#include <cuda_bf16.h>

#include <type_traits>

#include "rr_common.cuh"

namespace rr {

__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_f32(float v)
{
    if constexpr (sizeof(T) == 4) return v;
    else return __float2bfloat16_rn(v);
}
// v as a value of T holds it
template <class T>
__device__ __forceinline__ float rounded(float v) { return as_f32(from_f32<T>(v)); }

// How a load or store treats the caches: kStream for what is touched once, kKeep for what comes again, kConst for what comes again and
// what nothing in the launch writes to.
enum Cache { kKeep, kStream, kConst };
// A single bf16 goes as the 16-bit word it is: cuda_bf16.h states its cached loads as pure functions of the address, which the compiler may then
// make before the condition that guards them (a missing vector was read from address zero) or move across a store to the same place.
template <Cache C, class V>
__device__ __forceinline__ V fetch(const V *p)
{
    if constexpr (std::is_same<V, __nv_bfloat16>::value) return __ushort_as_bfloat16(fetch<C>(reinterpret_cast<const unsigned short *>(p)));
    else if constexpr (C == kStream) return __ldcs(p);
    else if constexpr (C == kConst) return __ldg(p);
    else return *p;
}
template <Cache C, class V>
__device__ __forceinline__ void place(V *p, V v)
{
    if constexpr (std::is_same<V, __nv_bfloat16>::value) place<C>(reinterpret_cast<unsigned short *>(p), __bfloat16_as_ushort(v));
    else if constexpr (C == kStream) __stcs(p, v);
    else *p = v;
}

template <class T, bool kVec>
struct Eight;

template <>
struct Eight<float, true> {
    float4 a, b;
    template <Cache C = kStream>
    __device__ __forceinline__ void load(const float *p, int, int)
    {
        a = fetch<C>(reinterpret_cast<const float4 *>(p));
        b = fetch<C>(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        a = make_float4(v[0], v[1], v[2], v[3]);
        b = make_float4(v[4], v[5], v[6], v[7]);
    }
    template <Cache C = kStream>
    __device__ __forceinline__ void store(float *p, int, int) const
    {
        place<C>(reinterpret_cast<float4 *>(p), a);
        place<C>(reinterpret_cast<float4 *>(p) + 1, b);
    }
};

template <>
struct Eight<__nv_bfloat16, true> {
    uint4 u;
    template <Cache C = kStream>
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, int, int) { u = fetch<C>(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void zero() { u = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        u = make_uint4(w[0], w[1], w[2], w[3]);
    }
    template <Cache C = kStream>
    __device__ __forceinline__ void store(__nv_bfloat16 *p, int, int) const { place<C>(reinterpret_cast<uint4 *>(p), u); }
};

// p points at the thread's first element, `left` elements of the row are there from it on (elements behind are read as zero and not written)
template <class T>
struct Eight<T, false> {
    T e[8];
    template <Cache C = kStream>
    __device__ __forceinline__ void load(const T *p, int step, int left)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = j * step < left ? fetch<C>(p + j * step) : from_f32<T>(0.f);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = from_f32<T>(0.f);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = as_f32(e[j]);
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = from_f32<T>(v[j]);
    }
    template <Cache C = kStream>
    __device__ __forceinline__ void store(T *p, int step, int left) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * step < left) place<C>(p + j * step, e[j]);
    }
};

}  // namespace rr
