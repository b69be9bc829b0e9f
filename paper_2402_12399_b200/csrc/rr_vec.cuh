// Eight elements of a row per thread and step, bf16 or fp32, as they lie in memory: the access shared by the memory-bound operators of a
// training step (norm, embedding, clip).
#pragma once
#include <cuda_bf16.h>

#include <type_traits>

#include "rr_common.cuh"
#include "rr_tc.cuh"

namespace rr {

__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_f32(float v)
{
    if constexpr (sizeof(T) == 4) return v;
    else return __float2bfloat16_rn(v);
}

// How a load or store treats the caches: kStream for what is touched once, kKeep for what comes again.  (No loads past the coherent path: a kernel
// that is made ready while the one in front of it still writes must not promise that what it reads stays as it is while it runs.)
enum Cache { kKeep, kStream };
// A single bf16 goes as the 16-bit word it is: cuda_bf16.h states its cached loads as pure functions of the address, which the compiler may then
// make before the condition that guards them (a missing vector was read from address zero) or move across a store to the same place.
template <Cache C, class V>
__device__ __forceinline__ V fetch(const V *p)
{
    if constexpr (std::is_same<V, __nv_bfloat16>::value) return __ushort_as_bfloat16(fetch<C>(reinterpret_cast<const unsigned short *>(p)));
    else if constexpr (C == kStream) return __ldcs(p);
    else return __ldca(p);  // (which, as __ldcs, stays where it is written: loads asked for together are asked for together)
}
template <Cache C, class V>
__device__ __forceinline__ void place(V *p, V v)
{
    if constexpr (std::is_same<V, __nv_bfloat16>::value) place<C>(reinterpret_cast<unsigned short *>(p), __bfloat16_as_ushort(v));
    else if constexpr (C == kStream) __stcs(p, v);
    else *p = v;
}

using tc::f32x2;

// two bf16 of a word as an fp32 pair, and back
__device__ __forceinline__ f32x2 pair_of(uint32_t w) { return tc::pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t word_of(f32x2 v) { return tc::pack_bf16x2(v); }

// kN consecutive elements at an address that is a multiple of their size: 16 bytes, or the four bf16 beside four fp32; or one element
template <class T, int kN>
struct Unit {
    using Raw = std::conditional_t<kN == 1, std::conditional_t<sizeof(T) == 4, float, unsigned short>,
                                   std::conditional_t<sizeof(T) * kN == 8, uint2, std::conditional_t<sizeof(T) == 4, float4, uint4>>>;
    Raw raw;
    template <Cache C>
    __device__ __forceinline__ void load(const T *p) { raw = fetch<C>(reinterpret_cast<const Raw *>(p)); }
    template <Cache C>
    __device__ __forceinline__ void store(T *p) const { place<C>(reinterpret_cast<Raw *>(p), raw); }
    __device__ __forceinline__ void get(float (&v)[kN]) const
    {
        if constexpr (kN == 1) {
            if constexpr (sizeof(T) == 4) v[0] = raw;
            else v[0] = __uint_as_float((uint32_t)raw << 16);
        } else if constexpr (sizeof(T) == 4) {
            v[0] = raw.x; v[1] = raw.y; v[2] = raw.z; v[3] = raw.w;
        } else {
            tc::unpack2(pair_of(raw.x), v[0], v[1]);
            tc::unpack2(pair_of(raw.y), v[2], v[3]);
            if constexpr (kN == 8) {
                tc::unpack2(pair_of(raw.z), v[4], v[5]);
                tc::unpack2(pair_of(raw.w), v[6], v[7]);
            }
        }
    }
    __device__ __forceinline__ void set(const float (&v)[kN])
    {
        if constexpr (kN == 1) {
            if constexpr (sizeof(T) == 4) raw = v[0];
            else raw = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
        } else if constexpr (sizeof(T) == 4) {
            raw = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            raw.x = word_of(tc::pack2(v[0], v[1]));
            raw.y = word_of(tc::pack2(v[2], v[3]));
            if constexpr (kN == 8) {
                raw.z = word_of(tc::pack2(v[4], v[5]));
                raw.w = word_of(tc::pack2(v[6], v[7]));
            }
        }
    }
};
template <int kN, class A, class B>
__device__ __forceinline__ void scaled(const Unit<A, kN> &from, Unit<B, kN> &to, float f)
{
    float v[kN];
    from.get(v);
    if constexpr (kN == 1) {
        v[0] *= f;
    } else {
        const f32x2 two = tc::pack2(f, f);
#pragma unroll
        for (int j = 0; j < kN; j += 2) tc::unpack2(tc::mul2(tc::pack2(v[j], v[j + 1]), two), v[j], v[j + 1]);
    }
    to.set(v);
}

// Where the eight elements of a thread lie, so that the threads of a group read and write whole 32-byte sectors side by side:
//   kEights  eight next to each other, 16 bytes of bf16 (in fp32 a warp would touch every sector twice)
//   kQuads   four next to each other and four more `step` elements on: 16 bytes of fp32, 8 of bf16
//   kOne     eight elements `step` apart: any width, any alignment
enum Layout { kOne, kQuads, kEights };

__device__ __forceinline__ void quad_of(const float4 &q, f32x2 &a, f32x2 &b) { a = tc::pack2(q.x, q.y); b = tc::pack2(q.z, q.w); }
__device__ __forceinline__ void quad_of(const uint2 &q, f32x2 &a, f32x2 &b) { a = pair_of(q.x); b = pair_of(q.y); }
__device__ __forceinline__ void quad_from(float4 &q, f32x2 a, f32x2 b) { tc::unpack2(a, q.x, q.y); tc::unpack2(b, q.z, q.w); }
__device__ __forceinline__ void quad_from(uint2 &q, f32x2 a, f32x2 b) { q = make_uint2(word_of(a), word_of(b)); }

// p points at the thread's first element; `left` elements of the row are there from it on.  What lies behind the row is read as zero and not
// written (with kEights the width is a multiple of eight, with kQuads of four).
template <class T, Layout L>
struct Eight;

template <class T>
struct Eight<T, kEights> {
    uint4 q[sizeof(T) / 2];
    template <Cache C = kStream>
    __device__ __forceinline__ void load(const T *p, int, int)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = fetch<C>(reinterpret_cast<const uint4 *>(p) + i);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void get(f32x2 (&v)[4]) const
    {
        if constexpr (sizeof(T) == 2) {
            v[0] = pair_of(q[0].x); v[1] = pair_of(q[0].y); v[2] = pair_of(q[0].z); v[3] = pair_of(q[0].w);
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                quad_of(make_float4(__uint_as_float(q[i].x), __uint_as_float(q[i].y), __uint_as_float(q[i].z), __uint_as_float(q[i].w)), v[2 * i], v[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void set(const f32x2 (&v)[4])
    {
        if constexpr (sizeof(T) == 2) {
            q[0] = make_uint4(word_of(v[0]), word_of(v[1]), word_of(v[2]), word_of(v[3]));
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
                float4 f;
                quad_from(f, v[2 * i], v[2 * i + 1]);
                q[i] = make_uint4(__float_as_uint(f.x), __float_as_uint(f.y), __float_as_uint(f.z), __float_as_uint(f.w));
            }
        }
    }
    template <Cache C = kStream>
    __device__ __forceinline__ void store(T *p, int, int) const
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) place<C>(reinterpret_cast<uint4 *>(p) + i, q[i]);
    }
};

template <class T>
struct Eight<T, kQuads> {
    using Quad = std::conditional_t<sizeof(T) == 4, float4, uint2>;
    Quad a, b;
    template <Cache C = kStream>
    __device__ __forceinline__ void load(const T *p, int step, int left)
    {
        a = fetch<C>(reinterpret_cast<const Quad *>(p));
        b = Quad{};
        if (step < left) b = fetch<C>(reinterpret_cast<const Quad *>(p + step));
    }
    __device__ __forceinline__ void zero() { a = b = Quad{}; }
    __device__ __forceinline__ void get(f32x2 (&v)[4]) const
    {
        quad_of(a, v[0], v[1]);
        quad_of(b, v[2], v[3]);
    }
    __device__ __forceinline__ void set(const f32x2 (&v)[4])
    {
        quad_from(a, v[0], v[1]);
        quad_from(b, v[2], v[3]);
    }
    template <Cache C = kStream>
    __device__ __forceinline__ void store(T *p, int step, int left) const
    {
        place<C>(reinterpret_cast<Quad *>(p), a);
        if (step < left) place<C>(reinterpret_cast<Quad *>(p + step), b);
    }
};

template <class T>
struct Eight<T, kOne> {
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
    __device__ __forceinline__ void get(f32x2 (&v)[4]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = tc::pack2(as_f32(e[2 * j]), as_f32(e[2 * j + 1]));
    }
    __device__ __forceinline__ void set(const f32x2 (&v)[4])
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x, y;
            tc::unpack2(v[j], x, y);
            e[2 * j] = from_f32<T>(x);
            e[2 * j + 1] = from_f32<T>(y);
        }
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
