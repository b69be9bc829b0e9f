// Epilogue of the dense linear layer: bias, activation, dropout, residual on tiles of the fp32 accumulator, and the
// activations' derivatives for its backward pass.
#pragma once
#include <cuda_bf16.h>

#include "rr_common.cuh"
#include "rr_philox.cuh"
#include "rr_tc.cuh"

namespace rr {

struct Epilogue {
    const __nv_bfloat16 *bias;  // [N] or null
    const void *residual;       // y's type, pitch ldr, or null; may be y
    long long ldr;
    int act;                    // RR_ACT_*
    int y_f32;                  // y and residual are fp32, else bf16
    int save_z;                 // z = accumulator + bias leaves as bf16
    DropoutParams drop;
    float alpha;                // factor of the accumulator
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float sigmoid(float v) { return rcp(1.0f + ex2(-kLog2e * v)); }

// The normal distribution function and density.  Phi(v) = erfc(|v| / sqrt 2) / 2 mirrored, with
// erfc(t) = (a1 u + a2 u^2 + .. + a5 u^5) e^{-t^2}, u = 1 / (1 + 0.3275911 t)   (Abramowitz and Stegun 7.1.26,
// absolute error below 1.5e-7): the exponential is the density's, so the derivative costs nothing more.
__device__ __forceinline__ void normal_cdf_pdf(float v, float &cdf, float &pdf)
{
    const float t = fabsf(v) * 0.70710678f;
    const float e = ex2(-kLog2e * t * t);
    const float u = rcp(fmaf(0.3275911f, t, 1.0f));
    float q = fmaf(1.061405429f, u, -1.453152027f);
    q = fmaf(q, u, 1.421413741f);
    q = fmaf(q, u, -0.284496736f);
    q = fmaf(q, u, 0.254829592f);
    const float half_tail = 0.5f * q * u * e;
    cdf = v < 0.0f ? half_tail : 1.0f - half_tail;
    pdf = 0.39894228f * e;
}

constexpr float kTanhA = 1.5957691216f;  // 2 sqrt(2 / pi)
constexpr float kTanhB = 0.044715f;

// A NaN stays a NaN; at +-infinity the limits: v or 0 (v sigmoid(v) is -inf * 0 there, so the product is guarded).
template <int kAct>
__device__ __forceinline__ float act_value(float v)
{
    if constexpr (kAct == RR_ACT_RELU) return v > 0.0f ? v : (v != v ? v : 0.0f);
    if constexpr (kAct == RR_ACT_SILU || kAct == RR_ACT_GELU_TANH) {
        // both are v sigmoid(w): w = v, or (0.5 v (1 + tanh(w / 2)))  w = 2 sqrt(2/pi) (v + 0.044715 v^3)
        const float s = sigmoid(kAct == RR_ACT_SILU ? v : kTanhA * v * fmaf(kTanhB * v, v, 1.0f));
        return s == 0.0f ? 0.0f : v * s;
    }
    if constexpr (kAct == RR_ACT_GELU) {
        float cdf, pdf;
        normal_cdf_pdf(v, cdf, pdf);
        return cdf == 0.0f ? 0.0f : v * cdf;
    }
    return v;
}
template <int kAct>
__device__ __forceinline__ float act_slope(float v)
{
    if constexpr (kAct == RR_ACT_RELU) return v > 0.0f ? 1.0f : 0.0f;
    if constexpr (kAct == RR_ACT_SILU) {
        const float s = sigmoid(v);
        return s == 0.0f ? 0.0f : s == 1.0f ? 1.0f : s * fmaf(v, 1.0f - s, 1.0f);
    }
    if constexpr (kAct == RR_ACT_GELU_TANH) {
        const float s = sigmoid(kTanhA * v * fmaf(kTanhB * v, v, 1.0f));
        return s == 0.0f ? 0.0f : s == 1.0f ? 1.0f : fmaf(v * s * (1.0f - s), kTanhA * fmaf(3.0f * kTanhB * v, v, 1.0f), s);
    }
    if constexpr (kAct == RR_ACT_GELU) {
        float cdf, pdf;
        normal_cdf_pdf(v, cdf, pdf);
        return pdf == 0.0f ? cdf : fmaf(v, pdf, cdf);
    }
    return 1.0f;
}

__device__ __forceinline__ void unpack8(const uint4 &u, float (&v)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float *v)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int kAct>
__device__ __forceinline__ void act8(float *v)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = act_value<kAct>(v[j]);
}

// One epilogue warp: 32 rows (lane = row) x 32 columns at a time.  Results leave through the warp's 4 KB staging tile
// by TMA stores, which clip at the matrix's edges: lane r writes its row in 16-byte pieces, piece j at
// j ^ (r & 7) of 128-byte rows (fp32) or j ^ ((r >> 1) & 3) of 64-byte rows (bf16: two tiles of 2 KB in turn).
struct EpilogueWarp {
    PhiloxKey key;
    uint32_t stores;

    __device__ __forceinline__ explicit EpilogueWarp(const Epilogue &e) : key{}, stores(0)
    {
        if (e.drop.rng) key = philox_key(e.drop.rng);
    }

    // sends 32 x 32 bf16 through the next 2 KB tile
    __device__ __forceinline__ void send_bf16(const float *v, uint8_t *st, const CUtensorMap *map, int col0, int row0, int lane)
    {
        uint8_t *bt = st + (stores & 1u) * 2048;
        if (stores >= 2) {  // the store before the last one has read this tile
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            __syncwarp();
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4 *>(bt + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = pack8(v + 8 * j);
        finish(bt, map, col0, row0, lane);
    }
    __device__ __forceinline__ void send_f32(const float *v, uint8_t *st, const CUtensorMap *map, int col0, int row0, int lane)
    {
        if (stores >= 1) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            *reinterpret_cast<float4 *>(st + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        finish(st, map, col0, row0, lane);
    }
    __device__ __forceinline__ void finish(uint8_t *bt, const CUtensorMap *map, int col0, int row0, int lane)
    {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            tc::tma_store_2d(map, bt, col0, row0);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        ++stores;
    }

    // accumulator columns [col0, col0+32) of rows [row0, row0+32), lane = row; N is a multiple of 8
    __device__ __forceinline__ void chunk(const Epilogue &e, float (&v)[32], int row0, int col0, int M, int N, int lane, uint8_t *st,
                                          const CUtensorMap *mapY, const CUtensorMap *mapZ)
    {
        const int row = row0 + lane;
        const bool live = row < M;
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= e.alpha;
        if (e.bias) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (col0 + 8 * j < N) {
                    float b[8];
                    unpack8(__ldg(reinterpret_cast<const uint4 *>(e.bias + col0 + 8 * j)), b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[8 * j + i] += b[i];
                }
            }
        }
        if (e.save_z) {
            if (e.y_f32 && stores >= 1) {  // (the fp32 tile of the store before lies over both bf16 tiles)
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                __syncwarp();
            }
            send_bf16(v, st, mapZ, col0, row0, lane);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            switch (e.act) {
            case RR_ACT_RELU: act8<RR_ACT_RELU>(v + 8 * j); break;
            case RR_ACT_GELU: act8<RR_ACT_GELU>(v + 8 * j); break;
            case RR_ACT_GELU_TANH: act8<RR_ACT_GELU_TANH>(v + 8 * j); break;
            case RR_ACT_SILU: act8<RR_ACT_SILU>(v + 8 * j); break;
            default: break;
            }
        }
        if (e.drop.rng) {
            const unsigned long long g0 = ((unsigned long long)row * (unsigned)N + (unsigned)col0) >> 3;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t keep = philox_keep8(key, g0 + j, e.drop.drop);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * j + i] = (keep >> i) & 1u ? v[8 * j + i] * e.drop.factor : 0.0f;
            }
        }
        if (e.residual && live) {
            if (e.y_f32) {
                const float *r = static_cast<const float *>(e.residual) + row * e.ldr + col0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (col0 + 4 * j < N) {
                        const float4 a = *reinterpret_cast<const float4 *>(r + 4 * j);
                        v[4 * j] += a.x; v[4 * j + 1] += a.y; v[4 * j + 2] += a.z; v[4 * j + 3] += a.w;
                    }
                }
            } else {
                const __nv_bfloat16 *r = static_cast<const __nv_bfloat16 *>(e.residual) + row * e.ldr + col0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (col0 + 8 * j < N) {
                        float a[8];
                        unpack8(*reinterpret_cast<const uint4 *>(r + 8 * j), a);
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[8 * j + i] += a[i];
                    }
                }
            }
        }
        if (e.y_f32) send_f32(v, st, mapY, col0, row0, lane);
        else send_bf16(v, st, mapY, col0, row0, lane);
    }
};

}  // namespace rr
