// Epilogue of the dense linear layer: bias, activation, dropout, residual on tiles of the fp32 accumulator, and the
// activations' derivatives for its backward pass.
#pragma once
#include <cuda_bf16.h>
#include <float.h>

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

using tc::ex2;
using tc::kLog2e;
using tc::rcp;

// The normal distribution function of a pair as copysign(h, v) + 1/2, and e^(-v^2/2), 2.5 times the density:
// Phi(v) = erfc(|v| / sqrt 2) / 2 mirrored, with erfc(t) = (a1 u + a2 u^2 + .. + a5 u^5) e^{-t^2}, u = 1 / (1 + 0.3275911 t)
// (Abramowitz and Stegun 7.1.26, absolute error below 1.5e-7); h = 1/2 - half of that.
__device__ __forceinline__ void normal_pair(float v0, float v1, float &h0, float &h1, tc::f32x2 &e)
{
    using namespace tc;
    const f32x2 x = pack2(v0, v1);
    float a, b;
    unpack2(mul2(mul2(x, x), pack2(-0.5f * kLog2e, -0.5f * kLog2e)), a, b);
    e = pack2(ex2(a), ex2(b));
    constexpr float p = 0.3275911f * 0.70710678f;
    const f32x2 u = pack2(rcp(fmaf(fabsf(v0), p, 1.0f)), rcp(fmaf(fabsf(v1), p, 1.0f)));
    f32x2 q = fma2(pack2(-0.5f * 1.061405429f, -0.5f * 1.061405429f), u, pack2(0.5f * 1.453152027f, 0.5f * 1.453152027f));
    q = fma2(q, u, pack2(-0.5f * 1.421413741f, -0.5f * 1.421413741f));
    q = fma2(q, u, pack2(0.5f * 0.284496736f, 0.5f * 0.284496736f));
    q = fma2(q, u, pack2(-0.5f * 0.254829592f, -0.5f * 0.254829592f));
    unpack2(fma2(mul2(q, u), e, pack2(0.5f, 0.5f)), h0, h1);
}

constexpr float kTanhA = 1.5957691216f;  // 2 sqrt(2 / pi)
constexpr float kTanhB = 0.044715f;

// -log2(e) times the argument of the sigmoid that SiLU and the tanh form of GELU multiply v by
template <int kAct>
__device__ __forceinline__ tc::f32x2 sigmoid_argument(tc::f32x2 x)
{
    using namespace tc;
    if (kAct == RR_ACT_SILU) return mul2(x, pack2(-kLog2e, -kLog2e));
    constexpr float b = -kLog2e * kTanhA * kTanhB, a = -kLog2e * kTanhA;
    return mul2(x, fma2(mul2(x, x), pack2(b, b), pack2(a, a)));
}
__device__ __forceinline__ float finite(float v) { return fminf(fmaxf(v, -FLT_MAX), FLT_MAX); }  // (a NaN becomes a number)

// act'(v) of eight values, in packed fp32 pairs where the operation exists for pairs.  A NaN stays a NaN (through the exponential);
// at +-infinity, where the other factor is 0, the bounded v keeps the product from being a NaN.
template <int kAct>
__device__ __forceinline__ void act_slope8(float *v)
{
    using namespace tc;
    const f32x2 one = pack2(1.0f, 1.0f);
    if constexpr (kAct == RR_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = v[j] > 0.0f ? 1.0f : 0.0f;
    }
    if constexpr (kAct == RR_ACT_SILU || kAct == RR_ACT_GELU_TANH) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float a, b;
            unpack2(sigmoid_argument<kAct>(pack2(v[j], v[j + 1])), a, b);
            unpack2(add2(pack2(ex2(a), ex2(b)), one), a, b);
            const f32x2 s = pack2(rcp(a), rcp(b)), minus = pack2(-1.0f, -1.0f);
            // s + x dw/dv s (1 - s);   (1 - s as -(s - 1)); where v is large enough for v^3 to overflow, s (1 - s) is 0 and v bounded
            const f32x2 x = pack2(fminf(fmaxf(v[j], -1e4f), 1e4f), fminf(fmaxf(v[j + 1], -1e4f), 1e4f));
            f32x2 xw = x;
            if (kAct == RR_ACT_GELU_TANH)
                xw = mul2(x, fma2(mul2(x, x), pack2(3.0f * kTanhA * kTanhB, 3.0f * kTanhA * kTanhB), pack2(kTanhA, kTanhA)));
            unpack2(fma2(mul2(xw, s), fma2(s, minus, one), s), v[j], v[j + 1]);
        }
    }
    if constexpr (kAct == RR_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float h0, h1;
            f32x2 e;
            normal_pair(v[j], v[j + 1], h0, h1, e);
            const f32x2 cdf = add2(pack2(copysignf(h0, v[j]), copysignf(h1, v[j + 1])), pack2(0.5f, 0.5f));
            unpack2(fma2(pack2(finite(v[j]), finite(v[j + 1])), mul2(e, pack2(0.39894228f, 0.39894228f)), cdf), v[j], v[j + 1]);
        }
    }
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

// The activation of eight values, likewise.
template <int kAct>
__device__ __forceinline__ void act8(float *v)
{
    using namespace tc;
    if constexpr (kAct == RR_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = v[j] <= 0.0f ? 0.0f : v[j];
    }
    if constexpr (kAct == RR_ACT_SILU || kAct == RR_ACT_GELU_TANH) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float a, b;
            unpack2(sigmoid_argument<kAct>(pack2(v[j], v[j + 1])), a, b);
            unpack2(add2(pack2(ex2(a), ex2(b)), pack2(1.0f, 1.0f)), a, b);
            unpack2(mul2(pack2(fmaxf(v[j], -FLT_MAX), fmaxf(v[j + 1], -FLT_MAX)), pack2(rcp(a), rcp(b))), v[j], v[j + 1]);
        }
    }
    if constexpr (kAct == RR_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float h0, h1;
            f32x2 e;
            normal_pair(v[j], v[j + 1], h0, h1, e);
            unpack2(mul2(pack2(fmaxf(v[j], -FLT_MAX), fmaxf(v[j + 1], -FLT_MAX)), add2(pack2(copysignf(h0, v[j]), copysignf(h1, v[j + 1])), pack2(0.5f, 0.5f))),
                    v[j], v[j + 1]);
        }
    }
}

__device__ __forceinline__ void add_pair(float *v, float a, float b)
{
    tc::unpack2(tc::add2(tc::pack2(v[0], v[1]), tc::pack2(a, b)), v[0], v[1]);
}

template <int kAct>
__device__ __forceinline__ void act32(float *v)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) act8<kAct>(v + 8 * j);
}
// the activation of eight values
__device__ __forceinline__ void activate8(int act, float *v)
{
    switch (act) {
    case RR_ACT_RELU: act8<RR_ACT_RELU>(v); break;
    case RR_ACT_GELU: act8<RR_ACT_GELU>(v); break;
    case RR_ACT_GELU_TANH: act8<RR_ACT_GELU_TANH>(v); break;
    case RR_ACT_SILU: act8<RR_ACT_SILU>(v); break;
    default: break;
    }
}
// dropout of eight consecutive elements whose generator words are w
__device__ __forceinline__ void drop8(const uint32_t (&w)[4], uint32_t bound, float factor, float *v)
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float a, b;
        tc::unpack2(tc::mul2(tc::pack2(v[i], v[i + 1]), tc::pack2(factor, factor)), a, b);
        v[i] = keep(w, i, bound) ? a : 0.0f;
        v[i + 1] = keep(w, i + 1, bound) ? b : 0.0f;
    }
}

// The whole epilogue of eight consecutive columns [col, col+8) of one row, results written straight to memory.
__device__ __forceinline__ void finish8(const Epilogue &e, const PhiloxKey &key, float (&v)[8], long long row, int col, int N, void *y,
                                        long long ldy, __nv_bfloat16 *z, long long ldz)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= e.alpha;
    if (e.bias) {
        float b[8];
        unpack8(__ldg(reinterpret_cast<const uint4 *>(e.bias + col)), b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += b[i];
    }
    if (z) *reinterpret_cast<uint4 *>(z + row * ldz + col) = pack8(v);
    activate8(e.act, v);
    if (e.drop.rng) {
        uint32_t w[1][4];
        philox_words<1>(key, ((unsigned long long)row * (unsigned)N + (unsigned)col) >> 3, e.drop.drop, w);
        drop8(w[0], keep_bound(e.drop.drop), e.drop.factor, v);
    }
    if (e.y_f32) {
        float4 *out = reinterpret_cast<float4 *>(static_cast<float *>(y) + row * ldy + col);
        if (e.residual) {
            const float4 *r = reinterpret_cast<const float4 *>(static_cast<const float *>(e.residual) + row * e.ldr + col);
            const float4 a = r[0], b = r[1];
            v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
        }
        out[0] = make_float4(v[0], v[1], v[2], v[3]);
        out[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        if (e.residual) {
            float a[8];
            unpack8(*reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(e.residual) + row * e.ldr + col), a);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += a[i];
        }
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(y) + row * ldy + col) = pack8(v);
    }
}

// One epilogue warp of the tiled kernel: 32 rows (lane = row) x 32 columns at a time.  Results leave through the warp's
// 2 KB staging tile by TMA stores, which clip at the matrix's edges: 64-byte rows, lane r writes its row in 16-byte
// pieces, piece j at j ^ ((r >> 1) & 3); bf16 in one piece of 32 columns, fp32 in two of 16.
struct EpilogueWarp {
    PhiloxKey key;
    uint4 ahead[4];  // bf16 residual of the next chunk: requested before the accumulator is waited for

    float ahead_bias;  // and its bias, of column col0 + lane

    template <bool kForward>
    __device__ __forceinline__ void fetch(const Epilogue &e, int row, int col0, int M, int N, int lane)
    {
        if (kForward && e.bias) ahead_bias = col0 + lane < N ? __bfloat162float(e.bias[col0 + lane]) : 0.0f;
        if (!e.residual || e.y_f32) return;
        const __nv_bfloat16 *r = static_cast<const __nv_bfloat16 *>(e.residual) + row * e.ldr + col0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            ahead[j] = make_uint4(0u, 0u, 0u, 0u);
            if (row < M && col0 + 8 * j < N) ahead[j] = *reinterpret_cast<const uint4 *>(r + 8 * j);
        }
    }

    __device__ __forceinline__ static void reuse_tile(int lane)  // the store before has read the staging tile
    {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }
    __device__ __forceinline__ static void send(const uint8_t *st, const CUtensorMap *map, int col0, int row0, int lane)
    {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            tc::tma_store_2d(map, st, col0, row0);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    }
    __device__ __forceinline__ static void send_bf16(const float *v, uint8_t *st, const CUtensorMap *map, int col0, int row0, int lane)
    {
        reuse_tile(lane);
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4 *>(st + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = pack8(v + 8 * j);
        send(st, map, col0, row0, lane);
    }

    // accumulator columns [col0, col0+32) of rows [row0, row0+32); N is a multiple of 8; `next` < 0: no chunk follows
    // `bias`: 32 floats of shared memory of this warp; `shift`: rows between these and their place behind mapY
    template <bool kForward>
    __device__ __forceinline__ void chunk(const Epilogue &e, float (&v)[32], float *bias, int row0, int shift, int col0, int next, int M, int N,
                                          int lane, uint8_t *st, const CUtensorMap *mapY, const CUtensorMap *mapZ)
    {
        const int row = row0 + lane;
        if constexpr (kForward) {
            if (e.bias) {
                __syncwarp();
                bias[lane] = ahead_bias;
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float4 b = *reinterpret_cast<const float4 *>(bias + 4 * j);
                    add_pair(v + 4 * j, b.x, b.y);
                    add_pair(v + 4 * j + 2, b.z, b.w);
                }
            }
            if (e.save_z) send_bf16(v, st, mapZ, col0, row0, lane);
            switch (e.act) {
            case RR_ACT_RELU: act32<RR_ACT_RELU>(v); break;
            case RR_ACT_GELU: act32<RR_ACT_GELU>(v); break;
            case RR_ACT_GELU_TANH: act32<RR_ACT_GELU_TANH>(v); break;
            case RR_ACT_SILU: act32<RR_ACT_SILU>(v); break;
            default: break;
            }
            if (e.drop.rng) {
                uint32_t w[4][4];
                philox_words<4>(key, ((unsigned long long)row * (unsigned)N + (unsigned)col0) >> 3, e.drop.drop, w);
                const uint32_t bound = keep_bound(e.drop.drop);
#pragma unroll
                for (int j = 0; j < 4; ++j) drop8(w[j], bound, e.drop.factor, v + 8 * j);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; j += 2) tc::unpack2(tc::mul2(tc::pack2(v[j], v[j + 1]), tc::pack2(e.alpha, e.alpha)), v[j], v[j + 1]);
        }
        if (!e.y_f32) {
            if (e.residual) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float a[8];
                    unpack8(ahead[j], a);
#pragma unroll
                    for (int i = 0; i < 8; i += 2) add_pair(v + 8 * j + i, a[i], a[i + 1]);
                }
            }
            if (next >= 0) fetch<kForward>(e, row, next, M, N, lane);
            send_bf16(v, st, mapY, col0, row0 + shift, lane);
        } else {
            if (next >= 0) fetch<kForward>(e, row, next, M, N, lane);
            const float *r = static_cast<const float *>(e.residual) + row * e.ldr + col0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (col0 + 16 * h >= N) break;
                reuse_tile(lane);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = 16 * h + 4 * j;
                    float4 a = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
                    if (e.residual && row < M && col0 + c < N) {
                        const float4 b = *reinterpret_cast<const float4 *>(r + c);
                        a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
                    }
                    *reinterpret_cast<float4 *>(st + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = a;
                }
                send(st, mapY, col0 + 16 * h, row0 + shift, lane);
            }
        }
    }
};

}  // namespace rr
