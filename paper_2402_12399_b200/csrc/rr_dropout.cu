// Dropout with the residual add of the branch around an expert (or dense) layer, and its gradient:
//     y_i = residual_i + keep_i x_i / (1 - p),      dx_i = keep_i dy_i / (1 - p)   (+ dx_i when accumulating),
// keep from the counter-based generator of rr_philox.cuh: no mask is written or read, the backward pass computes
// it again.  A dropped element is selected away, not multiplied by zero, so a NaN or infinity in a dropped place
// does not reach y.  One thread takes eight consecutive elements (one generator block).
#include <cuda_bf16.h>

#include "rr_ffn.cuh"
#include "rr_philox.cuh"

namespace rr {

namespace {

constexpr int kDropThreads = 256;

// eight consecutive elements at 16-byte aligned addresses; plain (coherent) loads, because y may be x or residual
__device__ __forceinline__ void read8(const float *p, float (&v)[8])
{
    const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void read8(const __nv_bfloat16 *p, float (&v)[8])
{
    const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(p));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void write8(float *p, const float (&v)[8])
{
    __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void write8(__nv_bfloat16 *p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    __stcs(reinterpret_cast<uint4 *>(p), make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

template <class TX, class TY>
__global__ void __launch_bounds__(kDropThreads) k_dropout(long long n, const TX *x, const TY *residual, DropoutParams d, TY *y)
{
    PhiloxKey key = {};
    if (d.rng) key = philox_key(d.rng);
    const long long groups = (n + 7) >> 3, step = (long long)gridDim.x * kDropThreads;
    for (long long g = (long long)blockIdx.x * kDropThreads + threadIdx.x; g < groups; g += step) {
        const long long i = g * 8;
        if (i + 8 <= n) {
            float v[8], r[8] = {};
            read8(x + i, v);
            if (residual) read8(residual + i, r);
            const uint32_t keep = d.rng ? philox_keep8(key, (unsigned long long)g, d.drop) : 0xffu;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (keep >> j) & 1u ? fmaf(v[j], d.factor, r[j]) : r[j];
            write8(y + i, v);
        } else {  // the last, partial group
            const uint32_t keep = d.rng ? philox_keep8(key, (unsigned long long)g, d.drop) : 0xffu;
            for (int j = 0; i + j < n; ++j) {
                const float r = residual ? as_float(residual[i + j]) : 0.0f;
                put(y + i + j, (keep >> j) & 1u ? fmaf(as_float(x[i + j]), d.factor, r) : r);
            }
        }
    }
}

template <class TX, class TY>
rr_status run(long long n, const void *x, const void *residual, const DropoutParams &d, void *y, cudaStream_t st)
{
    const long long groups = (n + 7) / 8, want = (groups + kDropThreads - 1) / kDropThreads;
    const int grid = (int)(want < 148 * 8 ? want : 148 * 8);
    k_dropout<TX, TY><<<grid, kDropThreads, 0, st>>>(n, static_cast<const TX *>(x), static_cast<const TY *>(residual), d,
                                                     static_cast<TY *>(y));
    return cudaGetLastError() == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

}  // namespace

rr_status launch_dropout(long long n, int x_dtype, int y_dtype, const void *x, const void *residual, float p, const void *rng,
                         void *y, cudaStream_t st)
{
    const DropoutParams d = dropout_params(p, rng);
    if (x_dtype == RR_F32)
        return y_dtype == RR_F32 ? run<float, float>(n, x, residual, d, y, st) : run<float, __nv_bfloat16>(n, x, residual, d, y, st);
    return y_dtype == RR_F32 ? run<__nv_bfloat16, float>(n, x, residual, d, y, st)
                             : run<__nv_bfloat16, __nv_bfloat16>(n, x, residual, d, y, st);
}

}  // namespace rr
