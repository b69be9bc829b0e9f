// Dropout with the residual add of the branch around an expert (or dense) layer, and its gradient:
//     y_i = residual_i + keep_i x_i / (1 - p),      dx_i = keep_i dy_i / (1 - p)   (+ dx_i when accumulating),
// keep from the counter-based generator of rr_philox.cuh: no mask is written or read, the backward pass computes
// it again.  A dropped element is selected away, not multiplied by zero, so a NaN or infinity in a dropped place
// does not reach y.  A thread takes two groups of eight consecutive elements at a time (a generator block each): their loads are in
// flight together and they share the key schedule, which leaves about 110 instructions a group (162 one by one).
// 2^26 elements: fp32 + bf16 residual -> bf16 81.8 us (1.00 of the measured copy rate of HBM), bf16 -> bf16 48 us (0.85, about half of
// the time is the generator's; 64 us with one group at a time), fp32 + residual -> fp32 142 us (0.86).
#include <cuda_bf16.h>

#include "rr_ffn.cuh"
#include "rr_philox.cuh"

namespace rr {

namespace {

constexpr int kDropThreads = 256;

// Blocks per SM, all resident at once.  Where every element moves 6 bytes or more HBM is the bound and fewer streams of reads and writes
// suit it better (2^26 elements, fp32 + bf16 residual -> bf16: 81.8 us with three, 84.7 with four, 95 with five; bf16 -> fp32: 69 and 78);
// with 4 bytes the generator's integer work is as long and wants the warps (bf16 -> bf16: 52.2 with three, 48.0 with four).
template <class TX, class TY>
constexpr int drop_blocks() { return sizeof(TX) + sizeof(TY) == 4 ? 4 : 3; }

// Eight consecutive elements at a 16-byte aligned address as they lie in memory, and as fp32.  Plain (coherent) loads, because y
// may be x or residual.
template <class T>
struct Raw8;
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void read(const float *p)
    {
        a = __ldcs(reinterpret_cast<const float4 *>(p));
        b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
template <>
struct Raw8<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void read(const __nv_bfloat16 *p) { u = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
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

template <class TX, class TY, bool kResidual>
__global__ void __launch_bounds__(kDropThreads, (drop_blocks<TX, TY>())) k_dropout(long long n, const TX *x, const TY *residual, DropoutParams d, TY *y)
{
    dependent_start();
    PhiloxKey key = {};
    if (d.rng) key = philox_key(d.rng);
    const uint32_t bound = keep_bound(d.drop);
    const long long groups = (n + 7) >> 3, whole = n >> 3, step = (long long)gridDim.x * kDropThreads;
    const long long g0 = (long long)blockIdx.x * kDropThreads + threadIdx.x;
    auto one = [&](long long g, const Raw8<TX> &rx, const Raw8<TY> &rr, const uint32_t (&w)[4]) {
        float v[8], r[8] = {};
        rx.get(v);
        if (kResidual) rr.get(r);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = !d.rng || keep(w, j, bound) ? fmaf(v[j], d.factor, r[j]) : r[j];
        write8(y + g * 8, v);
    };
    long long g = g0;
    for (; g + step < whole; g += 2 * step) {  // two groups at once: loads in flight together, one key schedule
        Raw8<TX> xa, xb;
        Raw8<TY> ra, rb;
        xa.read(x + g * 8);
        xb.read(x + (g + step) * 8);
        if (kResidual) {
            ra.read(residual + g * 8);
            rb.read(residual + (g + step) * 8);
        }
        uint32_t w[2][4];
        if (d.rng) philox_words<2>(key, (unsigned long long)g, d.drop, w, (unsigned long long)step);
        one(g, xa, ra, w[0]);
        one(g + step, xb, rb, w[1]);
    }
    if (g < whole) {
        Raw8<TX> xa;
        Raw8<TY> ra;
        xa.read(x + g * 8);
        if (kResidual) ra.read(residual + g * 8);
        uint32_t w[1][4];
        if (d.rng) philox_words<1>(key, (unsigned long long)g, d.drop, w);
        one(g, xa, ra, w[0]);
    }
    if (whole < groups && whole % step == g0) {  // the last, partial group
        uint32_t w[1][4];
        if (d.rng) philox_words<1>(key, (unsigned long long)whole, d.drop, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const long long i = whole * 8 + j;
            if (i >= n) break;
            const float r = kResidual ? as_float(residual[i]) : 0.0f;
            put(y + i, !d.rng || keep(w[0], j, bound) ? fmaf(as_float(x[i]), d.factor, r) : r);
        }
    }
}

template <class TX, class TY>
rr_status run(long long n, const void *x, const void *residual, const DropoutParams &d, void *y, cudaStream_t st)
{
    const long long groups = (n + 7) / 8, want = (groups + kDropThreads - 1) / kDropThreads;
    const int sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    const int most = sms * drop_blocks<TX, TY>(), grid = (int)(want < most ? want : most);
    const TX *px = static_cast<const TX *>(x);
    const TY *pr = static_cast<const TY *>(residual);
    const cudaError_t err = launch_dependent(residual ? k_dropout<TX, TY, true> : k_dropout<TX, TY, false>, dim3(grid), kDropThreads, 0, 1, st, n, px, pr, d,
                                             static_cast<TY *>(y));
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
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
