// The norm in front of a branch, with the residual add of the branch before it, and its gradients.  Layer norm and RMS norm:
//     h = residual + x  (rounded to the stream's type),   mu = mean(h) (RMS: 0),   rstd = 1 / sqrt(mean((h - mu)^2) + eps)
//     y = (h - mu) rstd w + b
//     xh = (h - mu) rstd,  g = dy w:   dx = dh + rstd (g - [mean(g)] - xh mean(g xh)),   dw = sum over rows dy xh,   db = sum over rows dy
// (mean(g) for the layer norm only).  A row is read once and held in registers, so the variance is that of differences from the mean
// and not a difference of squares; both passes are bound by HBM, and by latency where rows are few.  Statistics and sums are fp32.
// Measured: forward 16384 x 4096, fp32 + bf16 residual 99 us (6.8 TB/s), 65536 x 1024 in bf16 43.5 (6.2 TB/s), one row of 4096 2.1.  Gradients in bf16,
// joined with the stream's: 16384 x 4096 RMS 88 us (6.1 TB/s), 65536 x 1024 layer norm 90, 65536 x 1023 167 (elements one by one), one row 4.1.
#pragma once
#include <type_traits>

#include "rr_ffn.cuh"
#include "rr_vec.cuh"

namespace rr {

namespace {

using bf16 = __nv_bfloat16;
using namespace tc;

struct NormArgs {
    int M, N;
    int group;       // threads of a row, a power of two
    int layer;       // mean taken off
    int ahead;       // backward: buffers for rows in shared memory: 2, the next row comes while one is worked on; 1, then; 0, straight from global memory
    float eps, inv_n;
    long long stride;                                   // rows from one set of a block to its next,
    long long sx, sr, sh, sy, sdy, sdh, sdx;            // and as many pitches
    long long ldx, ldr, ldh, ldy, lddy, lddh, lddx;
    const void *x, *residual, *dy, *dh, *w, *b;
    void *h, *y, *dx;  // (backward: h is read only)
    int w_f32;
    float *mean, *rstd;
    float *dw, *db;  // final place (one block), or the parts [blocks][N] in the workspace
    int add;         // dw, db: add to what is there
};

// A row is shared out over `group` threads (G of them; 0: fewer than 32, told at run time).  Thread t holds kSlots times eight columns: those
// of slot s are first_column + 8 group s on, the eight of them as Layout says with steps of step_of.
template <Layout L>
__device__ __forceinline__ int first_column(int t) { return L == kEights ? t * 8 : L == kQuads ? t * 4 : t; }
template <Layout L>
__device__ __forceinline__ int step_of(int group) { return L == kQuads ? 4 * group : group; }
// values behind the row set to zero
template <Layout L>
__device__ __forceinline__ void cut(f32x2 (&v)[4], int step, int left)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (L == kOne) {
            float x, y;
            unpack2(v[j], x, y);
            v[j] = pack2(2 * j * step < left ? x : 0.f, (2 * j + 1) * step < left ? y : 0.f);
        } else if ((L == kQuads && j >= 2 ? step : 0) >= left) {
            v[j] = pack2(0.f, 0.f);
        }
    }
}

// ---- rows on their way into shared memory -----------------------------------------------------------------------
// kEights, kQuads: a thread copies its own pieces ahead of their use and reads back nothing but what it copied, so all it needs is its own
// wait.  kOne: the threads of a row copy it in 16-byte pieces from the boundary before its start on, wherever that lies; a barrier later they read
// elements.  Nothing behind the end of a row is read.
__host__ __device__ constexpr int row_bytes(int size, int N) { return (N * size + 15) / 16 * 16 + 16; }
__host__ __device__ constexpr int tensor_bytes(Layout L, int size, int slots, int threads, int rows, int N)
{
    return L == kOne ? rows * row_bytes(size, N) : slots * 8 * size * threads;
}
__device__ __forceinline__ void copy16(uint32_t to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_some(uint32_t to, const void *from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t to, const void *from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
// `own`: the thread's first column in the row; `to`: its tensor's place in shared memory
template <class T, Layout L, int kSlots, int kThreads>
__device__ __forceinline__ void copy_row(uint32_t to, const T *own, int t, int group, int N)
{
    if constexpr (L == kOne) {
        const T *row = own - t;
        const uint32_t dst = to + threadIdx.x / group * row_bytes(sizeof(T), N);
        const int lead = (int)(reinterpret_cast<uintptr_t>(row) & 15), bytes = lead + N * (int)sizeof(T);
        const char *src = reinterpret_cast<const char *>(row) - lead;
        for (int g = t * 16; g < bytes; g += group * 16) copy_some(dst + g, src + g, min(16, bytes - g));
    } else {
        const int left = N - first_column<L>(t);
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            if constexpr (L == kEights) {
                if (s * 8 * group < left) copy16(to + (s * kThreads + threadIdx.x) * 16, own + s * 8 * group);
            } else {
                constexpr int kPiece = 4 * sizeof(T);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const uint32_t dst = to + ((2 * s + q) * kThreads + threadIdx.x) * kPiece;
                    const T *src = own + s * 8 * group + q * 4 * group;
                    if (s * 8 * group + q * 4 * group >= left) continue;
                    if constexpr (kPiece == 16) copy16(dst, src);
                    else copy8(dst, src);
                }
            }
        }
    }
}
// slot s of the thread out of a copied row (`own`: where it lies in global memory, which says where it lies in its buffer)
template <class T, Layout L, int kThreads>
__device__ __forceinline__ void take(const char *from, const T *own, int s, int t, int group, int N, Eight<T, L> &e)
{
    if constexpr (L == kOne) {
        const int left = N - t - s * 8 * group;
        const T *p = reinterpret_cast<const T *>(from + threadIdx.x / group * row_bytes(sizeof(T), N) + (reinterpret_cast<uintptr_t>(own - t) & 15)) + t + s * 8 * group;
#pragma unroll
        for (int j = 0; j < 8; ++j) e.e[j] = j * group < left ? p[j * group] : from_f32<T>(0.f);
    } else if constexpr (L == kEights) {
        e.q[0] = *reinterpret_cast<const uint4 *>(from + (s * kThreads + threadIdx.x) * 16);
    } else {
        using Quad = typename Eight<T, L>::Quad;
        const Quad *p = reinterpret_cast<const Quad *>(from) + 2 * s * kThreads + threadIdx.x;
        e.a = p[0];
        e.b = Quad{};
        if (s * 8 * group + 4 * group < N - 4 * t) e.b = p[kThreads];
    }
}
__device__ __forceinline__ void copies_asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kOpen>
__device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(kOpen) : "memory"); }
// the threads of a row meet
template <int G>
__device__ __forceinline__ void row_barrier()
{
    if constexpr (G <= 32) __syncwarp();
    else __syncthreads();
}

__device__ __forceinline__ float both(f32x2 v)
{
    float a, b;
    unpack2(v, a, b);
    return a + b;
}

// Sums of one or two values over the threads of a row, the same in each of them, in a fixed order.  `turn` alternates between calls (a
// buffer is written again only behind the barrier of the call between).
template <int G, bool kTwo>
__device__ __forceinline__ void row_sums(float &a, float &b, int group, float2 (*buf)[32], int &turn)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if ((G ? G : group) <= o) continue;
        a += __shfl_xor_sync(0xffffffffu, a, o);
        if (kTwo) b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if constexpr (G > 32) {
        constexpr int kPerRow = G / 32;
        const int warp = threadIdx.x >> 5;
        if ((threadIdx.x & 31) == 0) buf[turn][warp] = make_float2(a, b);
        __syncthreads();
        const float2 *mine = &buf[turn][warp & ~(kPerRow - 1)];
        a = mine[0].x;
        b = mine[0].y;
#pragma unroll
        for (int q = 1; q < kPerRow; ++q) {
            a += mine[q].x;
            if (kTwo) b += mine[q].y;
        }
        turn ^= 1;
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------
// Threads of a row (a power of two) that hold `slots` eights of columns each, threads of a block (`least` or more) and rows of it side by side.
struct NormLayout {
    int group, threads, slots, rows;
};
inline NormLayout norm_layout(int N, int slots, int least)
{
    const int eights = (N + 7) / 8;
    NormLayout l;
    l.slots = slots;
    l.group = 1;
    while (l.group * l.slots < eights) l.group <<= 1;
    l.threads = l.group > least ? l.group : least;
    l.rows = l.threads / l.group;
    return l;
}
// how rows are read: `pitch % 4`, `% 8` of every matrix in the call
struct Access {
    bool all_bf16 = true, quads, eights;
    explicit Access(int N) : quads(N % 4 == 0), eights(N % 8 == 0) {}
    void matrix(const void *p, int dtype, long long pitch)
    {
        if (!p) return;
        all_bf16 = all_bf16 && dtype == RR_BF16;
        quads = quads && pitch % 4 == 0;
        eights = eights && pitch % 8 == 0;
    }
    Layout layout() const { return all_bf16 && eights ? kEights : quads ? kQuads : kOne; }
};

// calls f(layout, slots, threads, group) with its arguments as compile-time constants
template <Layout L, int kSlots, int kThreads, int G, class F>
cudaError_t call(F f)
{
    return f(std::integral_constant<Layout, L>{}, std::integral_constant<int, kSlots>{}, std::integral_constant<int, kThreads>{}, std::integral_constant<int, G>{});
}
template <class T>
struct Type {
    using type = T;
};
template <class F>
cudaError_t with_type(int dtype, F f) { return dtype == RR_F32 ? f(Type<float>{}) : f(Type<bf16>{}); }

constexpr int kMostShared = SharedAllowance::kMost;

inline NormArgs norm_args(const rr_norm_shape &s, const NormLayout &l, int blocks)
{
    NormArgs a = {};
    a.M = s.M;
    a.N = s.N;
    a.group = l.group;
    a.layer = s.kind == RR_NORM_LAYER;
    a.eps = s.eps;
    a.inv_n = 1.0f / (float)s.N;
    a.stride = (long long)blocks * l.rows;
    a.sx = a.stride * (a.ldx = s.ldx);
    a.sr = a.stride * (a.ldr = s.ldr);
    a.sh = a.stride * (a.ldh = s.ldh);
    a.sy = a.stride * (a.ldy = s.ldy);
    a.sdy = a.stride * (a.lddy = s.lddy);
    a.sdh = a.stride * (a.lddh = s.lddh);
    a.sdx = a.stride * (a.lddx = s.lddx);
    a.w_f32 = s.w_dtype == RR_F32;
    return a;
}

}  // namespace

}  // namespace rr
