// The norm in front of a branch, with the residual add of the branch before it, and its gradients.  Layer norm and RMS norm:
//     h = residual + x  (rounded to the stream's type),   mu = mean(h) (RMS: 0),   rstd = 1 / sqrt(mean((h - mu)^2) + eps)
//     y = (h - mu) rstd w + b
//     xh = (h - mu) rstd,  g = dy w:   dx = dh + rstd (g - [mean(g)] - xh mean(g xh)),   dw = sum over rows dy xh,   db = sum over rows dy
// (mean(g) for the layer norm only).  A row is read once and held in registers, so the variance is that of differences from the mean
// and not a difference of squares; both passes are bound by HBM, and by latency where rows are few.  Statistics and sums are fp32.
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
    int ahead;       // rows come through shared memory, the next set while the present one is worked on; else straight from global memory
    float eps, inv_n;
    long long ldx, ldr, ldh, ldy, lddy, lddh, lddx;
    const void *x, *residual, *dy, *dh, *w, *b;
    void *h, *y, *dx;  // (backward: h is read only)
    int w_f32;
    float *mean, *rstd;
    float *dw, *db;  // final place (one block), or the parts [blocks][N] in the workspace
    int add;         // dw, db: add to what is there
};

// Columns of slot s of a thread: first_column on, the eight of them as Layout says with steps of step_of.
template <Layout L>
__device__ __forceinline__ int first_column(int s, int t, int group)
{
    return L == kEights ? (s * group + t) * 8 : L == kQuads ? s * 8 * group + t * 4 : s * 8 * group + t;
}
template <Layout L>
__device__ __forceinline__ int step_of(int group) { return L == kQuads ? 4 * group : group; }
// values behind the row set to zero
template <Layout L>
__device__ __forceinline__ void cut(f32x2 (&v)[4], int at, int step, int N)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (L == kOne) {
            float x, y;
            unpack2(v[j], x, y);
            v[j] = pack2(at + 2 * j * step < N ? x : 0.f, at + (2 * j + 1) * step < N ? y : 0.f);
        } else if (at + (L == kQuads && j >= 2 ? step : 0) >= N) {
            v[j] = pack2(0.f, 0.f);
        }
    }
}

template <Layout L>
__device__ __forceinline__ void parameter(const void *p, int f32, int at, int step, int left, float none, f32x2 (&v)[4])
{
    if (!p) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = pack2(none, none);
    } else if (f32) {
        Eight<float, L> e;
        e.template load<kConst>(static_cast<const float *>(p) + at, step, left);
        e.get(v);
    } else {
        Eight<bf16, L> e;
        e.template load<kConst>(static_cast<const bf16 *>(p) + at, step, left);
        e.get(v);
    }
}

// ---- rows on their way into shared memory -----------------------------------------------------------------------
// kEights, kQuads: a thread copies its own pieces ahead of their use and reads back nothing but what it copied, so all it needs is its own
// wait.  kOne: the threads of a row copy it in 16-byte pieces from the boundary before its start on, wherever that lies; a barrier later they read
// elements.  Nothing behind the end of a row is read.
__host__ __device__ constexpr int tensor_bytes(Layout L, int size, int slots, int threads, int rows, int N)
{
    return L == kOne ? rows * ((N * size + 15) / 16 * 16 + 16) : slots * 8 * size * threads;
}
__device__ __forceinline__ void copy16(uint32_t to, const void *from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t to, const void *from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
template <class T, Layout L, int kSlots, int kThreads>
__device__ __forceinline__ void copy_row(char *to, const T *row, int t, int group, int N)
{
    if constexpr (L == kOne) {
        const uint32_t dst = smem_u32(to) + threadIdx.x / group * tensor_bytes(kOne, sizeof(T), 0, 0, 1, N);
        const int lead = (int)(reinterpret_cast<uintptr_t>(row) & 15), bytes = lead + N * (int)sizeof(T);
        const char *src = reinterpret_cast<const char *>(row) - lead;
        for (int g = t * 16; g < bytes; g += group * 16) copy16(dst + g, src + g, min(16, bytes - g));
    } else {
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = first_column<L>(s, t, group), step = step_of<L>(group);
            if (at >= N) break;
            if constexpr (L == kEights) {
                copy16(smem_u32(to) + (s * kThreads + threadIdx.x) * 16, row + at, 16);
            } else {
                constexpr int kPiece = 4 * sizeof(T);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if (at + q * step >= N) break;
                    const uint32_t dst = smem_u32(to) + ((2 * s + q) * kThreads + threadIdx.x) * kPiece;
                    if constexpr (kPiece == 16) copy16(dst, row + at + q * step, 16);
                    else copy8(dst, row + at + q * step);
                }
            }
        }
    }
}
// slot s of the thread out of a copied row (`row`: where it lies in global memory, which says where it lies in its buffer)
template <class T, Layout L, int kThreads>
__device__ __forceinline__ void take(const char *from, const T *row, int s, int t, int group, int N, Eight<T, L> &e)
{
    const int at = first_column<L>(s, t, group), step = step_of<L>(group);
    if constexpr (L == kOne) {
        const T *p = reinterpret_cast<const T *>(from + threadIdx.x / group * tensor_bytes(kOne, sizeof(T), 0, 0, 1, N) + (reinterpret_cast<uintptr_t>(row) & 15));
#pragma unroll
        for (int j = 0; j < 8; ++j) e.e[j] = at + j * step < N ? p[at + j * step] : from_f32<T>(0.f);
    } else if constexpr (L == kEights) {
        e.q[0] = *reinterpret_cast<const uint4 *>(from + (s * kThreads + threadIdx.x) * 16);
    } else {
        using Quad = typename Eight<T, L>::Quad;
        const Quad *p = reinterpret_cast<const Quad *>(from) + 2 * s * kThreads + threadIdx.x;
        e.a = p[0];
        e.b = Quad{};
        if (at + step < N) e.b = p[kThreads];
    }
}
__device__ __forceinline__ void copies_asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kOpen>
__device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(kOpen) : "memory"); }
// the threads of a row meet
__device__ __forceinline__ void row_barrier(int group)
{
    if (group <= 32) __syncwarp();
    else __syncthreads();
}

__device__ __forceinline__ float both(f32x2 v)
{
    float a, b;
    unpack2(v, a, b);
    return a + b;
}

// Sums of two values over the `group` threads of a row, the same in each of them, in a fixed order.  `turn` alternates between calls (a
// buffer is written again only behind the barrier of the call between).
__device__ __forceinline__ void row_sums(float &a, float &b, int group, float2 (*buf)[32], int &turn)
{
    const int in_warp = group < 32 ? group : 32;
    for (int o = in_warp >> 1; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if (group <= 32) return;
    const int warp = threadIdx.x >> 5, per_row = group >> 5;
    if ((threadIdx.x & 31) == 0) buf[turn][warp] = make_float2(a, b);
    __syncthreads();
    const float2 *mine = &buf[turn][warp & ~(per_row - 1)];
    a = b = 0.f;
    for (int q = 0; q < per_row; ++q) {
        a += mine[q].x;
        b += mine[q].y;
    }
    turn ^= 1;
}

// ---- host ---------------------------------------------------------------------------------------------------------
// Threads of a row (a power of two), eights of columns that a thread holds, threads of a block and rows of it side by side.
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

// calls f(layout, slots, threads) with its arguments as compile-time constants
template <Layout L, int kSlots, int kThreads, class F>
cudaError_t call(F f)
{
    return f(std::integral_constant<Layout, L>{}, std::integral_constant<int, kSlots>{}, std::integral_constant<int, kThreads>{});
}
template <class T>
struct Type {
    using type = T;
};
template <class F>
cudaError_t with_type(int dtype, F f) { return dtype == RR_F32 ? f(Type<float>{}) : f(Type<bf16>{}); }

constexpr int kMostShared = 226 << 10;  // for the rows (beside a little of the kernels' own)

// `smem` bytes of dynamic shared memory for a kernel
template <class K>
cudaError_t allow(K kernel, size_t smem)
{
    return smem <= 40 << 10 ? cudaSuccess : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
}

inline NormArgs norm_args(const rr_norm_shape &s, const NormLayout &l)
{
    NormArgs a = {};
    a.M = s.M;
    a.N = s.N;
    a.group = l.group;
    a.layer = s.kind == RR_NORM_LAYER;
    a.eps = s.eps;
    a.inv_n = 1.0f / (float)s.N;
    a.ldx = s.ldx;
    a.ldr = s.ldr;
    a.ldh = s.ldh;
    a.ldy = s.ldy;
    a.lddy = s.lddy;
    a.lddh = s.lddh;
    a.lddx = s.lddx;
    a.w_f32 = s.w_dtype == RR_F32;
    return a;
}

}  // namespace

}  // namespace rr
