// Clipping by the global norm of many gradients:
//     norm = sqrt(sum of the squares of all elements of all tensors),  f = min(1, bound / (norm + 1e-6)),  dst = f src
// in place or into other buffers.  The tensors are cut into chunks of equal length; a first kernel adds up squares, a second takes the
// factor from the blocks' sums and scales (its blocks find their tensor before the sums are there).  The factor needs every element, so gradients
// that exceed the L2 cache are read twice; the second kernel goes backwards, so that what was read last is found in the cache.  In place
// with f = 1 nothing is written.  Squares are added in fp32 eight at a time and these sums in 64 bits in a fixed order, so that neither the
// length nor the order costs anything; eights whose squares leave the range of fp32 are squared in 64 bits, so finite gradients never
// overflow or vanish.
// Measured: 0.59 G fp32 (one layer of 64 experts, its block and its table) into other buffers 1071 us, 6.6 TB/s over the two reads and the write;
// 0.18 G fp32 357 us, with no common 16-byte boundary 356 (an element at a time and one load after the other 2340); the norm alone 6.5 TB/s from
// 0.18 G on (bf16 5.6), and in tensors of about a million elements each, where every chunk of a block lies in another one and has to be looked up, 5.4 to 5.7
// (bf16 3.6 to 4.0: 576 tensors, 0.82 G, 609 and 458 us); 0.5 M in 12 tensors 5.4 us (the latencies of two kernels that depend on each other; with the factor made by the last block of
// the first kernel 6.9).
#include "rr_ffn.cuh"
#include "rr_vec.cuh"

namespace rr {

namespace {

using bf16 = __nv_bfloat16;

constexpr int kClipThreads = 256;
constexpr int kClipBlocks = 4;       // an SM, all resident at once (64 registers a thread)
constexpr int kClipMost = 2048;      // parts in the workspace
constexpr int kClipUnroll = 4;

struct GradEntry {
    const void *src;
    void *dst;           // null: only in the norm
    long long n;
    long long first;     // its first chunk; the entry behind the last tensor holds the number of chunks
    int src_f32, dst_f32;
    int head;            // elements up to the first that both src and dst hold at a 16-byte boundary; -1: there is none
    int src_head;        // the same for the squares, which read src alone: head, or where there is none up to src's first
};

constexpr int kPlanEntries = 64;     // written by one launch (3 KB of parameters)
struct PlanPiece {
    GradEntry e[kPlanEntries];
};
__global__ void k_grad_plan(const __grid_constant__ PlanPiece piece, int count, GradEntry *plan)
{
    if ((int)threadIdx.x < count) plan[threadIdx.x] = piece.e[threadIdx.x];
}

__device__ __forceinline__ GradEntry entry(const GradEntry *plan, int i)
{
    GradEntry e;
    const longlong2 *p = reinterpret_cast<const longlong2 *>(plan + i);
    longlong2 *q = reinterpret_cast<longlong2 *>(&e);
#pragma unroll
    for (int j = 0; j < (int)sizeof(GradEntry) / 16; ++j) q[j] = p[j];
    return e;
}
static_assert(sizeof(GradEntry) == 48, "read in pieces of 16 bytes");

// Block b takes the chunks b, b + gridDim, ... (all blocks sweep the memory together).  The tensor of a chunk is looked up by the whole
// block at once: one round of loads for up to 256 tensors, two for 65536.
struct Place {
    GradEntry e;
    long long end;  // first chunk behind the tensor
};
__device__ __forceinline__ void seek(Place &p, const GradEntry *plan, int tensors, long long chunk)
{
    int lo = 0, len = tensors;  // the last tensor whose first chunk is not behind this one (those without a chunk lie before one with)
    while (len > 1) {
        const int stride = (len + kClipThreads - 1) / kClipThreads, at = (int)threadIdx.x * stride;
        const int count = __syncthreads_count(at < len && plan[lo + at].first <= chunk) - 1;  // (the first of the range always is)
        lo += count * stride;
        len = min(stride, len - count * stride);
    }
    p.e = entry(plan, lo);
    p.end = plan[lo + 1].first;
}

// Range of chunk `c` of a tensor: elements [lo, hi), of which [body, body + 8 eights) lie at 16-byte boundaries.
struct Range {
    long long lo, hi, body;
    int eights;
};
__device__ __forceinline__ Range range_of(const GradEntry &e, int head, long long c, int chunk)
{
    Range r;
    if (head < 0) {
        r.lo = c * chunk;
        r.hi = min(e.n, r.lo + chunk);
        r.body = r.hi;
        r.eights = 0;
    } else {
        r.body = min(e.n, head + c * chunk);
        r.lo = c ? r.body : 0;
        r.hi = min(e.n, head + (c + 1) * chunk);
        r.eights = (int)((r.hi - r.body) >> 3);
    }
    return r;
}

// sum of the squares of kN values
template <int kN>
__device__ __forceinline__ double squares(const float (&v)[kN])
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < kN; ++j) s = fmaf(v[j], v[j], s);
    // in range: no overflow, and what an underflowing square loses is below 2^-126 / 2^-80 of the sum
    if (s >= 0x1p-80f && s <= 0x1p120f) return s;
    double d = 0;
#pragma unroll
    for (int j = 0; j < kN; ++j) d = fma((double)v[j], (double)v[j], d);
    return d;
}
__device__ __forceinline__ double block_sum(double v, double *buf)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int q = 0; q < kClipThreads / 32; ++q) v += buf[q];
    return v;
}

// f(k, element k) for every element of the range that the body leaves over, in front of it (all of a tensor without common boundaries: eight at
// a time) and behind it
template <class T, class F>
__device__ __forceinline__ void edges(const T *src, const Range &r, F f)
{
    long long k = r.lo + threadIdx.x;
    for (; k + 7 * kClipThreads < r.body; k += 8 * kClipThreads) {
        Unit<T, 1> e[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) e[u].template load<kKeep>(src + k + u * kClipThreads);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            float v[1];
            e[u].get(v);
            f(k + u * kClipThreads, v[0]);
        }
    }
    for (; k < r.body; k += kClipThreads) f(k, as_f32(src[k]));
    k = r.body + 8ll * r.eights + threadIdx.x;
    if (k < r.hi) f(k, as_f32(src[k]));
}

template <class T>
__device__ __forceinline__ double chunk_squares(const T *src, const Range &r)
{
    constexpr int kN = 16 / sizeof(T), kAtOnce = kClipUnroll * 8 / kN;  // 16 bytes, and how many of them a thread has in flight (a chunk has that many)
    const int units = r.eights * (8 / kN);
    const T *p = src + r.body;
    double sum = 0;
    int i = threadIdx.x;
    for (; i + (kAtOnce - 1) * kClipThreads < units; i += kAtOnce * kClipThreads) {
        Unit<T, kN> e[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) e[u].template load<kKeep>(p + (long long)(i + u * kClipThreads) * kN);
#pragma unroll
        for (int u = 0; u < kAtOnce; u += 8 / kN) {  // eight values at a time
            float v[8];
#pragma unroll
            for (int k = 0; k < 8 / kN; ++k) e[u + k].get(reinterpret_cast<float(&)[kN]>(v[k * kN]));
            sum += squares<8>(v);
        }
    }
    for (; i < units; i += kClipThreads) {
        Unit<T, kN> e;
        e.template load<kKeep>(p + (long long)i * kN);
        float v[kN];
        e.get(v);
        sum += squares<kN>(v);
    }
    edges(src, r, [&](long long, float x) {
        const double v = x;
        sum += v * v;
    });
    return sum;
}

// The next kernel may be made ready once this one has seen the plan, so that it can read it without waiting for the sums.
__global__ void __launch_bounds__(kClipThreads) k_grad_squares(const GradEntry *plan, int tensors, long long chunks, int chunk, double *part)
{
    __shared__ double buf[kClipThreads / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    double sum = 0;
    Place p;
    p.end = 0;
    for (long long c = blockIdx.x; c < chunks; c += gridDim.x) {
        if (c >= p.end) seek(p, plan, tensors, c);
        const Range r = range_of(p.e, p.e.src_head, c - p.e.first, chunk);
        sum += p.e.src_f32 ? chunk_squares(static_cast<const float *>(p.e.src), r) : chunk_squares(static_cast<const bf16 *>(p.e.src), r);
    }
    sum = block_sum(sum, buf);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

template <class TS, class TD>
__device__ __forceinline__ void chunk_scale(const TS *src, TD *dst, const Range &r, float f)
{
    constexpr int kN = sizeof(TS) + sizeof(TD) == 4 ? 8 : 4, kAtOnce = kClipUnroll * 8 / kN;
    const int units = r.eights * (8 / kN);
    const TS *p = src + r.body;
    TD *q = dst + r.body;
    int i = threadIdx.x;
    for (; i + (kAtOnce - 1) * kClipThreads < units; i += kAtOnce * kClipThreads) {
        Unit<TS, kN> e[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) e[u].template load<kStream>(p + (long long)(i + u * kClipThreads) * kN);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            Unit<TD, kN> o;
            scaled<kN>(e[u], o, f);
            o.template store<kStream>(q + (long long)(i + u * kClipThreads) * kN);
        }
    }
    for (; i < units; i += kClipThreads) {
        Unit<TS, kN> e;
        Unit<TD, kN> o;
        e.template load<kStream>(p + (long long)i * kN);
        scaled<kN>(e, o, f);
        o.template store<kStream>(q + (long long)i * kN);
    }
    edges(src, r, [&](long long k, float x) { dst[k] = from_f32<TD>(x * f); });
}

__global__ void __launch_bounds__(kClipThreads)
k_grad_scale(const GradEntry *plan, int tensors, long long chunks, int chunk, const double *part, int parts, float bound, float *norm, int *status)
{
    __shared__ double buf[kClipThreads / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    long long c = chunks > blockIdx.x ? blockIdx.x + (chunks - 1 - blockIdx.x) / gridDim.x * gridDim.x : -1;  // the last chunk of the block
    Place p;
    if (c >= 0) seek(p, plan, tensors, c);  // (the plan is older than the sums: see above)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double sum = 0;
    for (int i = threadIdx.x; i < parts; i += kClipThreads) sum += __ldcg(part + i);
    sum = block_sum(sum, buf);
    const double root = sqrt(sum);
    const bool finite = isfinite(sum);
    // (gradients that are not finite are left as they are)
    const float f = finite ? (float)fmin(1.0, (double)bound / (root + 1e-6)) : 1.0f;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        norm[0] = (float)root;
        norm[1] = f;
        if (!finite) latch_status(status, RR_ERR_NONFINITE);
    }
    for (; c >= 0; c -= gridDim.x) {
        if (c < p.e.first) seek(p, plan, tensors, c);
        const GradEntry &e = p.e;
        if (!e.dst || (e.dst == e.src && f == 1.0f)) continue;
        const Range r = range_of(e, e.head, c - e.first, chunk);
        if (e.src_f32) {
            if (e.dst_f32) chunk_scale(static_cast<const float *>(e.src), static_cast<float *>(e.dst), r, f);
            else chunk_scale(static_cast<const float *>(e.src), static_cast<bf16 *>(e.dst), r, f);
        } else {
            if (e.dst_f32) chunk_scale(static_cast<const bf16 *>(e.src), static_cast<float *>(e.dst), r, f);
            else chunk_scale(static_cast<const bf16 *>(e.src), static_cast<bf16 *>(e.dst), r, f);
        }
    }
}

int size_of(int dtype) { return dtype == RR_F32 ? 4 : 2; }

// elements up to the first at which both addresses (of elements of ss and ds bytes) are multiples of 16 bytes, -1 if there is none
int common_head(const void *src, int ss, const void *dst, int ds)
{
    const uintptr_t s = (uintptr_t)src, d = (uintptr_t)dst;
    for (int h = 0; h < 8; ++h)
        if ((s + (uintptr_t)h * ss) % 16 == 0 && (d + (uintptr_t)h * ds) % 16 == 0) return h;
    return -1;
}

}  // namespace

size_t grad_plan_size(int tensors) { return ((size_t)tensors + 1) * sizeof(GradEntry); }
size_t clip_workspace() { return kHeaderBytes + kClipMost * sizeof(double); }

rr_status launch_grad_plan(int tensors, const rr_grad *list, void *plan, rr_grad_set *set, cudaStream_t st)
{
    const int sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    // Chunks: 8192 elements, fewer where that would leave SMs without one.
    long long total = 0;
    for (int i = 0; i < tensors; ++i) total += list[i].n;
    int chunk = kClipThreads * 8 * kClipUnroll;
    while (chunk > kClipThreads * 8 && total / chunk < 4ll * sms) chunk >>= 1;
    long long first = 0;
    PlanPiece piece;
    GradEntry *out = static_cast<GradEntry *>(plan);
    for (int i = 0, k = 0; i <= tensors; ++i) {
        GradEntry &e = piece.e[k];
        e = GradEntry{};
        e.first = first;
        if (i < tensors) {
            const rr_grad &g = list[i];
            e.src = g.src;
            e.dst = g.dst;
            e.n = g.n;
            e.src_f32 = g.src_dtype == RR_F32;
            e.dst_f32 = g.dst_dtype == RR_F32;
            const int ss = size_of(g.src_dtype), src_head = common_head(g.src, ss, g.src, ss);
            e.head = g.dst ? common_head(g.src, ss, g.dst, size_of(g.dst_dtype)) : src_head;
            // (without a common one there is a chunk for every `chunk` elements from the first on, which reach as far from src's)
            e.src_head = e.head < 0 ? src_head : e.head;
            const long long body = e.head < 0 ? g.n : g.n > e.head ? g.n - e.head : 0;
            first += g.n == 0 ? 0 : body == 0 ? 1 : (body + chunk - 1) / chunk;
        }
        if (++k == kPlanEntries || i == tensors) {
            k_grad_plan<<<1, kPlanEntries, 0, st>>>(piece, k, out);
            if (cudaGetLastError() != cudaSuccess) return RR_ERR_CUDA;
            out += k;
            k = 0;
        }
    }
    set->plan = plan;
    set->tensors = tensors;
    set->chunk = chunk;
    set->chunks = first;
    return RR_OK;
}

rr_status launch_clip_grads(const rr_grad_set &set, float bound, float *norm, void *ws, cudaStream_t st)
{
    const int sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    const GradEntry *plan = static_cast<const GradEntry *>(set.plan);
    double *part = reinterpret_cast<double *>(static_cast<char *>(ws) + kHeaderBytes);
    long long most = (long long)sms * kClipBlocks;
    if (most > kClipMost) most = kClipMost;
    const int grid = set.chunks < 1 ? 1 : (int)(set.chunks < most ? set.chunks : most);
    cudaError_t err = launch_dependent(k_grad_squares, dim3(grid), kClipThreads, 0, 1, st, plan, (int)set.tensors, (long long)set.chunks, (int)set.chunk, part);
    // From 310 M elements on eight times the resident blocks scale: short ones drift apart, and reads and writes mix better (0.59 G fp32 1133 -> 1073 us).
    // Where f is 1 their starts cost 10 to 16 us, which fewer elements do not pay for.
    const int many = set.chunks >= 256ll * sms ? 32 * sms : grid;
    if (err == cudaSuccess)
        err = launch_dependent(k_grad_scale, dim3(many), kClipThreads, 0, 1, st, plan, (int)set.tensors, (long long)set.chunks, (int)set.chunk, (const double *)part,
                               grid, bound, norm, static_cast<int *>(ws));
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

}  // namespace rr
