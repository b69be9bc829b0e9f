// Balance loss over all k choices of a router, per segment of tokens, with a token mask; per-expert counts;
// the z-loss on the log of the softmax's denominator; and the gradient of both.  Segment s holds the tokens
// [s L, (s+1) L); n_s of them are live (mask non-zero), n is the sum of the n_s, S' the number of segments with
// a live token.
//     count_se = #{ (i, r) : i live in s, r < k, choice r of i is e },   f_se = count_se / (k n_s)
//     P_se     = (1/n_s) sum_{i live in s} g_ie,    g_i = softmax(a_i),   lse_i = log sum_e exp(a_ie)
//     L_b = alpha E / S' sum_s sum_e f_se P_se,     L_z = beta / n sum_{i live} lse_i^2
//     dL/da_ij = live_i g_ij ( alpha E / (S' n_s) (f_sj - sum_e f_se g_ie) + 2 beta / n lse_i )    (f constant)
// One read of the scores forward, one read and one write (or read-modify-write) backward: HBM at sizes above L2,
// launch latency below.  The row of a dead token is read and selected away (its load does not wait for the
// mask), so what it holds -- NaN, infinities -- reaches no sum.  All sums are fp32 in a fixed order (counts are
// integers), so the results repeat bit for bit.
// 65536 x 64, top-2, 32 padded segments: forward 10.9 us, gradient 8.6 (latency: a few dependent loads, the joining of the parts); 2^20
// tokens: 68 us, 4.2 TB/s read (loads in flight: registers hold two tokens a lane group) and 97 us, 5.5 TB/s.
#include <type_traits>

#include "rr_ffn.cuh"
#include "rr_rows.cuh"
#include "rr_tc.cuh"

namespace rr {

namespace {

constexpr int kBalThreads = 512;
constexpr int kBalWarps = kBalThreads / 32;
constexpr int kBalBlocks = 296;     // blocks wanted: two per SM, all resident at once
constexpr int kBalFinal = 1024;     // threads of the second forward kernel

// the columns of one row that a lane keeps; minus infinity past E and where there is no row.  kReadOnly: nothing in the launch
// writes to the scores (the gradient may be written over them, which loads past the coherent path would not be allowed to meet).
template <int GS, int CPL, bool VEC, bool kReadOnly>
__device__ __forceinline__ void load_row(const float *a, bool in, int E, int gl, float (&g)[CPL])
{
    auto get = [](const auto *p) { return kReadOnly ? __ldg(p) : *p; };
    if constexpr (VEC) {
#pragma unroll
        for (int q = 0; q < CPL / 4; ++q) {
            const int j = column_of<GS, true>(4 * q, gl);
            float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (in && j < E) v = get(reinterpret_cast<const float4 *>(a + j));
            g[4 * q] = v.x; g[4 * q + 1] = v.y; g[4 * q + 2] = v.z; g[4 * q + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const int j = column_of<GS, false>(c, gl);
            g[c] = (in && j < E) ? get(a + j) : -INFINITY;
        }
    }
}
// g becomes exp(a - m), m the row's maximum; returns log sum_e exp(a_e) and, in inv, the factor that makes g the softmax.  These
// kernels are bound by the instructions they issue, so: packed pairs of columns, the hardware's exponential, logarithm and reciprocal
// (relative errors of about 2^-22).  The maximum is taken off before anything is multiplied, so that a row whose scores are all the type's
// lowest value (a mask that leaves nothing) is a uniform one and not a difference of infinities.  The row of a dead token gives
// garbage that its group keeps to itself.
template <int GS, int CPL>
__device__ __forceinline__ float softmax_lse(float (&g)[CPL], float &inv)
{
    using namespace tc;
    float m = -INFINITY;
#pragma unroll
    for (int c = 0; c < CPL; ++c) m = fmaxf(m, g[c]);
    m = group_max<GS>(m);
    float z = 0.f;
    if constexpr (CPL % 2 == 0) {
        f32x2 sum = pack2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < CPL; c += 2) {
            unpack2(mul2(add2(pack2(g[c], g[c + 1]), pack2(-m, -m)), pack2(kLog2e, kLog2e)), g[c], g[c + 1]);
            g[c] = ex2(g[c]);  // (exp(-inf) = 0 for the columns past E)
            g[c + 1] = ex2(g[c + 1]);
            sum = add2(sum, pack2(g[c], g[c + 1]));
        }
        float a, b;
        unpack2(sum, a, b);
        z = a + b;
    } else {
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            g[c] = ex2((g[c] - m) * kLog2e);
            z += g[c];
        }
    }
    z = group_sum<GS>(z);
    inv = rcp(z);
    return fmaf(lg2(z), 0.693147180559945f, m);
}
// acc += inv * g
template <int CPL>
__device__ __forceinline__ void add_scaled(float (&acc)[CPL], const float (&g)[CPL], float inv)
{
    using namespace tc;
    if constexpr (CPL % 2 == 0) {
#pragma unroll
        for (int c = 0; c < CPL; c += 2)
            unpack2(fma2(pack2(g[c], g[c + 1]), pack2(inv, inv), pack2(acc[c], acc[c + 1])), acc[c], acc[c + 1]);
    } else {
#pragma unroll
        for (int c = 0; c < CPL; ++c) acc[c] = fmaf(g[c], inv, acc[c]);
    }
}

__device__ __forceinline__ bool is_live(const uint8_t *__restrict__ live, bool in, long long t)
{
    return in && (!live || __ldg(live + t) != 0);
}

struct BalShape {
    int E, k, stride;
    long long L;   // tokens of a segment
    int S;         // segments
    int cps;       // blocks per segment (forward)
    int slab;      // tokens of a block (forward)
    int one;       // the first forward kernel finishes the segments itself
};

struct BalScratch {
    Header *hdr;
    float *partial;  // [S*cps][E] softmax sums
    int *pcount;     // [S*cps][E] choices
    float *plse;     // [S*cps] sums of lse^2
    int *pn;         // [S*cps] live tokens
    float *dot;      // [S] sum_e f P of each segment
    float *slse;     // [S]
    int *sn;         // [S]
};

// sums over the warp, the same in every lane, and over the block (any number of warps up to 32), in a fixed order
template <class T>
__device__ __forceinline__ T warp_sum(T v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <class... T>
__device__ __forceinline__ void block_sums(uint32_t (*buf)[32], T &...v)
{
    const int lane = threadIdx.x & 31, warps = (int)(blockDim.x >> 5);
    int k = 0;
    auto store = [&](auto &x) {
        x = warp_sum(x);
        if (lane == 0) buf[k][threadIdx.x >> 5] = *reinterpret_cast<const uint32_t *>(&x);
        ++k;
    };
    __syncthreads();  // (buf may still be read from the call before)
    (store(v), ...);
    __syncthreads();
    k = 0;
    auto load = [&](auto &x) {
        const uint32_t u = lane < warps ? buf[k][lane] : 0u;  // (the bits of a zero of either type)
        x = warp_sum(*reinterpret_cast<const typename std::remove_reference<decltype(x)>::type *>(&u));
        ++k;
    };
    (load(v), ...);
}

// What the forward pass writes.
struct BalOut {
    float alpha, beta;
    float *loss, *P;
    int *count, *n_live;
};

// A sum of another block: past L1 when that block is of the same kernel (else its 32 warps share what the first of them fetched).
template <bool kFresh, class T>
__device__ __forceinline__ T other_block(const T *p)
{
    return kFresh ? __ldcg(p) : *p;
}

// Adds up the blocks of segment s; the caller that finishes last of the S adds up the segments.  NT threads.  Thread (r, j) takes the rows
// r, r + R, ... of column j (of the four columns from j on when VEC); the R sums of a column are then added in two steps.
template <bool VEC, int NT, bool kFresh>
__device__ __forceinline__ void finish_segment(const BalShape &b, const BalScratch &w, const BalOut &o, int s)
{
    constexpr int V = VEC ? 4 : 1, kParts = NT / kMaxE;
    __shared__ float sp[NT * V];
    __shared__ int sc[NT * V];
    __shared__ float tp[kParts][kMaxE];
    __shared__ int tc[kParts][kMaxE];
    __shared__ uint32_t buf[4][32];
    __shared__ int last;
    const int E = b.E, tid = threadIdx.x, lane = tid & 31;
    int epad = V;
    while (epad < E) epad <<= 1;
    const int cols = epad / V, R = NT / cols, r = tid / cols, j = (tid % cols) * V;
    const size_t row0 = (size_t)s * b.cps;
    float sum[V] = {}, lse2 = 0.f;
    int cnt[V] = {}, n = 0;
    for (int c = lane; c < b.cps; c += 32) { lse2 += other_block<kFresh>(w.plse + row0 + c); n += other_block<kFresh>(w.pn + row0 + c); }  // (every warp for itself: no barrier)
    if (j < E) {
#pragma unroll 4
        for (int c = r; c < b.cps; c += R) {
            if constexpr (VEC) {
                const float4 x = other_block<kFresh>(reinterpret_cast<const float4 *>(w.partial + (row0 + c) * E + j));
                const int4 y = other_block<kFresh>(reinterpret_cast<const int4 *>(w.pcount + (row0 + c) * E + j));
                sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
                cnt[0] += y.x; cnt[1] += y.y; cnt[2] += y.z; cnt[3] += y.w;
            } else {
                sum[0] += other_block<kFresh>(w.partial + (row0 + c) * E + j);
                cnt[0] += other_block<kFresh>(w.pcount + (row0 + c) * E + j);
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        sp[r * epad + j + v] = sum[v];
        sc[r * epad + j + v] = cnt[v];
    }
    n = warp_sum(n);
    lse2 = warp_sum(lse2);
    __syncthreads();
    {
        const int c = tid % kMaxE, part = tid / kMaxE, rows = min(R, b.cps);  // (the other rows are zero)
        float t = 0.f;
        int m = 0;
        if (c < E)
            for (int q = part; q < rows; q += kParts) { t += sp[q * epad + c]; m += sc[q * epad + c]; }
        tp[part][c] = t;
        tc[part][c] = m;
    }
    __syncthreads();
    float prod = 0.f;
    if (tid < E) {
        float tot = 0.f;
        int m = 0;
#pragma unroll
        for (int q = 0; q < kParts; ++q) { tot += tp[q][tid]; m += tc[q][tid]; }
        const float p = n > 0 ? tot / (float)n : 0.f;
        o.count[(size_t)s * E + tid] = m;
        o.P[(size_t)s * E + tid] = p;
        if (n > 0) prod = (float)m / ((float)b.k * (float)n) * p;
    }
    block_sums(buf, prod);
    float dots = 0.f, z = 0.f;
    int segs = 0, live = 0;
    if (b.S == 1) {
        if (tid) return;
        o.n_live[0] = n;
        dots = prod;
        z = lse2;
        segs = n > 0 ? 1 : 0;
        live = n;
    } else {
        if (tid == 0) {
            o.n_live[s] = n;
            w.dot[s] = prod;
            w.slse[s] = lse2;
            w.sn[s] = n;
            __threadfence();
            last = atomicAdd(&w.hdr->sync[8], 1) == b.S - 1;
        }
        __syncthreads();
        if (!last) return;
        __threadfence();
        for (int q = tid; q < b.S; q += NT) {
            dots += __ldcg(w.dot + q);
            z += __ldcg(w.slse + q);
            const int m = __ldcg(w.sn + q);
            live += m;
            segs += m > 0 ? 1 : 0;
        }
        block_sums(buf, dots, z, segs, live);
        if (tid) return;
        w.hdr->sync[8] = 0;
    }
    o.loss[0] = segs > 0 ? o.alpha * (float)E / (float)segs * dots : 0.f;
    o.loss[1] = live > 0 && o.beta != 0.f ? o.beta / (float)live * z : 0.f;  // (the sum may be infinite)
}

// Forward, second kernel: block s finishes segment s.
template <bool VEC>
__global__ void __launch_bounds__(kBalFinal) k_balance_final(const BalShape b, const BalScratch w, const BalOut o)
{
    dependent_start();  // (the first kernel has completed and its sums are visible)
    finish_segment<VEC, kBalFinal, false>(b, w, o, blockIdx.x);
}

// Forward, first kernel: block (s, c) adds up the tokens of its slab of segment s.  With kOne it is the only kernel: the block of a
// segment that ends last finishes it.
template <int GS, int CPL, bool VEC, bool kOne>
__global__ void __launch_bounds__(kBalThreads)
k_balance_partial(const BalShape b, const float *__restrict__ logits, const int32_t *__restrict__ topk,
                  const uint8_t *__restrict__ live, const BalScratch w, const BalOut o)
{
    constexpr int TPW = 32 / GS;
    __shared__ float red[kBalWarps][kMaxE];
    __shared__ int cnt[kMaxE];
    __shared__ float red_lse[kBalWarps];
    __shared__ int red_n[kBalWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, grp = lane / GS, gl = lane % GS, E = b.E;
    for (int j = threadIdx.x; j < E; j += kBalThreads) cnt[j] = 0;
    __syncthreads();
    dependent_start();
    const int s = blockIdx.x / b.cps, c0 = blockIdx.x - s * b.cps;
    const long long seg0 = s * b.L, t0 = seg0 + (long long)c0 * b.slab;
    const long long t1 = min(seg0 + b.L, t0 + b.slab);
    float acc[CPL] = {}, lse2 = 0.f;
    int n = 0;
    auto count_choice = [&](int e) {
        if (e >= 0 && e < E) atomicAdd(&cnt[e], 1);
        else latch_status(&w.hdr->status, RR_ERR_INVALID_ARG);
    };
    for (long long base = t0 + warp * TPW; base < t1; base += 2 * kBalWarps * TPW) {  // two tokens in flight per group
        const long long ta = base + grp, tb = ta + kBalWarps * TPW;
        const bool ina = ta < t1, inb = tb < t1;
        // rows, marks and choices are requested together, whatever the marks will say
        float ga[CPL], gb[CPL];
        load_row<GS, CPL, VEC, true>(logits + (ina ? ta : 0) * E, ina, E, gl, ga);
        load_row<GS, CPL, VEC, true>(logits + (inb ? tb : 0) * E, inb, E, gl, gb);
        const bool la = is_live(live, ina, ta), lb = is_live(live, inb, tb);
        const int ea = ina && gl < b.k ? __ldg(topk + ta * b.stride + gl) : 0, eb = inb && gl < b.k ? __ldg(topk + tb * b.stride + gl) : 0;
        if (la && gl < b.k) count_choice(ea);
        if (lb && gl < b.k) count_choice(eb);
        if (GS < kMaxK) {  // (a group smaller than k)
            for (int r = gl + GS; r < b.k; r += GS) {
                if (la) count_choice(__ldg(topk + ta * b.stride + r));
                if (lb) count_choice(__ldg(topk + tb * b.stride + r));
            }
        }
        float ia, ib;
        const float za = softmax_lse<GS, CPL>(ga, ia), zb = softmax_lse<GS, CPL>(gb, ib);
        if (la) {
            add_scaled<CPL>(acc, ga, ia);
            lse2 = fmaf(za, za, lse2);
        }
        if (lb) {
            add_scaled<CPL>(acc, gb, ib);
            lse2 = fmaf(zb, zb, lse2);
        }
        n += (la ? 1 : 0) + (lb ? 1 : 0);
    }
    // groups of the warp, then warps of the block, in a fixed order
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
#pragma unroll
        for (int o = GS; o < 32; o <<= 1) acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], o);
        const int j = column_of<GS, VEC>(c, gl);
        if (grp == 0 && j < E) red[warp][j] = acc[c];
    }
#pragma unroll
    for (int o = GS; o < 32; o <<= 1) {
        lse2 += __shfl_xor_sync(0xffffffffu, lse2, o);
        n += __shfl_xor_sync(0xffffffffu, n, o);
    }
    if (lane == 0) { red_lse[warp] = lse2; red_n[warp] = n; }
    __syncthreads();
    for (int j = threadIdx.x; j < E; j += kBalThreads) {
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < kBalWarps; ++q) sum += red[q][j];
        w.partial[(size_t)blockIdx.x * E + j] = sum;
        w.pcount[(size_t)blockIdx.x * E + j] = cnt[j];
    }
    if (threadIdx.x == 0) {
        float sum = 0.f;
        int m = 0;
        for (int q = 0; q < kBalWarps; ++q) { sum += red_lse[q]; m += red_n[q]; }
        w.plse[blockIdx.x] = sum;
        w.pn[blockIdx.x] = m;
    }
    if constexpr (kOne) {
        if (b.cps > 1) {
            __shared__ int last;
            __threadfence();  // (every thread's sums are visible before the block is counted)
            __syncthreads();
            if (threadIdx.x == 0) {
                last = atomicAdd(&w.hdr->segs[s], 1) == b.cps - 1;
                if (last) w.hdr->segs[s] = 0;
            }
            __syncthreads();
            if (!last) return;
            __threadfence();
        } else {
            __syncthreads();  // (its own sums)
        }
        finish_segment<VEC, kBalThreads, true>(b, w, o, s);
    }
}

// Backward: items of up to `slab` tokens of one segment, dealt to the blocks in turn.
template <int GS, int CPL, bool VEC>
__global__ void __launch_bounds__(kBalThreads)
k_balance_bwd(const BalShape b, const float *logits, const int *__restrict__ count, const int *__restrict__ n_live,
              const uint8_t *__restrict__ live, float coef_b, float coef_z, int accumulate, float *dlogits)
{
    constexpr int TPW = 32 / GS;
    __shared__ uint32_t buf[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, grp = lane / GS, gl = lane % GS, E = b.E;
    int segs = 0, tokens = 0;
    dependent_start();
    for (int q = threadIdx.x; q < b.S; q += kBalThreads) {
        const int m = __ldg(n_live + q);
        tokens += m;
        segs += m > 0 ? 1 : 0;
    }
    block_sums(buf, segs, tokens);
    const float cz = tokens > 0 ? coef_z / (float)tokens : 0.f;
    for (long long item = blockIdx.x; item < (long long)b.S * b.cps; item += gridDim.x) {
        const int s = (int)(item / b.cps);
        const long long seg0 = s * b.L, t0 = seg0 + (item - (long long)s * b.cps) * b.slab, t1 = min(seg0 + b.L, t0 + b.slab);
        const int ns = __ldg(n_live + s);
        const float inv = ns > 0 ? 1.0f / ((float)b.k * (float)ns) : 0.f;
        const float cb = ns > 0 ? coef_b / ((float)segs * (float)ns) : 0.f;
        float fj[CPL];
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const int j = column_of<GS, VEC>(c, gl);
            fj[c] = j < E ? (float)__ldg(count + (size_t)s * E + j) * inv : 0.f;
        }
        for (long long base = t0 + warp * TPW; base < t1; base += kBalWarps * TPW) {
            const long long t = base + grp;
            const bool in = t < t1;
            float g[CPL];
            load_row<GS, CPL, VEC, false>(logits + (in ? t : 0) * E, in, E, gl, g);
            const bool l = is_live(live, in, t);
            float inv, dot = 0.f;
            const float lse = softmax_lse<GS, CPL>(g, inv);
#pragma unroll
            for (int c = 0; c < CPL; ++c) dot = fmaf(fj[c], g[c], dot);
            dot = group_sum<GS>(dot) * inv;
            if (!in || (!l && accumulate)) continue;
            float *o = dlogits + t * E;
            const float zz = cz * lse;
#pragma unroll
            for (int c = 0; c < CPL; ++c) g[c] = l ? g[c] * inv * fmaf(cb, fj[c] - dot, zz) : 0.f;
            if constexpr (VEC) {
#pragma unroll
                for (int q = 0; q < CPL / 4; ++q) {
                    const int j = column_of<GS, true>(4 * q, gl);
                    if (j >= E) continue;
                    float4 *dst = reinterpret_cast<float4 *>(o + j);
                    float4 v = make_float4(g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]);
                    if (accumulate) {
                        const float4 old = *dst;
                        v = make_float4(__fadd_rn(old.x, v.x), __fadd_rn(old.y, v.y), __fadd_rn(old.z, v.z), __fadd_rn(old.w, v.w));
                    }
                    *dst = v;
                }
            } else {
#pragma unroll
                for (int c = 0; c < CPL; ++c) {
                    const int j = column_of<GS, false>(c, gl);
                    if (j < E) o[j] = accumulate ? __fadd_rn(o[j], g[c]) : g[c];
                }
            }
        }
    }
}

// Blocks per segment and tokens per block, for about `want` blocks in all and no fewer than `pass` tokens in one.
BalShape balance_shape(int T, int E, int k, int stride, int S, int want, int pass)
{
    BalShape b;
    b.E = E;
    b.k = k;
    b.stride = stride;
    b.S = S;
    b.L = T / S;
    long long cps = want / S, most = (b.L + pass - 1) / pass;
    if (cps > most) cps = most;
    if (cps < 1) cps = 1;
    b.slab = (int)((b.L + cps - 1) / cps);
    if (b.slab < 1) b.slab = 1;
    b.cps = (int)((b.L + b.slab - 1) / b.slab);
    if (b.cps < 1) b.cps = 1;
    // One launch where the header has a counter for every segment (32 words were spare) and a block adds up a segment's parts in about the
    // time that the second kernel takes to start.  The device takes as long, the caller 2 us less (with a mask, E = 64; in brackets with two launches:
    // four segments of 16 tokens 6.2 us [7.8], 32 of 256 8.4 [8.9], 32 of 2048 11.0 [11.3], 4 of 4096 in 32 parts each 9.5 [9.3]).  A segment in
    // more parts keeps the second kernel, whose blocks are twice as large (one of 16384 in 128 parts: 8.5 [7.6]).
    b.one = S <= 32 && b.cps <= 32;
    return b;
}
BalShape forward_shape(int T, int E, int k, int stride, int S)
{
    return balance_shape(T, E, k, stride, S, kBalBlocks, 2 * kBalWarps * (32 / layout_of(E).gs));
}

size_t balance_layout(void *ws, int T, int E, int S, BalScratch *out)
{
    const BalShape b = forward_shape(T, E, 1, 1, S);
    const size_t rows = (size_t)b.S * b.cps;
    Carver c(ws);
    BalScratch w;
    w.hdr = c.take<Header>(1);
    w.partial = c.take<float>(rows * E);
    w.pcount = c.take<int>(rows * E);
    w.plse = c.take<float>(rows);
    w.pn = c.take<int>(rows);
    w.dot = c.take<float>(S);
    w.slse = c.take<float>(S);
    w.sn = c.take<int>(S);
    if (out) *out = w;
    return align_up(c.off, 256);
}

template <int GS, int CPL, bool VEC>
rr_status run_fwd(const BalShape &b, const float *logits, const int32_t *topk, const uint8_t *live, const BalScratch &w,
                  const BalOut &o, cudaStream_t st)
{
    return launch_dependent(b.one ? k_balance_partial<GS, CPL, VEC, true> : k_balance_partial<GS, CPL, VEC, false>, dim3((unsigned)(b.S * b.cps)), kBalThreads, 0, 1, st, b, logits, topk, live, w,
                            o) == cudaSuccess
               ? RR_OK : RR_ERR_CUDA;
}

template <int GS, int CPL, bool VEC>
rr_status run_bwd(const BalShape &b, const float *logits, const int *count, const int *n, const uint8_t *live, float coef_b,
                  float coef_z, int accumulate, float *dlogits, cudaStream_t st)
{
    const long long items = (long long)b.S * b.cps;
    const int grid = (int)(items < kBalBlocks ? items : kBalBlocks);
    return launch_dependent(k_balance_bwd<GS, CPL, VEC>, dim3(grid), kBalThreads, 0, 1, st, b, logits, count, n, live, coef_b, coef_z, accumulate,
                            dlogits) == cudaSuccess
               ? RR_OK : RR_ERR_CUDA;
}

}  // namespace

size_t balance_workspace(int T, int E, int S) { return balance_layout(nullptr, T, E, S, nullptr); }

rr_status launch_balance_fwd(int T, int E, int k, int stride, int S, const float *logits, const int32_t *topk,
                             const uint8_t *live, float alpha, float beta, float *loss, int32_t *count, int32_t *n_live, float *P,
                             void *workspace, cudaStream_t st)
{
    const BalShape b = forward_shape(T, E, k, stride, S);
    BalScratch w;
    balance_layout(workspace, T, E, S, &w);
    rr_status rc = RR_OK;
    const BalOut o = {alpha, beta, loss, P, count, n_live};
    RR_ROWS_DISPATCH(rc = run_fwd, E, b, logits, topk, live, w, o, st);
    if (rc || b.one) return rc;
    const cudaError_t err = launch_dependent(E % 4 == 0 ? k_balance_final<true> : k_balance_final<false>, dim3(S), kBalFinal, 0, 1, st, b, w, o);
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

rr_status launch_balance_bwd(int T, int E, int k, int S, const float *logits, const int32_t *count, const int32_t *n_live,
                             const uint8_t *live, float coef_b, float coef_z, int accumulate, float *dlogits, cudaStream_t st)
{
    // (with few segments one item per block; with many, smaller items even out their lengths)
    const BalShape b = balance_shape(T, E, k, 1, S, (S > kBalBlocks / 4 ? 4 : 1) * kBalBlocks, kBalWarps * (32 / layout_of(E).gs));
    rr_status rc = RR_OK;
    RR_ROWS_DISPATCH(rc = run_bwd, E, b, logits, count, n_live, live, coef_b, coef_z, accumulate, dlogits, st);
    return rc;
}

}  // namespace rr
