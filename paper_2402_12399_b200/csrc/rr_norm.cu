// The norm in front of a branch, with the residual add of the branch before it, and its gradients.  Layer norm and RMS norm:
//     h = residual + x  (rounded to the stream's type),   mu = mean(h) (RMS: 0),   rstd = 1 / sqrt(mean((h - mu)^2) + eps)
//     y = (h - mu) rstd w + b
//     xh = (h - mu) rstd,  g = dy w:   dx = dh + rstd (g - [mean(g)] - xh mean(g xh)),   dw = sum over rows dy xh,   db = sum over rows dy
// (mean(g) for the layer norm only).  A row is read once and held in registers, so the variance is that of differences from the mean
// and not a difference of squares; both passes are bound by HBM, and by latency where rows are few.  Statistics and sums are fp32.
#include <type_traits>

#include "rr_ffn.cuh"
#include "rr_vec.cuh"

namespace rr {

namespace {

using bf16 = __nv_bfloat16;

constexpr int kNormThreads = 256;  // of a block, unless a row takes more

struct NormArgs {
    int M, N;
    int group;       // threads of a row, a power of two
    int layer;       // mean taken off
    float eps, inv_n;
    long long ldx, ldr, ldh, ldy, lddy, lddh, lddx;
    const void *x, *residual, *dy, *dh, *w, *b;
    void *h, *y, *dx;  // (backward: h is read only)
    int w_f32;
    float *mean, *rstd;
    float *dw, *db;  // final place (one block), or the parts [blocks][N] in the workspace
    int add;         // dw, db: add to what is there
};

// columns of slot v of a thread: eight from `at` on, `step` apart
template <bool kVec>
__device__ __forceinline__ int first_column(int v, int t, int group) { return kVec ? (v * group + t) * 8 : v * 8 * group + t; }

template <bool kVec>
__device__ __forceinline__ void parameter(const void *p, int f32, int at, int step, int left, float none, float (&v)[8])
{
    if (!p) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = none;
    } else if (f32) {
        Eight<float, kVec> e;
        e.template load<kConst>(static_cast<const float *>(p) + at, step, left);
        e.get(v);
    } else {
        Eight<bf16, kVec> e;
        e.template load<kConst>(static_cast<const bf16 *>(p) + at, step, left);
        e.get(v);
    }
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

// TH: type of the residual stream, void without one
template <class TX, class TH, class TY, int kSlots, int kThreads, bool kVec>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) k_norm_fwd(const NormArgs a)
{
    constexpr bool kRes = !__is_same(TH, void);
    using TR = std::conditional_t<kRes, TH, float>;
    __shared__ float2 buf[2][32];
    dependent_start();
    const int t = threadIdx.x & (a.group - 1), step = kVec ? 1 : a.group, rows = blockDim.x / a.group;
    int turn = 0;
    for (long long first = (long long)blockIdx.x * rows; first < a.M; first += (long long)gridDim.x * rows) {
        const long long row = first + threadIdx.x / a.group;
        const bool in = row < a.M;
        float v[kSlots][8];
        {
            Eight<TX, kVec> ex[kSlots];
            Eight<TR, kVec> er[kSlots];
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                const int at = first_column<kVec>(s, t, a.group);
                if (in && at < a.N) {
                    ex[s].load(static_cast<const TX *>(a.x) + row * a.ldx + at, step, a.N - at);
                    if (kRes) er[s].load(static_cast<const TR *>(a.residual) + row * a.ldr + at, step, a.N - at);
                } else {
                    ex[s].zero();
                    if (kRes) er[s].zero();
                }
            }
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                ex[s].get(v[s]);
                if constexpr (kRes) {
                    float r[8];
                    er[s].get(r);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[s][j] += r[j];
                    er[s].set(v[s]);
                    er[s].get(v[s]);  // the norm is that of the stream as it is stored
                    const int at = first_column<kVec>(s, t, a.group);
                    if (a.h && in && at < a.N) er[s].store(static_cast<TR *>(a.h) + row * a.ldh + at, step, a.N - at);
                }
            }
        }
        float m = 0.f, none = 0.f;
        if (a.layer) {
#pragma unroll
            for (int s = 0; s < kSlots; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) m += v[s][j];
            row_sums(m, none, a.group, buf, turn);
            m *= a.inv_n;
        }
        float d1 = 0.f, d2 = 0.f;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = first_column<kVec>(s, t, a.group);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[s][j] = (kVec ? at : at + j * step) < a.N ? v[s][j] - m : 0.f;
                d1 += v[s][j];
                d2 = fmaf(v[s][j], v[s][j], d2);
            }
        }
        row_sums(d1, d2, a.group, buf, turn);
        // what rounding left of the mean is in d1 (a row far from zero against its spread)
        const float rest = a.layer ? d1 * a.inv_n : 0.f;
        const float rstd = __frsqrt_rn(fmaxf(fmaf(d2, a.inv_n, -rest * rest), 0.f) + a.eps);
        if (t == 0 && in) {
            if (a.mean) a.mean[row] = m + rest;
            if (a.rstd) a.rstd[row] = rstd;
        }
        if (!in) continue;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = first_column<kVec>(s, t, a.group);
            if (at >= a.N) continue;
            float w[8], b[8];
            parameter<kVec>(a.w, a.w_f32, at, step, a.N - at, 1.f, w);
            parameter<kVec>(a.b, a.w_f32, at, step, a.N - at, 0.f, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[s][j] = fmaf((v[s][j] - rest) * rstd, w[j], b[j]);
            Eight<TY, kVec> e;
            e.set(v[s]);
            e.store(static_cast<TY *>(a.y) + row * a.ldy + at, step, a.N - at);
        }
    }
}

// Backward.  A block takes every gridDim-th set of rows and keeps the sums of its columns over them in registers; the next rows are
// requested while the present ones are worked on (blocks of 1024 have no registers for that).  A row is kept as it lies in memory and
// turned into numbers twice, for the sums and for dx: cheaper than the registers.  TD: type of dx and dh.
template <class TY, class TH, class TD, int kSlots, int kThreads, bool kVec>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? 2 : 1) k_norm_bwd(const NormArgs a)
{
    constexpr bool kAhead = kThreads < 1024;
    extern __shared__ float sums[];  // [2][N] where a block has several rows side by side
    __shared__ float2 buf[2][32];
    dependent_start();
    const int t = threadIdx.x & (a.group - 1), step = kVec ? 1 : a.group, rows = blockDim.x / a.group, mine = threadIdx.x / a.group;
    int turn = 0;
    float aw[kSlots][8] = {}, ab[kSlots][8] = {};
    struct Row {
        Eight<TY, kVec> y[kSlots];
        Eight<TH, kVec> h[kSlots];
        Eight<TD, kVec> d[kSlots];
        float mean, rstd;
    };
    auto request = [&](long long row, Row &r) {
        const bool in = row < a.M;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = first_column<kVec>(s, t, a.group);
            if (in && at < a.N) {
                r.y[s].load(static_cast<const TY *>(a.dy) + row * a.lddy + at, step, a.N - at);
                r.h[s].load(static_cast<const TH *>(a.h) + row * a.ldh + at, step, a.N - at);
                if (a.dh) r.d[s].load(static_cast<const TD *>(a.dh) + row * a.lddh + at, step, a.N - at);
                else r.d[s].zero();
            } else {
                r.y[s].zero();
                r.h[s].zero();
                r.d[s].zero();
            }
        }
        r.mean = in && a.mean ? __ldg(a.mean + row) : 0.f;
        r.rstd = in ? __ldg(a.rstd + row) : 0.f;
    };
    const long long stride = (long long)gridDim.x * rows;
    long long first = (long long)blockIdx.x * rows;
    Row ahead;
    if (kAhead && first < a.M) request(first + mine, ahead);
    for (; first < a.M; first += stride) {
        const long long row = first + mine;
        if (!kAhead) request(row, ahead);
        const Row r = ahead;
        if (kAhead && first + stride < a.M) request(row + stride, ahead);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = first_column<kVec>(s, t, a.group);
            if (at >= a.N) continue;
            float w[8], g[8], xh[8];
            parameter<kVec>(a.w, a.w_f32, at, step, a.N - at, 1.f, w);
            r.y[s].get(g);
            r.h[s].get(xh);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                xh[j] = (xh[j] - r.mean) * r.rstd;
                aw[s][j] = fmaf(g[j], xh[j], aw[s][j]);
                ab[s][j] += g[j];
                g[j] *= w[j];
                s1 += g[j];
                s2 = fmaf(g[j], xh[j], s2);
            }
        }
        if (!a.dx) continue;  // (not wanted)
        row_sums(s1, s2, a.group, buf, turn);
        s1 = a.layer ? s1 * a.inv_n : 0.f;
        s2 *= a.inv_n;
        if (row >= a.M) continue;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = first_column<kVec>(s, t, a.group);
            if (at >= a.N) continue;
            float w[8], g[8], xh[8], o[8];
            parameter<kVec>(a.w, a.w_f32, at, step, a.N - at, 1.f, w);
            r.y[s].get(g);
            r.h[s].get(xh);
            r.d[s].get(o);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                xh[j] = (xh[j] - r.mean) * r.rstd;
                o[j] = fmaf(r.rstd, fmaf(-xh[j], s2, fmaf(g[j], w[j], -s1)), o[j]);
            }
            Eight<TD, kVec> e;
            e.set(o);
            e.store(static_cast<TD *>(a.dx) + row * a.lddx + at, step, a.N - at);
        }
    }
    if (!a.dw && !a.db) return;
    // the rows of the block side by side, one after the other
    if (rows > 1) {
        for (int q = rows - 1; q >= 0; --q) {
            __syncthreads();
            if (mine != q) continue;
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                const int at = first_column<kVec>(s, t, a.group);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = at + j * step;
                    if (c >= a.N) continue;
                    if (q < rows - 1) {
                        aw[s][j] += sums[c];
                        ab[s][j] += sums[a.N + c];
                    }
                    if (q > 0) {
                        sums[c] = aw[s][j];
                        sums[a.N + c] = ab[s][j];
                    }
                }
            }
        }
        if (mine) return;
    }
    const size_t part = (size_t)blockIdx.x * a.N;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
        const int at = first_column<kVec>(s, t, a.group);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = at + j * step;
            if (c >= a.N) continue;
            if (a.dw) a.dw[part + c] = a.add ? a.dw[part + c] + aw[s][j] : aw[s][j];
            if (a.db) a.db[part + c] = a.add ? a.db[part + c] + ab[s][j] : ab[s][j];
        }
    }
}

// out[c] (+)= sum of the blocks' parts of column c, in a fixed order: a thread adds up every kLanes-th part, then the lanes are added in turn
constexpr int kFoldLanes = 16;
__global__ void __launch_bounds__(32 * kFoldLanes) k_norm_fold(int blocks, int N, const float *pw, const float *pb, float *dw, float *db, int add)
{
    __shared__ float red[kFoldLanes][33];
    const float *p = blockIdx.y ? pb : pw;
    float *out = blockIdx.y ? db : dw;
    const int lane = threadIdx.x & 31, q = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    dependent_start();
    if (!out) return;
    float sum = 0.f;
    if (c < N) {
#pragma unroll 8
        for (int b = q; b < blocks; b += kFoldLanes) sum += __ldg(p + (size_t)b * N + c);
    }
    red[q][lane] = sum;
    __syncthreads();
    if (q || c >= N) return;
    sum = red[0][lane];
#pragma unroll
    for (int i = 1; i < kFoldLanes; ++i) sum += red[i][lane];
    out[c] = add ? out[c] + sum : sum;
}

// Threads of a row (a power of two) and eights of columns that a thread holds: two, four in rows of more than 16384 columns, where a block of
// 1024 would otherwise be too small.
struct NormLayout {
    int group, threads, slots, rows;
};
NormLayout norm_layout(int N)
{
    const int eights = (N + 7) / 8;
    NormLayout l;
    l.slots = eights > 2048 ? 4 : 2;
    l.group = 1;
    while (l.group * l.slots < eights) l.group <<= 1;
    l.threads = l.group > kNormThreads ? l.group : kNormThreads;
    l.rows = l.threads / l.group;
    return l;
}

// calls f(slots, threads, vec) with its arguments as compile-time constants
template <class F>
cudaError_t with_layout(const NormLayout &l, bool vec, F f)
{
    auto go = [&](auto slots, auto threads) {
        return vec ? f(slots, threads, std::integral_constant<bool, true>{}) : f(slots, threads, std::integral_constant<bool, false>{});
    };
    using std::integral_constant;
    if (l.slots == 4) return go(integral_constant<int, 4>{}, integral_constant<int, 1024>{});
    if (l.threads == 1024) return go(integral_constant<int, 2>{}, integral_constant<int, 1024>{});
    if (l.threads == 512) return go(integral_constant<int, 2>{}, integral_constant<int, 512>{});
    return go(integral_constant<int, 2>{}, integral_constant<int, 256>{});
}
template <class T>
struct Type {
    using type = T;
};
template <class F>
cudaError_t with_type(int dtype, F f) { return dtype == RR_F32 ? f(Type<float>{}) : f(Type<bf16>{}); }

bool in_eights(long long pitch, int dtype) { return pitch % (dtype == RR_F32 ? 4 : 8) == 0; }

constexpr int kNormBlocks = 2;  // blocks of 256 threads an SM (backward)

int bwd_blocks(int M, int N)
{
    const NormLayout l = norm_layout(N);
    const int sms = device_sm_count(), per_sm = l.threads > 256 ? 1 : kNormBlocks;
    const long long sets = ((long long)M + l.rows - 1) / l.rows, most = (long long)(sms > 0 ? sms : 148) * per_sm;
    return (int)(sets < most ? sets : most);
}

NormArgs norm_args(const rr_norm_shape &s, const NormLayout &l)
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

size_t norm_workspace(int M, int N) { return kHeaderBytes + align_up((size_t)bwd_blocks(M, N) * N * 4, 256) * 2; }

rr_status launch_norm_fwd(const rr_norm_shape &s, const void *x, const void *residual, const void *w, const void *b, void *h, void *y, float *mean,
                          float *rstd, cudaStream_t st)
{
    const NormLayout l = norm_layout(s.N);
    NormArgs a = norm_args(s, l);
    a.x = x;
    a.residual = residual;
    a.w = w;
    a.b = b;
    a.h = h;
    a.y = y;
    a.mean = a.layer ? mean : nullptr;
    a.rstd = rstd;
    const bool vec = s.N % 8 == 0 && in_eights(s.ldx, s.x_dtype) && in_eights(s.ldy, s.y_dtype) &&
                     (!residual || (in_eights(s.ldr, s.h_dtype) && in_eights(s.ldh, s.h_dtype)));
    const int sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    const long long sets = ((long long)s.M + l.rows - 1) / l.rows, most = (long long)sms * (2048 / l.threads);
    const dim3 grid((unsigned)(sets < most ? sets : most));
    auto types = [&](auto tx, auto th, auto ty) {
        return with_layout(l, vec, [&](auto slots, auto threads, auto v) {
            return launch_dependent(k_norm_fwd<typename decltype(tx)::type, typename decltype(th)::type, typename decltype(ty)::type, slots(), threads(), v()>,
                                    grid, l.threads, 0, 1, st, a);
        });
    };
    const cudaError_t err = with_type(s.x_dtype, [&](auto tx) {
        return with_type(s.y_dtype, [&](auto ty) {
            if (!residual) return types(tx, Type<void>{}, ty);
            return with_type(s.h_dtype, [&](auto th) { return types(tx, th, ty); });
        });
    });
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

rr_status launch_norm_bwd(const rr_norm_shape &s, const void *dy, const void *h, const void *w, const float *mean, const float *rstd, const void *dh,
                          void *dx, float *dw, float *db, void *workspace, cudaStream_t st)
{
    const NormLayout l = norm_layout(s.N);
    NormArgs a = norm_args(s, l);
    a.dy = dy;
    a.h = const_cast<void *>(h);
    a.w = w;
    a.mean = a.layer ? const_cast<float *>(mean) : nullptr;
    a.rstd = const_cast<float *>(rstd);
    a.dh = dh;
    a.dx = dx;
    const int blocks = bwd_blocks(s.M, s.N), add = (s.flags & RR_ADD_DW) != 0;
    const bool fold = blocks > 1 && (dw || db);
    Carver c(workspace);
    c.take<Header>(1);
    float *pw = c.take<float>((size_t)blocks * s.N), *pb = c.take<float>((size_t)blocks * s.N);
    a.dw = dw ? (fold ? pw : dw) : nullptr;
    a.db = db ? (fold ? pb : db) : nullptr;
    a.add = fold ? 0 : add;
    const bool vec = s.N % 8 == 0 && in_eights(s.lddy, s.y_dtype) && in_eights(s.ldh, s.h_dtype) && (!dh || in_eights(s.lddh, s.dx_dtype)) &&
                     (!dx || in_eights(s.lddx, s.dx_dtype));
    const size_t smem = l.rows > 1 && (dw || db) ? (size_t)2 * s.N * 4 : 0;  // (at most 2 x 2048 floats)
    cudaError_t err = with_type(s.y_dtype, [&](auto ty) {
        return with_type(s.h_dtype, [&](auto th) {
            return with_type(s.dx_dtype, [&](auto td) {
                return with_layout(l, vec, [&](auto slots, auto threads, auto v) {
                    return launch_dependent(k_norm_bwd<typename decltype(ty)::type, typename decltype(th)::type, typename decltype(td)::type, slots(), threads(), v()>,
                                            dim3(blocks), l.threads, smem, 1, st, a);
                });
            });
        });
    });
    if (err == cudaSuccess && fold)
        err = launch_dependent(k_norm_fold, dim3((s.N + 31) / 32, 2), 32 * kFoldLanes, 0, 1, st, blocks, s.N, (const float *)pw, (const float *)pb, dw, db, add);
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

}  // namespace rr
