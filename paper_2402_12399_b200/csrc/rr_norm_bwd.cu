// Gradients of the norm (rr_norm.cuh has the mathematics).
#include "rr_norm.cuh"

namespace rr {

namespace {

constexpr int bwd_blocks(int threads) { return threads == 256 ? 2 : 1; }  // an SM

__host__ __device__ constexpr int weight_bytes(int slots, int threads) { return slots * 8 * 4 * threads; }

// weights of eight columns from `at` on (1 where there are none)
template <Layout L>
__device__ __forceinline__ void weight(const NormArgs &a, int at, int step, f32x2 (&w)[4])
{
    if (!a.w || at >= a.N) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack2(1.f, 1.f);
    } else if (a.w_f32) {
        Eight<float, L> e;
        e.template load<kKeep>(static_cast<const float *>(a.w) + at, step, a.N - at);
        e.get(w);
    } else {
        Eight<bf16, L> e;
        e.template load<kKeep>(static_cast<const bf16 *>(a.w) + at, step, a.N - at);
        e.get(w);
    }
}

// A block takes every gridDim-th set of rows and keeps the sums of its columns over them in registers.  With four eights a thread there are no
// registers left to keep a row's numbers: they are worked out a second time.  TD: type of dx and dh.
template <class TY, class TH, class TD, Layout L, int kSlots, int kThreads, int G>
__global__ void __launch_bounds__(kThreads, bwd_blocks(kThreads)) k_norm_bwd(const NormArgs a)
{
    constexpr bool kHold = kSlots == 2;
    extern __shared__ __align__(16) char shared[];  // weights (kHold), then [2] dy, h, dh; afterwards the sums of the block's rows side by side
    __shared__ float2 buf[2][32];
    dependent_start();
    const int group = G ? G : a.group, rows = kThreads / group, t = threadIdx.x & (group - 1), step = step_of<L>(group), col = first_column<L>(t);
    long long row = (long long)blockIdx.x * rows + threadIdx.x / group;
    const int h_at = tensor_bytes(L, sizeof(TY), kSlots, kThreads, rows, a.N), d_at = h_at + tensor_bytes(L, sizeof(TH), kSlots, kThreads, rows, a.N);
    const int stage_bytes = d_at + (a.dh ? tensor_bytes(L, sizeof(TD), kSlots, kThreads, rows, a.N) : 0);
    // A thread's weights are the same in every row: they lie in shared memory as the numbers they are, each thread's its own.
    float4 *const weights = reinterpret_cast<float4 *>(shared) + threadIdx.x;
    char *const ring = shared + (kHold ? weight_bytes(kSlots, kThreads) : 0);
    if constexpr (kHold) {
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            f32x2 w[4];
            weight<L>(a, col + s * 8 * group, step, w);
#pragma unroll
            for (int q = 0; q < 2; ++q) quad_from(weights[(2 * s + q) * kThreads], w[2 * q], w[2 * q + 1]);
        }
    }
    const uint32_t ring_at = smem_u32(ring);
    // the thread's first column in the present rows
    const TY *py = static_cast<const TY *>(a.dy) + row * a.lddy + col;
    const TH *ph = static_cast<const TH *>(a.h) + row * a.ldh + col;
    const TD *pd = static_cast<const TD *>(a.dh) + row * a.lddh + col;
    TD *px = static_cast<TD *>(a.dx) + row * a.lddx + col;
    auto request = [&](long long r, const TY *y, const TH *h, const TD *d, int stage) {
        if (r < a.M) {
            const uint32_t to = ring_at + stage * stage_bytes;
            copy_row<TY, L, kSlots, kThreads>(to, y, t, group, a.N);
            copy_row<TH, L, kSlots, kThreads>(to + h_at, h, t, group, a.N);
            if (a.dh) copy_row<TD, L, kSlots, kThreads>(to + d_at, d, t, group, a.N);
        }
        copies_asked();
    };
    if (a.ahead) request(row, py, ph, pd, 0);
    float mean = 0.f, rstd = 0.f;
    if (row < a.M) {
        if (a.layer) mean = a.mean[row];
        rstd = a.rstd[row];
    }
    f32x2 aw[kSlots][4], ab[kSlots][4];
#pragma unroll
    for (int s = 0; s < kSlots; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) aw[s][j] = ab[s][j] = pack2(0.f, 0.f);
    int turn = 0, stage = 0;
    for (long long first = (long long)blockIdx.x * rows; first < a.M; first += a.stride) {
        const bool in = row < a.M;
        const char *here = ring + stage * stage_bytes;
        if (a.ahead) {
            stage = a.ahead == 2 ? stage ^ 1 : 0;
            if (L == kOne || a.ahead == 1) {
                copies_arrived<0>();
                if (L == kOne) row_barrier<G>();  // (the rows of the other buffer have been read by all, these have come for all)
            }
            if (a.ahead == 2) request(row + a.stride, py + a.sdy, ph + a.sh, pd + a.sdh, stage);
            if (L != kOne && a.ahead == 2) copies_arrived<1>();
        }
        const f32x2 centre = pack2(-mean, -mean), factor = pack2(rstd, rstd);
        mean = rstd = 0.f;
        if (row + a.stride < a.M) {  // (of the next row)
            if (a.layer) mean = a.mean[row + a.stride];
            rstd = a.rstd[row + a.stride];
        }
        // the numbers of slot s: dy, xh and dy w (behind the row: dy is 0, and so is all that is made of it)
        auto numbers = [&](int s, f32x2 (&y)[4], f32x2 (&x)[4], f32x2 (&g)[4]) {
            const int left = a.N - col - s * 8 * group;
            Eight<TY, L> ey;
            Eight<TH, L> eh;
            if (a.ahead) {
                take<TY, L, kThreads>(here, py, s, t, group, a.N, ey);
                take<TH, L, kThreads>(here + h_at, ph, s, t, group, a.N, eh);
            } else {
                ey.load(py + s * 8 * group, step, left);
                eh.load(ph + s * 8 * group, step, left);
            }
            ey.get(y);
            eh.get(x);
            f32x2 w[4];
            if constexpr (kHold) {
#pragma unroll
                for (int q = 0; q < 2; ++q) quad_of(weights[(2 * s + q) * kThreads], w[2 * q], w[2 * q + 1]);
            } else {
                weight<L>(a, col + s * 8 * group, step, w);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) g[j] = mul2(y[j], w[j]);
            if (a.layer) {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = add2(x[j], centre);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = mul2(x[j], factor);
        };
        f32x2 g[kHold ? kSlots : 1][4], xh[kHold ? kSlots : 1][4], p1 = pack2(0.f, 0.f), p2 = p1;
        if (in) {
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                const int k = kHold ? s : 0;
                if (col + s * 8 * group >= a.N) continue;
                f32x2 y[4];
                numbers(s, y, xh[k], g[k]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    aw[s][j] = fma2(y[j], xh[k][j], aw[s][j]);
                    p2 = fma2(g[k][j], xh[k][j], p2);
                }
                if (a.layer) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) p1 = add2(p1, g[k][j]);
                }
                if (a.db) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) ab[s][j] = add2(ab[s][j], y[j]);
                }
            }
        }
        if (a.dx) {
            float s1 = both(p1), s2 = both(p2);
            if (a.layer) row_sums<G, true>(s2, s1, group, buf, turn);
            else row_sums<G, false>(s2, s1, group, buf, turn);
            const f32x2 c1 = pack2(-s1 * a.inv_n, -s1 * a.inv_n), c2 = pack2(-s2 * a.inv_n, -s2 * a.inv_n);
            if (in) {
#pragma unroll
                for (int s = 0; s < kSlots; ++s) {
                    const int k = kHold ? s : 0, left = a.N - col - s * 8 * group;
                    if (left <= 0) continue;
                    if constexpr (!kHold) {
                        f32x2 y[4];
                        numbers(s, y, xh[0], g[0]);
                    }
                    Eight<TD, L> e;
                    f32x2 d[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = fma2(xh[k][j], c2, g[k][j]);
                    if (a.layer) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) d[j] = add2(d[j], c1);
                    }
                    if (a.dh) {
                        f32x2 o[4];
                        if (a.ahead) take<TD, L, kThreads>(here + d_at, pd, s, t, group, a.N, e);
                        else e.load(pd + s * 8 * group, step, left);
                        e.get(o);
#pragma unroll
                        for (int j = 0; j < 4; ++j) d[j] = fma2(d[j], factor, o[j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) d[j] = mul2(d[j], factor);
                    }
                    e.set(d);
                    e.store(px + s * 8 * group, step, left);
                }
            }
        }
        if (a.ahead == 1) {  // one buffer: the next row comes when this one has been read
            if (L == kOne) row_barrier<G>();
            request(row + a.stride, py + a.sdy, ph + a.sh, pd + a.sdh, 0);
        }
        row += a.stride;
        py += a.sdy;
        ph += a.sh;
        pd += a.sdh;
        px += a.sdx;
    }
    if (!a.dw && !a.db) return;
    // The sums of the rows side by side: of a warp by exchange (every lane adds the same pairs in the same order), of the block through shared memory
    for (int o = group; o < 32; o <<= 1) {
#pragma unroll
        for (int s = 0; s < kSlots; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                aw[s][j] = add2(aw[s][j], __shfl_xor_sync(0xffffffffu, aw[s][j], o));
                ab[s][j] = add2(ab[s][j], __shfl_xor_sync(0xffffffffu, ab[s][j], o));
            }
    }
    const size_t part = (size_t)blockIdx.x * a.N;
    const int sets = kThreads / (group < 32 ? 32 : group);
    if (sets == 1) {
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = col + s * 8 * group;
            if (at >= a.N) continue;
            float *const out[2] = {a.dw, a.db};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (!out[k]) continue;
                f32x2 o[4];
                Eight<float, L> e;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = k ? ab[s][j] : aw[s][j];
                if (a.add) {
                    f32x2 old[4];
                    e.load(out[k] + part + at, step, a.N - at);
                    e.get(old);
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = add2(old[j], o[j]);
                }
                e.set(o);
                e.template store<kKeep>(out[k] + part + at, step, a.N - at);
            }
        }
        return;
    }
    copies_arrived<0>();
    __syncthreads();  // (nobody reads rows any more)
    float *const sums = reinterpret_cast<float *>(ring);  // [sets][2][N]
    const int set = threadIdx.x / (group < 32 ? 32 : group);
    if (group >= 32 || (int)(threadIdx.x & 31) < group) {
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = col + s * 8 * group;
            if (at >= a.N) continue;
            Eight<float, kOne> e;  // (element by element: a row of sums starts anywhere)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float *out = sums + (2 * set + k) * a.N;
                e.set(k ? ab[s] : aw[s]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = L == kEights ? at + j : L == kQuads ? at + (j >> 2) * step + (j & 3) : at + j * step;
                    if (c < a.N) out[c] = e.e[j];
                }
            }
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.N; c += kThreads) {
        float *out = c < a.N ? a.dw : a.db;
        if (!out) continue;
        float sum = sums[c];
        for (int q = 1; q < sets; ++q) sum += sums[2 * q * a.N + c];
        float *o = out + part + (c < a.N ? c : c - a.N);
        *o = a.add ? *o + sum : sum;
    }
}

// out[c] (+)= sum of the blocks' parts of column c, in a fixed order: thread (q, lane) adds up every kFoldLanes-th part of column `lane`, then a warp
// adds up the kFoldLanes sums of a column in pairs
constexpr int kFoldLanes = 32;
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
        for (int b = q; b < blocks; b += kFoldLanes) sum += __ldcs(p + (size_t)b * N + c);
    }
    red[q][lane] = sum;
    __syncthreads();
    sum = red[lane][q];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const int column = blockIdx.x * 32 + q;
    if (lane == 0 && column < N) out[column] = add ? out[column] + sum : sum;
}

// Two eights a thread beside the sums of as many columns; four from 8192 columns on, where two would take a block of 1024.
NormLayout bwd_layout(int N) { return norm_layout(N, N > 8192 ? 4 : 2, 256); }

int bwd_parts(int M, int N)
{
    const NormLayout l = bwd_layout(N);
    const int sms = device_sm_count();
    const long long sets = ((long long)M + l.rows - 1) / l.rows, most = (long long)(sms > 0 ? sms : 148) * bwd_blocks(l.threads);
    if (sets <= 4) return 1;  // (one block after the other set of rows: no second kernel, the device takes as long and the caller 2 us less)
    return (int)(sets < most ? sets : most);
}

template <Layout L, class F>
cudaError_t with_layout(const NormLayout &l, F f)
{
    switch (l.group) {
    case 32: return call<L, 2, 256, 32>(f);
    case 64: return call<L, 2, 256, 64>(f);
    case 128: return call<L, 2, 256, 128>(f);
    case 256: return call<L, 2, 256, 256>(f);
    case 512: return l.slots == 2 ? call<L, 2, 512, 512>(f) : call<L, 4, 512, 512>(f);
    case 1024: return call<L, 4, 1024, 1024>(f);
    default: return call<L, 2, 256, 0>(f);
    }
}

}  // namespace

// (enough for narrower rows too, so that the workspace of a program's largest norm serves every other: up to 4096 columns there are two blocks an
// SM that leave a part, beyond that one)
size_t norm_workspace(int M, int N)
{
    const int narrow = N < 4096 ? N : 4096;
    const size_t own = (size_t)bwd_parts(M, N) * N, less = (size_t)bwd_parts(M, narrow) * narrow;
    return kHeaderBytes + align_up((own > less ? own : less) * 4, 256) * 2;
}

rr_status launch_norm_bwd(const rr_norm_shape &s, const void *dy, const void *h, const void *w, const float *mean, const float *rstd, const void *dh,
                          void *dx, float *dw, float *db, void *workspace, cudaStream_t st)
{
    Access access(s.N);
    access.matrix(dy, s.y_dtype, s.lddy);
    access.matrix(h, s.h_dtype, s.ldh);
    access.matrix(dh, s.dx_dtype, s.lddh);
    access.matrix(dx, s.dx_dtype, s.lddx);
    if (!dh && !dx) access.all_bf16 = access.all_bf16 && s.dx_dtype == RR_BF16;  // (its kernels are of that type all the same)
    const Layout L = access.layout();
    const NormLayout l = bwd_layout(s.N);
    const int parts = bwd_parts(s.M, s.N), add = (s.flags & RR_ADD_DW) != 0;
    NormArgs a = norm_args(s, l, parts);
    a.dy = dy;
    a.h = const_cast<void *>(h);
    a.w = w;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.dh = dh;
    a.dx = dx;
    // (gradients that start anywhere, in a flat buffer, are written one by one: the second kernel does; one row 4.8 us instead of 3.1)
    const bool fold = (dw || db) && (parts > 1 || ((uintptr_t)dw | (uintptr_t)db) % 16 != 0);
    Carver c(workspace);
    c.take<Header>(1);
    float *pw = c.take<float>((size_t)parts * s.N), *pb = c.take<float>((size_t)parts * s.N);
    a.dw = dw ? (fold ? pw : dw) : nullptr;
    a.db = db ? (fold ? pb : db) : nullptr;
    a.add = fold ? 0 : add;
    auto bytes = [&](int dtype) { return tensor_bytes(L, dtype == RR_F32 ? 4 : 2, l.slots, l.threads, l.rows, s.N); };
    const int weights = l.slots == 2 ? weight_bytes(2, l.threads) : 0;
    const int row = bytes(s.y_dtype) + bytes(s.h_dtype) + (dh ? bytes(s.dx_dtype) : 0), room = kMostShared / bwd_blocks(l.threads) - weights;
    // (a block with one set of rows has nothing to fetch ahead)
    a.ahead = (long long)s.M <= (long long)parts * l.rows ? 0 : 2 * row <= room ? 2 : row <= room ? 1 : 0;
    int smem = weights + a.ahead * row;
    const int sets = l.threads / (l.group < 32 ? 32 : l.group), sums = sets > 1 ? sets * 2 * s.N * 4 : 0;  // (32 KB at most)
    if (smem < weights + sums) smem = weights + sums;
    cudaError_t err = with_type(s.y_dtype, [&](auto ty) {
        return with_type(s.h_dtype, [&](auto th) {
            return with_type(s.dx_dtype, [&](auto td) {
                using TY = typename decltype(ty)::type;
                using TH = typename decltype(th)::type;
                using TD = typename decltype(td)::type;
                auto go = [&](auto layout, auto slots, auto threads, auto group) {
                    auto kernel = k_norm_bwd<TY, TH, TD, layout(), slots(), threads(), group()>;
                    static SharedAllowance allowance;
                    const cudaError_t e = allowance.ask(kernel, smem);
                    return e != cudaSuccess ? e : launch_dependent(kernel, dim3(parts), threads(), (size_t)smem, 1, st, a);
                };
                if constexpr (sizeof(TY) + sizeof(TH) + sizeof(TD) == 6) {
                    if (L == kEights) return with_layout<kEights>(l, go);
                }
                return L == kOne ? with_layout<kOne>(l, go) : with_layout<kQuads>(l, go);
            });
        });
    });
    if (err == cudaSuccess && fold)
        err = launch_dependent(k_norm_fold, dim3((s.N + 31) / 32, 2), 32 * kFoldLanes, 0, 1, st, parts, s.N, (const float *)pw, (const float *)pb, dw, db, add);
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

}  // namespace rr
