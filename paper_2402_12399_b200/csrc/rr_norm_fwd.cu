// The norm with the residual add of the branch before it, forward (rr_norm.cuh has the mathematics).
#include "rr_norm.cuh"

namespace rr {

namespace {

constexpr int fwd_blocks(int threads) { return threads == 128 ? 6 : threads == 256 ? 3 : threads == 512 ? 2 : 1; }  // an SM

// TH: type of the residual stream, void without one
template <class TX, class TH, class TY, Layout L, int kSlots, int kThreads>
__global__ void __launch_bounds__(kThreads, fwd_blocks(kThreads)) k_norm_fwd(const NormArgs a)
{
    constexpr bool kRes = !std::is_same<TH, void>::value;
    using TR = std::conditional_t<kRes, TH, float>;
    extern __shared__ __align__(16) char ring[];  // [2] x, then residual
    __shared__ float2 buf[2][32];
    dependent_start();
    const int t = threadIdx.x & (a.group - 1), step = step_of<L>(a.group), rows = kThreads / a.group;
    const long long stride = (long long)gridDim.x * rows;
    long long row = (long long)blockIdx.x * rows + threadIdx.x / a.group;
    const int residual_at = tensor_bytes(L, sizeof(TX), kSlots, kThreads, rows, a.N);
    const int stage_bytes = residual_at + (kRes ? tensor_bytes(L, sizeof(TR), kSlots, kThreads, rows, a.N) : 0);
    auto request = [&](long long r, char *to) {
        if (r < a.M) {
            copy_row<TX, L, kSlots, kThreads>(to, static_cast<const TX *>(a.x) + r * a.ldx, t, a.group, a.N);
            if (kRes) copy_row<TR, L, kSlots, kThreads>(to + residual_at, static_cast<const TR *>(a.residual) + r * a.ldr, t, a.group, a.N);
        }
        copies_asked();
    };
    if (a.ahead) request(row, ring);
    int turn = 0, stage = 0;
    for (long long first = (long long)blockIdx.x * rows; first < a.M; first += stride, row += stride) {
        const bool in = row < a.M;
        f32x2 v[kSlots][4];
        {
            Eight<TX, L> ex[kSlots];
            Eight<TR, L> er[kSlots];
            const char *here = ring + stage * stage_bytes;
            if (a.ahead) {
                stage ^= 1;
                if (L == kOne) {  // (the rows of the other buffer have been read by all, these have come for all)
                    copies_arrived<0>();
                    row_barrier(a.group);
                    request(row + stride, ring + stage * stage_bytes);
                } else {
                    request(row + stride, ring + stage * stage_bytes);
                    copies_arrived<1>();
                }
            }
            const TX *px = static_cast<const TX *>(a.x) + row * a.ldx;
            const TR *pr = static_cast<const TR *>(a.residual) + row * a.ldr;
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                const int at = first_column<L>(s, t, a.group);
                if (!in || at >= a.N) {
                    ex[s].zero();
                    if (kRes) er[s].zero();
                } else if (a.ahead) {
                    take<TX, L, kThreads>(here, px, s, t, a.group, a.N, ex[s]);
                    if (kRes) take<TR, L, kThreads>(here + residual_at, pr, s, t, a.group, a.N, er[s]);
                } else {
                    ex[s].load(px + at, step, a.N - at);
                    if (kRes) er[s].load(pr + at, step, a.N - at);
                }
            }
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                ex[s].get(v[s]);
                if constexpr (kRes) {
                    f32x2 r[4];
                    er[s].get(r);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[s][j] = add2(v[s][j], r[j]);
                    er[s].set(v[s]);
                    er[s].get(v[s]);  // the norm is that of the stream as it is stored
                    const int at = first_column<L>(s, t, a.group);
                    if (a.h && in && at < a.N) er[s].store(static_cast<TR *>(a.h) + row * a.ldh + at, step, a.N - at);
                }
            }
        }
        float m = 0.f, d1 = 0.f, d2 = 0.f;
        if (a.layer) {
            f32x2 sum = pack2(0.f, 0.f);
#pragma unroll
            for (int s = 0; s < kSlots; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = add2(sum, v[s][j]);
            m = both(sum);
            row_sums(m, d1, a.group, buf, turn);
            m *= a.inv_n;
            sum = pack2(0.f, 0.f);
            const f32x2 centre = pack2(-m, -m);
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[s][j] = add2(v[s][j], centre);
                cut<L>(v[s], first_column<L>(s, t, a.group), step, a.N);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = add2(sum, v[s][j]);
            }
            d1 = both(sum);
        }
        f32x2 square = pack2(0.f, 0.f);
#pragma unroll
        for (int s = 0; s < kSlots; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) square = fma2(v[s][j], v[s][j], square);
        d2 = both(square);
        row_sums(d1, d2, a.group, buf, turn);
        // what rounding left of the mean is in d1 (a row far from zero against its spread)
        const float rest = d1 * a.inv_n;
        const float rstd = __frsqrt_rn(fmaxf(fmaf(d2, a.inv_n, -rest * rest), 0.f) + a.eps);
        if (!in) continue;
        if (t == 0) {
            if (a.mean) a.mean[row] = m + rest;
            if (a.rstd) a.rstd[row] = rstd;
        }
        const f32x2 factor = pack2(rstd, rstd), shift = pack2(-rest * rstd, -rest * rstd);
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            const int at = first_column<L>(s, t, a.group);
            if (at >= a.N) break;
            f32x2 w[4];
            parameter<L>(a.w, a.w_f32, at, step, a.N - at, 1.f, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[s][j] = mul2(fma2(v[s][j], factor, shift), w[j]);
            if (a.b) {
                parameter<L>(a.b, a.w_f32, at, step, a.N - at, 0.f, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[s][j] = add2(v[s][j], w[j]);
            }
            Eight<TY, L> e;
            e.set(v[s]);
            e.store(static_cast<TY *>(a.y) + row * a.ldy + at, step, a.N - at);
        }
    }
}

// Four eights a thread, which has its registers for one row; two where elements go one by one, if that is enough.
NormLayout fwd_layout(int N, Layout L) { return norm_layout(N, L == kOne && N <= 16384 ? 2 : 4, 128); }

template <Layout L, class F>
cudaError_t with_layout(const NormLayout &l, F f)
{
    constexpr int kSlots = L == kOne ? 2 : 4;
    if (l.threads == 128) return call<L, kSlots, 128>(f);
    if (l.threads == 256) return call<L, kSlots, 256>(f);
    if (l.threads == 512) return call<L, kSlots, 512>(f);
    return l.slots == 4 ? call<L, 4, 1024>(f) : call<L, kSlots, 1024>(f);
}

}  // namespace

rr_status launch_norm_fwd(const rr_norm_shape &s, const void *x, const void *residual, const void *w, const void *b, void *h, void *y, float *mean,
                          float *rstd, cudaStream_t st)
{
    Access access(s.N);
    access.matrix(x, s.x_dtype, s.ldx);
    access.matrix(residual, s.h_dtype, s.ldr);
    access.matrix(h, s.h_dtype, s.ldh);
    access.matrix(y, s.y_dtype, s.ldy);
    const Layout L = access.layout();
    const NormLayout l = fwd_layout(s.N, L);
    NormArgs a = norm_args(s, l);
    a.x = x;
    a.residual = residual;
    a.w = w;
    a.b = b;
    a.h = h;
    a.y = y;
    a.mean = a.layer ? mean : nullptr;
    a.rstd = rstd;
    const int sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    const long long sets = ((long long)s.M + l.rows - 1) / l.rows;
    int smem = 2 * (tensor_bytes(L, s.x_dtype == RR_F32 ? 4 : 2, l.slots, l.threads, l.rows, s.N) +
                    (residual ? tensor_bytes(L, s.h_dtype == RR_F32 ? 4 : 2, l.slots, l.threads, l.rows, s.N) : 0));
    int per_sm = fwd_blocks(l.threads);
    a.ahead = sets > (long long)sms * per_sm && smem <= kMostShared;  // (a block with one set of rows has nothing to fetch ahead)
    if (!a.ahead) smem = 0;
    while (per_sm > 1 && per_sm * (smem + 1024) > kMostShared) --per_sm;
    const dim3 grid((unsigned)(sets < (long long)sms * per_sm ? sets : (long long)sms * per_sm));
    auto types = [&](auto tx, auto th, auto ty) {
        using TX = typename decltype(tx)::type;
        using TH = typename decltype(th)::type;
        using TY = typename decltype(ty)::type;
        auto go = [&](auto layout, auto slots, auto threads) {
            auto kernel = k_norm_fwd<TX, TH, TY, layout(), slots(), threads()>;
            const cudaError_t err = allow(kernel, smem);
            return err != cudaSuccess ? err : launch_dependent(kernel, grid, threads(), (size_t)smem, 1, st, a);
        };
        if constexpr (sizeof(TX) + sizeof(TY) == 4 && !std::is_same<TH, float>::value) {
            if (L == kEights) return with_layout<kEights>(l, go);
        }
        return L == kOne ? with_layout<kOne>(l, go) : with_layout<kQuads>(l, go);
    };
    const cudaError_t err = with_type(s.x_dtype, [&](auto tx) {
        return with_type(s.y_dtype, [&](auto ty) {
            if (!residual) return types(tx, Type<void>{}, ty);
            return with_type(s.h_dtype, [&](auto th) { return types(tx, th, ty); });
        });
    });
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

}  // namespace rr
