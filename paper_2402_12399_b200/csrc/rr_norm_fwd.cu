// The norm with the residual add of the branch before it, forward (rr_norm.cuh has the mathematics).
#include "rr_norm.cuh"

namespace rr {

namespace {

constexpr int fwd_blocks(int threads, int slots) { return (slots == 2 || threads > 256 ? 1024 : 768) / threads; }  // an SM

// v w + b of eight columns from `at` on (w and b come from the L1 cache: a block meets the same columns in every row)
template <class TW, Layout L>
__device__ __forceinline__ void apply(const NormArgs &a, int at, int step, f32x2 (&v)[4])
{
    Eight<TW, L> e;
    f32x2 p[4];
    if (a.w) {
        e.template load<kKeep>(static_cast<const TW *>(a.w) + at, step, a.N - at);
        e.get(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = mul2(v[j], p[j]);
    }
    if (a.b) {
        e.template load<kKeep>(static_cast<const TW *>(a.b) + at, step, a.N - at);
        e.get(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = add2(v[j], p[j]);
    }
}

// TH: type of the residual stream, void without one
template <class TX, class TH, class TY, Layout L, int kSlots, int kThreads, int G>
__global__ void __launch_bounds__(kThreads, fwd_blocks(kThreads, kSlots)) k_norm_fwd(const NormArgs a)
{
    constexpr bool kRes = !std::is_same<TH, void>::value;
    using TR = std::conditional_t<kRes, TH, float>;
    __shared__ float2 buf[2][32];
    dependent_start();
    const int group = G ? G : a.group, rows = kThreads / group, t = threadIdx.x & (group - 1), step = step_of<L>(group), col = first_column<L>(t);
    long long row = (long long)blockIdx.x * rows + threadIdx.x / group;
    const TX *px = static_cast<const TX *>(a.x) + row * a.ldx + col;
    const TR *pr = static_cast<const TR *>(a.residual) + row * a.ldr + col;
    TR *ph = static_cast<TR *>(a.h) + row * a.ldh + col;
    TY *py = static_cast<TY *>(a.y) + row * a.ldy + col;
    int turn = 0;
    for (long long first = (long long)blockIdx.x * rows; first < a.M; first += a.stride) {
        const bool in = row < a.M;
        f32x2 v[kSlots][4];
        {
            Eight<TX, L> ex[kSlots];
            Eight<TR, L> er[kSlots];
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                const int left = a.N - col - s * 8 * group;
                if (!in || left <= 0) {
                    ex[s].zero();
                    if (kRes) er[s].zero();
                } else {
                    ex[s].load(px + s * 8 * group, step, left);
                    if (kRes) er[s].load(pr + s * 8 * group, step, left);
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
                    const int left = a.N - col - s * 8 * group;
                    if (a.h && in && left > 0) er[s].store(ph + s * 8 * group, step, left);
                }
            }
        }
        float m = 0.f, d1 = 0.f, d2 = 0.f;
        if (a.layer) {
            f32x2 sum = pack2(0.f, 0.f);  // (in pairs: a mean is often small against its terms)
#pragma unroll
            for (int s = 0; s < kSlots; ++s) sum = add2(sum, add2(add2(v[s][0], v[s][1]), add2(v[s][2], v[s][3])));
            m = both(sum);
            row_sums<G, false>(m, d1, group, buf, turn);
            m *= a.inv_n;
            sum = pack2(0.f, 0.f);
            const f32x2 centre = pack2(-m, -m);
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[s][j] = add2(v[s][j], centre);
                cut<L>(v[s], step, a.N - col - s * 8 * group);
                sum = add2(sum, add2(add2(v[s][0], v[s][1]), add2(v[s][2], v[s][3])));
            }
            d1 = both(sum);
        }
        f32x2 square = pack2(0.f, 0.f);
#pragma unroll
        for (int s = 0; s < kSlots; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) square = fma2(v[s][j], v[s][j], square);
        d2 = both(square);
        if (a.layer) row_sums<G, true>(d2, d1, group, buf, turn);
        else row_sums<G, false>(d2, d1, group, buf, turn);
        // what rounding left of the mean is in d1 (a row far from zero against its spread)
        const float rest = a.layer ? d1 * a.inv_n : 0.f;
        const float spread = fmaf(d2, a.inv_n, -rest * rest);
        const float rstd = __frsqrt_rn((spread < 0.f ? 0.f : spread) + a.eps);  // (a NaN stays one)
        if (in) {
            if (t == 0) {
                // (`rest` is the mean of rounded differences: below a few of their half steps it says more about them than about m)
                if (a.mean) a.mean[row] = fabsf(rest) * rstd > 0x1p-22f ? m + rest : m;
                if (a.rstd) a.rstd[row] = rstd;
            }
            const f32x2 factor = pack2(rstd, rstd), shift = pack2(-rest * rstd, -rest * rstd);
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                const int at = col + s * 8 * group;
                if (at >= a.N) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[s][j] = fma2(v[s][j], factor, shift);
                if (a.w_f32) apply<float, L>(a, at, step, v[s]);
                else apply<bf16, L>(a, at, step, v[s]);
                Eight<TY, L> e;
                e.set(v[s]);
                e.store(py + s * 8 * group, step, a.N - at);
            }
        }
        row += a.stride;
        px += a.sx;
        py += a.sy;
        if (kRes) {
            pr += a.sr;
            ph += a.sh;
        }
    }
}

// Two eights a thread, or four: one matrix to read and rows enough to fill the SMs want more of it in flight (65536 x 1024 in bf16 44 us instead of 53), and a
// row beyond 4096 columns fewer threads that meet (8192 x 8192 52 us instead of 71).
NormLayout fwd_layout(int M, int N, Layout L, bool residual, int sms)
{
    NormLayout l = norm_layout(N, 2, 128);
    const bool fills = (long long)M > (long long)sms * fwd_blocks(l.threads, 2) * l.rows;
    if (N > 16384 || (L != kOne && N > 4096) || (L == kEights && !residual && fills)) l = norm_layout(N, 4, 128);
    return l;
}

template <Layout L, class F>
cudaError_t with_layout(const NormLayout &l, F f)
{
    if (l.slots == 2) {
        switch (l.group) {
        case 32: return call<L, 2, 128, 32>(f);
        case 64: return call<L, 2, 128, 64>(f);
        case 128: return call<L, 2, 128, 128>(f);
        case 256: return call<L, 2, 256, 256>(f);
        default:
            if constexpr (L == kOne) {
                if (l.group == 512) return call<L, 2, 512, 512>(f);
                if (l.group == 1024) return call<L, 2, 1024, 1024>(f);
            }
            return call<L, 2, 128, 0>(f);
        }
    }
    if constexpr (L != kOne) {
        if (l.group == 256) return call<L, 4, 256, 256>(f);
        if (l.group == 512) return call<L, 4, 512, 512>(f);
    }
    if constexpr (L == kEights) {
        switch (l.group) {
        case 32: return call<L, 4, 128, 32>(f);
        case 64: return call<L, 4, 128, 64>(f);
        case 128: return call<L, 4, 128, 128>(f);
        default:
            if (l.group < 32) return call<L, 4, 128, 0>(f);
        }
    }
    return call<L, 4, 1024, 1024>(f);
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
    const int sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    const NormLayout l = fwd_layout(s.M, s.N, L, residual != nullptr, sms);
    const long long sets = ((long long)s.M + l.rows - 1) / l.rows;
    // Blocks far beyond those resident: each is short, so that they drift apart and reads and writes mix, and the last ones leave few SMs idle
    // (16384 x 4096, fp32 + bf16 residual: 111 us with the resident ones, 99 so).
    const long long most = (long long)sms * 32;
    const dim3 grid((unsigned)(sets < most ? sets : most));
    NormArgs a = norm_args(s, l, grid.x);
    a.x = x;
    a.residual = residual;
    a.w = w;
    a.b = b;
    a.h = h;
    a.y = y;
    a.mean = a.layer ? mean : nullptr;
    a.rstd = rstd;
    auto types = [&](auto tx, auto th, auto ty) {
        using TX = typename decltype(tx)::type;
        using TH = typename decltype(th)::type;
        using TY = typename decltype(ty)::type;
        auto go = [&](auto layout, auto slots, auto threads, auto group) {
            return launch_dependent(k_norm_fwd<TX, TH, TY, layout(), slots(), threads(), group()>, grid, threads(), 0, 1, st, a);
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
