// Dense linear layer with its epilogue, and its gradients (bf16 operands, fp32 accumulation):
//     z = x W^T + b,   y = residual + D(act(z))                       x [M,K], W [N,K], y [M,N]
//     dz = D(dy) act'(z),   dx = dz W,   dW = dz^T x,   db = sum over rows of dz
// D is dropout with the counter-based mask of rr_philox.cuh on the flat index row*N + column: the backward pass
// computes the mask again.  The three products run on one GEMM kernel (k_dense): 256-row tiles on CTA pairs
// (cta_group::2), operands by TMA, two TMEM accumulators so that the epilogue of one tile overlaps the main loop
// of the next.  Operands are read as they lie in memory (K-major or MN-major), nothing is transposed.
#include <cuda.h>
#include <cuda_bf16.h>

#include "rr_ffn.cuh"
#include "rr_linear.cuh"
#include "rr_tc.cuh"

namespace rr {

using namespace tc;

namespace {

constexpr int kStageA = 128 * 128;       // this CTA's 128 rows of A, one k-block of 64
constexpr int kPanel = 64 * 128;         // MN-major panel: 64 k-rows x 64 columns
constexpr int kDenseProducers = 3, kDenseMma = 3, kDenseEpi0 = 4, kDenseEpiWarps = 8;
constexpr int kDenseThreads = 32 * (kDenseEpi0 + kDenseEpiWarps);
constexpr int kEpiBytes = 4096;          // staging of one epilogue warp

struct DenseShared {
    uint64_t full[12], empty[12], tfull[2], tempty[2];
    uint32_t tmem_base;
    int abort_flag;
};

template <int TN>
__host__ __device__ constexpr int dense_stage_bytes() { return kStageA + TN / 2 * 128; }
template <int TN>
__host__ __device__ constexpr int dense_stages() { return TN == 256 ? 6 : 8; }
template <int TN>
constexpr size_t dense_smem() { return 1024 + (size_t)dense_stages<TN>() * dense_stage_bytes<TN>() + kDenseEpiWarps * kEpiBytes + sizeof(DenseShared); }

struct DenseParams {
    int M, N;              // rows and columns of the result
    int m_tiles, n_tiles;  // 256-row and TN-column tiles
    int kblocks;
    Epilogue e;
    int *status;
};

// Tile `t` of the raster: bands of eight row tiles, inside a band column after column, so that the pairs running
// together share few A and B tiles (74 pairs: 8 x 9) and find them in L2.
struct Tile {
    int m, n;
};
__device__ __forceinline__ Tile tile_of(const DenseParams &p, int t)
{
    const int band = 8 * p.n_tiles, b = t / band, first = 8 * b, high = min(8, p.m_tiles - first), r = t - b * band;
    return {first + r % high, r / high};
}

// kAmn / kBmn: operand is MN-major, i.e. the contraction runs over its rows.
template <int TN, bool kAmn, bool kBmn>
__global__ void __launch_bounds__(kDenseThreads, 1)
k_dense(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapY,
        const __grid_constant__ CUtensorMap mapZ, const __grid_constant__ DenseParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kNS = dense_stages<TN>(), kStage = dense_stage_bytes<TN>(), kBRows = TN / 2;
    uint8_t *staging = tiles + (size_t)kNS * kStage;
    DenseShared *sh = reinterpret_cast<DenseShared *>(staging + kDenseEpiWarps * kEpiBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank(), pair = (int)(blockIdx.x >> 1), npairs = (int)(gridDim.x >> 1);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kNS; ++s) { mbar_init(&sh->full[s], 1); mbar_init(&sh->empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&sh->tfull[b], 1); mbar_init(&sh->tempty[b], 2 * 32 * kDenseEpiWarps); }
        sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&mapA);
        prefetch_map(&mapB);
        prefetch_map(&mapY);
    }
    if (warp == kDenseMma) {
        tmem_alloc_pair(&sh->tmem_base, 2 * TN);
        tmem_relinquish_pair();
    }
    fence_before_sync();
    __syncthreads();
    cluster_sync_all();  // the peer's barriers are initialised before anything signals them
    fence_after_sync();
    const uint32_t tmem_base = sh->tmem_base;
    volatile int *abort_flag = &sh->abort_flag;
    const int total = p.m_tiles * p.n_tiles;
    const uint32_t lead_full = map_to_cta(&sh->full[0], 0), lead_tempty = map_to_cta(&sh->tempty[0], 0);

    if (warp < kDenseProducers) {
        // TMA producers: producer j takes the k-blocks j, j + 3, ... of this CTA's stream
        if (lane == 0) {
            uint32_t s = warp % kNS, ph = 0;
            int kb = warp;
            bool ok = true;
            for (int t = pair; ok && t < total; t += npairs) {
                const Tile w = tile_of(p, t);
                const int row = w.m * 256 + 128 * rank, col = w.n * TN + kBRows * rank;  // this CTA's rows of A and of B
                for (; kb < p.kblocks; kb += kDenseProducers) {
                    if (!mbar_wait(&sh->empty[s], ph ^ 1u, abort_flag, p.status)) { ok = false; break; }
                    uint8_t *a = tiles + (size_t)s * kStage, *b = a + kStageA;
                    const uint32_t bar = lead_full + 8u * s;
                    if (rank == 0) mbar_expect_tx(&sh->full[s], 2u * kStage);  // bytes of both CTAs
                    if (kAmn) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) tma_tile_2d_pair(a + q * kPanel, &mapA, row + 64 * q, kb * 64, bar);
                    } else {
                        tma_tile_2d_pair(a, &mapA, kb * 64, row, bar);
                    }
                    if (kBmn) {
#pragma unroll
                        for (int q = 0; q < kBRows / 64; ++q) tma_tile_2d_pair(b + q * kPanel, &mapB, col + 64 * q, kb * 64, bar);
                    } else {
                        tma_tile_2d_pair(b, &mapB, kb * 64, col, bar);
                    }
                    s += kDenseProducers;
                    if (s >= (uint32_t)kNS) { s -= kNS; ph ^= 1u; }
                }
                kb -= p.kblocks;
            }
        }
    } else if (warp == kDenseMma) {
        if (rank == 0 && lane == 0) {
            const uint32_t idesc = instr_desc(1u, kAmn ? 1u : 0u, kBmn ? 1u : 0u, 256, TN);
            const uint32_t a0 = smem_u32(tiles);
            const uint64_t adesc0 = kAmn ? smem_desc(a0, kPanel, 1024) : smem_desc(a0, 16, 1024);
            const uint64_t bdesc0 = kBmn ? smem_desc(a0 + kStageA, kPanel, 1024) : smem_desc(a0 + kStageA, 16, 1024);
            constexpr uint32_t a_step = kAmn ? 128u : 2u, b_step = kBmn ? 128u : 2u;
            uint32_t s = 0, ph = 0, it = 0;
            bool ok = true;
            for (int t = pair; ok && t < total; t += npairs, ++it) {
                const uint32_t buf = it & 1u;
                if (!mbar_wait(&sh->tempty[buf], ((it >> 1) & 1u) ^ 1u, abort_flag, p.status)) break;
                fence_after_sync();
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    if (!mbar_wait(&sh->full[s], ph, abort_flag, p.status)) { ok = false; break; }
                    fence_after_sync();
                    const uint32_t off = s * (uint32_t)(kStage >> 4);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_ss_pair<false>(tmem_base + buf * TN, adesc0 + off + a_step * kk, bdesc0 + off + b_step * kk, idesc, (kb | kk) != 0);
                    mma_commit_pair(&sh->empty[s]);
                    if (++s == (uint32_t)kNS) { s = 0; ph ^= 1u; }
                }
                if (ok) mma_commit_pair(&sh->tfull[buf]);
            }
        }
    } else {
        // Epilogue: two warps per TMEM lane quarter take alternate chunks of 32 columns
        const int eg = (warp - kDenseEpi0) >> 2, q = warp & 3;
        uint8_t *st = staging + (size_t)(eg * 4 + q) * kEpiBytes;
        EpilogueWarp ew(p.e);
        uint32_t it = 0;
        for (int t = pair; t < total; t += npairs, ++it) {
            const Tile w = tile_of(p, t);
            const uint32_t buf = it & 1u;
            if (!warp_wait(&sh->tfull[buf], (it >> 1) & 1u, abort_flag, p.status)) break;
            fence_after_sync();
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + buf * TN;
            const int row0 = w.m * 256 + 128 * rank + q * 32;  // first of this warp's 32 rows
            if (row0 < p.M) {
#pragma unroll 1
                for (int c = eg; c < TN / 32; c += 2) {
                    const int col0 = w.n * TN + c * 32;
                    if (col0 >= p.N) break;
                    float v[32];
                    tmem_ld32(taddr + c * 32, v);
                    ew.chunk(p.e, v, row0, col0, p.M, p.N, lane, st, &mapY, &mapZ);
                }
            }
            fence_before_sync();
            mbar_arrive_cluster(lead_tempty + 8u * buf);
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }

    __syncwarp();
    __syncthreads();
    if (sh->abort_flag) __nanosleep(2000000);  // let copies that are still in flight land
    cluster_sync_all();  // neither CTA leaves while its peer may still signal its barriers
    if (warp == kDenseMma) {
        fence_after_sync();
        tmem_dealloc_pair(tmem_base, 2 * TN);
    }
}

// ---- dz and its column sums ---------------------------------------------------------------------------
constexpr int kDzThreads = 256, kDzCols = 256;  // 32 threads x 8 columns, 8 rows at a time

// Block (bx, by): columns [256 bx, ...), rows [by*slab, ...).  dz[row, col] = keep dy act'(z) without the dropout factor
// (the GEMMs and the column sums apply it), so that without an activation the rounding to bf16 loses nothing.
// `dz` may be null (only the sums are wanted), `partial` too.
template <int kAct>
__global__ void __launch_bounds__(kDzThreads)
k_dz(int M, int N, const __nv_bfloat16 *__restrict__ dy, long long lddy, const __nv_bfloat16 *__restrict__ z, long long ldz,
     DropoutParams d, int slab, __nv_bfloat16 *__restrict__ dz, float *__restrict__ partial)
{
    __shared__ float red[kDzThreads / 32][kDzCols];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, col = blockIdx.x * kDzCols + tx * 8;
    const int r0 = blockIdx.y * slab, r1 = min(M, r0 + slab);
    PhiloxKey key = {};
    if (d.rng) key = philox_key(d.rng);
    float acc[8] = {};
    if (col < N) {
        for (int r = r0 + ty; r < r1; r += kDzThreads / 32) {
            float g[8];
            unpack8(*reinterpret_cast<const uint4 *>(dy + r * lddy + col), g);
            if (d.rng) {
                const uint32_t keep = philox_keep8(key, ((unsigned long long)r * N + col) >> 3, d.drop);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = (keep >> j) & 1u ? g[j] : 0.0f;
            }
            if constexpr (kAct != RR_ACT_NONE) {
                float a[8];
                unpack8(*reinterpret_cast<const uint4 *>(z + r * ldz + col), a);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] *= act_slope<kAct>(a[j]);
            }
            if (dz) *reinterpret_cast<uint4 *>(dz + (size_t)r * N + col) = pack8(g);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += g[j];
        }
    }
    if (!partial) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) red[ty][tx * 8 + j] = acc[j];
    __syncthreads();
    const int c = blockIdx.x * kDzCols + threadIdx.x;
    if (c < N) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kDzThreads / 32; ++w) s += red[w][threadIdx.x];
        partial[(size_t)blockIdx.y * N + c] = s;
    }
}

// db[c] (+)= factor * sum over the slabs, in their order
__global__ void k_dbias(int N, int slabs, const float *__restrict__ partial, float factor, int add, float *db)
{
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c >= N) return;
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < slabs; ++i) s += partial[(size_t)i * N + c];
    db[c] = add ? __fadd_rn(db[c], factor * s) : factor * s;
}

int dz_slabs(int M, int N)
{
    const int cols = (N + kDzCols - 1) / kDzCols;
    int want = (148 * 4 + cols - 1) / cols, most = (M + 31) / 32;
    if (want > most) want = most;
    return want < 1 ? 1 : want;
}

struct LinearScratch {
    Header *hdr;
    __nv_bfloat16 *dz;  // [M,N]
    float *partial;     // [slabs][N]
};

size_t linear_layout(void *ws, int M, int N, LinearScratch *out)
{
    Carver c(ws);
    LinearScratch s;
    s.hdr = c.take<Header>(1);
    s.dz = c.take<__nv_bfloat16>((size_t)M * N);
    s.partial = c.take<float>((size_t)dz_slabs(M, N) * N);
    if (out) *out = s;
    return align_up(c.off, 256);
}

// ---- host ---------------------------------------------------------------------------------------------
// [rows, cols] with `pitch` elements between rows; box: box_cols x box_rows with a swizzle as wide as the box
bool map_2d(CUtensorMap *m, const void *base, long long rows, long long cols, long long pitch, bool f32, int box_cols, int box_rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const int es = f32 ? 4 : 2, bytes = box_cols * es;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(pitch * es)};
    cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return fn(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides,
              box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int device_sms()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return n;
}

struct Operand {
    const void *p;
    long long pitch;
};

template <int TN, bool kAmn, bool kBmn>
rr_status launch_dense(Operand a, Operand b, int M, int N, int K, void *y, long long ldy, void *z, long long ldz, const Epilogue &e,
                       int *status, cudaStream_t st)
{
    CUtensorMap mA, mB, mY, mZ;
    // K-major: [rows, K], box 64 of K x the CTA's rows; MN-major: [K, rows], box 64 rows' columns x 64 of K
    if (!(kAmn ? map_2d(&mA, a.p, K, M, a.pitch, false, 64, 64) : map_2d(&mA, a.p, M, K, a.pitch, false, 64, 128))) return RR_ERR_CUDA;
    if (!(kBmn ? map_2d(&mB, b.p, K, N, b.pitch, false, 64, 64) : map_2d(&mB, b.p, N, K, b.pitch, false, 64, TN / 2))) return RR_ERR_CUDA;
    if (!map_2d(&mY, y, M, N, ldy, e.y_f32, 32, 32)) return RR_ERR_CUDA;
    mZ = mY;
    if (z && !map_2d(&mZ, z, M, N, ldz, false, 32, 32)) return RR_ERR_CUDA;
    DenseParams p;
    p.M = M;
    p.N = N;
    p.m_tiles = (M + 255) / 256;
    p.n_tiles = (N + TN - 1) / TN;
    p.kblocks = (K + 63) / 64;
    p.e = e;
    p.status = status;
    const long long total = (long long)p.m_tiles * p.n_tiles;
    if (total >= (1ll << 30)) return RR_ERR_INVALID_ARG;
    const int pairs = device_sms() / 2;
    if (pairs < 1) return RR_ERR_CUDA;
    if (cudaFuncSetAttribute(k_dense<TN, kAmn, kBmn>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dense_smem<TN>()) != cudaSuccess)
        return RR_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (unsigned)(total < pairs ? total : pairs));
    cfg.blockDim = dim3(kDenseThreads);
    cfg.dynamicSmemBytes = dense_smem<TN>();
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_dense<TN, kAmn, kBmn>, mA, mB, mY, mZ, p) == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

template <int kAct>
void launch_dz(dim3 grid, cudaStream_t st, int M, int N, const void *dy, long long lddy, const void *z, long long ldz, const DropoutParams &d,
               int slab, __nv_bfloat16 *dz, float *partial)
{
    k_dz<kAct><<<grid, kDzThreads, 0, st>>>(M, N, static_cast<const __nv_bfloat16 *>(dy), lddy, static_cast<const __nv_bfloat16 *>(z), ldz, d,
                                            slab, dz, partial);
}

}  // namespace

size_t linear_fwd_workspace() { return kHeaderBytes; }
size_t linear_bwd_workspace(int M, int N) { return linear_layout(nullptr, M, N, nullptr); }

rr_status launch_linear_fwd(const rr_linear_shape &s, const void *x, const void *w, const void *bias, const void *residual, const void *rng,
                            void *y, void *z, void *workspace, cudaStream_t st)
{
    Epilogue e = {};
    e.bias = static_cast<const __nv_bfloat16 *>(bias);
    e.residual = residual;
    e.ldr = s.ldr;
    e.act = s.act;
    e.y_f32 = s.y_dtype == RR_F32;
    e.save_z = z != nullptr;
    e.drop = dropout_params(s.p, rng);
    e.alpha = 1.0f;
    return launch_dense<256, false, false>({x, s.ldx}, {w, s.K}, s.M, s.N, s.K, y, s.ldy, z, s.ldz, e, &static_cast<Header *>(workspace)->status, st);
}

rr_status launch_linear_bwd(const rr_linear_shape &s, const void *dy, const void *x, const void *w, const void *z, const void *rng, void *dx,
                            void *dw, float *dbias, void *workspace, cudaStream_t st)
{
    LinearScratch ws;
    linear_layout(workspace, s.M, s.N, &ws);
    const DropoutParams d = dropout_params(s.p, rng);
    const bool plain = s.act == RR_ACT_NONE && !d.rng;  // dz is dy itself
    const bool want_dz = !plain && (dx || dw);
    if (want_dz || dbias) {
        const int slabs = dz_slabs(s.M, s.N), slab = (s.M + slabs - 1) / slabs;
        const dim3 grid((s.N + kDzCols - 1) / kDzCols, slabs);
        __nv_bfloat16 *out = want_dz ? ws.dz : nullptr;
        float *partial = dbias ? ws.partial : nullptr;
        switch (s.act) {
        case RR_ACT_NONE: launch_dz<RR_ACT_NONE>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        case RR_ACT_RELU: launch_dz<RR_ACT_RELU>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        case RR_ACT_GELU: launch_dz<RR_ACT_GELU>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        case RR_ACT_GELU_TANH: launch_dz<RR_ACT_GELU_TANH>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        default: launch_dz<RR_ACT_SILU>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        }
        if (cudaGetLastError() != cudaSuccess) return RR_ERR_CUDA;
        if (dbias) {
            k_dbias<<<(s.N + 255) / 256, 256, 0, st>>>(s.N, slabs, ws.partial, d.rng ? d.factor : 1.0f, (s.flags & RR_ADD_DW) ? 1 : 0, dbias);
            if (cudaGetLastError() != cudaSuccess) return RR_ERR_CUDA;
        }
    }
    const Operand g = plain ? Operand{dy, s.lddy} : Operand{ws.dz, s.N};
    Epilogue e = {};
    e.alpha = d.rng ? d.factor : 1.0f;
    if (dx) {
        e.y_f32 = s.dx_dtype == RR_F32;
        e.residual = (s.flags & RR_ADD_DX) ? dx : nullptr;
        e.ldr = s.lddx;
        const rr_status rc = launch_dense<256, false, true>(g, {w, s.K}, s.M, s.K, s.N, dx, s.lddx, nullptr, 0, e, &ws.hdr->status, st);
        if (rc) return rc;
    }
    if (dw) {
        e.y_f32 = s.dw_dtype == RR_F32;
        e.residual = (s.flags & RR_ADD_DW) ? dw : nullptr;
        e.ldr = s.K;
        const rr_status rc = launch_dense<256, true, true>(g, {x, s.ldx}, s.N, s.K, s.M, dw, s.K, nullptr, 0, e, &ws.hdr->status, st);
        if (rc) return rc;
    }
    return RR_OK;
}

}  // namespace rr
