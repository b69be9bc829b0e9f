// Dense linear layer with its epilogue, and its gradients (bf16 operands, fp32 accumulation):
//     z = x W^T + b,   y = residual + D(act(z))                       x [M,K], W [N,K], y [M,N]
//     dz = D(dy) act'(z),   dx = dz W,   dW = dz^T x,   db = sum over rows of dz
// D is dropout with the counter-based mask of rr_philox.cuh on the flat index row*N + column: the backward pass
// computes the mask again.  The three products run on one GEMM kernel (k_dense): 256-row tiles on CTA pairs
// (cta_group::2), operands by TMA, two TMEM accumulators so that the epilogue of one tile overlaps the main loop
// of the next.  Operands are read as they lie in memory (K-major or MN-major), nothing is transposed.
#include <cuda.h>
#include <cuda_bf16.h>
#include <stdlib.h>

#include "rr_ffn.cuh"
#include "rr_linear.cuh"
#include "rr_tc.cuh"

namespace rr {

using namespace tc;

namespace {

constexpr int kStageA = 128 * 128;       // this CTA's 128 rows of A, one k-block of 64
constexpr int kPanel = 64 * 128;         // MN-major panel: 64 k-rows x 64 columns
// Warps: 0-2 TMA producers, 3 MMA issuer and TMEM owner, 4-19 epilogue.  Sixteen epilogue warps, four per scheduler: the
// epilogue of a forward tile is some forty instructions an element with long dependent chains (generator,
// activation), as much time as the main loop at K = 1024.
constexpr int kDenseProducers = 3, kDenseMma = 3, kDenseEpi0 = 4, kDenseEpiWarps = 16;
constexpr int kDenseThreads = 32 * (kDenseEpi0 + kDenseEpiWarps);
constexpr int kEpiBytes = 2048;          // staging of one epilogue warp

struct DenseShared {
    alignas(16) float bias[2][256];  // of the tile's columns, one buffer per accumulator
    uint64_t full[12], empty[12], tfull[2], tempty[2];
    uint32_t tmem_base;
    int abort_flag;
};

template <int TN>
__host__ __device__ constexpr int dense_stage_bytes() { return kStageA + TN / 2 * 128; }
template <int TN>
__host__ __device__ constexpr int dense_stages() { return TN == 256 ? 6 : 8; }
template <int TN>
constexpr size_t dense_smem() { return (size_t)dense_stages<TN>() * dense_stage_bytes<TN>() + kDenseEpiWarps * kEpiBytes + sizeof(DenseShared); }

// One product of a launch: C[M,N] = A B, tiles of 256 x TN.  *_mn: the operand is MN-major, its rows are the contraction.
struct DenseJob {
    CUtensorMap mapA, mapB, mapY, mapZ;
    int M, N, m_tiles, n_tiles, kblocks, tiles;
    int a_mn, b_mn;
    Epilogue e;
};
// Up to two products share a launch (dx and dW), the one with the longer contraction first.
struct DenseParams {
    DenseJob job[2];
    int total;
    int *status;
};

// Tile `t` of a job: bands of eight row tiles, inside a band column after column, so that the pairs running together share few
// A and B tiles (74 pairs: 8 x 9) and find them in L2.
struct Tile {
    int job, m, n;
};
// The it-th tile of this pair.  Pairs take every npairs-th item, every second band of npairs items walked backwards, so
// that the pairs which got the longer items of one band get the shorter end of the next.  -1: no more.
__device__ __forceinline__ int item_of(const DenseParams &p, int it, int pair, int npairs)
{
    const int first = it * npairs, n = min(npairs, p.total - first);
    if (n <= 0) return -1;
    const int at = (it & 1) ? npairs - 1 - pair : pair;  // (a last, partial band goes to those it reaches first)
    return at < n ? first + at : -1;
}
__device__ __forceinline__ Tile tile_of(const DenseParams &p, int t)
{
    const int j = t >= p.job[0].tiles ? 1 : 0;
    if (j) t -= p.job[0].tiles;
    const int nt = p.job[j].n_tiles, band = 8 * nt, b = t / band, first = 8 * b, high = min(8, p.job[j].m_tiles - first), r = t - b * band;
    return {j, first + r % high, r / high};
}

template <int TN, bool kForward>
__global__ void __launch_bounds__(kDenseThreads, 1)
k_dense(const __grid_constant__ DenseParams p)
{
    extern __shared__ __align__(1024) uint8_t tiles[];  // (128-byte swizzled tiles start at multiples of 1024)
    constexpr int kNS = dense_stages<TN>(), kStage = dense_stage_bytes<TN>(), kBRows = TN / 2;
    uint8_t *staging = tiles + (size_t)kNS * kStage;
    DenseShared *sh = reinterpret_cast<DenseShared *>(staging + kDenseEpiWarps * kEpiBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank(), pair = (int)(blockIdx.x >> 1), npairs = (int)(gridDim.x >> 1);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kNS; ++s) { mbar_init(&sh->full[s], 1); mbar_init(&sh->empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&sh->tfull[b], 1); mbar_init(&sh->tempty[b], 2 * kDenseEpiWarps); }
        sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&p.job[0].mapA);
        prefetch_map(&p.job[0].mapB);
        prefetch_map(&p.job[0].mapY);
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
    const uint32_t lead_full = map_to_cta(&sh->full[0], 0), lead_tempty = map_to_cta(&sh->tempty[0], 0);
    // Launched as a programmatic dependent: all of the above overlaps the end of the kernel in front; nothing it wrote is
    // read, and nothing written, before this wait.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp < kDenseProducers) {
        // TMA producers: producer j takes the k-blocks j, j + 3, ... of this CTA's stream
        if (lane == 0) {
            uint32_t s = warp % kNS, ph = 0;
            int kb = warp, t;
            bool ok = true;
            for (int it = 0; ok && (t = item_of(p, it, pair, npairs)) >= 0; ++it) {
                const Tile w = tile_of(p, t);
                const DenseJob &j = p.job[w.job];
                const int row = w.m * 256 + 128 * rank, col = w.n * TN + kBRows * rank;  // this CTA's rows of A and of B
                for (; kb < j.kblocks; kb += kDenseProducers) {
                    if (!mbar_wait_brisk(&sh->empty[s], ph ^ 1u, abort_flag, p.status)) { ok = false; break; }
                    uint8_t *a = tiles + (size_t)s * kStage, *b = a + kStageA;
                    const uint32_t bar = lead_full + 8u * s;
                    if (rank == 0) mbar_expect_tx(&sh->full[s], 2u * kStage);  // bytes of both CTAs
                    if (!kForward && j.a_mn) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) tma_tile_2d_pair(a + q * kPanel, &j.mapA, row + 64 * q, kb * 64, bar);
                    } else {
                        tma_tile_2d_pair(a, &j.mapA, kb * 64, row, bar);
                    }
                    if (!kForward && j.b_mn) {
#pragma unroll
                        for (int q = 0; q < kBRows / 64; ++q) tma_tile_2d_pair(b + q * kPanel, &j.mapB, col + 64 * q, kb * 64, bar);
                    } else {
                        tma_tile_2d_pair(b, &j.mapB, kb * 64, col, bar);
                    }
                    s += kDenseProducers;
                    if (s >= (uint32_t)kNS) { s -= kNS; ph ^= 1u; }
                }
                kb -= j.kblocks;
            }
        }
    } else if (warp == kDenseMma) {
        if (rank == 0 && lane == 0) {
            const uint32_t a0 = smem_u32(tiles);
            uint32_t s = 0, ph = 0;
            int t;
            bool ok = true;
            for (int it = 0; ok && (t = item_of(p, it, pair, npairs)) >= 0; ++it) {
                const DenseJob &j = p.job[tile_of(p, t).job];
                const bool amn = !kForward && j.a_mn, bmn = !kForward && j.b_mn;
                const uint32_t idesc = instr_desc(1u, amn ? 1u : 0u, bmn ? 1u : 0u, 256, TN);
                const uint64_t adesc0 = smem_desc(a0, amn ? kPanel : 16, 1024), bdesc0 = smem_desc(a0 + kStageA, bmn ? kPanel : 16, 1024);
                const uint32_t a_step = amn ? 128u : 2u, b_step = bmn ? 128u : 2u;
                const int kblocks = j.kblocks;
                const uint32_t buf = it & 1u;
                if (!mbar_wait_brisk(&sh->tempty[buf], ((it >> 1) & 1u) ^ 1u, abort_flag, p.status)) break;
                fence_after_sync();
                for (int kb = 0; kb < kblocks; ++kb) {
                    if (!mbar_wait_brisk(&sh->full[s], ph, abort_flag, p.status)) { ok = false; break; }
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
        // Epilogue: four warps per TMEM lane quarter take the chunks of 32 columns in turn
        const int eg = (warp - kDenseEpi0) >> 2, q = warp & 3;
        uint8_t *st = staging + (size_t)(eg * 4 + q) * kEpiBytes;
        EpilogueWarp ew;
        if (kForward && p.job[0].e.drop.rng) ew.key = philox_key(p.job[0].e.drop.rng);
        int t;
        for (int it = 0; (t = item_of(p, it, pair, npairs)) >= 0; ++it) {
            const Tile w = tile_of(p, t);
            const DenseJob &j = p.job[w.job];
            const uint32_t buf = it & 1u;
            const int row0 = w.m * 256 + 128 * rank + q * 32;  // first of this warp's 32 rows
            const int col00 = w.n * TN;
            const bool mine = row0 < j.M;
            if (mine) ew.fetch(j.e, row0 + lane, col00 + eg * 32, j.M, j.N);
            // one thread polls, the others sleep at a named barrier: sixteen polling warps would take issue slots from the
            // producers and the MMA issuer (K = 4096, one tile a pair: 41 us instead of 34)
            if (kForward && j.e.bias) {
                // (the barrier below also says that everyone has finished the tile before, whose buffer the next one takes)
                const int c = threadIdx.x - 32 * kDenseEpi0;
                if (c < TN) sh->bias[buf][c] = col00 + c < j.N ? __bfloat162float(j.e.bias[col00 + c]) : 0.0f;
            }
            if (warp == kDenseEpi0 && lane == 0) mbar_wait_brisk(&sh->tfull[buf], (it >> 1) & 1u, abort_flag, p.status);
            __syncwarp();
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kDenseEpiWarps) : "memory");
            if (*abort_flag) break;
            fence_after_sync();
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + buf * TN;
            if (mine) {
#pragma unroll 1
                for (int c = eg * 32; c < TN && col00 + c < j.N; c += 128) {
                    float v[32];
                    tmem_ld32(taddr + c, v);
                    ew.template chunk<kForward>(j.e, v, sh->bias[buf] + c, row0, col00 + c, c + 128 < TN ? col00 + c + 128 : -1, j.M, j.N, lane, st, &j.mapY, &j.mapZ);
                }
            }
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(lead_tempty + 8u * buf);
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

// ---- few tokens ------------------------------------------------------------------------------------------
// With few tokens the layer is one read of the weights.  Here the weights are the 128-row operand and the tokens the
// (narrow) other one, so the tensor cores spend nothing on absent tokens, and the contraction is split over the CTAs
// of a cluster (`split` = 1, 2, 4, 8), which keeps all SMs reading when there are few weight tiles.  The fp32 partial
// tiles meet in shared memory: each CTA of the cluster adds up its share of the features, in the order of the
// ranks (the result repeats bit for bit), and finishes them.  About 110 KB of shared memory a CTA: two share an SM.
//   kWmn: the weights are MN-major (dx = dz W: the features are the columns of W, the contraction runs over its rows).
constexpr int kSlimThreads = 320;  // warp 0: TMA, warp 1: MMA, warps 2-9: TMEM; all of them finish
template <int BN>
__host__ __device__ constexpr int slim_stage_bytes() { return kStageA + BN * 128; }
template <int BN>
__host__ __device__ constexpr int slim_stages() { return BN == 16 ? 6 : BN == 32 ? 5 : BN == 64 ? 4 : 3; }

struct SlimShared {
    uint64_t full[8], empty[8], done;
    uint32_t tmem_base;
    int abort_flag;
};
template <int BN>
constexpr size_t slim_smem() { return (size_t)slim_stages<BN>() * slim_stage_bytes<BN>() + sizeof(SlimShared); }

struct SlimParams {
    int features, tokens;  // columns and rows of y
    int t_tiles;           // tiles of BN tokens
    int kblocks, split;
    Epilogue e;
    void *y;
    long long ldy;
    __nv_bfloat16 *z;
    long long ldz;
    int *status;
};

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

template <int BN, bool kWmn>
__global__ void __launch_bounds__(kSlimThreads, 2)
k_slim(const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapX, const __grid_constant__ SlimParams p)
{
    extern __shared__ __align__(1024) uint8_t tiles[];
    constexpr int kNS = slim_stages<BN>(), kStage = slim_stage_bytes<BN>(), kCols = BN < 32 ? 32 : BN;
    static_assert(BN * 128 * 4 <= kNS * kStage, "the partial tile takes the place of the ring");
    SlimShared *sh = reinterpret_cast<SlimShared *>(tiles + (size_t)kNS * kStage);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = blockIdx.x / p.split, rank = blockIdx.x - tile * p.split;  // (the cluster is `split` consecutive blocks)
    const int f0 = tile / p.t_tiles * 128, t0 = tile % p.t_tiles * BN;
    const int kb0 = (int)((long long)p.kblocks * rank / p.split), kb1 = (int)((long long)p.kblocks * (rank + 1) / p.split);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kNS; ++s) { mbar_init(&sh->full[s], 1); mbar_init(&sh->empty[s], 1); }
        mbar_init(&sh->done, 1);
        sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&mapW);
        prefetch_map(&mapX);
    }
    if (warp == 1) {
        tmem_alloc_one(&sh->tmem_base, kCols);
        tmem_relinquish_one();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem_base = sh->tmem_base;
    volatile int *abort_flag = &sh->abort_flag;
    // Launched as a programmatic dependent: all of the above overlaps the kernel in front; nothing it wrote is read,
    // and nothing written, before this wait.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, ph = 1;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait_brisk(&sh->empty[s], ph, abort_flag, p.status)) break;
                uint8_t *a = tiles + (size_t)s * kStage;
                mbar_expect_tx(&sh->full[s], kStage);
                if (kWmn) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) tma_tile_2d(a + q * kPanel, &mapW, f0 + 64 * q, kb * 64, &sh->full[s]);
                } else {
                    tma_tile_2d(a, &mapW, kb * 64, f0, &sh->full[s]);
                }
                tma_tile_2d(a + kStageA, &mapX, kb * 64, t0, &sh->full[s]);
                if (++s == (uint32_t)kNS) { s = 0; ph ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = instr_desc(1u, kWmn ? 1u : 0u, 0u, 128, BN), a0 = smem_u32(tiles);
            const uint64_t adesc0 = kWmn ? smem_desc(a0, kPanel, 1024) : smem_desc(a0, 16, 1024), bdesc0 = smem_desc(a0 + kStageA, 16, 1024);
            constexpr uint32_t a_step = kWmn ? 128u : 2u;
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait_brisk(&sh->full[s], ph, abort_flag, p.status)) { ok = false; break; }
                fence_after_sync();
                const uint32_t off = s * (uint32_t)(kStage >> 4);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    mma_ss_one(tmem_base, adesc0 + off + a_step * kk, bdesc0 + off + 2u * kk, idesc, (kb != kb0) || kk != 0);
                mma_commit_one(&sh->empty[s]);
                if (++s == (uint32_t)kNS) { s = 0; ph ^= 1u; }
            }
            if (ok) mma_commit_one(&sh->done);
        }
    } else if (warp_wait(&sh->done, 0, abort_flag, p.status)) {
        // every load has landed and every MMA has read its operands: the ring's memory takes the partial tile,
        // [token][128 features]
        fence_after_sync();
        float *part = reinterpret_cast<float *>(tiles);
        const int q = warp & 3, tokens = min(BN, p.tokens - t0);  // (two warps per TMEM lane quarter, alternate columns)
#pragma unroll 1
        for (int c = warp < 6 ? 0 : 16; c < tokens; c += 32) {
            float v[16];
            tmem_ld16(tmem_base + ((uint32_t)(q * 32) << 16) + c, v);
#pragma unroll
            for (int j = 0; j < 16; ++j) part[(c + j) * 128 + q * 32 + lane] = v[j];
        }
        fence_before_sync();
    }
    __syncwarp();
    __syncthreads();
    if (p.split > 1) cluster_sync_all();
    if (!sh->abort_flag) {
        PhiloxKey key = {};
        if (p.e.drop.rng) key = philox_key(p.e.drop.rng);
        // This CTA's share of the tokens, two at a time in a warp: lane l adds up features [4l, 4l+4) of both (512
        // consecutive bytes of the partial tiles per access), then neighbours exchange halves, so that an even lane holds
        // eight features of the first token and an odd one of the second.
        const int tokens = min(BN, p.tokens - t0), first = tokens * rank / p.split, last = tokens * (rank + 1) / p.split;
        const int f = (lane >> 1) * 8;
        for (int t = first + 2 * warp; t < last; t += 2 * (kSlimThreads / 32)) {
            const float *mine = reinterpret_cast<const float *>(tiles) + t * 128 + lane * 4;
            float4 a[8], b[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) {  // all in flight together
                if (s < p.split) {
                    const uint32_t at = map_to_cta(mine, s);
                    a[s] = ld_cluster_f4(at);
                    if (t + 1 < last) b[s] = ld_cluster_f4(at + 512);
                }
            }
            float va[4] = {}, vb[4] = {}, v[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                if (s < p.split) {
                    va[0] += a[s].x; va[1] += a[s].y; va[2] += a[s].z; va[3] += a[s].w;
                    if (t + 1 < last) { vb[0] += b[s].x; vb[1] += b[s].y; vb[2] += b[s].z; vb[3] += b[s].w; }
                }
            }
            const bool odd = lane & 1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float got = __shfl_xor_sync(0xffffffffu, odd ? va[j] : vb[j], 1);
                v[j] = odd ? got : va[j];
                v[j + 4] = odd ? vb[j] : got;
            }
            if (t + odd < last && f0 + f < p.features) finish8(p.e, key, v, t0 + t + odd, f0 + f, p.features, p.y, p.ldy, p.z, p.ldz);
        }
    } else {
        __nanosleep(2000000);  // let copies that are still in flight land
    }
    __syncwarp();
    if (p.split > 1) cluster_sync_all();  // no CTA leaves while another may still read its partial tile
    if (warp == 1) {
        fence_after_sync();
        tmem_dealloc_one(tmem_base, kCols);
    }
}

// ---- dz and its column sums ---------------------------------------------------------------------------
constexpr int kDzThreads = 256, kDzCols = 256;  // 32 threads x 8 columns, 8 rows at a time

// Block (bx, by): columns [256 bx, ...), rows [by*slab, ...).  dz[row, col] = keep dy act'(z) without the dropout factor
// (the GEMMs and the column sums apply it), so that without an activation the rounding to bf16 loses nothing.
// `dz` may be null (only the sums are wanted), `partial` too.  Two rows in flight per thread.
template <int kAct>
__global__ void __launch_bounds__(kDzThreads)
k_dz(int M, int N, const __nv_bfloat16 *__restrict__ dy, long long lddy, const __nv_bfloat16 *__restrict__ z, long long ldz,
     DropoutParams d, int slab, __nv_bfloat16 *__restrict__ dz, float *__restrict__ partial)
{
    constexpr int kRows = kDzThreads / 32, kU = 2;
    __shared__ float red[kRows][kDzCols];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, col = blockIdx.x * kDzCols + tx * 8;
    const int r0 = blockIdx.y * slab, r1 = min(M, r0 + slab);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    PhiloxKey key = {};
    if (d.rng) key = philox_key(d.rng);
    const uint32_t bound = keep_bound(d.drop);
    float acc[8] = {};
    if (col < N) {
        for (int r = r0 + ty; r < r1; r += kU * kRows) {
            uint4 g4[kU], a4[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int row = r + u * kRows;
                g4[u] = a4[u] = make_uint4(0u, 0u, 0u, 0u);
                if (row < r1) {
                    g4[u] = __ldg(reinterpret_cast<const uint4 *>(dy + row * lddy + col));
                    if (kAct != RR_ACT_NONE) a4[u] = __ldg(reinterpret_cast<const uint4 *>(z + row * ldz + col));
                }
            }
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int row = r + u * kRows;
                if (row >= r1) break;
                float g[8], a[8];
                unpack8(g4[u], g);
                if constexpr (kAct != RR_ACT_NONE) {
                    unpack8(a4[u], a);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] *= act_slope<kAct>(a[j]);
                }
                if (d.rng) {
                    uint32_t w[1][4];
                    philox_words<1>(key, ((unsigned long long)row * N + col) >> 3, d.drop, w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = keep(w[0], j, bound) ? g[j] : 0.0f;
                }
                if (dz) *reinterpret_cast<uint4 *>(dz + (size_t)row * N + col) = pack8(g);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += g[j];
            }
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
        for (int w = 0; w < kRows; ++w) s += red[w][threadIdx.x];
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

struct Operand {
    const void *p;
    long long pitch;
};

// An operand of C[M,N] = A B: `mn` = its rows are the contraction
struct Matrix {
    const void *p;
    long long pitch;
    bool mn;
};

bool make_job(DenseJob *j, int TN, Matrix a, Matrix b, int M, int N, int K, void *y, long long ldy, void *z, long long ldz, const Epilogue &e)
{
    // K-major: [rows, K], box 64 of K x the CTA's rows; MN-major: [K, rows], box 64 of the rows x 64 of K
    if (!(a.mn ? map_2d(&j->mapA, a.p, K, M, a.pitch, false, 64, 64) : map_2d(&j->mapA, a.p, M, K, a.pitch, false, 64, 128))) return false;
    if (!(b.mn ? map_2d(&j->mapB, b.p, K, N, b.pitch, false, 64, 64) : map_2d(&j->mapB, b.p, N, K, b.pitch, false, 64, TN / 2))) return false;
    if (!map_2d(&j->mapY, y, M, N, ldy, e.y_f32, e.y_f32 ? 16 : 32, 32)) return false;
    j->mapZ = j->mapY;
    if (z && !map_2d(&j->mapZ, z, M, N, ldz, false, 32, 32)) return false;
    j->M = M;
    j->N = N;
    j->m_tiles = (M + 255) / 256;
    j->n_tiles = (N + TN - 1) / TN;
    j->kblocks = (K + 63) / 64;
    j->a_mn = a.mn;
    j->b_mn = b.mn;
    j->e = e;
    const long long tiles = (long long)j->m_tiles * j->n_tiles;
    if (tiles >= (1ll << 29)) return false;
    j->tiles = (int)tiles;
    return true;
}

template <class... P, class... A>
cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int TN, bool kForward>
rr_status launch_dense(const DenseParams &p, cudaStream_t st)
{
    const int pairs = device_sms() / 2;
    if (pairs < 1) return RR_ERR_CUDA;
    if (cudaFuncSetAttribute(k_dense<TN, kForward>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dense_smem<TN>()) != cudaSuccess)
        return RR_ERR_CUDA;
    return launch_dependent(k_dense<TN, kForward>, dim3(2 * (unsigned)(p.total < pairs ? p.total : pairs)), kDenseThreads, dense_smem<TN>(), 2,
                            st, p) == cudaSuccess
               ? RR_OK : RR_ERR_CUDA;
}

template <int BN, bool kWmn>
rr_status run_slim(const CUtensorMap &mW, const CUtensorMap &mX, const SlimParams &p, int f_tiles, cudaStream_t st)
{
    if (cudaFuncSetAttribute(k_slim<BN, kWmn>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)slim_smem<BN>()) != cudaSuccess)
        return RR_ERR_CUDA;
    return launch_dependent(k_slim<BN, kWmn>, dim3((unsigned)(f_tiles * p.t_tiles * p.split)), kSlimThreads, slim_smem<BN>(), p.split, st, mW, mX,
                            p) == cudaSuccess
               ? RR_OK : RR_ERR_CUDA;
}

int env_int(const char *n, int d) { const char *v = getenv(n); return v ? atoi(v) : d; }
// y [tokens, features] = x [tokens, K] . W; W is [features, K], or [K, features] with kWmn.
template <bool kWmn>
rr_status launch_slim(Operand w, Operand x, int tokens, int features, int K, void *y, long long ldy, void *z, long long ldz, const Epilogue &e,
                      int *status, cudaStream_t st)
{
    CUtensorMap mW, mX;
    const int BN = tokens <= 16 ? 16 : tokens <= 32 ? 32 : tokens <= 64 ? 64 : 128;
    if (!(kWmn ? map_2d(&mW, w.p, K, features, w.pitch, false, 64, 64) : map_2d(&mW, w.p, features, K, w.pitch, false, 64, 128))) return RR_ERR_CUDA;
    if (!map_2d(&mX, x.p, tokens, K, x.pitch, false, 64, BN)) return RR_ERR_CUDA;
    SlimParams p;
    p.features = features;
    p.tokens = tokens;
    p.t_tiles = (tokens + BN - 1) / BN;
    p.kblocks = (K + 63) / 64;
    p.e = e;
    p.y = y;
    p.ldy = ldy;
    p.z = static_cast<__nv_bfloat16 *>(z);
    p.ldz = ldz;
    p.status = status;
    const int f_tiles = (features + 127) / 128;
    const int maxc = env_int("SLIM_CTAS", 296), minkb = env_int("SLIM_KB", 2);
    p.split = 1;
    while (p.split < 8 && (long long)f_tiles * p.t_tiles * p.split * 2 <= maxc && p.kblocks >= 2 * minkb * p.split) p.split *= 2;
    switch (BN) {
    case 16: return run_slim<16, kWmn>(mW, mX, p, f_tiles, st);
    case 32: return run_slim<32, kWmn>(mW, mX, p, f_tiles, st);
    case 64: return run_slim<64, kWmn>(mW, mX, p, f_tiles, st);
    default: return run_slim<128, kWmn>(mW, mX, p, f_tiles, st);
    }
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
    if (s.M <= env_int("SLIM_M", 128))
        return launch_slim<false>({w, s.K}, {x, s.ldx}, s.M, s.N, s.K, y, s.ldy, z, s.ldz, e, &static_cast<Header *>(workspace)->status, st);
    DenseParams p;
    p.status = &static_cast<Header *>(workspace)->status;
    const int TN = env_int("TN", 256);
    if (!make_job(&p.job[0], TN, {x, s.ldx, false}, {w, s.K, false}, s.M, s.N, s.K, y, s.ldy, z, s.ldz, e)) return RR_ERR_CUDA;
    p.total = p.job[0].tiles;
    return TN == 256 ? launch_dense<256, true>(p, st) : launch_dense<128, true>(p, st);
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
    }
    Epilogue ew = {};
    ew.alpha = e.alpha;
    ew.y_f32 = s.dw_dtype == RR_F32;
    ew.residual = (s.flags & RR_ADD_DW) ? dw : nullptr;
    ew.ldr = s.K;
    if (dx && s.M <= env_int("SLIM_M", 128)) {
        const rr_status rc = launch_slim<true>({w, s.K}, {g.p, g.pitch}, s.M, s.K, s.N, dx, s.lddx, nullptr, 0, e, &ws.hdr->status, st);
        if (rc) return rc;
        dx = nullptr;
    }
    if (!dx && !dw) return RR_OK;
    DenseParams p;
    p.status = &ws.hdr->status;
    p.total = 0;
    int n = 0;
    const int TN = env_int("TN", 256);
    for (int first = 0; first < 2; ++first) {  // the longer contraction first
        const bool is_dx = (s.N >= s.M) == (first == 0);
        if (is_dx ? !dx : !dw) continue;
        const bool ok = is_dx ? make_job(&p.job[n], TN, {g.p, g.pitch, false}, {w, s.K, true}, s.M, s.K, s.N, dx, s.lddx, nullptr, 0, e)
                              : make_job(&p.job[n], TN, {g.p, g.pitch, true}, {x, s.ldx, true}, s.N, s.K, s.M, dw, s.K, nullptr, 0, ew);
        if (!ok) return RR_ERR_CUDA;
        p.total += p.job[n++].tiles;
    }
    return TN == 256 ? launch_dense<256, false>(p, st) : launch_dense<128, false>(p, st);
}

}  // namespace rr
