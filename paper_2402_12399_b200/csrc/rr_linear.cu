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
// Warps: 0-2 TMA producers, 3 MMA issuer and TMEM owner, 4-15 epilogue.  The epilogue of a forward tile with everything in it is some
// thirty instructions an element with long dependent chains (generator, activation): at K = 1024 longer than the main loop.  Three warps
// per scheduler hide them best against the registers they leave each other (with twelve, eight, sixteen: 2048 x 4096 x 1024 with a
// residual 21.4, 21.8, 22.8 us, with GELU, dropout and z as well 30.8, 29.8, 31.2; 16384 x 4096 x 128 with everything 129, 140, 140,
// without the residual 111, 127, 105).
constexpr int kDenseProducers = 3, kDenseMma = 3, kDenseEpi0 = 4, kDenseEpiWarps = 12;
constexpr int kDenseThreads = 32 * (kDenseEpi0 + kDenseEpiWarps);
constexpr int kEpiBytes = 2048;          // staging of one epilogue warp
constexpr int kDenseStages = 6;          // of the ring (five cost the main loop 7 to 15 %)

struct DenseShared {
    alignas(16) float bias[kDenseEpiWarps][32];  // of the columns that an epilogue warp is working on
    uint64_t full[kDenseStages], empty[kDenseStages], tfull[2], tempty[2];
    uint32_t tmem_base;
    int abort_flag;
};

constexpr int kTN = 256;                                    // columns of a tile
constexpr int kDenseStage = kStageA + kTN / 2 * 128;        // bytes of one k-block in one CTA
constexpr int kStep = 32 * (kDenseEpiWarps / 4);            // columns between an epilogue warp's chunks
constexpr size_t kDenseSmem = (size_t)kDenseStages * kDenseStage + kDenseEpiWarps * kEpiBytes + sizeof(DenseShared);

// Division of 0 <= n < 2^31 by a divisor that the host knows: a product and a shift (the warps find their tiles with it; the
// compiler's division is some twenty dependent instructions, and there were six a tile in front of every epilogue).  With
// 2^s < d <= 2^(s+1) and mul = ceil(2^(32+s) / d), n mul / 2^(32+s) exceeds n / d by less than n 2^(s+1) / (d 2^(32+s)) <= 1 / d.
struct FastDiv {
    uint32_t d, mul, shift;
    __device__ __forceinline__ int operator()(int n) const { return mul ? (int)(__umulhi((uint32_t)n, mul) >> shift) : n; }
};
FastDiv fast_div(int d)
{
    FastDiv f = {(uint32_t)d, 0u, 0u};
    if (d == 1) return f;
    while ((2u << f.shift) < (uint32_t)d) ++f.shift;
    f.mul = (uint32_t)(((1ull << (32 + f.shift)) + d - 1) / d);
    return f;
}

// One product of a launch: C[M,N] = A B in tiles of 256 x 256.  *_mn: the operand is MN-major, its rows are the contraction.
// With split > 1 the contraction of every tile is cut into that many items, whose results go to consecutive matrices
// of part_rows rows (fp32) for k_combine to add up.
struct DenseJob {
    CUtensorMap mapA, mapB, mapY, mapZ;
    int M, N, m_tiles, n_tiles, kblocks, items;
    int split, part_rows;
    FastDiv by_split, by_band, by_last;  // by split, by the tiles of a band, by the row tiles of the last band
    int a_mn, b_mn;
    Epilogue e;
};
// db[c] (+)= factor * sum over the slabs of k_dz, in their order
struct BiasGrad {
    const float *partial;  // [slabs][n], null: none
    float *db;
    int n, slabs, add;
    float factor;
};
__device__ __forceinline__ void bias_grad(const BiasGrad &b, int c)
{
    if (c >= b.n) return;
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < b.slabs; ++i) s += b.partial[(size_t)i * b.n + c];
    b.db[c] = b.add ? __fadd_rn(b.db[c], b.factor * s) : b.factor * s;
}

// Up to two products share a launch (dx and dW), the one with the longer items first.
struct DenseParams {
    DenseJob job[2];
    int items[2];  // of each job
    int deal, more; // rounds of the first job's items that every pair takes part in, and how many pairs get another one
    int head;      // rounds of the second job's items that only pairs with fewer items of the first take part in
    BiasGrad bias; // (backward)
    int *status;
    unsigned long long tfull_limit_ns;  // of the epilogue's waits for accumulators
};

// The it-th item of this pair (job, index), index -1: no more.  The first job's items are dealt out in rounds; `more` pairs got
// one more than the others.  Of the second job's shorter items the others take `head` rounds alone (about the length
// of a longer one), then all pairs take part.
struct Item {
    int job, at;
};
__device__ __forceinline__ Item item_of(const DenseParams &p, int it, int pair, int npairs)
{
    const int more = p.more, mine = p.deal + (pair < more ? 1 : 0);
    if (it < mine) return {0, it * npairs + pair};
    const int k = it - mine, others = npairs - more;
    int at;
    if (pair < more) at = p.head * others + k * npairs + others + pair;
    else if (k < p.head) at = k * others + pair - more;
    else at = p.head * others + (k - p.head) * npairs + pair - more;
    return {1, at < p.items[1] ? at : -1};
}
// Tile and share of the contraction of an item.  Bands of eight row tiles, inside a band column after column, so that the pairs
// running together share few A and B tiles (74 pairs: 8 x 9) and find them in L2.
struct Work {
    int m, n, part, kb0, kb1;
};
__device__ __forceinline__ Work work_of(const DenseJob &j, int at)
{
    const int t = j.by_split(at), part = at - t * j.split;
    const int b = j.by_band(t), first = 8 * b, r = t - b * (8 * j.n_tiles);
    const bool whole = first + 8 <= j.m_tiles;
    const int n = whole ? r >> 3 : j.by_last(r), high = whole ? 8 : j.m_tiles - first;
    Work w = {first + r - n * high, n, part, 0, j.kblocks};
    if (j.split > 1) {
        w.kb0 = j.by_split(j.kblocks * part);
        w.kb1 = j.by_split(j.kblocks * (part + 1));
    }
    return w;
}

template <bool kForward>
__global__ void __launch_bounds__(kDenseThreads, 1)
k_dense(const __grid_constant__ DenseParams p)
{
    extern __shared__ __align__(1024) uint8_t tiles[];  // (128-byte swizzled tiles start at multiples of 1024)
    constexpr int TN = kTN, kNS = kDenseStages, kStage = kDenseStage, kBRows = TN / 2;
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
    // (all of the above overlaps the end of the kernel in front)
    dependent_start();

    if (warp < kDenseProducers) {
        // TMA producers: producer j takes the k-blocks j, j + 3, ... of this CTA's stream
        if (lane == 0) {
            uint32_t s = warp % kNS, ph = 0;
            int ahead = warp;  // k-blocks from the item's first one to this producer's next
            bool ok = true;
            for (int it = 0; ok; ++it) {
                const Item i = item_of(p, it, pair, npairs);
                if (i.at < 0) break;
                const DenseJob &j = p.job[i.job];
                const Work w = work_of(j, i.at);
                const int row = w.m * 256 + 128 * rank, col = w.n * TN + kBRows * rank;  // this CTA's rows of A and of B
                int kb = w.kb0 + ahead;
                for (; kb < w.kb1; kb += kDenseProducers) {
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
                ahead = kb - w.kb1;
            }
        }
    } else if (warp == kDenseMma) {
        if (rank == 0 && lane == 0) {
            const uint32_t a0 = smem_u32(tiles);
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (int it = 0; ok; ++it) {
                const Item i = item_of(p, it, pair, npairs);
                if (i.at < 0) break;
                const DenseJob &j = p.job[i.job];
                const Work w = work_of(j, i.at);
                const bool amn = !kForward && j.a_mn, bmn = !kForward && j.b_mn;
                const uint32_t idesc = instr_desc(1u, amn ? 1u : 0u, bmn ? 1u : 0u, 256, TN);
                const uint64_t adesc0 = smem_desc(a0, amn ? kPanel : 16, 1024), bdesc0 = smem_desc(a0 + kStageA, bmn ? kPanel : 16, 1024);
                const uint32_t a_step = amn ? 128u : 2u, b_step = bmn ? 128u : 2u;
                const uint32_t buf = it & 1u;
                if (!mbar_wait_brisk(&sh->tempty[buf], ((it >> 1) & 1u) ^ 1u, abort_flag, p.status)) break;
                fence_after_sync();
                for (int kb = w.kb0; kb < w.kb1; ++kb) {
                    if (!mbar_wait_brisk(&sh->full[s], ph, abort_flag, p.status)) { ok = false; break; }
                    fence_after_sync();
                    const uint32_t off = s * (uint32_t)(kStage >> 4);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_ss_pair<false>(tmem_base + buf * TN, adesc0 + off + a_step * kk, bdesc0 + off + b_step * kk, idesc, kb != w.kb0 || kk != 0);
                    mma_commit_pair(&sh->empty[s]);
                    if (++s == (uint32_t)kNS) { s = 0; ph ^= 1u; }
                }
                if (ok) mma_commit_pair(&sh->tfull[buf]);
            }
        }
    } else {
        // Epilogue: three warps per TMEM lane quarter take the chunks of 32 columns in turn
        const int eg = (warp - kDenseEpi0) >> 2, q = warp & 3;
        uint8_t *st = staging + (size_t)(eg * 4 + q) * kEpiBytes;
        EpilogueWarp ew;
        if (!kForward && p.bias.partial)  // before the first tile there is nothing else to do: 32 columns a warp, over all blocks
            for (int c = (warp - kDenseEpi0) * (int)gridDim.x + (int)blockIdx.x; c * 32 < p.bias.n; c += kDenseEpiWarps * (int)gridDim.x)
                bias_grad(p.bias, c * 32 + lane);
        if (kForward && p.job[0].e.drop.rng) ew.key = philox_key(p.job[0].e.drop.rng);
        for (int it = 0;; ++it) {
            const Item i = item_of(p, it, pair, npairs);
            if (i.at < 0) break;
            const DenseJob &j = p.job[i.job];
            const Work w = work_of(j, i.at);
            const uint32_t buf = it & 1u;
            const int row0 = w.m * 256 + 128 * rank + q * 32;  // first of this warp's 32 rows
            const int col00 = w.n * TN;
            const bool mine = row0 < j.M;
            if (mine) ew.template fetch<kForward>(j.e, row0 + lane, col00 + eg * 32, j.M, j.N, lane);
            // Every warp waits for itself, asleep: a dozen warps that poll take issue slots from the producers and the MMA issuer (one tile a
            // pair at K = 4096: 39 us instead of 34), and a barrier in front of the tile holds the early ones back.
            if (!warp_wait_brisk(&sh->tfull[buf], (it >> 1) & 1u, abort_flag, p.status, p.tfull_limit_ns)) break;
            fence_after_sync();
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + buf * TN;
            auto release = [&]() {  // (both CTAs' warps free the accumulator at the leader)
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_peer(lead_tempty + 8u * buf);
            };
            if (!mine || col00 + eg * 32 >= j.N) release();
            if (mine) {
#pragma unroll 1
                for (int c = eg * 32; c < TN && col00 + c < j.N; c += kStep) {
                    float v[32];
                    tmem_ld32(taddr + c, v);
                    if (c + kStep >= TN || col00 + c + kStep >= j.N) release();  // this warp's last look at the accumulator
                    ew.template chunk<kForward>(j.e, v, sh->bias[eg * 4 + q], row0, w.part * j.part_rows, col00 + c, c + kStep < TN ? col00 + c + kStep : -1, j.M,
                                                 j.N, lane, st, &j.mapY, &j.mapZ);
                }
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // (the staging tiles stay until they are read)
    }

    __syncwarp();
    __syncthreads();
    if (sh->abort_flag) __nanosleep(2000000);  // let copies that are still in flight land
    cluster_sync_all();  // neither CTA leaves before what its peer has signalled it has arrived (a release: it waits for that)
    if (warp == kDenseMma) {
        fence_after_sync();
        tmem_dealloc_pair(tmem_base, 2 * TN);
    }
}

// ---- few tokens ------------------------------------------------------------------------------------------
// With few tokens the layer is one read of the weights.  Here the weights are the 128-row operand and the tokens the
// (narrow) other one, so the tensor cores spend nothing on absent tokens, and the contraction is split over the CTAs
// of a cluster (`split` = 1, 2, 4, 8), which keeps all SMs reading when there are few weight tiles.  The fp32 partial
// tiles meet in shared memory: each CTA of the cluster adds up its share of the tokens, in the order of the
// ranks (the result repeats bit for bit), and finishes them.  About 110 KB of shared memory a CTA: two share an SM.
// 1 x 4096 x 4096: 8.3 us, 4.0 TB/s (256 CTAs; the read alone takes 5.1), 9.2 with bias and residual; 37 x 14336 x 4096: 23.2 us, 5.1 TB/s (0.79 of the measured copy
// rate).  With more tokens the parts' way through the SM-to-SM network counts, at about 4 TB/s over all SMs (128 x 4096 x 4096: 13.0 to 13.5 us;
// the library's product 9.6 to 10).
//   kWmn: the weights are MN-major (dx = dz W: the features are the columns of W, the contraction runs over its rows).
constexpr int kSlimTokens = 128;   // up to here always
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
    unsigned long long done_limit_ns;  // of the wait for the partial tile
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
    // (all of the above overlaps the kernel in front)
    dependent_start();

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
    } else if (warp_wait_brisk(&sh->done, 0, abort_flag, p.status, p.done_limit_ns)) {
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
    // No CTA leaves while another may still read its partial tile; every such read has been added up by now, and there is no other
    // traffic between the CTAs, so the barrier need not order anything.
    if (p.split > 1) cluster_sync_relaxed();
    if (warp == 1) {
        fence_after_sync();
        tmem_dealloc_one(tmem_base, kCols);
    }
}

// ---- the parts of a split contraction ------------------------------------------------------------------
// y = finish(sum of `split` fp32 matrices [M,N], part_rows rows apart, in their order)
__global__ void __launch_bounds__(256) k_combine(int M, int N, const float *__restrict__ parts, int split, int part_rows, Epilogue e, void *y, long long ldy)
{
    dependent_start();
    const int groups = N >> 3;
    const long long n = (long long)M * groups, step = (long long)part_rows * N;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const long long row = i / groups;
        const int col = (int)(i - row * groups) * 8;
        const float *src = parts + row * N + col;
        float v[8] = {};
#pragma unroll 4
        for (int s = 0; s < split; ++s, src += step) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(src)), b = __ldg(reinterpret_cast<const float4 *>(src) + 1);
            v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
        }
        finish8(e, PhiloxKey{}, v, row, col, N, y, ldy, nullptr, 0);
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
    dependent_start();
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
            uint32_t w[kU][4];
            if (d.rng) philox_words<kU>(key, ((unsigned long long)r * N + col) >> 3, d.drop, w, (unsigned long long)kRows * N >> 3);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int row = r + u * kRows;
                if (row >= r1) break;
                float g[8], a[8];
                unpack8(g4[u], g);
                if constexpr (kAct != RR_ACT_NONE) {
                    unpack8(a4[u], a);
                    act_slope8<kAct>(a);
#pragma unroll
                    for (int j = 0; j < 8; j += 2) unpack2(mul2(pack2(g[j], g[j + 1]), pack2(a[j], a[j + 1])), g[j], g[j + 1]);
                }
                if (d.rng) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = keep(w[u], j, bound) ? g[j] : 0.0f;
                }
                if (dz) *reinterpret_cast<uint4 *>(dz + (size_t)row * N + col) = pack8(g);
#pragma unroll
                for (int j = 0; j < 8; j += 2) add_pair(acc + j, g[j], g[j + 1]);
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

__global__ void __launch_bounds__(256) k_dbias(const BiasGrad b)
{
    dependent_start();
    bias_grad(b, blockIdx.x * 256 + threadIdx.x);
}

int dz_slabs(int M, int N)
{
    const int cols = (N + kDzCols - 1) / kDzCols;
    int want = (148 * 4 + cols - 1) / cols, most = (M + 31) / 32;
    if (want > most) want = most;
    return want < 1 ? 1 : want;
}

// How the backward products are cut into items: parts of dx's and dW's contractions (0: not on this kernel).
struct Plan {
    int dx, dw;
};
constexpr int kPlanPairs = 74;  // CTA pairs of a B200; fixed, because the workspace depends on it
long long tiles_of(int rows, int cols) { return ((long long)rows + 255) / 256 * ((cols + 255) / 256); }
int kblocks_of(int n) { return (n + 63) / 64; }
// A product with few tiles and a long contraction (dW of many tokens) would keep a few pairs busy long after the others have
// finished: its contraction is cut so that an item takes no longer than an even share of the whole launch (twelve k-blocks at
// least), where that saves more than the sixteen k-blocks' time (5 us) that writing and adding up the parts costs.
Plan plan_bwd(int M, int N, int K, bool dx, bool dw)
{
    const long long tx = dx ? tiles_of(M, K) : 0, tw = dw ? tiles_of(N, K) : 0;
    const int kx = kblocks_of(N), kw = kblocks_of(M);
    long long even = (tx * kx + tw * kw + kPlanPairs - 1) / kPlanPairs;
    if (even < 12) even = 12;
    auto parts = [&](long long tiles, int kb) {
        if (tiles == 0) return 0;
        if (kb <= even + 16) return 1;
        return (int)((kb + even - 1) / even);
    };
    return {parts(tx, kx), parts(tw, kw)};
}
int part_rows(int rows) { return (rows + 255) / 256 * 256; }  // (the last tile's rows may not run into the next part)

struct LinearScratch {
    Header *hdr;
    __nv_bfloat16 *dz;  // [M,N]
    float *partial;     // [slabs][N]
    float *parts_dx, *parts_dw;  // [parts][rows][K]
};

size_t linear_layout(void *ws, int M, int N, int K, LinearScratch *out)
{
    size_t px = 0, pw = 0;
    for (int want = 1; want < 4; ++want) {  // room for whichever gradients a call asks for
        const Plan p = plan_bwd(M, N, K, want & 1, want & 2);
        const size_t x = p.dx > 1 ? (size_t)p.dx * part_rows(M) * K : 0, w = p.dw > 1 ? (size_t)p.dw * part_rows(N) * K : 0;
        if (x > px) px = x;
        if (w > pw) pw = w;
    }
    Carver c(ws);
    LinearScratch s;
    s.hdr = c.take<Header>(1);
    s.dz = c.take<__nv_bfloat16>((size_t)M * N);
    s.partial = c.take<float>((size_t)dz_slabs(M, N) * N);
    s.parts_dx = c.take<float>(px);
    s.parts_dw = c.take<float>(pw);
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

// With split > 1, `parts` takes the results instead of y.
bool make_job(DenseJob *j, Matrix a, Matrix b, int M, int N, int K, void *y, long long ldy, void *z, long long ldz, const Epilogue &e, int split = 1,
              float *parts = nullptr)
{
    // K-major: [rows, K], box 64 of K x the CTA's rows; MN-major: [K, rows], box 64 of the rows x 64 of K
    if (!(a.mn ? map_2d(&j->mapA, a.p, K, M, a.pitch, false, 64, 64) : map_2d(&j->mapA, a.p, M, K, a.pitch, false, 64, 128))) return false;
    if (!(b.mn ? map_2d(&j->mapB, b.p, K, N, b.pitch, false, 64, 64) : map_2d(&j->mapB, b.p, N, K, b.pitch, false, 64, kTN / 2))) return false;
    j->M = M;
    j->N = N;
    j->m_tiles = (M + 255) / 256;
    j->n_tiles = (N + kTN - 1) / kTN;
    j->kblocks = kblocks_of(K);
    j->a_mn = a.mn;
    j->b_mn = b.mn;
    j->e = e;
    j->split = split;
    j->part_rows = part_rows(M);
    if (split > 1) {
        j->e = Epilogue{};
        j->e.alpha = 1.0f;
        j->e.y_f32 = 1;
        if (!map_2d(&j->mapY, parts, (long long)split * j->part_rows, N, N, true, 16, 32)) return false;
    } else {
        if (!map_2d(&j->mapY, y, M, N, ldy, e.y_f32, e.y_f32 ? 16 : 32, 32)) return false;
    }
    j->mapZ = j->mapY;
    if (z && !map_2d(&j->mapZ, z, M, N, ldz, false, 32, 32)) return false;
    const long long items = (long long)j->m_tiles * j->n_tiles * split;
    if (items >= (1ll << 29)) return false;
    j->items = (int)items;
    return true;
}

// The limit of the waits that a test may shorten.
unsigned long long short_wait_ns() { return test_wait_limit_ns() ? test_wait_limit_ns() : kWaitLimitNs; }

// `n` jobs of p, the one with the longer items first
template <bool kForward>
rr_status launch_dense(DenseParams &p, int n, cudaStream_t st)
{
    const int pairs = device_sm_count() / 2;
    if (pairs < 1) return RR_ERR_CUDA;
    p.tfull_limit_ns = short_wait_ns();
    p.items[0] = p.job[0].items;
    p.items[1] = n > 1 ? p.job[1].items : 0;
    for (int k = 0; k < n; ++k) {
        DenseJob &j = p.job[k];
        j.by_split = fast_div(j.split);
        j.by_band = fast_div(8 * j.n_tiles);
        j.by_last = fast_div(j.m_tiles % 8 ? j.m_tiles % 8 : 8);
    }
    p.head = 0;
    if (n > 1) {  // (an item's epilogue and start count as three k-blocks)
        const int a = p.job[0].kblocks / p.job[0].split + 3, b = p.job[1].kblocks / p.job[1].split + 3;
        p.head = (a + b / 2) / b;
    }
    const long long total = (long long)p.items[0] + p.items[1];
    if (cudaFuncSetAttribute(k_dense<kForward>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDenseSmem) != cudaSuccess) return RR_ERR_CUDA;
    const int used = (int)(total < pairs ? total : pairs);
    p.deal = p.items[0] / used;
    p.more = p.items[0] % used;
    return launch_dependent(k_dense<kForward>, dim3(2 * (unsigned)used), kDenseThreads, kDenseSmem, 2, st, p) == cudaSuccess
               ? RR_OK : RR_ERR_CUDA;
}

rr_status launch_combine(int M, int N, const float *parts, int split, const Epilogue &e, void *y, long long ldy, cudaStream_t st)
{
    const long long blocks = ((long long)M * (N / 8) + 255) / 256;
    return launch_dependent(k_combine, dim3((unsigned)(blocks < 148 * 8 ? blocks : 148 * 8)), 256, 0, 1, st, M, N, parts, split, part_rows(M), e, y,
                            ldy) == cudaSuccess
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

// y [tokens, features] = x [tokens, K] . W; W is [features, K], or [K, features] with kWmn.
template <bool kWmn>
rr_status launch_slim(Operand w, Operand x, int tokens, int features, int K, void *y, long long ldy, void *z, long long ldz, const Epilogue &e,
                      int *status, cudaStream_t st)
{
    CUtensorMap mW, mX;
    const int f_tiles = (features + 127) / 128;
    int BN = tokens <= 16 ? 16 : tokens <= 32 ? 32 : tokens <= 64 ? 64 : 128;
    // Where the tiles are few, narrower ones: the weights are read again, from L2, but the clusters join half as much each and there is room
    // to split (128 x 4096 x 4096: 13.0 us with 64 tokens a tile, 15.3 with 128; 512 x 1024 x 4096: 11.1 and 13.9).  The shorter the
    // contraction, the more the join is of the whole, and the narrower (128 x 1024 x 1024: 5.5 us with 32, 5.9 with 64; but 48 x 4096 x
    // 4096: 11.1 and 10.3; 200 x 256 x 256: 3.7 with 16, 4.3 with 32).
    const int least = kblocks_of(K) <= 4 ? 16 : kblocks_of(K) <= 32 ? 32 : 64;
    while (BN > least && (long long)f_tiles * ((tokens + BN / 2 - 1) / (BN / 2)) <= 74) BN /= 2;
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
    p.done_limit_ns = short_wait_ns();
    // two CTAs on every SM, if each is left four k-blocks (1 x 4096 x 4096 with bias and residual: 9.5 us with 256 CTAs, 10.0 with 128; 64 x 4096 x 1024: 6.9 us with
    // 128 CTAs of four k-blocks, 8.1 with 256 of two)
    p.split = 1;
    while (p.split < 8 && (long long)f_tiles * p.t_tiles * p.split * 2 <= 2 * 148 && p.kblocks >= 8 * p.split) p.split *= 2;
    switch (BN) {
    case 16: return run_slim<16, kWmn>(mW, mX, p, f_tiles, st);
    case 32: return run_slim<32, kWmn>(mW, mX, p, f_tiles, st);
    case 64: return run_slim<64, kWmn>(mW, mX, p, f_tiles, st);
    default: return run_slim<128, kWmn>(mW, mX, p, f_tiles, st);
    }
}

template <int kAct>
cudaError_t launch_dz(dim3 grid, cudaStream_t st, int M, int N, const void *dy, long long lddy, const void *z, long long ldz, const DropoutParams &d,
                      int slab, __nv_bfloat16 *dz, float *partial)
{
    return launch_dependent(k_dz<kAct>, grid, kDzThreads, 0, 0, st, M, N, static_cast<const __nv_bfloat16 *>(dy), lddy,
                            static_cast<const __nv_bfloat16 *>(z), ldz, d, slab, dz, partial);
}

}  // namespace

size_t linear_fwd_workspace() { return kHeaderBytes; }
size_t linear_bwd_workspace(int M, int N, int K) { return linear_layout(nullptr, M, N, K, nullptr); }

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
    // Few tokens, or tiles for no more than half of the SMs and a long contraction to split (measured, 256 x 256 tiles against the
    // split kernel: 512 x 4096 x 4096 28.5 against 21.3 us, 1024 x 1024 x 4096 20.9 against 15.4, 512 x 1024 x 1024 11.5 against 8.9; with more tiles or a
    // short contraction the larger tiles win: 768 x 4096 x 4096 28.5 against 35.6, 2048 x 1024 x 1024 10.1 against 10.7).
    const long long tiles = tiles_of(s.M, s.N);
    if (s.M <= kSlimTokens || tiles <= 16 || (tiles <= kPlanPairs / 2 && kblocks_of(s.K) >= 32))
        return launch_slim<false>({w, s.K}, {x, s.ldx}, s.M, s.N, s.K, y, s.ldy, z, s.ldz, e, &static_cast<Header *>(workspace)->status, st);
    DenseParams p;
    p.status = &static_cast<Header *>(workspace)->status;
    p.bias = {};
    if (!make_job(&p.job[0], {x, s.ldx, false}, {w, s.K, false}, s.M, s.N, s.K, y, s.ldy, z, s.ldz, e)) return RR_ERR_CUDA;
    return launch_dense<true>(p, 1, st);
}

rr_status launch_linear_bwd(const rr_linear_shape &s, const void *dy, const void *x, const void *w, const void *z, const void *rng, void *dx,
                            void *dw, float *dbias, void *workspace, cudaStream_t st)
{
    LinearScratch ws;
    linear_layout(workspace, s.M, s.N, s.K, &ws);
    const DropoutParams d = dropout_params(s.p, rng);
    const bool plain = s.act == RR_ACT_NONE && !d.rng;  // dz is dy itself
    const bool want_dz = !plain && (dx || dw);
    if (want_dz || dbias) {
        const int slabs = dz_slabs(s.M, s.N), slab = (s.M + slabs - 1) / slabs;
        const dim3 grid((s.N + kDzCols - 1) / kDzCols, slabs);
        __nv_bfloat16 *out = want_dz ? ws.dz : nullptr;
        float *partial = dbias ? ws.partial : nullptr;
        cudaError_t err;
        switch (s.act) {
        case RR_ACT_NONE: err = launch_dz<RR_ACT_NONE>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        case RR_ACT_RELU: err = launch_dz<RR_ACT_RELU>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        case RR_ACT_GELU: err = launch_dz<RR_ACT_GELU>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        case RR_ACT_GELU_TANH: err = launch_dz<RR_ACT_GELU_TANH>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        default: err = launch_dz<RR_ACT_SILU>(grid, st, s.M, s.N, dy, s.lddy, z, s.ldz, d, slab, out, partial); break;
        }
        if (err != cudaSuccess) return RR_ERR_CUDA;
    }
    BiasGrad bias = {};
    if (dbias) bias = {ws.partial, dbias, s.N, dz_slabs(s.M, s.N), (s.flags & RR_ADD_DW) ? 1 : 0, d.rng ? d.factor : 1.0f};
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
    if (dx && s.M <= kSlimTokens) {
        const rr_status rc = launch_slim<true>({w, s.K}, {g.p, g.pitch}, s.M, s.K, s.N, dx, s.lddx, nullptr, 0, e, &ws.hdr->status, st);
        if (rc) return rc;
        dx = nullptr;
    }
    if (!dx && !dw) {
        if (dbias && launch_dependent(k_dbias, dim3((s.N + 255) / 256), 256, 0, 1, st, bias) != cudaSuccess) return RR_ERR_CUDA;
        return RR_OK;
    }
    const Plan plan = plan_bwd(s.M, s.N, s.K, dx, dw);
    DenseParams p;
    p.status = &ws.hdr->status;
    p.bias = bias;
    int n = 0;
    for (int turn = 0; turn < 2; ++turn) {
        const bool is_dx = ((long long)kblocks_of(s.N) * (plan.dw ? plan.dw : 1) >= (long long)kblocks_of(s.M) * (plan.dx ? plan.dx : 1)) == (turn == 0);
        if (is_dx ? !dx : !dw) continue;
        const bool ok = is_dx ? make_job(&p.job[n], {g.p, g.pitch, false}, {w, s.K, true}, s.M, s.K, s.N, dx, s.lddx, nullptr, 0, e, plan.dx, ws.parts_dx)
                              : make_job(&p.job[n], {g.p, g.pitch, true}, {x, s.ldx, true}, s.N, s.K, s.M, dw, s.K, nullptr, 0, ew, plan.dw, ws.parts_dw);
        if (!ok) return RR_ERR_CUDA;
        ++n;
    }
    rr_status rc = launch_dense<false>(p, n, st);
    if (!rc && plan.dx > 1) rc = launch_combine(s.M, s.K, ws.parts_dx, plan.dx, e, dx, s.lddx, st);
    if (!rc && plan.dw > 1) rc = launch_combine(s.N, s.K, ws.parts_dw, plan.dw, ew, dw, s.K, st);
    return rc;
}

}  // namespace rr
