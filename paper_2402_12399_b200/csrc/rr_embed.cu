// The embedding in front of the first block, and its gradient.
//     y_i = scale table[id_i]          dtable_v = scale (sum over the tokens i with id_i = v, in token order, of dy_i)
// Forward: a gather, bound by HBM.  Backward without floating-point atomics, so that results repeat: the tokens are sorted by id (stably:
// equal ids stay in token order), the sorted tokens are cut into chunks of equal length, a block adds up the rows of a chunk in registers and
// writes the table's row whenever the id changes.  An id that fills a chunk, or lies across its ends, leaves parts in the workspace that a last
// kernel adds up in order: a frequent id costs no more than any other.  Rows that no token names are zeroed by blocks that run beside the
// sort and learn of the named rows from a bitmap of their own.  Sums are fp32.
#include <type_traits>

#include "rr_ffn.cuh"
#include "rr_vec.cuh"

namespace rr {

namespace {

using bf16 = __nv_bfloat16;

constexpr int kEmbThreads = 256;

// ---- forward ------------------------------------------------------------------------------------------------------
struct EmbArgs {
    long long n;
    int V, d;
    int wide;       // 64-bit ids
    float scale;
    long long ld;   // pitch of y or dy
    const void *ids, *in;
    void *out;
    int *status;
};

// id of token i: 0..V-1, or -1 for none (and, with the error latched, for one out of range)
__device__ __forceinline__ int token_id(const EmbArgs &a, long long i)
{
    const long long id = a.wide ? __ldg(static_cast<const long long *>(a.ids) + i) : (long long)__ldg(static_cast<const int *>(a.ids) + i);
    if (id >= 0 && id < a.V) return (int)id;
    if (id != -1) latch_status(a.status, RR_ERR_INVALID_ARG);
    return -1;
}

// A block takes tiles of kTile eights of the result, whatever the width of a row; row and place of each come from one division per
// tile and a product per eight.
constexpr int kEmbUnroll = 4;
template <class TX, class TY, bool kVec>
__global__ void __launch_bounds__(kEmbThreads) k_embed_fwd(const EmbArgs a, int per_row /* eights, or elements */, unsigned long long magic, long long row_step, unsigned at_step)
{
    constexpr int kTile = kEmbThreads * kEmbUnroll;
    dependent_start();
    const long long total = a.n * per_row;
    long long row0 = (long long)blockIdx.x * kTile / per_row;
    unsigned at0 = (unsigned)((long long)blockIdx.x * kTile - row0 * per_row);
    for (long long tile = (long long)blockIdx.x * kTile; tile < total; tile += (long long)gridDim.x * kTile) {
        int id[kEmbUnroll];
        long long row[kEmbUnroll];
        unsigned at[kEmbUnroll];
#pragma unroll
        for (int u = 0; u < kEmbUnroll; ++u) {
            const unsigned l = u * kEmbThreads + threadIdx.x, w = at0 + l;
            const unsigned q = magic ? (unsigned)__umul64hi(w, magic) : w;  // w / per_row (the host says why)
            row[u] = row0 + q;
            at[u] = w - q * per_row;
            id[u] = tile + l < total ? token_id(a, row[u]) : -2;
        }
        if constexpr (kVec) {
            Eight<TX, true> e[kEmbUnroll];
#pragma unroll
            for (int u = 0; u < kEmbUnroll; ++u) {
                e[u].zero();
                if (id[u] >= 0) e[u].template load<kKeep>(static_cast<const TX *>(a.in) + (long long)id[u] * a.d + at[u] * 8, 1, 8);
            }
#pragma unroll
            for (int u = 0; u < kEmbUnroll; ++u) {
                if (id[u] == -2) continue;
                float v[8];
                e[u].get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = id[u] < 0 ? 0.f : v[j] * a.scale;
                Eight<TY, true> o;
                o.set(v);
                o.store(static_cast<TY *>(a.out) + row[u] * a.ld + at[u] * 8, 1, 8);
            }
        } else {
            TX e[kEmbUnroll];
#pragma unroll
            for (int u = 0; u < kEmbUnroll; ++u)
                if (id[u] >= 0) e[u] = static_cast<const TX *>(a.in)[(long long)id[u] * a.d + at[u]];
#pragma unroll
            for (int u = 0; u < kEmbUnroll; ++u)
                if (id[u] != -2) place<kStream>(static_cast<TY *>(a.out) + row[u] * a.ld + at[u], from_f32<TY>(id[u] < 0 ? 0.f : as_f32(e[u]) * a.scale));
        }
        row0 += row_step;  // gridDim tiles on
        at0 += at_step;
        if (at0 >= (unsigned)per_row) {
            at0 -= per_row;
            ++row0;
        }
    }
}

// ---- backward: the sort -------------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigitBits = 8, kDigits = 1 << kDigitBits;
constexpr int kSortMost = 16;                            // tokens a thread of a sorting block holds
constexpr int kSlab = kSortThreads * kSortMost;          // tokens of a sorting block
constexpr int kMapWords = 8192;                          // bitmap of a zeroing block: 2^18 rows at a time

struct SortArgs {
    EmbArgs e;
    int slabs, slab;       // sorting blocks and tokens of each (the last may have fewer)
    int passes;
    int *key, *pos;        // [n] sorted ids (V: no id) and their tokens, slab by slab
    int fill;              // rows without a token are zeroed
    int out_f32;
};

// zeros in `bytes` (512 or more) bytes at p: an even number at an even address
__device__ __forceinline__ void zero_bytes(char *p, long long bytes, int lane)
{
    const int head = (int)(-(uintptr_t)p & 15), tail = (int)((bytes - head) & 15);
    if (2 * lane < head) *reinterpret_cast<uint16_t *>(p + 2 * lane) = 0;
    if (2 * lane < tail) *reinterpret_cast<uint16_t *>(p + bytes - tail + 2 * lane) = 0;
    uint4 *q = reinterpret_cast<uint4 *>(p + head);
    for (long long i = lane; i < (bytes - head) / 16; i += 32) __stcs(q + i, make_uint4(0u, 0u, 0u, 0u));
}

// Rows of this zeroing block that no token names.  A warp zeroes a row at a time; rows shorter than 512 bytes, which would leave lanes idle,
// are shared out by elements.
__device__ void zero_rows(const SortArgs &a, int block, int blocks, uint32_t *map)
{
    const long long V = a.e.V, lo = V * block / blocks, hi = V * (block + 1) / blocks;
    const int es = a.out_f32 ? 4 : 2;
    const long long width = (long long)a.e.d * es;
    char *out = static_cast<char *>(a.e.out);
    for (long long r0 = lo; r0 < hi; r0 += kMapWords * 32) {
        const long long r1 = min(hi, r0 + kMapWords * 32);
        const int words = (int)((r1 - r0 + 31) / 32);
        __syncthreads();
        for (int i = threadIdx.x; i < words; i += kSortThreads) map[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (long long i = threadIdx.x; i < a.e.n; i += kSortThreads) {
            const int id = token_id(a.e, i);
            if (id >= r0 && id < r1) atomicOr(&map[(id - r0) >> 5], 1u << ((id - r0) & 31));
        }
        __syncthreads();
        if (width >= 512) {
            for (long long r = r0 + (threadIdx.x >> 5); r < r1; r += kSortWarps)
                if (!(map[(r - r0) >> 5] >> ((r - r0) & 31) & 1)) zero_bytes(out + r * width, width, threadIdx.x & 31);
        } else {
            const int d = a.e.d;
            const long long elements = (r1 - r0) * d;
            for (long long i = threadIdx.x; i < elements; i += kSortThreads) {
                const int r = (int)(i / d);
                if (map[r >> 5] >> (r & 31) & 1) continue;
                if (es == 4) reinterpret_cast<float *>(out)[r0 * d + i] = 0.f;
                else reinterpret_cast<uint16_t *>(out)[r0 * d + i] = 0;
            }
        }
    }
}

// Stable sort of a slab by id, least significant digit first.  A thread holds K consecutive-by-warp tokens (token w*32*K + k*32 + lane of
// the slab): in a pass every warp counts its tokens digit by digit in its own column of the table (`__match_any_sync` gives a token its
// place among the equal digits of its warp), the table is scanned digit by digit and warp by warp, and the tokens move in shared memory.
// Blocks behind the sorting ones zero the rows that nobody names.
template <int K>
__global__ void __launch_bounds__(kSortThreads) k_embed_sort(const SortArgs a)
{
    extern __shared__ __align__(16) uint32_t shared[];
    dependent_start();
    if ((int)blockIdx.x >= a.slabs) {
        zero_rows(a, blockIdx.x - a.slabs, gridDim.x - a.slabs, shared);
        return;
    }
    uint32_t *const count = shared;                        // [kDigits][kSortWarps + 1]
    uint32_t *const sk = count + kDigits * (kSortWarps + 1);  // [1024 K]
    uint16_t *const sp = reinterpret_cast<uint16_t *>(sk + kSortThreads * K);
    __shared__ uint32_t warp_total[kSortWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long base = (long long)blockIdx.x * a.slab;
    const int n = (int)min((long long)a.slab, a.e.n - base);
    uint32_t key[K];
    uint32_t pos[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = warp * 32 * K + k * 32 + lane;
        int id = -1;
        if (i < n) id = token_id(a.e, base + i);
        key[k] = i >= n ? 0xffffffffu : id < 0 ? (uint32_t)a.e.V : (uint32_t)id;  // (places behind the end stay behind all others)
        pos[k] = i;
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * kDigitBits;
        for (int i = threadIdx.x; i < kDigits * (kSortWarps + 1); i += kSortThreads) count[i] = 0;
        __syncthreads();
        uint32_t rank[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t digit = key[k] >> shift & (kDigits - 1);
            const uint32_t same = __match_any_sync(0xffffffffu, digit), below = same & ((1u << lane) - 1);
            uint32_t *c = &count[digit * (kSortWarps + 1) + warp];
            const uint32_t before = *c;
            __syncwarp();
            if (below == 0) *c = before + __popc(same);
            __syncwarp();
            rank[k] = before + __popc(below);
        }
        __syncthreads();
        // exclusive scan over (digit, warp): thread t owns eight warps of digit t / 4
        uint32_t v[8], sum = 0;
        uint32_t *c = &count[(threadIdx.x >> 2) * (kSortWarps + 1) + (threadIdx.x & 3) * 8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = sum;
            sum += c[j];
        }
        uint32_t inclusive = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, inclusive, o);
            if (lane >= o) inclusive += up;
        }
        if (lane == 31) warp_total[warp] = inclusive;
        __syncthreads();
        uint32_t before = lane < warp ? warp_total[lane] : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
        before += inclusive - sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = before + v[j];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t to = rank[k] + count[(key[k] >> shift & (kDigits - 1)) * (kSortWarps + 1) + warp];
            sk[to] = key[k];
            sp[to] = (uint16_t)pos[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = warp * 32 * K + k * 32 + lane;
            key[k] = sk[i];
            pos[k] = sp[i];
        }
        // (the next pass writes to sk and sp behind two barriers)
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = warp * 32 * K + k * 32 + lane;
        if (i < n) {
            a.key[base + i] = (int)key[k];
            a.pos[base + i] = (int)(base + pos[k]);
        }
    }
}

// Sorted slabs into one order: a token's place is the number of tokens in front of it in every slab (equal ids: earlier slabs only).
__global__ void __launch_bounds__(kEmbThreads) k_embed_merge(long long n, int slabs, int slab, const int *__restrict__ key, const int *__restrict__ pos, int *out_key,
                                                             int *out_pos)
{
    dependent_start();
    const long long i = (long long)blockIdx.x * kEmbThreads + threadIdx.x;
    if (i >= n) return;
    const int mine = (int)(i / slab), id = __ldg(key + i);
    long long to = i - (long long)mine * slab;
    for (int s = 0; s < slabs; ++s) {
        if (s == mine) continue;
        const long long base = (long long)s * slab;
        int lo = 0, hi = (int)min((long long)slab, n - base);
        while (lo < hi) {  // tokens of slab s below id, or in earlier slabs not above it
            const int mid = (lo + hi) >> 1, k = __ldg(key + base + mid);
            if (k < id || (k == id && s < mine)) lo = mid + 1;
            else hi = mid;
        }
        to += lo;
    }
    out_key[to] = id;
    out_pos[to] = __ldg(pos + i);
}

// ---- backward: the sums -------------------------------------------------------------------------------------------
struct SumArgs {
    EmbArgs e;
    const int *key, *pos;  // [n] sorted
    float *part;           // [chunks][2][d]: the first and the last run of a chunk where they go on beyond it
    long long chunks;
    int add;
};

constexpr int kChunk = 32;    // sorted tokens of a chunk
constexpr int kAhead = 8;     // rows in flight

template <class TO, bool kVec>
__device__ __forceinline__ void write_row(const SumArgs &a, int id, int at, int step, float (&v)[8])
{
    TO *p = static_cast<TO *>(a.e.out) + (long long)id * a.e.d + at;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= a.e.scale;
    if (a.add) {
        Eight<TO, kVec> old;
        old.load(p, step, a.e.d - at);
        float o[8];
        old.get(o);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += o[j];
    }
    Eight<TO, kVec> e;
    e.set(v);
    e.store(p, step, a.e.d - at);
}
template <bool kVec>
__device__ __forceinline__ void write_part(const SumArgs &a, long long chunk, int which, int at, int step, const float (&v)[8])
{
    Eight<float, kVec> e;
    e.set(v);
    e.template store<kKeep>(a.part + (chunk * 2 + which) * a.e.d + at, step, a.e.d - at);
}

// One chunk of sorted tokens and 8 blockDim columns
template <class TY, class TO, bool kVec>
__global__ void __launch_bounds__(kEmbThreads) k_embed_sum(const SumArgs a)
{
    __shared__ int sk[kChunk + 2], sp[kChunk];
    dependent_start();
    const long long chunk = blockIdx.x, i0 = chunk * kChunk;
    const int n = (int)min((long long)kChunk, a.e.n - i0);
    for (int i = threadIdx.x; i < kChunk + 2; i += blockDim.x) {
        const long long at = i0 + i - 1;
        sk[i] = at >= 0 && at < a.e.n && i <= n + 1 ? __ldg(a.key + at) : -1;
        if (i < n) sp[i] = __ldg(a.pos + i0 + i);
    }
    __syncthreads();
    const int step = kVec ? 1 : blockDim.x, at = (kVec ? (blockIdx.y * blockDim.x + threadIdx.x) * 8 : blockIdx.y * blockDim.x * 8 + threadIdx.x);
    if (at >= a.e.d) return;
    const TY *dy = static_cast<const TY *>(a.e.in) + at;
    float acc[8] = {};
    bool started = sk[0] != sk[1];  // the run of ids at hand began in this chunk
    for (int i = 0; i < n; i += kAhead) {
        if (sk[i + 1] == a.e.V) return;  // (tokens without an id are the last)
        Eight<TY, kVec> row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < n && sk[i + u + 1] != a.e.V) row[u].load(dy + (long long)sp[i + u] * a.e.ld, step, a.e.d - at);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= n) break;
            const int id = sk[i + u + 1];
            if (id == a.e.V) return;
            float v[8];
            row[u].get(v);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += v[j];
            const bool ends = sk[i + u + 2] != id;
            if (!ends && i + u + 1 < n) continue;
            if (started && ends) write_row<TO, kVec>(a, id, at, step, acc);
            else write_part<kVec>(a, chunk, started ? 1 : 0, at, step, acc);
            started = true;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        }
    }
}

// Runs across chunks: the block of the chunk in which one begins adds up its parts, every kJoin-th by one row of threads, those in order.
constexpr int kJoin = 8, kJoinCols = 32;
template <class TO, bool kVec>
__global__ void __launch_bounds__(kJoin *kJoinCols) k_embed_join(const SumArgs a)
{
    __shared__ float red[kJoin][8][kJoinCols + 1];
    dependent_start();
    const long long chunk = blockIdx.x, last = (chunk + 1) * kChunk - 1;  // (the last chunk is not in the grid)
    const int id = __ldg(a.key + last);
    if (id == a.e.V || __ldg(a.key + last + 1) != id) return;             // no run goes on from this chunk
    if (__ldg(a.key + chunk * kChunk) == id && chunk > 0 && __ldg(a.key + chunk * kChunk - 1) == id) return;  // it began earlier
    long long lo = last + 1, hi = a.e.n;  // end of the run
    while (lo < hi) {
        const long long mid = (lo + hi) >> 1;
        if (__ldg(a.key + mid) == id) lo = mid + 1;
        else hi = mid;
    }
    const long long end = (lo - 1) / kChunk;  // its last chunk
    const int c = threadIdx.x % kJoinCols, q = threadIdx.x / kJoinCols;
    const int step = kVec ? 1 : kJoinCols;
    for (int tile = blockIdx.y * kJoinCols * 8; tile < a.e.d; tile += gridDim.y * kJoinCols * 8) {
        const int at = tile + (kVec ? c * 8 : c);
        float acc[8] = {};
        if (at < a.e.d) {
#pragma unroll 4
            for (long long k = chunk + q; k <= end; k += kJoin) {
                Eight<float, kVec> e;
                e.template load<kKeep>(a.part + (k * 2 + (k == chunk ? 1 : 0)) * a.e.d + at, step, a.e.d - at);
                float v[8];
                e.get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += v[j];
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) red[q][j][c] = acc[j];
        __syncthreads();
        if (q || at >= a.e.d) continue;
#pragma unroll
        for (int i = 1; i < kJoin; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += red[i][j][c];
        write_row<TO, kVec>(a, id, at, step, acc);
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------
template <class T>
struct Type {
    using type = T;
};
template <class F>
cudaError_t with_type(int dtype, F f) { return dtype == RR_F32 ? f(Type<float>{}) : f(Type<bf16>{}); }
template <class F>
cudaError_t with_vec(bool vec, F f) { return vec ? f(std::integral_constant<bool, true>{}) : f(std::integral_constant<bool, false>{}); }

struct BwdLayout {
    Header *hdr;
    int *key, *pos, *key2, *pos2;
    float *part;
    long long chunks;
    int slabs, slab;
};
size_t bwd_layout(void *ws, long long n, int d, BwdLayout *out)
{
    BwdLayout l;
    l.chunks = (n + kChunk - 1) / kChunk;
    l.slabs = (int)((n + kSlab - 1) / kSlab);
    l.slab = l.slabs ? (int)((n + l.slabs - 1) / l.slabs) : 0;
    Carver c(ws);
    l.hdr = c.take<Header>(1);
    l.key = c.take<int>(n);
    l.pos = c.take<int>(n);
    l.key2 = l.slabs > 1 ? c.take<int>(n) : l.key;
    l.pos2 = l.slabs > 1 ? c.take<int>(n) : l.pos;
    l.part = c.take<float>(l.chunks > 1 ? (size_t)l.chunks * 2 * d : 0);
    if (out) *out = l;
    return align_up(c.off, 256);
}

EmbArgs emb_args(const rr_embed_shape &s, const void *ids, const void *in, void *out, void *ws)
{
    EmbArgs a;
    a.n = s.n;
    a.V = s.V;
    a.d = s.d;
    a.wide = s.wide_ids != 0;
    a.scale = s.scale;
    a.ld = s.ldy;
    a.ids = ids;
    a.in = in;
    a.out = out;
    a.status = static_cast<int *>(ws);
    return a;
}

template <int K>
cudaError_t launch_sort(const SortArgs &a, int blocks, cudaStream_t st)
{
    const size_t tables = (size_t)kDigits * (kSortWarps + 1) * 4 + (size_t)kSortThreads * K * 6, map = (size_t)kMapWords * 4;
    const size_t smem = tables > map ? tables : map;
    const cudaError_t err = cudaFuncSetAttribute(k_embed_sort<K>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
    return launch_dependent(k_embed_sort<K>, dim3(blocks), kSortThreads, smem, 1, st, a);
}

}  // namespace

size_t embed_bwd_workspace(long long n, int d) { return bwd_layout(nullptr, n, d, nullptr); }

rr_status launch_embed_fwd(const rr_embed_shape &s, const void *ids, const void *table, void *y, void *ws, cudaStream_t st)
{
    const EmbArgs a = emb_args(s, ids, table, y, ws);
    const bool vec = s.d % 8 == 0 && s.ldy % (s.y_dtype == RR_F32 ? 4 : 8) == 0;
    const int per_row = vec ? s.d / 8 : s.d, sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    // w / per_row is the high word of w * magic, magic = ceil(2^64 / per_row): what the rounding up adds to the quotient is below
    // w / 2^64 < 2^-32, less than the 1 / per_row that would be missing to the next whole number.  (A divisor of one has no such factor.)
    const unsigned long long magic = per_row == 1 ? 0 : ~0ull / (unsigned)per_row + 1;
    const long long tiles = (s.n * per_row + kEmbThreads * kEmbUnroll - 1) / (kEmbThreads * kEmbUnroll), most = (long long)sms * 8;
    const dim3 grid((unsigned)(tiles < most ? tiles : most));
    const long long step = (long long)grid.x * kEmbThreads * kEmbUnroll, row_step = step / per_row;
    const unsigned at_step = (unsigned)(step % per_row);
    const cudaError_t err = with_type(s.table_dtype, [&](auto tx) {
        return with_type(s.y_dtype, [&](auto ty) {
            return with_vec(vec, [&](auto v) {
                return launch_dependent(k_embed_fwd<typename decltype(tx)::type, typename decltype(ty)::type, v()>, grid, kEmbThreads, 0, 1, st, a, per_row, magic, row_step, at_step);
            });
        });
    });
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

rr_status launch_embed_bwd(const rr_embed_shape &s, const void *ids, const void *dy, void *dtable, void *ws, cudaStream_t st)
{
    const int sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    BwdLayout l;
    bwd_layout(ws, s.n, s.d, &l);
    const bool add = (s.flags & RR_ADD_DW) != 0;
    SortArgs a;
    a.e = emb_args(s, ids, dy, dtable, ws);
    a.slabs = l.slabs;
    a.slab = l.slab;
    a.passes = 1;
    while (a.passes < 4 && ((unsigned long long)s.V >> (kDigitBits * a.passes)) != 0) ++a.passes;  // (V itself is a key)
    a.key = l.key;
    a.pos = l.pos;
    a.fill = !add;
    a.out_f32 = s.table_dtype == RR_F32;
    int fillers = 0;
    if (!add) {  // zeroing blocks: one an SM, but none with less than 64 KB
        const long long bytes = (long long)s.V * s.d * (a.out_f32 ? 4 : 2), want = (bytes + 65535) / 65536;
        const int most = sms - l.slabs > sms / 4 ? sms - l.slabs : sms / 4;  // (one block an SM: all at once)
        fillers = (int)(want < most ? want : most);
        if (fillers > s.V) fillers = s.V;
    }
    cudaError_t err = l.slab <= kSortThreads * 2 ? launch_sort<2>(a, l.slabs + fillers, st)
                      : l.slab <= kSortThreads * 4 ? launch_sort<4>(a, l.slabs + fillers, st)
                                                   : launch_sort<kSortMost>(a, l.slabs + fillers, st);
    if (err == cudaSuccess && l.slabs > 1)
        err = launch_dependent(k_embed_merge, dim3((unsigned)((s.n + kEmbThreads - 1) / kEmbThreads)), kEmbThreads, 0, 1, st, (long long)s.n, l.slabs, l.slab,
                               (const int *)l.key, (const int *)l.pos, l.key2, l.pos2);
    if (err != cudaSuccess) return RR_ERR_CUDA;
    SumArgs b;
    b.e = a.e;
    b.key = l.key2;
    b.pos = l.pos2;
    b.part = l.part;
    b.chunks = l.chunks;
    b.add = add;
    const bool vec = s.d % 8 == 0 && s.ldy % (s.y_dtype == RR_F32 ? 4 : 8) == 0;
    int threads = 32;
    while (threads < kEmbThreads && threads * 8 < s.d) threads <<= 1;
    const dim3 grid((unsigned)l.chunks, (unsigned)((s.d + threads * 8 - 1) / (threads * 8)));
    err = with_type(s.y_dtype, [&](auto ty) {
        return with_type(s.table_dtype, [&](auto to) {
            return with_vec(vec, [&](auto v) {
                return launch_dependent(k_embed_sum<typename decltype(ty)::type, typename decltype(to)::type, v()>, grid, threads, 0, 1, st, b);
            });
        });
    });
    if (err == cudaSuccess && l.chunks > 1) {
        const int tiles = (s.d + kJoinCols * 8 - 1) / (kJoinCols * 8);
        err = with_type(s.table_dtype, [&](auto to) {
            return with_vec(vec, [&](auto v) {
                return launch_dependent(k_embed_join<typename decltype(to)::type, v()>, dim3((unsigned)(l.chunks - 1), tiles < 16 ? tiles : 16), kJoin * kJoinCols, 0, 1, st, b);
            });
        });
    }
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

}  // namespace rr
