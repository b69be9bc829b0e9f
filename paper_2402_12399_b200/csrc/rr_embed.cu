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

// A block takes tiles of kTile units of the result (kN elements each), whatever the width of a row; row and place of a unit come from a
// product, and those of the next tile from those of the last.
constexpr int kEmbUnroll = 4;
template <class TX, class TY, int kN>
__global__ void __launch_bounds__(kEmbThreads) k_embed_fwd(const EmbArgs a, int per_row, unsigned long long magic, long long row_step, unsigned at_step)
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
        Unit<TX, kN> e[kEmbUnroll];
#pragma unroll
        for (int u = 0; u < kEmbUnroll; ++u) {
            e[u].raw = {};
            if (id[u] >= 0) e[u].template load<kKeep>(static_cast<const TX *>(a.in) + (long long)id[u] * a.d + (long long)at[u] * kN);
        }
#pragma unroll
        for (int u = 0; u < kEmbUnroll; ++u) {
            if (id[u] == -2) continue;
            Unit<TY, kN> o;
            scaled<kN>(e[u], o, a.scale);
            if (id[u] < 0) o.raw = {};  // (not -0)
            o.template store<kStream>(static_cast<TY *>(a.out) + row[u] * a.ld + (long long)at[u] * kN);
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
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits; // at most
constexpr int kSortMost = 16;                            // tokens a thread of a sorting block holds
constexpr int kSlab = kSortThreads * kSortMost;          // tokens of a sorting block
constexpr int kMapWords = 8192;                          // bitmap of a zeroing block: 2^18 rows at a time

struct SortArgs {
    EmbArgs e;
    int slabs, slab;       // sorting blocks and tokens of each (the last may have fewer)
    int passes, bits;      // digits, and bits of each
    int *key, *pos;        // [n] sorted ids (V: no id) and their tokens, slab by slab
    int *runs;             // counter of the long runs (k_embed_sum), set to zero here
    int out_f32;
};

// Rows of this zeroing block that no token names.  `lanes` lanes of a warp zero a row, as many as it has 16-byte pieces.
__device__ void zero_rows(const SortArgs &a, int block, int blocks, uint32_t *map)
{
    const long long V = a.e.V, lo = V * block / blocks, hi = V * (block + 1) / blocks;
    const long long width = (long long)a.e.d * (a.out_f32 ? 4 : 2);
    int lanes = 1;
    while (lanes < 32 && lanes * 16 < width) lanes <<= 1;
    const int lane = threadIdx.x & (lanes - 1), step = kSortThreads / lanes;
    constexpr int kAtOnce = 16;
    for (long long r0 = lo; r0 < hi; r0 += kMapWords * 32) {
        const long long r1 = min(hi, r0 + kMapWords * 32);
        const int words = (int)((r1 - r0 + 31) / 32);
        __syncthreads();
        for (int i = threadIdx.x; i < words; i += kSortThreads) map[i] = 0;
        __syncthreads();
        for (long long i0 = threadIdx.x; i0 < a.e.n; i0 += kAtOnce * kSortThreads) {
            int id[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) id[u] = i0 + u * kSortThreads < a.e.n ? token_id(a.e, i0 + u * kSortThreads) : -1;
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
                if (id[u] >= r0 && id[u] < r1) atomicOr(&map[(id[u] - r0) >> 5], 1u << ((id[u] - r0) & 31));
        }
        __syncthreads();
        for (long long r = r0 + threadIdx.x / lanes; r < r1; r += step) {
            if (map[(r - r0) >> 5] >> ((r - r0) & 31) & 1) continue;
            char *p = static_cast<char *>(a.e.out) + r * width;  // (an even address, an even number of bytes)
            const int head = (int)min(width, (long long)(-(uintptr_t)p & 15)), tail = (int)((width - head) & 15);
            for (int i = 2 * lane; i < head; i += 2 * lanes) *reinterpret_cast<uint16_t *>(p + i) = 0;
            for (int i = 2 * lane; i < tail; i += 2 * lanes) *reinterpret_cast<uint16_t *>(p + width - tail + i) = 0;
            uint4 *q = reinterpret_cast<uint4 *>(p + head);
            for (long long i = lane; i < (width - head) / 16; i += lanes) __stcs(q + i, make_uint4(0u, 0u, 0u, 0u));
        }
    }
}

// lanes of the warp with the same digit (`bits` bits) as this one
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, int bits)
{
    uint32_t same = 0xffffffffu;
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        if (b >= bits) break;
        const uint32_t with = __ballot_sync(0xffffffffu, digit >> b & 1);
        same &= digit >> b & 1 ? with : ~with;
    }
    return same;
}

// Stable sort of a slab by id, least significant digit first.  A thread holds K tokens (token w 32 K + k 32 + lane of the slab): in a
// pass every warp counts its tokens digit by digit in its own column of a table, which gives a token its place among the equal digits of the
// warp; the table is scanned digit by digit and warp by warp, and the tokens move in shared memory.
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
    constexpr int kRow = kSortWarps + 1;                   // (a column of the table in every bank)
    uint32_t *const count = shared;                        // [kDigits][kRow]
    uint32_t *const total = count + kDigits * kRow;        // [kDigits] tokens of a digit, then those of lower ones
    uint32_t *const sk = total + kDigits;                  // [1024 K]
    uint16_t *const sp = reinterpret_cast<uint16_t *>(sk + kSortThreads * K);
    __shared__ uint32_t warp_total[kSortWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, digits = 1 << a.bits;
    const long long base = (long long)blockIdx.x * a.slab;
    const int n = (int)min((long long)a.slab, a.e.n - base);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.runs = 0;
    uint32_t key[K], pos[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = warp * 32 * K + k * 32 + lane;
        int id = -1;
        if (i < n) id = token_id(a.e, base + i);
        key[k] = i >= n ? 0xffffffffu : id < 0 ? (uint32_t)a.e.V : (uint32_t)id;  // (places behind the end stay behind all others)
        pos[k] = i;
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.bits;
        for (int i = threadIdx.x; i < digits * kRow; i += kSortThreads) count[i] = 0;
        __syncthreads();
        uint32_t rank[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t digit = key[k] >> shift & (digits - 1), same = same_digit(digit, a.bits), below = same & ((1u << lane) - 1);
            uint32_t *c = &count[digit * kRow + warp];
            const uint32_t before = *c;
            __syncwarp();
            if (below == 0) *c = before + __popc(same);
            __syncwarp();
            rank[k] = before + __popc(below);
        }
        __syncthreads();
        for (int d = warp; d < digits; d += kSortWarps) {  // a digit's tokens in the warps before
            const uint32_t own = count[d * kRow + lane];
            uint32_t sum = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += up;
            }
            count[d * kRow + lane] = sum - own;
            if (lane == 31) total[d] = sum;
        }
        __syncthreads();
        uint32_t own = 0, sum = 0;  // lower digits' tokens
        if ((int)threadIdx.x < digits) sum = own = total[threadIdx.x];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 31) warp_total[warp] = sum;
        __syncthreads();
        if (warp < digits / 32 || warp == 0) {
            uint32_t before = lane < warp ? warp_total[lane] : 0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
            if ((int)threadIdx.x < digits) total[threadIdx.x] = before + sum - own;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t digit = key[k] >> shift & (digits - 1), to = rank[k] + total[digit] + count[digit * kRow + warp];
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
        // (the next pass writes to sk and sp behind further barriers)
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
// Four slabs are searched side by side.
__global__ void __launch_bounds__(kEmbThreads) k_embed_merge(long long n, int slabs, int slab, const int *__restrict__ key, const int *__restrict__ pos, int *out_key,
                                                             int *out_pos)
{
    constexpr int kSide = 4;
    dependent_start();
    const long long i = (long long)blockIdx.x * kEmbThreads + threadIdx.x;
    if (i >= n) return;
    const int mine = (int)(i / slab), id = __ldg(key + i);
    const int token = __ldg(pos + i);
    long long to = i - (long long)mine * slab;
    int steps = 1;
    while (1 << steps <= slab) ++steps;
    for (int s0 = 0; s0 < slabs; s0 += kSide) {
        int lo[kSide], hi[kSide];
#pragma unroll
        for (int u = 0; u < kSide; ++u) {
            const int s = s0 + u;
            lo[u] = 0;
            hi[u] = s < slabs && s != mine ? (int)min((long long)slab, n - (long long)s * slab) : 0;
        }
        for (int step = 0; step < steps; ++step) {
#pragma unroll
            for (int u = 0; u < kSide; ++u) {  // tokens of slab s below id, or in earlier slabs not above it
                if (lo[u] >= hi[u]) continue;
                const int mid = (lo[u] + hi[u]) >> 1, k = __ldg(key + (long long)(s0 + u) * slab + mid);
                if (k < id || (k == id && s0 + u < mine)) lo[u] = mid + 1;
                else hi[u] = mid;
            }
        }
#pragma unroll
        for (int u = 0; u < kSide; ++u) to += lo[u];
    }
    out_key[to] = id;
    out_pos[to] = token;
}

// ---- backward: the sums -------------------------------------------------------------------------------------------
// A run is all the tokens of one id.  A block takes a chunk of sorted tokens, and of the runs that begin in it those of up to kLong tokens
// to their end: most runs are short, and need no second look.  Of a longer run every chunk adds up its own piece (the first piece is part 1
// of its chunk, every other the part 0), and k_embed_join adds up the pieces in order.
struct SumArgs {
    EmbArgs e;
    const int *key, *pos;  // [n] sorted
    float *part;           // [chunks][2][d]
    int *runs, *list;      // long runs: how many, and the chunks in which they begin (in any order)
    int add;
};

constexpr int kChunk = 32;             // sorted tokens of a chunk
constexpr int kLong = 64;
constexpr int kReach = kChunk + kLong; // tokens that a block may have to look at from the start of its chunk on
constexpr int kAhead = 8;              // rows in flight

template <class TO, Layout L>
__device__ __forceinline__ void write_row(const SumArgs &a, int id, int at, int step, f32x2 (&v)[4])
{
    TO *p = static_cast<TO *>(a.e.out) + (long long)id * a.e.d + at;
    const f32x2 scale = tc::pack2(a.e.scale, a.e.scale);
    if (a.add) {
        Eight<TO, L> old;
        old.template load<kKeep>(p, step, a.e.d - at);
        f32x2 o[4];
        old.get(o);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = tc::add2(tc::mul2(v[j], scale), o[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = tc::mul2(v[j], scale);
    }
    Eight<TO, L> e;
    e.set(v);
    e.store(p, step, a.e.d - at);
}

// the number of lanes from lane 0 on without a gap
__device__ __forceinline__ int leading(bool p)
{
    const int gap = __ffs(~__ballot_sync(0xffffffffu, p));
    return gap ? gap - 1 : 32;
}

// One chunk of sorted tokens and 8 blockDim columns
template <class TY, class TO, Layout L>
__global__ void __launch_bounds__(kEmbThreads) k_embed_sum(const SumArgs a)
{
    __shared__ int sk[kLong + kReach];  // ids of the tokens from kLong before the chunk on; -1 where there is none
    __shared__ int sp[kReach];
    dependent_start();
    const long long chunk = blockIdx.x, i0 = chunk * kChunk;
    for (int i = threadIdx.x; i < kLong + kReach; i += blockDim.x) {
        const long long at = i0 + i - kLong;
        sk[i] = at >= 0 && at < a.e.n ? __ldg(a.key + at) : -1;
        if (i >= kLong) sp[i - kLong] = at < a.e.n ? __ldg(a.pos + at) : 0;
    }
    __syncthreads();
    const int *const id = sk + kLong;
    const int lane = threadIdx.x & 31, n = (int)min((long long)kChunk, a.e.n - i0), V = a.e.V;
    int begin = 0, end = n;
    bool head = false, tail = false;  // the first, the last run is a piece of a long one that began before, that begins here
    if (id[0] == V) return;           // (tokens without an id are the last)
    if (id[-1] == id[0]) {
        int back = leading(id[-1 - lane] == id[0]), on = leading(id[lane] == id[0]);
        if (back == 32) back += leading(id[-33 - lane] == id[0]);
        if (on == 32) on += leading(id[32 + lane] == id[0]);
        if (on == 64) on += leading(id[64 + lane] == id[0]);
        head = back + on > kLong;
        if (!head) begin = on;        // (the chunk in which it began takes all of it)
        if (begin >= n) return;
    }
    const int last = id[n - 1];
    if (last != V && id[n] == last && !(head && last == id[0])) {
        const int back = leading(id[n - 1 - lane] == last);  // (it begins in this chunk)
        int on = leading(id[n + lane] == last);
        if (on == 32) on += leading(id[n + 32 + lane] == last);
        tail = back + on > kLong;
        if (!tail) end = n + on;
        else if (threadIdx.x == 0 && blockIdx.y == 0) a.list[atomicAdd(a.runs, 1)] = (int)chunk;
    }
    const int threads = blockDim.x, step = L == kQuads ? 4 * threads : threads, block = blockIdx.y * threads * 8,
              at = block + (int)threadIdx.x * (L == kEights ? 8 : L == kQuads ? 4 : 1);
    if (at >= a.e.d) return;
    const TY *dy = static_cast<const TY *>(a.e.in) + at;
    f32x2 acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = tc::pack2(0.f, 0.f);
    for (int i = begin; i < end; i += kAhead) {
        Eight<TY, L> row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < end && id[i + u] != V) row[u].load(dy + (long long)sp[i + u] * a.e.ld, step, a.e.d - at);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= end) break;
            const int now = id[i + u];
            if (now == V) return;
            f32x2 v[4];
            row[u].get(v);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = tc::add2(acc[j], v[j]);
            if (i + u + 1 < end && id[i + u + 1] == now) continue;
            const bool piece = (head && now == id[0]) || (tail && now == last);
            if (piece) {
                Eight<float, L> e;
                e.set(acc);
                e.template store<kKeep>(a.part + (chunk * 2 + (head && now == id[0] ? 0 : 1)) * a.e.d + at, step, a.e.d - at);
            } else {
                write_row<TO, L>(a, now, at, step, acc);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = tc::pack2(0.f, 0.f);
        }
    }
}

// Long runs: a block adds up the pieces of kJoinCols 8 columns of one, every kJoin-th piece by a row of threads, those in order.
constexpr int kJoin = 8, kJoinCols = 32;
template <class TO, Layout L>
__global__ void __launch_bounds__(kJoin *kJoinCols) k_embed_join(const SumArgs a, int tiles)
{
    __shared__ float red[kJoin][8][kJoinCols + 1];
    dependent_start();
    const long long items = (long long)*a.runs * tiles;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long chunk = __ldg(a.list + item / tiles);
        const int id = __ldg(a.key + (chunk + 1) * kChunk - 1);
        long long end = chunk;  // its last chunk: those behind the first that begin with it
        for (int more = kJoin * kJoinCols; more == kJoin * kJoinCols; end += more) {
            const long long at = (end + 1 + threadIdx.x) * kChunk;
            more = __syncthreads_count(at < a.e.n && __ldg(a.key + at) == id);
        }
        const int c = threadIdx.x % kJoinCols, q = threadIdx.x / kJoinCols, step = L == kQuads ? 4 * kJoinCols : kJoinCols;
        const int at = (int)(item % tiles) * kJoinCols * 8 + c * (L == kEights ? 8 : L == kQuads ? 4 : 1);
        f32x2 acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = tc::pack2(0.f, 0.f);
        if (at < a.e.d) {
#pragma unroll 4
            for (long long k = chunk + q; k <= end; k += kJoin) {
                Eight<float, L> e;
                e.template load<kKeep>(a.part + (k * 2 + (k == chunk ? 1 : 0)) * a.e.d + at, step, a.e.d - at);
                f32x2 v[4];
                e.get(v);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = tc::add2(acc[j], v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) tc::unpack2(acc[j], red[q][2 * j][c], red[q][2 * j + 1][c]);
        __syncthreads();
        if (q == 0 && at < a.e.d) {
#pragma unroll
            for (int i = 1; i < kJoin; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = tc::add2(acc[j], tc::pack2(red[i][2 * j][c], red[i][2 * j + 1][c]));
            write_row<TO, L>(a, id, at, step, acc);
        }
        // (the next item writes to red behind the barrier in its search)
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------
template <class T>
struct Type {
    using type = T;
};
template <class F>
cudaError_t with_type(int dtype, F f) { return dtype == RR_F32 ? f(Type<float>{}) : f(Type<bf16>{}); }

struct BwdLayout {
    Header *hdr;
    int *key, *pos, *key2, *pos2, *runs, *list;
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
    l.runs = c.take<int>(1);
    l.list = c.take<int>(n / kLong + 1);
    l.part = c.take<float>(n > kLong ? (size_t)l.chunks * 2 * d : 0);
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

// bf16 alone goes eight at a time, with fp32 four: 16-byte accesses of the wider type
Layout layout_of(const rr_embed_shape &s)
{
    if (s.table_dtype == RR_BF16 && s.y_dtype == RR_BF16 && s.d % 8 == 0 && s.ldy % 8 == 0) return kEights;
    return s.d % 4 == 0 && s.ldy % 4 == 0 ? kQuads : kOne;
}

template <int K>
cudaError_t launch_sort(const SortArgs &a, int blocks, cudaStream_t st)
{
    constexpr size_t smem = (size_t)kDigits * (kSortWarps + 2) * 4 + (size_t)kSortThreads * K * 6;
    static_assert(smem >= kMapWords * 4 && smem <= 227 << 10, "a zeroing block's bitmap lies in the same memory");
    const cudaError_t err = cudaFuncSetAttribute(k_embed_sort<K>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
    return launch_dependent(k_embed_sort<K>, dim3(blocks), kSortThreads, smem, 1, st, a);
}

}  // namespace

size_t embed_bwd_workspace(long long n, int d) { return bwd_layout(nullptr, n, d, nullptr); }

rr_status launch_embed_fwd(const rr_embed_shape &s, const void *ids, const void *table, void *y, void *ws, cudaStream_t st)
{
    const EmbArgs a = emb_args(s, ids, table, y, ws);
    const Layout L = layout_of(s);
    const int per_row = L == kEights ? s.d / 8 : L == kQuads ? s.d / 4 : s.d, sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    // w / per_row is the high word of w * magic, magic = ceil(2^64 / per_row): what the rounding up adds to the quotient is below
    // w / 2^64 < 2^-32, less than the 1 / per_row that would be missing to the next whole number.  (A divisor of one has no such factor.)
    const unsigned long long magic = per_row == 1 ? 0 : ~0ull / (unsigned)per_row + 1;
    const long long tiles = ((long long)s.n * per_row + kEmbThreads * kEmbUnroll - 1) / (kEmbThreads * kEmbUnroll), most = (long long)sms * 8;
    const dim3 grid((unsigned)(tiles < most ? tiles : most));
    const long long step = (long long)grid.x * kEmbThreads * kEmbUnroll, row_step = step / per_row;
    const unsigned at_step = (unsigned)(step % per_row);
    const cudaError_t err = with_type(s.table_dtype, [&](auto tx) {
        return with_type(s.y_dtype, [&](auto ty) {
            using TX = typename decltype(tx)::type;
            using TY = typename decltype(ty)::type;
            auto go = [&](auto kernel) { return launch_dependent(kernel, grid, kEmbThreads, 0, 1, st, a, per_row, magic, row_step, at_step); };
            if constexpr (sizeof(TX) + sizeof(TY) == 4) {
                if (L == kEights) return go(k_embed_fwd<TX, TY, 8>);
            }
            return L == kOne ? go(k_embed_fwd<TX, TY, 1>) : go(k_embed_fwd<TX, TY, 4>);
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
    int bits = 1;
    while (bits < 31 && s.V >> bits) ++bits;  // (V itself is a key)
    a.passes = (bits + kDigitBits - 1) / kDigitBits;
    a.bits = (bits + a.passes - 1) / a.passes;
    a.key = l.key;
    a.pos = l.pos;
    a.runs = l.runs;
    a.out_f32 = s.table_dtype == RR_F32;
    int fillers = 0;
    if (!add) {  // zeroing blocks: one an SM, but none with less than 64 KB
        const long long bytes = (long long)s.V * s.d * (a.out_f32 ? 4 : 2), want = (bytes + 65535) / 65536;
        const int most = sms - l.slabs > sms / 4 ? sms - l.slabs : sms / 4;  // (one block an SM: all at once)
        fillers = (int)(want < most ? want : most);
        if (fillers > s.V) fillers = s.V;
    }
    const int blocks = l.slabs + fillers, K = (l.slab + kSortThreads - 1) / kSortThreads;
    cudaError_t err = K <= 2 ? launch_sort<2>(a, blocks, st) : K <= 4 ? launch_sort<4>(a, blocks, st) : K <= 8 ? launch_sort<8>(a, blocks, st)
                                                                                                                : launch_sort<kSortMost>(a, blocks, st);
    if (err == cudaSuccess && l.slabs > 1)
        err = launch_dependent(k_embed_merge, dim3((unsigned)((s.n + kEmbThreads - 1) / kEmbThreads)), kEmbThreads, 0, 1, st, (long long)s.n, l.slabs, l.slab,
                               (const int *)l.key, (const int *)l.pos, l.key2, l.pos2);
    if (err != cudaSuccess) return RR_ERR_CUDA;
    SumArgs b;
    b.e = a.e;
    b.key = l.key2;
    b.pos = l.pos2;
    b.part = l.part;
    b.runs = l.runs;
    b.list = l.list;
    b.add = add;
    const Layout L = layout_of(s);
    int threads = 32;
    while (threads < kEmbThreads && threads * 8 < s.d) threads <<= 1;
    const dim3 grid((unsigned)l.chunks, (unsigned)((s.d + threads * 8 - 1) / (threads * 8)));
    const int tiles = (s.d + kJoinCols * 8 - 1) / (kJoinCols * 8);
    const long long most_items = (long long)(s.n / kLong + 1) * tiles;
    const dim3 join((unsigned)(most_items < 2 * sms ? most_items : 2 * sms));
    err = with_type(s.table_dtype, [&](auto to) {
        using TO = typename decltype(to)::type;
        cudaError_t e = with_type(s.y_dtype, [&](auto ty) {
            using TY = typename decltype(ty)::type;
            auto go = [&](auto kernel) { return launch_dependent(kernel, grid, threads, 0, 1, st, b); };
            if constexpr (sizeof(TY) + sizeof(TO) == 4) {
                if (L == kEights) return go(k_embed_sum<TY, TO, kEights>);
            }
            return L == kOne ? go(k_embed_sum<TY, TO, kOne>) : go(k_embed_sum<TY, TO, kQuads>);
        });
        if (e != cudaSuccess || s.n <= kLong) return e;  // (no run is long)
        auto go = [&](auto kernel) { return launch_dependent(kernel, join, kJoin * kJoinCols, 0, 1, st, b, tiles); };
        if constexpr (sizeof(TO) == 2) {
            if (L == kEights) return go(k_embed_join<TO, kEights>);
        }
        return L == kOne ? go(k_embed_join<TO, kOne>) : go(k_embed_join<TO, kQuads>);
    });
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

}  // namespace rr
