// The embedding in front of the first block, and its gradient.
//     y_i = scale table[id_i]          dtable_v = scale (sum over the tokens i with id_i = v, in token order, of dy_i)
// Forward: a gather, bound by HBM.  Backward without floating-point atomics, so that results repeat: the tokens are sorted by id (stably:
// equal ids stay in token order), the sorted tokens are cut into chunks of equal length, a block adds up the rows of a chunk in registers and
// writes the table's row whenever the id changes.  An id with many tokens leaves pieces in the workspace that a last kernel adds up in order: a
// frequent id costs no more than any other.  Rows that no token names are zeroed by blocks that run beside the sort and learn of the named
// rows from a bitmap of their own.  Few tokens need no sort.  Sums are fp32.
// Measured, bf16: forward 65536 x 1024 27.7 us (5.7 TB/s counting every row of the table that is named once), 37 x 4096 1.7 us.  Gradient of a table of
// 32000 rows, 16384 x 4096 into fp32 129 us (5.1 TB/s; 80 of them the zeroed rows, which hide the sort), 16384 x 1024 42, 65536 x 1024 86 (sort
// beside rows to zero 28, merge 8, sums 33, long runs 8, starts).
#include <type_traits>
#include <utility>

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

// Ids of the kN tokens first, first + step, ...: 0..V-1, or -1 for none (and, with the error latched, for one out of range); -2 from token
// `end` on.  All are asked for before the first is looked at.
template <int kN>
__device__ __forceinline__ void token_ids(const EmbArgs &a, const long long (&token)[kN], long long end, int (&id)[kN])
{
    long long raw[kN];
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        raw[k] = -1;
        if (token[k] >= end) continue;
        if (a.wide) raw[k] = static_cast<const long long *>(a.ids)[token[k]];
        else raw[k] = static_cast<const int *>(a.ids)[token[k]];
    }
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        const bool fits = raw[k] >= 0 && raw[k] < a.V;
        bad |= !fits && raw[k] != -1;
        id[k] = token[k] >= end ? -2 : fits ? (int)raw[k] : -1;
    }
    if (bad) latch_status(a.status, RR_ERR_INVALID_ARG);
}

// `units` units of kN elements, kStep units apart, at most kEmbUnroll of them: all read before the first is written.  live: y is a row of the table
// and not of zeros.
constexpr int kEmbUnroll = 4;
template <class TX, class TY, int kN, int kStep>
__device__ __forceinline__ void copy_units(const TX *from, TY *to, int units, bool live, float scale)
{
    Unit<TX, kN> e[kEmbUnroll];
#pragma unroll
    for (int u = 0; u < kEmbUnroll; ++u) {
        e[u].raw = {};
        if (live && u < units) e[u].template load<kKeep>(from + u * kStep * kN);
    }
#pragma unroll
    for (int u = 0; u < kEmbUnroll; ++u) {
        if (u >= units) break;
        Unit<TY, kN> o;
        if constexpr (std::is_same<TX, TY>::value) o.raw = e[u].raw;
        if (scale != 1.0f || !std::is_same<TX, TY>::value) scaled<kN>(e[u], o, scale);
        if (!live) o.raw = {};  // (not -0)
        o.template store<kStream>(to + u * kStep * kN);
    }
}

// Wide rows: a warp takes pieces of a row, 32 kEmbUnroll units each.  One look at the id and one division for four units a lane: the kernel
// below, which divides for every unit, is bound by instructions (65536 x 1024 in bf16 30.5 us).
template <class TX, class TY, int kN>
__global__ void __launch_bounds__(kEmbThreads) k_embed_rows(const EmbArgs a, int per_row, int pieces, unsigned long long magic)
{
    constexpr int kPiece = 32 * kEmbUnroll;
    dependent_start();
    const int lane = threadIdx.x & 31;
    const long long items = a.n * pieces, step = (long long)gridDim.x * (kEmbThreads / 32);
    for (long long item = (long long)blockIdx.x * (kEmbThreads / 32) + (threadIdx.x >> 5); item < items; item += step) {
        const long long row = magic ? (long long)__umul64hi((unsigned long long)item, magic) : item;  // item / pieces (the host says why)
        const int first = (int)(item - row * pieces) * kPiece + lane;
        const long long token[1] = {row};
        int id[1];
        token_ids(a, token, a.n, id);
        copy_units<TX, TY, kN, 32>(static_cast<const TX *>(a.in) + (long long)max(id[0], 0) * a.d + (long long)first * kN, static_cast<TY *>(a.out) + row * a.ld + (long long)first * kN,
                                   (per_row - first + 31) / 32, id[0] >= 0, a.scale);
    }
}

// Narrow rows: a block takes tiles of units, whatever the width of a row; row and place of a unit come from a product, and those of the next
// tile from those of the last.
template <class TX, class TY, int kN>
__global__ void __launch_bounds__(kEmbThreads) k_embed_units(const EmbArgs a, int per_row, unsigned long long magic, long long row_step, unsigned at_step)
{
    constexpr int kTile = kEmbThreads * kEmbUnroll;
    dependent_start();
    const long long total = a.n * per_row;  // (a unit behind the last has a row behind the last)
    long long row0 = (long long)blockIdx.x * kTile / per_row;
    unsigned at0 = (unsigned)((long long)blockIdx.x * kTile - row0 * per_row);
    for (long long tile = (long long)blockIdx.x * kTile; tile < total; tile += (long long)gridDim.x * kTile) {
        int id[kEmbUnroll];
        long long row[kEmbUnroll];
        unsigned at[kEmbUnroll];
#pragma unroll
        for (int u = 0; u < kEmbUnroll; ++u) {
            const unsigned l = u * kEmbThreads + threadIdx.x, w = at0 + l;
            const unsigned q = magic ? (unsigned)__umul64hi(w, magic) : w;  // w / per_row
            row[u] = row0 + q;
            at[u] = w - q * per_row;
        }
        token_ids(a, row, a.n, id);
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
constexpr int kDigitBits = 5, kDigits = 1 << kDigitBits; // at most
constexpr int kSortMost = 16;                            // tokens a thread of a sorting block holds
constexpr int kSlab = kSortThreads * kSortMost;          // tokens of a sorting block (20 us; four of 4096 and their merge take as long)
constexpr int kPlaceBits = 14;                           // a token's place in its slab
static_assert(kSlab <= 1 << kPlaceBits && kSortMost <= 16, "a place fits into its bits, a thread's count of a digit into four");
constexpr int kTableWords = kDigits * (kSortThreads / 2 / 16 * 17);
constexpr int kMapWords = 8192;                          // bitmap of a zeroing block: 2^18 rows at a time

struct SortArgs {
    EmbArgs e;
    int slabs, slab;       // sorting blocks and tokens of each (the last may have fewer)
    int passes, bits;      // digits, and bits of each
    int *key, *pos;        // [n] sorted ids (V: no id) and their tokens, slab by slab
    int *runs;             // counter of the long runs (k_embed_sum), set to zero here
    int out_f32;
};

// Rows of this zeroing block that no token names (`size`: bytes of an element).  `lanes` lanes of a warp zero a row, as many as it has 16-byte
// pieces.
template <int kThreads>
__device__ void zero_rows(const EmbArgs &e, int size, int block, int blocks, uint32_t *map)
{
    const long long V = e.V, lo = V * block / blocks, hi = V * (block + 1) / blocks;
    const long long width = (long long)e.d * size;
    int lanes = 1;
    while (lanes < 32 && lanes * 16 < width) lanes <<= 1;
    const int lane = threadIdx.x & (lanes - 1), step = kThreads / lanes;
    constexpr int kAtOnce = 8;
    for (long long r0 = lo; r0 < hi; r0 += kMapWords * 32) {
        const long long r1 = min(hi, r0 + kMapWords * 32);
        const int words = (int)((r1 - r0 + 31) / 32);
        __syncthreads();
        for (int i = threadIdx.x; i < words; i += kThreads) map[i] = 0;
        __syncthreads();
        for (long long i0 = threadIdx.x; i0 < e.n; i0 += kAtOnce * kThreads) {
            long long token[kAtOnce];
            int id[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) token[u] = i0 + u * kThreads;
            token_ids(e, token, e.n, id);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
                if (id[u] >= r0 && id[u] < r1) atomicOr(&map[(id[u] - r0) >> 5], 1u << ((id[u] - r0) & 31));
        }
        __syncthreads();
        for (long long r = r0 + threadIdx.x / lanes; r < r1; r += step) {
            if (map[(r - r0) >> 5] >> ((r - r0) & 31) & 1) continue;
            char *p = static_cast<char *>(e.out) + r * width;  // (an even address, an even number of bytes)
            const int head = (int)min(width, (long long)(-(uintptr_t)p & 15)), tail = (int)((width - head) & 15);
            for (int i = 2 * lane; i < head; i += 2 * lanes) *reinterpret_cast<uint16_t *>(p + i) = 0;
            for (int i = 2 * lane; i < tail; i += 2 * lanes) *reinterpret_cast<uint16_t *>(p + width - tail + i) = 0;
            uint4 *q = reinterpret_cast<uint4 *>(p + head);
            for (long long i = lane; i < (width - head) / 16; i += lanes) __stcs(q + i, make_uint4(0u, 0u, 0u, 0u));
        }
    }
}

// Stable sort of a slab by id, least significant digit first, of words T that hold an id and below it the token's place in the slab.  Thread t
// holds the K words t K, t K + 1, ...: in a pass it counts them digit by digit in its own column of a table (32 digits of 1024 threads, 16 bits
// each) and remembers how many of a word's digit it had before; the table is scanned digit by digit and thread by thread, and the words
// move in shared memory.  (Counted by warps with ballots instead, a token cost 150 instructions a pass: 16384 tokens 40 us.)
// Blocks behind the sorting ones zero the rows that nobody names.
template <int K, class T>
__global__ void __launch_bounds__(kSortThreads) k_embed_sort(const SortArgs a)
{
    extern __shared__ __align__(16) uint32_t shared[];
    dependent_start();
    if ((int)blockIdx.x >= a.slabs) {
        zero_rows<kSortThreads>(a.e, a.out_f32 ? 4 : 2, blockIdx.x - a.slabs, gridDim.x - a.slabs, shared);
        return;
    }
    // Table and words have gaps, so that threads next to each other meet in different banks: two entries after every 32, one word after every K.
    uint16_t *const count = reinterpret_cast<uint16_t *>(shared);  // [digits][kSortThreads]
    T *const words = reinterpret_cast<T *>(shared + kTableWords);
    auto entry = [](uint32_t digit, int thread) { return digit * (kSortThreads / 16 * 17) + thread + (thread >> 5) * 2; };
    __shared__ uint32_t warp_total[kSortWarps];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, digits = 1 << a.bits;
    const long long base = (long long)blockIdx.x * a.slab;
    const int n = (int)min((long long)a.slab, a.e.n - base);
    if (blockIdx.x == 0 && t == 0) *a.runs = 0;
    constexpr int kAtOnce = K < 8 ? K : 8;
#pragma unroll
    for (int k0 = 0; k0 < K; k0 += kAtOnce) {
        long long token[kAtOnce];
        int id[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) token[k] = base + (k0 + k) * kSortThreads + t;
        token_ids(a.e, token, base + n, id);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int i = (k0 + k) * kSortThreads + t;  // (places behind the end stay behind all others)
            words[i + i / K] = (id[k] == -2 ? ~(T)0 << kPlaceBits : (T)(id[k] < 0 ? a.e.V : id[k]) << kPlaceBits) | (T)i;
        }
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = kPlaceBits + pass * a.bits;
        uint4 *const table = reinterpret_cast<uint4 *>(count);
        for (int i = t; i < digits * (kSortThreads / 128 * 17); i += kSortThreads) table[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        T e[K];
        uint32_t at[K];  // a word's entry in the table, and below it how many of its digit the thread had before
#pragma unroll
        for (int k = 0; k < K; ++k) e[k] = words[t * (K + 1) + k];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t c = entry((uint32_t)(e[k] >> shift) & (digits - 1), t), before = count[c];
            count[c] = (uint16_t)(before + 1);
            at[k] = c << 4 | before;
        }
        __syncthreads();
        // exclusive scan: thread t owns `digits` entries next to each other, pairs of 16 bits in a word
        uint32_t *const own = shared + t * (digits / 2) + t * (digits / 2) / 16;
        uint32_t pairs = 0;
#pragma unroll
        for (int i = 0; i < kDigits / 2; ++i)
            if (i < digits / 2) pairs += own[i];  // (no half leaves 16 bits: there are no more tokens)
        uint32_t sum = (pairs & 0xffff) + (pairs >> 16), upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += up;
        }
        if (lane == 31) warp_total[warp] = upto;
        __syncthreads();
        uint32_t run = lane < warp ? warp_total[lane] : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) run += __shfl_xor_sync(0xffffffffu, run, o);
        run += upto - sum;
#pragma unroll
        for (int i = 0; i < kDigits / 2; ++i) {
            if (i >= digits / 2) break;
            const uint32_t two = own[i], low = two & 0xffff;
            own[i] = run | (run + low) << 16;
            run += low + (two >> 16);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t to = count[at[k] >> 4] + (at[k] & 15);
            words[to + to / K] = e[k];
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = k * kSortThreads + t;
        if (i >= n) break;
        const T e = words[i + i / K];
        a.key[base + i] = (int)(e >> kPlaceBits);
        a.pos[base + i] = (int)(base + (long long)(e & ((1 << kPlaceBits) - 1)));
    }
}

// Every kSide sorted slabs into one: a token's place is the number of tokens in front of it in each of them (equal ids: earlier slabs only).  The
// slabs are searched side by side, all of a step's loads in flight together.
template <int kSide>
__global__ void __launch_bounds__(kEmbThreads) k_embed_merge(int n, int slab, const int *key, const int *pos, int *out_key, int *out_pos)
{
    dependent_start();
    const int i = blockIdx.x * kEmbThreads + threadIdx.x;
    if (i >= n) return;
    const int mine = i / slab, first = mine / kSide * kSide, id = key[i], token = pos[i];
    int to = i - (mine - first) * slab;  // (places are below 2^30)
    int lo[kSide], hi[kSide], start[kSide], steps = 1;
    while (1 << steps <= slab) ++steps;
#pragma unroll
    for (int u = 0; u < kSide; ++u) {
        const long long at = (long long)(first + u) * slab;
        const bool other = at < n && first + u != mine;
        start[u] = other ? (int)at : 0;
        lo[u] = 0;
        hi[u] = other ? (int)min((long long)slab, n - at) : 0;
    }
    for (int step = 0; step < steps; ++step) {
        int k[kSide];
#pragma unroll
        for (int u = 0; u < kSide; ++u) k[u] = key[start[u] + min((lo[u] + hi[u]) >> 1, max(hi[u] - 1, 0))];
#pragma unroll
        for (int u = 0; u < kSide; ++u) {  // tokens of that slab below id, or in earlier slabs not above it
            const int mid = (lo[u] + hi[u]) >> 1;
            const bool before = k[u] < id || (k[u] == id && first + u < mine), open = lo[u] < hi[u];
            if (open && before) lo[u] = mid + 1;
            if (open && !before) hi[u] = mid;
        }
    }
#pragma unroll
    for (int u = 0; u < kSide; ++u) to += lo[u];
    out_key[to] = id;
    out_pos[to] = token;
}

// ---- backward: the sums -------------------------------------------------------------------------------------------
// A run is all the tokens of one id.  A block takes a chunk of sorted tokens, and of the runs that begin in it those of up to two chunks'
// length to their end: most runs are short, and need no second look.  Of a longer run every chunk adds up its own piece (the first piece is
// part 1 of its chunk, every other the part 0), and k_embed_join adds up the pieces in order.
struct SumArgs {
    EmbArgs e;
    const int *key, *pos;  // [n] sorted
    float *part;           // [chunks][2][d]
    int *runs, *list;      // long runs: how many, and the chunks in which they begin (in any order)
    int chunk;             // sorted tokens of a chunk, kLeastChunk to kMostChunk
    int add;
};

constexpr int kLeastChunk = 8, kMostChunk = 32;
constexpr int kBefore = 2 * kMostChunk, kReach = 3 * kMostChunk;  // tokens that a block looks at before its chunk, and from its start on
constexpr int kAhead = 8;                                         // rows in flight

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
    __shared__ int sk[kBefore + kReach];  // ids of the tokens from kBefore before the chunk on; -1 where there is none
    __shared__ int sp[kReach];
    dependent_start();
    const long long chunk = blockIdx.x, i0 = chunk * a.chunk;
    constexpr int kLooks = (kBefore + kReach) / 32;  // (of a block of 32; all asked for at once)
    int k[kLooks], p[kLooks];
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
        const int i = threadIdx.x + u * blockDim.x;
        const long long at = i0 + i - kBefore;
        k[u] = -1;
        p[u] = 0;
        if (i >= kBefore + kReach || at < 0 || at >= a.e.n) continue;
        k[u] = a.key[at];
        if (i >= kBefore) p[u] = a.pos[at];
    }
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
        const int i = threadIdx.x + u * blockDim.x;
        if (i >= kBefore + kReach) break;
        sk[i] = k[u];
        if (i >= kBefore) sp[i - kBefore] = p[u];
    }
    __syncthreads();
    const int *const id = sk + kBefore;
    const int lane = threadIdx.x & 31, n = (int)min((long long)a.chunk, a.e.n - i0), V = a.e.V, longest = 2 * a.chunk;
    int begin = 0, end = n;
    bool head = false, tail = false;  // the first, the last run is a piece of a long one that began before, that begins here
    if (id[0] == V) return;           // (tokens without an id are the last)
    if (id[-1] == id[0]) {
        int back = leading(id[-1 - lane] == id[0]), on = leading(id[lane] == id[0]);
        if (back == 32) back += leading(id[-33 - lane] == id[0]);
        if (on == 32) on += leading(id[32 + lane] == id[0]);
        if (on == 64) on += leading(id[64 + lane] == id[0]);
        head = back + on > longest;
        if (!head) begin = on;        // (the chunk in which it began takes all of it)
        if (begin >= n) return;
    }
    const int last = id[n - 1];
    if (last != V && id[n] == last && !(head && last == id[0])) {
        const int back = leading(id[n - 1 - lane] == last);  // (it begins in this chunk)
        int on = leading(id[n + lane] == last);
        if (on == 32) on += leading(id[n + 32 + lane] == last);
        tail = back + on > longest;
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

// Few tokens: one kernel instead of three.  Every block looks at all ids; the block of a token that is the first of its id adds up the rows of
// all of them, those of other tokens have nothing to do, and the blocks behind zero the rows that nobody names.
constexpr int kDirect = 128;
template <class TY, class TO, Layout L>
__global__ void __launch_bounds__(kEmbThreads) k_embed_direct(const SumArgs a, int tiles)
{
    extern __shared__ __align__(16) uint32_t shared[];  // (the bitmap of a zeroing block)
    dependent_start();
    const int n = (int)a.e.n, token = blockIdx.x / tiles;
    if (token >= n) {
        zero_rows<kEmbThreads>(a.e, sizeof(TO), blockIdx.x - n * tiles, gridDim.x - n * tiles, shared);
        return;
    }
    int *const same = reinterpret_cast<int *>(shared);  // the tokens of this one's id, in order
    __shared__ int ids[kDirect];
    __shared__ int count;
    if (threadIdx.x < kDirect) {
        const long long at[1] = {(long long)threadIdx.x};
        int id[1];
        token_ids(a.e, at, a.e.n, id);
        ids[threadIdx.x] = id[0];
    }
    __syncthreads();
    const int id = ids[token];
    if (id < 0) return;
    if (threadIdx.x < 32) {
        int found = 0;
        bool first = true;
#pragma unroll
        for (int k = 0; k < kDirect; k += 32) {
            const int at = k + threadIdx.x;
            const uint32_t with = __ballot_sync(0xffffffffu, ids[at] == id);
            if (ids[at] == id) same[found + __popc(with & ((1u << threadIdx.x) - 1))] = at;
            if (found == 0 && with) first = k + __ffs(with) - 1 == token;
            found += __popc(with);
        }
        if (threadIdx.x == 0) count = first ? found : 0;
    }
    __syncthreads();
    const int step = L == kQuads ? 4 * kEmbThreads : kEmbThreads,
              at = (int)(blockIdx.x % tiles) * kEmbThreads * 8 + (int)threadIdx.x * (L == kEights ? 8 : L == kQuads ? 4 : 1);
    if (at >= a.e.d) return;
    const TY *dy = static_cast<const TY *>(a.e.in) + at;
    f32x2 acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = tc::pack2(0.f, 0.f);
    for (int i = 0; i < count; i += kAhead) {
        Eight<TY, L> row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < count) row[u].load(dy + (long long)same[i + u] * a.e.ld, step, a.e.d - at);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= count) break;
            f32x2 v[4];
            row[u].get(v);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = tc::add2(acc[j], v[j]);
        }
    }
    if (count) write_row<TO, L>(a, id, at, step, acc);
}

// Long runs: a block adds up the pieces of 8 kJoinCols columns of one, every kJoin-th piece by a row of threads, then the rows of threads in order.
constexpr int kJoin = 16, kJoinCols = 32;
template <class TO, Layout L>
__global__ void __launch_bounds__(kJoin *kJoinCols) k_embed_join(const SumArgs a, int tiles)
{
    __shared__ float red[kJoin][8][kJoinCols + 1];
    dependent_start();
    const long long items = (long long)*a.runs * tiles;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long chunk = a.list[item / tiles];
        const int id = a.key[(chunk + 1) * a.chunk - 1];
        long long end = chunk;  // its last chunk: those behind the first that begin with it
        for (int more = kJoin * kJoinCols; more == kJoin * kJoinCols; end += more) {
            const long long at = (end + 1 + threadIdx.x) * a.chunk;
            more = __syncthreads_count(at < a.e.n && a.key[at] == id);
        }
        const int c = threadIdx.x % kJoinCols, q = threadIdx.x / kJoinCols, step = L == kQuads ? 4 * kJoinCols : kJoinCols;
        const int at = (int)(item % tiles) * kJoinCols * 8 + c * (L == kEights ? 8 : L == kQuads ? 4 : 1);
        f32x2 acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = tc::pack2(0.f, 0.f);
        if (at < a.e.d) {
#pragma unroll 8
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
        if (q < 8) {  // the q-th of the eight values
            float sum = red[0][q][c];
#pragma unroll
            for (int i = 1; i < kJoin; ++i) sum += red[i][q][c];
            red[0][q][c] = sum;  // (nobody else reads it before the barrier)
        }
        __syncthreads();
        if (q == 0 && at < a.e.d) {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = tc::pack2(red[0][2 * j][c], red[0][2 * j + 1][c]);
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

// Floats of the pieces of `n` tokens, and of any fewer or narrower ones, so that the workspace of a program's largest batch serves every other:
// two rows a chunk.  Chunks are shorter where tokens are few, and then a row of each makes at most 2^23 + d floats in all: chunks of 8 (16) are taken
// below n ceil(d / 256) = 2^18 (2^19), so that n d / 8 (n d / 16) stays below 2^26 / 8 (2^27 / 16), and the last chunk adds a row.
size_t piece_floats(long long n, int d)
{
    const size_t least = (size_t)((n + kMostChunk - 1) / kMostChunk) * d, most = (size_t)((n + kLeastChunk - 1) / kLeastChunk) * d, cap = (1ull << 23) + d;
    const size_t few = most < cap ? most : cap;
    return 2 * (least > few ? least : few);
}

struct BwdLayout {
    Header *hdr;
    int *key, *pos, *key2, *pos2, *runs, *list;
    float *part;
    long long chunks;
    int chunk;
};
size_t bwd_layout(void *ws, long long n, int d, BwdLayout *out)
{
    BwdLayout l;
    // chunks: shorter ones where the SMs would be short of warps
    const long long warps = (d + 255) / 256;
    l.chunk = kMostChunk;
    while (l.chunk > kLeastChunk && n * warps < 16384ll * l.chunk) l.chunk >>= 1;
    l.chunks = (n + l.chunk - 1) / l.chunk;
    Carver c(ws);
    l.hdr = c.take<Header>(1);
    l.key = c.take<int>(n);
    l.pos = c.take<int>(n);
    l.key2 = n > kSlab ? c.take<int>(n) : l.key;
    l.pos2 = n > kSlab ? c.take<int>(n) : l.pos;
    l.runs = c.take<int>(1);
    l.list = c.take<int>(n / (2 * kLeastChunk) + 1);
    l.part = c.take<float>(n > kDirect ? piece_floats(n, d) : 0);  // (fewer tokens are not sorted)
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

template <int K, class T>
cudaError_t launch_sort(const SortArgs &a, int blocks, cudaStream_t st)
{
    constexpr size_t smem = (size_t)kTableWords * 4 + (size_t)kSortThreads * (K + 1) * sizeof(T);
    static_assert(smem >= kMapWords * 4 && smem <= SharedAllowance::kMost, "a zeroing block's bitmap lies in the same memory");
    static SharedAllowance allowance;
    const cudaError_t err = allowance.ask(k_embed_sort<K, T>, (int)smem);
    if (err != cudaSuccess) return err;
    return launch_dependent(k_embed_sort<K, T>, dim3(blocks), kSortThreads, smem, 1, st, a);
}
template <class T>
cudaError_t launch_sort(const SortArgs &a, int blocks, cudaStream_t st)
{
    const int K = (a.slab + kSortThreads - 1) / kSortThreads;
    return K <= 2 ? launch_sort<2, T>(a, blocks, st) : K <= 4 ? launch_sort<4, T>(a, blocks, st) : K <= 8 ? launch_sort<8, T>(a, blocks, st)
                                                                                                          : launch_sort<kSortMost, T>(a, blocks, st);
}

}  // namespace

size_t embed_bwd_workspace(long long n, int d) { return bwd_layout(nullptr, n, d, nullptr); }

rr_status launch_embed_fwd(const rr_embed_shape &s, const void *ids, const void *table, void *y, void *ws, cudaStream_t st)
{
    const EmbArgs a = emb_args(s, ids, table, y, ws);
    const Layout L = layout_of(s);
    const int per_row = L == kEights ? s.d / 8 : L == kQuads ? s.d / 4 : s.d, sms = device_sm_count();
    if (sms < 1) return RR_ERR_CUDA;
    // i / q is the high word of i * magic, magic = ceil(2^64 / q), for i < 2^40 and q < 2^23 (there is no memory for more): what the rounding up adds to the quotient is below
    // i / 2^64 < 2^-24, less than the 1 / q that would be missing to the next whole number.  (For i < 2^32: q < 2^31.)  A divisor of one has no such
    // factor.
    auto factor = [](int q) { return q == 1 ? 0 : ~0ull / (unsigned)q + 1; };
    constexpr int kPiece = 32 * kEmbUnroll;
    const int pieces = (per_row + kPiece - 1) / kPiece;
    const bool wide = (long long)pieces * kPiece * 3 <= (long long)per_row * 4;  // (at most a quarter of a row's last piece is idle)
    const long long blocks = wide ? ((long long)s.n * pieces + kEmbThreads / 32 - 1) / (kEmbThreads / 32)
                                  : ((long long)s.n * per_row + kEmbThreads * kEmbUnroll - 1) / (kEmbThreads * kEmbUnroll);
    const long long most = (long long)sms * 16;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    const long long step = (long long)grid.x * kEmbThreads * kEmbUnroll, row_step = step / per_row;
    const unsigned at_step = (unsigned)(step % per_row);
    const cudaError_t err = with_type(s.table_dtype, [&](auto tx) {
        return with_type(s.y_dtype, [&](auto ty) {
            using TX = typename decltype(tx)::type;
            using TY = typename decltype(ty)::type;
            auto go = [&](auto n) {
                constexpr int kN = n();
                return wide ? launch_dependent(k_embed_rows<TX, TY, kN>, grid, kEmbThreads, 0, 1, st, a, per_row, pieces, factor(pieces))
                            : launch_dependent(k_embed_units<TX, TY, kN>, grid, kEmbThreads, 0, 1, st, a, per_row, factor(per_row), row_step, at_step);
            };
            if constexpr (sizeof(TX) + sizeof(TY) == 4) {
                if (L == kEights) return go(std::integral_constant<int, 8>{});
            }
            return L == kOne ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 4>{});
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
    // (eights in fp32 too: its loads meet in the L1 cache; a table that starts anywhere, in a flat buffer, goes one by one: 65536 x 1024 into fp32
    // 119 us instead of 85)
    const Layout L = (uintptr_t)dtable % 16 != 0 ? kOne : s.d % 8 == 0 && s.ldy % 8 == 0 ? kEights : layout_of(s);
    const EmbArgs e = emb_args(s, ids, dy, dtable, ws);
    const long long zeroing = add ? 0 : ((long long)s.V * s.d * (s.table_dtype == RR_F32 ? 4 : 2) + 65535) / 65536;  // blocks that have 64 KB to zero
    // calls f(type of dy, type of dtable, layout)
    auto with_types = [&](auto f) {
        return with_type(s.table_dtype, [&](auto to) {
            return with_type(s.y_dtype, [&](auto ty) {
                using std::integral_constant;
                return L == kEights ? f(ty, to, integral_constant<Layout, kEights>{}) : L == kOne ? f(ty, to, integral_constant<Layout, kOne>{}) : f(ty, to, integral_constant<Layout, kQuads>{});
            });
        });
    };
    if (s.n <= kDirect) {
        SumArgs b = {};
        b.e = e;
        b.add = add;
        const int tiles = (s.d + kEmbThreads * 8 - 1) / (kEmbThreads * 8);
        const long long most = zeroing < 4 * sms ? zeroing : 4 * sms;
        const dim3 grid((unsigned)((long long)s.n * tiles + (most < s.V ? most : s.V)));
        const cudaError_t err = with_types([&](auto ty, auto to, auto layout) {
            return launch_dependent(k_embed_direct<typename decltype(ty)::type, typename decltype(to)::type, layout()>, grid, kEmbThreads, kMapWords * 4, 1, st, b, tiles);
        });
        return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
    }
    SortArgs a;
    a.e = e;
    a.slabs = (s.n + kSlab - 1) / kSlab;
    a.slab = (s.n + a.slabs - 1) / a.slabs;
    int bits = 1;
    while (bits < 31 && s.V >> bits) ++bits;  // (V itself is a key)
    a.passes = (bits + kDigitBits - 1) / kDigitBits;
    a.bits = (bits + a.passes - 1) / a.passes;
    a.key = l.key;
    a.pos = l.pos;
    a.runs = l.runs;
    a.out_f32 = s.table_dtype == RR_F32;
    int fillers = 0;
    if (!add) {
        const int most = sms - a.slabs > sms / 4 ? sms - a.slabs : sms / 4;  // (one block an SM: all at once)
        fillers = (int)(zeroing < most ? zeroing : most);
        if (fillers > s.V) fillers = s.V;
    }
    // (ids of up to 18 bits fit into a 32-bit word beside the place)
    cudaError_t err = bits <= 32 - kPlaceBits ? launch_sort<uint32_t>(a, a.slabs + fillers, st) : launch_sort<uint64_t>(a, a.slabs + fillers, st);
    int *key = l.key, *pos = l.pos, *key2 = l.key2, *pos2 = l.pos2;
    long long sorted = a.slab;
    while (err == cudaSuccess && sorted < s.n) {
        const bool few = sorted * 4 >= s.n;
        err = launch_dependent(few ? k_embed_merge<4> : k_embed_merge<8>, dim3((unsigned)((s.n + kEmbThreads - 1) / kEmbThreads)), kEmbThreads, 0, 1, st, (int)s.n,
                               (int)sorted, (const int *)key, (const int *)pos, key2, pos2);
        std::swap(key, key2);
        std::swap(pos, pos2);
        sorted *= few ? 4 : 8;
    }
    if (err != cudaSuccess) return RR_ERR_CUDA;
    SumArgs b;
    b.e = a.e;
    b.key = key;
    b.pos = pos;
    b.part = l.part;
    b.runs = l.runs;
    b.list = l.list;
    b.chunk = l.chunk;
    b.add = add;
    int threads = 32;
    while (threads < kEmbThreads && threads * 8 < s.d) threads <<= 1;
    const dim3 grid((unsigned)l.chunks, (unsigned)((s.d + threads * 8 - 1) / (threads * 8)));
    const int tiles = (s.d + kJoinCols * 8 - 1) / (kJoinCols * 8);
    const long long most_items = (long long)(s.n / (2 * l.chunk) + 1) * tiles;
    const dim3 join((unsigned)(most_items < 4 * sms ? most_items : 4 * sms));
    err = with_types([&](auto ty, auto to, auto layout) {
        return launch_dependent(k_embed_sum<typename decltype(ty)::type, typename decltype(to)::type, layout()>, grid, threads, 0, 1, st, b);
    });
    if (err == cudaSuccess)
        err = with_types([&](auto, auto to, auto layout) {
            return launch_dependent(k_embed_join<typename decltype(to)::type, layout()>, join, kJoin * kJoinCols, 0, 1, st, b, tiles);
        });
    return err == cudaSuccess ? RR_OK : RR_ERR_CUDA;
}

}  // namespace rr
