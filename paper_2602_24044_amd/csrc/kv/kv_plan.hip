// Block tables and slot maps of a step from its requests' lengths, and the list of pieces that its attention is cut into.
//
// Request i has l_i tokens in the cache and n_i new ones; it holds h_i blocks of 64 tokens, needs w_i = ceil((l_i + n_i) / 64), and
// takes max(0, w_i - h_i) blocks more: the lowest free ones, request after request.  A free block is a zero bit of `used`; the k-th
// free one is found by counting.  Everything is a prefix sum over requests or over bitmap words, integer and so the same whatever
// order the lanes run in.  The work is nothing and the time is latency: reads that hang on each other (row -> blocks held -> bitmap ->
// table) and barriers.  One launch for decode steps, two otherwise; one token 5.2 us, 32 requests 6.4, 29 prompts of 20462 tokens 7.9 + 4.0,
// 1000 requests of one token 16 + 4, 4000 of them 49 + 5.
#include "kv_internal.hpp"

#include <algorithm>

namespace lora {
namespace kv {
namespace {

// Exclusive sum over the workgroup's WAVES * 64 threads of N values each; total[] receives the sums.  sums: [WAVES][N] in LDS.
template <int WAVES, int N>
__device__ inline void scan(int (&v)[N], int (&total)[N], int (*sums)[N])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int own[N];
#pragma unroll
    for (int k = 0; k < N; ++k) own[k] = v[k];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int o = __shfl_up(v[k], d);
            if (lane >= d) v[k] += o;
        }
    __syncthreads();                       // the sums of the scan before have been read
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < N; ++k) sums[wave][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int s = sums[w][k];
            if (w < wave) before += s;
            all += s;
        }
        total[k] = all;
        v[k] += before - own[k];
    }
}

// Request i's lengths against its table row (own: the row exists and no earlier request has it).
__device__ inline bool lengths_ok(const PlanArgs& a, const Request& q, int add, bool own)
{
    return own && q.len >= 0 && add >= 0 && add <= a.max_new && q.len <= a.t.max_seq_tokens && add <= a.t.max_seq_tokens - q.len &&
           (q.len + kBlock - 1) / kBlock <= q.held;
}
// Token rows: `before` of the requests in front of it.  The sums stop at T + 1: what lies behind is outside of the step in any case.
__device__ inline int wanted_rows(const PlanArgs& a, int add) { return add < 0 ? 0 : min(add, a.T + 1); }
__device__ inline bool place_rows(const PlanArgs& a, Request& q, int before, int add, bool ok)
{
    const int rows = wanted_rows(a, add), first = min(before, a.T + 1);
    ok = ok && first + rows <= a.T;
    q.rows = max(0, min(first + rows, a.T) - first);
    q.first = min(first, a.T);
    q.want = ok ? max(q.held, (q.len + rows + kBlock - 1) / kBlock) : 0;
    return ok;
}
__device__ inline int blocks_of(const Request& q) { return q.held >= 0 ? (q.len + q.rows + kBlock - 1) / kBlock : 0; }
// Column tiles of a request's attention; returns the blocks that they read, all tiles together.  (A refused request's rows are set to
// zero by the kernel of few columns, however many they are.)
__device__ inline unsigned long long cut_columns(Request& q, int group)
{
    const int cols = q.rows * group;
    q.many = q.held >= 0 && cols > kFewMost;
    q.tiles = q.many ? (cols + kManyCols - 1) / kManyCols : (cols + kFewCols - 1) / kFewCols;
    return (unsigned long long)q.tiles * (unsigned)blocks_of(q);
}
// Blocks of a piece: the keys of every tile are cut so that all tiles and key heads together (`work` blocks a key head) make `items` pieces,
// and at most one more per tile.
__device__ inline int piece_blocks(unsigned long long work, int n_kv, int items, int least)
{
    const unsigned long long per = (work * n_kv + items - 1) / items;
    return ((int)(per < (unsigned)least ? least : per > kMaxBlocks ? kMaxBlocks : per) + 1) & ~1;
}
__device__ inline int merge_columns(const Request& q) { return q.splits < kMergeMany ? kMergeCols : 1; }
// v: entries (few, many), partial results (few, many), merges of the request.  A tile of few columns is cut into pieces of `chunk` blocks at
// most, one of many columns (whose pieces cost more to merge) stays whole up to one and a half.
__device__ inline void cut_keys(Request& q, int group, int chunk_few, int chunk_many, int (&v)[5])
{
    const int blocks = blocks_of(q), chunk = q.many ? chunk_many : chunk_few;
    q.splits = max(1, (blocks + (q.many ? chunk / 2 : chunk - 1)) / chunk);
    q.chunk = (blocks + q.splits - 1) / q.splits;
    const int pieces = q.tiles * q.splits, together = merge_columns(q);
    v[0] = q.many ? 0 : pieces;
    v[1] = q.many ? pieces : 0;
    v[2] = q.splits > 1 ? v[0] : 0;
    v[3] = q.splits > 1 ? v[1] : 0;
    v[4] = q.splits > 1 ? (q.rows * group + together - 1) / together : 0;
}
// Ends the lists behind their entries: what the step before had there is no longer any.  (The kernel of many columns reads how many there are.)
template <int THREADS> __device__ inline void end_lists(const Tables& t, int few, int many, int merge)
{
    const int tid = threadIdx.x;
    for (int k = few + tid; k < t.head->n_few; k += THREADS) t.few[k].rows = 0;
    for (int k = merge + tid; k < t.head->n_merge; k += THREADS) t.merge[k].rows = 0;
    __syncthreads();
    if (tid == 0) {
        t.head->n_few = few;
        t.head->n_many = many;
        t.head->n_merge = merge;
    }
}
__device__ inline uint32_t free_bits(const Tables& t, int w)
{
    if (w >= t.n_words) return 0u;
    const uint32_t free = ~t.used[w];
    return w == t.n_words - 1 && (t.n_blocks & 31) ? free & ((1u << (t.n_blocks & 31)) - 1) : free;
}

// What the plan has decided, written out: position and slot of row j of a request, entry k of its pieces, entry k of its merges.
// row: its row of the block table; fresh: the step's new blocks.
__device__ inline int block_at(const Request& q, const int32_t* row, const int32_t* fresh, int b) { return b < q.held ? row[b] : fresh[q.fresh + b - q.held]; }
__device__ inline void write_row(const Tables& t, const Request& q, const int32_t* row, const int32_t* fresh, int j)
{
    int position = -1, slot = -1;
    if (q.held >= 0) {
        position = q.len + j;
        slot = block_at(q, row, fresh, position / kBlock) * kBlock + position % kBlock;
    }
    t.position[q.first + j] = position;
    t.slot[q.first + j] = slot;
}
__device__ inline void write_entry(const Tables& t, const Request& q, const int32_t* row, const int32_t* fresh, int group, int k)
{
    const int cols = q.many ? kManyCols : kFewCols;
    Entry e = {};
    e.first = q.first;
    e.rows = q.rows;
    e.len = q.len;
    e.row = q.held >= 0 ? q.row : 0;
    e.tile = q.tiles - 1 - k / q.splits;               // the last tiles see the most keys: they come first
    e.block = (k % q.splits) * q.chunk;
    // the last token of the tile sees this many blocks
    const int last = min(q.rows - 1, ((e.tile + 1) * cols - 1) / group);
    const int seen = q.held >= 0 ? (q.len + last) / kBlock + 1 : 0;
    e.blocks = max(0, min(q.chunk, seen - e.block));
    e.part = q.splits > 1 ? q.part + k : -1;
#pragma unroll
    for (int j = 0; j < kEntryIds; ++j)
        if (j < e.blocks) e.id[j] = block_at(q, row, fresh, e.block + j);
    (q.many ? t.many : t.few)[q.entry + k] = e;
}
__device__ inline void write_merge(const Tables& t, const Request& q, int k)
{
    const int together = merge_columns(q), place = q.tiles - 1 - k * together / (q.many ? kManyCols : kFewCols);
    t.merge[q.merge + k] = Merge{q.first, q.rows, k * together, together, q.part + place * q.splits, q.splits, q.many, 0};
}
__device__ inline int32_t* table_row(const Tables& t, const Request& q) { return t.table + (size_t)(q.held >= 0 ? q.row : 0) * t.row_blocks; }

// Steps of up to kSmallThreads requests: a thread per request, which stays in registers (plan_kernel, which goes over lists in memory and
// has four times the waves at each barrier, takes 8.8 us for one request where this takes 3.9, 10.0 against 4.6 for 256).  Where no
// request has more than kSmallNew new tokens (so none needs more than one block) the same launch writes everything out: 5.2 us for one
// request where the second launch makes it 3.9 + 2.2, 7.5 for 256 requests of four tokens where it makes it 4.6 + 3.2.
constexpr int kSmallThreads = 256, kSmallNew = 4, kSmallRows = 1024;
__global__ __launch_bounds__(kSmallThreads) void plan_small_kernel(PlanArgs a)
{
    constexpr int W = kSmallThreads / 64, WORDS = 4;
    __shared__ int claim[kMaxSeqs];
    __shared__ int sums[W][5];
    __shared__ unsigned long long work[2];
    __shared__ int most;
    __shared__ int32_t fresh[kSmallThreads];
    __shared__ Request requests[kSmallThreads];
    const int i = threadIdx.x;
    const Tables& t = a.t;
    const int n = a.n;
    const bool mine = i < n;

    // everything that no other request decides is asked for first
    Request q = {};
    int add = 0;
    if (mine) {
        q.row = a.seq[i];
        q.len = a.len[i];
        add = a.add[i];
    }
    uint32_t free[WORDS];
#pragma unroll
    for (int k = 0; k < WORDS; ++k) free[k] = free_bits(t, kSmallThreads * k + i);
    const bool exists = mine && (unsigned)q.row < (unsigned)t.max_seqs;
    q.held = exists ? t.held[q.row] : -1;
    if (i < 2) work[i] = 0;
    if (i == 0) most = 0;
    // a row named twice belongs to the first request that names it
    if (exists) claim[q.row] = n;
    __syncthreads();
    if (exists) atomicMin(&claim[q.row], i);
    __syncthreads();
    bool ok = lengths_ok(a, q, add, exists && claim[q.row] == i);

    int v[1] = {wanted_rows(a, add)}, total[1];
    scan<W>(v, total, reinterpret_cast<int(*)[1]>(sums));
    ok = place_rows(a, q, v[0], add, ok) && mine;
    if (mine) t.start[i] = q.first;
    if (i == 0) {
        t.start[n] = min(total[0], a.T);
        t.head->rows = min(total[0], a.T);
    }
    v[0] = ok ? q.want - q.held : 0;
    scan<W>(v, total, reinterpret_cast<int(*)[1]>(sums));
    q.fresh = v[0];
    if (!ok) q.held = -1;
    const int need = total[0];

    // the first `need` free blocks in ascending order, which are in use from here on
    int found = 0;
    for (int base = 0; base < t.n_words && found < need; base += WORDS * kSmallThreads) {
        if (base)
#pragma unroll
            for (int k = 0; k < WORDS; ++k) free[k] = free_bits(t, base + kSmallThreads * k + i);
        int f[WORDS], in_words[WORDS];
#pragma unroll
        for (int k = 0; k < WORDS; ++k) f[k] = (int)__popc(free[k]);
        scan<W>(f, in_words, reinterpret_cast<int(*)[WORDS]>(sums));
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            int at = found + f[k];
            uint32_t bits = free[k];
            while (bits && at < need) {
                const int b = (base + kSmallThreads * k + i) * 32 + __ffs(bits) - 1;
                bits &= bits - 1;
                t.fresh[at] = b;
                if (at < kSmallThreads) fresh[at] = b;
                ++at;
            }
            if (bits != free[k]) t.used[base + kSmallThreads * k + i] = ~bits;
            found += in_words[k];
        }
    }
    found = min(found, need);

    // who gets them; how much attention has to read
    uint32_t flags = mine && !ok ? kFlagRefused : 0u;
    if (q.held >= 0 && q.want > q.held) {
        if (q.fresh + (q.want - q.held) > found) {
            flags |= kFlagExhausted;
            q.held = -1;
        } else {
            atomicMax(&most, q.fresh + (q.want - q.held));
        }
    }
    const unsigned long long w = cut_columns(q, a.group);
    if (w) atomicAdd(&work[q.many], w);
    __syncthreads();
    for (int k = most + i; k < found; k += kSmallThreads) {        // what nobody has got is free again
        const int b = t.fresh[k];
        atomicAnd(&t.used[b >> 5], ~(1u << (b & 31)));
    }
    int c[5], all[5];
    cut_keys(q, a.group, piece_blocks(work[0], a.n_kv, kFewItems, kFewChunk), piece_blocks(work[1], a.n_kv, kManyItems, kManyChunk), c);
    const int pieces = c[0] + c[1];
    scan<W>(c, all, sums);
    q.entry = q.many ? c[1] : c[0];
    q.part = q.many ? c[3] : c[2];
    q.merge = c[4];
    end_lists<kSmallThreads>(t, all[0], all[1], all[4]);
    if (flags) atomicOr(&t.head->flags, flags);
    if (!a.whole) {
        if (mine) t.request[i] = q;
        return;
    }

    int32_t* row = table_row(t, q);
    requests[i] = q;
    claim[i] = c[0] + c[1];                            // entries of the requests in front of it, in both lists together
    for (int j = 0; j < q.rows; ++j) write_row(t, q, row, fresh, j);
    if (pieces && q.splits > 1)
        for (int k = 0; k * merge_columns(q) < q.rows * a.group; ++k) write_merge(t, q, k);
    __syncthreads();
    for (int e = i; e < all[0] + all[1]; e += kSmallThreads) {
        int r = 0;                                     // the last request that begins at or before e
#pragma unroll
        for (int d = kSmallThreads / 2; d; d >>= 1)
            if (r + d < n && claim[r + d] <= e) r += d;
        write_entry(t, requests[r], table_row(t, requests[r]), fresh, a.group, e - claim[r]);
    }
    __syncthreads();                                   // the table has been read: the blocks that the step takes
    if (q.held >= 0 && q.want > q.held) {
        for (int b = q.held; b < q.want; ++b) row[b] = fresh[q.fresh + b - q.held];
        t.held[q.row] = q.want;
    }
}

// Steps of more requests, kPlanThreads at a time.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a)
{
    constexpr int W = kPlanThreads / 64;
    __shared__ int claim[kMaxSeqs];
    __shared__ int sums[W][5];
    __shared__ unsigned long long work[2];
    __shared__ int most;
    const int tid = threadIdx.x;
    const Tables& t = a.t;
    const int n = a.n;
    uint32_t flags = 0;

    for (int r = tid; r < t.max_seqs; r += kPlanThreads) claim[r] = n;
    if (tid < 2) work[tid] = 0;
    if (tid == 0) most = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kPlanThreads) {
        const int row = a.seq[i];
        if ((unsigned)row < (unsigned)t.max_seqs) atomicMin(&claim[row], i);
    }
    __syncthreads();

    // token rows and blocks of every request
    int rows0 = 0, need0 = 0;
    for (int base = 0; base < n; base += kPlanThreads) {
        const int i = base + tid;
        const bool mine = i < n;
        Request q = {};
        int add = 0;
        bool ok = false;
        if (mine) {
            q.row = a.seq[i];
            q.len = a.len[i];
            add = a.add[i];
            const bool own = (unsigned)q.row < (unsigned)t.max_seqs && claim[q.row] == i;
            q.held = own ? t.held[q.row] : -1;
            ok = lengths_ok(a, q, add, own);
        }
        int v[1] = {mine ? wanted_rows(a, add) : 0}, total[1];
        scan<W>(v, total, reinterpret_cast<int(*)[1]>(sums));
        ok = place_rows(a, q, rows0 + v[0], add, ok) && mine;
        rows0 = min(rows0 + total[0], a.T + 1);
        v[0] = ok ? q.want - q.held : 0;
        scan<W>(v, total, reinterpret_cast<int(*)[1]>(sums));
        q.fresh = need0 + v[0];
        need0 += total[0];
        if (!ok) q.held = -1;
        if (mine) {
            if (!ok) flags |= kFlagRefused;
            t.start[i] = q.first;
            t.request[i] = q;
        }
    }
    if (tid == 0) {
        t.start[n] = min(rows0, a.T);
        t.head->rows = min(rows0, a.T);
    }

    // the first need0 free blocks in ascending order, which are in use from here on; 32 of them a bitmap word
    int found = 0;
    for (int base = 0; base < t.n_words && found < need0; base += kPlanThreads) {
        uint32_t free = free_bits(t, base + tid);
        int v[1] = {(int)__popc(free)}, total[1];
        scan<W>(v, total, reinterpret_cast<int(*)[1]>(sums));
        int at = found + v[0];
        const uint32_t before = free;
        while (free && at < need0) {
            t.fresh[at++] = (base + tid) * 32 + __ffs(free) - 1;
            free &= free - 1;
        }
        if (free != before) t.used[base + tid] = ~free;
        found += total[0];
    }
    found = min(found, need0);

    // who gets them; how much attention has to read
    for (int i = tid; i < n; i += kPlanThreads) {
        Request q = t.request[i];
        if (q.held >= 0 && q.want > q.held) {
            if (q.fresh + (q.want - q.held) > found) {
                flags |= kFlagExhausted;
                q.held = -1;
            } else {
                atomicMax(&most, q.fresh + (q.want - q.held));
            }
        }
        const unsigned long long w = cut_columns(q, a.group);
        if (w) atomicAdd(&work[q.many], w);
        t.request[i] = q;
    }
    __syncthreads();
    for (int k = most + tid; k < found; k += kPlanThreads) {       // what nobody has got is free again
        const int b = t.fresh[k];
        atomicAnd(&t.used[b >> 5], ~(1u << (b & 31)));
    }

    const int chunk_few = piece_blocks(work[0], a.n_kv, kFewItems, kFewChunk), chunk_many = piece_blocks(work[1], a.n_kv, kManyItems, kManyChunk);
    int at[5] = {0, 0, 0, 0, 0};
    for (int base = 0; base < n; base += kPlanThreads) {
        const int i = base + tid;
        Request q = {};
        int v[5] = {0, 0, 0, 0, 0}, total[5];
        if (i < n) {
            q = t.request[i];
            cut_keys(q, a.group, chunk_few, chunk_many, v);
        }
        scan<W>(v, total, sums);
        if (i < n) {
            q.entry = q.many ? at[1] + v[1] : at[0] + v[0];
            q.part = q.many ? at[3] + v[3] : at[2] + v[2];
            q.merge = at[4] + v[4];
            t.request[i] = q;
        }
#pragma unroll
        for (int k = 0; k < 5; ++k) at[k] += total[k];
    }
    end_lists<kPlanThreads>(t, at[0], at[1], at[4]);
    if (flags) atomicOr(&t.head->flags, flags);
}

// Writes out what the plan of a longer step has decided: a workgroup per request and kFillRows of its token rows.
constexpr int kFillRows = 1024;
__global__ __launch_bounds__(256) void fill_kernel(PlanArgs a)
{
    const Tables& t = a.t;
    const Request q = t.request[blockIdx.x];
    int32_t* row = table_row(t, q);
    // (a refused request may have more rows than max_new, for which the grid was made)
    for (int j = blockIdx.y * 256 + (int)threadIdx.x; j < q.rows; j += gridDim.y * 256) write_row(t, q, row, t.fresh, j);
    if (blockIdx.y) return;
    if (q.held >= 0) {
        for (int b = q.held + (int)threadIdx.x; b < q.want; b += 256) row[b] = t.fresh[q.fresh + b - q.held];
        if (threadIdx.x == 0) t.held[q.row] = q.want;
    }
    for (int k = threadIdx.x; k < q.tiles * q.splits; k += 256) write_entry(t, q, row, t.fresh, a.group, k);
    if (q.splits > 1)
        for (int k = threadIdx.x; k * merge_columns(q) < q.rows * a.group; k += 256) write_merge(t, q, k);
}

__global__ __launch_bounds__(64) void release_kernel(Tables t, const int32_t* seq, const int32_t* keep)
{
    const int i = blockIdx.x;
    const int row = seq[i], tokens = keep ? keep[i] : 0;
    if ((unsigned)row >= (unsigned)t.max_seqs || tokens < 0) {
        if (threadIdx.x == 0) atomicOr(&t.head->flags, kFlagRefused);
        return;
    }
    const int k = (int)(((long)tokens + kBlock - 1) / kBlock);
    int held = 0;
    // a row named twice: whoever lowers the count gives back what lies in between
    if (threadIdx.x == 0) held = atomicMin(&t.held[row], k);
    held = __shfl(held, 0);
    int32_t* blocks = t.table + (size_t)row * t.row_blocks;
    // Blocks that a row got together mostly lie side by side: lanes whose bits are in one word put them together, and the last of them
    // takes them out (many rows' atomics on one word take their turns: 5.5 us for 29 rows of 11 blocks without this).
    const int lane = threadIdx.x;
    for (int from = k; from < held; from += 64) {
        const int b = from + lane;
        int word = -1;
        uint32_t bits = 0;
        if (b < held) {
            const int blk = blocks[b];
            blocks[b] = -1;
            word = blk >> 5;
            bits = 1u << (blk & 31);
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t other = __shfl_up(bits, d);
            const int its = __shfl_up(word, d);
            if (lane >= d && its == word) bits |= other;
        }
        const int next = __shfl_down(word, 1);
        if (word >= 0 && (lane == 63 || next != word)) atomicAnd(&t.used[word], ~bits);
    }
}

}  // namespace

hipError_t launch_plan(const PlanArgs& a, hipStream_t stream)
{
    PlanArgs b = a;
    // (T bounds what a refused request's rows cost one thread)
    b.whole = a.n <= kSmallThreads && a.max_new <= kSmallNew && a.T <= kSmallRows;
    if (a.n <= kSmallThreads) plan_small_kernel<<<1, kSmallThreads, 0, stream>>>(b);
    else plan_kernel<<<1, kPlanThreads, 0, stream>>>(b);
    if (a.n > 0 && !b.whole) {
        const int chunks = std::max(1, (a.max_new + kFillRows - 1) / kFillRows);
        fill_kernel<<<dim3(a.n, chunks), 256, 0, stream>>>(b);
    }
    return hipGetLastError();
}

hipError_t launch_release(const Tables& t, int n, const int32_t* seq, const int32_t* keep, hipStream_t stream)
{
    if (n > 0) release_kernel<<<n, 64, 0, stream>>>(t, seq, keep);
    return hipGetLastError();
}

}  // namespace kv
}  // namespace lora
