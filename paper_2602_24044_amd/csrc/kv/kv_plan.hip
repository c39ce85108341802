// Block tables and slot maps of a step from its requests' lengths, and the list of pieces that its attention is cut into.
//
// Request i has l_i tokens in the cache and n_i new ones; it holds h_i blocks of 64 tokens, needs w_i = ceil((l_i + n_i) / 64), and
// takes max(0, w_i - h_i) blocks more: the lowest free ones, request after request.  A free block is a zero bit of `used`; the k-th
// free one is found by counting.  Everything is a prefix sum over requests or over bitmap words, integer and so the same whatever
// order the lanes run in.
#include "kv_internal.hpp"

#include <algorithm>

namespace lora {
namespace kv {
namespace {

constexpr int kWaves = kPlanThreads / 64;

// Exclusive sum over the workgroup's threads of N values each; total[] receives the sums.  sums: [kWaves][N] in LDS.
template <int N>
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
        for (int w = 0; w < kWaves; ++w) {
            const int s = sums[w][k];
            if (w < wave) before += s;
            all += s;
        }
        total[k] = all;
        v[k] += before - own[k];
    }
}

// What the plan has decided, written out.  Position and slot of row j of a request; entry k of its list of pieces.
__device__ inline void write_row(const Tables& t, const Request& q, const int32_t* row, int j)
{
    int position = -1, slot = -1;
    if (q.held >= 0) {
        position = q.len + j;
        const int b = position / kBlock;
        slot = (b < q.held ? row[b] : t.fresh[q.fresh + b - q.held]) * kBlock + position % kBlock;
    }
    t.position[q.first + j] = position;
    t.slot[q.first + j] = slot;
}
__device__ inline void write_entry(const Tables& t, const Request& q, const int32_t* row, int group, int k)
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
    for (int j = 0; j < kEntryIds; ++j) {
        const int b = e.block + j;
        if (j < e.blocks) e.id[j] = b < q.held ? row[b] : t.fresh[q.fresh + b - q.held];
    }
    (q.many ? t.many : t.few)[q.entry + k] = e;
}
__device__ inline int merge_columns(const Request& q) { return q.splits < kMergeMany ? kMergeCols : 1; }
__device__ inline void write_merge(const Tables& t, const Request& q, int k)
{
    const int together = merge_columns(q), place = q.tiles - 1 - k * together / (q.many ? kManyCols : kFewCols);
    t.merge[q.merge + k] = Merge{q.first, q.rows, k * together, together, q.part + place * q.splits, q.splits, q.many, 0};
}
__device__ inline int32_t* table_row(const Tables& t, const Request& q) { return t.table + (size_t)(q.held >= 0 ? q.row : 0) * t.row_blocks; }

// A step of up to kPlanThreads requests with a few tokens each is written out by the same workgroup, a thread per request and then per entry.
constexpr int kSmallNew = 4;
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a)
{
    __shared__ int claim[kMaxSeqs];
    __shared__ int sums[kWaves][5];
    __shared__ unsigned long long work[2];
    const int tid = threadIdx.x;
    const Tables& t = a.t;
    const int n = a.n, T = a.T;
    uint32_t flags = 0;

    // a row named twice belongs to the first request that names it
    for (int r = tid; r < t.max_seqs; r += kPlanThreads) claim[r] = n;
    if (tid < 2) work[tid] = 0;
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
        Request q = {};
        bool ok = false;
        int add = 0;
        if (i < n) {
            q.row = a.seq[i];
            q.len = a.len[i];
            add = a.add[i];
            const bool own = (unsigned)q.row < (unsigned)t.max_seqs && claim[q.row] == i;
            q.held = own ? t.held[q.row] : -1;
            ok = own && q.len >= 0 && add >= 0 && add <= a.max_new && q.len <= t.max_seq_tokens && add <= t.max_seq_tokens - q.len &&
                 (q.len + kBlock - 1) / kBlock <= q.held;
        }
        // the sums stop at T + 1: what lies behind is outside of the step in any case
        int v[1] = {add < 0 ? 0 : min(add, T + 1)}, total[1];
        const int mine = v[0];
        scan<1>(v, total, reinterpret_cast<int(*)[1]>(sums));
        q.first = min(rows0 + v[0], T + 1);
        rows0 = min(rows0 + total[0], T + 1);
        ok = ok && q.first + mine <= T;
        if (i < n) {
            q.rows = max(0, min(q.first + mine, T) - q.first);
            q.first = min(q.first, T);
            t.start[i] = q.first;
            q.want = ok ? max(q.held, (q.len + mine + kBlock - 1) / kBlock) : 0;
            if (!ok) flags |= kFlagRefused;
        }
        int w[1] = {ok ? q.want - q.held : 0}, wt[1];
        scan<1>(w, wt, reinterpret_cast<int(*)[1]>(sums));
        q.fresh = need0 + w[0];
        need0 += wt[0];
        if (i < n) {
            if (!ok) q.held = -1;
            t.request[i] = q;
        }
    }
    if (tid == 0) {
        t.start[n] = min(rows0, T);
        t.head->rows = min(rows0, T);
    }

    // the first need0 free blocks in ascending order; 32 of them a bitmap word
    int found = 0;
    for (int base = 0; base < t.n_words && found < need0; base += kPlanThreads) {
        const int w = base + tid;
        uint32_t free = w < t.n_words ? ~t.used[w] : 0u;
        if (w == t.n_words - 1 && (t.n_blocks & 31)) free &= (1u << (t.n_blocks & 31)) - 1;
        int v[1] = {(int)__popc(free)}, total[1];
        scan<1>(v, total, reinterpret_cast<int(*)[1]>(sums));
        int at = found + v[0];
        while (free && at < need0) {
            const int b = __ffs(free) - 1;
            free &= free - 1;
            t.fresh[at++] = w * 32 + b;
        }
        found += total[0];
    }
    found = min(found, need0);

    // who gets them; how much attention has to read
    int taken = 0;
    unsigned long long mine0 = 0, mine1 = 0;
    for (int i = tid; i < n; i += kPlanThreads) {
        Request q = t.request[i];
        if (q.held >= 0) {
            if (q.want > q.held && q.fresh + (q.want - q.held) > found) {
                flags |= kFlagExhausted;
                q.held = -1;
            } else {
                taken = max(taken, q.want > q.held ? q.fresh + (q.want - q.held) : 0);
            }
        }
        // (a refused request's rows are set to zero by the kernel of few columns, however many they are)
        const int cols = q.rows * a.group;
        q.many = q.held >= 0 && cols > kFewMost;
        q.tiles = q.many ? (cols + kManyCols - 1) / kManyCols : (cols + kFewCols - 1) / kFewCols;
        if (q.held >= 0) {
            const unsigned long long w = (unsigned long long)q.tiles * (unsigned)((q.len + q.rows + kBlock - 1) / kBlock);
            (q.many ? mine1 : mine0) += w;
        }
        t.request[i] = q;
    }
    if (mine0) atomicAdd(&work[0], mine0);
    if (mine1) atomicAdd(&work[1], mine1);
    for (int d = 32; d; d >>= 1) taken = max(taken, __shfl_xor(taken, d));
    __syncthreads();
    if ((tid & 63) == 0) sums[tid >> 6][0] = taken;
    __syncthreads();
    taken = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) taken = max(taken, sums[w][0]);
    for (int k = tid; k < taken; k += kPlanThreads) {
        const int b = t.fresh[k];
        atomicOr(&t.used[b >> 5], 1u << (b & 31));
    }

    // pieces of attention: the keys of every tile are cut so that all tiles and key heads together make kFewItems (kManyItems) pieces, and
    // at most one more per tile; a tile of up to one and a half pieces stays whole
    auto cut = [&](unsigned long long w, int items, int least) {
        const unsigned long long per = (w * a.n_kv + items - 1) / items;
        return ((int)(per < (unsigned)least ? least : per > kMaxBlocks ? kMaxBlocks : per) + 3) & ~3;
    };
    const int chunk0 = cut(work[0], kFewItems, kFewChunk), chunk1 = cut(work[1], kManyItems, kManyChunk);
    int at[5] = {0, 0, 0, 0, 0};                       // entries, partial results (few, many), merges
    for (int base = 0; base < n; base += kPlanThreads) {
        const int i = base + tid;
        Request q = {};
        int v[5] = {0, 0, 0, 0, 0}, total[5];
        if (i < n) {
            q = t.request[i];
            const int blocks = q.held >= 0 ? (q.len + q.rows + kBlock - 1) / kBlock : 0;
            const int chunk = q.many ? chunk1 : chunk0;
            q.splits = max(1, (blocks + (q.many ? chunk / 2 : chunk - 1)) / chunk);
            q.chunk = (blocks + q.splits - 1) / q.splits;
            const int pieces = q.tiles * q.splits;
            v[0] = q.many ? 0 : pieces;
            v[1] = q.many ? pieces : 0;
            v[2] = q.splits > 1 ? v[0] : 0;
            v[3] = q.splits > 1 ? v[1] : 0;
            const int together = merge_columns(q);
            v[4] = q.splits > 1 ? (q.rows * a.group + together - 1) / together : 0;
        }
        scan<5>(v, total, sums);
        if (i < n) {
            q.entry = q.many ? at[1] + v[1] : at[0] + v[0];
            q.part = q.many ? at[3] + v[3] : at[2] + v[2];
            q.merge = at[4] + v[4];
            t.request[i] = q;
        }
#pragma unroll
        for (int k = 0; k < 5; ++k) at[k] += total[k];
    }
    // what the lists of the step before had behind these
    for (int k = at[0] + tid; k < t.head->n_few; k += kPlanThreads) t.few[k].rows = 0;
    for (int k = at[1] + tid; k < t.head->n_many; k += kPlanThreads) t.many[k].rows = 0;
    for (int k = at[4] + tid; k < t.head->n_merge; k += kPlanThreads) t.merge[k].rows = 0;
    __syncthreads();
    if (tid == 0) {
        t.head->n_few = at[0];
        t.head->n_many = at[1];
        t.head->n_merge = at[4];
    }
    if (flags) atomicOr(&t.head->flags, flags);
    if (!a.whole) return;

    // (claim[] becomes the requests' first entries, in both lists together)
    __syncthreads();
    Request q = {};
    if (tid < n) {
        q = t.request[tid];
        int32_t* row = table_row(t, q);
        for (int j = 0; j < q.rows; ++j) write_row(t, q, row, j);
        if (q.splits > 1)
            for (int k = 0; k * merge_columns(q) < q.rows * a.group; ++k) write_merge(t, q, k);
    }
    int v[1] = {tid < n ? q.tiles * q.splits : 0}, total[1];
    scan<1>(v, total, reinterpret_cast<int(*)[1]>(sums));
    claim[tid] = v[0];
    __syncthreads();
    for (int e = tid; e < total[0]; e += kPlanThreads) {
        int i = 0;                                     // the last request that begins at or before e
#pragma unroll
        for (int d = kPlanThreads / 2; d; d >>= 1)
            if (i + d < n && claim[i + d] <= e) i += d;
        const Request r = t.request[i];
        write_entry(t, r, table_row(t, r), a.group, e - claim[i]);
    }
    __syncthreads();                                   // the table has been read: the blocks that the step takes
    if (tid < n && q.held >= 0 && q.want > q.held) {
        int32_t* row = table_row(t, q);
        for (int b = q.held; b < q.want; ++b) row[b] = t.fresh[q.fresh + b - q.held];
        t.held[q.row] = q.want;
    }
}

// Longer steps: a workgroup per request and kFillRows of its token rows.
constexpr int kFillRows = 1024;
__global__ __launch_bounds__(256) void fill_kernel(PlanArgs a)
{
    const Tables& t = a.t;
    const Request q = t.request[blockIdx.x];
    int32_t* row = table_row(t, q);
    // (a refused request may have more rows than max_new, for which the grid was made)
    for (int j = blockIdx.y * 256 + (int)threadIdx.x; j < q.rows; j += gridDim.y * 256) write_row(t, q, row, j);
    if (blockIdx.y) return;
    if (q.held >= 0) {
        for (int b = q.held + (int)threadIdx.x; b < q.want; b += 256) row[b] = t.fresh[q.fresh + b - q.held];
        if (threadIdx.x == 0) t.held[q.row] = q.want;
    }
    for (int k = threadIdx.x; k < q.tiles * q.splits; k += 256) write_entry(t, q, row, a.group, k);
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
    for (int b = k + (int)threadIdx.x; b < held; b += 64) {
        const int blk = blocks[b];
        blocks[b] = -1;
        atomicAnd(&t.used[blk >> 5], ~(1u << (blk & 31)));
    }
}

}  // namespace

hipError_t launch_plan(const PlanArgs& a, hipStream_t stream)
{
    // (T bounds what a refused request's rows cost one thread)
    const bool whole = a.n <= kPlanThreads && a.T <= 4 * kPlanThreads && a.max_new <= kSmallNew;
    PlanArgs b = a;
    b.whole = whole;
    plan_kernel<<<1, kPlanThreads, 0, stream>>>(b);
    if (a.n > 0 && !whole) {
        const int chunks = std::max(1, (a.max_new + kFillRows - 1) / kFillRows);
        fill_kernel<<<dim3(a.n, chunks), 256, 0, stream>>>(a);
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
