// Host side of the key/value cache in four bits: argument checks, layout of the slab, launches behind the lora_kv_* calls.
#include "../../../include/lora_mi355.h"
#include "../lora_internal.hpp"
#include "kv_internal.hpp"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

using namespace lora;
using namespace lora::kv;

#define KV_HIP_FAIL(call) note_hip_failure((call), #call)

namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

bool valid_heads(int32_t n_heads, int32_t n_kv, int32_t dim)
{
    return n_kv >= 1 && n_heads >= n_kv && n_heads <= kMaxHeads && n_heads % n_kv == 0 && (dim == 64 || dim == 128);
}

int row_blocks_of(const lora_kv_config* c) { return (c->max_seq_tokens + kBlock - 1) / kBlock; }

lora_status check_config(const lora_kv_config* c)
{
    if (!c) return LORA_ERR_INVALID_ARG;
    if (c->n_layers < 1 || c->n_layers > kMaxLayers || c->n_blocks < 1 || c->n_blocks > kMaxBlocks || c->max_seqs < 1 ||
        c->max_seqs > kMaxSeqs || c->max_seq_tokens < 1 || c->max_seq_tokens > kMaxSeqTokens || c->max_tokens < 1 ||
        c->max_tokens > kMaxTokens)
        return LORA_ERR_INVALID_ARG;
    if ((long)c->max_seqs * row_blocks_of(c) >= (1l << 31)) return LORA_ERR_INVALID_ARG;
    if (!valid_heads(c->n_heads, c->n_kv_heads, c->head_dim)) return LORA_ERR_SHAPE;
    return LORA_OK;
}

struct Layout {
    size_t layer_bytes = 0;
    size_t cache = 0, table = 0, held = 0, used = 0, head = 0, fresh = 0, start = 0, position = 0, slot = 0, request = 0, few = 0,
           many = 0, merge = 0, few_acc = 0, few_ml = 0, many_acc = 0, many_ml = 0, total = 0;
};

// Entries that the lists of a step of T tokens in n requests can have: one a tile, and at most kFewItems (kManyItems) more, counted
// with the key heads, where tiles are cut along their keys.
long most_few(long T, long n, int group, int n_kv) { return T * group / kFewCols + n + kFewItems / n_kv + 1; }
long most_many(long T, long n, int group, int n_kv) { return T * group / kManyCols + std::min(n, T * group / kFewMost) + kManyItems / n_kv + 1; }

Layout make_layout(const lora_kv_config* c)
{
    Layout L;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes); return at; };
    const size_t seqs = c->max_seqs, T = c->max_tokens, group = c->n_heads / c->n_kv_heads;
    L.layer_bytes = align_up((size_t)c->n_blocks * c->n_kv_heads * part_bytes(c->head_dim));
    L.cache = take(L.layer_bytes * (size_t)c->n_layers);
    L.table = take(4 * seqs * (size_t)row_blocks_of(c));
    L.held = take(4 * seqs);
    L.used = take(4 * (((size_t)c->n_blocks + 31) / 32));
    L.head = take(sizeof(Header));
    L.fresh = take(4 * std::min<size_t>((size_t)c->n_blocks, T / kBlock + seqs + 1));
    L.start = take(4 * (seqs + 1));
    L.position = take(4 * T);
    L.slot = take(4 * T);
    L.request = take(sizeof(Request) * seqs);
    const int n_kv = c->n_kv_heads;
    const size_t few = (size_t)most_few(T, seqs, (int)group, n_kv), many = (size_t)most_many(T, seqs, (int)group, n_kv);
    // (and one that says that the list has ended)
    L.few = take(sizeof(Entry) * (few + 1));
    L.many = take(sizeof(Entry) * many);
    L.merge = take(sizeof(Merge) * (T * group + 1));
    // a cut tile has a partial result per piece, and its pieces are at least half of what a cut is aimed at; nor are there more than the
    // smallest pieces make
    auto parts = [&](size_t items, size_t entries, int least) {
        const size_t splits = ((size_t)row_blocks_of(c) + least - 1) / least;
        return std::min((2 * items / n_kv + 2), splits > 1 ? entries * splits : 0) * n_kv;
    };
    const size_t pf = parts(kFewItems, few, kFewChunk), pm = T * group > (size_t)kFewMost ? parts(kManyItems, many, kManyChunk) : 0;
    L.few_acc = take(4 * pf * kFewCols * (size_t)c->head_dim);
    L.few_ml = take(4 * pf * kFewCols * 2);
    L.many_acc = take(4 * pm * kManyCols * (size_t)c->head_dim);
    L.many_ml = take(4 * pm * kManyCols * 2);
    L.total = o;
    return L;
}

int compute_units()
{
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) {
        (void)hipGetLastError();
        return 256;
    }
    return n;
}

// Strides of 0 become dense ones; false: a stride or an address that the kernels do not take.
bool fix_operand(const void* p, int64_t& stride, int64_t width)
{
    if (!p) return true;
    if (stride == 0) stride = width;
    return stride >= width && stride % 8 == 0 && stride < (1ll << 40) && !misaligned(p, 16);
}

bool fill_heads(const lora_heads* h, int n_heads, int n_kv, int dim, HeadsArgs& a)
{
    std::memset(&a, 0, sizeof a);
    a.q = static_cast<const uint16_t*>(h->d_q);
    a.k = static_cast<const uint16_t*>(h->d_k);
    a.v = static_cast<const uint16_t*>(h->d_v);
    a.q_out = static_cast<uint16_t*>(h->d_q_out);
    a.k_out = static_cast<uint16_t*>(h->d_k_out);
    a.q_stride = h->q_stride;
    a.k_stride = h->k_stride;
    a.v_stride = h->v_stride;
    a.q_out_stride = h->q_out_stride;
    a.k_out_stride = h->k_out_stride;
    const int64_t wq = (int64_t)n_heads * dim, wk = (int64_t)n_kv * dim;
    if (!fix_operand(a.q, a.q_stride, wq) || !fix_operand(a.q_out, a.q_out_stride, wq) || !fix_operand(a.k, a.k_stride, wk) ||
        !fix_operand(a.k_out, a.k_out_stride, wk) || !fix_operand(a.v, a.v_stride, wk))
        return false;
    if ((a.q != nullptr) != (a.q_out != nullptr)) return false;
    if ((a.q && a.q == a.q_out && a.q_stride != a.q_out_stride) || (a.k && a.k == a.k_out && a.k_stride != a.k_out_stride)) return false;
    a.q_norm = static_cast<const uint16_t*>(h->d_q_norm);
    a.k_norm = static_cast<const uint16_t*>(h->d_k_norm);
    a.inv_freq = h->d_inv_freq;
    if (misaligned(a.q_norm, 16) || misaligned(a.k_norm, 16) || misaligned(a.inv_freq, 4)) return false;
    if (!(h->eps >= 0.f) || std::isinf(h->eps)) return false;
    if (h->pairing != LORA_ROTATE_HALVES && h->pairing != LORA_ROTATE_NEIGHBOURS) return false;
    a.eps = h->eps;
    a.pairs = h->pairing == LORA_ROTATE_NEIGHBOURS;
    a.n_heads = n_heads;
    a.n_kv = n_kv;
    return true;
}

}  // namespace

struct lora_kv {
    lora_kv_config cfg;
    Layout L;
    char* base = nullptr;
    int device = -1;
    int n_cus = 256;
    hipEvent_t ev = nullptr;
    hipStream_t last = nullptr;     // stream of the latest call that enqueued work outside of a capture
    bool have_last = false;
    uint64_t epoch = 0;             // of the latest lora_kv_extend / lora_kv_release
    int32_t step_n = -1, step_T = -1;   // of the latest step, -1: none, or ended by a release
    int32_t step_most = 0;              // no request of it has more new tokens

    template <typename Tp> Tp* at(size_t off) const { return reinterpret_cast<Tp*>(base + off); }
    uint8_t* layer(int l) const { return at<uint8_t>(L.cache + L.layer_bytes * (size_t)l); }
    Tables tables() const
    {
        Tables t;
        t.head = at<Header>(L.head);
        t.table = at<int32_t>(L.table);
        t.held = at<int32_t>(L.held);
        t.used = at<uint32_t>(L.used);
        t.fresh = at<int32_t>(L.fresh);
        t.start = at<int32_t>(L.start);
        t.position = at<int32_t>(L.position);
        t.slot = at<int32_t>(L.slot);
        t.request = at<Request>(L.request);
        t.few = at<Entry>(L.few);
        t.many = at<Entry>(L.many);
        t.merge = at<Merge>(L.merge);
        t.n_blocks = cfg.n_blocks;
        t.n_words = (cfg.n_blocks + 31) / 32;
        t.max_seqs = cfg.max_seqs;
        t.row_blocks = row_blocks_of(&cfg);
        t.max_seq_tokens = cfg.max_seq_tokens;
        return t;
    }

    // Called in front of every launch: the cache's device must be current, and a stream other than the previous call's waits for
    // that call, unless it is being captured (see the header).  Where the previous call's is, an event recorded on it would draw the
    // other stream into the capture: such a call is refused.
    lora_status enter(hipStream_t s)
    {
        int dev = -1;
        if (KV_HIP_FAIL(hipGetDevice(&dev))) return LORA_ERR_HIP;
        if (dev != device) return LORA_ERR_INVALID_ARG;
        hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
        if (KV_HIP_FAIL(hipStreamIsCapturing(s, &cs))) return LORA_ERR_HIP;
        if (cs != hipStreamCaptureStatusNone) return LORA_OK;
        if (have_last && last != s) {
            // (the default stream is never captured, and asking about it is an error while others are)
            bool ordered = !last || !KV_HIP_FAIL(hipStreamIsCapturing(last, &cs));
            if (cs != hipStreamCaptureStatusNone) return LORA_ERR_INVALID_ARG;
            ordered = ordered && !KV_HIP_FAIL(hipEventRecord(ev, last)) && !KV_HIP_FAIL(hipStreamWaitEvent(s, ev, 0));
            // (its stream is gone, against the header: the device's work is waited for, and later calls do not meet it again)
            if (!ordered && KV_HIP_FAIL(hipDeviceSynchronize())) return LORA_ERR_HIP;
        }
        last = s;
        have_last = true;
        return LORA_OK;
    }
    // In front of the launches that change the tables: where one of them fails, others may have run.
    void end_step()
    {
        ++epoch;
        step_n = step_T = -1;
    }
    bool current(const lora_kv_step* st) const
    {
        return st && step_n >= 0 && st->epoch == epoch && st->n == step_n && st->T == step_T;
    }
};

extern "C" {

size_t lora_kv_slab_bytes(const lora_kv_config* cfg)
{
    return check_config(cfg) == LORA_OK ? make_layout(cfg).total : 0;
}

lora_status lora_kv_create(const lora_kv_config* cfg, lora_kv** out)
{
    if (!out) return LORA_ERR_INVALID_ARG;
    *out = nullptr;
    if (const lora_status st = check_config(cfg); st != LORA_OK) return st;
    if (!cfg->slab || misaligned(cfg->slab, kAlign)) return LORA_ERR_INVALID_ARG;
    lora_kv* k = new (std::nothrow) lora_kv();
    if (!k) return LORA_ERR_OOM;
    k->cfg = *cfg;
    k->L = make_layout(cfg);
    k->base = static_cast<char*>(cfg->slab);
    if (cfg->slab_bytes < k->L.total) {
        delete k;
        return LORA_ERR_OOM;
    }
    bool ok = !KV_HIP_FAIL(hipGetDevice(&k->device)) && !KV_HIP_FAIL(hipEventCreateWithFlags(&k->ev, hipEventDisableTiming));
    if (ok) {
        k->n_cus = compute_units();
        // everything starts at zero: stale codes and exponents stand for finite numbers from the start.  (The memory may be fresh from
        // another use whose last write is still in a stream's queue, which the fills do not wait for by themselves.)
        ok = !KV_HIP_FAIL(hipDeviceSynchronize()) && !KV_HIP_FAIL(launch_fill_i32(k->at<int32_t>(0), 0, k->L.total / 4, nullptr)) &&
             !KV_HIP_FAIL(launch_fill_i32(k->at<int32_t>(k->L.table), -1, (size_t)cfg->max_seqs * row_blocks_of(cfg), nullptr)) &&
             !KV_HIP_FAIL(hipDeviceSynchronize());
    }
    if (!ok) {
        lora_kv_destroy(k);
        return LORA_ERR_HIP;
    }
    *out = k;
    return LORA_OK;
}

lora_status lora_kv_destroy(lora_kv* k)
{
    if (!k) return LORA_ERR_INVALID_ARG;
    if (k->ev) {
        int dev = -1;
        (void)hipGetDevice(&dev);
        if (dev != k->device) (void)hipSetDevice(k->device);
        (void)hipDeviceSynchronize();
        (void)hipEventDestroy(k->ev);
        if (dev >= 0 && dev != k->device) (void)hipSetDevice(dev);
    }
    delete k;
    return LORA_OK;
}

lora_status lora_kv_extend(lora_kv* k, int32_t n, const int32_t* d_seq, const int32_t* d_len, const int32_t* d_new, int32_t T, int32_t max_new,
                           lora_kv_step* out, void* stream)
{
    if (!k || !out || n < 0 || n > k->cfg.max_seqs || T < 0 || T > k->cfg.max_tokens || max_new < 0) return LORA_ERR_INVALID_ARG;
    if (n > 0 && (!d_seq || !d_len || !d_new || misaligned(d_seq, 4) || misaligned(d_len, 4) || misaligned(d_new, 4))) return LORA_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (const lora_status st = k->enter(s); st != LORA_OK) return st;
    PlanArgs a;
    a.t = k->tables();
    a.seq = d_seq;
    a.len = d_len;
    a.add = d_new;
    a.n = n;
    a.T = T;
    a.max_new = std::min(max_new, T);
    a.n_kv = k->cfg.n_kv_heads;
    a.group = k->cfg.n_heads / k->cfg.n_kv_heads;
    a.whole = 0;
    k->end_step();
    if (KV_HIP_FAIL(launch_plan(a, s))) return LORA_ERR_HIP;
    k->step_n = n;
    k->step_T = T;
    k->step_most = a.max_new;
    out->start = a.t.start;
    out->position = a.t.position;
    out->slot = a.t.slot;
    out->table = a.t.table;
    out->held = a.t.held;
    out->row_blocks = a.t.row_blocks;
    out->n = n;
    out->T = T;
    out->epoch = k->epoch;
    return LORA_OK;
}

lora_status lora_kv_release(lora_kv* k, int32_t n, const int32_t* d_seq, const int32_t* d_keep, void* stream)
{
    if (!k || n < 0 || (n > 0 && (!d_seq || misaligned(d_seq, 4))) || misaligned(d_keep, 4)) return LORA_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (const lora_status st = k->enter(s); st != LORA_OK) return st;
    k->end_step();
    return KV_HIP_FAIL(launch_release(k->tables(), n, d_seq, d_keep, s)) ? LORA_ERR_HIP : LORA_OK;
}

lora_status lora_head_norm_rotate(int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, const int32_t* d_position,
                                  const lora_heads* heads, void* stream)
{
    if (!heads || T < 0 || T > kMaxTokens || heads->d_v) return LORA_ERR_INVALID_ARG;
    if (!valid_heads(n_heads, n_kv_heads, head_dim)) return LORA_ERR_SHAPE;
    HeadsArgs a;
    if (!fill_heads(heads, n_heads, n_kv_heads, head_dim, a)) return LORA_ERR_INVALID_ARG;
    if ((a.k != nullptr) != (a.k_out != nullptr) || (!a.q && !a.k)) return LORA_ERR_INVALID_ARG;
    if (a.inv_freq && T > 0 && (!d_position || misaligned(d_position, 4))) return LORA_ERR_INVALID_ARG;
    a.position = d_position;
    a.T = T;
    return KV_HIP_FAIL(launch_heads(a, head_dim, static_cast<hipStream_t>(stream))) ? LORA_ERR_HIP : LORA_OK;
}

lora_status lora_kv_store(lora_kv* k, int32_t layer, const lora_kv_step* step, const lora_heads* heads, void* stream)
{
    if (!k || !heads || layer < 0 || layer >= k->cfg.n_layers || !k->current(step)) return LORA_ERR_INVALID_ARG;
    HeadsArgs a;
    if (!fill_heads(heads, k->cfg.n_heads, k->cfg.n_kv_heads, k->cfg.head_dim, a) || a.k_out) return LORA_ERR_INVALID_ARG;
    if (step->T == 0) return LORA_OK;
    if (!a.k || !a.v) return LORA_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (const lora_status st = k->enter(s); st != LORA_OK) return st;
    const Tables t = k->tables();
    a.position = t.position;
    a.slot = t.slot;
    a.head = t.head;
    a.cache = k->layer(layer);
    a.T = step->T;
    return KV_HIP_FAIL(launch_heads(a, k->cfg.head_dim, s)) ? LORA_ERR_HIP : LORA_OK;
}

lora_status lora_kv_attend(lora_kv* k, int32_t layer, const lora_kv_step* step, float scale, const void* d_q, int64_t q_stride, void* d_out,
                           int64_t out_stride, void* stream)
{
    if (!k || layer < 0 || layer >= k->cfg.n_layers || !k->current(step) || !std::isfinite(scale)) return LORA_ERR_INVALID_ARG;
    if (step->T == 0) return LORA_OK;
    const int64_t width = (int64_t)k->cfg.n_heads * k->cfg.head_dim;
    if (!d_q || !d_out || d_q == d_out || !fix_operand(d_q, q_stride, width) || !fix_operand(d_out, out_stride, width)) return LORA_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (const lora_status st = k->enter(s); st != LORA_OK) return st;
    AttendArgs a;
    a.t = k->tables();
    a.cache = k->layer(layer);
    a.q = static_cast<const uint16_t*>(d_q);
    a.out = static_cast<uint16_t*>(d_out);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.few_acc = k->at<float>(k->L.few_acc);
    a.few_ml = k->at<float>(k->L.few_ml);
    a.many_acc = k->at<float>(k->L.many_acc);
    a.many_ml = k->at<float>(k->L.many_ml);
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.T = step->T;
    a.n_kv = k->cfg.n_kv_heads;
    a.group = k->cfg.n_heads / k->cfg.n_kv_heads;
    const long few = most_few(step->T, step->n, a.group, a.n_kv);
    const long many = (long)k->step_most * a.group > kFewMost ? most_many(step->T, step->n, a.group, a.n_kv) : 0;
    a.n_few = (int)few;
    a.n_many = (int)many;
    a.n_merge = step->T * a.group;
    a.n_cus = k->n_cus;
    return KV_HIP_FAIL(launch_attend(a, k->cfg.head_dim, step->n, s)) ? LORA_ERR_HIP : LORA_OK;
}

lora_status lora_kv_read(lora_kv* k, int32_t layer, int32_t n, const int32_t* d_seq, const int32_t* d_position, void* d_k_out, void* d_v_out,
                         void* stream)
{
    if (!k || layer < 0 || layer >= k->cfg.n_layers || n < 0 || n > kMaxTokens * 16) return LORA_ERR_INVALID_ARG;
    if (n > 0 && (!d_seq || !d_position || misaligned(d_seq, 4) || misaligned(d_position, 4))) return LORA_ERR_INVALID_ARG;
    if (misaligned(d_k_out, 16) || misaligned(d_v_out, 16)) return LORA_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (const lora_status st = k->enter(s); st != LORA_OK) return st;
    ReadArgs a;
    a.t = k->tables();
    a.cache = k->layer(layer);
    a.seq = d_seq;
    a.position = d_position;
    a.k_out = static_cast<uint16_t*>(d_k_out);
    a.v_out = static_cast<uint16_t*>(d_v_out);
    a.n = n;
    a.n_kv = k->cfg.n_kv_heads;
    return KV_HIP_FAIL(launch_read(a, k->cfg.head_dim, s)) ? LORA_ERR_HIP : LORA_OK;
}

lora_status lora_kv_poll_flags(lora_kv* k, uint32_t* flags, void* stream)
{
    if (!k) return LORA_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (KV_HIP_FAIL(hipStreamIsCapturing(s, &cs))) return LORA_ERR_HIP;
    if (cs != hipStreamCaptureStatusNone) return LORA_ERR_INVALID_ARG;
    if (const lora_status st = k->enter(s); st != LORA_OK) return st;
    uint32_t word = 0;
    uint32_t* d = &k->tables().head->flags;
    if (KV_HIP_FAIL(hipMemcpyAsync(&word, d, sizeof word, hipMemcpyDeviceToHost, s)) ||
        KV_HIP_FAIL(launch_fill_i32(reinterpret_cast<int32_t*>(d), 0, 1, s)) || KV_HIP_FAIL(hipStreamSynchronize(s)))
        return LORA_ERR_HIP;
    if (flags) *flags = word;
    if (word & kFlagRefused) return LORA_ERR_KV_REFUSED;
    if (word & kFlagExhausted) return LORA_ERR_KV_EXHAUSTED;
    if (word & kFlagNotFinite) return LORA_ERR_NOT_FINITE;
    return LORA_OK;
}

}  // extern "C"
