// Internal declarations of the key/value cache in four bits: its block tables, what fills it and the attention that reads it.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lora {

// The text behind lora_last_hip_error (lora_api.hip): true if e is a failure, which it then holds.
bool note_hip_failure(hipError_t e, const char* what);

namespace kv {

constexpr int kBlock = 64;             // tokens of a block
constexpr int kGroup = 32;             // values of a head that share an exponent
constexpr int kMaxSeqs = 8192;         // rows of the block table: the plan keeps one int per row in LDS
constexpr int kMaxBlocks = 1 << 20;
constexpr int kMaxSeqTokens = 1 << 24;
constexpr int kMaxTokens = 1 << 20;
constexpr int kMaxHeads = 1024;
constexpr int kPlanThreads = 1024;
// Attention works on tiles of columns (token, query head of a key head).  Requests of up to kFewMost columns take tiles of
// kFewCols, whose waves each convert the codes that they need; longer ones take tiles of kManyCols, whose waves share them.  Where one
// overtakes the other, with 32 query heads on 8 key heads of 128 (few / many columns, us): 40 columns, 256 requests with 200 cached
// tokens 45 / 62, 64 with 1000 44 / 46, 4 with 1000 10 / 16; 64 columns, 64 with 1000 46 / 48; 128 columns 78 / 54.
constexpr int kFewCols = 16, kManyCols = 128;
constexpr int kFewMost = 64;
// Pieces that the keys of the tiles are cut into, over all tiles and key heads; at most one more per tile (piece_blocks).  Few columns:
// eleven waves a CU find room, 256 requests of mixed lengths take 86 - 90 us with 2048 pieces and more with 1536 or 2816 - 6144.  Many
// columns, 256 / 512 / 1024 pieces: 500 tokens behind 16000 178 / 160 / 172 us, 2000 tokens alone 60 / 60 / 70, and a merge of 7 / 9 / 12.
constexpr int kFewItems = 2048, kManyItems = 512;
// Blocks of the smallest piece.  (Few columns, 2 / 3 / 4: one request of 2000 tokens 6.9 / 8.0 / 9.1 us, 8 of 1000 9.0 / 9.6 / 10.3, 32 of 700
// 14.9 / 14.5 / 14.5.)
constexpr int kFewChunk = 2, kManyChunk = 8;
constexpr int kMinExp = -100, kMaxExp = 125;

// Bits of the device flag word (LORA_KV_FLAG_*).
constexpr uint32_t kFlagRefused = 1u, kFlagExhausted = 2u, kFlagNotFinite = 4u;

// Where things are in a head's part of a block, in bytes; D = head size.  A key's codes are one row: dimension d in nibble d.
// Values are kept for the product with the probabilities: chunks of four tokens, in a chunk D / 16 dimensions of token 0, the same
// of token 1, 2, 3, then the next D / 16 dimensions.  Every token owns whole bytes.
template <int D> struct Part {
    static constexpr int kRow = D / 2;                 // bytes of a token's codes
    static constexpr int kGroups = D / kGroup;
    static constexpr int kK = 0;
    static constexpr int kV = kBlock * kRow;
    static constexpr int kKExp = 2 * kBlock * kRow;
    static constexpr int kVExp = kKExp + kBlock * kGroups;
    static constexpr int kBytes = kVExp + kBlock * kGroups;
    static constexpr int kE = D / 16;                  // dimensions of a token that lie together in V
    // dimension d (a multiple of kE) of token k, in bytes from kV
    __host__ __device__ static constexpr int v_at(int k, int d) { return (k / 4) * 4 * kRow + (d / kE) * 2 * kE + (k % 4) * (kE / 2); }
    // exponents: those of the four tokens of equal k % 16 side by side
    __host__ __device__ static constexpr int k_exp_at(int k, int g) { return ((k % 16) * kGroups + g) * 4 + k / 16; }
    // exponents of V: those of a lane's 16 tokens side by side (token 16 t + 4 q + i of lane quarter q)
    __host__ __device__ static constexpr int v_exp_at(int k, int g) { return (((k % 16) / 4) * kGroups + g) * 16 + (k / 16) * 4 + k % 4; }
};

inline size_t part_bytes(int dim) { return dim == 64 ? Part<64>::kBytes : Part<128>::kBytes; }

// A request of the step (device).
struct Request {
    int32_t row;       // row of the block table
    int32_t len;       // tokens cached before the step
    int32_t rows;      // token rows of the step that are its own
    int32_t first;     // the first of them
    int32_t held;      // blocks of its table row before the step, -1: refused
    int32_t want;      // and with it
    int32_t fresh;     // its new blocks start here in the list of new blocks
    int32_t chunk;     // blocks of a split of its attention
    int32_t tiles;     // column tiles of its attention
    int32_t splits;    // splits over the keys of each tile
    int32_t entry;     // its first work entry
    int32_t part;      // its first partial result (splits > 1)
    int32_t merge;     // its first merge entry (splits > 1)
    int32_t many;      // its tiles have kManyCols columns
    int32_t pad_[2];
};

// A piece of a step's attention: a tile of columns against a range of blocks, for every key head.  It has with it what a kernel would
// otherwise fetch one after the other from the request and the block table (a piece is short: that chain of round trips would be a good
// part of it).
constexpr int kEntryIds = 8;
struct Entry {
    int32_t first;     // token row of the step that the request starts at
    int32_t rows;      // its token rows; 0: the list has ended (every entry behind the last one says so)
    int32_t len;       // its tokens cached before the step
    int32_t tile;
    int32_t block;     // first block of the range
    int32_t blocks;    // 0: nothing to read, the rows are set to zero
    int32_t part;      // partial result that it writes, -1: the output itself
    int32_t row;       // row of the block table
    uint32_t id[kEntryIds];   // the range's first blocks in the cache
};
static_assert(sizeof(Entry) == 64, "one line");
// Columns whose tile's range was split: the partial results are merged behind.  kMergeCols columns an entry, or one where there are at least
// kMergeMany pieces (all lanes of a workgroup then work on it: 8 requests of 32 pieces 4.8 us, 7.9 without that; from four pieces on
// it is the same either way).
constexpr int kMergeCols = 16, kMergeMany = 16;
struct Merge {
    int32_t first, rows;   // as in Entry
    int32_t col, cols; // first column, and how many
    int32_t part;      // first partial result of their tile
    int32_t splits;
    int32_t many;      // a tile of kManyCols columns
    int32_t pad_;
};

struct Header {
    uint32_t flags;
    int32_t rows;      // token rows of the step that belong to a request
    int32_t n_few;     // work entries
    int32_t n_many;
    int32_t n_merge;
    int32_t pad_[59];
};

struct Tables {
    Header* head;
    int32_t* table;    // [max_seqs][row_blocks], -1: none
    int32_t* held;     // [max_seqs]
    uint32_t* used;    // [n_words] bit b: block b is taken
    int32_t* fresh;    // blocks taken by the step
    int32_t* start;    // [n + 1]
    int32_t* position; // [T], -1: the row's request was refused
    int32_t* slot;     // [T], -1: likewise
    Request* request;  // [n]
    Entry* few;
    Entry* many;
    Merge* merge;
    int32_t n_blocks, n_words, max_seqs, row_blocks, max_seq_tokens;
};

struct PlanArgs {
    Tables t;
    const int32_t* seq;
    const int32_t* len;
    const int32_t* add;
    int32_t n, T, max_new;
    int32_t n_kv, group;
    int32_t whole;     // the first launch writes everything out (launch_plan)
};

struct HeadsArgs {
    const uint16_t *q, *k, *v;          // bf16; null: none
    uint16_t *q_out, *k_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;   // elements from token to token
    const uint16_t *q_norm, *k_norm;    // bf16 [D] or null
    const float* inv_freq;              // [D / 2] or null
    const int32_t* position;
    const int32_t* slot;                // of the tokens (cache != null)
    Header* head;                       // its row count limits the tokens (cache != null)
    uint8_t* cache;                     // the layer's part of the cache, or null
    float eps;
    int32_t T, n_heads, n_kv;
    int32_t pairs;                      // rotation of neighbours (2 p, 2 p + 1) instead of (p, p + D / 2)
};

struct ReadArgs {
    Tables t;
    const uint8_t* cache;
    const int32_t* seq;
    const int32_t* position;
    uint16_t *k_out, *v_out;            // [n][n_kv D]
    int32_t n, n_kv;
};

struct AttendArgs {
    Tables t;
    const uint8_t* cache;
    const uint16_t* q;
    uint16_t* out;
    int64_t q_stride, out_stride;
    float *few_acc, *few_ml;            // partial results: [part][key head][kFewCols][D] and [..][2] (m, l)
    float *many_acc, *many_ml;          // likewise with kManyCols
    float scale_log2;                   // scale * log2(e)
    int32_t T, n_kv, group;
    int32_t n_few, n_many, n_merge;     // entries that the lists can have (n_many 0: none)
    int32_t n_cus;
};

hipError_t launch_plan(const PlanArgs& a, hipStream_t stream);
hipError_t launch_release(const Tables& t, int n, const int32_t* seq, const int32_t* keep, hipStream_t stream);
hipError_t launch_heads(const HeadsArgs& a, int dim, hipStream_t stream);
hipError_t launch_read(const ReadArgs& a, int dim, hipStream_t stream);
// n: requests of the step
hipError_t launch_attend(const AttendArgs& a, int dim, int n, hipStream_t stream);

}  // namespace kv
}  // namespace lora
