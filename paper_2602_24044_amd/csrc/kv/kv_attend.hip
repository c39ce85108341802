// Attention of a step's tokens over the cache in four bits.
//
//   out[t, head] = sum_k p_k v_k,   p = softmax_k(scale q . k) over the keys at positions <= that of t
//
// in one pass over the keys: a running maximum m and sum l of the weights 2^(s - m), the accumulated values scaled down when m
// grows.  Scores, sums, m and the accumulated values are fp32; the weights are rounded to bf16 for the matrix units (2^-8 of each at
// most, like the values' own rounding in a cache of 16 bits), and l is the sum of the rounded ones, so that equal values stay what they are.
//
// Two kernels share the work.  A tile of 16 columns is a wave's: requests with few queries, where the cache's bytes are the bound.
// A tile of 128 columns is four waves', which share the converted values through LDS: chunks of prompts, where the matrix units and the
// weights' exponentials are.
//
// A column is a query: (token j, head g of the key head's group), column j * group + g, so a group's heads share the keys that they
// read.  S^T = K Q^T on MFMAs that take the keys' four-bit codes and exponents as they are in the cache (16x16x128, 32x32x64), O^T = V^T
// P^T on bf16 MFMAs (16x16x32, 32x32x16) with the values converted.  A lane's results belong to one column; the accumulator of S^T
// (lane (column, quarter): keys 4 quarter + i of a 16-key tile) is the operand that the second product wants once its keys are counted in
// that order, and the codes of four keys that a lane loads with one instruction are its own part of V^T, so the weights never cross lanes.
#include "kv_device.hpp"

#include <algorithm>

namespace lora {
namespace kv {
namespace {

__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

// Weights may grow to 2^kSlack times those of the running maximum before the sums are scaled down: most blocks then leave them alone.
constexpr float kSlack = 8.f;
// A weight is 2^(s scale - m) with the product unrounded and m the rounded product of the largest.  From this maximum on half a step of it
// is a factor of two, and more further on: the largest key's weight itself would leave the range.  A wave with such a column rounds all
// products first, and looks at every block as at one that makes m grow (limit -inf), so that the others' blocks do not ask for it (a pass over
// 8192 tokens 517 -> 522 us; with a question of its own in every block another 3 - 4).
constexpr float kFar = 16777216.f;

// The largest over lanes 32 apart, and over lanes 16 and 32 apart: rows of a register change places with rows of its copy on the vector
// unit.  (The copy is hidden from the compiler, which otherwise takes both results for one and drops the comparison.)
__device__ inline float max_halves(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    uint32_t v = u;
    asm("" : "+v"(v));
    const auto r = __builtin_amdgcn_permlane32_swap(u, v, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ inline float max_quarters(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    uint32_t v = u;
    asm("" : "+v"(v));
    const auto r = __builtin_amdgcn_permlane16_swap(u, v, false, false);
    return max_halves(fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1])));
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- tiles of few columns ----
// A wave takes a piece of a tile by itself, eleven waves on a CU.  Its blocks are copied to LDS as they are, the next block's keys as
// soon as this block's scores are there, its values at the end of the block: what is on its way hangs on no register (four waves that
// share a tile's blocks and fetch them through registers: 91 us instead of 86 for 256 requests; one place for keys and sixteen waves a
// CU: slower too).  The cache's bytes bound it: those 256 requests (383 MB) at 4.5 TB/s, one of 130000 tokens (143 MB) in 30 us, 4.8
// TB/s.  The matrix units are busy for 16 % of that and the vector unit for 37 %; what is missing is that all pieces start at once and the
// longest end alone.
template <int D> struct Stage {
    static constexpr int kKeys = 2, kExpPlaces = 4;
    static constexpr int kHalf = kBlock * Part<D>::kRow, kExps = 2 * kBlock * Part<D>::kGroups;
    static constexpr int kCopies = kHalf / 1024;       // copy instructions of a half; the exponents take one
    static constexpr int kV = kKeys * kHalf, kE = kV + kHalf, kBytes = kE + kExpPlaces * kExps;
};

// Keys in LDS: a row of codes per key as in the cache, but for the 16-byte pieces of a row, which change places (by the bits of the key above
// those that 256 bytes hold) so that lanes that read the same piece of neighbouring keys meet different banks.  A copy writes LDS in
// lane order, so it is the lanes' addresses in memory that are dealt out; keys 16 (32 with heads of 64) apart are alike.
template <int D> __device__ inline int key_at(int k, int piece)
{
    return k * Part<D>::kRow + 16 * (piece ^ (D == 128 ? (k >> 2) & 3 : (k >> 3) & 1));
}
template <int D> __device__ inline uint32_t key_from(int lane)
{
    return 16 * (lane ^ (D == 128 ? lane >> 4 : (lane >> 4) & 1));
}

// 16 bytes per active lane, `offset` behind `from`, to LDS at lds + 16 * lane.  m0 carries the LDS address (the compiler writes it itself
// directly in front of its own uses); the copy wants a wait state behind the write.
__device__ inline void copy16(const uint8_t* from, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(from), "s"(lds) : "memory");
}
// All but the wave's latest N requests to memory have come back.
template <int N> __device__ inline void landed() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// What has been read from LDS is in registers: its place may be overwritten.
__device__ inline void read_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// lds: where the stage is; b: number of the block in its piece.
template <int D> __device__ inline void copy_keys(uint32_t lds, int b, const uint8_t* part, int lane)
{
    using T = Stage<D>;
    if (16 * lane < T::kExps) copy16(part + Part<D>::kKExp, 16 * lane, lds + T::kE + b % T::kExpPlaces * T::kExps);
#pragma unroll
    for (int c = 0; c < T::kCopies; ++c) copy16(part + Part<D>::kK + 1024 * c, key_from<D>(lane), lds + b % T::kKeys * T::kHalf + 1024 * c);
}
template <int D> __device__ inline void copy_values(uint32_t lds, const uint8_t* part, int lane)
{
#pragma unroll
    for (int c = 0; c < Stage<D>::kCopies; ++c) copy16(part + Part<D>::kV + 1024 * c, 16 * lane, lds + Stage<D>::kV + 1024 * c);
}

template <int W> __device__ inline void load_words(uint32_t (&d)[W], const uint8_t* p)
{
    if constexpr (W == 4) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = x[j];
    } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(p);
        d[0] = x[0];
        d[1] = x[1];
    }
}

// m of the lane's column, l[i] the sum of its weights (every i the same: a product with ones, of the weights as they are rounded for
// the values), acc[j][i]: dimension E (4 quarter + i) + j of it.
template <int D> struct Running {
    float m;
    float limit, by;                                   // a score that makes m grow; what scores are multiplied by: their scale, or 1 (kFar)
    f32x4 l, acc[D / 16];
};

// Scores on the MFMA that takes four-bit operands with a power of two for every 32 values, as the cache holds the keys: they need no
// conversion.  The other operand has eight bits then: a query is taken apart into two e4m3 numbers, q = 2^n (a + b / 16), a the nearest
// to q / 2^n and b to what is left.  With the largest of the head's values at 2^7 .. 2^8 that is exact for the eight significant bits of bf16
// down to 2^-14 of it, and off by at most 2^-21 of it below.
// Lane (column, quarter) of the 16x16x128 MFMA has four-bit operands k = 32 quarter .. + 31 and eight-bit ones k = 16 quarter .. + 15 and
// 64 + 16 quarter .. + 15; the exponent of operands 32 j .. + 31 comes from quarter j.  With heads of 128, a and b take an MFMA each; with
// heads of 64, operands 64 .. 127 are b, against the same keys.
typedef __attribute__((ext_vector_type(8))) int i32x8;
template <int D> struct Query {
    static constexpr int kTerms = D / 64;
    i32x8 x[kTerms];
    int e[kTerms];                                     // biased exponent
};

__device__ inline i32x8 four_dwords(u32x4 v)
{
    const i32x8 r = {(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
    return r;                                          // (four-bit operands are the first half)
}

__device__ inline float positive(float scale_log2) { return scale_log2 == 0.f ? 1.f : __builtin_fabsf(scale_log2); }

// The two numbers of N * 16 values of a column (their runs at p + at(j)): hi and lo, four to a dword; returns n.  The column's other
// values are in lanes that largest() goes over.  The scale of the scores comes in here by its sign: it is positive from here on.
template <int N, typename At, typename Largest>
__device__ inline int split_values(int (&hi)[4 * N], int (&lo)[4 * N], const uint16_t* p, float scale_log2, At&& run, Largest&& largest)
{
    u32x4 raw[2 * N];
#pragma unroll
    for (int j = 0; j < 2 * N; ++j) raw[j] = load16(p + run(j / 2) + 8 * (j % 2));
    float top = 0.f, odd = 0.f;                        // odd: a NaN where a value is a NaN or an infinity, which makes the column one
#pragma unroll
    for (int j = 0; j < 2 * N; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __builtin_fabsf(lo_f32(raw[j][i])), y = __builtin_fabsf(hi_f32(raw[j][i]));
            odd = __builtin_fmaf(x, 0.f, __builtin_fmaf(y, 0.f, odd));
            top = fmaxf(top, fmaxf(x, y));
        }
    top = largest(top);
    const int n = max((int)(__builtin_bit_cast(uint32_t, top) >> 23) - 127 - 7, -120);
    const float power = __builtin_bit_cast(float, (uint32_t)(127 - n) << 23);
    const float down = scale_log2 > 0.f ? power : scale_log2 < 0.f ? -power : 0.f;
#pragma unroll
    for (int j = 0; j < 2 * N; ++j)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const float y[4] = {__builtin_fmaf(lo_f32(raw[j][i]), down, odd), __builtin_fmaf(hi_f32(raw[j][i]), down, odd),
                                __builtin_fmaf(lo_f32(raw[j][i + 1]), down, odd), __builtin_fmaf(hi_f32(raw[j][i + 1]), down, odd)};
            int a = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], a, true);
            const f32x2 a0 = __builtin_amdgcn_cvt_pk_f32_fp8(a, false), a1 = __builtin_amdgcn_cvt_pk_f32_fp8(a, true);
            int b = __builtin_amdgcn_cvt_pk_fp8_f32((y[0] - a0[0]) * 16.f, (y[1] - a0[1]) * 16.f, 0, false);
            b = __builtin_amdgcn_cvt_pk_fp8_f32((y[2] - a1[0]) * 16.f, (y[3] - a1[1]) * 16.f, b, true);
            hi[2 * j + i / 2] = a;
            lo[2 * j + i / 2] = b;
        }
    return n;
}

// row: the column's query.
template <int D> __device__ inline void split_query(Query<D>& q, const uint16_t* row, float scale_log2, int lane)
{
    constexpr int N = D / 64;                          // 16 dimensions, twice with heads of 128
    const int quad = lane >> 4;
    int hi[4 * N], lo[4 * N];
    const int n = split_values<N>(hi, lo, row, scale_log2, [&](int j) { return 64 * j + 16 * quad; }, [](float x) { return max_quarters(x); });
#pragma unroll
    for (int j = 0; j < 4 * N; ++j) {
        q.x[0][j] = hi[j];
        if constexpr (D == 128) q.x[1][j] = lo[j];
        else q.x[0][4 + j] = lo[j];
    }
    q.e[0] = n + 127 - (D == 64 && quad >= 2 ? 4 : 0);
    if constexpr (D == 128) q.e[1] = n + 127 - 4;
}

// s[t][i]: score of key 16 t + 4 quarter + i of a block.
template <int D> __device__ inline void scores(f32x4 (&s)[4], const uint8_t* keys, const uint8_t* exps, const Query<D>& q, int lane)
{
    const int m = lane & 15, g = D == 128 ? lane >> 4 : (lane >> 4) & 1;
    const int e = *reinterpret_cast<const int*>(exps + Part<D>::k_exp_at(m, g));
    i32x8 k[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        k[t] = four_dwords(*reinterpret_cast<const u32x4*>(keys + key_at<D>(16 * t + m, g)));
        s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // (formats: 4 = e2m1, 0 = e4m3; the number behind is the byte of the exponents)
#pragma unroll
    for (int x = 0; x < Query<D>::kTerms; ++x) {
        s[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k[0], q.x[x], s[0], 4, 0, 0, e, 0, q.e[x]);
        s[1] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k[1], q.x[x], s[1], 4, 0, 1, e, 0, q.e[x]);
        s[2] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k[2], q.x[x], s[2], 4, 0, 2, e, 0, q.e[x]);
        s[3] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k[3], q.x[x], s[3], 4, 0, 3, e, 0, q.e[x]);
    }
}

// Weights of a block's scores; limit: the last key position of the lane's column, relative to the block's first; masked: some column does
// not see the whole block.
template <int D> __device__ inline void weights(Running<D>& r, uint32_t (&p)[4][2], f32x4 (&s)[4], float scale, int limit, bool masked, int lane)
{
    const int quad = lane >> 4;
    float top = -INFINITY;
    if (masked)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (16 * t + 4 * quad + i > limit) s[t][i] = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
    top = max_quarters(top) * scale;
    if (__any(top > r.limit)) {
        const float m = fmaxf(r.m, top), from = m == -INFINITY ? 0.f : m;
        const float down = exp2_fast(r.m - from);
        const bool far = __any(__builtin_fabsf(from) > kFar);
        r.l *= down;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) r.acc[j] *= down;
        r.m = m;
        r.limit = far ? -INFINITY : m + kSlack;
        r.by = far ? 1.f : scale;
        if (far)
#pragma unroll
            for (int t = 0; t < 4; ++t) s[t] *= scale;
    }
    // a column that has seen no key yet keeps m = -inf: its weights are 2^-inf = 0, not 2^(-inf + inf)
    const float base = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = exp2_fast(__builtin_fmaf(s[t][i], r.by, -base));
        p[t][0] = pack_bf16(w[0], w[1]);
        p[t][1] = pack_bf16(w[2], w[3]);
    }
}

// The weighted values of 64 keys.  V^T of 32 keys: keys 4 quarter .. + 3 of tile 2 h, then of tile 2 h + 1.  A key's codes come two
// dimensions at a time; two keys' results are dealt into the two dimensions' operands.
template <int D> __device__ inline void add_values(Running<D>& r, const uint32_t (&p)[4][2], const uint8_t* values, const uint8_t* exps, int lane)
{
    constexpr int W = D / 32;
    const int m = lane & 15, quad = lane >> 4;
    const u32x4 ve = *reinterpret_cast<const u32x4*>(exps + kBlock * Part<D>::kGroups + Part<D>::v_exp_at(4 * quad, m * Part<D>::kE / kGroup));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t c[2][W];
#pragma unroll
        for (int t = 0; t < 2; ++t) load_words(c[t], values + Part<D>::v_at(16 * (2 * h + t) + 4 * quad, m * Part<D>::kE));
        const u32x4 w = {p[2 * h][0], p[2 * h][1], p[2 * h + 1][0], p[2 * h + 1][1]};
        r.l = mfma16(u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}, w, r.l);
#pragma unroll
        for (int d = 0; d < D / 16; d += 4) {          // four dimensions at a time: 16 registers of operands
            u32x4 f[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {              // keys 2 x, 2 x + 1 of the eight
                const int t = x / 2, i = 2 * (x & 1);
                const uint32_t e = ve[2 * h + t];
                const uint32_t e0 = i == 0 ? e << 23 : e << 7, e1 = i == 0 ? e << 15 : e >> 1;
                auto deal = [&](int j, uint32_t a, uint32_t b) {
                    f[j][x] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                    f[j + 1][x] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                };
                if constexpr (D == 128) {
                    const uint32_t a = c[t][i], b = c[t][i + 1];
                    deal(0, d == 0 ? two_bf16<0>(a, e0) : two_bf16<2>(a, e0), d == 0 ? two_bf16<0>(b, e1) : two_bf16<2>(b, e1));
                    deal(2, d == 0 ? two_bf16<1>(a, e0) : two_bf16<3>(a, e0), d == 0 ? two_bf16<1>(b, e1) : two_bf16<3>(b, e1));
                } else {
                    const uint32_t a = c[t][i / 2];    // both keys in one dword, four codes each
                    deal(0, two_bf16<0>(a, e0), two_bf16<2>(a, e1));
                    deal(2, two_bf16<1>(a, e0), two_bf16<3>(a, e1));
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) r.acc[d + j] = mfma16(f[j], w, r.acc[d + j]);
        }
    }
}

// Token and head that a request's (an entry's) column is; false: there is none in the step.
template <typename Of> __device__ inline bool column(const Of& r, int group, int T, int col, int& token, int& head)
{
    token = col / group;
    head = col - token * group;
    return token < r.rows && r.first + token < T;
}

// Where the blocks of a piece are in the cache: 64 numbers at a time, one per lane; those behind the ones that came with the entry are
// fetched when the first of them is asked for, which is in order.
struct Numbers {
    uint32_t ids;
    __device__ Numbers(const Entry& e, int lane) : ids(e.id[lane & (kEntryIds - 1)]) {}
    // block b of the n of the piece, which blocks[] has in the table.  (A row that has been released since the plan has none: any will do.)
    __device__ uint32_t at(int b, const int32_t* blocks, int n, int n_blocks, int lane)
    {
        if (b == kEntryIds || (b && b % 64 == 0)) ids = min((unsigned)blocks[min((b & ~63) + lane, n - 1)], (unsigned)n_blocks - 1);
        return __builtin_amdgcn_readlane(ids, b & 63);
    }
};

template <int D> __global__ __launch_bounds__(64, 3) void attend_few_kernel(AttendArgs a)
{
    using St = Stage<D>;
    constexpr int A = St::kCopies + 1, B = St::kCopies;             // requests for a block's keys (with the exponents), and for its values
    __shared__ __align__(1024) uint8_t stage[St::kBytes];
    const uint32_t lds = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)stage;
    const int lane = threadIdx.x, c = lane & 15, quad = lane >> 4;
    const float scale = positive(a.scale_log2);
    for (int item = blockIdx.x; item < a.n_few * a.n_kv; item += gridDim.x) {
        const Entry& r = a.t.few[item / a.n_kv];
        if (r.rows == 0) return;
        const int h = item % a.n_kv;
        int token, head;
        const bool real = column(r, a.group, a.T, r.tile * kFewCols + c, token, head);
        const int limit = r.len + token;                            // last key that the lane's column sees
        const int32_t* blocks = a.t.table + (size_t)r.row * a.t.row_blocks + r.block;
        const int n = r.blocks, first = r.block, len = r.len;
        Running<D> run;
        run.m = run.limit = -INFINITY;
        run.by = scale;
        run.l = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < D / 16; ++j) run.acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (n > 0) {
            Numbers numbers(r, lane);
            auto part = [&](int b) { return a.cache + ((size_t)numbers.at(b, blocks, n, a.t.n_blocks, lane) * a.n_kv + h) * Part<D>::kBytes; };
            const uint8_t *now = part(0), *next = now;
            copy_keys<D>(lds, 0, now, lane);
            if (n > 1) {
                next = part(1);
                copy_keys<D>(lds, 1, next, lane);
            }
            copy_values<D>(lds, now, lane);
            Query<D> q;
            split_query<D>(q, a.q + (size_t)min(r.first + (real ? token : 0), a.T - 1) * a.q_stride + ((size_t)h * a.group + (real ? head : 0)) * D, a.scale_log2, lane);
            for (int b = 0; b < n; ++b) {
                const bool one_more = b + 1 < n, two_more = b + 2 < n;
                const int at = (first + b) * kBlock;
                const uint8_t* exps = stage + St::kE + b % St::kExpPlaces * St::kExps;
                if (one_more) landed<A + B>();
                else landed<B>();
                f32x4 s[4];
                scores<D>(s, stage + b % St::kKeys * St::kHalf, exps, q, lane);
                read_done();
                const uint8_t* after = next;
                if (two_more) {
                    after = part(b + 2);
                    copy_keys<D>(lds, b + 2, after, lane);
                }
                uint32_t p[4][2];
                weights<D>(run, p, s, scale, limit - at, at + kBlock - 1 > len, lane);
                if (two_more) landed<A>();
                else landed<0>();
                add_values<D>(run, p, stage + St::kV, exps, lane);
                read_done();
                if (one_more) copy_values<D>(lds, next, lane);
                next = after;
            }
        }
        const float l = run.l[0];
        if (!real) continue;
        // the lane's values: dimensions E (4 quarter + i) + j of its column, D / 4 in a row
        if (r.part >= 0) {
            const size_t slot = ((size_t)r.part * a.n_kv + h) * kFewCols + c;
            float* o = a.few_acc + slot * D + quad * (D / 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < D / 16; j += 4)
                    *reinterpret_cast<f32x4*>(o + (D / 16) * i + j) = f32x4{run.acc[j][i], run.acc[j + 1][i], run.acc[j + 2][i], run.acc[j + 3][i]};
            if (quad == 0) {
                a.few_ml[slot * 2] = run.m;
                a.few_ml[slot * 2 + 1] = l;
            }
        } else {
            // (no block: a refused request, its rows are zero.  No weight behind keys: every score lies below the range, 0 / 0)
            const float f = n == 0 ? 0.f : 1.0f / l;
            uint16_t* o = a.out + (size_t)(r.first + token) * a.out_stride + ((size_t)h * a.group + head) * D + quad * (D / 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < D / 16; j += 4)
                    *reinterpret_cast<u32x2*>(o + (D / 16) * i + j) = u32x2{pack_bf16(run.acc[j][i] * f, run.acc[j + 1][i] * f),
                                                                          pack_bf16(run.acc[j + 2][i] * f, run.acc[j + 3][i] * f)};
        }
    }
}

// ---- tiles of many columns ----
// Four waves of 32 columns each on 32x32 MFMAs.  A block's keys are copied to LDS as they are (four-bit operands); its values go through
// registers, where each thread converts an eighth of 16 tokens to bf16 operands of V^T in LDS, once for all four waves.  Two stages: the next
// block is made while this one is used.
//
// A prompt of 8192 tokens, 32 heads on 8 of 128 (550 GFLOP) takes 485 - 515 us, by the card: 1.07 - 1.13 PFLOP/s, where a large bf16 product
// reaches 1.25 (heads of 64: 301 us, 0.9).
// Matrix and vector units are busy for half of the time each, LDS for a third; leaving out any one of them (scores, exponentials,
// conversion, products with the values) takes 5 - 17 % off, so it is the chain through all of them, twice on each SIMD, that counts.
// Not kept: 64 columns a wave, alone on its SIMD (694 us: scores and sums change places between the two kinds of registers);
// conversion and maximum between the products with the values (545 - 563, with and without priorities); the conversion's lanes dealt
// out otherwise (570).
//
// Values, as the 256 threads load them: a chunk of four tokens, kE dimensions.  That is half of an operand of V^T for each of these: the
// other half are the four tokens eight further.
template <int D> struct Raw {
    uint32_t v[D / 32], e;
};
struct Place {
    int u, c, h, m;            // tokens 16 u + 8 c + 4 h .. + 3, dimensions kE m ..
};
__device__ inline Place place()
{
    const int t = threadIdx.x;
    return Place{t >> 6, (t >> 5) & 1, (t >> 4) & 1, t & 15};
}

template <int D> __device__ inline void load_values(Raw<D>& r, const uint8_t* part, const Place& p)
{
    using P = Part<D>;
    const int k = 16 * p.u + 8 * p.c + 4 * p.h;
    load_words(r.v, part + P::kV + P::v_at(k, p.m * P::kE));
    r.e = *reinterpret_cast<const uint32_t*>(part + P::kVExp + P::v_exp_at(k, p.m * P::kE / kGroup));
}

// A block in LDS.  Values: every operand of an MFMA is 64 lanes * 16 bytes, in lane order but for a permutation inside groups of four that
// spreads a wave's writes over the banks: [d / 32][key / 16].  (Reads take lanes four by four, not all of them neighbours.)
template <int D> struct Tile {
    uint8_t k[kBlock * Part<D>::kRow], e[kBlock * Part<D>::kGroups];
    u32x4 v[(D / 32) * 4 * 64];
    __device__ static int v_at(int dt, int u, int h, int i) { return (dt * 4 + u) * 64 + h * 32 + (i ^ (2 * ((i >> 4) & 1) + (dt & 1))); }
};

template <int D> __device__ inline void convert(Tile<D>& t, const Raw<D>& r, const Place& p)
{
    constexpr int E = Part<D>::kE;
    u32x2 f[E];
#pragma unroll
    for (int x = 0; x < 2; ++x) {                      // tokens 2 x, 2 x + 1 of the four
        const uint32_t e0 = x == 0 ? r.e << 23 : r.e << 7, e1 = x == 0 ? r.e << 15 : r.e >> 1;
        const uint32_t a = D == 128 ? r.v[2 * x] : r.v[x], b = D == 128 ? r.v[2 * x + 1] : r.v[x] >> 16;
        auto deal = [&](int d, uint32_t y, uint32_t z) {
            f[d][x] = __builtin_amdgcn_perm(z, y, 0x05040100u);
            f[d + 1][x] = __builtin_amdgcn_perm(z, y, 0x07060302u);
        };
        deal(0, two_bf16<0>(a, e0), two_bf16<0>(b, e1));
        deal(2, two_bf16<1>(a, e0), two_bf16<1>(b, e1));
        if constexpr (D == 128) {
            deal(4, two_bf16<2>(a, e0), two_bf16<2>(b, e1));
            deal(6, two_bf16<3>(a, e0), two_bf16<3>(b, e1));
        }
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int d = E * p.m + j;
        reinterpret_cast<u32x2*>(&t.v[Tile<D>::v_at(d >> 5, p.u, p.h, d & 31)])[p.c] = f[j];
    }
}

// A block's keys and their exponents to LDS (lds: where the tile is): 1 KB a wave, the exponents by the last of these waves.
template <int D> __device__ inline void copy_block_keys(uint32_t lds, const uint8_t* part, int wave, int lane)
{
    constexpr int keys = kBlock * Part<D>::kRow, exps = kBlock * Part<D>::kGroups;
    if (wave < keys / 1024) copy16(part + Part<D>::kK + 1024 * wave, key_from<D>(lane), lds + 1024 * wave);
    if (wave == keys / 1024 - 1 && 16 * lane < exps) copy16(part + Part<D>::kKExp, 16 * lane, lds + keys);
}

template <int D> __global__ __launch_bounds__(256, 2) void attend_many_kernel(AttendArgs a)
{
    constexpr int X = D / 64, N = D / 32;
    __shared__ __align__(1024) Tile<D> tiles[2];
    const uint32_t lds = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)tiles;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, h = lane >> 5;
    // Entries of a request begin with the longest; requests follow each other as they are.  Where all entries find room at once, two a CU, the
    // second of a CU is taken from the list's end, so that a request's long ones share with short ones (a prompt of 2000 tokens 54 -> 49 us, two
    // of 900 34 -> 30; six of 300 - 1000 in no order 48 -> 49); where they do not, the list's order stands and the rest follows as CUs become free.
    const int there = a.t.head->n_many * a.n_kv, at_once = 2 * a.n_cus;
    if ((int)blockIdx.x >= there) return;
    const int item = there <= at_once && (int)blockIdx.x >= a.n_cus ? there - 1 - ((int)blockIdx.x - a.n_cus) : (int)blockIdx.x;
    const Entry& e = a.t.many[item / a.n_kv];
    const int hk = item % a.n_kv;
    int token, head;
    const bool real = column(e, a.group, a.T, e.tile * kManyCols + wave * 32 + i, token, head);
    const int limit = real ? e.len + token : -1;
    const int seen = e.len + (e.tile * kManyCols + wave * 32) / a.group;   // the last key that all of the wave's columns see
    const Place pl = place();
    const int32_t* blocks = a.t.table + (size_t)e.row * a.t.row_blocks + e.block;
    const int n = __builtin_amdgcn_readfirstlane(e.blocks), first = e.block;
    Numbers numbers(e, lane);

    // 32x32x64: lane (column, h) has eight-bit operands k = 16 h .. + 15 and 32 + 16 h .. + 15, four-bit ones k = 32 h .. + 31
    i32x8 q[X][2];
    int qe;
    {
        const size_t row = min(e.first + (real ? token : 0), a.T - 1);
        int hi[8 * X], lo[8 * X];
        qe = 127 + split_values<2 * X>(hi, lo, a.q + row * a.q_stride + ((size_t)hk * a.group + (real ? head : 0)) * D, a.scale_log2,
                                       [&](int j) { return 32 * j + 16 * h; }, [](float x) { return max_halves(x); });
#pragma unroll
        for (int x = 0; x < X; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q[x][0][j] = hi[8 * x + j];
                q[x][1][j] = lo[8 * x + j];
            }
    }
    f32x16 o[N];
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[d][x] = 0.f;
    float m = -INFINITY, l = 0.f;
    const float scale = positive(a.scale_log2);
    float most = -INFINITY, by = scale;                // as in Running

    Raw<D> raw;
    // A block's keys out of LDS, and one of the 4 X products that make its scores.
    struct Keys {
        i32x8 k[X][2];
        int e[X];
    };
    auto read_keys = [&](Keys& f, const Tile<D>& t) {
#pragma unroll
        for (int x = 0; x < X; ++x) {
            // exponents of keys i % 16, + 16, + 32, + 48: those of key i and i + 32 in bytes 0 and 2
            f.e[x] = *reinterpret_cast<const int*>(t.e + Part<D>::k_exp_at(i & 15, 2 * x + h)) >> (i & 16 ? 8 : 0);
#pragma unroll
            for (int k = 0; k < 2; ++k) f.k[x][k] = four_dwords(*reinterpret_cast<const u32x4*>(t.k + key_at<D>(32 * k + i, 2 * x + h)));
        }
    };
    auto score = [&](f32x16 (&s)[2], const Keys& f, int j) {
        const int x = j / 4, y = (j / 2) & 1;
        if (j & 1) s[1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f.k[x][1], q[x][y], s[1], 4, 0, 2, f.e[x], 0, qe - 4 * y);
        else s[0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f.k[x][0], q[x][y], s[0], 4, 0, 0, f.e[x], 0, qe - 4 * y);
    };
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    // The loop is one block of scores ahead, so that the matrix units have work while the vector unit forms a block's weights: at the top of
    // iteration b the scores of block b are there, its values and the next block's keys are in LDS (places b % 2 and (b + 1) % 2), and the
    // next block's values are in registers or on their way.
    f32x16 s[2];
    auto at = [&](uint32_t id) { return a.cache + ((size_t)__builtin_amdgcn_readfirstlane(id) * a.n_kv + hk) * Part<D>::kBytes; };
    if (n > 0) {
        const uint32_t one = numbers.at(0, blocks, n, a.t.n_blocks, lane);
        const uint32_t two = n > 1 ? numbers.at(1, blocks, n, a.t.n_blocks, lane) : one;
        copy_block_keys<D>(lds, at(one), wave, lane);
        copy_block_keys<D>(lds + (uint32_t)sizeof(Tile<D>), at(two), wave, lane);
        load_values<D>(raw, at(one), pl);
        convert<D>(tiles[0], raw, pl);                 // (waits for everything asked for so far)
        load_values<D>(raw, at(two), pl);
        __syncthreads();
        Keys f;
        read_keys(f, tiles[0]);
        s[0] = s[1] = zero;
#pragma unroll
        for (int j = 0; j < 4 * X; ++j) score(s, f, j);
    }
    auto step = [&](int b, f32x16 (&s)[2], f32x16 (&s_next)[2]) {
        __syncthreads();                               // what the comment above says holds for all waves, and the other places have been read
        const int key0 = (first + b) * kBlock;
        const Tile<D>&t = tiles[b & 1], &ahead = tiles[(b + 1) & 1];
        // (in this order: the compiler waits for all requests in front of the first use of `raw`, and it should be for the ones that the
        // iteration before has made)
        convert<D>(tiles[(b + 1) & 1], raw, pl);
        if (b + 2 < n) {
            const uint32_t two = numbers.at(b + 2, blocks, n, a.t.n_blocks, lane);
            copy_block_keys<D>(lds + (b & 1) * (uint32_t)sizeof(Tile<D>), at(two), wave, lane);
            load_values<D>(raw, at(two), pl);
        }
        if (key0 + kBlock - 1 > seen) {                // some column does not see the whole block
            const int room = limit - key0 - 4 * h;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    if (32 * k + 8 * (x / 4) + x % 4 > room) s[k][x] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int x = 0; x < 16; ++x) top = fmaxf(top, s[k][x]);
        top = max_halves(top) * scale;
        if (__any(top > most)) {
            const float grown = fmaxf(m, top), from = grown == -INFINITY ? 0.f : grown;
            const float down = exp2_fast(m - from);
            const bool far = __any(__builtin_fabsf(from) > kFar);
            l *= down;
#pragma unroll
            for (int d = 0; d < N; ++d) o[d] *= down;
            m = grown;
            most = far ? -INFINITY : m + kSlack;
            by = far ? 1.f : scale;
            if (far)
#pragma unroll
                for (int k = 0; k < 2; ++k) s[k] *= scale;
        }
        const float base = m == -INFINITY ? 0.f : m;
        // The order is pinned here: an MFMA of the next scores (of no use in the last iteration: what is in LDS then are older codes), and in
        // its time a part of this block's weights on the vector unit; values from LDS a group of operands ahead of the MFMAs that want
        // them.  Left to itself the compiler asks LDS for an operand right in front of each MFMA.
        // Priority over the SIMD's other wave from here on, whose conversion and maximum fill what the matrix units leave (8192 tokens: 565 ->
        // 547 us, 1900 behind 6100 268 -> 253; for the products with the values alone 570 and 268, the other way round 557 and 256).
        __builtin_amdgcn_s_setprio(1);
        Keys keys;
        read_keys(keys, ahead);
        s_next[0] = s_next[1] = zero;
        u32x4 w[4], f[2][N];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 4 * X; ++j) {
            score(s_next, keys, j);
            __builtin_amdgcn_sched_barrier(0);
            if (j == 4 * X - 1)
#pragma unroll
                for (int d = 0; d < N; ++d) f[0][d] = t.v[Tile<D>::v_at(d, 0, h, i)];
            constexpr int P = 32 / (4 * X);            // weights of a part
#pragma unroll
            for (int y = P * j; y < P * (j + 1); y += 2) {
                const int k = y / 16, x = y % 16;
                const float p0 = exp2_fast(__builtin_fmaf(s[k][x], by, -base)), p1 = exp2_fast(__builtin_fmaf(s[k][x + 1], by, -base));
                const uint32_t two = pack_bf16(p0, p1);
                l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3f803f80u), l, false);
                w[2 * k + x / 8][(x % 8) / 2] = two;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u < 3)
#pragma unroll
                for (int d = 0; d < N; ++d) f[(u + 1) & 1][d] = t.v[Tile<D>::v_at(d, u + 1, h, i)];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < N; ++d) o[d] = mfma32(as_bf16x8(f[u & 1][d]), as_bf16x8(w[u]), o[d]);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        landed<0>();
    };
    f32x16 s_other[2];
    for (int b = 0; b < n; b += 2) {                   // (two steps, whose scores change places without being moved)
        step(b, s, s_other);
        if (b + 1 < n) step(b + 1, s_other, s);
    }
    l += __shfl_xor(l, 32);
    if (!real) return;
    if (e.part >= 0) {
        const size_t slot = ((size_t)e.part * a.n_kv + hk) * kManyCols + wave * 32 + i;
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(a.many_acc + slot * D + 32 * d + 8 * g + 4 * h) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
        if (h == 0) {
            a.many_ml[slot * 2] = m;
            a.many_ml[slot * 2 + 1] = l;
        }
    } else {
        const float f = 1.0f / l;                      // (a column sees its own key at least)
        uint16_t* out = a.out + (size_t)(e.first + token) * a.out_stride + ((size_t)hk * a.group + head) * D + 4 * h;
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<u32x2*>(out + 32 * d + 8 * g) =
                    u32x2{pack_bf16(o[d][4 * g] * f, o[d][4 * g + 1] * f), pack_bf16(o[d][4 * g + 2] * f, o[d][4 * g + 3] * f)};
    }
}

// The partial results of tiles that were cut along their keys, in one pass with a running maximum.  D / 4 lanes take a column, four
// dimensions each; the groups of lanes of a workgroup have a column each, or share the pieces of one where there are many.
// Nearly all of it is waiting for the pieces, which other CUs have just written: 256 pieces of 32 columns take 6.8 us, of which 4.6 are an empty
// launch's (with 256 threads, half the groups, 8.8; with 1024 8.2; eight pieces' requests at once instead of four: no less).
constexpr int kMergeThreads = 512;
template <int D> __global__ __launch_bounds__(kMergeThreads) void merge_kernel(AttendArgs a)
{
    constexpr int L = D / 4, GROUPS = kMergeThreads / L;
    __shared__ float sAcc[GROUPS][D], sM[GROUPS], sL[GROUPS];
    const int tid = threadIdx.x, lane = tid % L, group = tid / L;
    for (int item = blockIdx.x; item < a.n_merge * a.n_kv; item += gridDim.x) {
        const Merge g = a.t.merge[item / a.n_kv];
        if (g.rows == 0) return;
        const int h = item % a.n_kv, cols = g.many ? kManyCols : kFewCols;
        const bool share = g.cols == 1;                // (the same for the whole workgroup, like everything but `group` and `lane`)
        for (int c = share ? 0 : group; c < g.cols; c += GROUPS) {
            int token, head;
            if (!column(g, a.group, a.T, g.col + c, token, head)) break;
            const size_t step = (size_t)a.n_kv * cols, slot0 = ((size_t)g.part * a.n_kv + h) * cols + g.col % cols + c;
            const float* ml = (g.many ? a.many_ml : a.few_ml) + 2 * slot0;
            const float* p = (g.many ? a.many_acc : a.few_acc) + slot0 * D + 4 * lane;
            float m = -INFINITY, l = 0.f;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            auto add = [&](float m1, float l1, f32x4 x) {
                const float grown = fmaxf(m, m1), base = grown == -INFINITY ? 0.f : grown;
                const float f0 = exp2_fast(m - base), f1 = exp2_fast(m1 - base);
                l = l * f0 + l1 * f1;
                acc = acc * f0 + x * f1;
                m = grown;
            };
#pragma unroll 4
            for (int s = share ? group : 0; s < g.splits; s += share ? GROUPS : 1)
                add(ml[2 * step * s], ml[2 * step * s + 1], *reinterpret_cast<const f32x4*>(p + step * D * s));
            if (share) {
                __syncthreads();
                *reinterpret_cast<f32x4*>(&sAcc[group][4 * lane]) = acc;
                if (lane == 0) {
                    sM[group] = m;
                    sL[group] = l;
                }
                __syncthreads();
                if (group) continue;
#pragma unroll
                for (int w = 1; w < GROUPS; ++w) add(sM[w], sL[w], *reinterpret_cast<const f32x4*>(&sAcc[w][4 * lane]));
            }
            const float f = 1.0f / l;                      // (no weight at all: every score lies below the range, 0 / 0)
            uint16_t* o = a.out + (size_t)(g.first + token) * a.out_stride + ((size_t)h * a.group + head) * D + 4 * lane;
            *reinterpret_cast<u32x2*>(o) = u32x2{pack_bf16(acc[0] * f, acc[1] * f), pack_bf16(acc[2] * f, acc[3] * f)};
        }
    }
}

template <int D> hipError_t attend(const AttendArgs& a, int n, hipStream_t stream)
{
    if (a.n_many > 0) attend_many_kernel<D><<<(unsigned)a.n_many * a.n_kv, 256, 0, stream>>>(a);
    // a workgroup per piece: which of them end early is for the hardware to fill (apart from refused requests a request has kFewMost
    // columns at most; more pieces than that go round)
    const long few = std::min<long>(a.n_few, (long)n * (kFewMost / kFewCols) + kFewItems / a.n_kv + 1);
    attend_few_kernel<D><<<(unsigned)std::min<long>(few * a.n_kv, 1 << 20), 64, 0, stream>>>(a);
    merge_kernel<D><<<(unsigned)std::min<long>((long)a.n_merge * a.n_kv, 4L * a.n_cus), kMergeThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const AttendArgs& a, int dim, int n, hipStream_t stream)
{
    if (a.T == 0) return hipSuccess;
    return dim == 64 ? attend<64>(a, n, stream) : attend<128>(a, n, stream);
}

}  // namespace kv
}  // namespace lora
