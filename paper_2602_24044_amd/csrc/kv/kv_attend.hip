// Attention of a step's tokens over the cache in four bits.
//
//   out[t, head] = sum_k p_k v_k,   p = softmax_k(scale q . k) over the keys at positions <= that of t
//
// in one pass over the keys: a running maximum m and sum l of the weights 2^(s - m), the accumulated values scaled down when m
// grows.  Scores, weights' sums, m and the accumulated values are fp32; the weights are rounded to bf16 for the matrix units (2^-9 of
// each, like the values' own rounding in a cache of 16 bits).
//
// Two kernels share the work.  Of a request with few columns (one-token requests) a wave takes whole blocks and converts what it
// needs itself: the cache's bytes bound it.  For long chunks four waves share the converted keys and values through LDS.
//
// A column is a query: (token j, head g of the key head's group), column j * group + g, so a group's heads share the keys that they
// read.  S^T = K Q^T and O^T = V^T P^T on 16x16x32 MFMAs (32x32x16 in the second kernel): a lane's results belong to one column, the
// accumulator of S^T (lane (c, quarter): keys 4 quarter + i of a 16-key tile) is the operand that the second product wants once its 32
// keys are counted in that order, and the codes of four keys and eight dimensions that a lane loads with one instruction are
// its own part of V^T, so neither the weights nor the values cross lanes or LDS.
#include "kv_device.hpp"

#include <algorithm>

namespace lora {
namespace kv {
namespace {

__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <int D> struct Codes {
    static constexpr int W = D / 32;      // dwords of a lane's part of a key tile (32 or 16 codes) and of a value tile
    uint32_t k[4][W], v[4][W];
    uint32_t ke;
    u32x4 ve;
};

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

template <int D> __device__ inline void load_keys(Codes<D>& c, const uint8_t* part, int lane)
{
    const int m = lane & 15, quad = lane >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words(c.k[t], part + Part<D>::kK + (16 * t + m) * Part<D>::kRow + quad * (D / 8));
    c.ke = *reinterpret_cast<const uint32_t*>(part + Part<D>::kKExp + Part<D>::k_exp_at(m, quad * (D / 4) / kGroup));
}
template <int D> __device__ inline void load_values(Codes<D>& c, const uint8_t* part, int lane)
{
    const int m = lane & 15, quad = lane >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words(c.v[t], part + Part<D>::kV + Part<D>::v_at(16 * t + 4 * quad, m * Part<D>::kE));
    c.ve = *reinterpret_cast<const u32x4*>(part + Part<D>::kVExp + Part<D>::v_exp_at(4 * quad, m * Part<D>::kE / kGroup));
}

// Weighted sum of a tile's columns: m and l for the lane's column (l: of the lane's own keys only), acc[j][i]: dimension
// E (4 quarter + i) + j of the lane's column.
template <int D> struct Running {
    float m, l;
    f32x4 acc[D / 16];
};

// One block of 64 keys, and the request for the codes of the wave's next one (at `next`) as soon as this one's have been used: keys
// travel during the second half of the block, values during the first half of the next.  limit: the last key position of the lane's
// column, relative to the block's first; masked: some column does not see the whole block.
template <int D> __device__ inline void one_block(Running<D>& r, Codes<D>& c, const u32x4 (&q)[D / 32], float scale_log2, int limit, bool masked,
                                                  const uint8_t* next, int lane)
{
    constexpr int S = D / 32;
    const int quad = lane >> 4;
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t e = t == 0 ? c.ke << 23 : t == 1 ? c.ke << 15 : t == 2 ? c.ke << 7 : c.ke >> 1;
        s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < S; ++k) s[t] = mfma16(eight_bf16(c.k[t][k], e), q[k], s[t]);
    }
    load_keys<D>(c, next, lane);
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[t][i] *= scale_log2;
            if (masked && 16 * t + 4 * quad + i > limit) s[t][i] = -INFINITY;
            top = fmaxf(top, s[t][i]);
        }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m = fmaxf(r.m, top);
    // a column that has seen no key yet keeps m = -inf: its weights are 2^-inf = 0, not 2^(-inf + inf)
    const float base = m == -INFINITY ? 0.f : m;
    if (__any(m > r.m)) {
        const float down = exp2_fast(r.m - base);
        r.l *= down;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) r.acc[j] *= down;
        r.m = m;
    }
    uint32_t p[4][2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = exp2_fast(s[t][i] - base);
            r.l += w[i];
        }
        p[t][0] = pack_bf16(w[0], w[1]);
        p[t][1] = pack_bf16(w[2], w[3]);
    }
    // V^T of 32 keys: keys 4 quarter .. + 3 of tile 2 h, then of tile 2 h + 1.  A key's codes come two dimensions at a time; two keys'
    // results are dealt into the two dimensions' operands.
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32x4 w = {p[2 * h][0], p[2 * h][1], p[2 * h + 1][0], p[2 * h + 1][1]};
        u32x4 f[D / 16];
#pragma unroll
        for (int x = 0; x < 4; ++x) {                  // keys 2 x, 2 x + 1 of the eight
            const int t = 2 * h + x / 2, i = 2 * (x & 1);
            const uint32_t e = c.ve[t];
            const uint32_t e0 = i == 0 ? e << 23 : e << 7, e1 = i == 0 ? e << 15 : e >> 1;
            auto deal = [&](int d, uint32_t a, uint32_t b) {
                f[d][x] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                f[d + 1][x] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            };
            if constexpr (D == 128) {
                const uint32_t a = c.v[t][i], b = c.v[t][i + 1];
                deal(0, two_bf16<0>(a, e0), two_bf16<0>(b, e1));
                deal(2, two_bf16<1>(a, e0), two_bf16<1>(b, e1));
                deal(4, two_bf16<2>(a, e0), two_bf16<2>(b, e1));
                deal(6, two_bf16<3>(a, e0), two_bf16<3>(b, e1));
            } else {
                const uint32_t a = c.v[t][i / 2];      // both keys in one dword, four codes each
                deal(0, two_bf16<0>(a, e0), two_bf16<2>(a, e1));
                deal(2, two_bf16<1>(a, e0), two_bf16<3>(a, e1));
            }
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) r.acc[j] = mfma16(f[j], w, r.acc[j]);
    }
    load_values<D>(c, next, lane);
}

// Token and head that a request's column is; false: there is none in the step.
__device__ inline bool column(const Request& r, int group, int T, int col, int& token, int& head)
{
    token = col / group;
    head = col - token * group;
    return token < r.rows && r.first + token < T;
}

template <int D> __global__ __launch_bounds__(256, 3) void attend_few_kernel(AttendArgs a)
{
    constexpr int kPad = 4;
    __shared__ float sAcc[4][kFewCols][D + kPad];
    __shared__ float sM[4][kFewCols], sL[4][kFewCols];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c = lane & 15, quad = lane >> 4;
    const int n_items = a.t.head->n_few * a.n_kv;
    for (int item = blockIdx.x; item < n_items; item += gridDim.x) {
        const Entry e = a.t.few[item / a.n_kv];
        const int h = item % a.n_kv;
        const Request r = a.t.request[e.request];
        int token, head;
        const bool real = column(r, a.group, a.T, e.tile * kFewCols + c, token, head);
        const int limit = r.len + token;                                    // last key that the lane's column sees
        Running<D> run;
        run.m = -INFINITY;
        run.l = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) run.acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 q[D / 32];
        {
            const size_t row = min(r.first + (real ? token : 0), a.T - 1);
            const uint16_t* p = a.q + row * a.q_stride + ((size_t)h * a.group + head) * D + quad * (D / 4);
#pragma unroll
            for (int k = 0; k < D / 32; ++k) q[k] = load16(p + 8 * k);
        }
        const int32_t* blocks = a.t.table + (size_t)(r.held >= 0 ? r.row : 0) * a.t.row_blocks;
        // (a row that has been released since the plan has no block there)
        auto part = [&](int b) {
            return a.cache + ((size_t)min((unsigned)blocks[b], (unsigned)a.t.n_blocks - 1) * a.n_kv + h) * Part<D>::kBytes;
        };
        const int end = e.block + e.blocks;
        int b = e.block + wave;
        if (b < end) {
            Codes<D> codes;
            const uint8_t* next = part(b);
            load_keys<D>(codes, next, lane);
            load_values<D>(codes, next, lane);
            next = part(min(b + 4, end - 1));
            for (; b < end; b += 4) {
                const uint8_t* after = part(min(b + 8, end - 1));
                one_block<D>(run, codes, q, a.scale_log2, limit - b * kBlock, b * kBlock + kBlock - 1 > r.len, next, lane);
                next = after;
            }
        }
        // the four waves' results
        run.l += __shfl_xor(run.l, 16);
        run.l += __shfl_xor(run.l, 32);
        __syncthreads();                                                    // the tile before has been read
        if (quad == 0) {
            sM[wave][c] = run.m;
            sL[wave][c] = run.l;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 16; j += 4)
                *reinterpret_cast<f32x4*>(&sAcc[wave][c][(D / 16) * (4 * quad + i) + j]) =
                    f32x4{run.acc[j][i], run.acc[j + 1][i], run.acc[j + 2][i], run.acc[j + 3][i]};
        __syncthreads();
        constexpr int V = D * kFewCols / 256;                               // values of a thread
        const int cc = tid / 16, d0 = (tid % 16) * V;
        if (!column(r, a.group, a.T, e.tile * kFewCols + cc, token, head)) continue;    // (no barrier behind this in the loop but the next item's first)
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, sM[w][cc]);
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f, acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = exp2_fast(sM[w][cc] - base);
            l += f * sL[w][cc];
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += f * sAcc[w][cc][d0 + j];
        }
        if (e.part >= 0) {
            const size_t slot = ((size_t)e.part * a.n_kv + h) * kFewCols + cc;
#pragma unroll
            for (int j = 0; j < V; ++j) a.few_acc[slot * D + d0 + j] = acc[j];
            if (tid % 16 == 0) {
                a.few_ml[slot * 2] = m;
                a.few_ml[slot * 2 + 1] = l;
            }
        } else {
            const float f = l == 0.f ? 0.f : 1.0f / l;                      // no key at all: a refused request, its rows are zero
            uint16_t* o = a.out + (size_t)(r.first + token) * a.out_stride + ((size_t)h * a.group + head) * D + d0;
#pragma unroll
            for (int j = 0; j < V; j += 2) *reinterpret_cast<uint32_t*>(o + j) = pack_bf16(acc[j] * f, acc[j + 1] * f);
        }
    }
}

// ---- tiles of many columns ----
// A workgroup's codes of a block of 64 keys, as its 256 threads load them: K: key tid / 4, a quarter of its dimensions; V: two
// chunks of four keys (those that a lane of the second product wants together), kE dimensions, of which the thread converts half.
template <int D> struct Raw {
    uint32_t k[D / 32], v[2][D / 32], ke, ve[2];
};

struct Place {
    int key, quarter;          // K
    int u, h, half, m;         // V: keys 16 u + 4 h .. + 3 and 16 u + 8 + 4 h .. + 3, dimensions kE m .. 
};
__device__ inline Place place()
{
    const int t = threadIdx.x;
    return Place{t >> 2, t & 3, t >> 6, (t >> 5) & 1, (t >> 4) & 1, t & 15};
}

template <int D> __device__ inline void load_raw(Raw<D>& r, const uint8_t* part, const Place& p)
{
    using P = Part<D>;
    load_words(r.k, part + P::kK + p.key * P::kRow + p.quarter * (D / 8));
    r.ke = part[P::kKExp + P::k_exp_at(p.key, p.quarter * (D / 4) / kGroup)];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        load_words(r.v[c], part + P::kV + P::v_at(16 * p.u + 8 * c + 4 * p.h, p.m * P::kE));
        r.ve[c] = *reinterpret_cast<const uint32_t*>(part + P::kVExp + P::v_exp_at(16 * p.u + 8 * c + 4 * p.h, p.m * P::kE / kGroup));
    }
}

// The block in LDS: every operand of an MFMA is 64 lanes * 16 bytes, in lane order but for a permutation inside groups of eight that
// spreads a wave's writes over the banks.  K: [key / 32][D / 16], V: [d / 32][key / 16].
template <int D> struct Tile {
    static constexpr int kKFrags = 2 * (D / 16), kVFrags = (D / 32) * 4;
    u32x4 k[kKFrags * 64], v[kVFrags * 64];
    __device__ static int k_at(int tile, int s, int h, int i) { return (tile * (D / 16) + s) * 64 + h * 32 + (i ^ (2 * (s * 16 / (D / 4)))); }
    __device__ static int v_at(int dt, int u, int h, int i) { return (dt * 4 + u) * 64 + h * 32 + (i ^ (2 * ((i >> 3) & 3) + (dt & 1))); }
};

template <int D> __device__ inline void convert(Tile<D>& t, const Raw<D>& r, const Place& p)
{
    constexpr int E = Part<D>::kE;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        const int d = p.quarter * (D / 4) + 8 * j;
        t.k[Tile<D>::k_at(p.key >> 5, d >> 4, (d >> 3) & 1, p.key & 31)] = eight_bf16(r.k[j], r.ke << 23);
    }
    u32x4 f[E / 2];
#pragma unroll
    for (int x = 0; x < 4; ++x) {                      // keys 2 x, 2 x + 1 of the thread's eight
        const int c = x / 2, i = 2 * (x & 1);
        const uint32_t e0 = i == 0 ? r.ve[c] << 23 : r.ve[c] << 7, e1 = i == 0 ? r.ve[c] << 15 : r.ve[c] >> 1;
        uint32_t a, b;
        if constexpr (D == 128) {
            a = r.v[c][i] >> (16 * p.half);
            b = r.v[c][i + 1] >> (16 * p.half);
        } else {
            a = r.v[c][i / 2] >> (8 * p.half);
            b = a >> 16;
        }
#pragma unroll
        for (int j = 0; j < E / 4; ++j) {
            const uint32_t y = j == 0 ? two_bf16<0>(a, e0) : two_bf16<1>(a, e0), z = j == 0 ? two_bf16<0>(b, e1) : two_bf16<1>(b, e1);
            f[2 * j][x] = __builtin_amdgcn_perm(z, y, 0x05040100u);
            f[2 * j + 1][x] = __builtin_amdgcn_perm(z, y, 0x07060302u);
        }
    }
#pragma unroll
    for (int j = 0; j < E / 2; ++j) {
        const int d = E * p.m + (E / 2) * p.half + j;
        t.v[Tile<D>::v_at(d >> 5, p.u, p.h, d & 31)] = f[j];
    }
}

__device__ inline float max_halves(float x)
{
    return fmaxf(x, __shfl_xor(x, 32));
}

// Weights may grow to 2^kSlack times those of the running maximum before the sums are scaled down: most blocks then leave them alone.
constexpr float kSlack = 8.f;

template <int D> __global__ __launch_bounds__(256, 2) void attend_many_kernel(AttendArgs a)
{
    constexpr int S = D / 16, N = D / 32;
    __shared__ Tile<D> tiles[2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 31, h = lane >> 5;
    const int item = blockIdx.x;
    if (item >= a.t.head->n_many * a.n_kv) return;
    const Entry e = a.t.many[item / a.n_kv];
    const int hk = item % a.n_kv;
    const Request r = a.t.request[e.request];
    int token, head;
    const bool real = column(r, a.group, a.T, e.tile * kManyCols + wave * 32 + i, token, head);
    const int limit = real ? r.len + token : -1;
    const Place pl = place();
    const int32_t* blocks = a.t.table + (size_t)(r.held >= 0 ? r.row : 0) * a.t.row_blocks;
    const uint8_t* cache = a.cache + (size_t)hk * Part<D>::kBytes;
    const size_t stride = (size_t)a.n_kv * Part<D>::kBytes;
    // (a row that has been released since the plan has no block there)
    auto part = [&](int b) { return cache + (size_t)min((unsigned)blocks[b], (unsigned)a.t.n_blocks - 1) * stride; };

    u32x4 q[S];
    {
        const size_t row = min(r.first + (real ? token : 0), a.T - 1);
        const uint16_t* p = a.q + row * a.q_stride + ((size_t)hk * a.group + (real ? head : 0)) * D + 8 * h;
#pragma unroll
        for (int s = 0; s < S; ++s) q[s] = load16(p + 16 * s);
    }
    f32x16 o[N];
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[d][x] = 0.f;
    float m = -INFINITY, l = 0.f;
    const float scale = a.scale_log2 > 0.f ? a.scale_log2 : 1.f;

    Raw<D> raw;
    const int end = e.block + e.blocks;
    if (e.blocks > 0) {
        load_raw<D>(raw, part(e.block), pl);
        convert<D>(tiles[0], raw, pl);
        load_raw<D>(raw, part(min(e.block + 1, end - 1)), pl);
    }
    for (int b = e.block, at = 0; b < end; ++b, at ^= 1) {
        __syncthreads();                               // this block's tile is complete, and the other one has been read
        if (b + 1 < end) {
            convert<D>(tiles[at ^ 1], raw, pl);
            load_raw<D>(raw, part(min(b + 2, end - 1)), pl);
        }
        const Tile<D>& t = tiles[at];
        f32x16 s[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int x = 0; x < 16; ++x) s[k][x] = 0.f;
#pragma unroll
            for (int j = 0; j < S; ++j) s[k] = mfma32(as_bf16x8(t.k[Tile<D>::k_at(k, j, h, i)]), as_bf16x8(q[j]), s[k]);
        }
        // (a positive scale is applied in the exponent below; it keeps the order of the scores)
        if (a.scale_log2 <= 0.f) {
#pragma unroll
            for (int k = 0; k < 2; ++k) s[k] *= a.scale_log2;
        }
        if (b * kBlock + kBlock - 1 > r.len) {         // some column may not see the whole block
            const int room = limit - b * kBlock - 4 * h;
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
        if (__any(top > m + kSlack)) {
            const float grown = fmaxf(m, top);
            const float down = exp2_fast(m - (grown == -INFINITY ? 0.f : grown));
            l *= down;
#pragma unroll
            for (int d = 0; d < N; ++d) o[d] *= down;
            m = grown;
        }
        const float base = m == -INFINITY ? 0.f : m;
        u32x4 w[4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int x = 0; x < 16; x += 2) {
                const float p0 = exp2_fast(__builtin_fmaf(s[k][x], scale, -base)), p1 = exp2_fast(__builtin_fmaf(s[k][x + 1], scale, -base));
                l += p0 + p1;
                w[2 * k + x / 8][(x % 8) / 2] = pack_bf16(p0, p1);
            }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int d = 0; d < N; ++d) o[d] = mfma32(as_bf16x8(t.v[Tile<D>::v_at(d, u, h, i)]), as_bf16x8(w[u]), o[d]);
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
        const float f = l == 0.f ? 0.f : 1.0f / l;
        uint16_t* out = a.out + (size_t)(r.first + token) * a.out_stride + ((size_t)hk * a.group + head) * D + 4 * h;
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<u32x2*>(out + 32 * d + 8 * g) =
                    u32x2{pack_bf16(o[d][4 * g] * f, o[d][4 * g + 1] * f), pack_bf16(o[d][4 * g + 2] * f, o[d][4 * g + 3] * f)};
    }
}

// The partial results of tiles that were cut along their keys.  D / 4 lanes take a column, four dimensions each.  Where there are many
// pieces, a workgroup's groups of lanes share those of one column (blockIdx.y).
template <int D> __global__ __launch_bounds__(256) void merge_kernel(AttendArgs a)
{
    constexpr int L = D / 4, GROUPS = 256 / L;
    __shared__ float sAcc[GROUPS][D], sL[GROUPS];
    const int tid = threadIdx.x, lane = tid % L, group = tid / L;
    const int n_items = a.t.head->n_merge * a.n_kv;
    for (int item = blockIdx.x; item < n_items; item += gridDim.x) {
        const Merge g = a.t.merge[item / a.n_kv];
        const int h = item % a.n_kv, splits = abs(g.splits), cols = g.splits < 0 ? kManyCols : kFewCols;
        const float* part_acc = g.splits < 0 ? a.many_acc : a.few_acc;
        const float* part_ml = g.splits < 0 ? a.many_ml : a.few_ml;
        const Request r = a.t.request[g.request];
        const size_t slot0 = ((size_t)g.part * a.n_kv + h) * cols + g.col % cols, step = (size_t)a.n_kv * cols;
        const bool share = splits >= 2 * GROUPS;       // (the same for the whole workgroup, like everything but `group` and `lane`)
        if (!share && blockIdx.y) continue;
        for (int c = share ? (int)blockIdx.y : group; c < kMergeCols; c += share ? (int)gridDim.y : GROUPS) {
            int token, head;
            if (!column(r, a.group, a.T, g.col + c, token, head)) break;
            float m = -INFINITY, l = 0.f;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            const float* ml = part_ml + 2 * (slot0 + c);
            for (int s = share ? lane : 0; s < splits; s += share ? L : 1) m = fmaxf(m, ml[2 * step * s]);
            if (share)
                for (int d = 1; d < L; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
            const float base = m == -INFINITY ? 0.f : m;
            const float* p = part_acc + (slot0 + c) * D + 4 * lane;
#pragma unroll 4
            for (int s = share ? group : 0; s < splits; s += share ? GROUPS : 1) {
                const float f = exp2_fast(ml[2 * step * s] - base);
                l += f * ml[2 * step * s + 1];
                acc += f * *reinterpret_cast<const f32x4*>(p + step * D * s);
            }
            if (share) {
                __syncthreads();
                *reinterpret_cast<f32x4*>(&sAcc[group][4 * lane]) = acc;
                if (lane == 0) sL[group] = l;
                __syncthreads();
                acc = f32x4{0.f, 0.f, 0.f, 0.f};
                l = 0.f;
#pragma unroll
                for (int w = 0; w < GROUPS; ++w) {
                    acc += *reinterpret_cast<const f32x4*>(&sAcc[w][4 * lane]);
                    l += sL[w];
                }
                if (group) continue;
            }
            const float f = l == 0.f ? 0.f : 1.0f / l;
            uint16_t* o = a.out + (size_t)(r.first + token) * a.out_stride + ((size_t)h * a.group + head) * D + 4 * lane;
            *reinterpret_cast<u32x2*>(o) = u32x2{pack_bf16(acc[0] * f, acc[1] * f), pack_bf16(acc[2] * f, acc[3] * f)};
        }
    }
}

template <int D> hipError_t attend(const AttendArgs& a, int n_cus, long most_few, long most_many, hipStream_t stream)
{
    if (most_many > 0) attend_many_kernel<D><<<(unsigned)(most_many * a.n_kv), 256, 0, stream>>>(a);
    const int grid = (int)std::max<long>(1, std::min<long>(most_few * a.n_kv, 3L * n_cus));
    attend_few_kernel<D><<<grid, 256, 0, stream>>>(a);
    merge_kernel<D><<<dim3(4 * n_cus, 4), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const AttendArgs& a, int dim, int n_cus, long most_few, long most_many, hipStream_t stream)
{
    if (a.T == 0) return hipSuccess;
    return dim == 64 ? attend<64>(a, n_cus, most_few, most_many, stream) : attend<128>(a, n_cus, most_few, most_many, stream);
}

}  // namespace kv
}  // namespace lora
