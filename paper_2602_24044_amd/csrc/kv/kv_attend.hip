// Attention of a step's tokens over the cache in four bits.
//
//   out[t, head] = sum_k p_k v_k,   p = softmax_k(scale q . k) over the keys at positions <= that of t
//
// in one pass over the keys: a running maximum m and sum l of the weights 2^(s - m), the accumulated values scaled down when m
// grows.  Scores, weights' sums, m and the accumulated values are fp32; the weights are rounded to bf16 for the matrix units (2^-9 of
// each, like the values' own rounding in a cache of 16 bits).
//
// A column is a query: (token j, head g of the key head's group), column j * group + g, so a group's heads share the keys that they
// read.  S^T = K Q^T and O^T = V^T P^T on 16x16x32 MFMAs, 16 columns a tile: a lane's results belong to one column, the
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

template <int D> __device__ inline void load_block(Codes<D>& c, const uint8_t* part, int lane)
{
    const int m = lane & 15, quad = lane >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words(c.k[t], part + Part<D>::kK + (16 * t + m) * Part<D>::kRow + quad * (D / 8));
    c.ke = *reinterpret_cast<const uint32_t*>(part + Part<D>::kKExp + Part<D>::k_exp_at(m, quad * (D / 4) / kGroup));
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

// One block of 64 keys.  limit: the last key position of the lane's column, relative to the block's first; masked: some column does
// not see the whole block.
template <int D> __device__ inline void one_block(Running<D>& r, const Codes<D>& c, const u32x4 (&q)[D / 32], float scale_log2, int limit, bool masked,
                                                  int quad)
{
    constexpr int S = D / 32;
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t e = t == 0 ? c.ke << 23 : t == 1 ? c.ke << 15 : t == 2 ? c.ke << 7 : c.ke >> 1;
        s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < S; ++k) s[t] = mfma16(eight_bf16(c.k[t][k], e), q[k], s[t]);
    }
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
}

// Row of the output and of the queries that column c of a tile is; false: there is none.
__device__ inline bool column(const Request& r, int group, int T, int tile, int c, int& token, int& head)
{
    const int col = tile * kFewCols + c;
    token = col / group;
    head = col - token * group;
    return token < r.rows && r.first + token < T;
}

template <int D> __global__ __launch_bounds__(256) void attend_few_kernel(AttendArgs a)
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
        const bool real = column(r, a.group, a.T, e.tile, c, token, head);
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
        for (int b = e.block + wave; b < e.block + e.blocks; b += 4) {
            const int at = blocks[b];
            if ((unsigned)at >= (unsigned)a.t.n_blocks) continue;           // the row has been released since the plan
            Codes<D> codes;
            load_block<D>(codes, a.cache + ((size_t)at * a.n_kv + h) * Part<D>::kBytes, lane);
            one_block<D>(run, codes, q, a.scale_log2, limit - b * kBlock, b * kBlock + kBlock - 1 > r.len, quad);
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
        if (!column(r, a.group, a.T, e.tile, cc, token, head)) continue;    // (no barrier behind this in the loop but the next item's first)
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
            for (int j = 0; j < V; ++j) a.part_acc[slot * D + d0 + j] = acc[j];
            if (tid % 16 == 0) {
                a.part_ml[slot * 2] = m;
                a.part_ml[slot * 2 + 1] = l;
            }
        } else {
            const float f = l == 0.f ? 0.f : 1.0f / l;                      // no key at all: a refused request, its rows are zero
            uint16_t* o = a.out + (size_t)(r.first + token) * a.out_stride + ((size_t)h * a.group + head) * D + d0;
#pragma unroll
            for (int j = 0; j < V; j += 2) *reinterpret_cast<uint32_t*>(o + j) = pack_bf16(acc[j] * f, acc[j + 1] * f);
        }
    }
}

// The partial results of a tile that was cut along its keys.
template <int D> __global__ __launch_bounds__(256) void merge_kernel(AttendArgs a)
{
    constexpr int V = D * kFewCols / 256;
    const int tid = threadIdx.x, cc = tid / 16, d0 = (tid % 16) * V;
    const int n_items = a.t.head->n_merge * a.n_kv;
    for (int item = blockIdx.x; item < n_items; item += gridDim.x) {
        const Merge g = a.t.merge[item / a.n_kv];
        const int h = item % a.n_kv;
        const Request r = a.t.request[g.request];
        int token, head;
        if (!column(r, a.group, a.T, g.tile, cc, token, head)) continue;
        float m = -INFINITY;
        for (int s = 0; s < g.splits; ++s) m = fmaxf(m, a.part_ml[(((size_t)(g.part + s) * a.n_kv + h) * kFewCols + cc) * 2]);
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f, acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
        for (int s = 0; s < g.splits; ++s) {
            const size_t slot = ((size_t)(g.part + s) * a.n_kv + h) * kFewCols + cc;
            const float f = exp2_fast(a.part_ml[slot * 2] - base);
            l += f * a.part_ml[slot * 2 + 1];
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += f * a.part_acc[slot * D + d0 + j];
        }
        const float f = l == 0.f ? 0.f : 1.0f / l;
        uint16_t* o = a.out + (size_t)(r.first + token) * a.out_stride + ((size_t)h * a.group + head) * D + d0;
#pragma unroll
        for (int j = 0; j < V; j += 2) *reinterpret_cast<uint32_t*>(o + j) = pack_bf16(acc[j] * f, acc[j + 1] * f);
    }
}

template <int D> hipError_t attend(const AttendArgs& a, int n_cus, long max_entries, hipStream_t stream)
{
    const int grid = (int)std::max<long>(1, std::min<long>(max_entries * a.n_kv, 4L * n_cus));
    attend_few_kernel<D><<<grid, 256, 0, stream>>>(a);
    merge_kernel<D><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const AttendArgs& a, int dim, int n_cus, long max_entries, hipStream_t stream)
{
    if (a.T == 0) return hipSuccess;
    return dim == 64 ? attend<64>(a, n_cus, max_entries, stream) : attend<128>(a, n_cus, max_entries, stream);
}

}  // namespace kv
}  // namespace lora
