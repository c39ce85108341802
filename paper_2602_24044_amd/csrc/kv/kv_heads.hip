// Norm of queries and keys for each head with the position rotation in the same pass, on its own and on the way into the cache in
// four bits; and the way out of the cache.
//
//   u = x / sqrt(mean(x^2) + eps) * w            (where there is a weight)
//   y_p = u_p cos a - u_p' sin a,  y_p' = u_p' cos a + u_p sin a,   a = position * f_p,  p' = p + D/2 (or its neighbour)
//
// One read and one write of every head, so the copy rate bounds it: 4099 tokens of 28 + 4 heads of 128 with norm, 67 MB, in 14.9 us (4.5
// TB/s); 8190 tokens of 64 + 8 heads with norm into the cache, 313 MB, in 65 us (4.8 TB/s; the vector unit is busy for half of it), and
// their keys and values out of it in 15.8.  D / 8 lanes share a head's row, 16 bytes each; the other half of a rotated pair sits D / 16
// lanes away.  Angles are taken in 64 bits (a far position times a frequency has few bits left behind the point in 32) once per token and
// pair, and shared by all heads through LDS.  Keys on the way to four bits are computed in 64 bits throughout and rounded to 32 once: next
// to a border between two codes an error of 2^-24 would pick the wrong one now and then.
#include "kv_device.hpp"

#include <algorithm>
#include <type_traits>

namespace lora {
namespace kv {
namespace {

// sin and cos of a in 64 bits: a - n pi/2 with pi/2 in two parts, then the Taylor sums up to r^17 (|r| <= pi/4: the next term is
// below 2^-56).
__device__ inline void sin_cos(double a, double& s, double& c)
{
    const double n = __builtin_rint(a * 0.63661977236758134308);
    double r = __builtin_fma(-n, 1.5707963267948966192, a);
    r = __builtin_fma(-n, 6.1232339957367658e-17, r);
    const double z = r * r;
    double ps = 1.0 / 355687428096000.0;
    ps = __builtin_fma(ps, z, -1.0 / 1307674368000.0);
    ps = __builtin_fma(ps, z, 1.0 / 6227020800.0);
    ps = __builtin_fma(ps, z, -1.0 / 39916800.0);
    ps = __builtin_fma(ps, z, 1.0 / 362880.0);
    ps = __builtin_fma(ps, z, -1.0 / 5040.0);
    ps = __builtin_fma(ps, z, 1.0 / 120.0);
    ps = __builtin_fma(ps, z, -1.0 / 6.0);
    const double sr = __builtin_fma(ps * z, r, r);
    double pc = 1.0 / 20922789888000.0;
    pc = __builtin_fma(pc, z, -1.0 / 87178291200.0);
    pc = __builtin_fma(pc, z, 1.0 / 479001600.0);
    pc = __builtin_fma(pc, z, -1.0 / 3628800.0);
    pc = __builtin_fma(pc, z, 1.0 / 40320.0);
    pc = __builtin_fma(pc, z, -1.0 / 720.0);
    pc = __builtin_fma(pc, z, 1.0 / 24.0);
    pc = __builtin_fma(pc, z, -0.5);
    const double cr = __builtin_fma(pc, z, 1.0);
    // quarter turns: n modulo 4 (n itself may not fit an int)
    const int k = (int)(n - 4.0 * __builtin_floor(n * 0.25));
    s = (k & 1) ? cr : sr;
    c = (k & 1) ? sr : cr;
    if (k == 2 || k == 3) s = -s;
    if (k == 1 || k == 2) c = -c;
}


// Over the L lanes of a row: the value of the lane L / 2 away, and the sum.  With 16 lanes a row is one of the vector unit's.
template <int L, typename T> __device__ inline T across(T v)
{
    static_assert(sizeof(T) == 4, "");
    if constexpr (L == 16) return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x128, 0xf, 0xf, true));
    else return __shfl_xor(v, L / 2);
}
template <int L> __device__ inline float row_sum(float v)
{
    if constexpr (L == 16) {
        auto turn = [](float x, auto by) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(by)::value, 0xf, 0xf, true)); };
        v += turn(v, std::integral_constant<int, 0x128>());
        v += turn(v, std::integral_constant<int, 0x124>());
        v += turn(v, std::integral_constant<int, 0x122>());
        return v + turn(v, std::integral_constant<int, 0x121>());
    } else {
#pragma unroll
        for (int d = 1; d < L; d <<= 1) v += __shfl_xor(v, d);
        return v;
    }
}
template <int L> __device__ inline double row_sum(double v)
{
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

template <int L> __device__ inline float row_max(float v)
{
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

__device__ inline float reciprocal_root(float x) { return __builtin_amdgcn_rsqf(x); }
// The unit's estimate has some 23 bits or more: two Newton steps, y += y (1 - x y^2) / 2.  (Zero and infinity keep what the estimate says.)
__device__ inline double reciprocal_root(double x)
{
    double y = __builtin_amdgcn_rsq(x);
    if (y < 1e300 && y > 0.0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) y = __builtin_fma(0.5 * y, __builtin_fma(-x * y, y, 1.0), y);
    }
    return y;
}

// What the rows of a token share: y = (x a + x' b) / rms for every value x and its partner x', a = w cos and b = -+ w' sin with the weights
// of the norm in them (the angle's sine with the sign that the value's place in its pair has).  In LDS in the order in which lanes read: 16
// bytes each, lanes side by side.  R = float (queries, and keys that stay bf16) or double (keys on their way to four bits).
template <typename R> struct Pair {
    R a, b;
};
template <int D, typename R> __device__ inline int pair_at(int d)
{
    constexpr int L = D / 8, per = sizeof(R) == 4 ? 2 : 1;
    return ((d % 8) / per * L + d / 8) * per + d % per;
}
template <int D, typename R> struct Turn {
    Pair<R> p[8];
    __device__ void load(const Pair<R>* of, int l)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = of[pair_at<D, R>(8 * l + j)];
    }
};

__device__ inline double bf16_at(const uint16_t* w, int d) { return w ? (double)__builtin_bit_cast(float, (uint32_t)w[d] << 16) : 1.0; }

// The two values of pair k, which turns by the angle of (sine, cosine).
template <int D, typename R> __device__ inline void put_pair(Pair<R>* to, int k, bool pairs, double sine, double cosine, const uint16_t* w)
{
    const int d0 = pairs ? 2 * k : k, d1 = pairs ? 2 * k + 1 : k + D / 2;
    const double w0 = bf16_at(w, d0), w1 = bf16_at(w, d1);
    to[pair_at<D, R>(d0)] = Pair<R>{(R)(cosine * w0), (R)(-sine * w1)};
    to[pair_at<D, R>(d1)] = Pair<R>{(R)(cosine * w1), (R)(sine * w0)};
}

// A power of two that a row of 32-bit numbers can be multiplied by for its norm, which does not hang on it as long as eps is multiplied by its
// square: the largest value, or the root of eps where that is larger, comes to 1 .. 2 or near it.
template <int L> __device__ inline float norm_power(const u32x4 raw, float eps)
{
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(__builtin_fabsf(lo_f32(raw[j])), __builtin_fabsf(hi_f32(raw[j]))));
    const int k = (int)(__builtin_bit_cast(uint32_t, row_max<L>(top)) >> 23) - 127;
    const int root = eps == 0.f ? -126 : ((int)(__builtin_bit_cast(uint32_t, eps) >> 23) - 126) >> 1;
    return __builtin_bit_cast(float, (uint32_t)(127 - min(max(max(k, root), -126), 126)) << 23);
}

// Norm and rotation of one row of D values, eight of them in a lane.  False, to all of the row's lanes alike: computed in 32 bits, and the mean
// square lies outside of 2^-40 .. 2^40, where squares begin to leave the type's range; y is of no use then, and the row has to be multiplied by
// its norm_power.  (The question costs rows of ordinary size 2 %: a pass over the 4099 tokens above 15.4 instead of 15.0 us.)
template <int D, typename R, bool SCALED = false>
__device__ inline bool norm_rotate(const u32x4 raw, bool norm, float eps, const Turn<D, R>& t, bool rotate, bool pairs, R (&y)[8], float power = 1.f)
{
    constexpr int L = D / 8;
    auto in = [&](float v) { return (R)(SCALED ? v * power : v); };
    R x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = in(lo_f32(raw[j]));
        x[2 * j + 1] = in(hi_f32(raw[j]));
    }
    if (!rotate) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = norm ? x[j] * t.p[j].a : x[j];
    } else if (pairs) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j] * t.p[j].a + x[j ^ 1] * t.p[j].b;
    } else {
        // the partners as they were read (half the exchange)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t o = across<L>(raw[j]);
            y[2 * j] = x[2 * j] * t.p[2 * j].a + in(lo_f32(o)) * t.p[2 * j].b;
            y[2 * j + 1] = x[2 * j + 1] * t.p[2 * j + 1].a + in(hi_f32(o)) * t.p[2 * j + 1].b;
        }
    }
    if (norm) {
        R sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[j] * x[j];
        const R mean = row_sum<L>(sum) * (R)(1.0 / D) + (R)(SCALED ? eps * power * power : eps);
        const R inv = reciprocal_root(mean);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= inv;
        if (sizeof(R) == 4 && !SCALED) return mean >= (R)0x1p-40 && mean <= (R)0x1p40;
    }
    return true;
}

// Eight fp32 values of a lane into codes, their group's exponent shared by four lanes.
__device__ inline uint32_t to_codes(float (&v)[8], int& exponent, bool& odd)
{
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (!(__builtin_fabsf(v[j]) <= 3.4028235e38f)) odd = true;
        if (v[j] != v[j]) v[j] = 0.f;
        top = fmaxf(top, __builtin_fabsf(v[j]));
    }
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    exponent = group_exponent(top);
    return eight_codes(v, __builtin_bit_cast(float, (uint32_t)exponent << 23));
}

template <int D> __device__ inline void put_v(uint8_t* part, int k, int l, uint32_t codes)
{
    uint8_t* v = part + Part<D>::kV;
    if constexpr (D == 128) {
        *reinterpret_cast<uint32_t*>(v + Part<D>::v_at(k, 8 * l)) = codes;
    } else {
        *reinterpret_cast<uint16_t*>(v + Part<D>::v_at(k, 8 * l)) = (uint16_t)codes;
        *reinterpret_cast<uint16_t*>(v + Part<D>::v_at(k, 8 * l + 4)) = (uint16_t)(codes >> 16);
    }
}
template <int D> __device__ inline uint32_t get_v(const uint8_t* part, int k, int l)
{
    const uint8_t* v = part + Part<D>::kV;
    if constexpr (D == 128) return *reinterpret_cast<const uint32_t*>(v + Part<D>::v_at(k, 8 * l));
    return *reinterpret_cast<const uint16_t*>(v + Part<D>::v_at(k, 8 * l)) |
           (uint32_t)*reinterpret_cast<const uint16_t*>(v + Part<D>::v_at(k, 8 * l + 4)) << 16;
}

// A workgroup takes a token: rows of queries (and of keys that stay bf16) go through its lane groups four at a time, then those that
// end in the cache, keys and values side by side.  (Four tokens a workgroup: 25.4 us instead of 25.2 for the rotation of 4096 tokens of 32 + 8
// heads out of HBM, 16.2 instead of 14.1 for 2048; into the cache 33.4 instead of 36.6, but 21.8 instead of 20.0.)
template <int D, bool CACHE> __global__ __launch_bounds__(256) void heads_kernel(HeadsArgs a)
{
    using K = std::conditional_t<CACHE, double, float>;
    constexpr int L = D / 8, ROWS = 256 / L, U = 4, KV = 2;
    __shared__ __align__(16) Pair<float> q_pairs[D];
    __shared__ __align__(16) Pair<K> k_pairs[D];
    const size_t t = blockIdx.x;
    if (CACHE && (int)t >= a.head->rows) return;
    const bool rotate = a.inv_freq != nullptr;
    const int l = threadIdx.x % L, group = threadIdx.x / L;
    const int slot = CACHE ? a.slot[t] : 0;
    // The first rows on their way to the cache are asked for in front of everything else.
    u32x4 rows[KV];
    auto fetch = [&](int from) {
#pragma unroll
        for (int u = 0; u < KV; ++u) {
            const int h = from + u * ROWS;
            if (h < 2 * a.n_kv) rows[u] = load16((h < a.n_kv ? a.k + t * a.k_stride + (size_t)h * D : a.v + t * a.v_stride + (size_t)(h - a.n_kv) * D) + 8 * l);
        }
    };
    if constexpr (CACHE) fetch(group);
    if (rotate || a.q_norm || a.k_norm) {
        for (int k = threadIdx.x; k < D / 2; k += 256) {
            double s = 0.0, c = 1.0;
            if (rotate) sin_cos((double)a.position[t] * (double)a.inv_freq[k], s, c);
            if (a.q) put_pair<D, float>(q_pairs, k, a.pairs, s, c, a.q_norm);
            if (a.k) put_pair<D, K>(k_pairs, k, a.pairs, s, c, a.k_norm);
        }
        __syncthreads();
    }

    auto dense = [&](const uint16_t* in, int64_t in_stride, uint16_t* out, int64_t out_stride, const Pair<float>* shared, bool norm, int heads) {
        Turn<D, float> turn;
        if (rotate || norm) turn.load(shared, l);
        const uint16_t* from = in + t * in_stride + 8 * l;
        uint16_t* to = out + t * out_stride + 8 * l;
        auto put = [&](int h, const float (&y)[8]) {
            u32x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = slot >= 0 ? pack_bf16(y[2 * j], y[2 * j + 1]) : 0u;
            *reinterpret_cast<u32x4*>(to + (size_t)h * D) = o;
        };
        static_assert(kMaxHeads <= 64 * ROWS, "a bit for each of a lane group's rows");
        uint64_t left = 0;
        for (int h0 = group; h0 < heads; h0 += U * ROWS) {
            u32x4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h0 + u * ROWS < heads) raw[u] = load16(from + (size_t)(h0 + u * ROWS) * D);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * ROWS;
                if (h >= heads) continue;
                float y[8];
                if (norm_rotate<D>(raw[u], norm, a.eps, turn, rotate, a.pairs, y)) put(h, y);
                else left |= 1ull << (h / ROWS);
            }
        }
        // rows far from 1, which have not been written yet (in 64 bits they would cost every row twice the registers)
#pragma unroll 1
        for (int h = group; left; h += ROWS, left >>= 1) {
            if (!(left & 1)) continue;
            const u32x4 raw = load16(from + (size_t)h * D);
            float y[8];
            norm_rotate<D, float, true>(raw, norm, a.eps, turn, rotate, a.pairs, y, norm_power<L>(raw, a.eps));
            put(h, y);
        }
    };
    if (a.q) dense(a.q, a.q_stride, a.q_out, a.q_out_stride, q_pairs, a.q_norm, a.n_heads);
    if constexpr (!CACHE) {
        if (a.k) dense(a.k, a.k_stride, a.k_out, a.k_out_stride, k_pairs, a.k_norm, a.n_kv);
    } else {
        if (slot < 0) return;                          // a refused request's
        bool odd = false;
        Turn<D, double> turn;
        if (rotate || a.k_norm) turn.load(k_pairs, l);
        for (int from = group; from < 2 * a.n_kv; from += KV * ROWS) {
            if (from != group) fetch(from);
#pragma unroll
            for (int u = 0; u < KV; ++u) {
                const int h = from + u * ROWS;
                if (h >= 2 * a.n_kv) continue;
                const bool is_k = h < a.n_kv;
                const int hk = is_k ? h : h - a.n_kv;
                float v[8];
                if (is_k) {
                    double y[8];
                    norm_rotate<D>(rows[u], a.k_norm, a.eps, turn, rotate, a.pairs, y);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = (float)y[j];
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v[2 * j] = lo_f32(rows[u][j]);
                        v[2 * j + 1] = hi_f32(rows[u][j]);
                    }
                }
                int exponent;
                const uint32_t codes = to_codes(v, exponent, odd);
                uint8_t* part = a.cache + ((size_t)(slot / kBlock) * a.n_kv + hk) * Part<D>::kBytes;
                const int k = slot % kBlock;
                if (is_k) *reinterpret_cast<uint32_t*>(part + Part<D>::kK + k * Part<D>::kRow + 4 * l) = codes;
                else put_v<D>(part, k, l, codes);
                if (l % 4 == 0)
                    part[is_k ? Part<D>::kKExp + Part<D>::k_exp_at(k, l / 4) : Part<D>::kVExp + Part<D>::v_exp_at(k, l / 4)] = (uint8_t)exponent;
            }
        }
        if (odd) atomicOr(&a.head->flags, kFlagNotFinite);
    }
}

template <int D> __global__ __launch_bounds__(256) void read_kernel(ReadArgs a)
{
    constexpr int L = D / 8, ROWS = 256 / L;
    const int l = threadIdx.x % L;
    const long r = (long)blockIdx.x * ROWS + threadIdx.x / L;
    const int per = 2 * a.n_kv;
    if (r >= (long)a.n * per) return;
    const int t = (int)(r / per), h = (int)(r - (long)t * per);
    const bool is_v = h >= a.n_kv;
    const int hk = is_v ? h - a.n_kv : h;
    const int row = a.seq[t], position = a.position[t];
    int block = -1;
    if ((unsigned)row < (unsigned)a.t.max_seqs && position >= 0 && position / kBlock < a.t.held[row])
        block = a.t.table[(size_t)row * a.t.row_blocks + position / kBlock];
    u32x4 o = {0, 0, 0, 0};
    if ((unsigned)block < (unsigned)a.t.n_blocks) {
        const uint8_t* part = a.cache + ((size_t)block * a.n_kv + hk) * Part<D>::kBytes;
        const int k = position % kBlock, g = l / 4;
        const uint32_t codes = is_v ? get_v<D>(part, k, l) : *reinterpret_cast<const uint32_t*>(part + Part<D>::kK + k * Part<D>::kRow + 4 * l);
        const uint32_t e = part[is_v ? Part<D>::kVExp + Part<D>::v_exp_at(k, g) : Part<D>::kKExp + Part<D>::k_exp_at(k, g)];
        o = eight_bf16(codes, e << 23);
    } else if (h == 0 && l == 0) {
        atomicOr(&a.t.head->flags, kFlagRefused);
    }
    uint16_t* out = is_v ? a.v_out : a.k_out;
    if (out) *reinterpret_cast<u32x4*>(out + (size_t)t * a.n_kv * D + (size_t)hk * D + 8 * l) = o;
}

template <int D> hipError_t heads(const HeadsArgs& a, hipStream_t stream)
{
    if (a.cache) heads_kernel<D, true><<<a.T, 256, 0, stream>>>(a);
    else heads_kernel<D, false><<<a.T, 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <int D> hipError_t read(const ReadArgs& a, hipStream_t stream)
{
    constexpr int rows = 256 / (D / 8);
    const int most = (1 << 26) / a.n_kv;               // tokens of a launch: its threads are counted in 32 bits
    for (int at = 0; at < a.n; at += most) {
        ReadArgs b = a;
        const size_t skip = (size_t)at * a.n_kv * D;
        b.n = std::min(most, a.n - at);
        b.seq += at;
        b.position += at;
        b.k_out = a.k_out ? a.k_out + skip : nullptr;
        b.v_out = a.v_out ? a.v_out + skip : nullptr;
        const long n = (long)b.n * 2 * b.n_kv;
        read_kernel<D><<<(unsigned)((n + rows - 1) / rows), 256, 0, stream>>>(b);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_heads(const HeadsArgs& a, int dim, hipStream_t stream)
{
    if (a.T == 0) return hipSuccess;
    return dim == 64 ? heads<64>(a, stream) : heads<128>(a, stream);
}

hipError_t launch_read(const ReadArgs& a, int dim, hipStream_t stream)
{
    if (a.n == 0) return hipSuccess;
    return dim == 64 ? read<64>(a, stream) : read<128>(a, stream);
}

}  // namespace kv
}  // namespace lora
