// What the two kernels of the attention over a span share: a row's key ranges, the units a tile of rows walks, and the test for
// values of V that a weight of zero would not make vanish.
#pragma once
#include "kv4_format.h"
#include "tidar_internal.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLag = 16.f;                             // log2 of how far scores may outgrow the softmax reference
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// What one query row sees: cache keys [0, sk) and [lo, hi), mask rows [m0, ms) and [ml, m1).
struct RowSpan {
    int lo, hi, sk;
    int m0, ms, ml, m1;
};
__device__ inline RowSpan row_span(const RowDesc &d, int r, int L, int window, int sinks) {
    const RowInfo ri = row_info(d, r, L);
    RowSpan s;
    s.hi = L + ri.vis;
    s.lo = window > 0 ? max(0, ri.pos - window + 1) : 0;
    s.sk = window > 0 ? min(sinks, s.hi) : 0;
    s.m0 = s.ms = s.ml = s.m1 = 0;
    if (ri.blk >= 0) {                                   // mask row m of the block sits at position hi + m - m0
        s.m0 = ri.blk * d.bl;
        s.m1 = min(s.m0 + d.bl, d.nm);
        s.ml = max(s.m0, s.m0 + s.lo - s.hi);
        s.ms = window > 0 ? min(s.m1, s.m0 + sinks - s.hi) : s.m0;
    }
    return s;
}
__device__ inline unsigned bits16(int lo, int hi) {      // bits [lo, hi) of 16
    lo = min(max(lo, 0), 16);
    hi = min(max(hi, 0), 16);
    return hi > lo ? ((1u << hi) - 1u) & ~((1u << lo) - 1u) : 0u;
}

// The least and largest bounds over some rows (of rows that are there).
struct RowBounds {
    int lo0, lo1, hi0, hi1, sk0, sk1, m0, m1;
};
__device__ inline RowBounds bounds_of(const RowSpan &s, bool row) {
    const int most = 0x7fffffff;
    const bool mask = row && s.m1 > s.m0;
    return {row ? s.lo : most, row ? s.lo : 0, row ? s.hi : most, row ? s.hi : 0,
            row ? s.sk : most, row ? s.sk : 0, mask ? s.m0 : most, mask ? s.m1 : 0};
}
__device__ inline RowBounds join(const RowBounds &x, const RowBounds &y) {
    return {min(x.lo0, y.lo0), max(x.lo1, y.lo1), min(x.hi0, y.hi0), max(x.hi1, y.hi1),
            min(x.sk0, y.sk0), max(x.sk1, y.sk1), min(x.m0, y.m0), max(x.m1, y.m1)};
}
// over LANES lanes that hold a row each, in scalar registers
template <int LANES>
__device__ inline RowBounds wave_bounds(RowBounds x) {
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1)
        x = join(x, {__shfl_xor(x.lo0, o), __shfl_xor(x.lo1, o), __shfl_xor(x.hi0, o), __shfl_xor(x.hi1, o),
                     __shfl_xor(x.sk0, o), __shfl_xor(x.sk1, o), __shfl_xor(x.m0, o), __shfl_xor(x.m1, o)});
    auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return {u(x.lo0), u(x.lo1), u(x.hi0), u(x.hi1), u(x.sk0), u(x.sk1), u(x.m0), u(x.m1)};
}

// The units that rows within these bounds walk: cache units [0, n_s), [w0, w0 + n_w), then mask units [um0, um0 + n_m).
struct Walk {
    int n_s, w0, n_w, um0, n_m;
    int n1, n2;                                          // iterations over the cache and over the mask tiles
    __device__ int cache_unit(int w) const { return w < n_s ? w : w < n_s + n_w ? w0 + (w - n_s) : -1; }
    __device__ int mask_unit(int w) const { return w < n_m ? um0 + w : -1; }
};
__device__ inline Walk walk_of(const RowBounds &r, int window) {
    Walk w;
    w.n_s = window > 0 ? (r.sk1 + 15) >> 4 : 0;
    w.w0 = r.lo0 >> 4;
    const int w1 = (r.hi1 + 15) >> 4;
    if (w.n_s >= w.w0) {                                 // sinks and window meet
        w.n_s = 0;
        w.w0 = 0;
    }
    w.n_w = max(0, w1 - w.w0);
    w.um0 = r.m1 > 0 ? r.m0 >> 4 : 0;
    w.n_m = r.m1 > 0 ? ((r.m1 + 15) >> 4) - w.um0 : 0;
    w.n1 = (w.n_s + w.n_w + 1) >> 1;
    w.n2 = (w.n_m + 1) >> 1;
    return w;
}
// whether all of these rows see all of a cache unit
__device__ inline bool all_see(const RowBounds &r, int u) {
    return u >= 0 && 16 * u + 16 <= r.hi0 && (16 * u >= r.lo1 || 16 * u + 16 <= r.sk0);
}
// the keys of a unit that a row sees
__device__ inline unsigned cache_bits(const RowSpan &s, int u) {
    return u < 0 ? 0u : bits16(s.lo - 16 * u, s.hi - 16 * u) | bits16(-16 * u, s.sk - 16 * u);
}
__device__ inline unsigned mask_bits(const RowSpan &s, int u) {
    return u < 0 ? 0u : bits16(s.ml - 16 * u, s.m1 - 16 * u) | bits16(s.m0 - 16 * u, s.ms - 16 * u);
}

// ---- a drafted tree's rows: all of the cached prefix, and of the tree what their bits say (a word to two units of 16 rows)
constexpr int kTreeWords = TIDAR_MAX_TREE / 32;
// Sequence b's range of rows [s0, s0 + n); n is 0 where it is not one of the call's rows or has more than `most`.  Entries that are not in
// order can give two sequences the same rows, each range in order by itself: they are the earlier sequence's (tree_taken).
__device__ inline int tree_range(const int32_t *row_start, int n_rows, int most, int b, int &s0) {
    s0 = row_start[b];
    const int e0 = row_start[b + 1];
    return s0 >= 0 && e0 <= n_rows && e0 > s0 && e0 - s0 <= most ? e0 - s0 : 0;
}
// Whether an earlier sequence's range has a row of [s0, s0 + n): thread i of `threads` (whole waves) asks for sequences i, i + threads ..;
// true where one of the wave's has.  (The attentions share the question among a workgroup's threads and take the answer with their
// stores: 512 trees of 4 rows 43.2 us, without the question 42.1, asked by every wave in front 48.1; 200 trees of 48 rows 168.0
// and 166.4.)
__device__ inline bool tree_taken(const int32_t *row_start, int n_rows, int most, int b, int s0, int n, int i, int threads) {
    bool taken = false;
    for (int x = i; x < b; x += threads) {
        int s;
        const int m = tree_range(row_start, n_rows, most, x, s);
        taken |= (m > 0) & (s < s0 + n) & (s + m > s0);
    }
    return __any(taken);
}
// Sequence b's rows, of which nobody else has one; asked by a whole wave
__device__ inline int tree_rows(const int32_t *row_start, int n_rows, int most, int b, int &s0) {
    const int n = tree_range(row_start, n_rows, most, b, s0);
    return tree_taken(row_start, n_rows, most, b, s0, n, threadIdx.x & 63, 64) ? 0 : n;
}
__device__ inline RowSpan tree_span(int n, int L) {
    RowSpan s = {};
    s.hi = L;
    s.m1 = n;
    return s;
}
// the bounds of any rows of a tree: they all walk the same
__device__ inline RowBounds tree_bounds(int n, int L) { return {0, 0, L, L, 0, 0, 0, n}; }
// the rows of units 2 i and 2 i + 1 that a row with this word of bits sees, of a tree of n
__device__ inline unsigned tree_bits(unsigned word, int i, int n) {
    const int left = n - 32 * i;
    return left >= 32 ? word : word & ((1u << max(left, 0)) - 1u);
}
// whether a row, with these words of bits, sees any key; asked only where a sum is 0: of no key, which makes zeros, or of scores that are all
// -inf, which makes NaN
__device__ inline bool tree_sees(const uint32_t *bits, int n, int L) {
    bool any = L > 0;
    for (int i = 0; i < kTreeWords; ++i) any = any || tree_bits(bits[i], i, n) != 0;
    return any;
}

// a score, or -inf where bit `bit` of `seen` is not set
__device__ inline float seen_or_not(unsigned seen, int bit, float s) {
    const unsigned m = (unsigned)((int)(seen << (31 - bit)) >> 31);
    return __uint_as_float((__float_as_uint(s) & m) | (0xff800000u & ~m));
}
// the larger magnitudes of two pairs of bf16 values (as bits; of `top` magnitudes already)
__device__ inline unsigned top2(unsigned top, unsigned x) {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, x & 0x7fff7fffu)));
}
// of two bf16 values: bits where one is not finite; and zeros in the places of those
__device__ inline unsigned nonfinite2(unsigned x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ inline unsigned nonfinite8(bf16x8 v) {        // the same as bits 0 .. 7 of eight values
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned x = nonfinite2(w[i]);
        m |= (((x >> 15) & 1u) | ((x >> 30) & 2u)) << (2 * i);
    }
    return m;
}
__device__ inline bf16x8 finite_only(bf16x8 v) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
        if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
    }
    return __builtin_bit_cast(bf16x8, w);
}

}  // namespace
