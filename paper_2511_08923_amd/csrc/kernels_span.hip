// Hybrid-mask attention over a span of the paged cache: a sliding window and a few first tokens (sinks), or all of it, from
// exact pages or 4-bit pages.
//
// The mask.  A row at position p sees the cache below its own bound (causal row r: L + r + 1; a row of mask block j: L + cond0
// + j) and, a mask row, its own block.  With a window w and t sinks a key at position x is left out where x <= p - w, unless
// x < t.  For one row the visible keys are thus two ranges of the cache, [0, sk) and [lo, hi), and two of the mask rows.
//
// The walk.  A workgroup takes a tile of 16 query rows of a kv head (the rows of all its query heads, head-major) and walks only the
// units of 16 keys (cache pages, then mask tiles) that any of its rows sees; any two units make an iteration of 32 keys.  Pages
// between the sinks and the window are never read, not even their table entries.  The waves take
// turns with the iterations, each with its own softmax state, straight from memory into registers (no LDS, no barrier in the loop),
// and are folded through LDS at the end.  Where the tiles do not fill the chip the walk is cut into key splits, evenly by its
// real length, and the partial results are joined by a second kernel.  Bound by the bytes where few rows read many keys (32
// sequences of up to 8192 4-bit keys, one token each: 49 us, 4.4 TB/s), else by what a wave waits for (8 waves to a unit).
//
// The softmax.  Scores are formed transposed, S^T[key][q], so that a lane holds one query row's scores of its keys and they are,
// without moving, the B operand of O^T[d][q] += V^T[d][key] P^T[key][q].  Numerators are taken against a power of two that is
// moved only when the scores outgrow it by 2^16 (and from -inf by a row's first key): every rescale is exact, and no common
// path reduces a maximum across lanes.  (A reference may lag behind the waves' and splits' common maximum by the 2^16, and
// what is folded with a factor below 2^-126 is lost: weights below 2^-110 of a row's largest.)  bf16: numerators are rounded to
// bf16 for the matrix product (by at most 2^-8 of each, as in tidar_hybrid_attention: fp32 operands would take the products to a tenth
// of the rate), and the denominator sums the rounded values in fp32.  With normal inputs outputs come 2.3e-3 off the definition in the
// norm, 1.7e-3 of it their own rounding.
//
// What a masked place holds never shows: scores are replaced by -inf, and infinities and NaN of V, which a weight of zero would
// turn into NaN, are taken out of the product in units that are not wholly visible, and put back for the rows that see them.
#include <algorithm>
#include <type_traits>

#include "span_device.h"

namespace {

// T: bf16 (head_dim 128) or float; KV4: 4-bit pages; HT: head_dim tiles of 16; W: waves.
template <class T, bool KV4, int HT, int W>
__global__ __launch_bounds__(64 * W, 2) void span_attn_kernel(SpanArgs a) {
    constexpr bool BF = sizeof(T) == 2;
    constexpr int HD = 16 * HT;                          // head_dim, padded to the tiles
    constexpr int Q4 = HD / 4;                           // fp32: head-dim values of a lane's quarter
    constexpr bool QUADS = !BF || KV4;                   // a lane's eight keys: two quads, or a run of eight
    __shared__ float red[W][16][HD + 4];
    __shared__ float m_lds[W][16], l_lds[W][16];
    const SpanCall &c = a.c;
    const RowDesc &d = c.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 15, kg = lane >> 4;
    const int n_kv = KV4 ? c.kv4.n_kv : c.kv.n_kv, hd = BF ? HD : (KV4 ? c.kv4.hd : c.kv.hd);
    const int pps = KV4 ? c.kv4.pages_per_seq : c.kv.pages_per_seq, n_pages = KV4 ? c.kv4.n_pages : c.kv.n_pages;
    // workgroup i of a launch runs on XCD i % 8: where the heads divide evenly over the eight, those of a head share one's L2
    const bool xcds = c.B * n_kv % 8 == 0;
    const int i_wg = xcds ? blockIdx.x >> 3 : blockIdx.x, tile = i_wg % a.tiles, split = blockIdx.y;
    const int grp = xcds ? (i_wg / a.tiles) * 8 + (blockIdx.x & 7) : i_wg / a.tiles;
    const int b = grp / n_kv, g = grp - b * n_kv;
    const int F = a.group * d.R;
    const int L_raw = c.prefix_len[d.seq_base + b];
    const bool fits = L_raw >= 0 && (long long)L_raw + d.nc <= (long long)pps * 16;
    const int L = fits ? L_raw : 0;
    const int f = tile * 16 + lq;
    const bool row = f < F;
    const int hq = row ? f / d.R : 0, r = row ? f - hq * d.R : 0;
    RowSpan rs = row_span(d, r, L, c.window, c.sinks);
    const RowBounds rb = wave_bounds<16>(bounds_of(rs, row));
    const Walk wk = walk_of(rb, c.window);
    if (!row) rs.hi = rs.lo = rs.sk = rs.m0 = rs.ms = rs.ml = rs.m1 = 0;
    const int n_it = fits ? wk.n1 + wk.n2 : 0, per = (n_it + a.splits - 1) / a.splits;
    const int it0 = min(n_it, split * per), it1 = min(n_it, it0 + per);
    const int32_t *pt = (KV4 ? c.kv4.page_table : c.kv.page_table) + (size_t)(d.seq_base + b) * pps;
    const int n_mt = (d.nm + 15) >> 4;
    bool bad = !fits;                                    // a page id outside the pool: the rows come out as NaN

    // ---- Q: B operand, lane = (row, quarter).  bf16 step s of 32: head-dim values 32 kg + 8 s .. (4-bit pages: a lane's
    // quarter is one block) or 32 s + 8 kg .. ; fp32 step s of 4: value Q4 kg + s
    const T *qp = (const T *)c.q + (((size_t)b * d.R + r) * c.n_q + (g * a.group + hq)) * hd;
    bf16x8 qb[4];
    float qf[BF ? 1 : Q4];
    if constexpr (BF) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            qb[s] = (bf16x8){0, 0, 0, 0, 0, 0, 0, 0};
            if (row) qb[s] = *(const bf16x8 *)(qp + (KV4 ? 32 * kg + 8 * s : 32 * s + 8 * kg));
        }
    } else {
#pragma unroll
        for (int s = 0; s < Q4; ++s) qf[s] = row && Q4 * kg + s < hd ? qp[Q4 * kg + s] : 0.f;
    }
    // of a score in the softmax.  fp32: the scores are scaled before it, so that their distances from the reference are exact at any
    // size (s * scale - m in one is off by 2^7 from 2^31 on, and a row lost its largest numerator or had an infinite one; with the
    // factor in Q its values are waited for before the first tile is asked for: one token 21.4 -> 22.8 us)
    const float to_log2 = kLog2e / sqrtf((float)hd), scale = BF ? to_log2 : 1.f;
    f32x4 acc[HT];
#pragma unroll
    for (int t = 0; t < HT; ++t) acc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    // Page ids of this wave's next 32 iterations, a lane each (0 for a unit that is not there): lane 2 i + t holds unit t's of its
    // i-th iteration from `first` on.  (One scalar load per iteration had to be waited for in each, together with all of LDS.)
    auto load_pages = [&](int first) {
        const int w = 2 * (first + W * (lane >> 1)) + (lane & 1), u = wk.cache_unit(w);
        int page = first + W * (lane >> 1) < it1 && u >= 0 ? pt[u] : 0;
        if ((unsigned)page >= (unsigned)n_pages) {
            bad = true;
            page = 0;
        }
        return page;
    };
    int pages = 0, pages_at = 0;
    auto page_of = [&](int n, int t) { return __builtin_amdgcn_readlane(pages, 2 * (n - pages_at) / W + t); };      // iteration n, unit t
    auto pages_for = [&](int n) {                        // before iteration n's pages are asked for (n in steps of W)
        if (n - pages_at >= 32 * W) {
            pages = load_pages(n);
            pages_at = n;
        }
    };
    pages_at = it0 + wave;
    pages = load_pages(pages_at);

    // softmax of one iteration's scores (two tiles of 16 keys; key of register e of tile t: bit key_bit(t, e))
    auto key_bit = [&](int t, int e) { return QUADS ? 16 * t + 4 * kg + e : 8 * kg + 4 * t + e; };
    auto softmax = [&](bool whole, f32x4 (&s)[2], unsigned vis, float (&p)[8]) __attribute__((always_inline)) {
        float mx = -INFINITY;
        if (!whole)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][e] = ((vis >> key_bit(t, e)) & 1u) ? s[t][e] : -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
        if (__any(!(mx * scale <= m_run + kLag))) {      // rare: a row's first keys, or scores that outgrow the reference
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            if (!(mx * scale <= m_run + kLag)) {
                const float m_new = fmaxf(m_run, ceilf(mx * scale));
                const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
                l_run *= alpha;
#pragma unroll
                for (int t = 0; t < HT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][e] *= alpha;
                m_run = m_new;
            }
        }
        const float m_safe = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) p[4 * t + e] = __builtin_amdgcn_exp2f(fmaf(s[t][e], scale, -m_safe));
    };

    // The one-token step: the new row's K/V are not in the cache yet.  The wave whose iteration holds position L takes them from
    // where they are instead of its slot (which nobody else sees), and stores them.
    const int new_unit = !KV4 && c.k_one ? L >> 4 : -2;
    const size_t new_row = ((size_t)b * n_kv + g) * hd;
    auto store_new = [&]() {
        const int page = pt[L >> 4];
        if ((unsigned)page >= (unsigned)n_pages) return;
        const size_t at = ((size_t)page * n_kv + g) * 16 * hd;
        T *kd = (T *)const_cast<void *>(c.kv.k_pages) + at + (L & 15) * hd, *vd = (T *)const_cast<void *>(c.kv.v_pages) + at + (L & 15);
#pragma unroll 1
        for (int e = lane; e < hd; e += 64) {
            kd[e] = ((const T *)c.k_one)[new_row + e];
            vd[(size_t)e * 16] = ((const T *)c.v_one)[new_row + e];
        }
    };

    if constexpr (BF) {
        // ---- bf16: 16x16x32 MFMAs
        auto body = [&](bool whole, const bf16x8 (&kf)[2][4], bf16x8 (&vf)[HT], unsigned vis) __attribute__((always_inline)) {
            f32x4 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][j], qb[j], s[t], 0, 0, 0);
            }
            float p[8];
            softmax(whole, s, vis, p);
            const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
            bf16x8 pf;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const bf16x2 pk = {(bf16_t)p[e], (bf16_t)p[e + 1]};
                l_run = __builtin_amdgcn_fdot2_f32_bf16(pk, ones, l_run, false);
                pf[e] = pk[0];
                pf[e + 1] = pk[1];
            }
            if (!whole) {
                unsigned top = 0;
#pragma unroll
                for (int t = 0; t < HT; ++t) {
                    const u32x4 w = __builtin_bit_cast(u32x4, vf[t]);
                    top = top2(top2(top2(top2(top, w[0]), w[1]), w[2]), w[3]);
                }
                if (__builtin_expect(__any(nonfinite2(top) != 0), 0)) {
                    // taken out of the fragments, and added for the rows that see them, key by key through the wave's share of
                    // LDS (rare, and written to need few registers; what lies in slots that no row sees costs the first step only)
                    unsigned short *v = reinterpret_cast<unsigned short *>(&red[wave][0][0]);
                    unsigned mine = 0, keys = 0;
#pragma unroll
                    for (int t = 0; t < HT; ++t) mine |= nonfinite8(vf[t]);
#pragma unroll
                    for (int o = 1; o < 16; o <<= 1) mine |= __shfl_xor(mine, o);
#pragma unroll
                    for (int q8 = 0; q8 < 4; ++q8) keys |= __builtin_amdgcn_readlane(mine, 16 * q8) << (8 * q8);
#pragma unroll
                    for (int t = 0; t < HT; ++t) *(bf16x8 *)(v + (16 * t + lq) * 32 + 8 * kg) = vf[t];
#pragma unroll 1
                    for (int i = 0; i < 32; ++i) {       // slot i % 8 of the lanes of quarter i / 8
                        const int q8 = i >> 3, e = i & 7;
                        const bool seen = (vis >> (QUADS ? 16 * (e >> 2) + 4 * q8 + (e & 3) : i)) & 1u;
                        if (!((keys >> i) & 1u) || !__any(seen)) continue;
#pragma unroll
                        for (int t = 0; t < HT; ++t)
#pragma unroll
                            for (int r4 = 0; r4 < 4; ++r4) {
                                const float x = __uint_as_float((unsigned)v[(16 * t + 4 * kg + r4) * 32 + i] << 16);
                                acc[t][r4] += seen && !(fabsf(x) < INFINITY) ? x : 0.f;
                            }
                    }
#pragma unroll
                    for (int t = 0; t < HT; ++t) vf[t] = finite_only(vf[t]);
                }
            }
#pragma unroll
            for (int t = 0; t < HT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[t], pf, acc[t], 0, 0, 0);
        };
        // exact tiles, K [16][128] and V [128][16]: of a page or of the mask rows
        auto load_exact = [&](const bf16_t *k0, const bf16_t *k1, const bf16_t *v0, const bf16_t *v1, bf16x8 (&kf)[2][4],
                              bf16x8 (&vf)[HT]) __attribute__((always_inline)) {
            if constexpr (KV4) {                         // two quads, blocks of 32 head-dim values to a quarter
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    kf[0][j] = *(const bf16x8 *)(k0 + lq * HD + 32 * kg + 8 * j);
                    kf[1][j] = *(const bf16x8 *)(k1 + lq * HD + 32 * kg + 8 * j);
                }
#pragma unroll
                for (int t = 0; t < HT; ++t) {
                    const u32x2 x = *(const u32x2 *)(v0 + (HT * lq + t) * 16 + 4 * kg);
                    const u32x2 y = *(const u32x2 *)(v1 + (HT * lq + t) * 16 + 4 * kg);
                    vf[t] = __builtin_bit_cast(bf16x8, (u32x4){x[0], x[1], y[0], y[1]});
                }
            } else {                                     // eight keys in a row: tile t, row 4a + e is key 8a + 4t + e of the 32
                const bf16_t *kb = (lq >> 3) ? k1 : k0, *vb = (kg >> 1) ? v1 : v0;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        kf[t][j] = *(const bf16x8 *)(kb + (8 * ((lq >> 2) & 1) + 4 * t + (lq & 3)) * HD + 32 * j + 8 * kg);
#pragma unroll
                for (int t = 0; t < HT; ++t) vf[t] = *(const bf16x8 *)(vb + (16 * t + lq) * 16 + 8 * (kg & 1));
            }
        };
        auto mask_tile = [&](int u) { return ((((size_t)b * n_kv + g) * n_mt + max(u, 0)) * 16) * HD; };
        // an iteration's codes (4-bit pages) or tiles (exact pages), asked for AHEAD iterations before they are needed
        constexpr int AHEAD = KV4 ? 2 : 1;
        struct Raw4 {
            u32x4 k[2], v[2];
            unsigned ks[2], vs[2];
        };
        struct RawExact {
            bf16x8 k[2][4], v[HT];
        };
        typedef std::conditional_t<KV4, Raw4, RawExact> Raw;
        auto fetch = [&](int n) __attribute__((always_inline)) {
            Raw x;
            pages_for(n);
            if constexpr (KV4) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const unsigned char *p = c.kv4.pages + kv4_offset(c.kv4, page_of(n, t), g);
                    x.k[t] = *(const u32x4 *)(p + kg * 256 + lq * 16);
                    x.v[t] = *(const u32x4 *)(p + kv4_v_codes(4) + kg * 256 + lq * 16);
                    x.ks[t] = p[kv4_k_scales(4) + kg * 16 + lq];
                    x.vs[t] = *(const unsigned *)(p + kv4_v_scales(4) + (lq >> 2) * 16 + 4 * kg);
                }
            } else {
                const size_t o0 = ((size_t)page_of(n, 0) * n_kv + g) * 16 * HD, o1 = ((size_t)page_of(n, 1) * n_kv + g) * 16 * HD;
                load_exact((const bf16_t *)c.kv.k_pages + o0, (const bf16_t *)c.kv.k_pages + o1,
                           (const bf16_t *)c.kv.v_pages + o0, (const bf16_t *)c.kv.v_pages + o1, x.k, x.v);
            }
            return x;
        };
        auto block = [&](int n, Raw &x) __attribute__((always_inline)) {
            const int u0 = wk.cache_unit(2 * n), u1 = wk.cache_unit(2 * n + 1);
            const bool whole = all_see(rb, u0) && all_see(rb, u1);
            const unsigned vis = whole ? ~0u : cache_bits(rs, u0) | (cache_bits(rs, u1) << 16);
            if constexpr (KV4) {
                bf16x8 kf[2][4], vf[HT];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const float s = kv4_scale(x.ks[t]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const bf16x2 x0 = kv4_pair_bf16<0>(x.k[t][j], s), x1 = kv4_pair_bf16<1>(x.k[t][j], s),
                                     x2 = kv4_pair_bf16<2>(x.k[t][j], s), x3 = kv4_pair_bf16<3>(x.k[t][j], s);
                        kf[t][j] = (bf16x8){x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {        // token 4 kg + e: eight head-dim values of lane lq
                        const float sv = kv4_scale((x.vs[t] >> (8 * e)) & 255u);
                        const bf16x2 x0 = kv4_pair_bf16<0>(x.v[t][e], sv), x1 = kv4_pair_bf16<1>(x.v[t][e], sv),
                                     x2 = kv4_pair_bf16<2>(x.v[t][e], sv), x3 = kv4_pair_bf16<3>(x.v[t][e], sv);
                        const int at = 4 * t + e;
                        vf[0][at] = x0[0]; vf[1][at] = x0[1]; vf[2][at] = x1[0]; vf[3][at] = x1[1];
                        vf[4][at] = x2[0]; vf[5][at] = x2[1]; vf[6][at] = x3[0]; vf[7][at] = x3[1];
                    }
                }
                body(whole, kf, vf, vis);
            } else {
                if (u0 == new_unit || u1 == new_unit) {
                    const int key = (u1 == new_unit ? 16 : 0) + (L & 15);        // of the 32: tile t, row 4a + e is key 8a + 4t + e
                    const bf16_t *kn = (const bf16_t *)c.k_one + new_row, *vn = (const bf16_t *)c.v_one + new_row;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        bf16x8 y;                        // (the row need not be aligned)
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = kn[32 * j + 8 * kg + e];
#pragma unroll
                        for (int t = 0; t < 2; ++t) x.k[t][j] = 8 * (lq >> 2) + 4 * t + (lq & 3) == key ? y : x.k[t][j];
                    }
#pragma unroll
                    for (int t = 0; t < HT; ++t) {
                        const bf16_t y = vn[16 * t + lq];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x.v[t][e] = 8 * kg + e == key ? y : x.v[t][e];
                    }
                    store_new();
                }
                body(whole, x.k, x.v, vis);
            }
        };
        const int end1 = min(it1, wk.n1);
        int n = it0 + wave;
        if (n < end1) {
            Raw x0 = fetch(n), x1;
            if (AHEAD == 2 && n + W < end1) x1 = fetch(n + W);
            for (; n < end1; n += W) {
                Raw now = x0;
                if constexpr (AHEAD == 2) x0 = x1;
                if (n + W * AHEAD < end1) (AHEAD == 2 ? x1 : x0) = fetch(n + W * AHEAD);
                block(n, now);
            }
        }
        for (; n < it1; n += W) {
            const int w = 2 * (n - wk.n1), u0 = wk.mask_unit(w), u1 = wk.mask_unit(w + 1);
            bf16x8 kf[2][4], vf[HT];
            load_exact((const bf16_t *)c.k_scr + mask_tile(u0), (const bf16_t *)c.k_scr + mask_tile(u1),
                       (const bf16_t *)c.v_scr + mask_tile(u0), (const bf16_t *)c.v_scr + mask_tile(u1), kf, vf);
            body(false, kf, vf, mask_bits(rs, u0) | (mask_bits(rs, u1) << 16));
        }
    } else {
        // ---- fp32: 16x16x4 MFMAs.  A lane's head-dim values of O^T tile t are HT i + t.
        const bool vec = hd % 4 == 0;
        typedef f32x4 any_f32x4 __attribute__((aligned(4)));     // (a new row need not be aligned)
        auto load_k = [&](const float *kp, float (&k)[Q4]) __attribute__((always_inline)) {      // token lq: hd values from kp on
            const float *src = kp + Q4 * kg;
            const int n = hd - Q4 * kg;
#pragma unroll
            for (int j = 0; j < Q4; j += 4) {
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
                if (vec) {
                    if (j < n) x = *(const any_f32x4 *)(src + j);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = j + e < n ? src[j + e] : 0.f;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) k[j + e] = x[e];
            }
        };
        auto load_v = [&](const float *vp, f32x4 (&v)[HT]) __attribute__((always_inline)) {      // tokens 4 kg .. of [hd][16]
#pragma unroll
            for (int t = 0; t < HT; ++t) {
                v[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
                if (HT * lq + t < hd) v[t] = *(const f32x4 *)(vp + (HT * lq + t) * 16 + 4 * kg);
            }
        };
        auto load_k4 = [&](const unsigned char *blk, float (&k)[Q4]) __attribute__((always_inline)) {
            const int nb = kv4_blocks(hd);
#pragma unroll
            for (int j = 0; j < Q4; j += 4) {
                const int e0 = Q4 * kg + j, bl = e0 >> 5;
                kv4_f32x2 x = {0.f, 0.f}, y = {0.f, 0.f};
                if (e0 < hd) {
                    const unsigned w = *(const unsigned short *)(blk + bl * 256 + lq * 16 + ((e0 & 31) >> 1));
                    const float s = kv4_scale(blk[kv4_k_scales(nb) + bl * 16 + lq]);
                    x = kv4_pair_f32<0>(w, s);
                    y = kv4_pair_f32<1>(w, s);
                }
                k[j] = x[0]; k[j + 1] = x[1]; k[j + 2] = y[0]; k[j + 3] = y[1];
            }
        };
        auto load_v4 = [&](const unsigned char *blk, f32x4 (&v)[HT]) __attribute__((always_inline)) {
            const int nb = kv4_blocks(hd), e0 = HT * lq;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                unsigned w = 0;
                float s = 0.f;
                if (e0 < hd) {
                    const unsigned char *src = blk + kv4_v_codes(nb) + (kg * 4 * nb + (e0 >> 3)) * 16 + e * 4 + ((e0 & 7) >> 1);
                    if constexpr (HT == 8) w = *(const unsigned *)src;
                    else if constexpr (HT == 4) w = *(const unsigned short *)src;
                    else w = *src;
                    s = kv4_scale(blk[kv4_v_scales(nb) + (e0 >> 5) * 16 + 4 * kg + e]);
                }
                const kv4_f32x2 x0 = kv4_pair_f32<0>(w, s), x1 = kv4_pair_f32<1>(w, s), x2 = kv4_pair_f32<2>(w, s),
                                x3 = kv4_pair_f32<3>(w, s);
                const float x[8] = {x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
#pragma unroll
                for (int t = 0; t < HT; ++t) v[t][e] = x[t];
            }
        };
        // the unit at hand: its scores, and what its weights add to the output
        auto scores = [&](const float (&k)[Q4]) __attribute__((always_inline)) {
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < Q4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j], qf[j], s, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] *= to_log2;
            return s;
        };
        auto weigh = [&](f32x4 (&v)[HT], const float *p, unsigned vis16) __attribute__((always_inline)) {
            unsigned top = 0;
#pragma unroll
            for (int t = 0; t < HT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(v[t][e]) & 0x7fffffffu);
            if (__builtin_expect(__any(top >= 0x7f800000u), 0)) {        // as above: set aside, and added key by key
                float (*vl)[HD + 4] = red[wave];
                unsigned mine = 0, keys = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t = 0; t < HT; ++t) {
                        vl[4 * kg + e][HT * lq + t] = v[t][e];
                        if (!(fabsf(v[t][e]) < INFINITY)) {
                            mine |= 1u << e;
                            v[t][e] = 0.f;
                        }
                    }
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) mine |= __shfl_xor(mine, o);
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) keys |= __builtin_amdgcn_readlane(mine, 16 * q4) << (4 * q4);
#pragma unroll 1
                for (int key = 0; key < 16; ++key) {
                    const bool seen = (vis16 >> key) & 1u;
                    if (!((keys >> key) & 1u) || !__any(seen)) continue;
#pragma unroll
                    for (int t = 0; t < HT; ++t)
#pragma unroll
                        for (int r4 = 0; r4 < 4; ++r4) {
                            const float x = vl[key][HT * (4 * kg + r4) + t];
                            acc[t][r4] += seen && !(fabsf(x) < INFINITY) ? x : 0.f;
                        }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < HT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[t][e], p[e], acc[t], 0, 0, 0);
        };
        for (int n = it0 + wave; n < it1; n += W) {
            const bool cache = n < wk.n1;
            const int w = cache ? 2 * n : 2 * (n - wk.n1);
            const int u[2] = {cache ? wk.cache_unit(w) : wk.mask_unit(w), cache ? wk.cache_unit(w + 1) : wk.mask_unit(w + 1)};
            pages_for(n);
            size_t at[2];
            f32x4 s[2], v[HT];
            float k[Q4], p[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const size_t piece = cache ? (size_t)page_of(n, t) * n_kv + g : ((size_t)b * n_kv + g) * n_mt + max(u[t], 0);
                at[t] = piece * 16 * hd;
                if (KV4 && cache) load_k4(c.kv4.pages + piece * kv4_head_bytes(hd), k);
                else load_k(!KV4 && cache && u[t] == new_unit && lq == (L & 15) ? (const float *)c.k_one + new_row
                                : (const float *)(cache ? c.kv.k_pages : c.k_scr) + at[t] + lq * hd, k);
                if (KV4 && cache) at[t] = piece * kv4_head_bytes(hd);
                s[t] = scores(k);
            }
            const unsigned vis = cache ? cache_bits(rs, u[0]) | (cache_bits(rs, u[1]) << 16)
                                       : mask_bits(rs, u[0]) | (mask_bits(rs, u[1]) << 16);
            softmax(false, s, vis, p);
#pragma unroll
            for (int e = 0; e < 8; ++e) l_run += p[e];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (KV4 && cache) load_v4(c.kv4.pages + at[t], v);
                else load_v((const float *)(cache ? c.kv.v_pages : c.v_scr) + at[t], v);
                if (!KV4 && cache && u[t] == new_unit) {
#pragma unroll
                    for (int i = 0; i < HT; ++i) {
                        const float y = HT * lq + i < hd ? ((const float *)c.v_one)[new_row + HT * lq + i] : 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[i][e] = 4 * kg + e == (L & 15) ? y : v[i][e];
                    }
                    store_new();
                }
                weigh(v, p + 4 * t, vis >> (16 * t));
            }
        }
    }

    // ---- fold the waves
    float l = l_run;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (__any(bad)) {
        l = __builtin_nanf("");
        if (m_run == -INFINITY) m_run = 0.f;
    }
    if (kg == 0) {
        m_lds[wave][lq] = m_run;
        l_lds[wave][lq] = l;
    }
#pragma unroll
    for (int t = 0; t < HT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 4 * kg + e;
            red[wave][lq][(BF && !KV4) ? 16 * t + i : HT * i + t] = acc[t][e];
        }
    __syncthreads();
    constexpr int LANES = 4 * W, PER = HD / LANES;       // a row's threads, and the values of each
    const int oq = tid / LANES, od = (tid % LANES) * PER, of = tile * 16 + oq;
    if (of >= F) return;
    float m = m_lds[0][oq];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, m_lds[w][oq]);
    float sum = 0.f, o[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const float mw = m_lds[w][oq];                   // -inf: saw nothing, sums of 0, or NaN scores alone, sums of NaN
        const float wgt = mw == m ? 1.f : __builtin_amdgcn_exp2f(mw - m);
        sum += wgt * l_lds[w][oq];
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] += wgt * red[w][oq][od + e];
    }
    const int ohq = of / d.R, orow = b * d.R + of - ohq * d.R;
    const size_t orh = (size_t)orow * c.n_q + g * a.group + ohq;
    if (a.splits > 1) {
        const size_t at = orh * a.splits + split;
        for (int e = 0; e < PER; ++e)
            if (od + e < hd) a.opart[at * hd + od + e] = o[e];
        if (tid % LANES == 0) {
            a.mpart[at] = m;
            a.lpart[at] = sum;
        }
        return;
    }
    T *out = (T *)c.out + orh * hd + od;
    if constexpr (BF) {
        typedef __attribute__((ext_vector_type(PER))) __bf16 bf16_per;
        bf16_per v;
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = (bf16_t)(o[e] / sum);
        *(bf16_per *)out = v;
    } else {
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (od + e < hd) out[e] = o[e] / sum;
    }
}

// out[row][head] = sum_s w_s O_s / sum_s w_s l_s, w_s = 2^(m_s - max m).  A wave per (row, head), lane = (8 head-dim values, one of 4
// split lanes); a lane asks for all of J splits at once (one after another, 31 splits cost 31 trips to memory: 16 us).
template <class T, int J>
__global__ __launch_bounds__(64) void span_combine_kernel(const float *__restrict__ opart, const float *__restrict__ mpart,
                                                          const float *__restrict__ lpart, int splits, int hd,
                                                          T *__restrict__ out) {
    const size_t at = (size_t)blockIdx.x * splits;
    const int lane = threadIdx.x, d0 = 8 * (lane & 15), sl = lane >> 4;
    const bool whole = d0 + 8 <= hd && hd % 4 == 0;
    float m_all = lane < splits ? mpart[at + lane] : -INFINITY;          // at most 64 splits
    float num[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, den = 0.f;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m_all = fmaxf(m_all, __shfl_xor(m_all, o));
    for (int s0 = sl; s0 < splits; s0 += 4 * J) {
        float m[J], l[J], x[J][8];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int s = min(s0 + 4 * j, splits - 1);
            m[j] = mpart[at + s];
            l[j] = lpart[at + s];
            const float *src = opart + (at + s) * hd + d0;
            if (whole) {
                const f32x4 a = *(const f32x4 *)src, b = *(const f32x4 *)(src + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[j][e] = a[e];
                    x[j][4 + e] = b[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = d0 + e < hd ? src[e] : 0.f;
            }
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (s0 + 4 * j >= splits || l[j] == 0.f) continue;           // (a split of NaN scores alone has a maximum of -inf too)
            const float w = m[j] == m_all ? 1.f : __builtin_amdgcn_exp2f(m[j] - m_all);
            den += w * l[j];
#pragma unroll
            for (int e = 0; e < 8; ++e) num[e] += w * x[j][e];
        }
    }
    den += __shfl_xor(den, 16);
    den += __shfl_xor(den, 32);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        num[e] += __shfl_xor(num[e], 16);
        num[e] += __shfl_xor(num[e], 32);
    }
    if (sl != 0) return;
    T *dst = out + (size_t)blockIdx.x * hd + d0;
    if constexpr (sizeof(T) == 2) {
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (bf16_t)(num[e] / den);
        *(bf16x8 *)dst = o;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d0 + e < hd) dst[e] = num[e] / den;
    }
}

}  // namespace

// Waves of a few-row workgroup.  bf16: eight, so that half as many splits have to be joined (32 sequences of 8192 keys in 4 bits:
// 50.6 us unsplit, with four waves 59.7 and 52 at best); fp32: four, the registers of head_dim 128 do not fit twice
// (from exact pages not even once: 56 of them are spilled).
static int span_waves(int dtype) { return dtype == TIDAR_BF16 ? 8 : 4; }
static int most_splits(int dtype, long long wgs) {
    const int slots = 2048 / span_waves(dtype);
    return wgs >= slots ? 1 : (int)std::min<long long>(64, slots / wgs);
}
static size_t few_part_floats(int dtype, long long wgs, int hd) {
    const int s = most_splits(dtype, wgs);
    return s == 1 ? 0 : (size_t)(wgs * 16 * s) * (hd + 2);
}

// Keys that a workgroup walks whose rows lie within `rows` positions, from the caller's bound on the prefix.
long long span_keys(const RowDesc &d, int rows, int window, int sinks, int max_prefix) {
    const long long all = (long long)max_prefix + d.R;
    return window > 0 ? std::min(all, (long long)window + sinks + rows) : all;
}

// 16 rows to a workgroup or 128: a wave that takes 16 rows starts and ends sooner, one that takes 32 reads its keys for twice as
// many and shares them with three others.  What decides is the work in 16 rows by 32 keys, all sequences and heads together, from
// exact pages in whole rounds of 256 workgroups, and that the rows fill enough of a workgroup's 128.  us with 16 and with 128 rows:
//   4-bit pages   8 sequences of 1000 keys and 168 rows of a head (23 k): 32.7, 34.0;  8 of 8000 and 120 (32 k): 31.6, 34.5;
//                 32 of 1000 and 252 (34 k): 41.9, 36.2;  8 of 1000 and 288 (39 k): 50.6, 36.6;  8 of 8000 and 48 (48 k): 44.3, 50.0
//   exact pages   one round with a window of 1000 (8.4 k): 19.1, 25.9;  2000 (16 k): 27.6, 27.6;  3000 (24 k): 36.7, 29.6;
//                 two rounds of 1000, 80 rows (16 k): 33.0, 26.8;  five, 288 rows (44 k): 73.1, 36.2
static bool many_rows(int dtype, bool four, int F, long long wgs, long long keys) {
    if (dtype != TIDAR_BF16) return false;
    const long long its = (keys + 31) / 32;
    if (four) return F > 64 && wgs * its > 33000;
    return F > 32 && (wgs > 256 ? (wgs + 255) / 256 * 256 : wgs) * its > 16200;
}

// The partial results' memory does not depend on that choice, nor on the keys: a caller's bound on the prefixes may differ from the
// one that it asked the workspace's size for.
SpanPlan plan_span(int dtype, bool four, int B, int n_q, int n_kv, int hd, const RowDesc &d, int window, int sinks, int max_prefix) {
    SpanPlan p = {};
    const int F = n_q / n_kv * d.R;
    const long long keys = span_keys(d, d.R, window, sinks, max_prefix);
    const long long wgs = (long long)B * n_kv * ((F + 15) / 16);
    if (dtype == TIDAR_BF16 && F > 32) plan_span_rows(B, n_kv, n_q / n_kv, d, window, sinks, max_prefix, &p);
    p.rows = many_rows(dtype, four, F, wgs, keys);
    if (p.rows) {
        p.part_floats = std::max(p.part_floats, few_part_floats(dtype, wgs, hd));
        return p;
    }
    p.tiles = (F + 15) / 16;
    // One round of workgroups, eight waves to a compute unit.  A wave's iteration takes about 0.75 us, the join of the splits 3 and
    // 4 ns per partial result: the least sum wins.  (us at 1, 2, 4, 8, 16 splits: 32 sequences of 1000 keys in 4 bits 12.1, 19.5,
    // 25.8, 37.5, 65.6; 8 of 8192 40.3, 26.5, 19.8, 25.3, 33.9; one over an exact window of 4096 43.5, 30.0, 19.8, 13.3, 11.3.)  fp32
    // waits for each tile: 3 us (72 rows over 570 keys of head_dim 128: 43 us unsplit, 22 in five)
    const int per_it = 32 * span_waves(dtype), bound = most_splits(dtype, wgs);
    p.splits = 1;
    const double it_us = dtype == TIDAR_BF16 ? 0.75 : 3.0;
    double best = 0.0;
    for (int s = 1; s <= bound; ++s) {
        const double t = it_us * (double)((keys + per_it * s - 1) / (per_it * s)) + (s > 1 ? 3.0 + 0.004 * (double)wgs * s : 0.0);
        if (s == 1 || t < best) {
            best = t;
            p.splits = s;
        }
    }
    p.part_floats = std::max(p.part_floats, few_part_floats(dtype, wgs, hd));
    return p;
}

static SpanArgs span_args(const SpanCall &c, const SpanPlan &p) {
    SpanArgs a;
    a.c = c;
    const int n_kv = c.kv.k_pages ? c.kv.n_kv : c.kv4.n_kv, hd = c.kv.k_pages ? c.kv.hd : c.kv4.hd;
    a.group = c.n_q / n_kv;
    a.tiles = p.tiles;
    a.splits = p.splits;
    a.span_rows = p.span_rows;
    a.whole = p.whole;
    a.per = p.per;
    const size_t rows = p.rows ? (size_t)(c.B * n_kv * p.tiles - p.whole) * p.splits * 128 : (size_t)c.B * c.d.R * c.n_q * p.splits;
    a.opart = c.part;
    a.mpart = c.part + rows * hd;
    a.lpart = a.mpart + rows;
    a.pieces = (int *)(a.lpart + rows);
    return a;
}

void launch_span_attention(int dtype, const SpanCall &c, const SpanPlan &p, hipStream_t st) {
    const SpanArgs a = span_args(c, p);
    if (p.rows) {
        launch_span_rows(a, st);
        return;
    }
    const bool four = c.kv.k_pages == nullptr;
    const int n_kv = four ? c.kv4.n_kv : c.kv.n_kv, hd = four ? c.kv4.hd : c.kv.hd;
    const dim3 grid(c.B * n_kv * p.tiles, p.splits);
    auto go = [&](auto kernel) { kernel<<<grid, 64 * span_waves(dtype), 0, st>>>(a); };
    if (dtype == TIDAR_BF16) {
        if (four) go(span_attn_kernel<bf16_t, true, 8, 8>);
        else go(span_attn_kernel<bf16_t, false, 8, 8>);
    } else if (four) {
        if (hd <= 32) go(span_attn_kernel<float, true, 2, 4>);
        else if (hd <= 64) go(span_attn_kernel<float, true, 4, 4>);
        else go(span_attn_kernel<float, true, 8, 4>);
    } else {
        if (hd <= 32) go(span_attn_kernel<float, false, 2, 4>);
        else if (hd <= 64) go(span_attn_kernel<float, false, 4, 4>);
        else go(span_attn_kernel<float, false, 8, 4>);
    }
}

void launch_span_combine(int dtype, const SpanCall &c, const SpanPlan &p, hipStream_t st) {
    if (p.splits == 1) return;
    const SpanArgs a = span_args(c, p);
    if (p.rows) {
        launch_span_rows_join(a, st);
        return;
    }
    const int hd = c.kv.k_pages ? c.kv.hd : c.kv4.hd;
    const int heads = c.B * c.d.R * c.n_q;
    auto go = [&](auto kernel, auto *out) { kernel<<<heads, 64, 0, st>>>(a.opart, a.mpart, a.lpart, p.splits, hd, out); };
    if (dtype == TIDAR_BF16) {
        if (p.splits <= 8) go(span_combine_kernel<bf16_t, 2>, (bf16_t *)c.out);
        else go(span_combine_kernel<bf16_t, 8>, (bf16_t *)c.out);
    } else {
        go(span_combine_kernel<float, 4>, (float *)c.out);
    }
}
