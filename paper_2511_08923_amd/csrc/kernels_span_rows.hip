// The attention over a span for many query rows (bf16): the walk, the mask and the softmax of kernels_span.hip with tiles of 32
// query rows to a wave, four waves to a workgroup, and K and V tiles of 32 keys that the four share in LDS.
//
// Scores are v_mfma_f32_32x32x16_bf16 products S^T = K Q^T; a lane's registers 8u .. 8u + 7 are its row's scores of keys 8 lh ..
// 8 lh + 7 of unit u, and after the exponential, packed, the B operand of O^T += V^T P^T.
//
// A wave works on two blocks at a time: the score products of block n + 1 stand between the vector instructions of block n's
// softmax, and the output products of block n between the conversions (4-bit pages) or nothing (exact pages) of a tile three
// blocks further on.  An MFMA takes 32 clocks and issues in 4; what stands between two of them is free up to eight vector
// instructions, and with one block at a time a SIMD had either its matrix or its vector unit idle.
//
// Tiles are staged in a ring of four.  Exact pages come by direct loads into LDS (lds_dma.h); of 4-bit pages every thread
// converts 16 elements of K and 16 of V per tile, so a tile is converted once for 128 query rows.  K rows of 256 bytes
// have their 16-byte pieces XOR-swizzled by the row and rows 4-7 and 8-11 of a unit exchanged; V^T is [unit][key half][position]
// 16-byte pieces, where position p is head-dim value p (exact pages) or 8 (p % 16) + p / 16 (4-bit pages: a wave's stores
// are contiguous then, and a lane's results are runs of eight values).
#include <algorithm>
#include <type_traits>

#include "lds_dma.h"
#include "span_device.h"

namespace {

constexpr int HD = 128, TILE = 32 * HD, RING = 4;

template <bool KV4>
__global__ __launch_bounds__(256, 2) void span_rows_kernel(SpanArgs a) {
    constexpr int KRING = KV4 ? RING : RING + 1;         // direct loads of K are asked for an iteration earlier
    __shared__ __attribute__((aligned(16))) bf16_t k_lds[KRING][TILE];
    __shared__ __attribute__((aligned(16))) bf16_t v_lds[RING][TILE];
    __shared__ RowBounds wave_rows[4];
    __shared__ int bad_lds;
    const SpanCall &c = a.c;
    const RowDesc &d = c.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 31, lh = lane >> 5;
    const int n_kv = KV4 ? c.kv4.n_kv : c.kv.n_kv;
    const int pps = KV4 ? c.kv4.pages_per_seq : c.kv.pages_per_seq, n_pages = KV4 ? c.kv4.n_pages : c.kv.n_pages;
    // The chunks of a (sequence, kv head) group run on one XCD where the groups divide evenly over the eight
    // (workgroup i of a launch runs on XCD i % 8): its L2 then fetches the head's K and V once
    const int n_groups = c.B * n_kv, chunks = a.tiles;
    int grp, chunk;
    if (n_groups % 8 == 0) {
        const int j = blockIdx.x >> 3;
        grp = (j / chunks) * 8 + (blockIdx.x & 7);
        chunk = j % chunks;
    } else {
        grp = blockIdx.x / chunks;
        chunk = blockIdx.x % chunks;
    }
    const int split = blockIdx.y, b = grp / n_kv, g = grp - b * n_kv;
    const int F = a.group * d.R;
    const int L_raw = c.prefix_len[d.seq_base + b];
    const bool fits = L_raw >= 0 && (long long)L_raw + d.nc <= (long long)pps * 16;
    const int L = fits ? L_raw : 0;
    const int tile = chunk * 4 + wave, f = tile * 32 + lq;
    const bool here = tile * 32 < F, row = f < F;        // (here: wave-uniform)
    const int hq = row ? f / d.R : 0, r = row ? f - hq * d.R : 0;
    RowSpan rs = row_span(d, r, L, c.window, c.sinks);
    const RowBounds rb = wave_bounds<32>(bounds_of(rs, row));
    if (!row) rs = RowSpan{};
    if (lane == 0) wave_rows[wave] = rb;
    if (tid == 0) bad_lds = 0;
    __syncthreads();
    const RowBounds all = join(join(wave_rows[0], wave_rows[1]), join(wave_rows[2], wave_rows[3]));
    auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const Walk wk = walk_of({uni(all.lo0), uni(all.lo1), uni(all.hi0), uni(all.hi1), uni(all.sk0), uni(all.sk1), uni(all.m0),
                             uni(all.m1)}, c.window);
    const int n_it = fits ? wk.n1 + wk.n2 : 0, per = (n_it + a.splits - 1) / a.splits;
    const int it0 = min(n_it, split * per), n_seq = min(n_it, it0 + per) - it0;
    const __attribute__((address_space(4))) int32_t *pt = (const __attribute__((address_space(4))) int32_t *)(
        (KV4 ? c.kv4.page_table : c.kv.page_table) + (size_t)(d.seq_base + b) * pps);
    const int n_mt = (d.nm + 15) >> 4;
    bool bad = !fits;

    // ---- Q: B operand, lane = (row, half of the 16 head-dim values of a step)
    bf16x8 qf[8];
    {
        const bf16_t *qp = (const bf16_t *)c.q + (((size_t)b * d.R + r) * c.n_q + (g * a.group + hq)) * HD + 8 * lh;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            qf[ks] = (bf16x8){0, 0, 0, 0, 0, 0, 0, 0};
            if (row) qf[ks] = *(const bf16x8 *)(qp + 16 * ks);
        }
    }
    const float scale = kLog2e / sqrtf((float)HD);
    f32x16 acc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    // ---- staging: wave w moves unit w / 2 of a tile's pair, of it K rows 8 (w % 2) .. + 7 and V key half w % 2
    const int u_w = wave >> 1, half_w = wave & 1;
    const unsigned k_lds0 = lds_address(reinterpret_cast<unsigned char *>(&k_lds[0][0]));
    const unsigned v_lds0 = lds_address(reinterpret_cast<unsigned char *>(&v_lds[0][0]));
    int k_voff[2], v_voff[2];
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) {
        const int lrow = 8 * half_w + 4 * jj + (lane >> 4);
        const int key = (lrow & 3) | ((lrow & 4) << 1) | ((lrow & 8) >> 1);
        k_voff[jj] = key * (HD * 2) + (((lane & 15) ^ lrow) << 4);
        const int p = 64 * jj + lane;
        v_voff[jj] = (KV4 ? 8 * (p & 15) + (p >> 4) : p) * 32 + half_w * 16;
    }
    const size_t scr0 = ((size_t)b * n_kv + g) * n_mt * 16 * HD;
    const int4v dks = raw_desc((const bf16_t *)c.k_scr + scr0, (size_t)n_mt * 16 * HD * 2);
    const int4v dvs = raw_desc((const bf16_t *)c.v_scr + scr0, (size_t)n_mt * 16 * HD * 2);
    const size_t layer_bytes = KV4 ? 0 : (size_t)c.kv.n_pages * n_kv * 16 * HD * 2;
    const int4v dk = raw_desc(c.kv.k_pages, layer_bytes), dv = raw_desc(c.kv.v_pages, layer_bytes);
    auto k_slot = [&](int m) { return KV4 ? m & (RING - 1) : m % KRING; };
    auto dma_k = [&](int4v desc, int base, int slot) __attribute__((always_inline)) {
        const unsigned to = k_lds0 + slot * (TILE * 2) + (u_w * 16 + 8 * half_w) * 256;
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) dma16(to + 1024 * jj, k_voff[jj], desc, base);
    };
    auto dma_v = [&](int4v desc, int base, int slot) __attribute__((always_inline)) {
        const unsigned to = v_lds0 + slot * (TILE * 2) + (u_w * 2 + half_w) * 2048;
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) dma16(to + 1024 * jj, v_voff[jj], desc, base);
    };
    // The page of this wave's unit of tile m (0: it has none), asked for an iteration before it is needed.  All of this is scalar
    // selects: with branches for the kinds of units an iteration took 2.5 times as long
    const int n_cache = wk.n_s + wk.n_w, last_unit = max(0, wk.w0 + wk.n_w - 1);
    auto page_at = [&](int m) {
        const int w = 2 * (it0 + m) + u_w;
        const bool in = m < n_seq && w < n_cache;
        const int page = pt[min(w < wk.n_s ? w : wk.w0 + (w - wk.n_s), last_unit)];
        return in ? page : 0;
    };
    auto checked = [&](int page) {
        const bool in = (unsigned)page < (unsigned)n_pages;
        bad = bad || !in;
        return in ? page : 0;
    };
    // byte offset of this wave's unit of tile m among the mask rows' tiles (one that is not there: the last again, masked)
    auto mask_base = [&](int m) {
        return max(0, min(wk.um0 + 2 * (it0 + m - wk.n1) + u_w, wk.um0 + wk.n_m - 1)) * (16 * HD * 2);
    };
    auto page_base = [&](int page) { return (int)((((size_t)page * n_kv + g) * 16 * HD) * 2); };
    // 4-bit pages: a thread's 8 bytes of K (16 elements of a token) and 8 of V (8 elements of two tokens)
    struct Raw {
        u32x2 k, v;
        unsigned ks, vs;
    };
    // (the LDS rows of a wave's tokens are those that its direct loads write)
    const int k_row = 8 * half_w + (lane & 7), kt = (k_row & 3) | ((k_row & 4) << 1) | ((k_row & 8) >> 1);     // K: row and token,
    const int kb = (lane >> 3) & 3, kp = lane >> 5;                                    // block, half of the block
    const int vi = lane & 15, vt = 8 * half_w + 4 * ((lane >> 4) & 1) + 2 * (lane >> 5);       // V: group of 8, first token
    const int k_src = kb * 256 + kt * 16 + kp * 8, ks_src = kv4_k_scales(4) + kb * 16 + kt;
    const int v_src = kv4_v_codes(4) + (vt >> 2) * 256 + vi * 16 + (vt & 3) * 4, vs_src = kv4_v_scales(4) + (vi >> 2) * 16 + vt;
    auto fetch = [&](int page) __attribute__((always_inline)) {
        const unsigned char *p = c.kv4.pages + kv4_offset(c.kv4, checked(page), g);
        return Raw{*(const u32x2 *)(p + k_src), *(const u32x2 *)(p + v_src), p[ks_src], *(const unsigned short *)(p + vs_src)};
    };
    auto convert = [&](const Raw &x, int slot) __attribute__((always_inline)) {
        unsigned char *kd = reinterpret_cast<unsigned char *>(&k_lds[slot][0]) + (u_w * 16 + k_row) * 256;
        unsigned char *vd = reinterpret_cast<unsigned char *>(&v_lds[slot][0]) + ((u_w * 2 + half_w) * 128 + vi) * 16 + (vt & 7) * 2;
        const float s = kv4_scale(x.ks), s0 = kv4_scale(x.vs & 255u), s1 = kv4_scale(x.vs >> 8);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bf16x2 x0 = kv4_pair_bf16<0>(x.k[j], s), x1 = kv4_pair_bf16<1>(x.k[j], s), x2 = kv4_pair_bf16<2>(x.k[j], s),
                         x3 = kv4_pair_bf16<3>(x.k[j], s);
            *(bf16x8 *)(kd + (((4 * kb + 2 * kp + j) ^ k_row) << 4)) =
                (bf16x8){x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
        }
        const bf16x2 a0 = kv4_pair_bf16<0>(x.v[0], s0), a1 = kv4_pair_bf16<1>(x.v[0], s0), a2 = kv4_pair_bf16<2>(x.v[0], s0),
                     a3 = kv4_pair_bf16<3>(x.v[0], s0);
        const bf16x2 b0 = kv4_pair_bf16<0>(x.v[1], s1), b1 = kv4_pair_bf16<1>(x.v[1], s1), b2 = kv4_pair_bf16<2>(x.v[1], s1),
                     b3 = kv4_pair_bf16<3>(x.v[1], s1);
        const bf16x2 o[8] = {{a0[0], b0[0]}, {a0[1], b0[1]}, {a1[0], b1[0]}, {a1[1], b1[1]},
                             {a2[0], b2[0]}, {a2[1], b2[1]}, {a3[0], b3[0]}, {a3[1], b3[1]}};
#pragma unroll
        for (int t = 0; t < 8; ++t) *(bf16x2 *)(vd + t * 256) = o[t];
    };
    // 4-bit pages: tile m into its slot of the ring, from registers, or, mask rows, by direct loads (rare: waited for at once).  A tile
    // that there is not is written all the same: its slot is free
    auto stage4 = [&](int m, const Raw &x) __attribute__((always_inline)) {
        convert(x, m & (RING - 1));
        if (m < n_seq && it0 + m >= wk.n1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // what this wave just wrote must not come later
            dma_k(dks, mask_base(m), m & (RING - 1));
            dma_v(dvs, mask_base(m), m & (RING - 1));
            wait_loads<0>();
        }
    };
    // exact pages and mask rows: two direct loads of K or V of tile m; of a tile that there is not, through a buffer of no bytes
    auto from = [&](int4v pages, int4v rows, int m) {
        int4v desc;
        const bool mask = it0 + m >= wk.n1;
#pragma unroll
        for (int i = 0; i < 4; ++i) desc[i] = mask ? rows[i] : pages[i];
        desc[2] = m < n_seq ? desc[2] : 0;
        return desc;
    };
    auto ask_k = [&](int m, int page) __attribute__((always_inline)) {
        dma_k(from(dk, dks, m), it0 + m >= wk.n1 ? mask_base(m) : page_base(page), k_slot(m));
    };
    auto ask_v = [&](int m, int page) __attribute__((always_inline)) {
        dma_v(from(dv, dvs, m), it0 + m >= wk.n1 ? mask_base(m) : page_base(page), m & (RING - 1));
    };

    // K as A operand: lane = (tile row, half of the step); V^T as A operand: lane = (position, key half of the unit)
    auto k_frags = [&](int m, bf16x8 (&kf)[8]) __attribute__((always_inline)) {
        const unsigned char *p = reinterpret_cast<const unsigned char *>(&k_lds[k_slot(m)][0]) + lq * 256;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) kf[ks] = *(const bf16x8 *)(p + (((2 * ks + lh) ^ (lq & 15)) << 4));
    };
    auto v_frags = [&](int m, bf16x8 (&vf)[4][2]) __attribute__((always_inline)) {
        const unsigned char *p = reinterpret_cast<const unsigned char *>(&v_lds[m & (RING - 1)][0]);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) vf[t][u] = *(const bf16x8 *)(p + (((u * 2 + lh) * 128 + 32 * t + lq) << 4));
    };
    auto scores = [&](const bf16x8 (&kf)[8], f32x16 &s) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
    };
    // V^T values that are not finite, of a block that not every row sees whole: taken out of the fragments, and added for the
    // rows that see them, key by key from LDS (rare, and written to need few registers)
    auto set_aside = [&](int m, bf16x8 (&vf)[4][2], unsigned vis32) __attribute__((always_inline)) {
        unsigned odd = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4 w = __builtin_bit_cast(u32x4, vf[t][u]);
                odd |= nonfinite2(w[0]) | nonfinite2(w[1]) | nonfinite2(w[2]) | nonfinite2(w[3]);
            }
        if (__builtin_expect(__any(odd != 0), 0)) {
            const unsigned short *v = reinterpret_cast<const unsigned short *>(&v_lds[m & (RING - 1)][0]);
#pragma unroll 1
            for (int key = 0; key < 32; ++key) {
                const unsigned short *p = v + (key >> 3) * 1024 + (key & 7) + 32 * lh;
                const bool seen = (vis32 >> key) & 1u;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = __uint_as_float((unsigned)p[(32 * t + 8 * (e >> 2) + (e & 3)) * 8] << 16);
                        acc[t][e] += seen && !(fabsf(x) < INFINITY) ? x : 0.f;
                    }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    u32x4 w = __builtin_bit_cast(u32x4, vf[t][u]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
                        if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
                    }
                    vf[t][u] = __builtin_bit_cast(bf16x8, w);
                }
        }
    };

    Raw r0 = {}, r1 = {};
    int page = 0, page_v = 0;                            // of the next tile to be asked for, and of the last one
    if constexpr (KV4) {
#pragma unroll
        for (int m = 0; m < 3; ++m) stage4(m, fetch(page_at(m)));
        r0 = fetch(page_at(3));
        r1 = fetch(page_at(4));
        page = page_at(5);
    } else {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            page_v = checked(page_at(m));
            ask_k(m, page_v);
            if (m < 3) ask_v(m, page_v);
        }
        page = page_at(4);
    }
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) asm volatile("" : "+v"(qf[ks]));      // no wait for Q inside the loop
    wait_loads<0>();
    lds_barrier();
    f32x16 s;
    bf16x8 kf[8];
    if (here) {
        k_frags(0, kf);
        scores(kf, s);
        k_frags(1, kf);
    }
    // the reference of a row, moved where the block's scores outgrow it (rare)
    auto reference = [&]() __attribute__((always_inline)) {
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
        if (__builtin_expect(__any(!(mx * scale <= m_run + kLag)), 0)) {
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const bool grow = !(mx * scale <= m_run + kLag);
            const float m_new = grow ? fmaxf(m_run, ceilf(mx * scale)) : m_run;
            const float alpha = grow ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[t][e] *= alpha;
            m_run = m_new;
        }
    };
    // scores of the next block between the numerators of this one
    auto numerators = [&](f32x16 &s_next, bf16x8 (&pf)[2]) __attribute__((always_inline)) {
        scores(kf, s_next);
        const float m_safe = m_run == -INFINITY ? 0.f : m_run;
        const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const bf16x2 pk = {(bf16_t)__builtin_amdgcn_exp2f(fmaf(s[e], scale, -m_safe)),
                               (bf16_t)__builtin_amdgcn_exp2f(fmaf(s[e + 1], scale, -m_safe))};
            l_run = __builtin_amdgcn_fdot2_f32_bf16(pk, ones, l_run, false);
            pf[e >> 3][e & 7] = pk[0];
            pf[e >> 3][(e & 7) + 1] = pk[1];
        }
    };
    auto outputs = [&](const bf16x8 (&vf)[4][2], const bf16x8 (&pf)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t][u], pf[u], acc[t], 0, 0, 0);
    };
    // the tiles to come: 4-bit pages, the tile three blocks on; exact pages, K of block n + 4 and V of n + 3, which are needed
    // two iterations on
    auto ahead = [&](int n) __attribute__((always_inline)) {
        if constexpr (KV4) {
            stage4(n + 3, r0);
            r0 = r1;
            r1 = fetch(page);
            page = page_at(n + 6);
        } else {
            const int page_k = checked(page);
            page = page_at(n + 5);
            ask_k(n + 4, page_k);
            ask_v(n + 3, page_v);
            page_v = page_k;
            wait_loads<4>();                             // what was asked for before has landed
        }
        lds_barrier_counted();
    };
    if (!here) {                                         // no rows: this wave only moves tiles
        for (int n = 0; n < n_seq; ++n) ahead(n);
    } else {
        // blocks [f0, f1) are cache units that every row of the wave sees whole: no predicate there
        const int base = wk.w0 - wk.n_s + 2 * it0;
        const int f0 = max(((wk.n_s + 1) >> 1) - it0, ((((rb.lo1 + 15) >> 4) - base) + 1) >> 1), f1 = ((rb.hi0 >> 4) - base) >> 1;
        for (int n = 0; n < n_seq; ++n) {
            bf16x8 vf[4][2], pf[2];
            f32x16 s_next;
            v_frags(n, vf);
            unsigned vis = 0;
            const bool masked = n < f0 || n >= f1;
            if (masked) {
                const int it = it0 + n, w = 2 * (it - wk.n1);
                const bool cache = it < wk.n1;
                const int u0 = cache ? wk.cache_unit(2 * it) : wk.mask_unit(w), u1 = cache ? wk.cache_unit(2 * it + 1) : wk.mask_unit(w + 1);
                vis = cache ? cache_bits(rs, u0) | (cache_bits(rs, u1) << 16) : mask_bits(rs, u0) | (mask_bits(rs, u1) << 16);
                const unsigned mine = vis >> (8 * lh);   // register e: key 8 lh + e % 8 of unit e / 8
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = ((mine >> ((e & 7) + 16 * (e >> 3))) & 1u) ? s[e] : -INFINITY;
            }
            reference();
            if (masked) set_aside(n, vf, vis);           // (behind the rescale: a factor of zero would make NaN of infinity)
            numerators(s_next, pf);
            k_frags(n + 2, kf);
            outputs(vf, pf);
            s = s_next;
            ahead(n);
        }
    }

    // ---- results
    if (bad) bad_lds = 1;
    __syncthreads();
    if (!here) return;
    float l = l_run;
    l += __shfl_xor(l, 32);
    if (bad_lds) {
        l = __builtin_nanf("");
        if (m_run == -INFINITY) m_run = 0.f;
    }
    if (!row) return;
    const size_t orh = ((size_t)b * d.R + r) * c.n_q + g * a.group + hq;
    const size_t at = orh * a.splits + split;
    const float inv = 1.f / l;
    if (a.splits > 1 && lh == 0) {
        a.mpart[at] = m_run;
        a.lpart[at] = l;
    }
    if constexpr (KV4) {                                 // runs of eight: values 8 i .. + 7 of i = 8 h + 4 lh + e
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d0 = 8 * (8 * h + 4 * lh + e);
                float x[8];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    x[2 * t] = acc[t][4 * h + e];
                    x[2 * t + 1] = acc[t][8 + 4 * h + e];
                }
                if (a.splits > 1) {
                    *(f32x4 *)(a.opart + at * HD + d0) = (f32x4){x[0], x[1], x[2], x[3]};
                    *(f32x4 *)(a.opart + at * HD + d0 + 4) = (f32x4){x[4], x[5], x[6], x[7]};
                } else {
                    bf16x8 o;
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = (bf16_t)(x[i] * inv);
                    *(bf16x8 *)((bf16_t *)c.out + orh * HD + d0) = o;
                }
            }
    } else {
        typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int d0 = 32 * t + 8 * h + 4 * lh;
                const f32x4 x = {acc[t][4 * h], acc[t][4 * h + 1], acc[t][4 * h + 2], acc[t][4 * h + 3]};
                if (a.splits > 1)
                    *(f32x4 *)(a.opart + at * HD + d0) = x;
                else
                    *(bf16x4 *)((bf16_t *)c.out + orh * HD + d0) =
                        (bf16x4){(bf16_t)(x[0] * inv), (bf16_t)(x[1] * inv), (bf16_t)(x[2] * inv), (bf16_t)(x[3] * inv)};
            }
    }
}

}  // namespace

void launch_span_rows(const SpanArgs &a, int chunks, hipStream_t st) {
    const bool four = a.c.kv.k_pages == nullptr;
    const dim3 grid(a.c.B * (four ? a.c.kv4.n_kv : a.c.kv.n_kv) * chunks, a.splits);
    if (four) span_rows_kernel<true><<<grid, 256, 0, st>>>(a);
    else span_rows_kernel<false><<<grid, 256, 0, st>>>(a);
}
