// The attention over a span for many query rows (bf16): the walk, the mask and the softmax of kernels_span.hip with a tile of 32
// query rows to a wave, four waves to a workgroup, and K and V tiles of 32 keys that the four share in LDS.
//
// Scores are v_mfma_f32_32x32x16_bf16 products S^T = K Q^T; a lane's registers 8u .. 8u + 7 are its row's scores of keys 8 lh ..
// 8 lh + 7 of unit u, and after the exponential, packed, the B operand of O^T += V^T P^T.
//
// Tiles are staged in a ring of four.  Exact pages come by direct loads into LDS (lds_dma.h), three blocks ahead; of 4-bit
// pages every thread converts 16 elements of K and 16 of V per tile, so a tile is converted once for 128 query rows.  K rows
// of 256 bytes have their 16-byte pieces XOR-swizzled by the row and rows 4-7 and 8-11 of a unit exchanged; V^T is
// [unit][key half][position] 16-byte pieces, where position p is head-dim value p (exact pages) or 8 (p % 16) + p / 16 (4-bit
// pages: a wave's stores are contiguous then, and a lane's results are runs of eight values).
//
// Two workgroups share a compute unit, 512 run at a time.  As many whole ones as make full rounds go first; the walks of the rest,
// whose round would leave most of the chip idle, are cut into pieces of equal length (SpanPlan), and only their partial results are
// written and joined.
//
// Bound by the loop: 16 MFMAs (512 clocks) and, from exact pages where nothing is masked, about 70 vector instructions, 16 of them
// exponentials, per wave and block (over 4-bit pages 108 with conversion, masks and the way in).  Of one wave they follow from each other,
// scores, numerators, products, and nothing holds the two waves of a SIMD in opposite phases, so that they overlap little (waves
// with nothing but one of them each do overlap: MFMAs alone 248 us, beside a wave of FMAs that takes 294 alone 317); 1.06 PFLOP/s in long
// walks.  A step of 8 sequences of up to 8192 4-bit keys, 272 rows of 32 heads each: 258 us with placement and join (890 TFLOP/s);
// 2064 rows over an exact window of 1024: 65 us.  Trees of 64 rows of 16 sequences, 4600 to 8200 exact keys, 32 heads: 126 to 132 us, the loop
// by itself 111 to 123 (matrix cores busy 34 %); of 24 rows of 32 sequences over 4-bit pages 114, where a head's 96 rows leave one of the four waves idle.
#include <algorithm>
#include <cmath>

#include "lds_dma.h"
#include "span_device.h"

namespace {

constexpr int HD = 128, TILE = 32 * HD, RING = 4, ROWS = 128;

// A workgroup's rows: which (sequence, kv head), and which of its rows.
struct Place {
    int b, g;
    int f0, f1;                                          // rows [f0, f1) of the kv head's (head-major) list
    int R, row0;                                         // the sequence's rows, and the first of them
};
template <bool TREE>
__device__ inline Place place_of(const SpanArgs &a, int n_kv, int item) {
    // The chunks of a (sequence, kv head) group run on one XCD where the groups divide evenly over the eight
    // (workgroup i of a launch runs on XCD i % 8): its L2 then fetches the head's K and V once
    const int n_groups = a.c.B * n_kv;
    int grp, chunk;
    if (n_groups % 8 == 0) {
        const int j = item >> 3;
        grp = (j / a.tiles) * 8 + (item & 7);
        chunk = j % a.tiles;
    } else {
        grp = item / a.tiles;
        chunk = item % a.tiles;
    }
    const int per_span = (a.span_rows + ROWS - 1) / ROWS, span = chunk / per_span;
    // every other span backwards: the chunks of causal rows grow, and with them in one order an XCD got the long ones of all heads
    const int at = chunk - span * per_span, spans = a.tiles / per_span;
    Place p;
    p.b = grp / n_kv;
    p.g = grp - p.b * n_kv;
    p.R = a.c.d.R;
    p.row0 = p.b * p.R;
    if constexpr (TREE) p.R = tree_range(a.c.row_start, a.c.n_rows, a.c.d.R, p.b, p.row0);      // (tree_taken: where rows are stored)
    const int F = a.group * p.R;
    p.f0 = span * a.span_rows + ((grp * spans + span) & 1 ? per_span - 1 - at : at) * ROWS;
    p.f1 = min(min(p.f0 + ROWS, (span + 1) * a.span_rows), F);
    return p;
}

// The bounds that a walk needs (lo0, hi1, sk1, m0, m1) of rows [r0, r1) of a query head, and of a workgroup's rows.
__device__ inline RowBounds head_bounds(const RowDesc &d, int L, int r0, int r1, int window, int sinks) {
    int first = 0x7fffffff, hi = 0, m0 = 0x7fffffff, m1 = 0;             // first: the least position of a row
    if (r0 < d.nc) {
        first = L + r0;
        hi = L + min(r1, d.nc);
    }
    if (r1 > d.nc) {
        const int a = max(r0, d.nc) - d.nc, j0 = a / d.bl, j1 = (r1 - 1 - d.nc) / d.bl;
        first = min(first, L + d.cond0 + j0 * d.cstride + a - j0 * d.bl);
        if (j1 > j0) first = min(first, L + d.cond0 + (j0 + 1) * d.cstride);
        hi = max(hi, L + d.cond0 + j1 * d.cstride);
        m0 = j0 * d.bl;
        m1 = min((j1 + 1) * d.bl, d.nm);
    }
    return {window > 0 ? max(0, first - window + 1) : 0, 0, 0, hi, 0, window > 0 ? min(sinks, hi) : 0, m0, m1};
}
template <bool TREE>
__device__ inline Walk walk_at(const SpanArgs &a, const Place &p, int L) {
    if constexpr (TREE) return walk_of(tree_bounds(p.R, L), 0);
    const RowDesc &d = a.c.d;
    const int h0 = p.f0 / d.R, h1 = (p.f1 - 1) / d.R, ra = p.f0 - h0 * d.R, rb = p.f1 - h1 * d.R;
    const int w = a.c.window, t = a.c.sinks;
    return walk_of(h0 == h1 ? head_bounds(d, L, ra, rb, w, t)
                            : h1 == h0 + 1 ? join(head_bounds(d, L, ra, d.R, w, t), head_bounds(d, L, 0, rb, w, t))
                                           : head_bounds(d, L, 0, d.R, w, t), w);
}
__device__ inline bool length_of(const SpanArgs &a, int b, int pps, int &L) {
    const int x = a.c.prefix_len[a.c.d.seq_base + b];
    const bool fits = x >= 0 && (long long)x + a.c.d.nc <= (long long)pps * 16;
    L = fits ? x : 0;
    return fits;
}

// A lane's results: 16 pieces of four values (t, h) of its row, normalised, into the output.  KV4: value e of piece (t, h) is
// head-dim value 8 (8 (h % 2) + 4 lh + e) + 2 t + h / 2; else 32 t + 8 h + 4 lh + e.
template <bool KV4>
__device__ inline void store_row(bf16_t *out, const f32x4 (&x)[4][4], float inv, int lh) {
    if constexpr (KV4) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bf16x8 o;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    o[2 * t] = (bf16_t)(x[t][h][e] * inv);
                    o[2 * t + 1] = (bf16_t)(x[t][h + 2][e] * inv);
                }
                *(bf16x8 *)(out + 8 * (8 * h + 4 * lh + e)) = o;
            }
    } else {
        typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int h = 0; h < 4; ++h)
                *(bf16x4 *)(out + 32 * t + 8 * h + 4 * lh) = (bf16x4){(bf16_t)(x[t][h][0] * inv), (bf16_t)(x[t][h][1] * inv),
                                                                      (bf16_t)(x[t][h][2] * inv), (bf16_t)(x[t][h][3] * inv)};
    }
}
// Where the partial results of tile `wave` of piece `part` are: 16 pieces as they lie in the registers, a store being one contiguous KiB.
__device__ inline f32x4 *partial_of(const SpanArgs &a, int part, int wave) {
    return (f32x4 *)a.opart + ((size_t)part * 4 + wave) * 16 * 64;
}

template <bool KV4, bool TREE>
__global__ __launch_bounds__(256, 2) void span_rows_kernel(SpanArgs a) {
    __shared__ __attribute__((aligned(16))) bf16_t k_lds[RING][TILE];
    __shared__ __attribute__((aligned(16))) bf16_t v_lds[RING][TILE];
    __shared__ int bad_lds, taken_lds[4];                // (taken: a tree whose rows are another one's too, which stores them)
    __shared__ __attribute__((aligned(16))) uint32_t tree_lds[TREE ? ROWS * kTreeWords : 4];      // who the rows see of their tree
    const SpanCall &c = a.c;
    const RowDesc &d = c.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 31, lh = lane >> 5;
    const int n_kv = KV4 ? c.kv4.n_kv : c.kv.n_kv;
    const int pps = KV4 ? c.kv4.pages_per_seq : c.kv.pages_per_seq, n_pages = KV4 ? c.kv4.n_pages : c.kv.n_pages;
    const int cut = (int)blockIdx.x - a.whole;           // >= 0: a piece of a walk
    int item = blockIdx.x, split = 0, splits = 1;
    int part = cut;                                      // where this piece's partial results go
    if constexpr (TREE) {
        if (cut >= 0) {
            const int e = __builtin_amdgcn_readfirstlane(a.items[cut]);
            if (e < 0) return;                           // fewer pieces than the bound allows for (whole workgroup)
            item = e & 1023;
            split = (e >> 10) & 127;
            splits = e >> 17;
            part = item * a.splits + split;
            item += a.whole;
        }
    } else if (cut >= 0) {
        // Piece `cut` of the walks that are cut, numbered walk by walk; each has as many as it is long (a table of their first
        // pieces, made by every workgroup for itself: a launch with empty pieces between the others left a quarter of the
        // compute units without work while others had three).  Two of at most 511 walks to a thread.
        int *first = reinterpret_cast<int *>(&k_lds[0][0]), *sums = first + 514;
        const int rest = c.B * n_kv * a.tiles - a.whole;
        int n[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            n[k] = 0;
            if (2 * tid + k < rest) {
                const Place p = place_of<false>(a, n_kv, a.whole + 2 * tid + k);
                int L;
                n[k] = 1;
                if (length_of(a, p.b, pps, L)) {
                    const Walk w = walk_at<false>(a, p, L);
                    n[k] = max(1, min(a.splits, (w.n1 + w.n2 + a.per - 1) / a.per));
                }
            }
        }
        int sum = n[0] + n[1];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(sum, o);
            if (lane >= o) sum += x;
        }
        if (lane == 63) sums[wave] = sum;
        __syncthreads();
        for (int w = 0; w < wave; ++w) sum += sums[w];
        first[2 * tid] = sum - n[0] - n[1];
        first[2 * tid + 1] = sum - n[1];
        if (tid == 255) first[512] = sum;
        __syncthreads();
        if (cut >= first[512]) return;                   // fewer pieces than the bound allows for (whole workgroup)
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (first[2 * tid + k] <= cut && cut < first[2 * tid + k] + n[k]) sums[4] = 2 * tid + k;
        __syncthreads();
        item = __builtin_amdgcn_readfirstlane(sums[4]);
        split = __builtin_amdgcn_readfirstlane(cut - first[item]);
        splits = __builtin_amdgcn_readfirstlane(first[item + 1] - first[item]);
        if (split == 0 && tid == 0) {                    // for the join
            a.pieces[2 * item] = cut;
            a.pieces[2 * item + 1] = splits;
        }
        item += a.whole;
        __syncthreads();                                 // the table's place is a tile's
    }
    const Place pl = place_of<TREE>(a, n_kv, item);
    if (TREE && pl.f0 >= pl.f1) return;                  // (whole workgroup)
    const int b = pl.b, g = pl.g;
    int L;
    const bool fits = length_of(a, b, pps, L);
    const int f = pl.f0 + wave * 32 + lq;
    const bool here = pl.f0 + wave * 32 < pl.f1, row = f < pl.f1;        // (here: wave-uniform)
    const int R = TREE ? pl.R : d.R, hq = row ? f / R : 0, r = row ? f - hq * R : 0;
    const size_t orh = ((TREE ? (size_t)pl.row0 : (size_t)b * d.R) + r) * c.n_q + g * a.group + hq;    // (row, head) in q and out
    RowSpan rs = TREE ? tree_span(pl.R, L) : row_span(d, r, L, c.window, c.sinks);
    if constexpr (TREE) {                                // two threads to a row, four words each
        const int fr = pl.f0 + (tid >> 1), rr = fr - fr / pl.R * pl.R;
        u32x4 x = {0, 0, 0, 0};
        if (fr < pl.f1) x = *(const u32x4 *)(c.ancestors + ((size_t)pl.row0 + rr) * kTreeWords + 4 * (tid & 1));
        *(u32x4 *)(tree_lds + 4 * tid) = x;
        const bool taken = tree_taken(c.row_start, c.n_rows, d.R, b, pl.row0, pl.R, tid, 256);
        if (lane == 0) taken_lds[wave] = taken;
    }
    RowBounds rb;
    if constexpr (TREE) rb = tree_bounds(pl.R, L);
    else rb = wave_bounds<32>(bounds_of(rs, row));
    if (!row) rs = RowSpan{};
    if (tid == 0) bad_lds = 0;
    const Walk wk = walk_at<TREE>(a, pl, L);
    const int n_it = fits ? wk.n1 + wk.n2 : 0, per = TREE ? (n_it + splits - 1) / splits : a.per;      // (a tree's pieces of a walk are even)
    const int it0 = min(n_it, split * per);
    const int n_seq = (split == splits - 1 ? n_it : min(n_it, it0 + per)) - it0;
    const int32_t *pt = (KV4 ? c.kv4.page_table : c.kv.page_table) + (size_t)(d.seq_base + b) * pps;
    const int n_mt = (d.nm + 15) >> 4;
    bool bad = !fits;

    // ---- Q: B operand, lane = (row, half of the 16 head-dim values of a step)
    bf16x8 qf[8];
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
        qf[ks] = (bf16x8){0, 0, 0, 0, 0, 0, 0, 0};
        if (row) qf[ks] = *(const bf16x8 *)((const bf16_t *)c.q + orh * HD + 8 * lh + 16 * ks);
    }
    const float scale = kLog2e / sqrtf((float)HD);
    const float inv_scale = 1.f / scale;
    f32x16 acc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    float m_neg = 0.f, m_most = -INFINITY;               // what is added to scores; scores beyond which the reference moves

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
    // Page ids of this wave's units, 64 tiles at a time: lane i holds tile page0 + i's (0 for a unit that is not there), the
    // next 64 are on their way.  (As scalar loads, one per iteration, they shared their counter with the LDS reads: every
    // wait for LDS, the one in front of the barrier too, then waited for the table as well.)
    const int n_cache = wk.n_s + wk.n_w;
    auto load_pages = [&](int m0) {
        const int m = m0 + lane, w = 2 * (it0 + m) + u_w;
        return m < n_seq && w < n_cache ? pt[w < wk.n_s ? w : wk.w0 + (w - wk.n_s)] : 0;
    };
    int page0 = 0, pages = load_pages(0), pages_next = load_pages(64);
    auto page_at = [&](int m) {
        if (m - page0 >= 64) {
            page0 += 64;
            pages = pages_next;
            pages_next = load_pages(page0 + 64);
        }
        const int page = __builtin_amdgcn_readlane(pages, m - page0);
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
        const unsigned char *p = c.kv4.pages + kv4_offset(c.kv4, page, g);
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
    auto stage4 = [&](int m, int slot, const Raw &x) __attribute__((always_inline)) {
        convert(x, slot);
        if (m < n_seq && it0 + m >= wk.n1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // what this wave just wrote must not come later
            dma_k(dks, mask_base(m), slot);
            dma_v(dvs, mask_base(m), slot);
            wait_loads<0>();
        }
    };
    // exact pages and mask rows: four direct loads of tile m; of a tile that there is not, through a buffer of no bytes
    auto ask = [&](int m, int slot, int page) __attribute__((always_inline)) {
        const bool mask = it0 + m >= wk.n1;
        int4v kd, vd;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kd[i] = mask ? dks[i] : dk[i];
            vd[i] = mask ? dvs[i] : dv[i];
        }
        kd[2] = m < n_seq ? kd[2] : 0;
        vd[2] = m < n_seq ? vd[2] : 0;
        const int base = mask ? mask_base(m) : page_base(page);
        dma_k(kd, base, slot);
        dma_v(vd, base, slot);
    };

    // K as A operand: lane = (tile row, half of the step); V^T as A operand: lane = (position, key half of the unit)
    auto k_frags = [&](int slot, bf16x8 (&kf)[8]) __attribute__((always_inline)) {
        const unsigned char *p = reinterpret_cast<const unsigned char *>(&k_lds[slot][0]) + lq * 256;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) kf[ks] = *(const bf16x8 *)(p + (((2 * ks + lh) ^ (lq & 15)) << 4));
    };
    auto scores = [&](const bf16x8 (&kf)[8], f32x16 &s) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
    };
    auto v_frags = [&](int slot, bf16x8 (&vf)[4][2]) __attribute__((always_inline)) {
        const unsigned char *p = reinterpret_cast<const unsigned char *>(&v_lds[slot][0]);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) vf[t][u] = *(const bf16x8 *)(p + (((u * 2 + lh) * 128 + 32 * t + lq) << 4));
    };
    // V^T values that are not finite, of a block that not every row sees whole: taken out of the fragments, and added for the
    // rows that see them, key by key from LDS (rare, and written to need few registers; what lies in slots that no row
    // sees, unset memory perhaps, costs the first step only)
    auto set_aside = [&](int slot, bf16x8 (&vf)[4][2], unsigned vis) __attribute__((always_inline)) {
        unsigned top = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4 w = __builtin_bit_cast(u32x4, vf[t][u]);
                top = top2(top2(top2(top2(top, w[0]), w[1]), w[2]), w[3]);
            }
        if (__builtin_expect(__any(nonfinite2(top) != 0), 0)) {
            const unsigned short *v = reinterpret_cast<const unsigned short *>(&v_lds[slot][0]);
            unsigned keys = 0;                           // this lane's: bit 8 u + e
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) keys |= nonfinite8(vf[t][u]) << (8 * u);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) keys |= __shfl_xor(keys, o);
            const unsigned other = __shfl_xor(keys, 32), lo = lh ? other : keys, hi = lh ? keys : other;
            keys = __builtin_amdgcn_readfirstlane((lo & 0xffu) | ((hi & 0xffu) << 8) | ((lo & 0xff00u) << 8) | ((hi & 0xff00u) << 16));
#pragma unroll 1
            for (int key = 0; key < 32; ++key) {
                if (!((keys >> key) & 1u) || !__any((vis >> key) & 1u)) continue;
                const unsigned short *p = v + (key >> 3) * 1024 + (key & 7) + 32 * lh;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = __uint_as_float((unsigned)p[(32 * t + 8 * (e >> 2) + (e & 3)) * 8] << 16);
                        const float y = fabsf(x) < INFINITY ? 0.f : x;
                        acc[t][e] += ((vis >> key) & 1u) ? y : 0.f;
                    }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) vf[t][u] = finite_only(vf[t][u]);
        }
    };

    // Tiles to come.  Exact pages: at the start of iteration n tile n + 3 is asked for, at its end tile n + 2 has landed.  4-bit
    // pages: at the end of iteration n the codes of tile n + 3 are converted and those of tile n + 5 asked for in their place: the
    // iterations take turns with two sets of registers (handed on from one to the next, a copy would wait for the newest load)
    Raw r0 = {}, r1 = {};
    if constexpr (KV4) {
#pragma unroll
        for (int m = 0; m < 3; ++m) stage4(m, m, fetch(page_at(m)));
        r0 = fetch(page_at(3));
        r1 = fetch(page_at(4));
    } else {
#pragma unroll
        for (int m = 0; m < 3; ++m) ask(m, m, page_at(m));
    }
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) asm volatile("" : "+v"(qf[ks]));      // no wait for Q inside the loop
    wait_loads<0>();
    lds_barrier();
    auto begin = [&](int n, int slot) __attribute__((always_inline)) {
        if constexpr (!KV4) ask(n + 3, (slot + 3) % RING, page_at(n + 3));
    };
    auto finish = [&](int n, int slot, Raw &x) __attribute__((always_inline)) {
        if constexpr (KV4) {
            stage4(n + 3, (slot + 3) % RING, x);
            x = fetch(page_at(n + 5));
        } else {
            wait_loads<4>();
        }
        lds_barrier_counted();
    };
    // four iterations at a time: a tile's place in the ring is then part of the LDS instructions (274.5 -> 267.5 us)
    auto take_turns = [&](auto &turn) __attribute__((always_inline)) {
        for (int n = 0; n < n_seq; ++n) {
            turn(n, 0, r0);
            if (++n == n_seq) break;
            turn(n, 1, r1);
            if (++n == n_seq) break;
            turn(n, 2, r0);
            if (++n == n_seq) break;
            turn(n, 3, r1);
        }
    };
    if (!here) {                                         // no rows: this wave only moves tiles
        auto turn = [&](int n, int slot, Raw &x) __attribute__((always_inline)) {
            begin(n, slot);
            finish(n, slot, x);
        };
        take_turns(turn);
    } else {
        // blocks [f0, f1) are cache units that every row of the wave sees whole: no predicate there
        const int base = wk.w0 - wk.n_s + 2 * it0;
        const int f0 = __builtin_amdgcn_readfirstlane(max(((wk.n_s + 1) >> 1) - it0, ((((rb.lo1 + 15) >> 4) - base) + 1) >> 1));
        const int f1 = __builtin_amdgcn_readfirstlane(((rb.hi0 >> 4) - base) >> 1);
        // K of tile n + 1 is read while tile n's numerators are formed (69.2 -> 66.7 us for a pass of 2064 rows of 32 heads from
        // exact pages, 263.5 -> 257.0 for a step of 8 sequences from 4-bit pages)
        bf16x8 k_next[8];
        k_frags(0, k_next);
        auto turn = [&](int n, int slot, Raw &x) __attribute__((always_inline)) {
            begin(n, slot);
            f32x16 s;
            bf16x8 vf[4][2];
            u32x4 pw[2];
            scores(k_next, s);
            v_frags(slot, vf);
            k_frags((slot + 1) % RING, k_next);
            unsigned vis = 0;
            const bool masked = n < f0 || n >= f1;
            if (masked) {
                const int it = it0 + n, w = 2 * (it - wk.n1);
                const bool cache = it < wk.n1;
                const int u0 = cache ? wk.cache_unit(2 * it) : wk.mask_unit(w), u1 = cache ? wk.cache_unit(2 * it + 1) : wk.mask_unit(w + 1);
                if (TREE && !cache) vis = tree_bits(tree_lds[(wave * 32 + lq) * kTreeWords + (it - wk.n1)], it - wk.n1, pl.R);
                else vis = cache ? cache_bits(rs, u0) | (cache_bits(rs, u1) << 16) : mask_bits(rs, u0) | (mask_bits(rs, u1) << 16);
                const unsigned mine = vis >> (8 * lh);   // register e: key 8 lh + e % 8 of unit e / 8
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = seen_or_not(mine, (e & 7) + 16 * (e >> 3), s[e]);
            }
            // the reference of a row, moved where the block's scores outgrow it (rare)
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
            if (__builtin_expect(__any(!(mx <= m_most)), 0)) {
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                if (!(mx <= m_most)) {
                    const float m_new = fmaxf(m_run, ceilf(mx * scale)), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
                    l_run *= alpha;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[t][e] *= alpha;
                    m_run = m_new;
                    m_neg = m_new == -INFINITY ? 0.f : -m_new;
                    m_most = (m_new + kLag) * inv_scale;
                }
            }
            if (masked) set_aside(slot, vf, vis);           // (behind the rescale: a factor of zero would make NaN of infinity)
            const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const bf16x2 pk = {(bf16_t)__builtin_amdgcn_exp2f(fmaf(s[e], scale, m_neg)),
                                   (bf16_t)__builtin_amdgcn_exp2f(fmaf(s[e + 1], scale, m_neg))};
                l_run = __builtin_amdgcn_fdot2_f32_bf16(pk, ones, l_run, false);
                pw[e >> 3][(e & 7) >> 1] = __builtin_bit_cast(unsigned, pk);
            }
            const bf16x8 pf[2] = {__builtin_bit_cast(bf16x8, pw[0]), __builtin_bit_cast(bf16x8, pw[1])};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t][u], pf[u], acc[t], 0, 0, 0);
            finish(n, slot, x);
        };
        take_turns(turn);
    }

    // ---- results
    if (bad) bad_lds = 1;
    __syncthreads();
    if (!here) return;
    if (TREE && (taken_lds[0] | taken_lds[1] | taken_lds[2] | taken_lds[3])) return;
    float l = l_run;
    l += __shfl_xor(l, 32);
    if (bad_lds) {
        l = __builtin_nanf("");
        if (m_run == -INFINITY) m_run = 0.f;
    }
    f32x4 x[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int h = 0; h < 4; ++h) x[t][h] = (f32x4){acc[t][4 * h], acc[t][4 * h + 1], acc[t][4 * h + 2], acc[t][4 * h + 3]};
    if (cut < 0) {
        if (TREE && row && l == 0.f && !tree_sees(c.ancestors + ((size_t)pl.row0 + r) * kTreeWords, pl.R, L)) l = 1.f;       // zeros
        if (row) store_row<KV4>((bf16_t *)c.out + orh * HD, x, 1.f / l, lh);
        return;
    }
    f32x4 *op = partial_of(a, part, wave) + lane;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int h = 0; h < 4; ++h) op[(4 * t + h) * 64] = x[t][h];
    if (lh == 0) {
        a.mpart[(size_t)part * ROWS + wave * 32 + lq] = m_run;
        a.lpart[(size_t)part * ROWS + wave * 32 + lq] = l;
    }
}

// out = sum_s w_s O_s / sum_s w_s l_s, w_s = 2^(m_s - max m), of the workgroups that were cut.  A wave takes half of the
// results of a tile of 32 rows: pieces (t, h) and (t, h + 2) of all t, whole runs of eight values with 4-bit pages.
template <bool KV4, bool TREE>
__global__ __launch_bounds__(128) void span_rows_join_kernel(SpanArgs a) {
    const SpanCall &c = a.c;
    const int lane = threadIdx.x & 63, lq = lane & 31, lh = lane >> 5, half = threadIdx.x >> 6, wave = blockIdx.x & 3;
    const int tail = blockIdx.x >> 2, n_kv = KV4 ? c.kv4.n_kv : c.kv.n_kv;
    const Place pl = place_of<TREE>(a, n_kv, a.whole + tail);
    const int f = pl.f0 + wave * 32 + lq;
    if (pl.f0 + wave * 32 >= pl.f1 || (TREE && tree_taken(c.row_start, c.n_rows, c.d.R, pl.b, pl.row0, pl.R, lane, 64))) return;
    const int part = a.pieces[2 * tail], S = a.pieces[2 * tail + 1];
    const float *mp = a.mpart + (size_t)part * ROWS + wave * 32 + lq, *lp = a.lpart + (size_t)part * ROWS + wave * 32 + lq;
    float m = -INFINITY;
#pragma unroll 8
    for (int s = 0; s < S; ++s) m = fmaxf(m, mp[(size_t)s * ROWS]);
    f32x4 num[4][2];
    float den = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) num[t][0] = num[t][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < S; s0 += 2) {
        f32x4 x[2][4][2];
        float ms[2], ls[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int s = min(s0 + j, S - 1);
            ms[j] = mp[(size_t)s * ROWS];
            ls[j] = s0 + j < S ? lp[(size_t)s * ROWS] : 0.f;
            const f32x4 *op = partial_of(a, part + s, wave) + lane;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) x[j][t][i] = op[(4 * t + half + 2 * i) * 64];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (ls[j] == 0.f) continue;                  // saw nothing (a piece of NaN scores alone has a maximum of -inf too)
            const float w = ms[j] == m ? 1.f : __builtin_amdgcn_exp2f(ms[j] - m);
            den += w * ls[j];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) num[t][i][e] += w * x[j][t][i][e];
        }
    }
    if (f >= pl.f1) return;
    const int R = TREE ? pl.R : c.d.R, hq = f / R, r = f - hq * R;
    if (TREE && den == 0.f && !tree_sees(c.ancestors + ((size_t)pl.row0 + r) * kTreeWords, pl.R, c.prefix_len[pl.b])) den = 1.f;
    const float inv = 1.f / den;
    bf16_t *out = (bf16_t *)c.out + (((TREE ? (size_t)pl.row0 : (size_t)pl.b * c.d.R) + r) * c.n_q + pl.g * a.group + hq) * HD;
    if constexpr (KV4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            bf16x8 o;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                o[2 * t] = (bf16_t)(num[t][0][e] * inv);
                o[2 * t + 1] = (bf16_t)(num[t][1][e] * inv);
            }
            *(bf16x8 *)(out + 8 * (8 * half + 4 * lh + e)) = o;
        }
    } else {
        typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *(bf16x4 *)(out + 32 * t + 8 * (half + 2 * i) + 4 * lh) =
                    (bf16x4){(bf16_t)(num[t][i][0] * inv), (bf16_t)(num[t][i][1] * inv), (bf16_t)(num[t][i][2] * inv),
                             (bf16_t)(num[t][i][3] * inv)};
    }
}

// Before the attention of trees: their K/V as tiles of 16 rows, K [16][128] and V [128][16], a workgroup to a tile, and, by the first
// workgroup, what the attention's workgroups (those that are not whole) do: walk | piece << 10 | pieces << 17, or -1.  (Made by every
// attention workgroup for itself, as other calls do, the table took each 2.6 us of 17 for 96 walks and 3.9 for 256.)
// Where all walks are cut, the pieces of a head's chunks that read the same keys stand eight apart, so that they run at once on one XCD, and
// the head's pieces go by their length: two workgroups share a compute unit, number x and x + 256, so the first half goes from long to
// short and the second from short to long (16 sequences of 4600 to 8200 keys, 64 rows: 138 us in the sequences' order, so 129).
__global__ __launch_bounds__(256) void tree_rows_prepare_kernel(SpanArgs a, const bf16_t *__restrict__ k_new, const bf16_t *__restrict__ v_new,
                                                                int n_kv, int pps, int first_tile, int n_items) {
    const SpanCall &c = a.c;
    const int tid = threadIdx.x, n_mt = (c.d.nm + 15) >> 4, groups = c.B * n_kv;
    if ((int)blockIdx.x >= first_tile) {
        __shared__ __attribute__((aligned(16))) bf16_t vt[16][HD + 2];
        const int at0 = blockIdx.x - first_tile, mt = at0 % n_mt, bg = at0 / n_mt, b = bg / n_kv, g = bg - b * n_kv;
        int row0;
        const int R = tree_range(c.row_start, c.n_rows, c.d.R, b, row0), n = R - 16 * mt;
        if (n <= 0) return;
        typedef bf16x8 any_bf16x8 __attribute__((aligned(2)));
        const int r = tid >> 4, e = (tid & 15) * 8;
        bf16x8 k = {0, 0, 0, 0, 0, 0, 0, 0}, v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (r < n) {                                     // behind the tree: zeros, the attention need not look closer
            const size_t at = (((size_t)row0 + 16 * mt + r) * n_kv + g) * HD + e;
            k = *(const any_bf16x8 *)(k_new + at);
            v = *(const any_bf16x8 *)(v_new + at);
        }
        *(bf16x8 *)((bf16_t *)c.k_scr + (size_t)at0 * 16 * HD + r * HD + e) = k;
#pragma unroll
        for (int j = 0; j < 8; ++j) vt[r][e + j] = v[j];
        __syncthreads();
        const int d = tid >> 1, s = (tid & 1) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = vt[s + j][d];
        *(bf16x8 *)((bf16_t *)c.v_scr + (size_t)at0 * 16 * HD + d * 16 + s) = v;
        return;
    }
    // ---- the table.  All walks of a sequence, of its heads and chunks of rows, have the same keys
    __shared__ int len[512], order[512], sums[4];        // (fewer than 512 walks are cut)
    const int rest = groups * a.tiles - a.whole, lane = tid & 63, wave = tid >> 6;
    auto pieces_of = [&](int b, int &keys) {             // of a walk of sequence b, and the iterations of one
        int L, row0;
        const int n = tree_range(c.row_start, c.n_rows, c.d.R, b, row0);
        keys = 0;
        if (n == 0) return 0;
        if (!length_of(a, b, pps, L)) return 1;
        const Walk w = walk_of(tree_bounds(n, L), 0);
        const int p = max(1, min(a.splits, (w.n1 + w.n2 + a.per - 1) / a.per));
        keys = (w.n1 + w.n2 + p - 1) / p;
        return p;
    };
    auto sum_to = [&](int x) {                           // of all threads before this one and itself; sums[] then holds the waves'
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(x, o);
            if (lane >= o) x += y;
        }
        if (lane == 63) sums[wave] = x;
        __syncthreads();
        for (int w = 0; w < wave; ++w) x += sums[w];
        return x;
    };
    for (int i = tid; i < n_items; i += 256) a.items[i] = -1;
    if (a.whole > 0) {                                   // the last walks of a large call: one after another
        int n[2], keys;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            n[k] = 0;
            if (2 * tid + k < rest) {
                const Place p = place_of<true>(a, n_kv, a.whole + 2 * tid + k);
                n[k] = p.f0 < p.f1 ? pieces_of(p.b, keys) : 0;
            }
        }
        int at = sum_to(n[0] + n[1]) - n[0] - n[1];      // (its barrier: items[] is cleared)
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (2 * tid + k < rest) {
                a.pieces[2 * (2 * tid + k)] = (2 * tid + k) * a.splits;
                a.pieces[2 * (2 * tid + k) + 1] = n[k];
                for (int s = 0; s < n[k]; ++s, ++at) a.items[at] = (2 * tid + k) | s << 10 | n[k] << 17;
            }
        return;
    }
    // sequences by the length of their pieces, and how many pieces of all heads come before each
    int pieces[2], rank[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int b = tid + 256 * k;
        int keys = -1;
        pieces[k] = b < c.B ? pieces_of(b, keys) : 0;
        len[b] = keys;
        order[b] = 0;
    }
    __syncthreads();
    for (int x = 0; x < c.B; ++x) {
        const int lx = len[x];
#pragma unroll
        for (int k = 0; k < 2; ++k) rank[k] += lx > len[tid + 256 * k] || (lx == len[tid + 256 * k] && x < tid + 256 * k);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (tid + 256 * k < c.B) order[rank[k]] = pieces[k] * n_kv;
    __syncthreads();
    const int x0 = order[2 * tid], x1 = order[2 * tid + 1], before = sum_to(x0 + x1) - x0 - x1;
    order[2 * tid] = before;
    order[2 * tid + 1] = before + x0;
    __syncthreads();
    const int total = sums[0] + sums[1] + sums[2] + sums[3];
    // (more than 32 chunks to a head: eight pieces of each are more workgroups than units, and all go from long to short; there are few such pieces,
    // and the other way round took as long: 7 trees of 256 rows of 32 heads over one of K/V, 4600 to 8000 keys, 185.2 and 185.6 us)
    const int half = a.tiles > 32 ? total : min(total, 256 / a.tiles / 8 * 8);
#pragma unroll
    for (int k = 0; k < 2; ++k)                          // (by sequence from here on: pieces, and where they begin)
        if (tid + 256 * k < c.B) len[tid + 256 * k] = pieces[k] | order[rank[k]] << 8;
    __syncthreads();
    for (int item = tid; item < rest; item += 256) {
        const Place p = place_of<true>(a, n_kv, item);
        const int of = len[p.b], n = p.f0 < p.f1 ? of & 255 : 0, first = (of >> 8) + p.g * (of & 255);
        const int chunk = groups % 8 == 0 ? (item >> 3) % a.tiles : item % a.tiles;
        a.pieces[2 * item] = item * a.splits;
        a.pieces[2 * item + 1] = n;
        for (int s = 0; s < n; ++s) {
            const int v = first + s, u = v < half ? v : half + total - 1 - v;
            a.items[(u >> 3) * 8 * a.tiles + chunk * 8 + (u & 7)] = item | s << 10 | n << 17;
        }
    }
}

int groups_of(const SpanArgs &a) { return a.c.B * (a.c.kv.k_pages ? a.c.kv.n_kv : a.c.kv4.n_kv); }

}  // namespace

// Whole workgroups first, then the pieces of the rest: of every round but the last 512 workgroups, two to a compute unit, run at a
// time.  The rest (fewer than 512) is cut into pieces of equal length, at most `splits` of each, as many as take the least time.
// An iteration counts 1.2 with two workgroups on every unit and 0.8 with one; a workgroup has a prologue of about eight iterations,
// and twelve more where its partial results (66 KB) go out and come back.  (Long even walks take 1.02 and 0.53 us an iteration, but
// with those numbers 8 sequences of 8000 4-bit keys and 1632 rows of 12 heads take 184 us instead of 151.)  No more than 1024 workgroups and one per four
// iterations: that bound sizes the workspace, which then depends on the rows alone.
void plan_span_rows(int B, int n_kv, int group, const RowDesc &d, int window, int sinks, int max_prefix, SpanPlan *p) {
    const int F = group * d.R;
    // rows of one head see one run of keys where they are many: chunks that run over the end of a head would walk all of them
    p->span_rows = d.nc >= ROWS ? d.R : F;
    const int per_span = (p->span_rows + ROWS - 1) / ROWS;
    p->tiles = F / p->span_rows * per_span;
    const int items = B * n_kv * p->tiles, rest = items % 512;
    const int most = rest ? std::min(64, 1024 / rest) : 1;
    const int iters = (int)((span_keys(d, p->span_rows == F ? d.R : ROWS, window, sinks, max_prefix) + 31) / 32);
    // workgroups that have something to do: without a window the causal rows of a chunk see what is before them only
    auto busy = [&](int s, int per) {
        if (s == 1 || window > 0 || p->span_rows == F) return (double)rest * s;
        double n = 0.0;
        for (int k = 1; k <= per_span; ++k) n += ((max_prefix + std::min(ROWS * k, d.R) + 31) / 32 + per - 1) / per;
        return n / per_span * rest;
    };
    p->splits = 1;
    p->per = 1 << 30;
    double best = 0.0;
    for (int s = 1; s <= most && (s == 1 || 4 * s <= iters); ++s) {
        const int per = (iters + s - 1) / s;
        const double rounds = std::ceil(busy(s, per) / 256.0);            // of one workgroup per unit
        const double full = std::floor(rounds / 2.0), t = (1.2 * full + 0.8 * (rounds - 2.0 * full)) * (per + (s == 1 ? 8 : 20));
        if (s == 1 || t < 0.97 * best) {
            best = t;
            p->splits = s;
            p->per = s == 1 ? 1 << 30 : per;
        }
    }
    p->whole = p->splits == 1 ? items : items - rest;
    p->part_floats = most > 1 ? (size_t)rest * (most * ROWS * (HD + 2) + 2) : 0;
    if (d.nc == 0 && most > 1) p->part_floats += tree_items(B * n_kv, items - rest, p->tiles, most);      // (a tree: and the workgroups' table)
}

// (eight pieces of each chunk at a time: the last eight may not be full)
int tree_items(int groups, int whole, int tiles, int splits) {
    return whole > 0 ? (groups * tiles - whole) * splits : (groups * splits + 7) / 8 * 8 * tiles;
}
static int items_cut(const SpanArgs &a) { return tree_items(groups_of(a), a.whole, a.tiles, a.splits); }

void launch_tree_rows_prepare(const SpanArgs &a, const bf16_t *k_new, const bf16_t *v_new, hipStream_t st) {
    const bool four = a.c.kv.k_pages == nullptr;
    const int n_kv = four ? a.c.kv4.n_kv : a.c.kv.n_kv, pps = four ? a.c.kv4.pages_per_seq : a.c.kv.pages_per_seq;
    const bool cut = a.splits > 1;
    const int grid = groups_of(a) * ((a.c.d.nm + 15) / 16) + (cut ? 1 : 0);
    tree_rows_prepare_kernel<<<grid, 256, 0, st>>>(a, k_new, v_new, n_kv, pps, cut ? 1 : 0, cut ? items_cut(a) : 0);
}

void launch_span_rows(const SpanArgs &a, hipStream_t st) {
    const int items = groups_of(a) * a.tiles, grid = a.whole + (a.c.row_start && a.splits > 1 ? items_cut(a) : (items - a.whole) * a.splits);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(a); };
    if (!a.c.row_start) go(a.c.kv.k_pages ? span_rows_kernel<false, false> : span_rows_kernel<true, false>);
    else go(a.c.kv.k_pages ? span_rows_kernel<false, true> : span_rows_kernel<true, true>);
}

void launch_span_rows_join(const SpanArgs &a, hipStream_t st) {
    const int tail = groups_of(a) * a.tiles - a.whole;
    auto go = [&](auto kernel) { kernel<<<tail * 4, 128, 0, st>>>(a); };
    if (!a.c.row_start) go(a.c.kv.k_pages ? span_rows_join_kernel<false, false> : span_rows_join_kernel<true, false>);
    else go(a.c.kv.k_pages ? span_rows_join_kernel<false, true> : span_rows_join_kernel<true, true>);
}
