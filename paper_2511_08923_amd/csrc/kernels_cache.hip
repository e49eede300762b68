// Kernels around the paged cache: page tables and slot maps from request lengths, rows of K and V into 4-bit pages and
// back, and the placement of a windowed attention's new rows.  All of them move bytes; what bounds each stands with it.
#include <algorithm>

#include "kv4_format.h"
#include "tidar_internal.h"

namespace {

// ------------------------------------------------------------------ page tables and slot maps
// Sequence b holds P_b positions, has h_b pages and gets n_b rows more: it needs ceil((P_b + n_b) / 16) - h_b pages of the
// free list (or none), in the order of the sequences.  Where a sequence's pages begin in the list, and its rows in the
// slot map, is an exclusive sum over the sequences before it.  Every workgroup adds up its predecessors by itself, so the
// whole is one launch: up to 512 workgroups read 12 bytes of each predecessor from L2 (batch 2048: 6 MB in all), which is less than
// the second launch that a scan in two steps costs.  A wave then takes a sequence at a time, its pages a lane each.  Bound by the
// launch and three dependent trips to memory: 4.4 us for six sequences, 6.7 us for 2048 that get 50 k rows.
struct TableArgs {
    int batch;
    const int32_t *prefix_len, *n_new, *held, *free_pages;
    int n_free;
    int32_t *page_table;
    int pages_per_seq, n_pages;
    int32_t *row_start, *slots;
    int slot_cap;
    int32_t *held_out, *granted, *n_taken;
    int per_wg;               // sequences of a workgroup
};

struct SeqNeed {
    int P, n;                 // n: rows, 0 where the count is out of range
    int held, need;           // need 0 where the sequence is not valid
    bool ok;
};
__device__ inline SeqNeed seq_need(const TableArgs &a, int b) {
    const int cap = a.pages_per_seq * 16, P = a.prefix_len[b], n = a.n_new[b], held = a.held[b];
    SeqNeed s;
    const bool rows_ok = n >= 0 && n <= cap;
    s.ok = rows_ok && P >= 0 && P <= cap - n && held <= a.pages_per_seq && ((P + 15) >> 4) <= held;
    s.P = s.ok ? P : 0;
    s.n = rows_ok ? n : 0;
    s.held = s.ok ? held : 0;
    s.need = s.ok ? max(0, ((P + n + 15) >> 4) - held) : 0;
    return s;
}
__device__ inline int saturate(long long v) { return v > 0x7fffffff ? 0x7fffffff : (int)v; }
__global__ __launch_bounds__(256) void table_extend_kernel(TableArgs a) {
    __shared__ long long sum_need[256], sum_rows[256];    // inclusive, of a run of up to 256 sequences
    __shared__ SeqNeed seqs[256];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b0 = blockIdx.x * a.per_wg, b1 = min(a.batch, b0 + a.per_wg);
    // what the sequences before this workgroup's need, and their rows
    long long base_need = 0, base_rows = 0;
    for (int b = tid; b < b0; b += 256) {
        const SeqNeed s = seq_need(a, b);
        base_need += s.need;
        base_rows += s.n;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        base_need += __shfl_xor(base_need, o);
        base_rows += __shfl_xor(base_rows, o);
    }
    if (lane == 0) {
        sum_need[wave] = base_need;
        sum_rows[wave] = base_rows;
    }
    __syncthreads();
    base_need = sum_need[0] + sum_need[1] + sum_need[2] + sum_need[3];
    base_rows = sum_rows[0] + sum_rows[1] + sum_rows[2] + sum_rows[3];
    // The sequences whose pages the list has and whose rows the slot map has are the first ones (both sums only grow), and so
    // what the list has lost is what they need together: the workgroup that they end in writes it
    const bool was_in = base_need <= a.n_free && base_rows <= a.slot_cap;
    long long taken = base_need;
    for (int c0 = b0; c0 < b1; c0 += 256) {
        const int m = min(256, b1 - c0);
        __syncthreads();
        SeqNeed mine = {};
        if (tid < m) mine = seq_need(a, c0 + tid);
        seqs[tid] = mine;
        long long x = mine.need, y = mine.n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long px = __shfl_up(x, o), py = __shfl_up(y, o);
            if (lane >= o) {
                x += px;
                y += py;
            }
        }
        sum_need[tid] = x;
        sum_rows[tid] = y;
        __syncthreads();
        for (int w = 0; w < wave; ++w) {
            x += sum_need[64 * w + 63];
            y += sum_rows[64 * w + 63];
        }
        __syncthreads();
        sum_need[tid] = x;
        sum_rows[tid] = y;
        if (tid < m && base_need + x <= a.n_free && base_rows + y <= a.slot_cap) taken = max(taken, base_need + x);
        __syncthreads();
        for (int i = wave; i < m; i += 4) {               // a wave to a sequence
            const int b = c0 + i;
            const SeqNeed s = seqs[i];
            const long long off = base_need + sum_need[i] - s.need;
            const long long row0 = base_rows + sum_rows[i] - s.n, row1 = row0 + s.n;
            int32_t *table = a.page_table + (size_t)b * a.pages_per_seq;
            const bool room = s.ok && (s.need == 0 || off + s.need <= a.n_free) && (s.n == 0 || row1 <= a.slot_cap);
            // the pages that the new rows go into: those that the sequence has, and those from the list; a lane each
            const int first = s.P >> 4, pages = s.n > 0 ? ((s.P + s.n + 15) >> 4) - first : 0;
            auto page_of = [&](int j) {                   // logical page first + j
                const int lp = first + j;
                return lp < s.held ? table[lp] : a.free_pages[off + (lp - s.held)];
            };
            bool ids = true;
            int page = 0;
            if (room)
                for (int j = lane; j < pages; j += 64) {
                    const int p = page_of(j);
                    if (j < 64) page = p;
                    ids = ids && (unsigned)p < (unsigned)a.n_pages;
                }
            ids = __all(ids);
            const int granted = !s.ok ? -1 : !room ? 0 : ids ? 1 : -1;
            for (int j0 = 0; j0 == 0 || j0 < pages; j0 += 64) {
                const int j = j0 + lane;
                if (j0 > 0 && granted == 1 && j < pages) page = page_of(j);
                if (granted == 1 && j < pages && first + j >= s.held) table[first + j] = page;
                // rows of these 64 pages
                const int p0 = max(s.P, 16 * (first + j0)), p1 = min(s.P + s.n, 16 * (first + j0 + 64));
                for (int p = p0; p < p1; p += 64) {       // (uniform, for the shuffle)
                    const int at = p + lane, slot = __shfl(page, (at >> 4) - first - j0) * 16 + (at & 15);
                    const long long r = row0 + (at - s.P);
                    if (at < p1 && r < a.slot_cap) a.slots[r] = granted == 1 ? slot : -1;
                }
            }
            if (lane == 0) {
                a.granted[b] = granted;
                a.held_out[b] = granted == 1 ? s.held + s.need : a.held[b];
                a.row_start[b + 1] = saturate(row1);
            }
        }
        base_need += sum_need[m - 1];
        base_rows += sum_rows[m - 1];
    }
    const bool is_in = base_need <= a.n_free && base_rows <= a.slot_cap, last = b1 == a.batch;
    if (blockIdx.x == 0 && tid == 0) a.row_start[0] = 0;
    if (last)                                             // padding of the slot map
        for (long long r = base_rows + tid; r < a.slot_cap; r += 256) a.slots[r] = -1;
    if (!was_in || (is_in && !last)) return;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) taken = max(taken, __shfl_xor(taken, o));
    __syncthreads();
    if (lane == 0) sum_need[wave] = taken;
    __syncthreads();
    if (tid == 0) a.n_taken[0] = (int)max(max(sum_need[0], sum_need[1]), max(sum_need[2], sum_need[3]));
}

// ------------------------------------------------------------------ rows into 4-bit pages and back
// A lane takes eight elements (16 bytes of bf16), the four lanes of a block agree on its scale by two shuffles, and 16 rows of a
// head follow one another: of rows that are neighbours a workgroup holds whole pages, whose lines then go through one XCD's L2
// (16000 rows of 8 heads in bf16, us to store and to load: sixteen rows at a time 22.2 and 14.0, four 25.2 and 21.7; pages put together
// in LDS and written 16 bytes a lane cost the store 5 %).  Bound by the bytes of the rows.
struct RowArgs {
    Kv4View kv;
    const int32_t *slots;
    int n_rows;
    int vec;                  // rows can be read and written 16 bytes at a time
};
__device__ inline bool row_piece(const RowArgs &a, size_t idx, int &row, int &h, int &grp) {
    const int ng = 4 * kv4_blocks(a.kv.hd);
    grp = (int)(idx % ng);
    const size_t t = idx / ng;
    const int rr = (int)(t & 15);
    const size_t u = t >> 4;
    h = (int)(u % a.kv.n_kv);
    const size_t rb = u / a.kv.n_kv;
    row = (int)(rb * 16 + rr);
    return rb * 16 + rr < (size_t)a.n_rows;
}

template <typename T>
__device__ inline void load8(const T *src, int n, bool vec, float (&x)[8]) {
    if (vec) {
        if constexpr (sizeof(T) == 2) {
            const bf16x8 v = *(const bf16x8 *)src;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
        } else {
            const f32x4 v = *(const f32x4 *)src, w = *(const f32x4 *)(src + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = v[e];
                x[4 + e] = w[e];
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n ? (float)src[e] : 0.f;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void kv4_store_kernel(RowArgs a, const T *__restrict__ k, const T *__restrict__ v) {
    const int nb = kv4_blocks(a.kv.hd), hd = a.kv.hd;
    const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
    int row, h, grp;
    const bool here = row_piece(a, idx, row, h, grp);
    const int slot = here ? a.slots[row] : -1;
    float x[2][8] = {};
    const int n = hd - 8 * grp;                           // elements of this group that there are
    if (here && n > 0) {                                  // (whatever the slot: one trip to memory for all three)
        const size_t src = ((size_t)row * a.kv.n_kv + h) * hd + 8 * grp;
        load8(k + src, n, a.vec && n >= 8, x[0]);
        load8(v + src, n, a.vec && n >= 8, x[1]);
    }
    unsigned codes[2], byte[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        unsigned amax = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[i][e]) & 0x7fffffffu);
        amax = max(amax, (unsigned)__shfl_xor((int)amax, 1));
        amax = max(amax, (unsigned)__shfl_xor((int)amax, 2));
        byte[i] = kv4_scale_byte(amax);
        codes[i] = 0x77777777u;                           // of a block that reads back as NaN
        if (byte[i] != kScaleNan) {
            const float scale = kv4_scale(byte[i]);
            codes[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[i][0], x[i][1], scale, 0);
            codes[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes[i], x[i][2], x[i][3], scale, 1);
            codes[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes[i], x[i][4], x[i][5], scale, 2);
            codes[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes[i], x[i][6], x[i][7], scale, 3);
        }
    }
    if (slot < 0 || slot >= (long long)a.kv.n_pages * 16) return;
    unsigned char *blk = a.kv.pages + kv4_offset(a.kv, slot >> 4, h);
    const int t = slot & 15, b = grp >> 2;
    *(unsigned *)(blk + b * 256 + t * 16 + (grp & 3) * 4) = codes[0];
    *(unsigned *)(blk + kv4_v_codes(nb) + ((t >> 2) * 4 * nb + grp) * 16 + (t & 3) * 4) = codes[1];
    if ((grp & 3) == 0) {
        blk[kv4_k_scales(nb) + b * 16 + t] = (unsigned char)byte[0];
        blk[kv4_v_scales(nb) + b * 16 + t] = (unsigned char)byte[1];
    }
}

// ONCE: more than the L2s hold together, written past them (16000 rows of 8 heads in bf16: a load takes 14.0 us, a store and a load
// together 35.6; without it 15.8 and 44.6)
template <typename T, bool ONCE>
__global__ __launch_bounds__(256) void kv4_load_kernel(RowArgs a, T *__restrict__ k, T *__restrict__ v) {
    const int nb = kv4_blocks(a.kv.hd), hd = a.kv.hd;
    const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
    int row, h, grp;
    if (!row_piece(a, idx, row, h, grp)) return;
    const int n = hd - 8 * grp;
    if (n <= 0) return;
    const int slot = a.slots[row];
    const bool ok = slot >= 0 && slot < (long long)a.kv.n_pages * 16;
    unsigned words[2] = {0, 0}, bytes[2] = {0, 0};
    if (ok) {
        const unsigned char *blk = a.kv.pages + kv4_offset(a.kv, slot >> 4, h);
        const int t = slot & 15, b = grp >> 2;
        words[0] = *(const unsigned *)(blk + b * 256 + t * 16 + (grp & 3) * 4);
        words[1] = *(const unsigned *)(blk + kv4_v_codes(nb) + ((t >> 2) * 4 * nb + grp) * 16 + (t & 3) * 4);
        bytes[0] = blk[kv4_k_scales(nb) + b * 16 + t];
        bytes[1] = blk[kv4_v_scales(nb) + b * 16 + t];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float s = kv4_scale(bytes[i]);
        const kv4_f32x2 p0 = kv4_pair_f32<0>(words[i], s), p1 = kv4_pair_f32<1>(words[i], s), p2 = kv4_pair_f32<2>(words[i], s),
                        p3 = kv4_pair_f32<3>(words[i], s);
        float x[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = !ok ? 0.f : bytes[i] == kScaleNan ? __builtin_nanf("") : x[e];
        T *dst = (i ? v : k) + ((size_t)row * a.kv.n_kv + h) * hd + 8 * grp;
        if (a.vec && n >= 8) {
            if constexpr (sizeof(T) == 2) {
                bf16x8 o;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = (bf16_t)x[e];
                if constexpr (ONCE) __builtin_nontemporal_store(o, (bf16x8 *)dst);
                else *(bf16x8 *)dst = o;
            } else {
                *(f32x4 *)dst = (f32x4){x[0], x[1], x[2], x[3]};
                *(f32x4 *)(dst + 4) = (f32x4){x[4], x[5], x[6], x[7]};
            }
        } else {
            for (int e = 0; e < 8 && e < n; ++e) dst[e] = (T)x[e];
        }
    }
}

// ------------------------------------------------------------------ new rows of an attention call
// A workgroup takes the rows of one unit of 16 keys (a cache page of the causal rows, or a tile of mask rows) of one kv head:
// V is turned to [hd][16] through LDS, so that a whole unit is written in runs of 16 tokens (row by row every 2-byte store
// had a cache sector to itself).  VEC: rows are read 16 bytes at a time.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void span_place_kernel(const T *__restrict__ k_new, const T *__restrict__ v_new, int n_rows,
                                                         int mask_row0, const int32_t *__restrict__ prefix_len, RowDesc d,
                                                         KvView kv, int n_cache_units, int units, T *__restrict__ k_scr,
                                                         T *__restrict__ v_scr) {
    __shared__ T vt[16][128 + 2];
    const int unit = blockIdx.x % units, bh = blockIdx.x / units, b = bh / kv.n_kv, h = bh - b * kv.n_kv;
    const int hd = kv.hd, tid = threadIdx.x;
    int r0, s0, n;                                        // first row of the unit, its slot, and how many
    T *kd, *vd;
    if (unit < n_cache_units) {
        const int L = prefix_len[d.seq_base + b];
        if (!seq_fits(kv, L, d.nc)) return;
        const int u = (L >> 4) + unit, p0 = max(L, 16 * u), p1 = min(L + d.nc, 16 * u + 16);
        if (p1 <= p0) return;
        const int page = kv.page_table[(size_t)(d.seq_base + b) * kv.pages_per_seq + u];
        if (!page_ok(kv, page)) return;
        r0 = p0 - L;
        s0 = p0 & 15;
        n = p1 - p0;
        kd = (T *)kv.k_pages + k_page_offset(kv, page, h, 0, 0);
        vd = (T *)kv.v_pages + v_page_offset(kv, page, h, 0, 0);
    } else {
        const int mt = unit - n_cache_units, n_mt = (d.nm + 15) >> 4;
        r0 = mask_row0 + 16 * mt;
        s0 = 0;
        n = min(16, d.nm - 16 * mt);
        const size_t tile = (((size_t)b * kv.n_kv + h) * n_mt + mt) * 16 * hd;
        kd = k_scr + tile;
        vd = v_scr + tile;
    }
    const size_t src = (((size_t)b * n_rows + r0) * kv.n_kv + h) * hd, stride = (size_t)kv.n_kv * hd;
    constexpr int E = 16 / sizeof(T);                     // elements of a 16-byte piece
    typedef __attribute__((ext_vector_type(E))) T piece_t;
    if (VEC) {
        const int pieces = hd / E;
        for (int i = tid; i < n * pieces; i += 256) {
            const int r = i / pieces, e = (i - r * pieces) * E;
            *(piece_t *)(kd + (s0 + r) * hd + e) = *(const piece_t *)(k_new + src + r * stride + e);
            const piece_t x = *(const piece_t *)(v_new + src + r * stride + e);
#pragma unroll
            for (int j = 0; j < E; ++j) vt[s0 + r][e + j] = x[j];
        }
    } else {
        for (int i = tid; i < n * hd; i += 256) {
            const int r = i / hd, e = i - r * hd;
            kd[(s0 + r) * hd + e] = k_new[src + r * stride + e];
            vt[s0 + r][e] = v_new[src + r * stride + e];
        }
    }
    if (unit >= n_cache_units) {                          // behind the mask rows: zeros, the attention need not look closer
        for (int i = tid; i < (16 - n) * hd; i += 256) vt[n + i / hd][i % hd] = (T)0.f;
        n = 16;
    }
    __syncthreads();
    for (int i = tid; i < hd * (16 / E); i += 256) {      // a run of E tokens of one element
        const int e = i / (16 / E), s = (i - e * (16 / E)) * E;
        if (s >= s0 && s + E <= s0 + n) {
            piece_t x;
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = vt[s + j][e];
            *(piece_t *)(vd + e * 16 + s) = x;
        } else {
            for (int j = max(s, s0); j < min(s + E, s0 + n); ++j) vd[e * 16 + j] = vt[j][e];
        }
    }
}

}  // namespace

void launch_span_place(int dtype, const void *k_new, const void *v_new, int n_rows, int mask_row0, const int32_t *prefix_len,
                       const RowDesc &d, int B, KvView kv, void *k_scr, void *v_scr, hipStream_t st) {
    const int cache_units = kv.k_pages ? (d.nc + 15) / 16 + 1 : 0, units = cache_units + (d.nm + 15) / 16;
    if (units == 0) return;
    const int grid = units * kv.n_kv * B;
    const bool vec = kv.hd % (dtype == TIDAR_BF16 ? 8 : 4) == 0 && (((uintptr_t)k_new | (uintptr_t)v_new) & 15) == 0;
    auto go = [&](auto kernel, auto t) {
        typedef decltype(t) T;
        kernel<<<grid, 256, 0, st>>>((const T *)k_new, (const T *)v_new, n_rows, mask_row0, prefix_len, d, kv, cache_units, units,
                                     (T *)k_scr, (T *)v_scr);
    };
    if (dtype == TIDAR_BF16 && vec) go(span_place_kernel<bf16_t, true>, bf16_t());
    else if (dtype == TIDAR_BF16) go(span_place_kernel<bf16_t, false>, bf16_t());
    else if (vec) go(span_place_kernel<float, true>, float());
    else go(span_place_kernel<float, false>, float());
}

void launch_table_extend(int batch, const int32_t *prefix_len, const int32_t *n_new, const int32_t *held,
                         const int32_t *free_pages, int n_free, int32_t *page_table, int pages_per_seq, int n_pages,
                         int32_t *row_start, int32_t *slots, int slot_cap, int32_t *held_out, int32_t *granted,
                         int32_t *n_taken, hipStream_t st) {
    const int wgs = batch < 2048 ? (batch + 3) / 4 : 512;
    const int per_wg = (batch + wgs - 1) / wgs;
    const TableArgs a = {batch, prefix_len, n_new, held, free_pages, n_free, page_table, pages_per_seq, n_pages,
                         row_start, slots, slot_cap, held_out, granted, n_taken, per_wg};
    table_extend_kernel<<<(batch + per_wg - 1) / per_wg, 256, 0, st>>>(a);
}

// A launch has fewer than 2^32 threads: `launch` gets rows [r0, r0 + n) in runs of at most 2^31 lanes, whole units of 16 rows but the last.
template <class F>
static void for_row_runs(const Kv4View &kv, const int32_t *slots, int n_rows, const void *k, const void *v, size_t esize, F launch) {
    const size_t row_lanes = (size_t)kv.n_kv * 4 * kv4_blocks(kv.hd), row_bytes = (size_t)kv.n_kv * kv.hd * esize;
    const size_t run = std::max<size_t>(16, ((size_t)1 << 31) / row_lanes & ~(size_t)15);
    const int vec = kv.hd % 8 == 0 && (((uintptr_t)k | (uintptr_t)v) & 15) == 0;
    for (size_t r0 = 0; r0 < (size_t)n_rows; r0 += run) {
        const int n = (int)std::min<size_t>(run, n_rows - r0);
        const size_t lanes = ((size_t)n + 15) / 16 * 16 * row_lanes;
        launch(RowArgs{kv, slots + r0, n, vec}, dim3((unsigned)((lanes + 255) / 256)), r0 * row_bytes);
    }
}
void launch_kv4_store(int dtype, const Kv4View &kv, const int32_t *slots, int n_rows, const void *k, const void *v,
                      hipStream_t st) {
    auto go = [&](auto t) {
        typedef decltype(t) T;
        for_row_runs(kv, slots, n_rows, k, v, sizeof(T), [&](const RowArgs &a, dim3 grid, size_t at) {
            kv4_store_kernel<<<grid, 256, 0, st>>>(a, (const T *)((const char *)k + at), (const T *)((const char *)v + at));
        });
    };
    if (dtype == TIDAR_BF16) go(bf16_t());
    else go(float());
}
void launch_kv4_load(int dtype, const Kv4View &kv, const int32_t *slots, int n_rows, void *k, void *v, hipStream_t st) {
    const bool once = (size_t)n_rows * kv.n_kv * kv.hd * 4 > 32u << 20;
    auto go = [&](auto kernel, auto t) {
        typedef decltype(t) T;
        for_row_runs(kv, slots, n_rows, k, v, sizeof(T), [&](const RowArgs &a, dim3 grid, size_t at) {
            kernel<<<grid, 256, 0, st>>>(a, (T *)((char *)k + at), (T *)((char *)v + at));
        });
    };
    if (dtype == TIDAR_BF16 && once) go(kv4_load_kernel<bf16_t, true>, bf16_t());
    else if (dtype == TIDAR_BF16) go(kv4_load_kernel<bf16_t, false>, bf16_t());
    else go(kv4_load_kernel<float, false>, float());
}
