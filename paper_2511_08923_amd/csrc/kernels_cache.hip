// Kernels around the paged cache: page tables and slot maps from request lengths, rows of K and V into 4-bit pages and
// back, and the placement of a windowed attention's new rows.  All of them move bytes; what bounds each stands with it.
#include "kv4_format.h"
#include "tidar_internal.h"

namespace {

// ------------------------------------------------------------------ page tables and slot maps
// Sequence b holds P_b positions, has h_b pages and gets n_b rows more: it needs ceil((P_b + n_b) / 16) - h_b pages of the
// free list (or none), in the order of the sequences.  Where a sequence's pages begin in the list, and its rows in the
// slot map, is an exclusive sum over the sequences before it.  Every workgroup adds up its predecessors by itself, so the
// whole is one launch: up to 512 workgroups read 8 bytes of each predecessor from L2 (batch 2048: 12 MB in all), which is less than
// the second launch that a scan in two steps costs.  A wave then takes a sequence at a time.
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
__device__ inline bool fits(const TableArgs &a, long long off, int need, int rows, long long rows_end) {
    return (need == 0 || off + need <= a.n_free) && (rows == 0 || rows_end <= a.slot_cap);
}

__global__ __launch_bounds__(256) void table_extend_kernel(TableArgs a) {
    __shared__ long long sum_need[256], sum_rows[256];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b0 = blockIdx.x * a.per_wg, b1 = min(a.batch, b0 + a.per_wg);
    const bool last = b1 == a.batch;
    // sums over a range of sequences, in every thread
    auto total = [&](int lo, int hi, long long &need, long long &rows) {
        long long x = 0, y = 0;
        for (int b = lo + tid; b < hi; b += 256) {
            const SeqNeed s = seq_need(a, b);
            x += s.need;
            y += s.n;
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            x += __shfl_xor(x, o);
            y += __shfl_xor(y, o);
        }
        __syncthreads();
        if (lane == 0) {
            sum_need[wave] = x;
            sum_rows[wave] = y;
        }
        __syncthreads();
        need = sum_need[0] + sum_need[1] + sum_need[2] + sum_need[3];
        rows = sum_rows[0] + sum_rows[1] + sum_rows[2] + sum_rows[3];
        __syncthreads();
    };
    long long base_need, base_rows;
    total(0, b0, base_need, base_rows);
    long long taken = 0;
    for (int c0 = b0; c0 < b1; c0 += 256) {
        const int m = min(256, b1 - c0);
        // inclusive sums of this run of sequences
        SeqNeed mine = {};
        if (tid < m) mine = seq_need(a, c0 + tid);
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
        __syncthreads();
        for (int i = wave; i < m; i += 4) {
            const int b = c0 + i;
            const SeqNeed s = seq_need(a, b);
            const long long off = base_need + sum_need[i] - s.need;
            const long long row0 = base_rows + sum_rows[i] - s.n, row1 = row0 + s.n;
            int32_t *table = a.page_table + (size_t)b * a.pages_per_seq;
            const bool room = s.ok && fits(a, off, s.need, s.n, row1);
            // the pages that the new rows go into: those that the sequence has, and those from the list
            bool ids = true;
            const int first = s.P >> 4, own_end = min(s.held, (s.P + s.n + 15) >> 4);
            if (room && s.n > 0)
                for (int j = first + lane; j < own_end; j += 64) ids = ids && (unsigned)table[j] < (unsigned)a.n_pages;
            if (room)
                for (int j = lane; j < s.need; j += 64) ids = ids && (unsigned)a.free_pages[off + j] < (unsigned)a.n_pages;
            ids = __all(ids);
            const int granted = !s.ok ? -1 : !room ? 0 : ids ? 1 : -1;
            if (granted == 1)
                for (int j = lane; j < s.need; j += 64) table[s.held + j] = a.free_pages[off + j];
            for (long long r = row0 + lane; r < row1 && r < a.slot_cap; r += 64) {
                const int p = s.P + (int)(r - row0), lp = p >> 4;
                int slot = -1;
                if (granted == 1) slot = (lp < s.held ? table[lp] : a.free_pages[off + (lp - s.held)]) * 16 + (p & 15);
                a.slots[r] = slot;
            }
            if (lane == 0) {
                a.granted[b] = granted;
                a.held_out[b] = granted == 1 ? s.held + s.need : a.held[b];
                a.row_start[b + 1] = saturate(row1);
            }
        }
        // what the list has lost: the furthest end of a valid sequence that it had room for
        if (tid < m && mine.need > 0 && fits(a, base_need + x - mine.need, mine.need, mine.n, base_rows + y)) {
            const long long end = base_need + x;
            taken = end > taken ? end : taken;
        }
        const long long n_need = sum_need[m - 1], n_rows = sum_rows[m - 1];
        __syncthreads();
        base_need += n_need;
        base_rows += n_rows;
    }
    if (blockIdx.x == 0 && tid == 0) a.row_start[0] = 0;
    if (!last) return;
    for (long long r = base_rows + tid; r < a.slot_cap; r += 256) a.slots[r] = -1;       // padding of the slot map
    // n_taken needs every sequence: ends only grow, so the largest that fits is found by one more pass over those before
    long long run_need = 0, run_rows = 0;
    for (int c0 = 0; c0 < b0; c0 += 256) {
        const int m = min(256, b0 - c0);
        SeqNeed mine = {};
        if (tid < m) mine = seq_need(a, c0 + tid);
        long long x = mine.need, y = mine.n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long px = __shfl_up(x, o), py = __shfl_up(y, o);
            if (lane >= o) {
                x += px;
                y += py;
            }
        }
        __syncthreads();
        if (lane == 63) {
            sum_need[wave] = x;
            sum_rows[wave] = y;
        }
        __syncthreads();
        long long all_need = 0, all_rows = 0;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) {
                x += sum_need[w];
                y += sum_rows[w];
            }
            all_need += sum_need[w];
            all_rows += sum_rows[w];
        }
        if (tid < m && mine.need > 0 && fits(a, run_need + x - mine.need, mine.need, mine.n, run_rows + y)) {
            const long long end = run_need + x;
            taken = end > taken ? end : taken;
        }
        run_need += all_need;
        run_rows += all_rows;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long t = __shfl_xor(taken, o);
        taken = t > taken ? t : taken;
    }
    __syncthreads();
    if (lane == 0) sum_need[wave] = taken;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < 4; ++w) taken = sum_need[w] > taken ? sum_need[w] : taken;
        a.n_taken[0] = (int)taken;
    }
}

// ------------------------------------------------------------------ rows into 4-bit pages and back
// A lane takes eight elements (16 bytes of bf16), the four lanes of a block agree on its scale by two shuffles, and a wave
// takes four rows of a head at head_dim 128: its stores into V's token quads are then whole runs of 16 bytes where the rows
// are neighbours.  Bound by the bytes of the rows.
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
    const int rr = (int)(t & 3);
    const size_t u = t >> 2;
    h = (int)(u % a.kv.n_kv);
    const size_t rb = u / a.kv.n_kv;
    row = (int)(rb * 4 + rr);
    return rb * 4 + rr < (size_t)a.n_rows;
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
    const bool ok = slot >= 0 && slot < (long long)a.kv.n_pages * 16;
    const T *src = blockIdx.y ? v : k;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int n = hd - 8 * grp;                           // elements of this group that there are
    if (ok && n > 0) load8(src + ((size_t)row * a.kv.n_kv + h) * hd + 8 * grp, n, a.vec && n >= 8, x);
    unsigned amax = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[e]) & 0x7fffffffu);
    amax = max(amax, (unsigned)__shfl_xor((int)amax, 1));
    amax = max(amax, (unsigned)__shfl_xor((int)amax, 2));
    if (!ok) return;
    const unsigned byte = kv4_scale_byte(amax);
    unsigned codes = 0x77777777u;                         // of a block that reads back as NaN
    if (byte != kScaleNan) {
        const float scale = kv4_scale(byte);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
    }
    unsigned char *blk = a.kv.pages + kv4_offset(a.kv, slot >> 4, h);
    const int t = slot & 15, b = grp >> 2;
    if (blockIdx.y == 0) {
        *(unsigned *)(blk + b * 256 + t * 16 + (grp & 3) * 4) = codes;
        if ((grp & 3) == 0) blk[kv4_k_scales(nb) + b * 16 + t] = (unsigned char)byte;
    } else {
        *(unsigned *)(blk + kv4_v_codes(nb) + ((t >> 2) * 4 * nb + grp) * 16 + (t & 3) * 4) = codes;
        if ((grp & 3) == 0) blk[kv4_v_scales(nb) + b * 16 + t] = (unsigned char)byte;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void kv4_load_kernel(RowArgs a, T *__restrict__ k, T *__restrict__ v) {
    const int nb = kv4_blocks(a.kv.hd), hd = a.kv.hd;
    const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
    int row, h, grp;
    if (!row_piece(a, idx, row, h, grp)) return;
    const int n = hd - 8 * grp;
    if (n <= 0) return;
    const int slot = a.slots[row];
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (slot >= 0 && slot < (long long)a.kv.n_pages * 16) {
        const unsigned char *blk = a.kv.pages + kv4_offset(a.kv, slot >> 4, h);
        const int t = slot & 15, b = grp >> 2;
        const unsigned word = blockIdx.y ? *(const unsigned *)(blk + kv4_v_codes(nb) + ((t >> 2) * 4 * nb + grp) * 16 + (t & 3) * 4)
                                         : *(const unsigned *)(blk + b * 256 + t * 16 + (grp & 3) * 4);
        const unsigned byte = blk[(blockIdx.y ? kv4_v_scales(nb) : kv4_k_scales(nb)) + b * 16 + t];
        const float s = kv4_scale(byte);
        const kv4_f32x2 p0 = kv4_pair_f32<0>(word, s), p1 = kv4_pair_f32<1>(word, s), p2 = kv4_pair_f32<2>(word, s),
                        p3 = kv4_pair_f32<3>(word, s);
        const float y[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = byte == kScaleNan ? __builtin_nanf("") : y[e];
    }
    T *dst = (blockIdx.y ? v : k) + ((size_t)row * a.kv.n_kv + h) * hd + 8 * grp;
    if (a.vec && n >= 8) {
        if constexpr (sizeof(T) == 2) {
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (bf16_t)x[e];
            *(bf16x8 *)dst = o;
        } else {
            *(f32x4 *)dst = (f32x4){x[0], x[1], x[2], x[3]};
            *(f32x4 *)(dst + 4) = (f32x4){x[4], x[5], x[6], x[7]};
        }
    } else {
        for (int e = 0; e < 8 && e < n; ++e) dst[e] = (T)x[e];
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

static RowArgs row_args(const Kv4View &kv, const int32_t *slots, int n_rows, const void *k, const void *v) {
    return {kv, slots, n_rows, kv.hd % 8 == 0 && (((uintptr_t)k | (uintptr_t)v) & 15) == 0};
}
static dim3 row_grid(const Kv4View &kv, int n_rows) {
    const size_t lanes = (size_t)((n_rows + 3) / 4) * 4 * kv.n_kv * 4 * kv4_blocks(kv.hd);
    return dim3((unsigned)((lanes + 255) / 256), 2);
}
void launch_kv4_store(int dtype, const Kv4View &kv, const int32_t *slots, int n_rows, const void *k, const void *v,
                      hipStream_t st) {
    const RowArgs a = row_args(kv, slots, n_rows, k, v);
    if (dtype == TIDAR_BF16) kv4_store_kernel<<<row_grid(kv, n_rows), 256, 0, st>>>(a, (const bf16_t *)k, (const bf16_t *)v);
    else kv4_store_kernel<<<row_grid(kv, n_rows), 256, 0, st>>>(a, (const float *)k, (const float *)v);
}
void launch_kv4_load(int dtype, const Kv4View &kv, const int32_t *slots, int n_rows, void *k, void *v, hipStream_t st) {
    const RowArgs a = row_args(kv, slots, n_rows, k, v);
    if (dtype == TIDAR_BF16) kv4_load_kernel<<<row_grid(kv, n_rows), 256, 0, st>>>(a, (bf16_t *)k, (bf16_t *)v);
    else kv4_load_kernel<<<row_grid(kv, n_rows), 256, 0, st>>>(a, (float *)k, (float *)v);
}
