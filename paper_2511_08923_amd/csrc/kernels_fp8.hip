// Matrix products in 8-bit floating point: rows into e4m3 blocks of 128 with a power of two each (fp8_format.h), and the product
// of two such operands.
#include <algorithm>
#include <type_traits>

#include "fp8_format.h"
#include "gemm_device.h"
#include "lds_dma.h"

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

// ------------------------------------------------------------------ rows into blocks
// s = 2^e with the least e for which the block's largest magnitude is at most 448 * 2^e; an element is x / s (exact: a power of two), rounded once,
// to the nearest of e4m3, ties to even.
// Eight lanes to a block, 16 elements each; a wave takes eight rows of one block, so that its stores are runs of 128 bytes.  Bound by memory
// for weights (24576 x 4096: 54.5 us, 5.6 TB/s), by the launch and one trip to memory for a step's rows (272 x 12288: 3.5 us).
struct PackArgs {
    int rows, K, tiles, tile_off, tile_stride;            // tiles: of the destination, where tile t of the source is tile tile_off + t * tile_stride
    unsigned char *codes;
    unsigned *scales;
};
// 16 elements from k0 on of a row (zeros from K on) as codes, with the largest magnitude of the block over eight lanes.
template <typename T>
__device__ inline i32x4 fp8_convert16(const T *__restrict__ row, int k0, int K, unsigned &byte) {
    float x[16];
    unsigned amax = 0;
    if (k0 < K) {                                         // K is a multiple of 16
#pragma unroll
        for (int j = 0; j < 16; j += 16 / sizeof(T)) {
            typedef __attribute__((ext_vector_type(16 / sizeof(T)))) T piece_t;
            const piece_t v = *(const piece_t *)(row + k0 + j);
#pragma unroll
            for (int e = 0; e < (int)(16 / sizeof(T)); ++e) x[j + e] = (float)v[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) amax = max(amax, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) amax = max(amax, (unsigned)__shfl_xor((int)amax, o));
    const unsigned b = fp8_scale_byte(amax);
    const float inv = __uint_as_float((254u - min(b, 247u)) << 23);      // 2^-(b - 127), exact
    i32x4 code;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w] * inv, x[4 * w + 1] * inv, 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w + 2] * inv, x[4 * w + 3] * inv, c, true);
        code[w] = b == 255u ? 0x7f7f7f7f : c;
    }
    byte = b == 255u ? 127u : b;
    return code;
}

template <typename T>
__global__ __launch_bounds__(256) void fp8_pack_kernel(PackArgs a, const T *__restrict__ src) {
    const int tid = threadIdx.x, p = tid & 7, r16 = (tid >> 3) & 15, nb = fp8_blocks(a.K), pairs = (nb + 1) / 2;
    const int t = blockIdx.x / pairs, kb = 2 * (blockIdx.x - t * pairs) + (tid >> 7), row = 16 * t + r16;
    if (kb >= nb || row >= a.rows) return;                // (all eight lanes of a block)
    unsigned byte;
    const i32x4 code = fp8_convert16(src + (size_t)row * a.K, 128 * kb + 16 * p, a.K, byte);
    const size_t tile = (size_t)a.tile_off + (size_t)t * a.tile_stride;
    *(i32x4 *)(a.codes + (((size_t)2 * kb + (p >> 2)) * a.tiles + tile) * 1024 + (p & 3) * 256 + r16 * 16) = code;
    if (p == 0) ((unsigned char *)(a.scales + ((size_t)(kb >> 2) * a.tiles + tile) * 16 + r16))[kb & 3] = (unsigned char)byte;
}

// ------------------------------------------------------------------ the product
struct Gemm8Args {
    const unsigned char *a, *w;                           // codes
    const unsigned *as, *ws;                              // scales
    void *out;
    int M, N, K, a_tiles, w_tiles, nb;
    int bf16_out;
};

__device__ inline i32x8 join16(i32x4 x, i32x4 y) { return (i32x8){x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]}; }

// Four values of one row, columns n .. n + 3 (N is a multiple of 16).
__device__ inline void store4(const Gemm8Args &g, int m, int n, f32x4 v) {
    if (m >= g.M || n >= g.N) return;
    const size_t at = (size_t)m * g.N + n;
    if (g.bf16_out) *(bf16x4 *)((bf16_t *)g.out + at) = (bf16x4){(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
    else *(f32x4 *)((float *)g.out + at) = v;
}

// Few rows: a workgroup takes a tile of 16 columns and MT of 16 rows, its W waves take turns with the blocks of K, operands straight from
// memory into registers; the waves' sums are folded through LDS.  Bound by HBM for up to 16 rows (1 x 24576 x 4096: 20 us, 5.0 TB/s), beyond
// by what a compute unit takes in, every workgroup reading all rows (52 GB/s per unit).
// SRC: void, or the type of the rows as the caller has them (MT 1): every workgroup then brings them into 8 bits by itself, in LDS, while
// its first weights, four blocks to a wave, are on their way, and there is no other launch (1 x 6144 x 4096 in two launches 9.0 us, so 6.7; with
// rows in 8 bits already registers for loads ahead cost more waves than they gain: 16 rows 9.0 -> 10.1).
template <int MT, int W, class SRC>
__global__ __launch_bounds__(64 * W, 6) void gemm8_few_kernel(Gemm8Args g, const SRC *__restrict__ src) {
    constexpr bool OWN = !std::is_void<SRC>::value;
    constexpr int DEPTH = 4;
    extern __shared__ __attribute__((aligned(16))) unsigned char few_smem[];         // OWN: codes [block][half, quarter][row][16], then scales
    __shared__ f32x4 red[W][MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wt = blockIdx.x, at0 = blockIdx.y * MT;
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    auto tile = [&](const unsigned char *p, const unsigned *s, int tiles, int t, int kb, i32x8 &x, int &sc) __attribute__((always_inline)) {
        const unsigned char *at = p + ((size_t)2 * kb * tiles + t) * 1024 + lane * 16;
        x = join16(*(const i32x4 *)at, *(const i32x4 *)(at + (size_t)tiles * 1024));
        sc = ((const unsigned char *)(s + ((size_t)(kb >> 2) * tiles + t) * 16 + (lane & 15)))[kb & 3];
    };
    if constexpr (OWN) {
        i32x8 wf[DEPTH];
        int wsc[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) tile(g.w, g.ws, g.w_tiles, wt, min(wave + d * W, g.nb - 1), wf[d], wsc[d]);
        unsigned char *scales = few_smem + (size_t)g.nb * g.M * 128;
        for (int i = threadIdx.x; i < g.M * g.nb * 8; i += 64 * W) {
            const int p = i & 7, r = (i >> 3) / g.nb, kb = (i >> 3) - r * g.nb;
            unsigned byte;
            const i32x4 code = fp8_convert16(src + (size_t)r * g.K, 128 * kb + 16 * p, g.K, byte);
            *(i32x4 *)(few_smem + ((kb * 8 + p) * g.M + r) * 16) = code;
            if (p == 0) scales[kb * g.M + r] = (unsigned char)byte;
        }
        __syncthreads();
        const int r = min(lane & 15, g.M - 1);
        for (int kb0 = wave; kb0 < g.nb; kb0 += DEPTH * W)
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int kb = kb0 + d * W;
                if (kb >= g.nb) break;
                const unsigned char *at = few_smem + ((kb * 8 + (lane >> 4)) * g.M + r) * 16;
                const i32x8 af = join16(*(const i32x4 *)at, *(const i32x4 *)(at + 64 * g.M));
                acc[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[d], af, acc[0], 0, 0, 0, wsc[d], 0, scales[kb * g.M + r]);
                if (kb0 + DEPTH * W < g.nb) tile(g.w, g.ws, g.w_tiles, wt, min(kb + DEPTH * W, g.nb - 1), wf[d], wsc[d]);
            }
    } else {
        for (int kb = wave; kb < g.nb; kb += W) {
            i32x8 wf, af[MT];
            int wsc, asc[MT];
            tile(g.w, g.ws, g.w_tiles, wt, kb, wf, wsc);
#pragma unroll
            for (int i = 0; i < MT; ++i) tile(g.a, g.as, g.a_tiles, min(at0 + i, g.a_tiles - 1), kb, af[i], asc[i]);     // (not there: the last again)
#pragma unroll
            for (int i = 0; i < MT; ++i)
                acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, af[i], acc[i], 0, 0, 0, wsc, 0, asc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) red[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MT; i += W) {
        f32x4 v = red[0][i][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) v += red[w][i][lane];
        store4(g, (at0 + i) * 16 + (lane & 15), wt * 16 + 4 * (lane >> 4), v);
    }
}

// Many rows: a workgroup of four waves, two by two, takes a tile of up to 256 rows and 64 CA columns, a wave RA x CA tiles of 32 x 32.  Both
// operands go from memory straight into LDS in chunks of 64 k, four of them on their way or in use; what the next chunk's MFMAs need is
// read, and the loads of the chunk after the next three go out, between this chunk's MFMAs.
// out[m][n] = sum over blocks of K of 2^(ea + ew) (codes . codes): the MFMA takes both powers of two, so a block costs no instruction of its own.
// 256 x 256 to a workgroup: 512 bytes from LDS for 131072 operations of a k, and 16 MFMAs of 64 clocks to each barrier; one wave to a
// SIMD, since the sums take 256 registers (four registers are spilled around the loop, none in it).  Conversion of the rows and all, in captured
// calls: 2064 x 24576 x 4096 179 us, 2.3 PFLOP/s, 8192^3 414 us, 2.66 (under a trace the kernel takes 436 by itself, at best 387).  Bound by the
// matrix cores at the clock they then run at (58 % busy at 1.9 to 2.0 GHz and 77 % at 1.82) and, with short K,
// by a workgroup's first loads and last stores, 2.3 and 6 us, which nothing else fills.
// RA: row tiles of a wave in the first n_tall passes over the rows; the others, n_short, have one less (the workgroups of a launch are
// started in order: short ones last fill up what the others leave).
constexpr int BUFS = 4;
constexpr int early(int loads) { return (3 * loads + 3) / 4; }           // of a chunk's loads, those that go out before the next chunk begins
template <int RA, int CA>
constexpr int tile_slot() { return (4 * RA + 4 * CA + 3) * 1024; }       // A tiles, W tiles, scales of A and of W, and what nobody reads

template <int RA, int CA>
__global__ __launch_bounds__(256) void gemm8_tile_kernel(Gemm8Args g, int splits, int per_split, int n_tall, int n_short, int n_colblk,
                                                         float *__restrict__ part) {
    constexpr int TILES = RA + CA, SLOT = tile_slot<RA, CA>();           // loads of a wave and chunk, but for the scales
    extern __shared__ __attribute__((aligned(16))) unsigned char smem8[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mh = wave >> 1, nh = wave & 1;
    // Workgroup i of a launch runs on XCD i % 8: each XCD takes one contiguous eighth of the (row pass, column block) plane, four
    // column blocks wide and passes downwards, so that what runs on it together shares rows and columns through its L2.
    const bool tall = (int)blockIdx.x < n_tall * n_colblk;
    int bx, bz;
    {
        const int n_pass = tall ? n_tall : n_short, n_wg = n_pass * n_colblk, l = blockIdx.x - (tall ? 0 : n_tall * n_colblk);
        const int q = n_wg >> 3, r = n_wg & 7, x = l & 7, i = x * q + min(x, r) + (l >> 3), band = 4 * n_pass;
        const int p = i / band, o = i - p * band, wd = min(4, n_colblk - 4 * p);
        bz = __builtin_amdgcn_readfirstlane(o / wd);     // (divisions are done in vector registers)
        bx = __builtin_amdgcn_readfirstlane(4 * p + o - bz * wd);
    }
    const int ra = tall ? RA : RA - 1, at0 = 4 * (tall ? bz * RA : n_tall * RA + bz * (RA - 1)), wt0 = bx * 4 * CA;        // first tiles of 16
    const int kb0 = blockIdx.y * per_split, kb1 = min(g.nb, kb0 + per_split), n_chunks = 2 * max(0, kb1 - kb0);

    // loads of a chunk: wave w brings A tiles w RA .. and W tiles w CA .., of every other chunk waves 0 and 1 the scales too (of four blocks each
    // time; the other waves ask for nothing, so that all have as many loads in flight).  One wave to a SIMD issues an instruction
    // every eight clocks or so, and what it issues besides the MFMAs is what bounds the loop: the loads of an operand share their addresses, and
    // nothing is masked but what runs past the end of the workgroup's K (tiles that are not there hold another row's codes, or zeros
    // at the end of the operand, and are never stored).
    const int lane16 = lane * 16, a_step = g.a_tiles * 1024, w_step = g.w_tiles * 1024;
    struct Run {                                         // a run of tiles, and the bytes to the end of the workgroup's K
        unsigned long long at;
        int left;
    };
    auto run_of = [&](const unsigned char *p, int step, int first) {
        return Run{(unsigned long long)(p + (size_t)2 * kb0 * step + (size_t)first * 1024), max(0, n_chunks * step - first * 1024)};
    };
    Run ra_run = run_of(g.a, a_step, at0 + wave * RA), w_run = run_of(g.w, w_step, wt0 + wave * CA);
    const unsigned long long s_at = (unsigned long long)(wave == 0 ? g.as : g.ws);
    auto desc = [&](unsigned long long at, int bytes) __attribute__((always_inline)) {
        return (int4v){(int)(unsigned)at, (int)((unsigned)(at >> 32) & 0xffff), bytes, 0x00020000};
    };
    const int s_step = (wave == 0 ? g.a_tiles : g.w_tiles) * 64, s_first = (wave == 0 ? at0 : wt0) * 64, s_end = wave > 1 ? 0 : ((g.nb + 3) >> 2) * s_step;
    const unsigned lds0 = lds_address(smem8), a_dst = lds0 + wave * RA * 1024, w_dst = lds0 + (4 * RA + wave * CA) * 1024,
                   s_dst = lds0 + (4 * RA + 4 * CA + min(wave, 2)) * 1024;
    auto advance = [&](Run &r, int step) __attribute__((always_inline)) {        // to the next chunk
        r.at += (unsigned)step;
        r.left = max(0, r.left - step);
        asm("" : "+s"(r.at), "+s"(r.left));              // (these stay in scalar registers)
    };
    // load i of chunk c: W tiles, A tiles, scales
    auto load = [&](int c, int i) __attribute__((always_inline)) {
        const unsigned slot = (c & (BUFS - 1)) * SLOT;
        if (i < CA) {
            dma16_run(w_dst + slot, lane16, desc(w_run.at, w_run.left), i);
            if (i == CA - 1) advance(w_run, w_step);
        } else if (i < CA + RA) {
            dma16_run(a_dst + slot, lane16, desc(ra_run.at, ra_run.left), i - CA);
            if (i == CA + RA - 1) advance(ra_run, a_step);
        } else {
            const int kb = kb0 + (c >> 1), at = (kb >> 2) * s_step + s_first;
            dma16_run(s_dst + slot, lane16, desc(s_at + (unsigned)at, kb < kb1 ? max(0, s_end - at) : 0), 0);
        }
    };

    f32x16 acc[RA][CA];
#pragma unroll
    for (int i = 0; i < RA; ++i)
#pragma unroll
        for (int j = 0; j < CA; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    i32x8 wf[2][CA], af[2][RA];
    int sc[CA + RA], sc_next[CA + RA];                   // scales of this block of 128 and the next, W first
    // lane (row, g) of a 32 x 32 x 64 operand: quarters g and 2 + g of its row
    const unsigned char *frag0 = smem8 + ((lane >> 4) & 1) * 1024 + (lane >> 5) * 256 + (lane & 15) * 16;
    auto k_loop = [&](auto ra_tag) __attribute__((always_inline)) {
        constexpr int RH = decltype(ra_tag)::value, N = RH * CA, FRAGS = CA + RH, FREE = RH > 1 ? CA : 1;
        static_assert(N > FREE, "no place for the reads");
        const unsigned char *a0 = frag0 + mh * 2 * RH * 1024, *w0 = frag0 + (4 * RA + nh * 2 * CA) * 1024;
        const unsigned char *as0 = smem8 + (4 * RA + 4 * CA) * 1024 + (mh * RH * 32 + (lane & 31)) * 4;
        const unsigned char *ws0 = smem8 + (4 * RA + 4 * CA + 1) * 1024 + (nh * CA * 32 + (lane & 31)) * 4;
        // read r of chunk c's 2 (CA + RH) halves of fragments, W first, then (even chunks) of its CA + RH scales
        auto read = [&](int s, int c, int r) __attribute__((always_inline)) {
            const int at = (c & (BUFS - 1)) * SLOT;
            if (r >= 2 * FRAGS) {
                const int f = r - 2 * FRAGS, byte = (kb0 + (c >> 1)) & 3;
                if (f < CA) sc_next[f] = ws0[at + f * 128 + byte];
                else sc_next[f] = as0[at + (f - CA) * 128 + byte];
                return;
            }
            const int f = r >> 1, k = r & 1;
            const i32x4 x = *(const i32x4 *)((f < CA ? w0 + f * 2048 : a0 + (f - CA) * 2048) + at + k * 512);
#pragma unroll
            for (int e = 0; e < 4; ++e) (f < CA ? wf[s][f < CA ? f : 0] : af[s][f < CA ? 0 : f - CA])[4 * k + e] = x[e];
        };
        auto next_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int f = 0; f < FRAGS; ++f) {
                sc[f] = sc_next[f];
                asm("" : "+v"(sc[f]));                   // (a word: taken for a byte across the loop, it is widened again in every pass)
            }
        };
        // Chunk c with fragment set s = c % 2.  The loads of chunk c + BUFS - 1 (whose place chunk c - 1 left) go out between the first
        // MFMAs, as far as they have not before; then chunk c + 1 has to have landed for everyone; then come the reads of its fragments, and the
        // first loads of chunk c + BUFS.  Spread evenly: four waves that ask at the same time wait for each other.
        auto chunk = [&](auto s_tag, int c) __attribute__((always_inline)) {
            constexpr int s = decltype(s_tag)::value, READS = 2 * FRAGS + (s ? FRAGS : 0);
            constexpr int LOADS = TILES + 1 - s, FIRST = early(LOADS), BEFORE = TILES + s, REST = BEFORE - early(BEFORE);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int i = n / CA, j = n - i * CA;
                __builtin_amdgcn_sched_barrier(0);
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[s][j], af[s][i], acc[i][j], 0, 0, 0, sc[j], 0, sc[CA + i]);
                __builtin_amdgcn_sched_barrier(0);
                if (n < FREE) {
#pragma unroll
                    for (int k = REST * n / FREE; k < REST * (n + 1) / FREE; ++k) load(c - 1 + BUFS, BEFORE - REST + k);
                    if (n + 1 < FREE) continue;
                    wait_loads<2 * TILES + 1>();         // those of chunks c + 2 and c + 3
                    lds_barrier_counted();
                    continue;
                }
                const int x = n - FREE;
#pragma unroll
                for (int k = READS * x / (N - FREE); k < READS * (x + 1) / (N - FREE); ++k) read(s ^ 1, c + 1, k);
#pragma unroll
                for (int k = FIRST * x / (N - FREE); k < FIRST * (x + 1) / (N - FREE); ++k) load(c + BUFS, k);
            }
            if constexpr (s == 1) next_scales();
        };
#pragma unroll
        for (int r = 0; r < 3 * FRAGS; ++r) read(0, 0, r);
        next_scales();
        for (int c = 0; c < n_chunks; c += 2) {
            chunk(std::integral_constant<int, 0>(), c);
            chunk(std::integral_constant<int, 1>(), c + 1);
        }
    };
#pragma unroll
    for (int c = 0; c < BUFS; ++c)
#pragma unroll
        for (int i = 0; i < (c < BUFS - 1 ? TILES + 1 - (c & 1) : early(TILES)); ++i) load(c, i);
    wait_loads<TILES + TILES + 1 + early(TILES)>();      // chunk 0 has landed
    lds_barrier_counted();
    if (RA == 1 || ra == RA) k_loop(std::integral_constant<int, RA>());
    else if constexpr (RA > 1) k_loop(std::integral_constant<int, RA - 1>());
    wait_loads<0>();
    lds_barrier_counted();

    // ---- results: a lane holds row `lane % 32` of a tile, columns 8 e + 4 (lane / 32) + 0 .. 3.  They are turned through LDS, 32 rows at
    // a time, so that whole runs of a row are stored; past the L2s, which all workgroups of a round fill at once (4096^3 67.9 -> 64.8 us)
    auto store = [&](auto t, auto *out) __attribute__((always_inline)) {
        typedef decltype(t) T;
        typedef __attribute__((ext_vector_type(4))) T T4;
        constexpr int ROW = 32 * CA * sizeof(T), STRIDE = ROW + 16, PIECES = ROW / 16, E = 16 / sizeof(T);
        unsigned char *mine = smem8 + wave * 32 * STRIDE;
        const int n0 = wt0 * 16 + nh * CA * 32;
#pragma unroll
        for (int i = 0; i < RA; ++i) {
            if (i >= ra) break;
            const int m0 = at0 * 16 + (mh * ra + i) * 32;
#pragma unroll
            for (int j = 0; j < CA; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *(T4 *)(mine + (lane & 31) * STRIDE + (32 * j + 8 * e + 4 * (lane >> 5)) * sizeof(T)) =
                        (T4){(T)acc[i][j][4 * e], (T)acc[i][j][4 * e + 1], (T)acc[i][j][4 * e + 2], (T)acc[i][j][4 * e + 3]};
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int x = 0; x < 32 * PIECES / 64; ++x) {
                const int idx = x * 64 + lane, r = idx / PIECES, p = idx - r * PIECES;
                const i32x4 v = *(const i32x4 *)(mine + r * STRIDE + p * 16);
                if (m0 + r < g.M && n0 + p * E < g.N) __builtin_nontemporal_store(v, (i32x4 *)(out + (size_t)(m0 + r) * g.N + n0 + p * E));
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    };
    if (splits > 1) store(0.f, part + (size_t)blockIdx.y * g.M * g.N);
    else if (g.bf16_out) store((bf16_t)0.f, (bf16_t *)g.out);
    else store(0.f, (float *)g.out);
}

// out = sum of the splits' partial sums, in their order
template <typename T>
__global__ __launch_bounds__(256) void gemm8_sum_kernel(const float *__restrict__ part, int splits, size_t n, T *__restrict__ out) {
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;       // n is a multiple of 16
    if (i >= n) return;
    f32x4 v = *(const f32x4 *)(part + i);
    for (int s = 1; s < splits; ++s) v += *(const f32x4 *)(part + s * n + i);
    if constexpr (sizeof(T) == 2) *(bf16x4 *)(out + i) = (bf16x4){(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
    else *(f32x4 *)(out + i) = v;
}

template <int RA, int CA>
void launch_tile(const Gemm8Args &g, const Gemm8Plan &p, float *part, hipStream_t st) {
    constexpr int SMEM = std::max(BUFS * tile_slot<RA, CA>(), 4 * 32 * (32 * CA * 4 + 16));      // the ring, then the waves' results
    static std::atomic<bool> granted[kLdsDevices];
    grant_lds((const void *)gemm8_tile_kernel<RA, CA>, SMEM, granted);
    const int n_colblk = (g.w_tiles + 4 * CA - 1) / (4 * CA);
    gemm8_tile_kernel<RA, CA><<<dim3((p.tall + p.shorts) * n_colblk, p.splits), 256, SMEM, st>>>(g, p.splits, p.per, p.tall, p.shorts, n_colblk, part);
}

}  // namespace

// Estimated time of the many-row kernel, us, but for partial sums: its workgroups in rounds on 256 compute units (the last one, where units stand
// idle, counts half of that: the others' clock rises).  us of a chunk of 64 k, measured with every unit busy: wave
// tiles of 32 rows 1, 2, 3, 4 by two of 32 columns .22, .33, .40, .46, by four .42, .47, .58, .69.
static double tile_wg_time(int ra, int ca, int per, int splits) {          // of a workgroup
    static const double chunk_us[2][4] = {{0.22, 0.33, 0.40, 0.46}, {0.42, 0.47, 0.58, 0.69}};
    return 2.5 + 2 * per * chunk_us[ca / 4][ra - 1] + 0.35 * ra * ca * (splits > 1 ? 2 : 1);
}
static double tile_time(const Gemm8Plan &p, int colblk) {
    auto wg = [&](int r) { return tile_wg_time(r, p.ca, p.per, p.splits); };
    const long long nt = (long long)p.tall * colblk * p.splits, ns = (long long)p.shorts * colblk * p.splits;
    const double T = wg(p.ra), S = ns ? wg(p.ra - 1) : 0.0;
    // the tall ones in rounds, the short ones where there is room first
    double at[2] = {(double)(nt / 256) * T, (double)(nt / 256 + 1) * T};
    const long long n[2] = {256 - nt % 256, nt % 256};
    double end = n[1] ? at[1] : at[0];
    for (long long left = ns; left > 0;) {
        const int k = n[1] == 0 || at[0] <= at[1] ? 0 : 1;
        at[k] += S;
        left -= n[k];
        end = std::max(end, at[k]);
    }
    return 0.5 * (end + std::max(T, (nt * T + ns * S) / 256.0));
}
static double part_time(int M, int N, int splits) { return 4.0 + (double)M * N * 4 * splits / 4.5e6; }      // partial sums, out and back

static int few_tiles(int M) { return M <= 16 ? 1 : M <= 32 ? 2 : 4; }     // row tiles of a workgroup of few rows

// The plans that there are for rows in `units` of 64, first that of few rows: what a compute unit takes in, at 52 GB/s, or the weights at 5
// TB/s.  us with few and with many rows' kernel, conversion and all:
// 64 x 6144 x 4096 13.3, 14.3;  64 x 24576 x 4096 42, 26.8;  64 x 4096 x 12288 23.1, 19.0;  32 x 6144 x 4096 9.8, 13.5;  32 x 24576 x 4096 29, 26.2
struct Gemm8Plans {
    int N, nb, n;
    Gemm8Plan plan[2 * 4 * 12];
    double us[2 * 4 * 12];
    Gemm8Plans(int units, int N, int nb) : N(N), nb(nb), n(0) {
        for (int ca = 2; ca <= 4; ca += 2)
            for (int ra = 1; ra <= 4 && ra <= units; ++ra) {
                Gemm8Plan q = {};
                const int passes = (units + ra - 1) / ra, colblk = (N + 64 * ca - 1) / (64 * ca);
                q.ra = ra;
                q.ca = ca;
                q.tall = units - passes * (ra - 1);       // as even as they go
                q.shorts = passes - q.tall;
                if (q.tall <= 0) continue;
                for (const int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
                    if (s > nb) break;
                    q.per = (nb + s - 1) / s;
                    q.splits = (nb + q.per - 1) / q.per;
                    if (q.splits != s) continue;
                    plan[n] = q;
                    us[n++] = tile_time(q, colblk);
                }
            }
    }
    Gemm8Plan best(int M) const {                         // for M rows, more than 16, of these units
        Gemm8Plan p = {};
        p.splits = 1;
        p.per = nb;
        const int mt = few_tiles(M), passes = (fp8_tiles(M) + mt - 1) / mt;
        const double bytes = (double)N * nb * 128;
        double best = M > 1 << 16 ? 1e30 : 1.5 + std::max((double)fp8_tiles(N) * passes * (mt + 1) * nb * 2048.0 / 256 / 52e3, bytes / 5e6);
        for (int i = 0; i < n; ++i) {
            const double t = std::max(us[i] + (plan[i].splits > 1 ? part_time(M, N, plan[i].splits) : 0.0), bytes / 4.6e6 + 2.0);
            if (t < best) {
                best = t;
                p = plan[i];
            }
        }
        return p;
    }
};

Gemm8Plan plan_gemm_fp8(int M, int N, int K) {
    const int nb = fp8_blocks(K);
    if (M > 16) return Gemm8Plans((M + 63) / 64, N, nb).best(M);
    Gemm8Plan p = {};
    p.splits = 1;
    p.per = nb;
    return p;
}
size_t gemm_fp8_part_bytes(const Gemm8Plan &p, int M, int N) {
    return p.splits > 1 ? (size_t)p.splits * M * N * 4 : 0;
}
// The most of any count of rows up to M: fewer rows can have more splits.  A split saves at most an unsplit workgroup's time (the round that is
// not full), so that no count is split from where its partial sums take longer on.
size_t gemm_fp8_most_part_bytes(int M, int N, int K) {
    const int nb = fp8_blocks(K);
    size_t most = 0;
    for (int m = 17; m <= M && part_time(m, N, 2) < tile_wg_time(4, 4, nb, 1);) {
        const Gemm8Plans plans((m + 63) / 64, N, nb);
        for (const int end = std::min((m + 63) / 64 * 64, M); m <= end; ++m)
            most = std::max(most, gemm_fp8_part_bytes(plans.best(m), m, N));
    }
    return most;
}

void launch_fp8_pack(int dtype, const void *src, int rows, int K, unsigned char *dst, int dst_rows, int tile_off, int tile_stride,
                     hipStream_t st) {
    const PackArgs a = {rows, K, fp8_tiles(dst_rows), tile_off, tile_stride, dst, (unsigned *)(dst + fp8_code_bytes(dst_rows, K))};
    const unsigned grid = (unsigned)fp8_tiles(rows) * ((fp8_blocks(K) + 1) / 2);
    if (dtype == TIDAR_BF16) fp8_pack_kernel<<<grid, 256, 0, st>>>(a, (const bf16_t *)src);
    else fp8_pack_kernel<<<grid, 256, 0, st>>>(a, (const float *)src);
}

void launch_gemm_fp8(const unsigned char *a, const unsigned char *w, void *out, int out_dtype, int M, int N, int K, const Gemm8Plan &p,
                     float *part, hipStream_t st) {
    const Gemm8Args g = {a, w, (const unsigned *)(a + fp8_code_bytes(M, K)), (const unsigned *)(w + fp8_code_bytes(N, K)), out, M, N, K,
                         fp8_tiles(M), fp8_tiles(N), fp8_blocks(K), out_dtype == TIDAR_BF16};
    if (p.ra) {
        auto tile = [&](auto ca) {
            constexpr int CA = decltype(ca)::value;
            if (p.ra == 4) launch_tile<4, CA>(g, p, part, st);
            else if (p.ra == 3) launch_tile<3, CA>(g, p, part, st);
            else if (p.ra == 2) launch_tile<2, CA>(g, p, part, st);
            else launch_tile<1, CA>(g, p, part, st);
        };
        if (p.ca == 4) tile(std::integral_constant<int, 4>());
        else tile(std::integral_constant<int, 2>());
        if (p.splits > 1) {
            const size_t n = (size_t)M * N;
            const unsigned grid = (unsigned)((n / 4 + 255) / 256);
            if (out_dtype == TIDAR_BF16) gemm8_sum_kernel<<<grid, 256, 0, st>>>(part, p.splits, n, (bf16_t *)out);
            else gemm8_sum_kernel<<<grid, 256, 0, st>>>(part, p.splits, n, (float *)out);
        }
        return;
    }
    auto go = [&](auto mt) {
        constexpr int MT = decltype(mt)::value;
        gemm8_few_kernel<MT, 8, void><<<dim3(g.w_tiles, (g.a_tiles + MT - 1) / MT), 512, 0, st>>>(g, nullptr);
    };
    if (few_tiles(M) == 1) go(std::integral_constant<int, 1>());
    else if (few_tiles(M) == 2) go(std::integral_constant<int, 2>());
    else go(std::integral_constant<int, 4>());
}

// Whether a product's workgroups bring the rows into 8 bits by themselves: as long as that is few blocks for each, and either few rows or few
// workgroups.  us by themselves and in a launch before: 1 x 24576 x 4096 19.8, 24.6;  4 x 24576 x 4096 22.1, 25.1;  1 x 4096 x 12288 11.8, 13.7;
// 4 x 4096 x 12288 (384 blocks) 15.5, 13.7;  8 x 6144 x 4096 (256) 10.2, 9.4;  16 x 6144 x 1536 (192) 7.2, 9.1;  16 x 17920 x 1536 13.2, 9.5
bool gemm_fp8_own_rows(int M, int N, int K) {
    return M <= 16 && M * fp8_blocks(K) <= 192 && (M <= 4 || fp8_tiles(N) <= 512);
}

void launch_gemm_fp8_own(int dtype, const void *a, const unsigned char *w, void *out, int out_dtype, int M, int N, int K, hipStream_t st) {
    const Gemm8Args g = {nullptr, w, nullptr, (const unsigned *)(w + fp8_code_bytes(N, K)), out, M, N, K,
                         fp8_tiles(M), fp8_tiles(N), fp8_blocks(K), out_dtype == TIDAR_BF16};
    const size_t smem = (size_t)M * g.nb * 129;
    auto go = [&](auto t) {
        typedef decltype(t) T;
        gemm8_few_kernel<1, 8, T><<<g.w_tiles, 512, smem, st>>>(g, (const T *)a);
    };
    if (dtype == TIDAR_BF16) go(bf16_t());
    else go(float());
}
