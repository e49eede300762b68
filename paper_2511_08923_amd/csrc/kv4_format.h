// The 4-bit cache's page format and its conversions, shared by the kernels that write and read it.
//
// One page of one kv head is a block of 544 * nb bytes, nb = ceil(head_dim / 32) (17 whole cache lines at head_dim 128):
//   K codes   [nb][16 tokens][16 bytes]               byte j of token t: elements 2j (low nibble), 2j + 1 of 32-element block
//   V codes   [4 token quads][4 nb groups][4 tokens][4 bytes]   byte j: elements 2j (low), 2j + 1 of 8-element group
//   K scales  [nb][16 tokens], V scales [nb][16 tokens]         one byte per token and block
// No two tokens share a byte, so rows are stored without reading their neighbours.  The orders are those of the MFMA
// operands: a wave's lane (token, block) finds its 32 elements of K in one 16-byte piece, lane (8 head-dim values, token
// quad) its 4 x 8 elements of V in one, and either read of a page is one contiguous KiB.
//
// A code is e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign), a scale byte s stands for 2^(s - 127), 2 <= s <= 252, or, 255,
// for a block that held an infinity or NaN and reads back as NaN.  Scales are powers of two: codes times scale are exact in
// bf16, and the quantiser's division is exact, so its result is the same in any precision.
#pragma once
#include "tidar_internal.h"

namespace {

__host__ __device__ inline int kv4_blocks(int hd) { return (hd + 31) / 32; }
__host__ __device__ inline int kv4_head_bytes(int hd) { return 544 * kv4_blocks(hd); }
__host__ __device__ inline int kv4_v_codes(int nb) { return 256 * nb; }
__host__ __device__ inline int kv4_k_scales(int nb) { return 512 * nb; }
__host__ __device__ inline int kv4_v_scales(int nb) { return 528 * nb; }
// address of (page, head): 64 bits, a layer may hold more than 4 GiB
__device__ inline size_t kv4_offset(const Kv4View &kv, int page, int h) {
    return ((size_t)page * kv.n_kv + h) * (size_t)kv4_head_bytes(kv.hd);
}

constexpr int kScaleNan = 255;
__device__ inline float kv4_scale(unsigned byte) { return __uint_as_float(byte << 23); }     // 255: infinity
// Scale byte of a block from the bits of its largest magnitude: the smallest exponent e with amax <= 7 * 2^e (values
// between 6 and 7 steps go to 6, at most half of the step between 4 and 6 away), held where 6 * 2^e and 2^(e-1) are normal.
__device__ inline unsigned kv4_scale_byte(unsigned amax_bits) {
    if (amax_bits >= 0x7f800000u) return kScaleNan;
    const int e = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (unsigned)(e < 2 ? 2 : e > 252 ? 252 : e);
}

typedef __attribute__((ext_vector_type(2))) __bf16 kv4_bf16x2;
typedef __attribute__((ext_vector_type(2))) float kv4_f32x2;
// Two elements of byte SEL of a word of codes, times the scale.
template <int SEL>
__device__ inline kv4_bf16x2 kv4_pair_bf16(unsigned word, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, SEL);
}
template <int SEL>
__device__ inline kv4_f32x2 kv4_pair_f32(unsigned word, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, SEL);
}

}  // namespace
