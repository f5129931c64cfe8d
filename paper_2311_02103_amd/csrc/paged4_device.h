// Device functions of the paged 4-bit KV cache (layout and meaning: relax_paged4_cache in relax_mi355.h), shared by the kernels that append to it and read it.
//
// A word holds eight codes of four bits.  A byte 0000uuuu is the fp8 (e4m3) number u 2^-9, subnormal or not, so the conversion of two fp8 numbers with a factor of 2^9
// makes two fp16 numbers u, exactly: seven instructions per word, of which three separate its halves.  (Masks alone make subnormal fp16 numbers u 2^-24, two instructions less, but the matrix
// instructions align products by the operands' exponent fields: sums were off by 2^-15 of their terms, with normal numbers by 2^-23.)
// The order of the codes in a word is the one that brings them out as fragments:
//   K  word [quarter = e / 8 % 4][t][e / 32]   lane (token = l % 16, quarter = l / 16): k step e / 32, elements 0 4 1 5 2 6 3 7 of its eight
//   V  word [t / 4][e % 16][e / 32]            lane (e % 16 = l % 16, quarter = l / 16): its four tokens as 0 2 1 3, for the element below 16 of 32 and for the one above
// Scales [t / 4][e / 32][t % 4]: the four tokens that a lane of the result of K Q^T, and of the operand V, holds in eight bytes.  The offset of 8 comes off the codes,
// u s + (-8 s), exactly, or off the sums: sum (u - 8) q = sum u q - 8 sum q.
#pragma once

#include "paged_device.h"

namespace relax {

constexpr int kGroup4 = RELAX_PAGED4_GROUP;

struct Paged4Args {
    uint8_t *k, *v;
    uint16_t *k_scale, *v_scale;
    const int32_t *pages;
    uint32_t *err;                   // flag word of the workspace
    int32_t n_pages, per_slot, slots, cap;
    int32_t shift;                   // log2 of the blocks per page
};

// Attention of the sequences with at least pl.least (row, head) pairs, in tiles of kPagedRowTile pairs (attn_paged4_rows.hip)
hipError_t launch_paged4_rows(const uint16_t *q, const Paged4Args &pa, const relax_layer_dims &dm, const PagedSeqs &st, const PagedPlan &pl, uint16_t *out, hipStream_t stream);

// The eight codes of a word as fp16 numbers 0..15: the low halves of its bytes 0 .. 3, then the high ones
__device__ __forceinline__ void word_codes(uint32_t w, half2p_t (&u)[4])
{
    const uint32_t lo = w & 0x0f0f0f0fu, hi = w >> 4 & 0x0f0f0f0fu;
    u[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false), u[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true);
    u[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false), u[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true);
}
__device__ __forceinline__ half8p_t operand(half2p_t a, half2p_t b, half2p_t c, half2p_t d) { return half8p_t{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y}; }

constexpr int block4_codes(int d) { return 8 * d; }            // bytes of a block's codes
constexpr int block4_scales(int d) { return d / 2; }           // fp16 numbers

}  // namespace relax
