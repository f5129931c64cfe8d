// Device functions of the paged 8-bit KV cache (layout and meaning: relax_paged_cache in relax_mi355.h), shared by the kernels that
// append to it (paged_append.hip) and read it (paged_append.hip, attn_paged.hip).
//
// A block is 16 tokens of one KV head: 16 * d codes of one byte, u = 128 + round(x / s) in 1..255, with one scale for keys and one for
// values.  Why 16: it is the token side of a 16 x 16 MFMA tile, so the scale of a tile is one scalar that multiplies scores or
// probabilities, and the codes go into the products as the integers they are (exact in fp16).  Both blocks are laid out as the fragments
// of those products, so that a wavefront loads 1 KB of consecutive bytes per instruction and nothing is shuffled afterwards:
//   K  [d / 16][16 tokens][16 elements]           lane (token = l % 16, quarter = l / 16) of load j holds elements 16 (4 j + quarter) .. + 15
//   V  [d / 64][4][16][4][4]: [e / 64][t / 4][e % 16][e / 16 % 4][t % 4]
//                                                 lane (e % 16 = l % 16, t / 4 = l / 16) of load j holds elements 64 j + 16 i + l % 16, four tokens each
// A code is offset by 128 because 0x64uu is the fp16 number 1024 + u: one byte permutation makes two halves, one packed subtraction of
// 1152 two signed integers.
#pragma once

#include "relax_common.h"

namespace relax {

typedef _Float16 half2p_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8p_t __attribute__((ext_vector_type(8)));
typedef float float4p_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2p_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4p_t __attribute__((ext_vector_type(4)));

struct SeqSpan {
    int32_t q_start, q_len, kv_len, slot;
};
__device__ inline SeqSpan seq_span(const SeqTable &st, int b)
{
    SeqSpan s;
    if (st.dev) {
        s.q_start = st.dev[b], s.q_len = st.dev[st.B + b], s.kv_len = st.dev[2 * st.B + b], s.slot = st.dev[3 * st.B + b];
    } else {
        s.q_start = st.q_start[0], s.q_len = st.q_len[0], s.kv_len = st.kv_len[0], s.slot = st.slot[0];
#pragma unroll
        for (int j = 1; j < kInlineSeqs; ++j)                  // static indices: see row_info
            if (j == b) s.q_start = st.q_start[j], s.q_len = st.q_len[j], s.kv_len = st.kv_len[j], s.slot = st.slot[j];
    }
    return s;
}

// Blocks of 16 tokens that a sequence's q_len rows can touch, wherever they begin
__host__ __device__ inline int paged_blocks_of(int q_len) { return (q_len + 30) >> 4; }

// Sequence b of the call that item `key` belongs to when sequence j brings count(q_len_j) items, and the item's place among its own.
// key is the same in all lanes of the wavefront; b = st.B: behind the last one.  A device table is searched 64 sequences at a time.
template <typename Count>
__device__ inline int seq_of(const SeqTable &st, int key, const Count &count, int &place)
{
    if (!st.dev) {
        int b = st.B, left = key;
#pragma unroll
        for (int j = 0; j < kInlineSeqs; ++j) {
            const int c = j < st.B ? count(st.q_len[j]) : 0;
            if (b == st.B && j < st.B) {
                if (left < c) b = j;
                else left -= c;
            }
        }
        place = left;
        return b;
    }
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < st.B; base += kWave) {
        const int own = base + lane < st.B ? count(st.dev[st.B + base + lane]) : 0;
        int sum = own;                                         // inclusive sum over the lanes up to this one
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int other = __shfl_up(sum, off, kWave);
            if (lane >= off) sum += other;
        }
        const unsigned long long past = __ballot(key < before + sum);
        if (past) {
            const int j = __ffsll((unsigned long long)past) - 1;
            place = key - before - (__shfl(sum, j, kWave) - __shfl(own, j, kWave));
            return base + j;
        }
        before += __shfl(sum, kWave - 1, kWave);
    }
    place = 0;
    return st.B;
}

struct PagedArgs {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    const int32_t *pages;
    const float *rope;
    uint32_t *err;                   // flag word of the workspace
    int32_t n_pages, per_slot, slots, cap;
    int32_t shift;                   // log2 of the blocks per page
};
constexpr uint32_t kBadPage = 4u;    // bit 2 of the flag word: a block had no page

// Number of a sequence's block `blk` in the pool for KV head kvh, -1 if its slot, its place in the slot's row of the page table or the page is
// out of range: the table is device data, so what it says is checked here and not on the host.
__device__ inline int paged_block(const PagedArgs &pa, int g, int kvh, int slot, int blk)
{
    const int at = blk >> pa.shift;
    if ((unsigned)slot >= (unsigned)pa.slots || blk < 0 || at >= pa.per_slot) return -1;
    const int page = pa.pages[(size_t)slot * pa.per_slot + at];
    if ((unsigned)page >= (unsigned)pa.n_pages) return -1;
    return ((page * g + kvh) << pa.shift) + (blk & ((1 << pa.shift) - 1));
}

// four codes -> four fp16 integers
__device__ __forceinline__ void codes_to_half(uint32_t w, half2p_t &lo, half2p_t &hi)
{
    const half2p_t off = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(half2p_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - off;
    hi = __builtin_bit_cast(half2p_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - off;
}
__device__ __forceinline__ half8p_t codes_to_half8(uint32_t w0, uint32_t w1)
{
    half2p_t a, b, c, d;
    codes_to_half(w0, a, b);
    codes_to_half(w1, c, d);
    return half8p_t{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

}  // namespace relax
