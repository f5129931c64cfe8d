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

// The ragged batch of a paged call, the FIRST argument of each of its kernels: they read it through the kernel argument segment with a
// uniform index, one scalar load per field.  (A struct of arrays in a parameter that is indexed with a variable is copied to scratch
// memory first, 264 bytes per lane for 16 sequences.)  Batches of up to kPagedInline sequences need no table in memory, and so no launch that writes
// one.  Both together: the append of 64 rows of the 70B heads and its read-back went from 26.6 us of kernels to 13.5
// (9.4 with what paged_append.hip describes).
constexpr int kPagedInline = 128;
struct PagedSeqs {
    const int32_t *dev;              // [4][B]: q_start, q_len, kv_len, slot; nullptr -> the arrays
    int32_t B, n, q_max, pad;
    int32_t q_start[kPagedInline], q_len[kPagedInline], kv_len[kPagedInline], slot[kPagedInline];
};
typedef const __attribute__((address_space(4))) PagedSeqs *SeqsArg;
__device__ __forceinline__ SeqsArg seqs_arg() { return (SeqsArg)__builtin_amdgcn_kernarg_segment_ptr(); }

struct SeqSpan {
    int32_t q_start, q_len, kv_len, slot;
};
__device__ __forceinline__ SeqSpan seq_span(SeqsArg st, int b)      // b: uniform
{
    const int32_t *dev = st->dev;
    const int B = st->B;
    if (dev) return {dev[b], dev[B + b], dev[2 * (size_t)B + b], dev[3 * (size_t)B + b]};
    return {st->q_start[b], st->q_len[b], st->kv_len[b], st->slot[b]};
}

// A length from device memory that the capacity does not cover: the sequence has no page, no row of the rotary table and no token.  (As unsigned numbers: one below
// zero is none either.)
__device__ __forceinline__ bool beyond_capacity(const SeqSpan &si, int cap) { return (uint32_t)si.kv_len > (uint32_t)cap; }

// Blocks of 16 tokens that a sequence's q_len rows can touch, wherever they begin
__host__ __device__ inline int paged_blocks_of(int q_len) { return (q_len + 30) >> 4; }

// Sequence b of the call that item `key` belongs to when sequence j brings count(j) items (seq_of: count(q_len_j)), and the item's place among its own.
// key is the same in all lanes of the wavefront; b = B: behind the last one.  64 sequences at a time, one per lane.
template <typename Count>
__device__ __forceinline__ int seq_at(SeqsArg st, int key, const Count &count, int &place)
{
    const int B = st->B;
    place = key;
    if (B == 1) return 0;                                      // (the caller finds a place behind the last one by the lengths)
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < B; base += kWave) {
        const int own = base + lane < B ? count(base + lane) : 0;
        int sum = own;                                         // inclusive sum over the lanes up to this one
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int other = __shfl_up(sum, off, kWave);
            if (lane >= off) sum += other;
        }
        const unsigned long long past = __ballot(key < before + sum);
        if (past) {
            const int j = __ffsll(past) - 1;
            place = key - before - __builtin_amdgcn_readlane(sum - own, j);
            return base + j;
        }
        before += __builtin_amdgcn_readlane(sum, kWave - 1);
    }
    return B;
}

template <typename Count>
__device__ __forceinline__ int seq_of(SeqsArg st, int key, const Count &count, int &place)
{
    const int32_t *dev = st->dev;
    const int B = st->B;
    return seq_at(st, key, [&](int j) { return count(dev ? dev[B + j] : st->q_len[j]); }, place);
}

// Tiles of a paged attention call are numbered sequence by sequence.  per_seq > 0: that many numbers for each, of which a short one leaves some unused;
// 0: as many as it has (a decode step's or one prompt's batch needs no search; a prompt among many rows would launch its own number for
// each of them).
template <typename Count>
__device__ __forceinline__ int tile_of(SeqsArg st, int item, int per_seq, const Count &count, int &place)
{
    place = 0;
    if (per_seq == 1) return item;
    if (per_seq == 0) return seq_of(st, item, count, place);
    const int b = item / per_seq;
    place = item - b * per_seq;
    return b;
}
constexpr int64_t kMaxThreads = (1LL << 32) - 1;      // of a launch's x dimension

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
template <typename Args>
__device__ inline int paged_block(const Args &pa, int g, int kvh, int slot, int blk)
{
    const int at = blk >> pa.shift;
    if ((unsigned)slot >= (unsigned)pa.slots || blk < 0 || at >= pa.per_slot) return -1;
    const int page = pa.pages[(size_t)slot * pa.per_slot + at];
    if ((unsigned)page >= (unsigned)pa.n_pages) return -1;
    return ((page * g + kvh) << pa.shift) + (blk & ((1 << pa.shift) - 1));
}

constexpr int kPagedPartials = 65536;             // partial results (row, head, split) of a paged attention call at most

// How a paged attention call is cut (attn_paged.hip): sequences that fill a tile of 256 pairs go to such tiles if there are row_tiles of them over all KV heads
struct PagedPlan {
    int32_t least;                   // pairs from which a sequence is the other kernel's
    int32_t row_items, items;        // tiles of 256 and of 16 pairs that are launched
    int32_t row_per_seq, per_seq;    // as tile_of takes them
    int32_t chunk, splits, waves;    // wavefronts per workgroup of 16-pair tiles
};
PagedPlan paged_plan(const relax_layer_dims &dm, const relax_seqs &sq, int32_t n, int32_t L_max, int32_t row_tiles);

// Attention of the sequences with at least `least` (row, head) pairs, in `items` tiles of kPagedRowTile pairs (attn_paged_rows.hip)
constexpr int kPagedRowTile = 256;
hipError_t launch_paged_rows(const uint16_t *q, const PagedArgs &pa, const relax_layer_dims &dm, const PagedSeqs &st, int32_t items, int32_t per_seq, int32_t least, uint16_t *out,
                             hipStream_t stream);

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
