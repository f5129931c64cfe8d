// Appending to the paged 4-bit KV cache, with norm and rotation of the heads on the way, and reading it back.
//
//   q'[i], k'[i]                       prepared heads (heads_device.h); k' stays fp32 until it is quantised
//   s = round8(x* / -8)                per 32 elements of a token, x* the one of the largest magnitude
//   u = 8 + clamp(rne(x / s), -8, 7)
//
// x / -8 puts the largest element on code 0 exactly and leaves the other end at 7/8 of it: sixteen levels where a scale of max / 7 has fifteen.  round8 is a
// rounding to bf16, and eight bits times a code are an fp16 number, so that nothing behind this kernel rounds a key or a value.
//
// One wavefront is four tokens that share the words of V (positions 4 j .. 4 j + 3) of `steps` KV heads' keys, or values: 16 lanes per token, eight
// elements per lane.  A group is four lanes.  Keys go out as the lane's own word; values change hands between the lanes of the four
// tokens through permlane swaps, into words that hold a byte of each.  Where the call brings fewer than four of them, bytes are stored: no token of another
// call is read or written.  q is prepared by further workgroups of the same launch.
//
// 2043 rows of 32 / 32 heads of 128, turned: 16.5 us for 76 MB, 4.6 TB/s, and 9.5 to read them back, 43 MB: both between a long stream's bytes (12.5 and 7) and the vector unit's
// instructions.  (Two steps of heads on their way instead of one: 26.5 us together for 25.7.)  One row: 5.4 us in a graph, two chains of three dependent loads, of which
// two launches are 3.7.
#include "heads_device.h"
#include "paged4_device.h"

namespace relax {

namespace {

struct KvRows {
    const uint16_t *k, *v;
    int64_t stride;                  // elements from one row to the next
};

__host__ __device__ inline int paged4_quads_of(int q_len) { return (q_len + 6) >> 2; }      // aligned groups of four positions that q_len rows can touch

// scale of a group from its largest and smallest element, rounded to eight significant bits (bf16), at most 8160 = 255 * 32: 8160 * 8 is an fp16 number
__device__ __forceinline__ _Float16 scale_of(float top, float low)
{
    const float s = (top >= -low ? top : low) * -0.125f;
    const uint32_t u = __builtin_bit_cast(uint32_t, s);
    const float r = __builtin_bit_cast(float, (u + 0x7fffu + (u >> 16 & 1u)) & 0xffff0000u);
    return (_Float16)fminf(fmaxf(r, -8160.0f), 8160.0f);
}
// rne(x / s) in -8..7 plus 8, of eight elements, four to a number: d0 = sum over j of the codes of elements i_j times 16^j, exact in fp32.
// x - a s is exact (a has 24 bits, s eight), inv the reciprocal of s within 2^-23, so q is the quotient rounded once but for 2^-22 of its last bit; and a quotient that is no tie is at least
// 0.501 of its last bit away from one, because s has eight bits: no value goes to the wrong side.  (The bounds are whole numbers: they may go in front of the rounding.)
__device__ __forceinline__ void codes_of(const float (&x)[8], float s, float (&c)[8])
{
    const float inv = s != 0.0f ? __builtin_amdgcn_rcpf(s) : 0.0f;      // (a scale of 0: all codes 8)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float a = x[j] * inv, q = fmaf(fmaf(-a, s, x[j]), inv, a);
        c[j] = rintf(__builtin_amdgcn_fmed3f(q, -8.0f, 7.0f));
    }
}
__device__ __forceinline__ uint32_t digits(float a, float b, float c, float d)      // nibbles a b c d, each plus 8
{
    return (uint32_t)fmaf(fmaf(fmaf(d, 16.0f, c), 16.0f, b), 16.0f, a + (float)0x8888);
}
__device__ __forceinline__ uint32_t dword_dpp_xor2(uint32_t v) { return __builtin_bit_cast(uint32_t, lane_xor<2>(__builtin_bit_cast(float, v))); }

// four nibbles to the low halves of four bytes
__device__ __forceinline__ uint32_t spread(uint32_t v)
{
    const uint32_t w = (v | v << 8) & 0x00ff00ffu;
    return (w | w << 4) & 0x0f0f0f0fu;
}

// the dwords that the lanes with the same l % 16 hold, by l / 16
__device__ __forceinline__ void gather_quarters(uint32_t v, uint32_t (&w)[4])
{
    const u32x2_t half = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const uint32_t lo = half.x, hi = half.y;                   // quarters 0 1 0 1 and 2 3 2 3
    const u32x2_t a = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), b = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
}

// Workgroups 0 .. kv_groups - 1: four wavefronts, four of the 2 * chunks (keys or values of `steps` steps of KV heads) of one item; the rest: rows of q
template <int D>
__global__ __launch_bounds__(256) void paged4_append_kernel(PagedSeqs, HeadRows hr, KvRows r, HeadPrep p, Paged4Args pa, int h, int g, int64_t kv_groups, int chunks, int steps,
                                                            int slices)
{
    constexpr int U = kUnits<D>, HS = 16 / U, J = D / 32;      // heads of a token side by side; groups of a head
    const SeqsArg st = seqs_arg();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (blockIdx.x >= kv_groups) {
        head_rows<D>(st, hr, p, h, 0, pa.cap, ((int64_t)blockIdx.x - kv_groups) * 4 + wave, slices, pa.err);
        return;
    }
    const int64_t w_all = (int64_t)blockIdx.x * 4 + wave;
    const int item = (int)(w_all / (2 * chunks)), part = (int)(w_all - (int64_t)item * (2 * chunks));
    const bool values = part & 1;
    int place, b = item;
    if (st->q_max == 1) place = 0;
    else b = seq_of(st, item, [](int q_len) { return paged4_quads_of(q_len); }, place);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, __builtin_amdgcn_readfirstlane(b));
    if (beyond_capacity(si, pa.cap)) {
        if (lane == 0) atomicOr(pa.err, kBadPage);
        return;
    }
    const int first = si.kv_len - si.q_len;                    // position of the sequence's first row
    if (first < 0) return;
    const int base = ((first >> 2) + place) * 4, low = max(first - base, 0), high = min(si.kv_len - base, 4);      // tokens low .. high - 1 of the four are the call's
    if (high <= low) return;
    const int quarter = lane >> 4, unit = lane & (U - 1), sub = (lane & 15) / U;
    const bool fresh = quarter >= low && quarter < high;
    const int tok = min(max(quarter, low), high - 1);          // (lanes of other tokens take the nearest one)
    const int64_t row = si.q_start + (base - first) + tok;
    const uint16_t *src = (values ? r.v : r.k) + row * r.stride + unit * 8;
    const int begin = (part >> 1) * steps * HS, end = min(g, begin + steps * HS);
    if (begin >= end) return;
    Unit in = *(const Unit *)(src + min(begin + sub, g - 1) * D);
    Unit wk = {};
    Angles a = {};
    if (!values) {
        if (p.k_norm) wk = *(const Unit *)(p.k_norm + unit * 8);
        if (p.rope) load_angles(a, p, base + tok, unit);
    }
    const int pool = paged_block(pa, g, 0, si.slot, base >> 4);
    if (pool < 0) {
        if (lane == 0) atomicOr(pa.err, kBadPage);
        return;
    }
    const int t16 = (base & 12) + quarter, j = unit >> 2;      // token of the block; group of the head
    for (int hd = begin; hd < end; hd += HS) {
        Unit ahead = in;
        if (hd + HS < end) ahead = *(const Unit *)(src + min(hd + HS + sub, g - 1) * D);
        float x[8];
        to_storable(in, x);
        if (!values) {
            if (p.k_norm) normalise<D>(x, wk, p.eps);
            if (p.rope) rotate<D>(x, a, p, unit, lane);
        }
        float top = x[0], bottom = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]), bottom = fminf(bottom, x[i]);
        top = fmaxf(top, lane_xor<1>(top)), bottom = fminf(bottom, lane_xor<1>(bottom));
        top = fmaxf(top, lane_xor<2>(top)), bottom = fminf(bottom, lane_xor<2>(bottom));
        const _Float16 s = scale_of(top, bottom);
        float c[8];
        codes_of(x, (float)s, c);
        const int kvh = hd + sub;
        const bool there = kvh < g;
        const size_t blk = (size_t)pool + ((size_t)kvh << pa.shift);
        if (!values) {
            const uint32_t w = digits(c[0], c[2], c[4], c[6]) | digits(c[1], c[3], c[5], c[7]) << 16;
            if (fresh && there) ((uint32_t *)(pa.k + blk * block4_codes(D)))[((unit & 3) * 16 + t16) * J + j] = w;
        } else {
            // lanes of elements below 16 of 32 and their partners above: bytes of elements 0 .. 3, resp. 4 .. 7, of the eight
            const bool above = unit & 2;
            const uint32_t mine = digits(c[0], c[1], c[2], c[3]), rest = digits(c[4], c[5], c[6], c[7]);
            const uint32_t given = dword_dpp_xor2(above ? mine : rest), kept = above ? rest : mine;
            // bytes of the four elements: the nibble of the lane below in the low half, of the lane above in the high one
            const uint32_t lows = spread(above ? given : kept), highs = spread(above ? kept : given);
            const uint32_t bytes = lows | highs << 4;
            uint32_t w4[4];
            gather_quarters(bytes, w4);
            const uint32_t sel = (uint32_t)quarter | (uint32_t)(quarter + 4) << 8;                     // byte `quarter` of either
            const uint32_t lo = __builtin_amdgcn_perm(w4[2], w4[0], sel), hi = __builtin_amdgcn_perm(w4[3], w4[1], sel);
            const uint32_t w = (lo & 0xffffu) | hi << 16;      // tokens 0 2 1 3
            uint32_t *dst = (uint32_t *)(pa.v + blk * block4_codes(D)) + ((base >> 2 & 3) * 16 + (unit & 1) * 8 + (above ? 4 : 0) + quarter) * J + j;
            if (there) {
                if (low == 0 && high == 4) *dst = w;
                else {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (t >= low && t < high) ((uint8_t *)dst)[(t & 1) * 2 + (t >> 1)] = (uint8_t)(w >> (8 * ((t & 1) * 2 + (t >> 1))));
                }
            }
        }
        if (fresh && there && (unit & 3) == 0)
            (values ? pa.v_scale : pa.k_scale)[blk * block4_scales(D) + ((base >> 2 & 3) * J + j) * 4 + quarter] = __builtin_bit_cast(uint16_t, s);
        in = ahead;
    }
}

// out[row, kvh, :] = code * scale, exact.  One wavefront is one (block, KV head) of keys or of values; words change hands in LDS so that a lane has eight consecutive
// elements of D / 32 tokens and a row of a head is written at once.
template <int D>
__global__ __launch_bounds__(256) void paged4_read_kernel(PagedSeqs, Paged4Args pa, uint16_t *k_out, uint16_t *v_out, int g)
{
    constexpr int J = D / 32, U = kUnits<D>, R = D / 32;       // R: tokens per lane
    constexpr int kPitch = 16 * J + 4;                         // words of a quarter in LDS: the 64 words of a load are on 64 banks
    __shared__ __align__(16) uint32_t turns[4][4 * kPitch];
    const SeqsArg st = seqs_arg();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t w_all = (int64_t)blockIdx.x * 4 + wave;
    const int item = (int)(w_all / (2 * g)), part = (int)(w_all - (int64_t)item * (2 * g)), kvh = part >> 1;
    const bool values = part & 1;
    uint16_t *out = values ? v_out : k_out;
    if (!out) return;
    int place, b = item;
    if (st->q_max == 1) place = 0;
    else b = seq_of(st, item, [](int q_len) { return paged_blocks_of(q_len); }, place);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, __builtin_amdgcn_readfirstlane(b));
    const bool beyond = beyond_capacity(si, pa.cap);
    // a length that the capacity does not cover: rows of zeros, as many as the call has
    const int first = beyond ? 0 : si.kv_len - si.q_len;
    if (first < 0) return;
    const int blk = (first >> 4) + place, lead = (first & 15) - place * 16;
    const int low = max(lead, 0), high = min(lead + si.q_len, 16);
    if (high <= low) return;
    const int pool = beyond ? -1 : paged_block(pa, g, kvh, si.slot, blk);
    if (pool < 0 && lane == 0) atomicOr(pa.err, kBadPage);
    const size_t at = (size_t)max(pool, 0);
    const uint32_t *codes = (const uint32_t *)((values ? pa.v : pa.k) + at * block4_codes(D));
    const uint16_t *scales = (values ? pa.v_scale : pa.k_scale) + at * block4_scales(D);
    uint32_t *turn = turns[wave];
    typedef uint32_t words_t __attribute__((ext_vector_type(J)));
    *(words_t *)(turn + (lane >> 4) * kPitch + (lane & 15) * J) = ((const words_t *)codes)[lane];
    const int unit = lane & (U - 1), j = unit >> 2, quarter = lane >> 4, t0 = D == 128 ? 0 : (lane >> 3 & 1) * 2;      // tokens 4 quarter + t0 + i
    typedef _Float16 scales_t __attribute__((ext_vector_type(R)));
    const scales_t s = *(const scales_t *)(scales + (quarter * J + j) * 4 + t0);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");     // (a wavefront's LDS instructions execute in order: only the compiler has to keep it)
    __builtin_amdgcn_wave_barrier();
    uint32_t w[8];
    if (values) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = turn[quarter * kPitch + ((unit & 1) * 8 + e) * J + j];
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) w[i] = turn[(unit & 3) * kPitch + (4 * quarter + t0 + i) * J + j];
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int t = t0 + i, tok = 4 * quarter + t;
        Unit x;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = values ? w[e] >> (8 * ((t & 1) * 2 + (t >> 1)) + 2 * (unit & 2)) & 15u
                                      : w[i] >> (8 * ((e & 1) * 2 + (e >> 2)) + 2 * (e & 2)) & 15u;
            x[e] = pool < 0 ? (_Float16)0.0f : (_Float16)((float)((int)u - 8) * (float)s[i]);
        }
        if (tok >= low && tok < high) *(Unit *)(out + ((size_t)(si.q_start - lead + tok) * g + kvh) * D + unit * 8) = x;
    }
}

}  // namespace

// quads: paged4_quads_of the call's sequences in all
hipError_t launch_paged4_append(const HeadRows &hr, const uint16_t *k, const uint16_t *v, int64_t kv_stride, const HeadPrep &p, const Paged4Args &pa, const relax_layer_dims &dm,
                                const PagedSeqs &st, const relax_seqs &sq, hipStream_t stream)
{
    int64_t quads = 0;
    for (int b = 0; b < sq.B; ++b) quads += st.q_max == 1 ? 1 : paged4_quads_of(sq.q_lens[b]);
    const int h = hr.q ? dm.n_heads : 0, g = dm.n_kv_heads, per_step = 16 * 8 / dm.head_dim, all_steps = (g + per_step - 1) / per_step;
    int steps = 1;                                             // of KV heads per wavefront (us, append and read-back of 2043 rows of 32 / 32 heads with 4096, 8192 and 16384 wavefronts: 25.6, 26.3, 29.5)
    while (steps < 16 && quads * (2 * ((all_steps + steps - 1) / steps)) > 4096) steps *= 2;
    const int chunks = (all_steps + steps - 1) / steps, slices = h ? head_slices(h, st.n, dm.head_dim) : 1;
    const int64_t kv_groups = (quads * 2 * chunks + 3) / 4, q_groups = h ? ((int64_t)st.n * slices + 3) / 4 : 0;
    if ((kv_groups + q_groups) * 256 > kMaxThreads) return hipErrorInvalidValue;
    const KvRows r = {k, v, kv_stride};
    const dim3 grid(kv_groups + q_groups);
    if (dm.head_dim == 128) hipLaunchKernelGGL(paged4_append_kernel<128>, grid, dim3(256), 0, stream, st, hr, r, p, pa, h, g, kv_groups, chunks, steps, slices);
    else hipLaunchKernelGGL(paged4_append_kernel<64>, grid, dim3(256), 0, stream, st, hr, r, p, pa, h, g, kv_groups, chunks, steps, slices);
    return hipGetLastError();
}

hipError_t launch_paged4_read(const Paged4Args &pa, uint16_t *k_out, uint16_t *v_out, const relax_layer_dims &dm, const PagedSeqs &st, int items, hipStream_t stream)
{
    const int64_t all = ((int64_t)items * 2 * dm.n_kv_heads + 3) / 4;
    if (all * 256 > kMaxThreads) return hipErrorInvalidValue;
    if (dm.head_dim == 128) hipLaunchKernelGGL(paged4_read_kernel<128>, dim3(all), dim3(256), 0, stream, st, pa, k_out, v_out, dm.n_kv_heads);
    else hipLaunchKernelGGL(paged4_read_kernel<64>, dim3(all), dim3(256), 0, stream, st, pa, k_out, v_out, dm.n_kv_heads);
    return hipGetLastError();
}

}  // namespace relax
