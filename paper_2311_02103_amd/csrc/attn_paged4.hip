// Causal attention over the paged 4-bit KV cache.
//
//   o[i] = sum_t p[i,t] v[t],   p[i,:] = softmax_t(q[i] . k[t] / sqrt d),  t = 0 .. pos_i,   k[t][e] = s_k[t][e / 32] (u_k[t][e] - 8), v likewise
//
// A tile is up to 32 consecutive (row, head) pairs against one KV head and one part of the tokens, S^T = K Q^T and O^T = V^T P^T, so that a pair is a column, a lane
// (quarter, column) of the scores holds tokens 4 quarter .. + 3 of a block, and the lane's eight weights of two blocks are what the second product wants from it.
//
// Up to eight pairs (a decode step with grouped heads): bytes and vector instructions are near each other, and a column costs little, so codes go into both products as fp16 integers 0..15
// (paged4_device.h) and the scales meet columns.  A scale is constant over a k step of 32 elements, so a step is a product of its own, S_j = sum u q, and x = sum_j s_kj S_j.  The
// accumulator of S_j starts at -8 sum q, which takes the codes' offset off.  The weight of a token times its value scale, w s_j, is rounded to fp16 once per group of 32 elements and is
// the operand; -8 sum (w s_j), from one more product per group, goes to the result.  The reference of a column, which the weights are exp2(score - reference) to, stands 12 below the
// largest score + log2 s of a lane's four tokens, s the root of the sum of squares of their scales, and moves when w s is about to leave fp16's range: the largest of these products is
// 2^12 .. 65000 whatever the size of the values, and an operand below fp16's normal range is off by 2^-37 of it.  (A reference that follows the score alone has to leave room for the
// largest scale, 8160, and rounds the tails of ordinary values away.)
// More pairs: a column costs more vector instructions than a token, so operands are the numbers that the cache stands for, (u - 8) s = u s + (-8 s), one multiply-add per two and
// exact (eight and four bits).  The products need no factor; the weight is rounded to fp16 and its sum is that of the rounded ones, from a product with ones.
// (300 rows of 32 / 8 heads on 1201 tokens beside eight sequences of five: 30.7 us; with codes and scales of columns as above 36.7.)
//
// Few pairs are bound by bytes, with what a workgroup's beginning and end and the merge take on top (about 3.8 and 3.9 us): heads of 128, 64 / 8 heads, one sequence of 120001 tokens 29.3 us, 4.7 TB/s
// (23.0 at a long stream's rate), 16 of 100 to 8000 tokens 21.7 (12.5).  17 to 32 pairs are bound by a wavefront's chain of decoding, products and exponentials, some 270
// instructions and 34 products per 32 tokens, with one to two wavefronts per SIMD: in the call above the vector unit is busy for 46 %, the matrix pipe for 15 %.
// (Tiles of 48 pairs, queries in LDS: 29.2 us for 30.6 in the call above, but 38.2 for 34.9 with 1200 rows on nothing.)
#include <algorithm>
#include <type_traits>

#include "paged4_device.h"

namespace relax {

namespace {

constexpr float kUnset = -1e30f;                 // reference of a column that has met no token: below every score, and finite
constexpr float kBias = 12.0f, kHead = 15.9f;    // up to eight pairs: log2 of the largest weight times scale behind a move of the reference, and before the next one
constexpr float kLeast2 = 0x1p-28f;              // square of the least scale that counts there: subnormal ones may be zeros in a product, and zeros leave the weights, up to 2^30, in fp32's range
constexpr float kPackedBias = 11.0f, kMost = 65000.0f;       // more: log2 of the weight at the reference, the largest weight before that moves

typedef _Float16 half4p_t __attribute__((ext_vector_type(4)));

// largest of a value over the four lanes of a column
__device__ __forceinline__ float column_max(float v)
{
    float2 both = pair_xor16(v);
    both = pair_xor32(fmaxf(both.x, both.y));
    return fmaxf(both.x, both.y);
}

// n / d for 0 <= n < 2^31 by a product: with s = ceil(log2 d) and m = floor(2^(31 + s) / d) + 1 the error n (m d - 2^(31 + s)) is below 2^(31 + s)
struct Divisor {
    uint32_t m, shift;
};
Divisor divisor(uint32_t d)
{
    uint32_t s = 0;
    while (s < 31 && (1u << s) < d) ++s;
    return {(uint32_t)((1ull << (31 + s)) / d + 1), 31 + s};
}
__device__ __forceinline__ int quotient(int n, const Divisor &d) { return (int)((uint64_t)(uint32_t)n * d.m >> d.shift); }

constexpr int kTile = 32;                        // (row, head) pairs of a tile at most
template <int D, int TILE, int W>
struct States {                                  // of the wavefronts, in LDS
    static constexpr int kPairs = TILE, kWaves = W, kPitch = D + 4;
    float o[W * TILE * kPitch], m[W * TILE], l[W * TILE];
};

// What a workgroup has to do: pairs p0 .. p0 + n_pairs - 1 of a sequence against tokens t_begin .. t_end - 1 and one KV head
struct Task {
    int q_start, slot, past, kvh, p0, n_pairs, t_begin, t_end;
    int rep;
    Divisor by_rep;
    int used, split, splits;         // parts of the sequence, this one, the partial results per row
};

// The workgroup's part of a tile, its wavefronts a share of the tokens each, a step two blocks.  CT: column tiles of 16 pairs, with decoded operands.  FOLD: up to eight pairs, every column twice,
// with codes as operands: a lane of the columns from 8 on takes the second block of a step (the products with keys meet queries in one half of the columns and zeros in the other), so
// that scores, exponentials and weights of two blocks are those of one.
template <int D, int CT, bool FOLD, typename Lds>
__device__ __forceinline__ void attend(Lds &lds, const Task &k, const uint16_t *q, const Paged4Args &pa, float *__restrict__ part, uint16_t *out, int h,
                                       int g)
{
    constexpr int J = D / 32;                    // k steps, words of a lane per block, scales of a token
    constexpr int NT = D / 16;                   // 16-element tiles of O^T
    constexpr int W = Lds::kWaves;
    static_assert(!FOLD || CT == 1, "eight pairs are one column tile");
    typedef uint32_t words_t __attribute__((ext_vector_type(J)));
    typedef _Float16 scales_t __attribute__((ext_vector_type(4 * J)));
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const half2p_t eight = {(_Float16)-8.0f, (_Float16)-8.0f}, one = {(_Float16)1.0f, (_Float16)1.0f};
    const float4p_t none = {0.0f, 0.0f, 0.0f, 0.0f};

    // ---- this wavefront's blocks: its share of the part, in pairs ----
    const int b_begin = (k.t_begin + 15) >> 4, b_end = k.t_end > k.t_begin ? (k.t_end + 15) >> 4 : b_begin;
    const int per = ((b_end - b_begin + 1) / 2 + W - 1) / W * 2;
    const int w_begin = b_begin + wave * per, w_end = min(b_end, w_begin + per);
    const int pos_min = k.past + quotient(k.p0, k.by_rep);

    // ---- lane j: number in the pool of the wavefront's block j; the next 64 when those are done ----
    auto lookup = [&](int seg) __attribute__((always_inline)) {
        int pool = -1;
        if (seg + lane < w_end) {
            pool = paged_block(pa, g, k.kvh, k.slot, seg + lane);
            if (pool < 0) atomicOr(pa.err, kBadPage);
        }
        return pool;
    };
    int pool = lookup(w_begin);

    // ---- queries: lane holds pair `col` of each column tile; k step j takes elements 32 j + 8 quarter .. + 7, in the order of the codes ----
    int pos[CT];
    half8p_t qf[CT][J];                          // FOLD: of the columns below 8, zeros in the others; qg: the other way round
    half8p_t qg[FOLD ? J : 1];
    float qs[FOLD ? J : 1];                      // -8 sum q of a step
    const float c = 1.44269504088896340736f / sqrtf((float)D);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int pair = k.p0 + min(FOLD ? col & 7 : ct * 16 + col, k.n_pairs - 1), row = quotient(pair, k.by_rep), head = k.kvh * k.rep + pair - row * k.rep;
        pos[ct] = k.past + row;
        const uint16_t *src = q + ((size_t)(k.q_start + row) * h + head) * D + quarter * 8;
#pragma unroll
        for (int j = 0; j < J; ++j) qf[ct][j] = *(const half8p_t *)(src + j * 32);
    }
    auto order_queries = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const half8p_t x = qf[ct][j];
                qf[ct][j] = half8p_t{x[0], x[4], x[1], x[5], x[2], x[6], x[3], x[7]};
                if constexpr (FOLD) {
                    float sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += (float)x[e];
                    qs[j] = xor32_sum(xor16_sum(sum)) * -8.0f;
                    const u32x4p_t raw = __builtin_bit_cast(u32x4p_t, qf[ct][j]), zero = {0, 0, 0, 0};
                    qg[j] = __builtin_bit_cast(half8p_t, col < 8 ? zero : raw), qf[ct][j] = __builtin_bit_cast(half8p_t, col < 8 ? raw : zero);
                }
            }
    };

    float4p_t O[CT][NT], off[FOLD ? J : 1];      // off: -8 times the sums of a group's operands
    float m[CT];                                 // the columns' references
    float4p_t l[CT];                             // sums of the weights: the same in all four, FOLD: the lane's own in the first
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = kUnset, l[ct] = none;
#pragma unroll
        for (int i = 0; i < NT; ++i) O[ct][i] = none;
    }
#pragma unroll
    for (int j = 0; j < (FOLD ? J : 1); ++j) off[j] = none;

    words_t kreg[2], vreg[2];
    scales_t ks[FOLD ? 1 : 2], vs[FOLD ? 1 : 2];               // (FOLD: of the lane's block)
    const int k_four = FOLD ? quarter : col >> 2;              // four tokens whose key scales the lane needs: those of its scores or that of its operand
    auto load = [&](words_t (&reg)[2], scales_t (&sc)[FOLD ? 1 : 2], const uint8_t *codes, const uint16_t *scales, int four, int s) __attribute__((always_inline)) {
        size_t at[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            at[t] = max(__builtin_amdgcn_readlane(pool, min(2 * s + t, 63)), 0);       // no such block: any that can be read
            reg[t] = stream_load((const words_t *)(codes + at[t] * block4_codes(D)) + lane);
        }
#pragma unroll
        for (int t = 0; t < (FOLD ? 1 : 2); ++t) sc[t] = *((const scales_t *)(scales + (FOLD ? (col < 8 ? at[0] : at[1]) : at[t]) * block4_scales(D)) + four);
    };
    bool ordered = false;
    for (int seg = w_begin; seg < w_end; seg += kWave) {
        if (seg != w_begin) pool = lookup(seg);
        const int ns = (min(w_end - seg, kWave) + 1) >> 1;
        // loads are issued without a condition, behind the last step the last one's again: behind a branch their number at a wait is not known
        load(kreg, ks, pa.k, pa.k_scale, k_four, 0), load(vreg, vs, pa.v, pa.v_scale, quarter, 0);
        if (!ordered) order_queries(), ordered = true;
        // a step's keys make room for the next one's as soon as the scores are there, its values when they are summed: one step is in flight all the time
        // (two in flight take 40 registers more and lose: 120001 tokens 30.6 us for 29.1)
#pragma unroll 1
        for (int s = 0; s < ns; ++s) {
            const int t0 = (seg + 2 * s) * 16;                 // first token of the step
            const bool there[2] = {__builtin_amdgcn_readlane(pool, min(2 * s, 63)) >= 0, __builtin_amdgcn_readlane(pool, min(2 * s + 1, 63)) >= 0};
            const bool gone = !there[0] || !there[1] || t0 + 31 > pos_min;      // uniform: some of the tokens are masked
            // the first token that the lane has a score of in (its) block t, and whether there is the block
            const auto first = [&](int t) { return t0 + 16 * (FOLD ? col >> 3 : t) + 4 * quarter; };
            const auto have = [&](int t) { return FOLD ? (col < 8 ? there[0] : there[1]) : there[t]; };
            const auto clean_scales = [&]() __attribute__((always_inline)) {    // a scale behind the last token, or of no block, is anything, and a weight of zero would not hide a NaN
#pragma unroll
                for (int t = 0; t < (FOLD ? 1 : 2); ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!have(t) || first(t) + i >= k.t_end)
#pragma unroll
                            for (int j = 0; j < J; ++j) vs[t][4 * j + i] = (_Float16)0.0f;
            };
            if constexpr (FOLD) {
                float4p_t S[J];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        half2p_t p[4];
                        word_codes(kreg[t][j], p);
                        S[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(p[0], p[1], p[2], p[3]), t ? qg[j] : qf[0][j], t ? S[j] : float4p_t{qs[j], qs[j], qs[j], qs[j]}, 0, 0, 0);
                    }
                float x[4], w[4];                              // scores over c, weights
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = fmaf(S[0][i], (float)ks[0][i], 0.0f);       // (as a multiply-add of mixed types: a product would convert its scale first)
#pragma unroll
                    for (int j = 1; j < J; ++j) x[i] = fmaf(S[j][i], (float)ks[0][4 * j + i], x[i]);
                }
                if (gone) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!have(0) || first(0) + i > pos[0]) x[i] = -INFINITY;
                }
                load(kreg, ks, pa.k, pa.k_scale, k_four, min(s + 1, ns - 1));
                if (gone) clean_scales();
                float square = kLeast2;                        // of the lane's scales: each is below the root
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const half2p_t two = {vs[0][4 * j + i], vs[0][4 * j + i + 1]};
                        square = __builtin_amdgcn_fdot2(two, two, square, false);
                    }
                const float level = 0.5f * __builtin_amdgcn_logf(square), mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), top = fmaf(mx, c, -m[0]) + level;      // above log2 of weights times scales
                if (__any(top > kHead)) {                      // rare behind the first tokens; every column is new there
                    const float high = column_max(fmaxf(top, lane_xor<8>(top))), at = fmaf(mx, c, level), near = column_max(fmaxf(at, lane_xor<8>(at))) - kBias;
                    // a column moves by itself: no row depends on the others of its tile.  (A little too far: by more than the rounding of a large reference, which would put it below)
                    const float to = high > kHead ? fmaf(fabsf(near), 0x1p-22f, near) : m[0], alpha = __builtin_amdgcn_exp2f(m[0] - to);
                    m[0] = to, l[0][0] *= alpha;
#pragma unroll
                    for (int i = 0; i < NT; ++i) O[0][i] *= alpha;
#pragma unroll
                    for (int j = 0; j < J; ++j) off[j] *= alpha;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c, -m[0])), l[0][0] += w[i];
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    half2p_t a[4], e[4], pw[4];                // pw: the weights of both blocks times their scales, tokens 0 2 | 1 3
                    word_codes(vreg[0][j], a);
                    word_codes(vreg[1][j], e);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float lo = fmaf(w[i], (float)vs[0][4 * j + i], 0.0f), hi = fmaf(w[i + 2], (float)vs[0][4 * j + i + 2], 0.0f);
                        asm("" : "+v"(lo), "+v"(hi));          // (the products in fp32 and one conversion of both: multiply-adds that write a half take twice the time)
                        pw[i] = half2p_t{(_Float16)lo, (_Float16)hi};
                        pw[2 + i] = __builtin_bit_cast(half2p_t, lane_xor<8>(__builtin_bit_cast(float, pw[i])));      // (columns from 8 on have the blocks the other way round, and no pair)
                    }
                    const half8p_t pf = operand(pw[0], pw[1], pw[2], pw[3]);
                    O[0][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(a[0], a[1], e[0], e[1]), pf, O[0][2 * j], 0, 0, 0);
                    O[0][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(a[2], a[3], e[2], e[3]), pf, O[0][2 * j + 1], 0, 0, 0);
                    off[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(eight, eight, eight, eight), pf, off[j], 0, 0, 0);
                }
            } else {
                float4p_t S[2][CT];                            // scores over c
                const uint32_t own = 0x01000100u + (lane & 3) * 0x02020202u;   // bytes of the lane's token of four, twice
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const uint32_t lo = __builtin_bit_cast(uint32_t, half2p_t{ks[t][4 * j], ks[t][4 * j + 1]}), hi = __builtin_bit_cast(uint32_t, half2p_t{ks[t][4 * j + 2], ks[t][4 * j + 3]});
                        const half2p_t scale = __builtin_bit_cast(half2p_t, __builtin_amdgcn_perm(hi, lo, own)), zero_point = scale * eight;
                        half2p_t p[4];
                        word_codes(kreg[t][j], p);
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[e] = __builtin_elementwise_fma(p[e], scale, zero_point);
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct)
                            S[t][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(p[0], p[1], p[2], p[3]), qf[ct][j], j ? S[t][ct] : none, 0, 0, 0);
                    }
                load(kreg, ks, pa.k, pa.k_scale, k_four, min(s + 1, ns - 1));
                if (gone) {
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (!have(t) || first(t) + i > pos[ct]) S[t][ct][i] = -INFINITY;
                }
                half8p_t pf[CT];
                const auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i)        // tokens 0 2 1 3, as the values lie
                                pf[ct][4 * t + (i & 1) * 2 + (i >> 1)] = (_Float16)__builtin_amdgcn_exp2f(fmaf(S[t][ct][i], c, kPackedBias - m[ct]));
                };
                weights();
                // The weights were computed against the reference as it was.  Where one is about to leave fp16's range (or every column is new) the reference moves to the
                // maximum of these scores: rare behind the first tokens, and a look at the packed weights costs a quarter of the maxima of the scores.
                half2p_t top = {(_Float16)0.0f, (_Float16)0.0f};
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, half2p_t{pf[ct][2 * i], pf[ct][2 * i + 1]});
                if (__any(fmaxf((float)top.x, (float)top.y) > kMost)) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        float mx = -INFINITY, most = 0.0f;     // a column moves by itself: no row depends on the others of its tile
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, S[t][ct][i] * c), most = fmaxf(most, (float)pf[ct][4 * t + i]);
                        mx = column_max(mx), most = column_max(most);
                        const float to = most > kMost && mx > m[ct] ? mx : m[ct], alpha = __builtin_amdgcn_exp2f(m[ct] - to);
                        m[ct] = to, l[ct] *= alpha;
#pragma unroll
                        for (int i = 0; i < NT; ++i) O[ct][i] *= alpha;
                    }
                    weights();
                }
                if (gone) clean_scales();
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    half2p_t a[2][4];
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        word_codes(vreg[t][j], a[t]);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {          // tokens i and i + 2
                            const half2p_t scale = {vs[t][4 * j + i], vs[t][4 * j + i + 2]}, zero_point = scale * eight;
                            a[t][i] = __builtin_elementwise_fma(a[t][i], scale, zero_point), a[t][2 + i] = __builtin_elementwise_fma(a[t][2 + i], scale, zero_point);
                        }
                    }
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        O[ct][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(a[0][0], a[0][1], a[1][0], a[1][1]), pf[ct], O[ct][2 * j], 0, 0, 0);
                        O[ct][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(a[0][2], a[0][3], a[1][2], a[1][3]), pf[ct], O[ct][2 * j + 1], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(one, one, one, one), pf[ct], l[ct], 0, 0, 0);
            }
            load(vreg, vs, pa.v, pa.v_scale, quarter, min(s + 1, ns - 1));
        }
    }

#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int at = wave * Lds::kPairs + (FOLD ? col & 7 : ct * 16 + col);
        float den = l[ct][0];
        if constexpr (FOLD) den = xor32_sum(xor16_sum(den + lane_xor<8>(den)));
        if (FOLD && col >= 8) continue;
#pragma unroll
        for (int i = 0; i < NT; ++i) *(float4p_t *)(lds.o + at * Lds::kPitch + i * 16 + quarter * 4) = FOLD ? O[ct][i] + off[FOLD ? i >> 1 : 0] : O[ct][i];
        if (quarter == 0) lds.m[at] = m[ct], lds.l[at] = den;
    }

    // ---- the wavefronts' states meet: T threads per pair, E times four elements each ----
    __syncthreads();
    constexpr int TW = FOLD ? 8 : 16 * CT, T = 64 * W / TW, E = D / 4 / T > 0 ? D / 4 / T : 1;
    const int pc = tid / T, e0 = tid % T * 4;
    if (pc >= k.n_pairs || e0 >= D) return;
    float mw[W], lw[W], mm = -INFINITY, den = 0.0f;
    float4p_t num[E], o[W][E];
#pragma unroll
    for (int w = 0; w < W; ++w) {
        mw[w] = lds.m[w * Lds::kPairs + pc], lw[w] = lds.l[w * Lds::kPairs + pc];
#pragma unroll
        for (int i = 0; i < E; ++i) o[w][i] = *(const float4p_t *)(lds.o + (w * Lds::kPairs + pc) * Lds::kPitch + e0 + i * 4 * T);
    }
#pragma unroll
    for (int w = 0; w < W; ++w) mm = fmaxf(mm, mw[w]);
#pragma unroll
    for (int i = 0; i < E; ++i) num[i] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const float f = __builtin_amdgcn_exp2f(mw[w] - mm);
        den += lw[w] * f;
#pragma unroll
        for (int i = 0; i < E; ++i) num[i] += o[w][i] * f;
    }
    const int pr = quotient(k.p0 + pc, k.by_rep);
    const size_t at = (size_t)(k.q_start + pr) * h + k.kvh * k.rep + k.p0 + pc - pr * k.rep;
    if (k.used > 1) {
        float *dst = part + (at * k.splits + k.split) * (D + 2);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            float2 *d2 = (float2 *)(dst + e0 + i * 4 * T);
            d2[0] = make_float2(num[i].x, num[i].y), d2[1] = make_float2(num[i].z, num[i].w);
        }
        if (e0 == 0) *(float2 *)(dst + D) = make_float2(mm, den);
    } else {
        const float inv = den > 0.0f ? 1.0f / den : den;       // a row that no token is left for is zeros; a NaN stays one
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float4p_t r = num[i] * inv;
            *(u32x2p_t *)(out + at * D + e0 + i * 4 * T) = u32x2p_t{f2h(r.x) | (uint32_t)f2h(r.y) << 16, f2h(r.z) | (uint32_t)f2h(r.w) << 16};
        }
    }
}

// grid: item * g + KV head, an item being a part of a tile (the tiles of a part side by side: they read the same tokens).  per_seq: as tile_of takes it.  part: [row][head][splits][D + 2], of
// rows that have more than one part.  FEW: no sequence has more than eight pairs; three wavefronts per SIMD (64 sequences of 100 to 730 tokens, 32 / 32 heads: 28.0 us for 31.2 with two; the fewest
// sequences as before).
struct Grid {
    int h, g, rep, per_seq, chunk, splits, least;
    Divisor by_g, by_rep, by_per_seq, by_chunk;
};
template <int D, bool FEW, int W>
__global__ __launch_bounds__(64 * W, FEW ? 3 : 2) void attn_paged4_kernel(PagedSeqs, const uint16_t *q, Paged4Args pa, float *__restrict__ part, uint16_t *out, Grid gr)
{
    __shared__ __align__(16) States<D, FEW ? 8 : kTile, W> lds;
    const int rep = gr.rep, item = quotient(blockIdx.x, gr.by_g), kvh = (int)blockIdx.x - item * gr.g;
    const SeqsArg st = seqs_arg();
    const auto tiles_of = [&](int q_len) { return q_len * rep < gr.least ? (q_len * rep + kTile - 1) / kTile : 0; };
    const auto parts_of = [&](int kv_len) { return min(max(quotient(kv_len + gr.chunk - 1, gr.by_chunk), 1), gr.splits); };
    int place = item, b = 0;
    if (gr.per_seq > 0) b = quotient(item, gr.by_per_seq), place = item - b * gr.per_seq;
    else b = seq_at(st, item, [&](int j) { return st->dev ? tiles_of(st->dev[st->B + j]) * gr.splits : tiles_of(st->q_len[j]) * parts_of(st->kv_len[j]); }, place);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, __builtin_amdgcn_readfirstlane(b));
    const int pairs = si.q_len * rep, tiles = tiles_of(si.q_len), split = tiles > 1 ? place / tiles : place, p0 = (tiles > 1 ? place - split * tiles : 0) * kTile;
    if (tiles == 0) return;
    const int n_pairs = min(kTile, pairs - p0);
    const bool beyond = beyond_capacity(si, pa.cap);
    const int past = beyond ? 0 : si.kv_len - si.q_len;
    const int vis = beyond ? 0 : past + quotient(p0 + n_pairs - 1, gr.by_rep) + 1;      // tokens that any of the pairs attends to
    // the tile's tokens in equal parts, as many as the sequence has chunks (more than the host's bound gives makes them longer)
    const int used = beyond ? 1 : parts_of(si.kv_len);
    if (split >= used) return;
    const int share = used == 1 ? vis : ((vis + used - 1) / used + 31) & ~31, t_begin = min(split * share, vis), t_end = min(vis, t_begin + share);
    if (beyond && threadIdx.x == 0) atomicOr(pa.err, kBadPage);
    const Task task = {si.q_start, si.slot, past, kvh, p0, n_pairs, t_begin, t_end, rep, gr.by_rep, used, split, gr.splits};
    if (FEW || n_pairs <= 8) attend<D, 1, true>(lds, task, q, pa, part, out, gr.h, gr.g);
    else if constexpr (!FEW) n_pairs <= 16 ? attend<D, 1, false>(lds, task, q, pa, part, out, gr.h, gr.g) : attend<D, 2, false>(lds, task, q, pa, part, out, gr.h, gr.g);
}

// Estimated times, us, fitted to 46 calls with up to 40 cuts each, of which they choose one that is 0.7 % behind the best in the mean and 12 % at most.  kGroupUs: a workgroup's beginning and end, with
// one, four and eight wavefronts (kWideGroupUs: with four and eight, where a sequence has more than 16 pairs); kStepUs: a step of 32 tokens with up to three wavefronts on a SIMD (kWideStepUs: up to
// two); heads of 64: times kHalfHead.  kTail: the share of the longest workgroup that comes on top when there are more of them than at a time.  A merge, and each of its partial results; the
// cache's bytes.
// One wavefront alone has no states to merge and the shortest end, which counts when there are several rounds of workgroups: 128 sequences of 20 to 530 tokens, 32 / 32 heads, 32.9 us for 40.8 with four;
// two are between them (never more than 12 % better than the best of the others) and are not built.
constexpr int kWaves[3] = {1, 4, 8};
constexpr float kGroupUs[3] = {3.0f, 3.5f, 5.4f}, kWideGroupUs[3] = {0.0f, 3.2f, 7.1f}, kStepUs[3] = {0.96f, 1.14f, 1.19f}, kWideStepUs[2] = {1.1f, 1.11f}, kHalfHead = 0.89f, kTail = 0.15f, kMergeUs = 3.45f,
                kMergeResultUs = 3.2e-4f, kBytesUs = 5.9f, kBytesPerUs = 7.0e6f;
// Tiles of 256 pairs over all KV heads from which the kernel of such tiles is faster: it has 256 workgroups at a time, each as slow alone as beside 255 others (us, these tiles / those: 1200 rows on 600
// cached tokens of 32 / 8 heads, 150 tiles, 52.7 / 59.7; 1600 rows, 200, 51.7 / 54.4 and on 600 cached tokens 76.2 / 71.4; 2043 rows, 255, 71.6 / 66.0; 4096 rows, 512, 227 / 141)
constexpr int kRowTiles = 200;
constexpr int kLeast = 128;                      // tokens of a part

// How the tiles are cut: a sequence of L tokens into ceil(L / chunk) equal parts
struct Cut {
    int64_t items;                   // parts of tiles
    int32_t chunk, splits;           // splits: the most parts of a sequence
    int32_t per_seq;                 // parts of every sequence, 0: not alike
    int32_t rows;                    // rows of sequences that have more than one part
    int32_t waves;                   // wavefronts per workgroup
    bool few;                        // no sequence has more than eight pairs
};
Cut cut(const PagedPlan &pl, const relax_layer_dims &dm, const PagedSeqs &st, const relax_seqs &sq, int32_t L_max)
{
    const int rep = dm.n_heads / dm.n_kv_heads, g = dm.n_kv_heads;
    const auto tiles_of = [&](int b) {
        const int64_t pairs = (int64_t)sq.q_lens[b] * rep;
        return pairs < pl.least ? (pairs + kTile - 1) / kTile : 0;
    };
    int64_t tiles = 0, tokens = 0, most = 0;
    float unique = 0.0f;
    for (int b = 0; b < sq.B; ++b) {
        const int64_t t = tiles_of(b);
        tiles += t, tokens += t * sq.kv_lens[b];
        if (t) most = std::max(most, (int64_t)sq.q_lens[b] * rep), unique += (float)sq.kv_lens[b];
    }
    const float bytes_us = kBytesUs + unique * (float)(g * 2 * (block4_codes(dm.head_dim) + 2 * block4_scales(dm.head_dim)) / 16) / kBytesPerUs;
    const float head = dm.head_dim == 64 ? kHalfHead : 1.0f;
    int32_t waves = 4;
    int64_t chunk = std::max<int64_t>(32, ((int64_t)L_max + 31) & ~31);
    float best = INFINITY;
    const auto up = [](float x) { return (float)(int32_t)(x + 0.9999f); };      // (ceilf is a function call here: 1 us of a call's host time with 64 sequences)
    // takes parts of up to c tokens if they are estimated to be faster than what was considered before.  Workgroups at a time: what three wavefronts per SIMD make of one and of four, two of eight;
    // with more than eight pairs two wavefronts per SIMD, and not one alone
    const bool few = most <= 8;
    const float slots[3] = {12.0f * 256.0f, few ? 3.0f * 256.0f : 2.0f * 256.0f, 256.0f};
    const auto consider = [&](int64_t c) {
        const float by_c = 1.0f / (float)c;
        float groups = 0.0f, merged = 0.0f, wide_groups = 0.0f;
        float steps[3] = {0.0f, 0.0f, 0.0f}, wide_steps[3] = {0.0f, 0.0f, 0.0f}, most_steps[3] = {0.0f, 0.0f, 0.0f}, most_wide[3] = {0.0f, 0.0f, 0.0f};
        for (int b = 0; b < sq.B; ++b) {
            const float t = (float)tiles_of(b), L = (float)sq.kv_lens[b];
            if (t == 0.0f) continue;
            const float parts = std::max(up(L * by_c), 1.0f), share = parts == 1.0f ? L : L / parts, k = t * parts;
            const bool wide = (int64_t)sq.q_lens[b] * rep > 16;
            for (int w = few ? 0 : 1; w < 3; ++w) {
                const float n = up(share * (1.0f / (float)(32 * kWaves[w])));
                if (wide) wide_steps[w] += n * k, most_wide[w] = std::max(most_wide[w], n);
                else steps[w] += n * k, most_steps[w] = std::max(most_steps[w], n);
            }
            groups += k;
            if (wide) wide_groups += k;
            if (parts > 1.0f) merged += (float)sq.q_lens[b] * parts;
        }
        const float all = groups * (float)g;
        for (int w = few ? 0 : 1; w < 3; ++w) {
            const float on_simd = all * (float)kWaves[w] * (1.0f / 1024.0f);
            const int n = on_simd <= 1.0f ? 0 : on_simd <= 2.0f || !few || w == 2 ? 1 : 2;
            const float step = kStepUs[n] * head, wide_step = kWideStepUs[std::min(n, 1)] * head;
            const float longest = std::max(most_steps[w] > 0.0f ? kGroupUs[w] + most_steps[w] * step : 0.0f, most_wide[w] > 0.0f ? kWideGroupUs[w] + most_wide[w] * wide_step : 0.0f);
            const float total = (groups - wide_groups) * kGroupUs[w] + steps[w] * step + wide_groups * kWideGroupUs[w] + wide_steps[w] * wide_step;
            float us = all <= slots[w] ? longest : total * (float)g / slots[w] + kTail * longest;
            us = std::max(us, bytes_us) + (merged > 0.0f ? kMergeUs + kMergeResultUs * merged * (float)dm.n_heads : 0.0f);
            if (us < best) best = us, chunk = c, waves = kWaves[w];
        }
    };
    consider(chunk);
    // From 2048 workgroups on no cut has been estimated to be faster (us, with the search / without: 64 sequences of 800 tokens, 32 / 32 heads, 41.9 / 42.2; 128 of 300 to 935 71.5 / 71.7), and the
    // search is host time
    if (tiles * g < 2048) {
        const int64_t most_parts = std::max<int64_t>(1, kPagedPartials / ((int64_t)st.n * dm.n_heads)), least = (std::max<int64_t>(kLeast, L_max / most_parts + 1) + 31) & ~31;
        for (int parts = 2; parts <= (sq.B <= 4 ? 64 : sq.B <= 24 ? 16 : 4); parts += parts < 4 ? 1 : parts / 2) {
            const int64_t c = (L_max / parts + 32) & ~31;
            if (c >= least) consider(c);
        }
        const int64_t even = (tokens * g / 512 + 32) & ~31;    // as many parts as workgroups at a time, for sequences alike
        if (even >= least && even < L_max) consider(even);
    }
    Cut c = {0, (int32_t)chunk, (int32_t)((L_max + chunk - 1) / chunk), -1, 0, waves, few};
    for (int b = 0; b < sq.B; ++b) {
        const int64_t parts = st.dev ? c.splits : (sq.kv_lens[b] + chunk - 1) / chunk, items = tiles_of(b) * parts;
        c.items += items;
        if (parts > 1) c.rows += sq.q_lens[b];
        if (c.per_seq < 0) c.per_seq = (int32_t)std::min<int64_t>(items, INT32_MAX);
        else if (c.per_seq != items) c.per_seq = 0;
    }
    return c;
}

// The sequences in order of their lengths, longest first, where they are in the arguments: the workgroups that take longest begin first
void longest_first(PagedSeqs &st)
{
    if (st.dev || st.B < 2) return;
    struct Entry {
        int32_t kv_len, b;
    } order[kPagedInline];
    bool sorted = true;
    for (int b = 0; b < st.B; ++b) order[b] = {st.kv_len[b], b}, sorted = sorted && (b == 0 || st.kv_len[b] <= st.kv_len[b - 1]);
    if (sorted) return;
    std::sort(order, order + st.B, [](const Entry &x, const Entry &y) { return x.kv_len != y.kv_len ? x.kv_len > y.kv_len : x.b < y.b; });
    int32_t from[3][kPagedInline];
    for (int b = 0; b < st.B; ++b) from[0][b] = st.q_start[b], from[1][b] = st.q_len[b], from[2][b] = st.slot[b];
    for (int b = 0; b < st.B; ++b) {
        const int i = order[b].b;
        st.q_start[b] = from[0][i], st.q_len[b] = from[1][i], st.slot[b] = from[2][i], st.kv_len[b] = order[b].kv_len;
    }
}

// out from the parts of the rows that have more than one: T * G threads per (row, head), a thread four elements of every G-th part.  The first F of them are asked for before the number of parts is
// known (there is memory for all that a row could have), so that they do not wait for the descriptor.  all: every row of the call, in its order; else the first rows of st's sequences.
template <int D, int G>
__global__ __launch_bounds__(256) void attn_paged4_merge_kernel(PagedSeqs, const float *__restrict__ part, uint16_t *out, Grid gr, Divisor by_h, int count, int cap, int all)
{
    constexpr int T = D / 4, F = 4, P = 256 / (T * G);
    __shared__ __align__(16) float sums[P][G][D];
    __shared__ float sm_m[P][G], sm_l[P][G];
    const SeqsArg st = seqs_arg();
    const int tid = threadIdx.x, p = __builtin_amdgcn_readfirstlane(tid / (T * G)), grp = tid / T % G, e = tid % T * 4;
    const int idx = min((int)blockIdx.x * P + p, count - 1), r = quotient(idx, by_h), hd = idx - r * gr.h;
    float ms[F], ls[F];
    float4p_t as[F];
    const auto load = [&](const float *src, int s0, int most) {
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const float2 *q2 = (const float2 *)(src + (size_t)min(s0 + j * G, most) * (D + 2));
            const float2 lo = q2[e / 2], hi = q2[e / 2 + 1], ml = q2[D / 2];
            ms[j] = ml.x, ls[j] = ml.y, as[j] = float4p_t{lo.x, lo.y, hi.x, hi.y};
        }
    };
    size_t at = idx;
    if (all) load(part + at * gr.splits * (D + 2), grp, gr.splits - 1);
    int place = 0, b = r;
    if (st->q_max != 1) b = seq_of(st, r, [](int q_len) { return q_len; }, place);
    const SeqSpan si = seq_span(st, __builtin_amdgcn_readfirstlane(min(b, st->B - 1)));
    if (!all) {
        at = (size_t)(si.q_start + place) * gr.h + hd;
        load(part + at * gr.splits * (D + 2), grp, gr.splits - 1);
    }
    const int used = beyond_capacity(si, cap) || si.q_len * gr.rep >= gr.least ? 1 : min(max(quotient(si.kv_len + gr.chunk - 1, gr.by_chunk), 1), gr.splits);
    float mm = -INFINITY, den = 0.0f;
    float4p_t num = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = grp;;) {
        float mx = mm;
#pragma unroll
        for (int j = 0; j < F; ++j) mx = s0 + j * G < used ? fmaxf(mx, ms[j]) : mx;
        const float ref = mx == -INFINITY ? 0.0f : mx, f0 = __builtin_amdgcn_exp2f(mm - ref);
        den *= f0, num *= f0;
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const bool there = s0 + j * G < used;              // (memory that no part was written to may hold anything)
            const float f = there ? __builtin_amdgcn_exp2f(ms[j] - ref) : 0.0f;
            den += there ? ls[j] * f : 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) num[i] += there ? as[j][i] * f : 0.0f;
        }
        mm = mx;
        s0 += G * F;
        if (s0 - grp >= used) break;                           // uniform
        load(part + at * gr.splits * (D + 2), s0, used - 1);
    }
    *(float4p_t *)&sums[p][grp][e] = num;
    if (e == 0) sm_m[p][grp] = mm, sm_l[p][grp] = den;
    __syncthreads();
    if (grp > 0 || used <= 1 || (int)blockIdx.x * P + p >= count) return;      // (one part: written already)
#pragma unroll
    for (int w = 0; w < G; ++w) mm = fmaxf(mm, sm_m[p][w]);
    num = float4p_t{0.0f, 0.0f, 0.0f, 0.0f}, den = 0.0f;
#pragma unroll
    for (int w = 0; w < G; ++w) {
        const float f = sm_m[p][w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_m[p][w] - mm);
        num += *(const float4p_t *)&sums[p][w][e] * f, den += sm_l[p][w] * f;
    }
    const float inv = den > 0.0f ? 1.0f / den : den;
    const uint32_t lo = f2h(num.x * inv) | (uint32_t)f2h(num.y * inv) << 16, hi = f2h(num.z * inv) | (uint32_t)f2h(num.w * inv) << 16;
    *(u32x2p_t *)(out + at * D + e) = u32x2p_t{lo, hi};
}

template <int D>
hipError_t launch_d(const uint16_t *q, const Paged4Args &pa, const relax_layer_dims &dm, const PagedSeqs &call, const PagedSeqs &st, const PagedPlan &pl, const Cut &c, uint16_t *out, float *partials,
                    hipStream_t stream)
{
    if (c.items * dm.n_kv_heads * 64 * c.waves > kMaxThreads) return hipErrorInvalidValue;
    const dim3 grid(c.items * dm.n_kv_heads);
    const int rep = dm.n_heads / dm.n_kv_heads;
    const Grid gr = {dm.n_heads, dm.n_kv_heads, rep, c.per_seq, c.chunk, c.splits, pl.least, divisor(dm.n_kv_heads), divisor(rep), divisor(std::max(c.per_seq, 1)), divisor(c.chunk)};
    const auto launch = [&](auto FEW, auto W) {
        hipLaunchKernelGGL((attn_paged4_kernel<D, FEW, W>), grid, dim3(64 * W), 0, stream, st, q, pa, partials, out, gr);
    };
    using four = std::integral_constant<int, 4>;
    using eight = std::integral_constant<int, 8>;
    if (c.waves == 1) launch(std::true_type{}, std::integral_constant<int, 1>{});
    else if (c.waves == 8) c.few ? launch(std::true_type{}, eight{}) : launch(std::false_type{}, eight{});
    else c.few ? launch(std::true_type{}, four{}) : launch(std::false_type{}, four{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.rows == 0) return e;
    const int all = c.rows == st.n, count = c.rows * dm.n_heads;
    const PagedSeqs &rows = all ? call : st;
    const auto merge = [&](auto G) {
        constexpr int P = 256 / (D / 4 * G);
        hipLaunchKernelGGL((attn_paged4_merge_kernel<D, G>), dim3((count + P - 1) / P), dim3(256), 0, stream, rows, partials, out, gr, divisor(dm.n_heads), count, pa.cap, all);
    };
    // threads that share a row's parts, four times as many or fewer (us of the call: one row of 64 / 8 heads with 28 parts 30.6 / 32.1, with nine 7.7 / 8.1; 16 rows of them with up to six parts
    // 24.1 / 23.3, 25 rows of 32 / 8 heads with two 32.0 / 31.1: many parts are few rows)
    if (c.splits > 16) merge(std::integral_constant<int, 1024 / D>{});
    else merge(std::integral_constant<int, 256 / D>{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged4_attention(const uint16_t *q, const Paged4Args &pa, const relax_layer_dims &dm, const PagedSeqs &st, const relax_seqs &sq, int32_t L_max,
                                   uint16_t *out, float *partials, hipStream_t stream)
{
    const PagedPlan pl = paged_plan(dm, sq, st.n, L_max, kRowTiles);
    if (pl.row_items > 0) {
        const hipError_t e = launch_paged4_rows(q, pa, dm, st, pl, out, stream);
        if (e != hipSuccess || pl.items == 0) return e;
    }
    const Cut c = cut(pl, dm, st, sq, L_max);
    PagedSeqs by_length = st;
    longest_first(by_length);
    return dm.head_dim == 128 ? launch_d<128>(q, pa, dm, st, by_length, pl, c, out, partials, stream) : launch_d<64>(q, pa, dm, st, by_length, pl, c, out, partials, stream);
}

}  // namespace relax
