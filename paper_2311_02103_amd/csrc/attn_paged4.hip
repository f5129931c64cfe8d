// Causal attention over the paged 4-bit KV cache.
//
//   o[i] = sum_t p[i,t] v[t],   p[i,:] = softmax_t(q[i] . k[t] / sqrt d),  t = 0 .. pos_i,   k[t][e] = s_k[t][e / 32] (u_k[t][e] - 8), v likewise
//
// Tiles, splits and the merge of partial results are those of attn_paged.hip: 16 consecutive (row, head) pairs against one KV head and one split of the
// tokens, S^T = K Q^T and O^T = V^T P^T, so that a pair is a column, a lane (quarter, column) of the scores holds tokens 4 quarter .. + 3 of a
// block, and the lane's eight probabilities of two blocks are what the second product wants from it.
//
// Codes go into both products as fp16 integers 0..15 (paged4_device.h).
// Scores.  A scale is constant over a k step of 32 elements, so a step is a product of its own, S_j = sum u q, and x = sum_j s_kj S_j.  The accumulator of S_j starts at
// -8 sum q, which takes the codes' offset off.
// Values.  The weight of a token times its value scale, w s_j, is rounded to fp16 once per group of 32 elements and is the operand; -8 sum (w s_j), from one more product
// per group, goes to the result.  Weights are exp2(score - reference + 1) with a reference that trails the maximum by at most 2: at most 8, and times 8160,
// the largest scale, an fp16 number.  The smallest ones lose bits: 2^-25 absolute, at most 2^-26 of the largest weight, per code.
#include <type_traits>

#include "paged4_device.h"

namespace relax {

namespace {

constexpr float kBias = 1.0f, kLag = 2.0f;       // log2: weight at the reference, and how far the reference may trail the maximum

typedef _Float16 half4p_t __attribute__((ext_vector_type(4)));

// largest of a value over the four lanes of a column
__device__ __forceinline__ float column_max(float v)
{
    float2 both = pair_xor16(v);
    both = pair_xor32(fmaxf(both.x, both.y));
    return fmaxf(both.x, both.y);
}

// grid: x = tile * g + KV head, y = split.  part: [row][head][splits][D + 2] when splits > 1.
template <int D, int W, bool FOLD>
__global__ __launch_bounds__(64 * W, FOLD ? 3 : 2) void attn_paged4_kernel(PagedSeqs, const uint16_t *__restrict__ q, Paged4Args pa, float *__restrict__ part,
                                                             uint16_t *__restrict__ out, int h, int g, int per_seq, int chunk, int splits, int least)
{
    constexpr int J = D / 32;                    // k steps, words of a lane per block, scales of a token
    constexpr int NT = D / 16;                   // 16-element tiles of O^T
    constexpr int P = D + 4;                     // pitch of a state in LDS
    constexpr int SB = FOLD ? 1 : 2;             // blocks of a step whose scores a lane holds
    typedef uint32_t words_t __attribute__((ext_vector_type(J)));
    typedef _Float16 scales_t __attribute__((ext_vector_type(4 * J)));
    __shared__ __align__(16) float states[W * 16 * P];
    __shared__ float sm_m[W * 16], sm_l[W * 16];

    const int rep = h / g, item = (int)blockIdx.x / g, kvh = (int)blockIdx.x - item * g, split = blockIdx.y;
    const SeqsArg st = seqs_arg();
    int tile;
    const int b = tile_of(st, item, per_seq, [&](int q_len) { return q_len * rep < least ? (q_len * rep + 15) >> 4 : 0; }, tile);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, __builtin_amdgcn_readfirstlane(b));
    const int pairs = si.q_len * rep, p0 = tile * 16;
    if (pairs >= least || p0 >= pairs) return;
    const int n_pairs = min(16, pairs - p0);
    const bool beyond = beyond_capacity(si, pa.cap);
    const int past = beyond ? 0 : si.kv_len - si.q_len;
    const int pos_min = past + p0 / rep, vis = beyond ? 0 : past + (p0 + n_pairs - 1) / rep + 1;      // tokens that any of the pairs attends to
    const int t_begin = split * chunk;
    if (split > 0 && t_begin >= vis) return;
    if (beyond && threadIdx.x == 0) atomicOr(pa.err, kBadPage);
    const int t_end = split + 1 == splits ? vis : min(vis, t_begin + chunk);      // the last split takes what a device table holds beyond the host's bound
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, quarter = lane >> 4;

    // ---- this wavefront's blocks: its share of the split, in pairs ----
    const int b_begin = t_begin >> 4, b_end = t_end > t_begin ? (t_end + 15) >> 4 : b_begin;
    const int per = ((b_end - b_begin + 1) / 2 + W - 1) / W * 2;
    const int w_begin = b_begin + wave * per, w_end = min(b_end, w_begin + per);

    // ---- queries: lane holds pair `col`; k step j takes elements 32 j + 8 quarter .. + 7, in the order of the codes ----
    const int pair = p0 + min(FOLD ? col & 7 : col, n_pairs - 1), row = pair / rep, head = kvh * rep + pair - row * rep, pos = past + row;
    half8p_t qf[J];
    float qs[J];                                 // -8 sum q of a step
    const float c = 1.44269504088896340736f / sqrtf((float)D);
    {
        const uint16_t *src = q + ((size_t)(si.q_start + row) * h + head) * D + quarter * 8;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const half8p_t x = *(const half8p_t *)(src + j * 32);
            qf[j] = half8p_t{x[0], x[4], x[1], x[5], x[2], x[6], x[3], x[7]};
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += (float)x[e];
            qs[j] = xor32_sum(xor16_sum(sum)) * -8.0f;
        }
    }

    float4p_t O[NT], off[J];                     // off: -8 times the sums of a group's operands
#pragma unroll
    for (int i = 0; i < NT; ++i) O[i] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < J; ++j) off[j] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
    float m_run = -INFINITY, l_run = 0.0f;

    for (int seg = w_begin; seg < w_end; seg += kWave) {
        // ---- lane j: number in the pool of block seg + j ----
        int pool = -1;
        if (seg + lane < w_end) {
            pool = paged_block(pa, g, kvh, si.slot, seg + lane);
            if (pool < 0) atomicOr(pa.err, kBadPage);
        }
        const int ns = (min(w_end - seg, kWave) + 1) >> 1;
        words_t kreg[2], vreg[2];                              // one step: two blocks
        scales_t ks[SB], vs[SB];                               // (FOLD: of the lane's block)
        auto load = [&](words_t (&reg)[2], scales_t (&sc)[SB], const uint8_t *codes, const uint16_t *scales, int s) __attribute__((always_inline)) {
            size_t at[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                at[t] = max(__builtin_amdgcn_readlane(pool, min(2 * s + t, 63)), 0);       // no such block: any that can be read
                reg[t] = stream_load((const words_t *)(codes + at[t] * block4_codes(D)) + lane);
            }
#pragma unroll
            for (int t = 0; t < SB; ++t) sc[t] = *((const scales_t *)(scales + (FOLD ? (col < 8 ? at[0] : at[1]) : at[t]) * block4_scales(D)) + quarter);
        };
        load(kreg, ks, pa.k, pa.k_scale, 0), load(vreg, vs, pa.v, pa.v_scale, 0);
        // a step's keys make room for the next one's as soon as the scores are there, its values when they are summed: one step is in flight all the time
        auto step = [&](int s, auto MORE) __attribute__((always_inline)) {
            float x[4 * SB];                                   // scores over c
            float4p_t S[2][J];
            const int t0 = (seg + 2 * s) * 16;                 // first token of the step
            const bool there0 = __builtin_amdgcn_readlane(pool, min(2 * s, 63)) >= 0, there1 = __builtin_amdgcn_readlane(pool, min(2 * s + 1, 63)) >= 0;
            const bool gone = !there0 || !there1 || t0 + 31 > pos_min;      // uniform: some of the tokens are masked
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    half2p_t p[4];
                    word_codes(kreg[t][j], p);
                    S[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(p[0], p[1], p[2], p[3]), qf[j], float4p_t{qs[j], qs[j], qs[j], qs[j]}, 0, 0, 0);
                }
#pragma unroll
            for (int t = 0; t < SB; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const auto score = [&](int j) { return FOLD ? (col < 8 ? S[0][j][i] : S[1][j][i]) : S[t][j][i]; };
                    float sum = score(0) * (float)ks[t][i];
#pragma unroll
                    for (int j = 1; j < J; ++j) sum = fmaf(score(j), (float)ks[t][4 * j + i], sum);
                    x[4 * t + i] = sum;
                }
            if (gone) {
#pragma unroll
                for (int t = 0; t < SB; ++t) {
                    const bool there = FOLD ? (col < 8 ? there0 : there1) : (t ? there1 : there0);
                    const int first = t0 + 16 * (FOLD ? col >> 3 : t) + 4 * quarter;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!there || first + i > pos) x[4 * t + i] = -INFINITY;
                }
            }
            float mx = x[0];
#pragma unroll
            for (int i = 1; i < 4 * SB; ++i) mx = fmaxf(mx, x[i]);
            if constexpr (MORE) load(kreg, ks, pa.k, pa.k_scale, s + 1);
            if constexpr (FOLD) mx = fmaxf(mx, lane_xor<8>(mx));
            mx = column_max(mx) * c;
            const bool move = mx > m_run + kLag;               // the first visible tokens: m_run = -inf
            if (__any(move)) {
                const float m_new = move ? mx : m_run, alpha = move ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.0f;
                l_run *= alpha;
                m_run = m_new;
#pragma unroll
                for (int i = 0; i < NT; ++i) O[i] *= alpha;
#pragma unroll
                for (int j = 0; j < J; ++j) off[j] *= alpha;
            }
            const float m_ref = m_run == -INFINITY ? 0.0f : m_run - kBias;      // nothing visible yet: every weight is exp2(-inf)
            float w[4 * SB];
#pragma unroll
            for (int i = 0; i < 4 * SB; ++i) {
                w[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c, -m_ref));
                l_run += w[i];
            }
            if (gone) {                                        // a scale behind the last token is anything
#pragma unroll
                for (int t = 0; t < SB; ++t)
#pragma unroll
                    for (int j = 0; j < J; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) vs[t][4 * j + i] = x[4 * t + i] == -INFINITY ? (_Float16)0.0f : vs[t][4 * j + i];
            }
#pragma unroll
            for (int j = 0; j < J; ++j) {
                half2p_t pw[4];                                // the weights of both blocks, tokens 0 2 | 1 3
#pragma unroll
                for (int t = 0; t < SB; ++t)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        pw[2 * t + i] = half2p_t{(_Float16)(w[4 * t + i] * (float)vs[t][4 * j + i]), (_Float16)(w[4 * t + i + 2] * (float)vs[t][4 * j + i + 2])};
                if constexpr (FOLD) {                          // (columns from 8 on have the blocks the other way round, and no pair)
#pragma unroll
                    for (int i = 0; i < 2; ++i) pw[2 + i] = __builtin_bit_cast(half2p_t, lane_xor<8>(__builtin_bit_cast(float, pw[i])));
                }
                const half8p_t pf = operand(pw[0], pw[1], pw[2], pw[3]);
                half2p_t a[4], e[4];
                word_codes(vreg[0][j], a);
                word_codes(vreg[1][j], e);
                O[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(a[0], a[1], e[0], e[1]), pf, O[2 * j], 0, 0, 0);
                O[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(a[2], a[3], e[2], e[3]), pf, O[2 * j + 1], 0, 0, 0);
                const half2p_t eight = {(_Float16)-8.0f, (_Float16)-8.0f};
                off[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(eight, eight, eight, eight), pf, off[j], 0, 0, 0);
            }
            if constexpr (MORE) load(vreg, vs, pa.v, pa.v_scale, s + 1);
        };
#pragma unroll 1
        for (int s = 0; s + 1 < ns; ++s) step(s, std::true_type{});
        step(ns - 1, std::false_type{});
    }

    // ---- the wavefronts' states meet in LDS ----
    if constexpr (FOLD) l_run += lane_xor<8>(l_run);
    l_run = xor32_sum(xor16_sum(l_run));
#pragma unroll
    for (int i = 0; i < NT; ++i)
        *(float4p_t *)(states + (wave * 16 + col) * P + i * 16 + quarter * 4) = O[i] + off[i >> 1];
    if (quarter == 0) sm_m[wave * 16 + col] = m_run, sm_l[wave * 16 + col] = l_run;
    __syncthreads();
    for (int u = tid; u < n_pairs * (D / 4); u += 64 * W) {
        const int pc = u / (D / 4), e = u % (D / 4) * 4;
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) mm = fmaxf(mm, sm_m[w * 16 + pc]);
        float4p_t num = {0.0f, 0.0f, 0.0f, 0.0f};
        float den = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float mw = sm_m[w * 16 + pc], fw = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - mm);
            num += *(const float4p_t *)(states + (w * 16 + pc) * P + e) * fw;
            den += sm_l[w * 16 + pc] * fw;
        }
        const int pr = (p0 + pc) / rep, ph = kvh * rep + p0 + pc - pr * rep;
        const size_t at = (size_t)(si.q_start + pr) * h + ph;
        if (splits > 1) {
            float *dst = part + (at * splits + split) * (D + 2);
            dst[e] = num.x, dst[e + 1] = num.y, dst[e + 2] = num.z, dst[e + 3] = num.w;
            if (e == 0) dst[D] = mm, dst[D + 1] = den;
        } else {
            const float inv = den > 0.0f ? 1.0f / den : den;   // a row that no token is left for is zeros; a NaN stays one
            const uint32_t lo = f2h(num.x * inv) | (uint32_t)f2h(num.y * inv) << 16, hi = f2h(num.z * inv) | (uint32_t)f2h(num.w * inv) << 16;
            *(u32x2p_t *)(out + at * D + e) = u32x2p_t{lo, hi};
        }
    }
}

template <int D>
hipError_t launch_d(const uint16_t *q, const Paged4Args &pa, const relax_layer_dims &dm, const PagedSeqs &st, const PagedPlan &pl, bool few, uint16_t *out, float *partials,
                    hipStream_t stream)
{
    if ((int64_t)pl.items * dm.n_kv_heads * 64 * pl.waves > kMaxThreads) return hipErrorInvalidValue;
    const dim3 grid(pl.items * dm.n_kv_heads, pl.splits);
    const auto launch = [&](auto W, auto FOLD) {
        hipLaunchKernelGGL((attn_paged4_kernel<D, W, FOLD>), grid, dim3(64 * W), 0, stream, st, q, pa, partials, out, dm.n_heads, dm.n_kv_heads, pl.per_seq, pl.chunk, pl.splits,
                           pl.least);
    };
    using four = std::integral_constant<int, 4>;
    using eight = std::integral_constant<int, 8>;
    if (pl.waves == 8) few ? launch(eight{}, std::true_type{}) : launch(eight{}, std::false_type{});
    else few ? launch(four{}, std::true_type{}) : launch(four{}, std::false_type{});
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || pl.splits == 1 ? e : launch_paged_merge(pl, partials, out, dm, pa.cap, st, stream);
}

}  // namespace

hipError_t launch_paged4_attention(const uint16_t *q, const Paged4Args &pa, const relax_layer_dims &dm, const PagedSeqs &st, const relax_seqs &sq, int32_t L_max,
                                   uint16_t *out, float *partials, hipStream_t stream)
{
    const PagedPlan pl = paged_plan(dm, sq, st.n, L_max);
    if (pl.row_items > 0) {
        const hipError_t e = launch_paged4_rows(q, pa, dm, st, pl, out, stream);
        if (e != hipSuccess || pl.items == 0) return e;
    }
    const bool few = (int64_t)st.q_max * (dm.n_heads / dm.n_kv_heads) <= 8;
    return dm.head_dim == 128 ? launch_d<128>(q, pa, dm, st, pl, few, out, partials, stream) : launch_d<64>(q, pa, dm, st, pl, few, out, partials, stream);
}

}  // namespace relax
