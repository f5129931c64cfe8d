// Causal attention over the paged 4-bit KV cache for sequences that bring many (row, head) pairs: prompts, and drafts of long groups.
//
// The mathematics are those of attn_paged4.hip, the tiles, the turns of the two halves of a workgroup and the barriers between them those of attn_paged_rows.hip: 256 pairs against
// one KV head and all tokens they see, 32 of them per wavefront, every tile of 64 tokens in LDS as fp16 in the order of the fragments.  A scale belongs to 32
// elements of one token here, so both operands are decoded to the numbers that the cache stands for, (u - 8) s = u s + (-8 s), one multiply-add per pair and exact
// (eight and four bits): the products need no factor, and the one rounding is that of the weights.
//
// 4096 rows of 32 / 8 heads of 128: 139 us, 0.99 PFLOP/s of the causal half (a large fp16 product reaches 1.35 here: 102 us).  Bound by the two halves' turns: one takes about 1050 cycles, of which
// its 34 matrix instructions need 571 alone; next to them a vector instruction of the other half takes 8.5 cycles instead of 5.4.
#include <type_traits>

#include "paged4_device.h"

namespace relax {

namespace {

constexpr float kBias = 11.0f, kMost = 65000.0f; // log2 of the weight at the reference; the largest packed weight before that moves
constexpr float kUnset = -1e30f;                 // reference of a row that has met no token: below every score, and finite

// LDS-only workgroup barrier: global loads stay in flight across it
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

constexpr int CT = 2;                            // column tiles of 16 pairs per wavefront
constexpr int kThreads = 512;
constexpr int kSegment = kThreads;               // blocks whose numbers are in LDS at a time

// grid: x = tile * g + KV head (the last tile of a sequence, with the longest prefix, first)
template <int D>
__global__ __launch_bounds__(kThreads, 2) void attn_paged4_rows_kernel(PagedSeqs, const uint16_t *q, Paged4Args pa, uint16_t *out, int h, int g, int per_seq,
                                                                       int least)
{
    constexpr int J = D / 32, NT = D / 16;       // words of a lane per block, also k steps; 16-element tiles of O^T
    constexpr int G = NT;                        // steps of either product of 32 tokens
    constexpr int PD = D == 128 ? 8 : 4;         // steps that operands are read ahead
    static_assert(2 * J == G && PD <= G, "both products of half a tile have as many operands");
    constexpr int kPairs = kPagedRowTile;
    static_assert(kPairs == 8 * 16 * CT, "eight wavefronts");
    constexpr int kTileBytes = 64 * D * 2;
    __shared__ __align__(16) unsigned char lds[4 * kTileBytes];        // keys: two buffers, values: two
    __shared__ __align__(16) int pools[kSegment];                      // numbers of the segment's blocks, -1: none
    __shared__ int bad_s;

    const int rep = h / g, item = (int)blockIdx.x / g, kvh = (int)blockIdx.x - item * g;
    const SeqsArg st = seqs_arg();
    const auto tiles_of = [&](int q_len) { return q_len * rep < least ? 0 : (q_len * rep + kPairs - 1) / kPairs; };
    int place;
    const int b = tile_of(st, item, per_seq, tiles_of, place);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, __builtin_amdgcn_readfirstlane(b));
    const int pairs = si.q_len * rep, p0 = (tiles_of(si.q_len) - 1 - place) * kPairs;
    if (pairs < least || p0 < 0) return;                          // (fewer pairs: the other kernel's)
    const int n_pairs = min(kPairs, pairs - p0);
    const bool beyond = beyond_capacity(si, pa.cap);
    const int past = beyond ? 0 : si.kv_len - si.q_len;
    const int vis = beyond ? 0 : past + (p0 + n_pairs - 1) / rep + 1;
    if (beyond && threadIdx.x == 0) atomicOr(pa.err, kBadPage);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int b_end = (max(vis, 0) + 15) >> 4;

    // ---- queries, in the order of the codes of a word ----
    const int wave_min = past + min(p0 + wave * 16 * CT, p0 + n_pairs - 1) / rep;
    half8p_t qf[CT][J];
    int pos[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int pair = min(p0 + (wave * CT + ct) * 16 + col, p0 + n_pairs - 1), row = pair / rep, head = kvh * rep + pair - row * rep;
        pos[ct] = past + row;
        const uint16_t *src = q + ((size_t)(si.q_start + row) * h + head) * D + quarter * 8;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const half8p_t x = *(const half8p_t *)(src + j * 32);
            qf[ct][j] = half8p_t{x[0], x[4], x[1], x[5], x[2], x[6], x[3], x[7]};
        }
    }
    const float c = 1.44269504088896340736f / sqrtf((float)D);

    float4p_t O[NT][CT];
    float m[CT];
    float4p_t l[CT];                                                   // sums of the weights, the same in all four
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = kUnset, l[ct] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NT; ++i) O[i][ct] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    struct Keys {                                                      // two words of the lane, and the scales of their groups for its token
        u32x2p_t w;
        uint16_t s[2];
    };
    struct Values {                                                    // two words, and the scales of their groups for the lane's four tokens
        u32x2p_t w;
        half8p_t s;
    };
    Keys rk[2];                                                        // of the next two tiles, by their parity
    Values rv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) rk[i] = Keys{}, rv[i] = Values{};
    half8p_t ring[PD], pf[CT];

    // ---- staging: a tile is 2 J packets of two words per lane of keys and as many of values; with heads of 128 a wavefront brings one of each, with heads of 64 one ----
    const bool brings_keys = J == 4 || wave < 4, brings_values = J == 4 || wave >= 4;
    const int blk_w = J == 4 ? wave >> 1 : wave & 3, load_w = J == 4 ? wave & 1 : 0;
    auto pool_of = [&](int t) { return pools[min(t * 4, kSegment - 4) + blk_w]; };
    auto load_keys = [&](int parity, int pool) {
        const size_t at = max(__builtin_amdgcn_readfirstlane(pool), 0);
        rk[parity].w = ((const u32x2p_t *)(pa.k + at * block4_codes(D)))[lane * (J / 2) + load_w];
        const uint16_t *s = pa.k_scale + at * block4_scales(D) + (((lane & 15) >> 2) * J + 2 * load_w) * 4 + (lane & 3);
        rk[parity].s[0] = s[0], rk[parity].s[1] = s[4];
    };
    auto load_values = [&](int parity, int pool) {
        const size_t at = max(__builtin_amdgcn_readfirstlane(pool), 0);
        rv[parity].w = ((const u32x2p_t *)(pa.v + at * block4_codes(D)))[lane * (J / 2) + load_w];
        rv[parity].s = *(const half8p_t *)(pa.v_scale + at * block4_scales(D) + (quarter * J + 2 * load_w) * 4);
    };
    // scales of values behind the last token, or of a block without a page, are anything, and a weight of zero would not hide a NaN
    auto clean_values = [&](int parity, int t, int t0, bool bad) {    // t: the tile in its segment, t0: its first position
        if (t0 + 64 > vis || bad) {                                    // uniform
            const bool there = pool_of(t) >= 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!there || t0 + 16 * blk_w + 4 * quarter + (i & 3) >= vis) rv[parity].s[i] = (_Float16)0.0f;
        }
    };
    auto store_key = [&](int kb, int i) {                              // word i of the packet; the buffer is the tile's parity
        if (!brings_keys) return;
        half2p_t u[4];
        word_codes(rk[kb].w[i], u);
        const _Float16 s = __builtin_bit_cast(_Float16, rk[kb].s[i]), off = s * (_Float16)-8.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = __builtin_elementwise_fma(u[e], half2p_t{s, s}, half2p_t{off, off});
        *(half8p_t *)(lds + kb * kTileBytes + ((blk_w * J + 2 * load_w + i) * 64 + lane) * 16) = operand(u[0], u[1], u[2], u[3]);
    };
    auto store_value = [&](int vb, int i) {                            // the four tokens of the low (i even) or high halves of word i / 2
        if (!brings_values) return;
        const uint32_t w = rv[vb].w[i >> 1], n = (i & 1 ? w >> 4 : w) & 0x0f0f0f0fu;
        const half8p_t s = rv[vb].s;
        const int at = (i >> 1) * 4;
        const half2p_t s0 = {s[at], s[at + 2]}, s1 = {s[at + 1], s[at + 3]}, eight = {(_Float16)-8.0f, (_Float16)-8.0f};
        const half2p_t u0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(n, 512.0f, false), u1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(n, 512.0f, true);
        const half2p_t lo = __builtin_elementwise_fma(u0, s0, s0 * eight), hi = __builtin_elementwise_fma(u1, s1, s1 * eight);
        *(u32x2p_t *)(lds + (2 + vb) * kTileBytes + (((blk_w >> 1) * NT + 4 * load_w + i) * 64 + lane) * 16 + (blk_w & 1) * 8) =
            u32x2p_t{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
    };

    // ---- half a tile: 32 tokens, two blocks ----
    struct Scores {
        float4p_t s[2][CT];
    };
    auto read_key = [&](int kb, int sub, int i) { return *(const half8p_t *)(lds + kb * kTileBytes + (sub * 2 * J * 64 + lane) * 16 + i * 1024); };
    auto read_value = [&](int vb, int sub, int i) { return *(const half8p_t *)(lds + (2 + vb) * kTileBytes + (sub * NT * 64 + lane) * 16 + i * 1024); };
    auto key_step = [&](Scores &S, int i) {
        const float4p_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            S.s[i / J][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ring[i % PD], qf[ct][i % J], i % J ? S.s[i / J][ct] : zero, 0, 0, 0);
    };
    auto value_step = [&](int i) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) O[i][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ring[i % PD], pf[ct], O[i][ct], 0, 0, 0);
    };
    auto weights = [&](const Scores &S) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const float off = kBias - m[ct];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)                            // tokens 0 2 1 3, as the values lie
                    pf[ct][4 * u + (i & 1) * 2 + (i >> 1)] = (_Float16)__builtin_amdgcn_exp2f(fmaf(S.s[u][ct][i], c, off));
        }
    };
    auto mask = [&](Scores &S, int at, int t0, bool bad) {             // at: the first of the two blocks in the segment
        if (t0 + 31 > wave_min || bad) {                               // uniform
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool there = pools[at + u] >= 0;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!there || t0 + 16 * u + 4 * quarter + i > pos[ct]) S.s[u][ct][i] = -INFINITY;
            }
        }
    };
    // The weights were computed against the reference as it was.  Where one is about to leave fp16's range (or every column is new), the reference
    // moves to the maximum of these scores, what was summed against the old one is rescaled and the weights are computed again: rare behind the first
    // tiles of a row, and a look at the packed weights costs a quarter of the maxima of the scores.
    auto settle = [&](const Scores &S) {
        half2p_t top = {(_Float16)0.0f, (_Float16)0.0f};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, half2p_t{pf[ct][2 * i], pf[ct][2 * i + 1]});
        if (__any(fmaxf((float)top.x, (float)top.y) > kMost)) {
            auto over_column = [](float v) {                           // maximum over the four lanes of a column
                float2 both = pair_xor16(v);
                both = pair_xor32(fmaxf(both.x, both.y));
                return fmaxf(both.x, both.y);
            };
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float mx = -INFINITY, most = 0.0f;                     // a column moves by itself: no row depends on the others of its tile
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, S.s[u][ct][i] * c), most = fmaxf(most, (float)pf[ct][4 * u + i]);
                mx = over_column(mx), most = over_column(most);
                const float to = most > kMost && mx > m[ct] ? mx : m[ct], alpha = __builtin_amdgcn_exp2f(m[ct] - to);
                m[ct] = to, l[ct] *= alpha;
#pragma unroll
                for (int i = 0; i < NT; ++i) O[i][ct] *= alpha;
            }
            weights(S);
        }
    };

    const bool second = wave >= 4;                                     // of the two halves that take turns
    for (int seg = 0; seg < b_end; seg += kSegment) {
        // ---- numbers of the segment's blocks, one per thread ----
        int pool = -1;
        if (seg + tid < b_end) {
            pool = paged_block(pa, g, kvh, si.slot, seg + tid);
            if (pool < 0) atomicOr(pa.err, kBadPage);
        }
        __syncthreads();                                               // the segment before is consumed
        if (tid == 0) bad_s = 0;
        __syncthreads();
        if (pool < 0 && seg + tid < b_end) bad_s = 1;
        pools[tid] = pool;
        __syncthreads();
        // a tile's last blocks may lie behind the end: masked like those without a page, but by their positions
        const bool bad = __builtin_amdgcn_readfirstlane(bad_s) != 0;

        // ---- the segment's tiles ----
        const int first = seg * 16, nt = (min(b_end - seg, kSegment) + 3) >> 2;
        // Loads are issued without a condition, behind the last tile of any block: behind a branch their number at a wait is not known, and each wait
        // would be for all of them.
        load_keys(0, pool_of(0)), load_values(0, pool_of(0)), load_keys(1, pool_of(1)), load_values(1, pool_of(1));
#pragma unroll
        for (int i = 0; i < 4; ++i) store_key(i >> 1, i & 1);
        clean_values(0, 0, first, bad);
#pragma unroll
        for (int i = 0; i < 4; ++i) store_value(0, i);
        load_keys(0, pool_of(2)), load_values(0, pool_of(2)), load_keys(1, pool_of(3));
        lds_barrier();
        if (second) lds_barrier();
        Scores S;
#pragma unroll
        for (int i = 0; i < PD; ++i) ring[i] = read_key(0, 0, i);
#pragma unroll
        for (int i = 0; i < G; ++i) {
            key_step(S, i);
            if (i + PD < G) ring[i % PD] = read_key(0, 0, i + PD);
        }
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
        // two turns of either kind per tile; PARITY: its buffers and registers
        auto tile_turns = [&](auto PARITY, int t) __attribute__((always_inline)) {
            constexpr int kb = PARITY;
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                // ---- turn of the vector unit: weights of these 32 tokens; the first operands of the products are asked for ----
                mask(S, min(t * 4 + 2 * sub, kSegment - 2), first + t * 64 + sub * 32, bad);
                weights(S);
                settle(S);
                if (sub == 0) clean_values(kb ^ 1, t + 1, first + t * 64 + 64, bad);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < PD; ++i) ring[i] = read_value(kb, sub, i);
                asm volatile("s_barrier" ::: "memory");                // (nothing written in this turn: no wait for the reads)
                // ---- turn of the matrix pipe: these weights with V, the keys of the next 32 tokens with Q, and what the wavefront brings: in the first turn of
                // a tile its values of the next one, in the second its keys of the one behind that.  The other half has read either buffer for
                // the last time one turn before at the latest, and neither is read before two turns have passed ----
                const int key_buf = sub ? kb ^ 1 : kb;                 // (behind the last tile: an old one, its scores are not used)
                __builtin_amdgcn_s_setprio(1);
                const int pool_ahead = pool_of(t + 3 + sub);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    value_step(i);
                    ring[i % PD] = i + PD < G ? read_value(kb, sub, i + PD) : read_key(key_buf, sub ^ 1, i + PD - G);
                    if (sub == 0 && i >= G / 4 - 1 && i < G / 4 + 3) store_value(kb ^ 1, i - (G / 4 - 1));   // (behind the last tile: the same once more, not read)
                    if (sub == 1 && i >= 1 && i < 3) store_key(kb, i - 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
                const half2p_t one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(one, one, one, one), pf[ct], l[ct], 0, 0, 0);
                if (sub == 0) load_values(kb ^ 1, pool_ahead);
                if (sub == 1) load_keys(kb, pool_ahead);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    key_step(S, i);
                    if (i + PD < G) ring[i % PD] = read_key(key_buf, sub ^ 1, i + PD);
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
                lds_barrier();
            }
        };
        for (int t = 0; t < nt; t += 2) {
            tile_turns(std::integral_constant<int, 0>{}, t);
            if (t + 1 < nt) tile_turns(std::integral_constant<int, 1>{}, t + 1);
        }
        if (!second) lds_barrier();
    }

    // ---- results: lane holds elements 16 i + 4 quarter .. + 3 of its columns ----
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const float den = l[ct][0];
        const int place = (wave * CT + ct) * 16 + col;
        if (place >= n_pairs) continue;
        const int pair = p0 + place, row = pair / rep;
        const size_t at = (size_t)(si.q_start + row) * h + kvh * rep + pair - row * rep;
        const float inv = den > 0.0f ? 1.0f / den : den;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const float4p_t o = O[i][ct] * inv;
            const uint32_t lo = f2h(o.x) | (uint32_t)f2h(o.y) << 16, hi = f2h(o.z) | (uint32_t)f2h(o.w) << 16;
            *(u32x2p_t *)(out + at * D + i * 16 + quarter * 4) = u32x2p_t{lo, hi};
        }
    }
}

template <int D>
hipError_t launch_one(const uint16_t *q, const Paged4Args &pa, const relax_layer_dims &dm, const PagedSeqs &st, const PagedPlan &pl, uint16_t *out, hipStream_t stream)
{
    if ((int64_t)pl.row_items * dm.n_kv_heads * kThreads > kMaxThreads) return hipErrorInvalidValue;
    hipLaunchKernelGGL(attn_paged4_rows_kernel<D>, dim3(pl.row_items * dm.n_kv_heads), dim3(kThreads), 0, stream, st, q, pa, out, dm.n_heads, dm.n_kv_heads, pl.row_per_seq, pl.least);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged4_rows(const uint16_t *q, const Paged4Args &pa, const relax_layer_dims &dm, const PagedSeqs &st, const PagedPlan &pl, uint16_t *out, hipStream_t stream)
{
    return dm.head_dim == 128 ? launch_one<128>(q, pa, dm, st, pl, out, stream) : launch_one<64>(q, pa, dm, st, pl, out, stream);
}

}  // namespace relax
