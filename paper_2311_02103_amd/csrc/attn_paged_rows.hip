// Causal attention over the paged 8-bit KV cache for sequences that bring many (row, head) pairs: prompts, and drafts of long groups.
//
// The mathematics, the transposed products, the fragments and the scales are those of attn_paged.hip; here the pairs are many enough to share
// what a tile of the cache costs.  A workgroup takes 256 pairs against one KV head and all tokens they see, each of its eight wavefronts 32 of
// them, and all eight meet every tile of 64 tokens in LDS, as fp16 integers in the order of the fragments: the codes are turned into halves
// once per workgroup (in the wavefronts they would cost as many issue slots as the softmax), and every read and write is 16 consecutive bytes per lane (V writes
// 8).  Keys and values have two buffers each.
//
// Per 32 tokens a wavefront has 34 MFMAs of 16 cycles and about 75 vector instructions and 16 exponentials: some 500 cycles of the matrix pipe and as many of
// the vector unit.  Two wavefronts share a SIMD, one of each half of the workgroup, and the halves
// take turns: while wavefronts 0 .. 3 multiply (this step's weights with V, the next step's keys with Q), wavefronts 4 .. 7 compute weights and stage their
// part of the next tile, then the other way round, with a barrier between the turns.  4096 tokens, 32 / 8 heads of 128: 147 us (0.93 PFLOP/s of the causal half); with
// four wavefronts per workgroup left to themselves, scores and exponentials in one stream of instructions, 170 (the matrix pipe busy 34 % of the time).
// A turn takes about 1000 cycles at 2 GHz where 544 of the matrix pipe would do: next to the other half's vector work its 34 MFMAs take 970, alone 660.
//
// The value scale of a block, relative to the largest so far, is 2^E mu with 1 <= mu < 2.  The power of two multiplies the codes on their way into LDS, which is
// exact down to 2^-24; mu is in the weights, as an addend of their exponent, so that the one rounding to fp16 stays that of the weights (with the whole
// scale on the codes outputs were off by 3.2e-4 instead of 2.8e-4, 2.0e-4 of it their own rounding).  The sums of the weights are one more MFMA: its other operand is
// 1 / mu of the token's block, as two halves in alternate rows, whose results add up to 1 / mu within 2^-22.
#include <type_traits>

#include "paged_device.h"

namespace relax {

namespace {

constexpr float kBias = 11.0f, kMost = 65000.0f; // as in attn_paged.hip: log2 of the weight at the reference; the largest packed weight before that moves (at 32768
                                                 // it moves more often: 4096 tokens of 32 / 8 heads 170 us for 159)
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
constexpr int kSegment = kThreads;               // blocks whose numbers and scales are in LDS at a time

// What a block needs: c k_scale, log2 mu + kBias, number in the pool (as bits), 2^E as two halves to multiply (as bits)
typedef float4p_t Block;

// grid: x = tile * g + KV head (the last tile of a sequence, with the longest prefix, first)
template <int D>
__global__ __launch_bounds__(kThreads, 2) void attn_paged_rows_kernel(PagedSeqs, const uint16_t *__restrict__ q, PagedArgs pa, uint16_t *__restrict__ out, int h, int g, int per_seq,
                                                                       int least)
{
    constexpr int J = D / 64, KS = D / 32, NT = D / 16;
    constexpr int G = NT;                        // steps of either product of 32 tokens
    constexpr int PD = D == 128 ? 8 : 4;         // steps that operands are read ahead
    static_assert(2 * KS == G && PD <= G, "both products of half a tile have as many operands");
    constexpr int kPairs = kPagedRowTile;
    static_assert(kPairs == 8 * 16 * CT, "eight wavefronts");
    constexpr int kTileBytes = 64 * D * 2;
    __shared__ __align__(16) unsigned char lds[4 * kTileBytes];        // keys: two buffers, values: two
    __shared__ __align__(16) Block blocks[kSegment];
    __shared__ __align__(8) uint32_t unscales[2][kSegment];            // 1 / mu: the two halves to add, each twice in a word
    __shared__ float v_tops[8];
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
    const int past = si.kv_len - si.q_len;
    const int n_pairs = min(kPairs, pairs - p0);
    const bool beyond = beyond_capacity(si, pa.cap);
    const int vis = beyond ? 0 : past + (p0 + n_pairs - 1) / rep + 1;
    if (beyond && threadIdx.x == 0) atomicOr(pa.err, kBadPage);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int b_end = (max(vis, 0) + 15) >> 4;

    // ---- queries ----
    const int wave_min = past + min(p0 + wave * 16 * CT, p0 + n_pairs - 1) / rep;
    half8p_t qf[CT][KS];
    int pos[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int pair = min(p0 + (wave * CT + ct) * 16 + col, p0 + n_pairs - 1), row = pair / rep, head = kvh * rep + pair - row * rep;
        pos[ct] = past + row;
        const uint16_t *src = q + ((size_t)(si.q_start + row) * h + head) * D + quarter * 16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ct][ks] = *(const half8p_t *)(src + (ks >> 1) * 64 + (ks & 1) * 8);
    }
    const float c = 1.44269504088896340736f / sqrtf((float)D);

    float4p_t O[NT][CT];
    float m[CT];
    float4p_t l[CT];                                                   // sums of the weights: the first two together
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = kUnset, l[ct] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NT; ++i) O[i][ct] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    float v_ref = 0.0f;
    u32x4p_t rk[2], rv[2];                                             // of the next two tiles, by their parity
    float vr[2];                                                       // 2^E of what is in rv
#pragma unroll
    for (int i = 0; i < 2; ++i) rk[i] = rv[i] = u32x4p_t{0, 0, 0, 0}, vr[i] = 0.0f;
    half8p_t ring[PD], pf[CT];

    // ---- staging: a tile is 4 J loads of keys and as many of values; with heads of 128 a wavefront brings one of each, with heads of 64 one ----
    const bool brings_keys = J == 2 || wave < 4, brings_values = J == 2 || wave >= 4;
    const int blk_w = J == 2 ? wave >> 1 : wave & 3, load_w = J == 2 ? wave & 1 : 0;
    auto info_of = [&](int t) { return blocks[min(t * 4, kSegment - 4) + blk_w]; };
    auto packet = [&](const uint8_t *codes, const Block &info) {
        const int p = max(__builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, (float)info[2])), 0);
        return ((const u32x4p_t *)(codes + (size_t)p * (16 * D)))[load_w * 64 + lane];
    };
    auto load_keys = [&](int parity, const Block &info) {
        rk[parity] = packet(pa.k, info);
    };
    auto load_values = [&](int parity, const Block &info) {
        rv[parity] = packet(pa.v, info), vr[parity] = info[3];
    };
    auto store_key = [&](int kb, int i) {                              // half i of the load; the buffer is the tile's parity
        if (!brings_keys) return;
        const u32x4p_t w = rk[kb];
        *(half8p_t *)(lds + kb * kTileBytes + ((blk_w * KS + 2 * load_w + i) * 64 + lane) * 16) = i ? codes_to_half8(w.z, w.w) : codes_to_half8(w.x, w.y);
    };
    auto store_value = [&](int vb, int i) {                            // the four tokens of element i of the load
        if (!brings_values) return;
        const half2p_t f = __builtin_bit_cast(half2p_t, vr[vb]);       // (the second factor rounds, where values below 2^-31 of the largest leave fp16's range)
        half2p_t lo, hi;
        codes_to_half(rv[vb][i], lo, hi);
        lo = lo * half2p_t{f.x, f.x} * half2p_t{f.y, f.y}, hi = hi * half2p_t{f.x, f.x} * half2p_t{f.y, f.y};
        *(u32x2p_t *)(lds + (2 + vb) * kTileBytes + (((blk_w >> 1) * NT + 4 * load_w + i) * 64 + lane) * 16 + (blk_w & 1) * 8) =
            u32x2p_t{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
    };

    // ---- half a tile: 32 tokens, two blocks ----
    struct Scores {
        float4p_t s[2][CT];
    };
    auto read_key = [&](int kb, int sub, int i) { return *(const half8p_t *)(lds + kb * kTileBytes + (sub * 2 * KS * 64 + lane) * 16 + i * 1024); };
    auto read_value = [&](int vb, int sub, int i) { return *(const half8p_t *)(lds + (2 + vb) * kTileBytes + (sub * NT * 64 + lane) * 16 + i * 1024); };
    auto key_step = [&](Scores &S, int i) {
        const float4p_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            S.s[i / KS][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ring[i % PD], qf[ct][i % KS], i % KS ? S.s[i / KS][ct] : zero, 0, 0, 0);
    };
    auto value_step = [&](int i) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) O[i][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ring[i % PD], pf[ct], O[i][ct], 0, 0, 0);
    };
    auto weights = [&](const Scores &S, const Block (&bl)[2]) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const float off = bl[u][1] - m[ct];
#pragma unroll
                for (int i = 0; i < 4; ++i) pf[ct][4 * u + i] = (_Float16)__builtin_amdgcn_exp2f(fmaf(S.s[u][ct][i], bl[u][0], off));
            }
        }
    };
    auto unscale_of = [&](int at) { return *(const u32x2p_t *)&unscales[lane & 1][min(at, kSegment - 2)]; };
    auto mask = [&](Scores &S, int at, int t0, bool bad) {             // at: the first of the two blocks in the segment
        if (t0 + 31 > wave_min || bad) {                               // uniform
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool there = __builtin_bit_cast(int, (float)blocks[at + u][2]) >= 0;
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
    auto settle = [&](const Scores &S, const Block (&bl)[2]) {
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
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, S.s[u][ct][i] * bl[u][0]), most = fmaxf(most, (float)pf[ct][4 * u + i]);
                mx = over_column(mx), most = over_column(most);
                const float to = most > kMost && mx > m[ct] ? mx : m[ct], alpha = __builtin_amdgcn_exp2f(m[ct] - to);
                m[ct] = to, l[ct] *= alpha;
#pragma unroll
                for (int i = 0; i < NT; ++i) O[i][ct] *= alpha;
            }
            weights(S, bl);
        }
    };

    const bool second = wave >= 4;                                     // of the two halves that take turns
    for (int seg = 0; seg < b_end; seg += kSegment) {
        // ---- numbers and scales of the segment's blocks, one per thread ----
        int pool = -1;
        float ks = 0.0f, vs = 0.0f;
        if (seg + tid < b_end) {
            pool = paged_block(pa, g, kvh, si.slot, seg + tid);
            if (pool < 0) atomicOr(pa.err, kBadPage);
            else ks = pa.k_scale[pool], vs = pa.v_scale[pool];
        }
        const float top = wave_max(vs);
        __syncthreads();                                               // the segment before is consumed
        if (tid == 0) bad_s = 0;
        if (lane == 0) v_tops[wave] = top;
        __syncthreads();
        float ref = v_ref;
#pragma unroll
        for (int w = 0; w < 8; ++w) ref = fmaxf(ref, v_tops[w]);
        if (pool < 0 && seg + tid < b_end) bad_s = 1;
        // (codes of a zero scale are zero; -inf times its factor has to stay -inf)
        const float scale = fmaxf(ref > 0.0f ? __builtin_amdgcn_logf(vs / ref) : 0.0f, -40.0f);       // (2^-40: codes of a zero scale, which become zeros in fp16)
        const float mu = __builtin_amdgcn_fractf(scale), inv = __builtin_amdgcn_exp2f(-mu);
        const int e = (int)(scale - mu), e1 = max(e, -14);
        const _Float16 inv_hi = (_Float16)inv, inv_lo = (_Float16)(inv - (float)inv_hi);
        blocks[tid] = Block{fmaxf(ks * c, 0x1p-100f), mu + kBias, __builtin_bit_cast(float, pool),
                            __builtin_bit_cast(float, half2p_t{(_Float16)ldexpf(1.0f, e1), (_Float16)ldexpf(1.0f, e - e1)})};
        unscales[0][tid] = __builtin_bit_cast(uint32_t, half2p_t{inv_hi, inv_hi}), unscales[1][tid] = __builtin_bit_cast(uint32_t, half2p_t{inv_lo, inv_lo});
        if (v_ref > 0.0f && ref > v_ref) {                             // O is in units of the largest value scale so far
            const float f = v_ref / ref;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) O[i][ct] *= f;
        }
        v_ref = ref;
        __syncthreads();
        // a tile's last blocks may lie behind the end: masked like those without a page, but by their positions
        const bool bad = __builtin_amdgcn_readfirstlane(bad_s) != 0;

        // ---- the segment's tiles ----
        const int first = seg * 16, nt = (min(b_end - seg, kSegment) + 3) >> 2;
        // Loads are issued without a condition, behind the last tile of any block: behind a branch their number at a wait is not known, and each wait
        // would be for all of them (turns of the matrix pipe 1000 cycles instead of 850).
        load_keys(0, info_of(0)), load_values(0, info_of(0)), load_keys(1, info_of(1)), load_values(1, info_of(1));
#pragma unroll
        for (int i = 0; i < 4; ++i) store_key(i >> 1, i & 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) store_value(0, i);
        load_keys(0, info_of(2)), load_values(0, info_of(2)), load_keys(1, info_of(3));
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
        Block bl[2] = {blocks[0], blocks[1]};
        u32x2p_t un = unscale_of(0);
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
        // two turns of either kind per tile; PARITY: its buffers and registers
        auto tile_turns = [&](auto PARITY, int t) __attribute__((always_inline)) {
            constexpr int kb = PARITY;
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                // ---- turn of the vector unit: weights of these 32 tokens; the first operands of the products are asked for ----
                mask(S, t * 4 + 2 * sub, first + t * 64 + sub * 32, bad);
                weights(S, bl);
                settle(S, bl);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < PD; ++i) ring[i] = read_value(kb, sub, i);
                asm volatile("s_barrier" ::: "memory");                // (nothing written in this turn: no wait for the reads)
                // ---- turn of the matrix pipe: these weights with V, the keys of the next 32 tokens with Q, and what the wavefront brings: in the first turn of
                // a tile its values of the next one, in the second its keys of the one behind that.  The other half has read either buffer for
                // the last time one turn before at the latest, and neither is read before two turns have passed ----
                const int key_buf = sub ? kb ^ 1 : kb;                 // (behind the last tile: an old one, its scores are not used)
                __builtin_amdgcn_s_setprio(1);
                bl[0] = blocks[min(t * 4 + 2 * sub + 2, kSegment - 2)], bl[1] = blocks[min(t * 4 + 2 * sub + 3, kSegment - 1)];
                const Block info_ahead = info_of(t + 3 + sub);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    value_step(i);
                    ring[i % PD] = i + PD < G ? read_value(kb, sub, i + PD) : read_key(key_buf, sub ^ 1, i + PD - G);
                    if (sub == 0 && i >= G / 4 - 1 && i < G / 4 + 3) store_value(kb ^ 1, i - (G / 4 - 1));   // (behind the last tile: the same once more, not read)
                    if (sub == 1 && i >= 1 && i < 3) store_key(kb, i - 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
                const half8p_t unscale = __builtin_bit_cast(half8p_t, u32x4p_t{un.x, un.x, un.y, un.y});
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(unscale, pf[ct], l[ct], 0, 0, 0);
                un = unscale_of(t * 4 + 2 * sub + 2);
                if (sub == 0) load_values(kb ^ 1, info_ahead);
                if (sub == 1) load_keys(kb, info_ahead);
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
        const float den = l[ct][0] + l[ct][1];
        const int place = (wave * CT + ct) * 16 + col;
        if (place >= n_pairs) continue;
        const int pair = p0 + place, row = pair / rep;
        const size_t at = (size_t)(si.q_start + row) * h + kvh * rep + pair - row * rep;
        const float inv = (den > 0.0f ? 1.0f / den : den) * v_ref;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const float4p_t o = O[i][ct] * inv;
            const uint32_t lo = f2h(o.x) | (uint32_t)f2h(o.y) << 16, hi = f2h(o.z) | (uint32_t)f2h(o.w) << 16;
            *(u32x2p_t *)(out + at * D + i * 16 + quarter * 4) = u32x2p_t{lo, hi};
        }
    }
}

template <int D>
hipError_t launch_one(const uint16_t *q, const PagedArgs &pa, const relax_layer_dims &dm, const PagedSeqs &st, int32_t items, int32_t per_seq, int32_t least, uint16_t *out, hipStream_t stream)
{
    if ((int64_t)items * dm.n_kv_heads * kThreads > kMaxThreads) return hipErrorInvalidValue;
    hipLaunchKernelGGL(attn_paged_rows_kernel<D>, dim3(items * dm.n_kv_heads), dim3(kThreads), 0, stream, st, q, pa, out, dm.n_heads, dm.n_kv_heads, per_seq, least);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_rows(const uint16_t *q, const PagedArgs &pa, const relax_layer_dims &dm, const PagedSeqs &st, int32_t items, int32_t per_seq, int32_t least, uint16_t *out,
                             hipStream_t stream)
{
    return dm.head_dim == 128 ? launch_one<128>(q, pa, dm, st, items, per_seq, least, out, stream) : launch_one<64>(q, pa, dm, st, items, per_seq, least, out, stream);
}

}  // namespace relax
