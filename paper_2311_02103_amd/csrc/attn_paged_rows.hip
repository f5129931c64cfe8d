// Causal attention over the paged 8-bit KV cache for sequences that bring many (row, head) pairs: prompts, and drafts of long groups.
//
// The mathematics, the transposed products, the fragments and the scales are those of attn_paged.hip; here the pairs are many enough to share
// what a tile of the cache costs.  A workgroup takes 64 CT pairs against one KV head and one split of the tokens, each of its four wavefronts 16 CT of
// them, and all four meet every tile of 64 tokens in LDS, as fp16 integers in the order of the fragments: the codes are turned into halves
// once per workgroup (in the wavefronts they would cost as many issue slots as the softmax), and every read and write is 16 consecutive bytes per lane (V writes
// 8).  Keys and values have two buffers each.
//
// Per 32 tokens and wavefront the matrix pipe has 16 CT MFMAs of 16 cycles, the vector unit about 7 issue slots of 4 cycles for each of 8 CT scores (four of them the
// exponential) next to staging, and LDS 16 KB for the four wavefronts: at CT = 2 512, 600 and 512 cycles.  None of the three may wait for another, so the
// order is written out: the scores of the next 32 tokens are computed between the exponentials of these, the products with V between the staging of the next
// tile, and the operands of both are read PD steps ahead.
//
// The value scale of a block goes into the exponent here, log2 of its ratio to the largest scale so far, and the block's sum of weights is
// multiplied by the inverse ratio: one operation per four scores instead of one per score.
#include "paged_device.h"

namespace relax {

namespace {

constexpr float kBias = 11.0f, kMost = 32768.0f; // as in attn_paged.hip: log2 of the weight at the reference; the largest weight before that moves
constexpr float kUnset = -1e30f;                 // reference of a row that has met no token: below every score, and finite

// LDS-only workgroup barrier: global loads stay in flight across it
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

constexpr int kSegment = 768;                    // blocks whose numbers and scales are in LDS at a time

// What a block needs: c k_scale, log2 of v_scale relative to the reference and its inverse, number in the pool (as bits)
typedef float4p_t Block;

// grid: x = KV head, y = split, z = sequence * tiles + tile (the last tile of a sequence, with the longest prefix, first)
template <int D, int CT>
__global__ __launch_bounds__(256, 2) void attn_paged_rows_kernel(PagedSeqs, const uint16_t *__restrict__ q, PagedArgs pa, float *__restrict__ part,
                                                                uint16_t *__restrict__ out, int h, int g, int tiles, int chunk, int splits, int least)
{
    constexpr int J = D / 64, KS = D / 32, NT = D / 16;
    constexpr int G = NT;                        // steps of either product of 32 tokens
    constexpr int PD = 4;                        // steps that operands are read ahead
    static_assert(2 * KS == G && PD <= G, "both products of half a tile have as many operands");
    constexpr int kPairs = 64 * CT;
    constexpr int kTileBytes = 64 * D * 2;
    __shared__ __align__(16) unsigned char lds[4 * kTileBytes];        // keys: two buffers, values: two
    __shared__ __align__(16) Block blocks[kSegment];
    __shared__ float v_tops[4];
    __shared__ int bad_s;

    const int b = tiles == 1 ? (int)blockIdx.z : (int)blockIdx.z / tiles, tile = tiles == 1 ? 0 : tiles - 1 - ((int)blockIdx.z - b * tiles);
    const int kvh = blockIdx.x, split = blockIdx.y;
    const SeqSpan si = seq_span(seqs_arg(), b);
    const int rep = h / g, pairs = si.q_len * rep, p0 = tile * kPairs;
    if (pairs < least || p0 >= pairs) return;                          // (fewer pairs: the other kernel's)
    const int past = si.kv_len - si.q_len;
    const int n_pairs = min(kPairs, pairs - p0);
    const int vis = min(past + (p0 + n_pairs - 1) / rep + 1, pa.cap);
    const int t_begin = split * chunk;
    if (split > 0 && t_begin >= vis) return;
    const int t_end = min(vis, t_begin + chunk);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int b_begin = t_begin >> 4, b_end = t_end > t_begin ? (t_end + 15) >> 4 : b_begin;

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
    float m[CT], l[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = kUnset, l[ct] = 0.0f;
#pragma unroll
        for (int i = 0; i < NT; ++i) O[i][ct] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    float v_ref = 0.0f;
    u32x4p_t rk[J], rv[J];
    half8p_t ring[PD], pf[CT];
    float sum[2][CT];

    // ---- staging: wavefront w brings block w of a tile ----
    auto pool_of = [&](int t) { return max(__builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, (float)blocks[t * 4 + wave][3])), 0); };
    auto load_keys = [&](int t) {
        const u32x4p_t *p = (const u32x4p_t *)(pa.k + (size_t)pool_of(t) * (16 * D));
#pragma unroll
        for (int j = 0; j < J; ++j) rk[j] = p[j * 64 + lane];
    };
    auto load_values = [&](int t) {
        const u32x4p_t *p = (const u32x4p_t *)(pa.v + (size_t)pool_of(t) * (16 * D));
#pragma unroll
        for (int j = 0; j < J; ++j) rv[j] = p[j * 64 + lane];
    };
    auto store_key = [&](int kb, int i) {                              // i of 2 J: half of load i / 2
        const u32x4p_t w = rk[i >> 1];
        *(half8p_t *)(lds + kb * kTileBytes + (wave * KS * 64 + lane) * 16 + i * 1024) = i & 1 ? codes_to_half8(w.z, w.w) : codes_to_half8(w.x, w.y);
    };
    auto store_value = [&](int vb, int i) {                            // i of 4 J: the four tokens of one element of load i / 4
        half2p_t lo, hi;
        const uint32_t w = rv[i >> 2][i & 3];
        codes_to_half(w, lo, hi);
        *(u32x2p_t *)(lds + (2 + vb) * kTileBytes + ((wave >> 1) * NT * 64 + lane) * 16 + (wave & 1) * 8 + i * 1024) =
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
    // piece i of 4 CT: two weights, in the order block, column tile, pair
    auto weights = [&](const Scores &S, const Block (&bl)[2], int i) {
        const int u = i / (2 * CT), ct = i / 2 % CT, e = i % 2 * 2;
        const float off = bl[u][1] + kBias - m[ct];
        float x0 = __builtin_amdgcn_exp2f(fmaf(S.s[u][ct][e], bl[u][0], off)), x1 = __builtin_amdgcn_exp2f(fmaf(S.s[u][ct][e + 1], bl[u][0], off));
        asm volatile("" : "+v"(x0), "+v"(x1));                         // computed here and not where they are first used
        sum[u][ct] = e ? sum[u][ct] + (x0 + x1) : x0 + x1;
        pf[ct][4 * u + e] = (_Float16)x0, pf[ct][4 * u + e + 1] = (_Float16)x1;
    };
    auto mask = [&](Scores &S, int at, int t0, bool bad) {             // at: the first of the two blocks in the segment
        if (t0 + 31 > wave_min || bad) {                               // uniform
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool there = __builtin_bit_cast(int, (float)blocks[at + u][3]) >= 0;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!there || t0 + 16 * u + 4 * quarter + i > pos[ct]) S.s[u][ct][i] = -INFINITY;
            }
        }
    };
    // The weights were computed against the reference as it was.  Where one has left fp16's range behind 2^15 (or every column is new), the reference
    // moves to the maximum of these scores, what was summed against the old one is rescaled and the weights are computed again: rare behind the first
    // tiles of a row, and a look at the packed weights costs a quarter of the maxima of the scores.
    auto settle = [&](const Scores &S, const Block (&bl)[2]) {
        half2p_t top = {(_Float16)0.0f, (_Float16)0.0f};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, half2p_t{pf[ct][2 * i], pf[ct][2 * i + 1]});
        if (__any(fmaxf((float)top.x, (float)top.y) > kMost)) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float mx = -INFINITY;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, S.s[u][ct][i] * bl[u][0]);
                float2 both = pair_xor16(mx);
                both = pair_xor32(fmaxf(both.x, both.y));
                mx = fmaxf(both.x, both.y);
                const float to = mx > m[ct] ? mx : m[ct], alpha = __builtin_amdgcn_exp2f(m[ct] - to);
                m[ct] = to, l[ct] *= alpha;
#pragma unroll
                for (int i = 0; i < NT; ++i) O[i][ct] *= alpha;
            }
#pragma unroll
            for (int i = 0; i < 4 * CT; ++i) weights(S, bl, i);
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) l[ct] = fmaf(sum[1][ct], bl[1][2], fmaf(sum[0][ct], bl[0][2], l[ct]));
    };

    for (int seg = b_begin; seg < b_end; seg += kSegment) {
        // ---- numbers and scales of the segment's blocks, three per thread ----
        int pool[kSegment / 256];
        float ks[kSegment / 256], vs[kSegment / 256], top = 0.0f;
        int bad_any = 0;
#pragma unroll
        for (int j = 0; j < kSegment / 256; ++j) {
            const int blk = seg + j * 256 + tid;
            pool[j] = -1, ks[j] = vs[j] = 0.0f;
            if (blk < b_end) {
                pool[j] = paged_block(pa, g, kvh, si.slot, blk);
                if (pool[j] < 0) bad_any = 1, atomicOr(pa.err, kBadPage);
                else ks[j] = pa.k_scale[pool[j]], vs[j] = pa.v_scale[pool[j]];
            }
        }
#pragma unroll
        for (int j = 0; j < kSegment / 256; ++j) top = fmaxf(top, vs[j]);
        top = wave_max(top);
        __syncthreads();                                               // the segment before is consumed
        if (tid == 0) bad_s = 0;
        if (lane == 0) v_tops[wave] = top;
        __syncthreads();
        const float ref = fmaxf(fmaxf(fmaxf(v_tops[0], v_tops[1]), fmaxf(v_tops[2], v_tops[3])), v_ref);
        if (bad_any) bad_s = 1;
#pragma unroll
        for (int j = 0; j < kSegment / 256; ++j) {
            const float lr = vs[j] > 0.0f ? fmaxf(__builtin_amdgcn_logf(vs[j] / ref), -60.0f) : 0.0f;
            // (codes of a zero scale are zero; -inf times its factor has to stay -inf)
            blocks[j * 256 + tid] = Block{fmaxf(ks[j] * c, 0x1p-100f), lr, __builtin_amdgcn_exp2f(-lr), __builtin_bit_cast(float, pool[j])};
        }
        if (v_ref > 0.0f && ref > v_ref) {                             // O is in units of the largest value scale so far
            const float f = v_ref / ref;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) O[i][ct] *= f;
        }
        v_ref = ref;
        __syncthreads();
        const bool bad = __builtin_amdgcn_readfirstlane(bad_s) != 0;

        // ---- the segment's tiles ----
        const int first = seg * 16, nt = (min(b_end - seg, kSegment) + 3) >> 2;
        load_keys(0), load_values(0);
#pragma unroll
        for (int i = 0; i < 2 * J; ++i) store_key(0, i);
#pragma unroll
        for (int i = 0; i < 4 * J; ++i) store_value(0, i);
        if (nt > 1) load_keys(1), load_values(1);
        lds_barrier();
        Scores S[2];
        Block bl[2];
#pragma unroll
        for (int i = 0; i < PD; ++i) ring[i] = read_key(0, 0, i);
#pragma unroll
        for (int i = 0; i < G; ++i) {
            key_step(S[0], i);
            if (i + PD < G) ring[i % PD] = read_key(0, 0, i + PD);
        }
        mask(S[0], 0, first, bad);
        for (int t = 0; t < nt; ++t) {
            const int kb = t & 1;
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                Scores &cur = S[sub], &ahead = S[sub ^ 1];
                // ---- scores of the next 32 tokens between the exponentials of these (behind the last tile: of an old one, not used) ----
                const int key_buf = sub ? kb ^ 1 : kb, at = t * 4 + 2 * sub;
#pragma unroll
                for (int i = 0; i < PD; ++i) ring[i] = read_key(key_buf, sub ^ 1, i);
                bl[0] = blocks[at], bl[1] = blocks[at + 1];
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    key_step(ahead, i);
                    ring[i % PD] = i + PD < G ? read_key(key_buf, sub ^ 1, i + PD) : read_value(kb, sub, i + PD - G);
#pragma unroll
                    for (int w = i * 4 * CT / G; w < (i + 1) * 4 * CT / G; ++w) weights(cur, bl, w);
                    __builtin_amdgcn_sched_barrier(0);
                }
                settle(cur, bl);
                // ---- products with V between the staging of the next tile: keys, then values ----
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    value_step(i);
                    if (i + PD < G) ring[i % PD] = read_value(kb, sub, i + PD);
                    if (sub == 0) {                                    // (behind the last tile: the same once more, not read)
#pragma unroll
                        for (int w = i * 2 * J / G; w < (i + 1) * 2 * J / G; ++w) store_key(kb ^ 1, w);
                    } else {
#pragma unroll
                        for (int w = i * 4 * J / G; w < (i + 1) * 4 * J / G; ++w) store_value(kb ^ 1, w);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                mask(ahead, min(at + 2, kSegment - 2), first + t * 64 + (sub + 1) * 32, bad);
                if (t + 2 < nt) {
                    if (sub == 0) load_keys(t + 2);
                    else load_values(t + 2);
                }
                lds_barrier();
            }
        }
    }

    // ---- results: lane holds elements 16 i + 4 quarter .. + 3 of its columns ----
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const float den = xor32_sum(xor16_sum(l[ct]));
        const int place = (wave * CT + ct) * 16 + col;
        if (place >= n_pairs) continue;
        const int pair = p0 + place, row = pair / rep;
        const size_t at = (size_t)(si.q_start + row) * h + kvh * rep + pair - row * rep;
        if (splits > 1) {
            float *dst = part + (at * splits + split) * (D + 2);
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) dst[i * 16 + quarter * 4 + j] = O[i][ct][j] * v_ref;
            if (quarter == 0) dst[D] = m[ct], dst[D + 1] = den;
        } else {
            const float inv = (den > 0.0f ? 1.0f / den : den) * v_ref;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const float4p_t o = O[i][ct] * inv;
                const uint32_t lo = f2h(o.x) | (uint32_t)f2h(o.y) << 16, hi = f2h(o.z) | (uint32_t)f2h(o.w) << 16;
                *(u32x2p_t *)(out + at * D + i * 16 + quarter * 4) = u32x2p_t{lo, hi};
            }
        }
    }
}

template <int D, int CT>
hipError_t launch_one(const uint16_t *q, const PagedArgs &pa, const relax_layer_dims &dm, const PagedSeqs &st, const PagedRows &pl, uint16_t *out, float *partials,
                      hipStream_t stream)
{
    const dim3 grid(dm.n_kv_heads, pl.splits, pl.tiles * st.B);
    hipLaunchKernelGGL((attn_paged_rows_kernel<D, CT>), grid, dim3(256), 0, stream, st, q, pa, partials, out, dm.n_heads, dm.n_kv_heads, pl.tiles, pl.chunk, pl.splits,
                       pl.least);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_rows(const uint16_t *q, const PagedArgs &pa, const relax_layer_dims &dm, const PagedSeqs &st, const PagedRows &pl, uint16_t *out,
                             float *partials, hipStream_t stream)
{
    if (dm.head_dim == 128) return pl.ct == 2 ? launch_one<128, 2>(q, pa, dm, st, pl, out, partials, stream) : launch_one<128, 1>(q, pa, dm, st, pl, out, partials, stream);
    return pl.ct == 2 ? launch_one<64, 2>(q, pa, dm, st, pl, out, partials, stream) : launch_one<64, 1>(q, pa, dm, st, pl, out, partials, stream);
}

}  // namespace relax
