// Causal attention over the paged 8-bit KV cache.
//
//   o[i] = sum_t p[i,t] v[t],   p[i,:] = softmax_t(q[i] . k[t] / sqrt d),  t = 0 .. pos_i,   k[t] = s_k[t / 16] (u_k[t] - 128), v likewise
//
// The query heads of a KV head and the rows of a sequence are one list of (row, head) pairs: pair p is row p / rep, head p % rep of the group.
// A workgroup takes 16 consecutive pairs, the columns of the MFMA tiles, against one KV head and one split of the tokens; its four
// or eight wavefronts take a share of the split each.  With S^T = K Q^T a pair is a column of the result and the lane (quarter, column) holds tokens
// 4 quarter .. + 3 of a block; the same lane's eight probabilities of two blocks are what the B operand of O^T = V^T P^T wants from it, and
// the codes come in as the A operands (paged_device.h), so nothing passes through LDS or another lane but the maxima.
//
// Scales.  The codes go into the products as integers.  A block's key scale times log2(e) / sqrt(d) multiplies its scores; its value scale,
// divided by the largest of the wavefront's blocks so that it is at most 1, multiplies the probabilities in front of their rounding to fp16, and the largest
// one the result.  exp2's argument is offset by 11 in return: the largest probability is at most 2^15 (the reference trails the maximum by
// at most 2^4) and one of 2^-39 of it still is a subnormal fp16 number.  Scores, sums and O are fp32; the rounding of the probabilities (2^-11 relative, independent
// from token to token) is the only one between the codes and the result.
#include <algorithm>
#include <type_traits>

#include "paged_device.h"

namespace relax {

namespace {

constexpr float kBias = 11.0f, kLag = 4.0f;      // log2: offset of the weights, and how far the reference may trail the maximum

// grid: x = tile * g + KV head (the heads of a tile on neighbouring dies, a head's tiles on one, with eight heads), y = split.  part: [row][head][splits][D + 2] when splits > 1.
template <int D, int W>
__global__ __launch_bounds__(64 * W, 4) void attn_paged_kernel(PagedSeqs, const uint16_t *__restrict__ q, PagedArgs pa, float *__restrict__ part,
                                                            uint16_t *__restrict__ out, int h, int g, int per_seq, int chunk, int splits, int least)
{
    constexpr int J = D / 64;                    // 1 KB loads per block
    constexpr int NT = D / 16;                   // 16-element tiles of O^T
    constexpr int P = D + 4;                     // pitch of a state in LDS
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
    const int past = si.kv_len - si.q_len;
    const int n_pairs = min(16, pairs - p0);
    const bool beyond = beyond_capacity(si, pa.cap);
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

    // ---- queries: lane holds pair `col`; k step 2 j + half takes elements 16 (4 j + quarter) + 8 half .. + 7 ----
    const int pair = p0 + min(col, n_pairs - 1), row = pair / rep, head = kvh * rep + pair - row * rep, pos = past + row;
    half8p_t qf[2 * J];
    {
        const uint16_t *src = q + ((size_t)(si.q_start + row) * h + head) * D + quarter * 16;
#pragma unroll
        for (int j = 0; j < 2 * J; ++j) qf[j] = *(const half8p_t *)(src + (j >> 1) * 64 + (j & 1) * 8);
    }
    const float c = 1.44269504088896340736f / sqrtf((float)D);

    float4p_t O[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) O[i] = float4p_t{0.0f, 0.0f, 0.0f, 0.0f};
    float m_run = -INFINITY, l_run = 0.0f, v_ref = 0.0f;

    for (int seg = w_begin; seg < w_end; seg += kWave) {
        // ---- lane j: number in the pool and scales of block seg + j ----
        int pool = -1;
        if (seg + lane < w_end) {
            pool = paged_block(pa, g, kvh, si.slot, seg + lane);
            if (pool < 0) atomicOr(pa.err, kBadPage);
        }
        float ks = pa.k_scale[max(pool, 0)], vs = pa.v_scale[max(pool, 0)];
        const int ns = (min(w_end - seg, kWave) + 1) >> 1;

        u32x4p_t kreg[2 * J], vreg[2 * J];                     // one step: two blocks
        auto load = [&](u32x4p_t (&reg)[2 * J], const uint8_t *codes, int s) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int at = max(__builtin_amdgcn_readlane(pool, min(2 * s + t, 63)), 0);       // no such block: any that can be read
                const u32x4p_t *p = (const u32x4p_t *)(codes + (size_t)at * (16 * D));
#pragma unroll
                for (int j = 0; j < J; ++j) reg[t * J + j] = stream_load(p + j * 64 + lane);
            }
        };
        // the first step is on its way before the scales are needed, and the scales ahead of it
        __builtin_amdgcn_sched_barrier(0);
        load(kreg, pa.k, 0), load(vreg, pa.v, 0);
        __builtin_amdgcn_sched_barrier(0);
        ks = pool < 0 ? 0.0f : ks * c, vs = pool < 0 ? 0.0f : vs;
        const float ref = fmaxf(v_ref, wave_max(vs));
        if (v_ref > 0.0f && ref > v_ref) {                     // later blocks have larger values: O is in units of the largest scale
            const float f = v_ref / ref;
#pragma unroll
            for (int i = 0; i < NT; ++i) O[i] *= f;
        }
        v_ref = ref;
        const float vr = ref > 0.0f ? vs / ref : 0.0f;
        // a step's keys make room for the next one's as soon as the scores are there, its values when they are summed: one step is in flight all the time
        auto step = [&](int s, auto MORE) __attribute__((always_inline)) {
            float x[8];
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float4p_t S = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const u32x4p_t w = kreg[t * J + j];
                    S = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half8(w.x, w.y), qf[2 * j], S, 0, 0, 0);
                    S = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half8(w.z, w.w), qf[2 * j + 1], S, 0, 0, 0);
                }
                const int at = min(2 * s + t, 63);
                const bool there = __builtin_amdgcn_readlane(pool, at) >= 0;
                const float kc = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ks), at));
                const int t0 = (seg + 2 * s + t) * 16;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[4 * t + i] = S[i] * kc;
                if (!there || t0 + 15 > pos_min) {             // uniform
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!there || t0 + 4 * quarter + i > pos) x[4 * t + i] = -INFINITY;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, x[4 * t + i]);
            }
            if constexpr (MORE) load(kreg, pa.k, s + 1);
            float2 both = pair_xor16(mx);
            both = pair_xor32(fmaxf(both.x, both.y));
            mx = fmaxf(both.x, both.y);
            const bool move = mx > m_run + kLag;               // the first visible tokens: m_run = -inf
            if (__any(move)) {
                const float m_new = move ? mx : m_run, alpha = move ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.0f;
                l_run *= alpha;
                m_run = m_new;
#pragma unroll
                for (int i = 0; i < NT; ++i) O[i] *= alpha;
            }
            const float m_ref = m_run == -INFINITY ? 0.0f : m_run - kBias;      // nothing visible yet: every weight is exp2(-inf)
            half8p_t pf;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float r = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, vr), min(2 * s + t, 63)));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(x[4 * t + i] - m_ref);
                    l_run += p;
                    pf[4 * t + i] = (_Float16)(p * r);
                }
            }
#pragma unroll
            for (int i = 0; i < NT; ++i)
                O[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half8(vreg[i >> 2][i & 3], vreg[J + (i >> 2)][i & 3]), pf, O[i], 0, 0, 0);
            if constexpr (MORE) load(vreg, pa.v, s + 1);
        };
#pragma unroll 1
        for (int s = 0; s + 1 < ns; ++s) step(s, std::true_type{});
        step(ns - 1, std::false_type{});
    }

    // ---- the wavefronts' states meet in LDS ----
    l_run = xor32_sum(xor16_sum(l_run));
#pragma unroll
    for (int i = 0; i < NT; ++i) *(float4p_t *)(states + (wave * 16 + col) * P + i * 16 + quarter * 4) = O[i] * v_ref;
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
            const float mw = sm_m[w * 16 + pc], f = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - mm);
            num += *(const float4p_t *)(states + (w * 16 + pc) * P + e) * f;
            den += sm_l[w * 16 + pc] * f;
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

// out of (row, head) from its splits, one workgroup each: D / 4 threads take four elements of a split, as many splits as there are such
// groups of threads side by side and four of each in flight, and the groups' results meet in LDS
template <int D>
__global__ __launch_bounds__(256) void attn_paged_merge_kernel(PagedSeqs, const float *__restrict__ part, uint16_t *__restrict__ out, int h, int g, int cap,
                                                               int chunk, int splits, int least)
{
    constexpr int T = D / 4, F = 4;
    __shared__ __align__(16) float sums[256 / T][D];
    __shared__ float sm_m[256 / T], sm_l[256 / T];
    const SeqsArg st = seqs_arg();
    const int i = blockIdx.x, r = i / h, hd = i - r * h, rep = h / g;
    const int tid = threadIdx.x, grp = tid / T, e = tid % T * 4, groups = blockDim.x / T;
    int place, b = r;
    if (st->q_max == 1) place = 0;
    else b = seq_of(st, r, [](int q_len) { return q_len; }, place);
    const SeqSpan si = seq_span(st, __builtin_amdgcn_readfirstlane(b));
    // the splits that the tile of this pair had: those of its last pair
    const int pairs = si.q_len * rep, pair = place * rep + hd % rep, last = min(pair | 15, pairs - 1) / rep;
    if (pairs >= least) return;                                // (not split: the other kernel's)
    const int vis = beyond_capacity(si, cap) ? 0 : si.kv_len - si.q_len + last + 1, used = min(max((vis + chunk - 1) / chunk, 1), splits);
    const float *src = part + (size_t)i * splits * (D + 2);
    float mm = -INFINITY, den = 0.0f;
    float4p_t num = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = grp; s0 < used; s0 += groups * F) {
        float ms[F], ls[F];
        float4p_t as[F];
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const float *p = src + (size_t)min(s0 + j * groups, used - 1) * (D + 2);
            ms[j] = p[D], ls[j] = p[D + 1], as[j] = float4p_t{p[e], p[e + 1], p[e + 2], p[e + 3]};
        }
        float mx = mm;
#pragma unroll
        for (int j = 0; j < F; ++j) mx = s0 + j * groups < used ? fmaxf(mx, ms[j]) : mx;
        const float ref = mx == -INFINITY ? 0.0f : mx, f0 = __builtin_amdgcn_exp2f(mm - ref);
        den *= f0, num *= f0;
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const float f = s0 + j * groups < used ? __builtin_amdgcn_exp2f(ms[j] - ref) : 0.0f;
            den += ls[j] * f, num += as[j] * f;
        }
        mm = mx;
    }
    *(float4p_t *)&sums[grp][e] = num;
    if (e == 0) sm_m[grp] = mm, sm_l[grp] = den;
    __syncthreads();
    if (grp > 0) return;
    for (int w = 0; w < groups; ++w) mm = fmaxf(mm, sm_m[w]);
    num = float4p_t{0.0f, 0.0f, 0.0f, 0.0f}, den = 0.0f;
    for (int w = 0; w < groups; ++w) {
        const float f = sm_m[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_m[w] - mm);
        num += *(const float4p_t *)&sums[w][e] * f, den += sm_l[w] * f;
    }
    const float inv = den > 0.0f ? 1.0f / den : den;
    const uint32_t lo = f2h(num.x * inv) | (uint32_t)f2h(num.y * inv) << 16, hi = f2h(num.z * inv) | (uint32_t)f2h(num.w * inv) << 16;
    *(u32x2p_t *)(out + (size_t)i * D + e) = u32x2p_t{lo, hi};
}

// Splits of a launch with `small` workgroups per split: from kUnsplit workgroups on none, below it as many as bring it to kPagedGroups workgroups, at most one
// per 128 tokens of the longest sequence (rounded up to 32 tokens, a split has 96 at least), and no more than kPagedPartials partial results (row, head, split).  The workgroups of a split launch have eight
// wavefronts where a split has 256 tokens and more, as many tokens in flight with half the partial results.
// us, unsplit / split: 16 x 3 rows of 64 / 8 heads (256 workgroups) 18.5 / 23, 4 x 17 rows of them (288) 20 / 25, 16 x 16 rows of 32 / 32 (512) 28 / 38.  16 decode rows
// of 64 / 8 heads with 768 workgroups 31.6, with 512 35.8, with 1024 32.7, with four wavefronts 36.
constexpr int kUnsplit = 256, kPagedGroups = 768;

// The kernel of 256-pair tiles takes the sequences that fill one, in calls that have kRowTiles such tiles over all KV heads: it halves the time of long prompts
// and loses on the rest, where its workgroups are few and each waits 5 us for its first tile (us, tiles of 16 / of 256; heads of 128): 2048 rows of 32 / 32 heads
// (256 tiles) 114 / 73, 1000 rows on 300 tokens of 40 / 40 (160) 59 / 51, 511 rows of 64 / 8 (128) 24 / 37, 300 rows on 1201 of 32 / 32 (64) 28 / 34,
// 600 rows on 500 tokens of 16 / 2 heads of 64 (38) 14.5 / 24.
constexpr int kRowTiles = 160;

// Tiles are searched for where a fixed number per sequence would launch more than twice as many (us: 300 rows on 1201 tokens beside 20 decode rows of 32 / 32 heads,
// 39 tiles per KV head numbered as 399, 46.8; searched for, 42.0)
void numbering(long long all, long long most, int32_t B, int32_t &items, int32_t &per_seq)
{
    const bool search = most * B > 2 * all;
    items = (int32_t)(search ? all : most * B);
    per_seq = (int32_t)(search ? 0 : most);
}

template <int D>
hipError_t launch_d(const uint16_t *q, const PagedArgs &pa, const relax_layer_dims &dm, const PagedSeqs &st, const PagedPlan &pl, uint16_t *out, float *partials,
                    hipStream_t stream)
{
    if ((int64_t)pl.items * dm.n_kv_heads * 64 * pl.waves > kMaxThreads) return hipErrorInvalidValue;
    const dim3 grid(pl.items * dm.n_kv_heads, pl.splits);
    if (pl.waves == 8)
        hipLaunchKernelGGL((attn_paged_kernel<D, 8>), grid, dim3(512), 0, stream, st, q, pa, partials, out, dm.n_heads, dm.n_kv_heads, pl.per_seq, pl.chunk, pl.splits, pl.least);
    else
        hipLaunchKernelGGL((attn_paged_kernel<D, 4>), grid, dim3(256), 0, stream, st, q, pa, partials, out, dm.n_heads, dm.n_kv_heads, pl.per_seq, pl.chunk, pl.splits, pl.least);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.splits == 1) return e;
    const int threads = pl.splits > 4 * 64 / (D / 4) ? 256 : 64;      // one round of four splits per group of threads, if that is enough
    hipLaunchKernelGGL(attn_paged_merge_kernel<D>, dim3(st.n * dm.n_heads), dim3(threads), 0, stream, st, partials, out, dm.n_heads, dm.n_kv_heads, pa.cap,
                       pl.chunk, pl.splits, pl.least);
    return hipGetLastError();
}

}  // namespace

PagedPlan paged_plan(const relax_layer_dims &dm, const relax_seqs &sq, int32_t n, int32_t L_max, int32_t row_tiles)
{
    const int rep = dm.n_heads / dm.n_kv_heads;
    auto pairs_of = [&](int b) { return (long long)sq.q_lens[b] * rep; };
    long long large = 0;
    for (int b = 0; b < sq.B; ++b)
        if (pairs_of(b) >= kPagedRowTile) large += (pairs_of(b) + kPagedRowTile - 1) / kPagedRowTile;
    PagedPlan p;
    p.least = large * dm.n_kv_heads >= row_tiles ? kPagedRowTile : INT32_MAX;
    long long small = 0, most_small = 0, most_large = 0;
    for (int b = 0; b < sq.B; ++b) {
        const long long pairs = pairs_of(b);
        if (pairs >= p.least) most_large = std::max(most_large, pairs);
        else small += (pairs + 15) / 16, most_small = std::max(most_small, pairs);
    }
    if (p.least == INT32_MAX) large = 0;
    numbering(large, (most_large + kPagedRowTile - 1) / kPagedRowTile, sq.B, p.row_items, p.row_per_seq);
    numbering(small, (most_small + 15) / 16, sq.B, p.items, p.per_seq);
    long long s = small && small * dm.n_kv_heads < kUnsplit ? kPagedGroups / (small * dm.n_kv_heads) : 1;
    s = std::min(s, (long long)(L_max + 127) / 128);
    s = std::min(s, (long long)kPagedPartials / ((long long)n * dm.n_heads));
    s = std::max(s, 1LL);
    p.chunk = (int32_t)(((L_max + s - 1) / s + 31) / 32 * 32);
    p.splits = (L_max + p.chunk - 1) / p.chunk;
    p.waves = p.splits > 1 && p.chunk >= 256 ? 8 : 4;
    return p;
}

// paged_plan() has splits <= ceil(L / 128) and, where it has more than one, n * heads * splits <= kPagedPartials
size_t paged_partial_floats(const relax_layer_dims &dm, int32_t n, int32_t L)
{
    const size_t most = kPagedPartials, mine = (size_t)n * dm.n_heads * (((size_t)L + 127) / 128);
    return (mine < most ? mine : most) * (dm.head_dim + 2);
}

hipError_t launch_paged_attention(const uint16_t *q, const PagedArgs &pa, const relax_layer_dims &dm, const PagedSeqs &st, const relax_seqs &sq, int32_t L_max,
                                  uint16_t *out, float *partials, hipStream_t stream)
{
    const PagedPlan pl = paged_plan(dm, sq, st.n, L_max, kRowTiles);
    if (pl.row_items > 0) {
        const hipError_t e = launch_paged_rows(q, pa, dm, st, pl.row_items, pl.row_per_seq, pl.least, out, stream);
        if (e != hipSuccess || pl.items == 0) return e;
    }
    return dm.head_dim == 128 ? launch_d<128>(q, pa, dm, st, pl, out, partials, stream) : launch_d<64>(q, pa, dm, st, pl, out, partials, stream);
}

}  // namespace relax
