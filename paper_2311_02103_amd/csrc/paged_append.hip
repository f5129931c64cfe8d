// Appending to the paged 8-bit KV cache, with the rotary embedding on the way, and reading it back.
//
//   q'[i] = R(pos_i) q[i]                        half-split pairs (e, e + d/2), angles from the table, rounded once to fp16
//   k'[i] = R(pos_i) k[i]                        stays fp32 until it is quantised
//   s_new = max(s_old, max|x| / 127)             per block of 16 tokens and KV head, over the call's tokens in it; s_old = 0 if the call's
//                                                first token of the block is the block's first
//   u = 128 + rne(x / s_new);  codes that were there: u' = 128 + rne((u - 128) s_old / s_new) if the scale grew
//
// One wavefront is one (block, KV head) of keys or of values: it alone reads and writes the block's codes and scale, whatever the number of
// tokens the call brings for it, so nothing is atomic and the result does not depend on any order.  Keys and values are wavefronts of
// their own, q is rotated by further workgroups of the same launch.  Bound by latency for a decode step and by bytes for a prompt: 2043 rows of
// 32 / 32 heads of 128 take 19.6 us, 4.3 TB/s, 64 rows of 64 / 8 heads 6.4, one row 5.8, of which a launch is 2.
#include "paged_device.h"

namespace relax {

namespace {

struct RowsView {
    const uint16_t *q, *k, *v;
    int64_t q_stride, kv_stride;     // elements from one row to the next
};

__device__ __forceinline__ void load8p(const uint16_t *p, float *v)
{
    const half8p_t x = *(const half8p_t *)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)x[e];
}

// what of an input is quantised: the ends of fp16's range for infinities, 0 for a NaN.  In front of the rotation: inf * 0 would be a NaN in both elements of the pair,
// and a finite pair may leave that range behind it, which an fp32 scale holds
__device__ __forceinline__ float storable(float x) { return x == x ? fminf(fmaxf(x, -65504.0f), 65504.0f) : 0.0f; }

// pairs (a[e], b[e]) at the angles cs[2 e], cs[2 e + 1]
__device__ __forceinline__ void rotate8(float *a, float *b, const float *cs)
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float4p_t c2 = *(const float4p_t *)(cs + 2 * e);
        const float a0 = a[e], b0 = b[e], a1 = a[e + 1], b1 = b[e + 1];
        a[e] = a0 * c2.x - b0 * c2.y, b[e] = a0 * c2.y + b0 * c2.x;
        a[e + 1] = a1 * c2.z - b1 * c2.w, b[e + 1] = a1 * c2.w + b1 * c2.z;
    }
}

struct NewScale {
    float s, inv, keep;              // scale, its reciprocal, factor of the codes that were there
    bool grew;
};
// amax: largest magnitude of the call's tokens in the block; old: the block's scale if it holds earlier tokens
__device__ __forceinline__ NewScale new_scale(float amax, bool has_old, float old)
{
    NewScale n;
    const float s_old = has_old && old > 0.0f && old < 1e30f ? old : 0.0f;      // (never written: whatever the memory held)
    const float need = amax / 127.0f;
    n.s = fmaxf(s_old, need);
    n.grew = has_old && n.s > s_old;
    n.inv = n.s > 1e-30f ? 1.0f / n.s : 0.0f;
    n.keep = n.s > 0.0f ? s_old / n.s : 0.0f;
    return n;
}
// x / s to the last bit but for the rarest: the plain product with the reciprocal would round one value in 10^5 to the other side
__device__ __forceinline__ uint32_t code_of(float x, const NewScale &n)
{
    const float a = x * n.inv, q = fmaf(fmaf(-a, n.s, x), n.inv, a);
    return (uint32_t)((int)fminf(fmaxf(rintf(q), -127.0f), 127.0f) + 128);
}
__device__ __forceinline__ uint32_t recode(uint32_t u, float keep) { return (uint32_t)((int)rintf((float)((int)u - 128) * keep) + 128); }

// Tokens low .. high - 1 of a block are the call's; row: the call's row of token 0 of the block (low's row minus low).  find() is the block's number in the pool, -1
// if there is none: the rows are on their way and their largest magnitude known before its answer is waited for, because a decode step is
// this chain of loads (page, scale, codes) and nothing else.
template <int D, typename Find>
__device__ __forceinline__ bool put_keys(const RowsView &r, const PagedArgs &pa, const Find &find, int kvh, int lane, int low, int high, int row, int pos)
{
    constexpr int U = D / 64;                                  // units of eight pairs per lane
    const int tok = lane & 15, quarter = lane >> 4;
    const bool fresh = tok >= low && tok < high;
    const int src = min(max(tok, low), high - 1);              // (lanes of other tokens load the nearest one)
    float a[U][8], b[U][8];
    const uint16_t *x = r.k + (row + src) * r.kv_stride + kvh * D;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int e = (quarter + 4 * i) * 8;
        load8p(x + e, a[i]);
        load8p(x + e + D / 2, b[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) a[i][j] = storable(a[i][j]), b[i][j] = storable(b[i][j]);
        if (pa.rope) rotate8(a[i], b[i], pa.rope + ((size_t)(pos + src) * (D / 2) + e) * 2);
    }
    const int pool = find();
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fmaxf(fabsf(a[i][j]), fabsf(b[i][j])));
    amax = wave_max(amax);
    if (pool < 0) return false;
    // unit (i, half): elements (quarter + 4 i) * 8 + half * D / 2 of the lane's token
    const auto at = [&](int i, int hh) {
        const int e = (quarter + 4 * i) * 8 + hh * (D / 2);
        return (u32x2p_t *)(pa.k + (size_t)pool * (16 * D) + (e >> 4) * 256 + tok * 16 + (e & 15));
    };
    float old = 0.0f;
    u32x2p_t w[U][2] = {};
    if (low > 0) {
        old = pa.k_scale[pool];
#pragma unroll
        for (int i = 0; i < 2 * U; ++i) w[i >> 1][i & 1] = *at(i >> 1, i & 1);
    }
    const NewScale n = new_scale(amax, low > 0, old);
    if (lane == 0) pa.k_scale[pool] = n.s;
    if (!fresh && !(tok < low && n.grew)) return true;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const float *val = hh ? b[i] : a[i];
            u32x2p_t c;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const uint32_t o = w[i][hh][p];
                if (fresh) c[p] = code_of(val[4 * p], n) | code_of(val[4 * p + 1], n) << 8 | code_of(val[4 * p + 2], n) << 16 | code_of(val[4 * p + 3], n) << 24;
                else c[p] = recode(o & 255u, n.keep) | recode(o >> 8 & 255u, n.keep) << 8 | recode(o >> 16 & 255u, n.keep) << 16 | recode(o >> 24, n.keep) << 24;
            }
            *at(i, hh) = c;
        }
    return true;
}

// Values change hands in LDS between rows and codes: lane (c, quarter) has D / 16 consecutive elements c * D / 16 .. of the tokens 4 quarter .. + 3 as rows, and so
// D / 16 words of four codes; as codes it has 16-byte packets of the block.  The 64 words of each [e / 64][t / 4] lie kTurnPitch apart, with
// which the 64 words of one store, or load, are on 64 banks.  (With rows of values element by element, 2 bytes per lane, reading back 2043 tokens of
// 32 / 32 heads of 128 took 15.2 us for 11.7 and 64 rows of 64 / 8 heads 9.3 for 5.7; appending is bound by other things.)
constexpr int kTurnPitch = 68;
template <int D>
using Turn = uint32_t[D / 16 * kTurnPitch];
template <int D>
__device__ __forceinline__ int turn_word(int c, int quarter, int j)      // element e = c * D / 16 + j
{
    const int e = c * (D / 16) + j;
    return ((e >> 6) * 4 + quarter) * kTurnPitch + (e & 15) * 4 + (e >> 4 & 3);
}
__device__ __forceinline__ u32x4p_t *turn_packet(uint32_t *turn, int lane, int j) { return (u32x4p_t *)(turn + (j * 4 + (lane >> 4)) * kTurnPitch + (lane & 15) * 4); }
// a wavefront's LDS instructions execute in order: only the compiler has to keep it
__device__ __forceinline__ void turn_done()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int D, typename Find>
__device__ __forceinline__ bool put_values(const RowsView &r, const PagedArgs &pa, const Find &find, int kvh, int lane, int low, int high, int row, uint32_t *turn)
{
    constexpr int E = D / 16;
    typedef _Float16 part_t __attribute__((ext_vector_type(E)));
    const int c = lane & 15, quarter = lane >> 4, t0 = quarter * 4;
    part_t in[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
        in[t] = *(const part_t *)(r.v + (row + min(max(t0 + t, low), high - 1)) * r.kv_stride + kvh * D + c * E);
    const int pool = find();
    float x[E][4], amax = 0.0f;
#pragma unroll
    for (int j = 0; j < E; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            x[j][t] = storable((float)in[t][j]);
            amax = fmaxf(amax, fabsf(x[j][t]));
        }
    amax = wave_max(amax);
    if (pool < 0) return false;
    uint32_t fresh = 0, there = 0;                             // bytes of the call's tokens and of earlier ones in the lane's words
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if (t0 + t >= low && t0 + t < high) fresh |= 255u << (8 * t);
        if (t0 + t < low) there |= 255u << (8 * t);
    }
    u32x4p_t *blk = (u32x4p_t *)(pa.v + (size_t)pool * (16 * D));
    float old = 0.0f;
    u32x4p_t w[D / 64] = {};
    if (low > 0 || high < 16) {
        if (low > 0) old = pa.v_scale[pool];
#pragma unroll
        for (int j = 0; j < D / 64; ++j) w[j] = blk[j * 64 + lane];
    }
    const NewScale n = new_scale(amax, low > 0, old);
    if (lane == 0) pa.v_scale[pool] = n.s;
#pragma unroll
    for (int j = 0; j < E; ++j)
        turn[turn_word<D>(c, quarter, j)] = code_of(x[j][0], n) | code_of(x[j][1], n) << 8 | code_of(x[j][2], n) << 16 | code_of(x[j][3], n) << 24;
    turn_done();
    if (!fresh && !(n.grew && there)) return true;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
        u32x4p_t to = *turn_packet(turn, lane, j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t o = w[j][i];
            if (n.grew) {
                const uint32_t moved = recode(o & 255u, n.keep) | recode(o >> 8 & 255u, n.keep) << 8 | recode(o >> 16 & 255u, n.keep) << 16 | recode(o >> 24, n.keep) << 24;
                o = (o & ~there) | (moved & there);
            }
            to[i] = (to[i] & fresh) | (o & ~fresh);
        }
        blk[j * 64 + lane] = to;
    }
    return true;
}

// Workgroups 0 .. kv_groups - 1: four wavefronts, four of the 2 g (KV head, keys or values) of one item; the rest: rows of q, `slices` workgroups per row
template <int D>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedSeqs, RowsView r, uint16_t *q_out, PagedArgs pa, int h, int g, int kv_groups, int slices)
{
    __shared__ __align__(16) Turn<D> turn[4];
    const SeqsArg st = seqs_arg();
    const int lane = threadIdx.x & 63;
    if ((int)blockIdx.x < kv_groups) {
        const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), per_item = (g + 1) / 2;
        const int item = (int)blockIdx.x / per_item, part = ((int)blockIdx.x - item * per_item) * 4 + wave, kvh = part >> 1;
        if (part >= 2 * g) return;
        int place, b = item;
        if (st->q_max == 1) place = 0;
        else b = seq_of(st, item, [](int q_len) { return paged_blocks_of(q_len); }, place);
        if (b >= st->B) return;
        const SeqSpan si = seq_span(st, b);
        const int first = si.kv_len - si.q_len;                // position of the sequence's first row
        const int blk = (first >> 4) + place, lead = (first & 15) - place * 16;      // (no position of the block itself: a device table's length may be any number)
        const int low = max(lead, 0), high = min(lead + si.q_len, 16);
        if (first < 0 || high <= low) return;
        if (beyond_capacity(si, pa.cap)) {
            if (lane == 0) atomicOr(pa.err, kBadPage);
            return;
        }
        const int row = si.q_start - lead;
        const auto find = [&] { return paged_block(pa, g, kvh, si.slot, blk); };
        if (!(part & 1 ? put_values<D>(r, pa, find, kvh, lane, low, high, row, turn[wave])
                       : put_keys<D>(r, pa, find, kvh, lane, low, high, row, blk * 16)) && lane == 0) atomicOr(pa.err, kBadPage);
        return;
    }
    const int wg = (int)blockIdx.x - kv_groups, i = wg / slices, slice = wg - i * slices;
    int place, b = i;
    if (st->q_max == 1) place = 0;
    else b = seq_of(st, i, [](int q_len) { return q_len; }, place);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, b);
    const int pos = min(max(si.kv_len - si.q_len + place, 0), pa.cap - 1);
    constexpr int per_head = D / 16;
    const uint16_t *row = r.q + i * r.q_stride;
    uint16_t *dst = q_out + (size_t)i * h * D;
    for (int u = slice * 256 + threadIdx.x; u < h * per_head; u += slices * 256) {
        const int e = u / per_head * D + u % per_head * 8;
        float a[8], c[8];
        load8p(row + e, a);
        load8p(row + e + D / 2, c);
        if (pa.rope) rotate8(a, c, pa.rope + ((size_t)pos * (D / 2) + u % per_head * 8) * 2);
        half8p_t lo, hi;
#pragma unroll
        for (int j = 0; j < 8; ++j) lo[j] = (_Float16)a[j], hi[j] = (_Float16)c[j];
        *(half8p_t *)(dst + e) = lo;
        *(half8p_t *)(dst + e + D / 2) = hi;
    }
}

// out[row, kvh, :] = fp16(code * scale).  One wavefront is one (block, KV head) of keys or of values.
template <int D>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedSeqs, PagedArgs pa, uint16_t *k_out, uint16_t *v_out, int g)
{
    __shared__ __align__(16) Turn<D> turns[4];
    const SeqsArg st = seqs_arg();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int per_item = (g + 1) / 2, item = (int)blockIdx.x / per_item, part = ((int)blockIdx.x - item * per_item) * 4 + wave, kvh = part >> 1;
    if (part >= 2 * g || !(part & 1 ? v_out : k_out)) return;
    int place, b = item;
    if (st->q_max == 1) place = 0;
    else b = seq_of(st, item, [](int q_len) { return paged_blocks_of(q_len); }, place);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, b);
    const int first = si.kv_len - si.q_len, blk = (first >> 4) + place, lead = (first & 15) - place * 16;
    const int low = max(lead, 0), high = min(lead + si.q_len, 16);
    if (first < 0 || high <= low) return;
    const int pool = beyond_capacity(si, pa.cap) ? -1 : paged_block(pa, g, kvh, si.slot, blk);
    if (pool < 0 && lane == 0) atomicOr(pa.err, kBadPage);
    const int row = si.q_start - lead, at = max(pool, 0);
    const float s = pool < 0 ? 0.0f : (part & 1 ? pa.v_scale : pa.k_scale)[at];       // no page: zeros
    const u32x4p_t *src = (const u32x4p_t *)((part & 1 ? pa.v : pa.k) + (size_t)at * (16 * D));
    const int c = lane & 15, quarter = lane >> 4;
    u32x4p_t code[D / 64];
#pragma unroll
    for (int j = 0; j < D / 64; ++j) code[j] = src[j * 64 + lane];
    const auto value = [&](uint32_t w, int byte) {
        float x = (float)((int)(w >> (8 * byte) & 255u) - 128) * s;
        asm("" : "+v"(x));                                     // the fp32 product itself, not the one instruction that rounds code * s to fp16 without it
        return (_Float16)x;
    };
    if (part & 1) {
        constexpr int E = D / 16;
        typedef _Float16 part_t __attribute__((ext_vector_type(E)));
        uint32_t *turn = turns[wave];
#pragma unroll
        for (int j = 0; j < D / 64; ++j) *turn_packet(turn, lane, j) = code[j];
        turn_done();
        uint32_t o[E];
#pragma unroll
        for (int j = 0; j < E; ++j) o[j] = turn[turn_word<D>(c, quarter, j)];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int tok = quarter * 4 + t;
            part_t x;
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = value(o[j], t);
            if (tok >= low && tok < high) *(part_t *)(v_out + ((size_t)(row + tok) * g + kvh) * D + c * E) = x;
        }
    } else if (c >= low && c < high) {
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            uint16_t *dst = k_out + ((size_t)(row + c) * g + kvh) * D + (j * 4 + quarter) * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                half8p_t x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = value(code[j][2 * i + (e >> 2)], e & 3);
                *(half8p_t *)(dst + 8 * i) = x;
            }
        }
    }
}

}  // namespace

hipError_t launch_paged_append(const uint16_t *q, int64_t q_stride, const uint16_t *k, const uint16_t *v, int64_t kv_stride, uint16_t *q_out,
                               const PagedArgs &pa, const relax_layer_dims &dm, const PagedSeqs &st, int items, hipStream_t stream)
{
    const RowsView r = {q, k, v, q_stride, kv_stride};
    const int units = dm.n_heads * (dm.head_dim / 16), slices = st.n >= 256 ? 1 : (units + 255) / 256;     // few rows: over several workgroups
    const int64_t kv_groups = (int64_t)items * ((dm.n_kv_heads + 1) / 2), all = kv_groups + (q ? (int64_t)st.n * slices : 0);
    if (all * 256 > kMaxThreads) return hipErrorInvalidValue;
    const dim3 grid(all);
    if (dm.head_dim == 128) hipLaunchKernelGGL(paged_append_kernel<128>, grid, dim3(256), 0, stream, st, r, q_out, pa, dm.n_heads, dm.n_kv_heads, (int)kv_groups, slices);
    else hipLaunchKernelGGL(paged_append_kernel<64>, grid, dim3(256), 0, stream, st, r, q_out, pa, dm.n_heads, dm.n_kv_heads, (int)kv_groups, slices);
    return hipGetLastError();
}

hipError_t launch_paged_read(const PagedArgs &pa, uint16_t *k_out, uint16_t *v_out, const relax_layer_dims &dm, const PagedSeqs &st, int items, hipStream_t stream)
{
    const int64_t all = (int64_t)items * ((dm.n_kv_heads + 1) / 2);
    if (all * 256 > kMaxThreads) return hipErrorInvalidValue;
    const dim3 grid(all);
    if (dm.head_dim == 128) hipLaunchKernelGGL(paged_read_kernel<128>, grid, dim3(256), 0, stream, st, pa, k_out, v_out, dm.n_kv_heads);
    else hipLaunchKernelGGL(paged_read_kernel<64>, grid, dim3(256), 0, stream, st, pa, k_out, v_out, dm.n_kv_heads);
    return hipGetLastError();
}

}  // namespace relax
