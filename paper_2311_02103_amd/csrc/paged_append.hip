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
// their own, q is rotated by further workgroups of the same launch.  Bound by latency for a decode step and by bytes for a prompt.
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

// what a value is quantised from: fp16's range, a NaN is 0
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

// Tokens low .. high - 1 of a block are the call's; row: the call's row of token 0 of the block (low's row minus low)
template <int D>
__device__ __forceinline__ void put_keys(const RowsView &r, const PagedArgs &pa, int pool, int kvh, int lane, int low, int high, int row, int pos)
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
        if (pa.rope) rotate8(a[i], b[i], pa.rope + ((size_t)(pos + src) * (D / 2) + e) * 2);
    }
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            a[i][j] = storable(a[i][j]), b[i][j] = storable(b[i][j]);
            amax = fmaxf(amax, fmaxf(fabsf(a[i][j]), fabsf(b[i][j])));
        }
    amax = wave_max(amax);
    const NewScale n = new_scale(amax, low > 0, low > 0 ? pa.k_scale[pool] : 0.0f);
    if (lane == 0) pa.k_scale[pool] = n.s;
    uint8_t *blk = pa.k + (size_t)pool * (16 * D);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const int e = (quarter + 4 * i) * 8 + hh * (D / 2);
            u32x2p_t *at = (u32x2p_t *)(blk + (e >> 4) * 256 + tok * 16 + (e & 15));
            u32x2p_t w;
            if (fresh) {
                const float *val = hh ? b[i] : a[i];
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    w[p] = code_of(val[4 * p], n) | code_of(val[4 * p + 1], n) << 8 | code_of(val[4 * p + 2], n) << 16 | code_of(val[4 * p + 3], n) << 24;
                *at = w;
            } else if (tok < low && n.grew) {
                w = *at;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const uint32_t o = w[p];
                    w[p] = recode(o & 255u, n.keep) | recode(o >> 8 & 255u, n.keep) << 8 | recode(o >> 16 & 255u, n.keep) << 16 | recode(o >> 24, n.keep) << 24;
                }
                *at = w;
            }
        }
}

template <int D>
__device__ __forceinline__ void put_values(const RowsView &r, const PagedArgs &pa, int pool, int kvh, int lane, int low, int high, int row)
{
    const int m = lane & 15, t0 = (lane >> 4) * 4;             // the lane's elements are m + 16 i, its tokens t0 .. t0 + 3
    float x[D / 16][4];
    float amax = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int src = min(max(t0 + t, low), high - 1);
        const uint16_t *at = r.v + (row + src) * r.kv_stride + kvh * D + m;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) x[i][t] = h2f(at[16 * i]);
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            x[i][t] = storable(x[i][t]);
            amax = fmaxf(amax, fabsf(x[i][t]));
        }
    amax = wave_max(amax);
    const NewScale n = new_scale(amax, low > 0, low > 0 ? pa.v_scale[pool] : 0.0f);
    if (lane == 0) pa.v_scale[pool] = n.s;
    const bool all_new = t0 >= low && t0 + 3 < high, none = t0 + 3 < low || t0 >= high;
    if (none && !(n.grew && t0 < low)) return;
    u32x4p_t *blk = (u32x4p_t *)(pa.v + (size_t)pool * (16 * D));
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
        u32x4p_t w = {0, 0, 0, 0};
        if (!all_new) w = blk[j * 64 + lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t o = w[i];
            uint32_t c = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint32_t u = o >> (8 * t) & 255u;
                if (t0 + t >= low && t0 + t < high) u = code_of(x[4 * j + i][t], n);
                else if (t0 + t < low && n.grew) u = recode(u, n.keep);
                c |= u << (8 * t);
            }
            w[i] = c;
        }
        blk[j * 64 + lane] = w;
    }
}

// Workgroups 0 .. kv_groups - 1: four wavefronts, each one (item, KV head, keys or values); the rest: rows of q, `slices` workgroups per row
template <int D>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedSeqs, RowsView r, uint16_t *q_out, PagedArgs pa, int h, int g, int items, int kv_groups, int slices)
{
    const SeqsArg st = seqs_arg();
    const int lane = threadIdx.x & 63;
    if ((int)blockIdx.x < kv_groups) {
        const int w = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6));
        const int item = w / (2 * g), part = w - item * 2 * g, kvh = part >> 1;
        if (item >= items) return;
        int place, b = item;
        if (st->q_max == 1) place = 0;
        else b = seq_of(st, item, [](int q_len) { return paged_blocks_of(q_len); }, place);
        if (b >= st->B) return;
        const SeqSpan si = seq_span(st, b);
        const int first = si.kv_len - si.q_len;                // position of the sequence's first row
        const int blk = (first >> 4) + place;
        const int low = max(first - blk * 16, 0), high = min(si.kv_len - blk * 16, 16);
        if (first < 0 || high <= low) return;
        const int pool = si.kv_len <= pa.cap ? paged_block(pa, g, kvh, si.slot, blk) : -1;
        if (pool < 0) {
            if (lane == 0) atomicOr(pa.err, kBadPage);
            return;
        }
        const int row = si.q_start + blk * 16 - first;
        if (part & 1) put_values<D>(r, pa, pool, kvh, lane, low, high, row);
        else put_keys<D>(r, pa, pool, kvh, lane, low, high, row, blk * 16);
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
__global__ __launch_bounds__(256) void paged_read_kernel(PagedSeqs, PagedArgs pa, uint16_t *k_out, uint16_t *v_out, int g, int items)
{
    const SeqsArg st = seqs_arg();
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6));
    const int item = w / (2 * g), part = w - item * 2 * g, kvh = part >> 1;
    if (item >= items || !(part & 1 ? v_out : k_out)) return;
    int place, b = item;
    if (st->q_max == 1) place = 0;
    else b = seq_of(st, item, [](int q_len) { return paged_blocks_of(q_len); }, place);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, b);
    const int first = si.kv_len - si.q_len, blk = (first >> 4) + place;
    const int low = max(first - blk * 16, 0), high = min(si.kv_len - blk * 16, 16);
    if (first < 0 || high <= low) return;
    const int pool = si.kv_len <= pa.cap ? paged_block(pa, g, kvh, si.slot, blk) : -1;
    if (pool < 0 && lane == 0) atomicOr(pa.err, kBadPage);
    const int row = si.q_start + blk * 16 - first, at = max(pool, 0);
    const float s = pool < 0 ? 0.0f : (part & 1 ? pa.v_scale : pa.k_scale)[at];       // no page: zeros
    const u32x4p_t *src = (const u32x4p_t *)((part & 1 ? pa.v : pa.k) + (size_t)at * (16 * D));
    const int c = lane & 15, quarter = lane >> 4;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
        const u32x4p_t code = src[j * 64 + lane];
        if (part & 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t o = code[i];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int tok = quarter * 4 + t;
                    if (tok >= low && tok < high)
                        v_out[((size_t)(row + tok) * g + kvh) * D + j * 64 + i * 16 + c] = f2h((float)((int)(o >> (8 * t) & 255u) - 128) * s);
                }
            }
        } else if (c >= low && c < high) {
            uint16_t *dst = k_out + ((size_t)(row + c) * g + kvh) * D + (j * 4 + quarter) * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                half8p_t x;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t o = code[2 * i + (e >> 2)];
                    x[e] = (_Float16)((float)((int)(o >> (8 * (e & 3)) & 255u) - 128) * s);
                }
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
    const int kv_groups = (items * 2 * dm.n_kv_heads + 3) / 4;
    const int units = dm.n_heads * (dm.head_dim / 16), slices = st.n >= 256 ? 1 : (units + 255) / 256;     // few rows: over several workgroups
    const dim3 grid(kv_groups + (q ? st.n * slices : 0));
    if (dm.head_dim == 128)
        hipLaunchKernelGGL(paged_append_kernel<128>, grid, dim3(256), 0, stream, st, r, q_out, pa, dm.n_heads, dm.n_kv_heads, items, kv_groups, slices);
    else
        hipLaunchKernelGGL(paged_append_kernel<64>, grid, dim3(256), 0, stream, st, r, q_out, pa, dm.n_heads, dm.n_kv_heads, items, kv_groups, slices);
    return hipGetLastError();
}

hipError_t launch_paged_read(const PagedArgs &pa, uint16_t *k_out, uint16_t *v_out, const relax_layer_dims &dm, const PagedSeqs &st, int items, hipStream_t stream)
{
    const dim3 grid((items * 2 * dm.n_kv_heads + 3) / 4);
    if (dm.head_dim == 128) hipLaunchKernelGGL(paged_read_kernel<128>, grid, dim3(256), 0, stream, st, pa, k_out, v_out, dm.n_kv_heads, items);
    else hipLaunchKernelGGL(paged_read_kernel<64>, grid, dim3(256), 0, stream, st, pa, k_out, v_out, dm.n_kv_heads, items);
    return hipGetLastError();
}

}  // namespace relax
