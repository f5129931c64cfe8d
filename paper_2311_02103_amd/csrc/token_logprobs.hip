// Log probabilities of given tokens, entropies and the most likely tokens of rows of logits.
//
//   m = max x,  S = sum_v e^(x_v - m),  log p_v = x_v - m - log S,  H = log S - (sum_v e^(x_v - m) (x_v - m)) / S
//
// S is kept as 1 + rest, with one maximum counted and not added: log S = log1p(rest) then keeps its digits on rows whose top token is all but
// certain, where log(1 + rest) would be 0.
//
// One workgroup per row.  The row is read once and stays in registers for three passes (maxima; sums; candidates), rows beyond 163833 logits
// are read again by each pass.  The k best without a sort: thread maxima are folded into 64 groups (equal lanes of all
// wavefronts, so that neighbouring logits are spread over the groups), and the k-th largest group maximum T bounds the k-th largest
// logit from below; whatever is not smaller than T -- a few more than k on any row whose large logits do not share few groups -- goes to a list in
// LDS and is ranked by counting.  More than the list holds (many equal logits): T is replaced by the k-th largest logit itself, by bisection
// over the 16-bit values, the list takes what is larger, and the lowest indexes among those equal to T follow, found by a scan in order.
//
// A few rows of a large vocabulary are cut into slices, one workgroup each, whose sums and k best meet in a second kernel (uncut / cut, us: 1 row of 70000 logits 15.0 /
// 11.1, of 152064 with 20 alternatives 19.9 / 14.8, of 262000 36.6 / 15.2, 16 rows of 128256 17.7 / 13.8; 1 row of 50257 10.5 / 11.4; both sides are some
// 7 % faster now that a packet's candidates are found as bits first).
//
// Bound by the passes of a row one after the other, between the other rows' reads: a logit takes nine issue slots in the sums (four of them the exponential) and one and
// a half in the other two passes, which look at pairs; eight instead of nine changed nothing.  2047 rows of 32000 logits: 32 us without alternatives (4.1 TB/s), 39 to 43 with 20; 1 row 7.2.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "relax_common.h"

namespace relax {

namespace {

typedef uint32_t u32x4l_t __attribute__((ext_vector_type(4)));
typedef _Float16 half2l_t __attribute__((ext_vector_type(2)));

constexpr int kListed = 1024;        // places of the candidate list
constexpr uint32_t kNone2 = 0xFC00FC00u;        // (-inf, -inf)
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// fp16 values as integers of the same order, -0 and 0 alike; NaN never gets here
__device__ __forceinline__ int order_of(float x)
{
    const int u = f2h(x + 0.0f);                               // -0 + 0 = 0
    return u & 0x8000 ? 0xFFFF - u : u | 0x8000;
}
__device__ __forceinline__ float value_of(int order) { return h2f((uint16_t)(order & 0x8000 ? order & 0x7FFF : 0xFFFF - order)); }
// place of a candidate in the order: larger logits first, then lower indexes.  order -1: NaN
__device__ __forceinline__ long long rank_key(int order, int id) { return (long long)order << 32 | (uint32_t)(0x7FFFFFFF - id); }

__device__ __forceinline__ float element(const u32x4l_t &w, int e) { const uint32_t v = w[e >> 1]; return h2f((uint16_t)(e & 1 ? v >> 16 : v & 0xFFFFu)); }
// x - base of the low and of the high half of a word, one instruction each
__device__ __forceinline__ float low_minus(uint32_t w, float base)
{
    float r;
    asm("v_fma_mix_f32 %0, %1, 1.0, -%2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(w), "v"(base));
    return r;
}
__device__ __forceinline__ float high_minus(uint32_t w, float base)
{
    float r;
    asm("v_fma_mix_f32 %0, %1, 1.0, -%2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(w), "v"(base));
    return r;
}
__device__ __forceinline__ half2l_t pairs_max(half2l_t a, uint32_t b) { return __builtin_elementwise_max(a, __builtin_bit_cast(half2l_t, b)); }   // the other where one is NaN
__device__ __forceinline__ half2l_t packet_max(const u32x4l_t &w)
{
    const uint32_t a = w.x, b = w.y, c = w.z, d = w.w;
    return __builtin_elementwise_max(pairs_max(__builtin_bit_cast(half2l_t, a), b), pairs_max(__builtin_bit_cast(half2l_t, c), d));
}

// What a slice of a row leaves: its maximum, how many logits have it, the sum of e^(x - m) over the others and the sum of e^(x - m) (x - m) / log 2;
// its `listed` best logits follow
struct Slice {
    float m, rest, t;
    int tops, listed, pad;
};
constexpr int kMaxTop = 32, kMaxSlices = 16, kSliceLogits = 512 * 8 * 4 - 8;
struct SliceList {
    Slice sums;
    long long best[kMaxTop];
};

struct Outputs {
    const int32_t *targets;
    float *logprobs, *entropy;
    int32_t *top_ids;
    float *top_logprobs;
    SliceList *slices;               // PART: [n][slices]
};

// What the logits of a row are taken relative to: its maximum, 0 where that is infinite.  The sum of a row with a +inf then is +inf, of one with a NaN it is NaN.
__device__ __forceinline__ float base_of(float m) { return fabsf(m) == INFINITY ? 0.0f : m; }

// The end of a row: `rest` is the sum without one maximum, both sums relative to base_of(m); target: its logit, -inf outside the vocabulary
struct RowEnd {
    float base, rest, log_s;
    bool empty;
    __device__ __forceinline__ RowEnd(float m, float rest_, int tops)
    {
        base = base_of(m);
        empty = m == -INFINITY && rest_ == 0.0f;               // no logit above -inf, and no NaN
        rest = rest_ + (float)(tops - 1);
        log_s = log1pf(fmaf(0.0f, rest, rest));                // (NaN where a +inf is in the row: only a token at -inf has a log probability then)
    }
    __device__ __forceinline__ float logp(float x) const { return empty || x == -INFINITY ? (rest == rest ? -INFINITY : rest) : x - base - log_s; }
    __device__ __forceinline__ float entropy(float t) const { return empty ? 0.0f : log_s - t * kLn2 / (1.0f + rest); }
    __device__ __forceinline__ void put(const Outputs &o, int row, int k, int rank, long long key) const
    {
        const int order = (int)(key >> 32);
        o.top_ids[(size_t)row * k + rank] = 0x7FFFFFFF - (int)(uint32_t)key;
        o.top_logprobs[(size_t)row * k + rank] = order < 0 ? NAN : logp(value_of(order));
    }
};

// NT threads, NP packets of eight logits each; RESIDENT: they hold the whole row; PART: the row is slice blockIdx.y of one, of `length` logits
template <int NT, int NP, bool RESIDENT, bool PART>
__global__ __launch_bounds__(NT) void token_logprobs_kernel(const uint16_t *__restrict__ logits, int64_t stride, Outputs o, int vocab, int k, int length)
{
    constexpr int W = NT / 64;
    const int from = PART ? (int)blockIdx.y * length : 0, V = PART ? min(length, vocab - from) : vocab;
    __shared__ float lane_max[W][64], wave_m[W], wave_rest[W], wave_t[W];
    __shared__ int wave_n[W], listed, scan[W];
    __shared__ long long list[kListed];
    __shared__ float bound_s;

    const uint16_t *row = logits + (int64_t)blockIdx.x * stride + from;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float target = -INFINITY;                                  // asked for before the row is
    if (!PART && o.targets) {
        const int id = o.targets[blockIdx.x];
        if (id >= 0 && id < V) target = h2f(row[id]);
    }
    // packets are aligned to 16 bytes: the first one begins `skip` elements in front of the row
    const int skip = (int)((reinterpret_cast<uintptr_t>(row) & 15) >> 1);
    const int packets = (V + skip + 7) >> 3;

    auto fetch = [&](int p) -> u32x4l_t {                      // packet p of the row, -inf outside it
        const int at = p * 8 - skip;
        if (at >= 0 && at + 8 <= V) return *(const u32x4l_t *)(row + at);
        u32x4l_t w = {kNone2, kNone2, kNone2, kNone2};
        if (at < V) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e >= 0 && at + e < V) {
                    const uint32_t v = row[at + e];
                    w[e >> 1] = e & 1 ? (w[e >> 1] & 0xFFFFu) | v << 16 : (w[e >> 1] & 0xFFFF0000u) | v;
                }
        }
        return w;
    };
    u32x4l_t held[RESIDENT ? NP : 1];
    // f(packet, its first element's index) for the thread's packets
    auto each = [&](const auto &f) __attribute__((always_inline)) {
        if constexpr (RESIDENT) {
#pragma unroll
            for (int i = 0; i < NP; ++i) f(held[i], (i * NT + tid) * 8 - skip);
        } else {
            for (int p = tid; p < packets; p += NT) f(fetch(p), p * 8 - skip);
        }
    };
    auto block_sum = [&](int v) {                              // over the workgroup, the same in all threads
#pragma unroll
        for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off, kWave);
        __syncthreads();
        if (lane == 0) scan[wave] = v;
        __syncthreads();
        int s = 0;
        for (int w = 0; w < W; ++w) s += scan[w];
        return s;
    };

    // ---- the maximum, and those of the threads ----
    if constexpr (RESIDENT) {
#pragma unroll
        for (int i = 0; i < NP; ++i) held[i] = fetch(i * NT + tid);
    }
    half2l_t mx2 = __builtin_bit_cast(half2l_t, kNone2);
    each([&](const u32x4l_t &w, int) __attribute__((always_inline)) { mx2 = __builtin_elementwise_max(mx2, packet_max(w)); });
    const float mine = fmaxf((float)mx2.x, (float)mx2.y);
    lane_max[wave][lane] = mine;
    const float wm = wave_max(mine);
    if (lane == 0) wave_m[wave] = wm;
    if (tid == 0) listed = 0;
    __syncthreads();
    float m = wave_m[0];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, wave_m[w]);

    // ---- the first wavefront: the k-th largest of the 64 group maxima ----
    if (wave == 0 && k > 0) {
        float gm = lane_max[0][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) gm = fmaxf(gm, lane_max[w][lane]);
        int rank = 0;
#pragma unroll
        for (int j = 0; j < 64; ++j) {
            const float o = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, gm), j));
            rank += o > gm || (o == gm && j < lane);
        }
        if (rank == min(k, V) - 1) bound_s = gm;
    }

    // ---- sums: exponents in units of log 2; the maxima themselves, in the wavefronts that hold one, are counted instead ----
    const float base = base_of(m);
    float rest = 0.0f, t = 0.0f;
    int tops = 0;
    auto add = [&](const u32x4l_t &w, bool count) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t v = w[e >> 1];
            const float y = (e & 1 ? high_minus(v, base) : low_minus(v, base)) * kLog2e;
            float x = __builtin_amdgcn_exp2f(y);
            t = fmaf(x, fmaxf(y, -300.0f), t);                 // (0 * -inf: exp2 is 0 there)
            if (count) tops += y == 0.0f, x = y == 0.0f ? 0.0f : x;
            rest += x;
        }
    };
    if (wm == m) each([&](const u32x4l_t &w, int) __attribute__((always_inline)) { add(w, true); });
    else each([&](const u32x4l_t &w, int) __attribute__((always_inline)) { add(w, false); });
    rest = wave_sum(rest), t = wave_sum(t);
#pragma unroll
    for (int off = 32; off; off >>= 1) tops += __shfl_xor(tops, off, kWave);
    if (lane == 0) wave_rest[wave] = rest, wave_t[wave] = t, wave_n[wave] = tops;
    __syncthreads();
    rest = 0.0f, t = 0.0f, tops = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) rest += wave_rest[w], t += wave_t[w], tops += wave_n[w];
    const RowEnd end(m, rest, tops);
    if (!PART && tid == 0) {
        if (o.targets) o.logprobs[blockIdx.x] = end.logp(target);
        if (o.entropy) o.entropy[blockIdx.x] = end.entropy(t);
    }
    SliceList *mine_out = PART ? o.slices + (size_t)blockIdx.x * gridDim.y + blockIdx.y : nullptr;
    if (PART && tid == 0) mine_out->sums = Slice{m, rest, t, tops, min(k, V), 0};
    if (k == 0) return;

    // ---- candidates ----
    float bound = bound_s;
    auto collect = [&](auto EQUAL) __attribute__((always_inline)) {
        each([&](const u32x4l_t &w, int at) __attribute__((always_inline)) {
            const half2l_t p = packet_max(w);
            const float most = fmaxf((float)p.x, (float)p.y);
            if (!__any(EQUAL ? most >= bound : most > bound)) return;
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = element(w, e);
                hits |= (EQUAL ? x >= bound : x > bound) ? 1u << e : 0u;
            }
            while (hits) {                                     // rarely more than one in a wavefront
                const int e = __ffs(hits) - 1;
                hits &= hits - 1;
                const uint32_t v = e < 4 ? (e < 2 ? w.x : w.y) : (e < 6 ? w.z : w.w);
                if (at + e < 0 || at + e >= V) continue;       // (outside the row is -inf, which the bound may be)
                const int place = atomicAdd(&listed, 1);
                if (place < kListed) list[place] = rank_key(order_of(h2f((uint16_t)(e & 1 ? v >> 16 : v & 0xFFFFu))), at + e);
            }
        });
        __syncthreads();
        return listed;
    };
    int found = collect(std::true_type{});
    const bool many = found > kListed;
    if (many) {
        // the k-th largest value: the smallest order with fewer than k logits above it
        int lo = order_of(bound), hi = order_of(m);
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            const float v = value_of(mid);
            int above = 0;
            each([&](const u32x4l_t &w, int) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) above += element(w, e) > v;
            });
            if (block_sum(above) < k) hi = mid;
            else lo = mid + 1;
        }
        bound = value_of(lo);
        __syncthreads();
        if (tid == 0) listed = 0;
        __syncthreads();
        found = collect(std::false_type{});
    }
    // ---- too few: the first of those equal to the bound, and behind -inf the NaNs ----
    for (int kind = many ? 0 : 1; kind < 2 && found < k; ++kind)
        for (int p0 = 0; p0 < packets && found < k; p0 += NT) {
            const u32x4l_t w = fetch(p0 + tid);
            const int at = (p0 + tid) * 8 - skip;
            uint32_t is = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = element(w, e);
                if (at + e >= 0 && at + e < V && (kind == 0 ? x == bound : x != x)) is |= 1u << e;
            }
            int sum = __popc(is);                              // inclusive sum over the workgroup's threads
#pragma unroll
            for (int off = 1; off < kWave; off <<= 1) {
                const int o = __shfl_up(sum, off, kWave);
                if (lane >= off) sum += o;
            }
            __syncthreads();
            if (lane == 63) scan[wave] = sum;
            __syncthreads();
            int place = found + sum - __popc(is), all = 0;
            for (int v = 0; v < W; ++v) {
                if (v < wave) place += scan[v];
                all += scan[v];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (is >> e & 1u) {
                    if (place < k) list[place] = rank_key(kind == 0 ? order_of(bound) : -1, at + e);
                    ++place;
                }
            found = min(found + all, k);
        }
    __syncthreads();

    // ---- ranks ----
    for (int i = tid; i < found; i += NT) {
        const long long own = list[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < found; ++j) rank += list[j] > own;
        if (rank >= k) continue;
        if (PART) mine_out->best[rank] = own - from;           // (its id counts down)
        else end.put(o, blockIdx.x, k, rank, own);
    }
}

// One workgroup per row: the slices' sums relative to the largest maximum, and the best of their best
__global__ __launch_bounds__(256) void token_logprobs_join_kernel(const uint16_t *__restrict__ logits, int64_t stride, Outputs o, int V, int k, int slices)
{
    __shared__ Slice sl[kMaxSlices];
    __shared__ long long list[kMaxSlices * kMaxTop];
    const int row = blockIdx.x, tid = threadIdx.x;
    const SliceList *src = o.slices + (size_t)row * slices;
    float target = -INFINITY;
    if (o.targets) {
        const int id = o.targets[row];
        if (id >= 0 && id < V) target = h2f(logits[(int64_t)row * stride + id]);
    }
    if (tid < slices) sl[tid] = src[tid].sums;
    for (int i = tid; i < slices * k; i += 256) {
        const int s = i / k, j = i - s * k;
        list[i] = j < src[s].sums.listed ? src[s].best[j] : LLONG_MIN;
    }
    __syncthreads();
    float m = -INFINITY, rest = 0.0f, t = 0.0f;
    int tops = 0;
    for (int s = 0; s < slices; ++s) m = fmaxf(m, sl[s].m);
    for (int s = 0; s < slices; ++s) {
        const Slice q = sl[s];
        if (q.m == m) {                                        // (-inf: a sum of 0, or NaN)
            rest += q.rest, t += q.t, tops += q.tops;
        } else if (q.m > -INFINITY) {
            const float d = (q.m - m) * kLog2e, f = __builtin_amdgcn_exp2f(d), all = q.rest + (float)q.tops;
            rest += all * f, t += f * fmaf(fmaxf(d, -300.0f), all, q.t);
        } else {
            rest += q.rest;                                    // 0, or NaN
        }
    }
    const RowEnd end(m, rest, tops);
    if (tid == 0) {
        if (o.targets) o.logprobs[row] = end.logp(target);
        if (o.entropy) o.entropy[row] = end.entropy(t);
    }
    for (int i = tid; i < slices * k; i += 256) {
        const long long own = list[i];
        if (own == LLONG_MIN) continue;
        int rank = 0;
#pragma unroll 4
        for (int s = 0; s < slices; ++s) {                     // each slice's list is in order: where `own` would stand in it
            int pos = 0;
#pragma unroll
            for (int step = kMaxTop; step; step >>= 1) {
                const bool larger = list[s * k + min(pos + step, k) - 1] > own;
                pos += pos + step <= k && larger ? step : 0;
            }
            rank += pos;
        }
        if (rank < k) end.put(o, row, k, rank, own);
    }
}

// A launch has fewer than 2^32 threads: rows beyond kLaunchThreads / NT follow in further ones
constexpr int64_t kLaunchThreads = 1LL << 31;
template <int NT, int NP, bool RESIDENT>
hipError_t launch_one(const uint16_t *logits, int64_t stride, const Outputs &o, int32_t n, int32_t V, int32_t k, hipStream_t stream)
{
    for (int64_t row = 0; row < n; row += kLaunchThreads / NT) {
        Outputs at = o;
        if (at.targets) at.targets += row, at.logprobs += row;
        if (at.entropy) at.entropy += row;
        if (k > 0) at.top_ids += row * k, at.top_logprobs += row * k;
        const dim3 rows((uint32_t)std::min(n - row, kLaunchThreads / NT));
        hipLaunchKernelGGL((token_logprobs_kernel<NT, NP, RESIDENT, false>), rows, dim3(NT), 0, stream, logits + row * stride, stride, at, V, k, V);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Slices of a row, as few as hold it: from 65530 logits on, where one workgroup takes longer than two kernels, and up to one slice per CU (more have not been
// measured; several fit on one)
constexpr int kUncut = 65529;
int slices_of(int32_t n, int32_t V)
{
    const int need = (V + kSliceLogits - 1) / kSliceLogits;
    return V > kUncut && need <= kMaxSlices && (int64_t)need * n <= 256 ? need : 1;
}

}  // namespace

size_t token_logprobs_partial_bytes(int32_t n, int32_t V)
{
    // (for n rows at most: fewer may be cut where n are not)
    const int64_t need = (V + kSliceLogits - 1) / kSliceLogits;
    return slices_of(1, V) > 1 ? sizeof(SliceList) * (size_t)std::min<int64_t>(need * n, 256) : 0;
}

hipError_t launch_token_logprobs(const uint16_t *logits, int64_t stride, const int32_t *targets, float *logprobs, float *entropy, int32_t *top_ids,
                                 float *top_logprobs, int32_t n, int32_t V, int32_t k, void *partials, hipStream_t stream)
{
    const Outputs o = {targets, logprobs, entropy, top_ids, top_logprobs, static_cast<SliceList *>(partials)};
    const int slices = partials ? slices_of(n, V) : 1;
    if (slices > 1) {
        const int length = (V + slices - 1) / slices;          // (the last slice is shorter, and never empty: (slices - 1) * length < V)
        hipLaunchKernelGGL((token_logprobs_kernel<512, 4, true, true>), dim3(n, slices), dim3(512), 0, stream, logits, stride, o, V, k, length);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(token_logprobs_join_kernel, dim3(n), dim3(256), 0, stream, logits, stride, o, V, k, slices);
        return hipGetLastError();
    }
    // The smallest workgroup that holds the row: several are on a CU, and one reads while another sums (us, 2047 rows of 1000 logits with 256 threads 14.7, with 512 31;
    // 1000 rows of 50257 with 512 threads and 16 packets 41, with 1024 and 20 88).  The last two kernels that hold their row keep 2 and 26 words of it in scratch
    // memory, which still is faster than reading it three times (500 rows of 128256 50 us against 69, 400 of 152064 60 against 76).  Rows that leave CUs idle take twice the threads.
    if (V + 7 <= 256 * 8 * 4) return launch_one<256, 4, true>(logits, stride, o, n, V, k, stream);
    if (V + 7 <= 1024 * 8 * 4 && n <= 512) return launch_one<1024, 4, true>(logits, stride, o, n, V, k, stream);
    if (V + 7 <= 512 * 8 * 8) return launch_one<512, 8, true>(logits, stride, o, n, V, k, stream);
    if (V + 7 <= 512 * 8 * 16) return launch_one<512, 16, true>(logits, stride, o, n, V, k, stream);
    if (V + 7 <= 1024 * 8 * 16) return launch_one<1024, 16, true>(logits, stride, o, n, V, k, stream);
    if (V + 7 <= 1024 * 8 * 20) return launch_one<1024, 20, true>(logits, stride, o, n, V, k, stream);
    return launch_one<1024, 1, false>(logits, stride, o, n, V, k, stream);
}

}  // namespace relax
