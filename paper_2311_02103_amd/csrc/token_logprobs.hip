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
// logit from below; whatever is larger than T -- a few more than k on any row whose large logits do not share few groups -- goes to a list in
// LDS and is ranked by counting.  Fewer than k larger ones: the lowest indexes among those equal to T follow, found by a scan in order.
// More than the list holds: T is replaced by the k-th largest logit itself, by bisection over the 16-bit values.
//
// Bound by the vector unit next to the read: a logit takes nine issue slots in the sums (four of them the exponential) and one and a half in the other
// two passes, which look at pairs.
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

// NT threads, NP packets of eight logits each; RESIDENT: they hold the whole row
template <int NT, int NP, bool RESIDENT>
__global__ __launch_bounds__(NT) void token_logprobs_kernel(const uint16_t *__restrict__ logits, int64_t stride, const int32_t *__restrict__ targets,
                                                            float *__restrict__ logprobs, float *__restrict__ entropy, int32_t *__restrict__ top_ids,
                                                            float *__restrict__ top_logprobs, int V, int k)
{
    constexpr int W = NT / 64;
    __shared__ float lane_max[W][64], wave_m[W], wave_rest[W], wave_t[W];
    __shared__ int wave_n[W], listed, scan[W];
    __shared__ long long list[kListed];
    __shared__ float bound_s;

    const uint16_t *row = logits + (int64_t)blockIdx.x * stride;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
        if (rank == k - 1) bound_s = gm;
    }

    // ---- sums: exponents in units of log 2; the maxima themselves, in the wavefronts that hold one, are counted instead ----
    const float base = m == -INFINITY ? 0.0f : m;
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
    const bool empty = m == -INFINITY && rest == 0.0f;         // no logit above -inf, and no NaN
    rest += (float)(tops - 1);
    const float log_s = log1pf(rest);
    auto logp = [&](float x) { return empty || x == -INFINITY ? (rest == rest ? -INFINITY : rest) : x - base - log_s; };
    if (tid == 0) {
        if (targets) {
            const int id = targets[blockIdx.x];
            logprobs[blockIdx.x] = logp(id >= 0 && id < V ? h2f(row[id]) : -INFINITY);
        }
        if (entropy) entropy[blockIdx.x] = empty ? 0.0f : log_s - t * kLn2 / (1.0f + rest);
    }
    if (k == 0) return;

    // ---- candidates: what is larger than the bound ----
    float bound = bound_s;
    auto collect = [&]() __attribute__((always_inline)) {
        each([&](const u32x4l_t &w, int at) __attribute__((always_inline)) {
            const half2l_t p = packet_max(w);
            if (!__any(fmaxf((float)p.x, (float)p.y) > bound)) return;
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
                const uint32_t v = e < 4 ? (e < 2 ? w.x : w.y) : (e < 6 ? w.z : w.w);
                const float x = h2f((uint16_t)(e & 1 ? v >> 16 : v & 0xFFFFu));
                if (x > bound) {
                    const int place = atomicAdd(&listed, 1);
                    if (place < kListed) list[place] = rank_key(order_of(x), at + e);
                }
            }
        });
        __syncthreads();
        return listed;
    };
    int found = collect();
    if (found > kListed) {
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
        found = collect();
    }
    // ---- too few: the first of those equal to the bound, and behind -inf the NaNs ----
    for (int kind = 0; kind < 2 && found < k; ++kind)
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
        if (rank < k) {
            const int order = (int)(own >> 32);
            top_ids[(size_t)blockIdx.x * k + rank] = 0x7FFFFFFF - (int)(uint32_t)own;
            top_logprobs[(size_t)blockIdx.x * k + rank] = order < 0 ? NAN : logp(value_of(order));
        }
    }
}

template <int NT, int NP, bool RESIDENT>
hipError_t launch_one(const uint16_t *logits, int64_t stride, const int32_t *targets, float *logprobs, float *entropy, int32_t *top_ids, float *top_logprobs,
                      int32_t n, int32_t V, int32_t k, hipStream_t stream)
{
    hipLaunchKernelGGL((token_logprobs_kernel<NT, NP, RESIDENT>), dim3(n), dim3(NT), 0, stream, logits, stride, targets, logprobs, entropy, top_ids, top_logprobs, V, k);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logprobs(const uint16_t *logits, int64_t stride, const int32_t *targets, float *logprobs, float *entropy, int32_t *top_ids,
                                 float *top_logprobs, int32_t n, int32_t V, int32_t k, hipStream_t stream)
{
    if (V + 7 <= 1024 * 8 * 4 && n <= 512) return launch_one<1024, 4, true>(logits, stride, targets, logprobs, entropy, top_ids, top_logprobs, n, V, k, stream);
    if (V + 7 <= 512 * 8 * 8) return launch_one<512, 8, true>(logits, stride, targets, logprobs, entropy, top_ids, top_logprobs, n, V, k, stream);
    if (V + 7 <= 1024 * 8 * 20) return launch_one<1024, 20, true>(logits, stride, targets, logprobs, entropy, top_ids, top_logprobs, n, V, k, stream);
    return launch_one<1024, 1, false>(logits, stride, targets, logprobs, entropy, top_ids, top_logprobs, n, V, k, stream);
}

}  // namespace relax
