// Device functions that prepare the heads of queries and keys -- norm and rotation, relax_head_prep in relax_mi355.h -- shared by the kernel that writes them
// (heads.hip) and the one that quantises them (paged4_append.hip).
//
// A lane holds a unit of eight consecutive elements, a head is d / 8 neighbouring lanes, so every access is 16 bytes per lane and d * 2 consecutive bytes per head.
// The sum of squares goes through DPP moves in fp64: the squares of fp16 numbers are exact in fp32, and their sum in fp64 is exact where a head's elements but zeros lie within 2^12 of each
// other, else off by 2^-49 of itself at most, so that the fp32 factor, and a quantised key, depends on the order of the sum for less than one in 2^24 of those.  The
// pair of an element of the halves layout lies rotary_dim / 16 lanes away.
#pragma once

#include "paged_device.h"

namespace relax {

// Frequencies of a rotary table: f_t = base^(-2 t / R) times w + (1 - w) / factor, w a ramp from 1 (at x = one) to 0 (at x = none) over x = t or x = turns_t
struct RopeFrequency {
    double log_base_2_r;             // -2 ln base / R
    double inv_factor, turns;        // turns: trained / 2 pi (wavelength ramp), 0: x = t
    double none, inv_width;          // w = clamp((x - none) * inv_width, 0, 1)
    double amplitude;
};
inline RopeFrequency rope_frequencies(const relax_rope_scaling &sc)
{
    constexpr double kTau = 6.283185307179586476925;
    RopeFrequency f = {-2.0 * log(sc.base) / sc.rotary_dim, sc.scaling == RELAX_ROPE_PLAIN ? 1.0 : 1.0 / sc.factor, 0.0, 0.0, 0.0, sc.amplitude == 0.0 ? 1.0 : sc.amplitude};
    if (sc.scaling == RELAX_ROPE_WAVELENGTH_RAMP) f.turns = sc.trained / kTau, f.none = sc.slow, f.inv_width = 1.0 / (sc.fast - sc.slow);
    if (sc.scaling == RELAX_ROPE_INDEX_RAMP) {
        const auto index = [&](double b) { return sc.rotary_dim * log(sc.trained / (kTau * b)) / (2.0 * log(sc.base)); };
        const double first = fmax(floor(index(sc.fast)), 0.0), last = fmin(ceil(index(sc.slow)), sc.rotary_dim - 1.0), width = fmax(last - first, 0.001);
        f.none = first + width, f.inv_width = -1.0 / width;
    }
    return f;
}
__device__ __forceinline__ double rope_frequency(const RopeFrequency &f, int t)
{
    const double plain = exp((double)t * f.log_base_2_r), x = f.turns > 0.0 ? f.turns * plain : (double)t;
    const double w = fmin(fmax((x - f.none) * f.inv_width, 0.0), 1.0);
    return plain * (w + (1.0 - w) * f.inv_factor);
}

struct HeadPrep {
    const uint16_t *q_norm, *k_norm; // nullptr: none
    const float *rope;               // nullptr: none
    float eps;
    int32_t rot, pairs;              // rotated elements; 1: neighbours, 0: halves
};

typedef half8p_t Unit;               // eight elements of a head
template <int D>
constexpr int kUnits = D / 8;        // lanes of a head

// What of a unit is quantised: the ends of fp16's range for infinities, 0 for a NaN.  A look at all eight (x * 0 is a NaN for either) costs less than treating each
__device__ __forceinline__ void to_storable(const Unit &in, float (&x)[8])
{
    const half2p_t zero = {(_Float16)0.0f, (_Float16)0.0f};
    half2p_t t = zero;
#pragma unroll
    for (int i = 0; i < 8; i += 2) t = __builtin_elementwise_fma(half2p_t{in[i], in[i + 1]}, zero, t);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)in[i];
    const float bad = (float)t.x + (float)t.y;
    if (__any(bad != bad)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -65504.0f), 65504.0f) : 0.0f;
    }
}

template <int OFF>
__device__ __forceinline__ double lane_xor(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const float lo = lane_xor<OFF>(__builtin_bit_cast(float, (uint32_t)u)), hi = lane_xor<OFF>(__builtin_bit_cast(float, (uint32_t)(u >> 32)));
    return __builtin_bit_cast(double, (uint64_t)__builtin_bit_cast(uint32_t, hi) << 32 | __builtin_bit_cast(uint32_t, lo));
}

// 1 / sqrt(ms) in fp32, the correctly rounded one but for one value in about 2^26: the hardware's estimate in fp64 (2^-24; the one in fp32 has no estimate of a subnormal number, which eps may be) and two steps of Newton's method (2^-46,
// then fp64's own 2^-52), a sixth of the instructions of a square root and a division.  0 for infinity and for 0
__device__ __forceinline__ float rsqrt_once(double ms)
{
    const double r0 = __builtin_amdgcn_rsq(ms), half = 0.5 * ms;
    const double r1 = r0 * __builtin_fma(-half * r0, r0, 1.5), r2 = r1 * __builtin_fma(-half * r1, r1, 1.5);
    return ms > 0.0 && ms < __builtin_inf() ? (float)r2 : ms == ms ? 0.0f : __builtin_nanf("");
}

// x *= w / sqrt(mean square + eps) over the lanes of a head
template <int D>
__device__ __forceinline__ void normalise(float (&x)[8], const Unit &w, float eps)
{
#pragma clang fp contract(off)
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)x[j], (double)x[j], sum);
    sum += lane_xor<1>(sum);
    sum += lane_xor<2>(sum);
    sum += lane_xor<4>(sum);
    if (D == 128) sum += lane_xor<8>(sum);
    const float r = rsqrt_once(sum * (1.0 / D) + (double)eps);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float y = x[j] * r;
        x[j] = y * (float)w[j];
    }
}

// The angles of a lane's unit at one position: (cos, sin) of its four pairs (neighbours), of the eight pairs that its elements belong to (halves; the sines of the first half's negated, so that
// either element is x cos + other sin)
struct Angles {
    float4p_t cs[4];
};
__device__ __forceinline__ void load_angles(Angles &a, const HeadPrep &p, int pos, int unit)
{
    const int low = p.rot >> 4;                                // units of half the rotated part
    const int at = p.pairs ? unit * 8 : (unit >= low ? unit - low : unit) * 16;
    const float4p_t *src = (const float4p_t *)(p.rope + (size_t)pos * p.rot + (unit * 8 < p.rot ? at : 0));
#pragma unroll
    for (int i = 0; i < 2; ++i) a.cs[i] = src[i];
    if (!p.pairs) {
#pragma unroll
        for (int i = 2; i < 4; ++i) a.cs[i] = src[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) a.cs[i].y = unit < low ? -a.cs[i].y : a.cs[i].y, a.cs[i].w = unit < low ? -a.cs[i].w : a.cs[i].w;
    }
}

// the rotation of a unit; lane: of the wavefront; every lane of the head is active
template <int D>
__device__ __forceinline__ void rotate(float (&x)[8], const Angles &a, const HeadPrep &p, int unit, int lane)
{
#pragma clang fp contract(off)
    float z[8];
    if (p.pairs) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float c = a.cs[j >> 1][(j & 1) * 2], s = a.cs[j >> 1][(j & 1) * 2 + 1];
            const float ac = x[2 * j] * c, bs = x[2 * j + 1] * s, as = x[2 * j] * s, bc = x[2 * j + 1] * c;
            z[2 * j] = ac - bs, z[2 * j + 1] = as + bc;
        }
    } else {
        float y[8];
        if (p.rot == D) {                                      // uniform
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = lane_xor<D / 16>(x[j]);
        } else {
            const int low = p.rot >> 4, from = unit * 8 < p.rot ? (unit < low ? lane + low : lane - low) : lane;
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = __shfl(x[j], from, kWave);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float own = x[j] * a.cs[j >> 1][(j & 1) * 2], other = y[j] * a.cs[j >> 1][(j & 1) * 2 + 1];
            z[j] = own + other;
        }
    }
    if (p.rot == D) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = z[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = unit * 8 < p.rot ? z[j] : x[j];
    }
}

// Rows of heads that are prepared and written as fp16
struct HeadRows {
    const uint16_t *q, *k;
    uint16_t *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
};

// Wavefront `wave` of the call: one row, every `slices`-th step of 64 / kUnits<D> heads of its [h of q; g of k].  h or g may be 0.
template <int D>
__device__ __forceinline__ void head_rows(SeqsArg st, const HeadRows &r, const HeadPrep &p, int h, int g, int cap, int64_t wave, int slices, uint32_t *err)
{
    constexpr int U = kUnits<D>, HS = kWave / U;
    const int i = (int)(wave / slices), slice = (int)(wave - (int64_t)i * slices);
    const int lane = threadIdx.x & 63, unit = lane & (U - 1), heads = h + g;
    if (i >= st->n) return;
    const auto src = [&](int hd) { return (const Unit *)((hd < h ? r.q + i * r.q_stride + (int64_t)hd * D : r.k + i * r.k_stride + (int64_t)(hd - h) * D) + unit * 8); };
    int hd = slice * HS + lane / U;
    Unit in = *src(min(hd, heads - 1));                        // on its way before the position is known
    Unit wq = {}, wk = {};
    if (p.q_norm) wq = *(const Unit *)(p.q_norm + unit * 8);
    if (p.k_norm) wk = *(const Unit *)(p.k_norm + unit * 8);
    int place, b = i;
    if (st->q_max == 1) place = 0;
    else b = seq_of(st, i, [](int q_len) { return q_len; }, place);
    if (b >= st->B) return;
    const SeqSpan si = seq_span(st, __builtin_amdgcn_readfirstlane(b));
    Angles a = {};
    if (p.rope) {
        const bool beyond = beyond_capacity(si, cap);
        const int at = si.kv_len < 0 ? 0 : beyond ? cap - 1 : si.kv_len - si.q_len + place, pos = min(max(at, 0), cap - 1);
        if ((beyond || at != pos) && slice == 0 && lane == 0) atomicOr(err, kBadPage);
        load_angles(a, p, pos, unit);
    }
    for (;;) {
        const int next = hd + slices * HS;
        const bool more = __builtin_amdgcn_readfirstlane(hd) + slices * HS < heads;      // (the first lane's head is the lowest)
        Unit ahead = in;
        if (more) ahead = *src(min(next, heads - 1));
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)in[j];
        const bool isq = hd < h;
        if (p.q_norm && p.k_norm) normalise<D>(x, isq ? wq : wk, p.eps);
        else if (p.q_norm || p.k_norm) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = x[j];
            normalise<D>(y, isq ? wq : wk, p.eps);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (isq ? p.q_norm : p.k_norm) ? y[j] : x[j];
        }
        if (p.rope) rotate<D>(x, a, p, unit, lane);
        if (hd < heads) {
            Unit out;
#pragma unroll
            for (int j = 0; j < 8; ++j) out[j] = (_Float16)x[j];
            *(Unit *)((isq ? r.q_out + i * r.q_out_stride + (int64_t)hd * D : r.k_out + i * r.k_out_stride + (int64_t)(hd - h) * D) + unit * 8) = out;
        }
        if (!more) return;
        in = ahead, hd = next;
    }
}

// wavefronts per row of head_rows: one per step of heads for few rows, few for many, whose angles and positions then serve more heads (us for 2043 rows of 32 / 8 heads with 2048, 4096 and
// 8192 wavefronts wanted: 11.2, 11.5, 13.0)
inline int head_slices(int heads, int n, int d)
{
    const int steps = (heads * d / 8 + kWave - 1) / kWave;     // of one row
    int slices = 1;
    while (slices < steps && (int64_t)n * slices < 2048) slices *= 2;
    return slices < steps ? slices : steps;
}

}  // namespace relax
