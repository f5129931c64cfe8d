// Rotary tables of scaled positions: table[p][t] = amplitude (cos, sin)(p f'_t), fp64 rounded to fp32 (frequencies: relax_rope_scaling in relax_mi355.h).
// A sine and cosine per entry made it bound by fp64 instructions: 131071 positions of 128 elements 32.7 us.  All entries of a thread from one, by rotation: 11.2 to 11.8 us, 5.7 to 6.0 TB/s
// written (9.8 at the rate of a fill).
#include <algorithm>
#include <cmath>

#include "heads_device.h"

namespace relax {

namespace {

constexpr int kThreads = 1 << 18;                // of a launch at most: four workgroups per CU, all at once (with up to 16 entries per thread, eight per CU and more: 14.3 us for 11.8)

// Thread i has pair i % half at positions i / half, + rows, + 2 rows ..: two sines and cosines, and a rotation by the angle of `rows` positions for each further entry (four multiply-adds in
// 64 bits, off by 2^-52 each: 32 of them with 131072 positions of 128 elements; a sine and cosine is some fifty instructions).
__global__ __launch_bounds__(256) void rope_scaled_kernel(float *table, RopeFrequency f, int rows, int positions, int half)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)rows * half) return;
    const int p0 = (int)(i / half), t = (int)(i - (int64_t)p0 * half);
    const double w = rope_frequency(f, t);
    double s, c, ds, dc;
    sincos((double)p0 * w, &s, &c);
    sincos((double)rows * w, &ds, &dc);
    s *= f.amplitude, c *= f.amplitude;
    float2 *dst = (float2 *)table + i;
    for (int64_t p = p0; p < positions; p += rows, dst += (int64_t)rows * half) {
        *dst = make_float2((float)c, (float)s);
        const double turned = c * dc - s * ds;
        s = c * ds + s * dc, c = turned;
    }
}

}  // namespace

hipError_t launch_rope_scaled(const relax_rope_scaling &sc, int32_t positions, float *table, hipStream_t stream)
{
    const int half = sc.rotary_dim / 2;
    const int rows = std::min(positions, kThreads / half);
    const int64_t groups = ((int64_t)rows * half + 255) / 256;
    hipLaunchKernelGGL(rope_scaled_kernel, dim3(groups), dim3(256), 0, stream, table, rope_frequencies(sc), rows, positions, half);
    return hipGetLastError();
}

}  // namespace relax
