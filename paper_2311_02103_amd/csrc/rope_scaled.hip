// Rotary tables of scaled positions: table[p][t] = amplitude (cos, sin)(p f'_t), fp64 rounded to fp32 (frequencies: relax_rope_scaling in relax_mi355.h).
#include <cmath>

#include "heads_device.h"

namespace relax {

namespace {

// one thread per entry
__global__ __launch_bounds__(256) void rope_scaled_kernel(float *table, RopeFrequency f, int64_t total, int half)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const int64_t p = i / half;
    double s, c;
    sincos((double)p * rope_frequency(f, (int)(i - p * half)), &s, &c);
    ((float2 *)table)[i] = make_float2((float)(f.amplitude * c), (float)(f.amplitude * s));
}

}  // namespace

hipError_t launch_rope_scaled(const relax_rope_scaling &sc, int32_t positions, float *table, hipStream_t stream)
{
    const int half = sc.rotary_dim / 2;
    const int64_t total = (int64_t)positions * half;
    const RopeFrequency f = rope_frequencies(sc);
    hipLaunchKernelGGL(rope_scaled_kernel, dim3((total + 255) / 256), dim3(256), 0, stream, table, f, total, half);
    return hipGetLastError();
}

}  // namespace relax
