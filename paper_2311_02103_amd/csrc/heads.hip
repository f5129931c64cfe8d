// Norm and rotation of the heads of queries and keys in one pass over them (relax_head_norm_rope): heads_device.h has the mathematics.  A wavefront takes heads of one row,
// so that the row's angles are loaded once for all of them; the next step's heads are on their way while these are prepared (two steps ahead: 11.6 us for 11.3).
// Bound by bytes for a prompt: 2043 rows of 32 / 8 heads of 128, normalised, half of each turned, 11.1 us, 3.8 TB/s (42 MB in and out: 7.1 at a long stream's
// rate), and by latency for a decode step: one row of 64 / 8 heads 3.0 us in a graph, of which a launch is 1.9.
#include "heads_device.h"

namespace relax {

namespace {

template <int D>
__global__ __launch_bounds__(256) void head_norm_rope_kernel(PagedSeqs, HeadRows r, HeadPrep p, int h, int g, int cap, int slices, uint32_t *err)
{
    head_rows<D>(seqs_arg(), r, p, h, g, cap, (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), slices, err);
}

}  // namespace

hipError_t launch_head_norm_rope(const HeadRows &r, const HeadPrep &p, const relax_layer_dims &dm, const PagedSeqs &st, uint32_t *err, hipStream_t stream)
{
    const int h = r.q ? dm.n_heads : 0, g = r.k ? dm.n_kv_heads : 0, slices = head_slices(h + g, st.n, dm.head_dim);
    const int64_t groups = ((int64_t)st.n * slices + 3) / 4;
    if (groups * 256 > kMaxThreads) return hipErrorInvalidValue;
    if (dm.head_dim == 128) hipLaunchKernelGGL(head_norm_rope_kernel<128>, dim3(groups), dim3(256), 0, stream, st, r, p, h, g, dm.kv_capacity, slices, err);
    else hipLaunchKernelGGL(head_norm_rope_kernel<64>, dim3(groups), dim3(256), 0, stream, st, r, p, h, g, dm.kv_capacity, slices, err);
    return hipGetLastError();
}

}  // namespace relax
