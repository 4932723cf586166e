// The kernels of the block-scaled product for the format HIDET_MX_A of A: compiled once for each.
#include "mx_gemm.hpp"

namespace hidet {
namespace mx {

template <int FA, int FB>
hipError_t launch(const GemmCut& c, const GemmArgs& p, hipStream_t stream) {
  const dim3 grid((unsigned)c.blocks);
  switch (c.kernel) {
    case KERNEL_TILE_256: hipLaunchKernelGGL((tile_kernel<FA, FB, 4, 4, 1>), grid, dim3(1024), 0, stream, p); break;
    case KERNEL_TILE_128: hipLaunchKernelGGL((tile_kernel<FA, FB, 2, 2, 1>), grid, dim3(256), 0, stream, p); break;
    case KERNEL_TILE_64X128: hipLaunchKernelGGL((tile_kernel<FA, FB, 1, 2, 2>), grid, dim3(256), 0, stream, p); break;
    case KERNEL_TILE_64: hipLaunchKernelGGL((tile_kernel<FA, FB, 1, 1, 4>), grid, dim3(256), 0, stream, p); break;
    case KERNEL_STREAM_16: hipLaunchKernelGGL((stream_kernel<FA, FB, false>), grid, dim3(512), 0, stream, p); break;
    default: hipLaunchKernelGGL((stream_kernel<FA, FB, true>), grid, dim3(512), 0, stream, p); break;
  }
  return hipGetLastError();
}

template <>
hipError_t launch_gemm<HIDET_MX_A>(int format_b, const GemmCut& c, const GemmArgs& p, hipStream_t stream) {
  if (format_b == HIDET_MX_E4M3) return launch<HIDET_MX_A, HIDET_MX_E4M3>(c, p, stream);
  if (format_b == HIDET_MX_E5M2) return launch<HIDET_MX_A, HIDET_MX_E5M2>(c, p, stream);
  return launch<HIDET_MX_A, HIDET_MX_E2M1>(c, p, stream);
}

}  // namespace mx
}  // namespace hidet
