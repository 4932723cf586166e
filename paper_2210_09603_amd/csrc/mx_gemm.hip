// Host side of the block-scaled product: its checks, which kernel serves it and how it is cut.
#include <algorithm>

#include "mx_gemm.hpp"

using namespace hidet;
using namespace hidet::mx;

namespace hidet {
namespace mx {
template <>
hipError_t launch_gemm<HIDET_MX_E4M3>(int, const GemmCut&, const GemmArgs&, hipStream_t);
template <>
hipError_t launch_gemm<HIDET_MX_E5M2>(int, const GemmCut&, const GemmArgs&, hipStream_t);
template <>
hipError_t launch_gemm<HIDET_MX_E2M1>(int, const GemmCut&, const GemmArgs&, hipStream_t);
}  // namespace mx
}  // namespace hidet

namespace {

constexpr long long kMaxLd = 1LL << 32;          // of C and the residual
constexpr long long kMaxGrid = (1LL << 22) - 1;  // workgroups of up to 512 threads: below 2^32 work items

// `room`: bytes of workspace
GemmCut cut_gemm(long long M, long long N, long long K, long long room) {
  (void)K;
  (void)room;
  GemmCut c;
  c.slices = 1;
  if (M <= 16) {
    c.kernel = KERNEL_STREAM_16;
    c.blocks = (M + 15) / 16 * ((N + 15) / 16);
  } else if (M <= 64) {
    c.kernel = KERNEL_STREAM_64;
    c.blocks = (M + 63) / 64 * ((N + 63) / 64);
  } else {
    c.kernel = KERNEL_TILE_128;
    c.blocks = (M + 127) / 128 * ((N + 127) / 128);
  }
  return c;
}

hidet_status_t check_epilogue(const hidet_epilogue_t* e, int out, long long M, long long N) {
  if (!e) return HIDET_OK;
  if (e->struct_size != sizeof(hidet_epilogue_t)) return HIDET_ERR_INVALID_ARG;
  if (e->bias_axis < 0 || e->bias_axis > 2 || e->act < 0 || e->act > 1 || e->out_map < 0 || e->out_map > 1 || e->prologue < 0 || e->prologue > 1)
    return HIDET_ERR_INVALID_ARG;
  if (e->out_map != HIDET_MAP_PLAIN || e->prologue != HIDET_PROLOGUE_NONE) return HIDET_ERR_UNSUPPORTED;
  if (!(e->alpha == e->alpha)) return HIDET_ERR_INVALID_ARG;
  if (e->bias_axis != HIDET_BIAS_NONE) {
    if (!e->bias) return HIDET_ERR_INVALID_ARG;
    if (!is_aligned(e->bias, size_of(out))) return HIDET_ERR_ALIGNMENT;
  }
  if (!e->residual || M == 0 || N == 0) return HIDET_OK;
  if (hidet_status_t st = check_rows(e->residual, out, M, N, e->ld_residual); st != HIDET_OK) return st;
  return e->ld_residual >= kMaxLd ? HIDET_ERR_UNSUPPORTED : HIDET_OK;
}

}  // namespace

extern "C" {

int64_t hidet_mx_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t format_a, int32_t format_b) {
  (void)format_a;
  (void)format_b;
  if (M <= 0 || N <= 0 || K <= 0 || M >= kMaxSide || N >= kMaxSide || K >= kMaxSide) return 0;
  const GemmCut c = cut_gemm(M, N, K, 1LL << 62);
  return c.slices > 1 ? 4LL * c.slices * M * N : 0;
}

hidet_status_t hidet_mx_gemm(int32_t out, int64_t M, int64_t N, int64_t K, const hidet_mx_t* A, const hidet_mx_t* B, void* C, int64_t ldc,
                             const hidet_epilogue_t* epi, void* workspace, int64_t workspace_bytes, void* stream) {
  if (out < 0 || out > 2 || M < 0 || N < 0 || K < 0 || workspace_bytes < 0) return HIDET_ERR_INVALID_ARG;
  if (M >= kMaxSide || N >= kMaxSide || K >= kMaxSide) return HIDET_ERR_UNSUPPORTED;
  hidet_status_t st = check_mx(A, M, K);
  if (st != HIDET_OK) return st;
  if (st = check_mx(B, N, K); st != HIDET_OK) return st;
  if (st = check_epilogue(epi, out, M, N); st != HIDET_OK) return st;
  if (workspace && !is_aligned(workspace, 16)) return HIDET_ERR_ALIGNMENT;
  if (M == 0 || N == 0) return HIDET_OK;
  if (st = check_rows(C, out, M, N, ldc); st != HIDET_OK) return st;
  if (ldc >= kMaxLd) return HIDET_ERR_UNSUPPORTED;
  if (epi && epi->residual == C && M > 1 && epi->ld_residual != ldc) return HIDET_ERR_INVALID_ARG;

  const GemmCut c = cut_gemm(M, N, K, workspace ? workspace_bytes : 0);
  if (c.blocks > kMaxGrid) return HIDET_ERR_UNSUPPORTED;
  GemmArgs p{};
  p.a = reinterpret_cast<const unsigned char*>(A->values);
  p.b = reinterpret_cast<const unsigned char*>(B->values);
  p.scales_a = reinterpret_cast<const unsigned char*>(A->scales);
  p.scales_b = reinterpret_cast<const unsigned char*>(B->scales);
  p.c = C;
  p.lda = (unsigned)A->stride_values;
  p.ldb = (unsigned)B->stride_values;
  p.ld_scales_a = (unsigned)A->stride_scales;
  p.ld_scales_b = (unsigned)B->stride_scales;
  p.ldc = (unsigned)ldc;
  p.M = (int)M;
  p.N = (int)N;
  p.blocks = (int)blocks_of(K);
  p.alpha = 1.0f;
  const size_t four = 4 * size_of(out);
  bool quads = is_aligned(C, four) && (M == 1 || ldc % 4 == 0);
  p.flags = (unsigned)out;
  if (epi) {
    p.alpha = epi->alpha;
    p.bias = epi->bias_axis ? epi->bias : nullptr;
    p.residual = epi->residual;
    p.ldr = epi->residual ? (unsigned)epi->ld_residual : 0;
    p.flags |= (unsigned)epi->bias_axis << 2 | (epi->act == HIDET_ACT_RELU ? 16u : 0u);
    if (epi->residual) quads = quads && is_aligned(epi->residual, four) && (M == 1 || epi->ld_residual % 4 == 0);
  }
  p.flags |= (quads ? 32u : 0u) | (unsigned)c.slices << 8;
  const int steps = (p.blocks + 3) / 4;
  p.slice = (steps + c.slices - 1) / c.slices;
  if (c.slices > 1) p.c = workspace;
  const hipStream_t s = (hipStream_t)stream;
  hipError_t e = A->format == HIDET_MX_E4M3   ? launch_gemm<HIDET_MX_E4M3>(B->format, c, p, s)
                 : A->format == HIDET_MX_E5M2 ? launch_gemm<HIDET_MX_E5M2>(B->format, c, p, s)
                                              : launch_gemm<HIDET_MX_E2M1>(B->format, c, p, s);
  if (e == hipSuccess && c.slices > 1) {
    p.c = C;
    const long long quads_all = M * ((N + 3) / 4), blocks = (quads_all + 255) / 256;
    const dim3 grid((unsigned)blocks);
    const float* sums = reinterpret_cast<const float*>(workspace);
    if (out == HIDET_F32)
      hipLaunchKernelGGL((join_slices_kernel<float>), grid, dim3(256), 0, s, p, sums);
    else if (out == HIDET_F16)
      hipLaunchKernelGGL((join_slices_kernel<f16>), grid, dim3(256), 0, s, p, sums);
    else
      hipLaunchKernelGGL((join_slices_kernel<bf16>), grid, dim3(256), 0, s, p, sums);
    e = hipGetLastError();
  }
  return e == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

}  // extern "C"
