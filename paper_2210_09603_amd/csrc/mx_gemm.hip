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
constexpr long long kMaxGrid = (1LL << 22) - 1;  // workgroups of up to 1024 threads: below 2^32 work items

constexpr int kUnits = 256;                      // compute units

// What a tile takes for a step of 128 k, in us: where each unit has one of them, and, by the unit's time, where there are more.  Both operands in 8
// bits, one, none.  (K = 4096; 333 x 5120, 1024 x 1024, 4096 x 4096 and 8192 x 8192.)  What the kernels on both sides of a border take at
// K = 4096 into bf16, 8 bits by 8, 8 by 4, 4 by 4, in us; * is the one that is chosen:
//   1024 x 1024   64 x 64    15.5* 13.8* 12.1*   64 x 128   19.1  17.3  16.2
//   1024 x 1536   64 x 64    27.7  25.3  14.5    64 x 128   18.9* 17.0* 15.3*
//   1024 x 2048   64 x 128   19.5* 17.4* 15.6*   128 x 128  23.7  25.5  24.9
//   2048 x 2048   64 x 128   37.4  23.2  20.6    128 x 128  27.0* 26.7* 19.5*
//   3000 x 4096   128 x 128  57.9* 56.3* 38.6*   256 x 256  53.1  50.0  35.6
//   4096 x 4096   128 x 128  70.3  66.7  47.3    256 x 256  60.2* 55.1* 38.9*
// (with slices of K where cut_slices makes them).  Of 381 products of 17 to 8192 rows the choice is within 3 % of the fastest kernel in 311 and within
// 10 % in 356.  It is off by most for 8 bits by 4, where two and three rounds of 64 x 128 tiles take less than the model has for them:
// 512 x 8192 x 8192 on 128 x 128 tiles 47.6, on 64 x 128 37.3.
struct TileCost {
  int kernel, rows, cols;
  float alone[3], among[3], once;  // once: of a tile, its first loads and its stores
};
constexpr TileCost kTiles[] = {
    {KERNEL_TILE_256, 256, 256, {1.60f, 1.45f, 1.05f}, {1.65f, 1.48f, 1.05f}, 5.0f},
    {KERNEL_TILE_128, 128, 128, {0.57f, 0.50f, 0.34f}, {0.47f, 0.41f, 0.30f}, 2.0f},
    {KERNEL_TILE_64X128, 64, 128, {0.42f, 0.34f, 0.27f}, {0.48f, 0.26f, 0.19f}, 2.0f},
    {KERNEL_TILE_64, 64, 64, {0.28f, 0.24f, 0.18f}, {0.35f, 0.31f, 0.16f}, 2.0f},
};
constexpr float kJoin = 4.0f;  // us, of the second launch of a product in slices
// The same of the workgroups of few rows, whose wavefronts take 8 steps at once; by rounds of one to a unit, and as far as they begin sooner than tiles.
// Them and tiles (those that are chosen, else the fastest), as above:
//   32 x 4096 x 4096    11.2  8.9* 8.1*   13.0* 11.0 10.6        64 x 4096 x 4096    12.9  9.4* 8.4*   14.2* 12.4 11.8
//   100 x 4096 x 4096   22.6 14.8* 13.1*  14.1* 13.9 12.0        128 x 4096 x 4096   22.7 15.0* 13.2*  14.4* 13.5 11.7
//   256 x 1024 x 1024   5.9* 5.1* 4.8*    8.3   8.1  7.3         512 x 1024 x 1024    9.1  6.6* 6.1*   8.4*  8.2  7.4
//   64 x 8192 x 2048    14.1 9.4* 8.5*    11.3* 9.9  8.8         48 x 8192 x 8192    40.0 25.0 22.0    21.5* 18.3* 16.5*
// (the last: 64 x 128 tiles 19.8, 16.1 and 14.9).  The time has no term for A, which every workgroup of columns reads again: at 100 and 128 rows it
// is up to 14 % off.  More than two rounds are left to the tiles.
constexpr float kStream[3] = {0.27f, 0.15f, 0.12f};

long long tiles_of(long long M, long long N, long long rows, long long cols) { return (M + rows - 1) / rows * ((N + cols - 1) / cols); }

// Cuts c along K where its workgroups leave units without work, and that saves more than the second launch takes.  each: steps that a slice is
// made of; per: us of a step; most: slices that the workspace has room for.  Gives the us of what follows its first loads.
float cut_slices(GemmCut& c, long long steps, long long each, float per, long long most) {
  const float whole = (float)steps * per;
  if (c.blocks > kUnits / 2) return whole * (float)((c.blocks + kUnits - 1) / kUnits);
  const long long slices = std::min(std::min<long long>(kUnits / c.blocks, steps / (2 * each)), most);
  if (slices < 2) return whole;
  const long long slice = ((steps + slices - 1) / slices + each - 1) / each * each, cut = (steps + slice - 1) / slice;
  if (cut < 2 || (float)(steps - slice) * per <= kJoin) return whole;
  c.slices = (int)cut;
  c.slice = (int)slice;
  c.blocks *= cut;
  return (float)slice * per + kJoin;
}

// `room`: bytes of workspace
GemmCut cut_gemm(long long M, long long N, long long K, int format_a, int format_b, long long room) {
  const long long steps = std::max(1LL, (K + 127) / 128);
  const int kind = 2 - (int)is_wide(format_a) - (int)is_wide(format_b);
  const long long most = room / 4 / M / N;
  if (M <= 16) {
    // (4 x 8192 x 4096, 8 bits by 4: 6.6 us; 64 columns a workgroup 7.9, 64 x 64 tiles 13.2.)
    GemmCut c{KERNEL_STREAM_16, 1, 1 << 24, tiles_of(M, N, 16, 16)};
    cut_slices(c, steps, 8, 0.06f, most);
    return c;
  }
  GemmCut tile{}, stream{KERNEL_STREAM_16X64, 1, 1 << 24, tiles_of(M, N, 16, 64)};
  float best = 0.0f, alone = 0.0f, once = 0.0f;
  for (const TileCost& t : kTiles) {
    const long long tiles = tiles_of(M, N, t.rows, t.cols);
    const float rounds = (float)((tiles + kUnits - 1) / kUnits);
    const float us = rounds * ((float)steps * (tiles <= kUnits ? t.alone[kind] : t.among[kind]) + t.once);
    if (best == 0.0f || us < best) {
      best = us;
      tile = GemmCut{t.kernel, 1, 1 << 24, tiles};
      alone = t.alone[kind];
      once = t.once;
    }
  }
  if (const float us = cut_slices(tile, steps, 4, alone, most); tile.slices > 1) best = us + once;
  if (stream.blocks > 2 * kUnits) return tile;
  return cut_slices(stream, steps, 8, kStream[kind], most) < best ? stream : tile;
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
  if (format_a < 0 || format_a > HIDET_MX_E2M1 || format_b < 0 || format_b > HIDET_MX_E2M1) return 0;
  if (M <= 0 || N <= 0 || K <= 0 || M >= kMaxSide || N >= kMaxSide || K >= kMaxSide) return 0;
  const GemmCut c = cut_gemm(M, N, K, format_a, format_b, 1LL << 62);
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

  const GemmCut c = cut_gemm(M, N, K, A->format, B->format, workspace ? workspace_bytes : 0);
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
  p.flags = (unsigned)out;
  if (epi) {
    p.alpha = epi->alpha;
    p.bias = epi->bias_axis ? epi->bias : nullptr;
    p.residual = epi->residual;
    p.ldr = epi->residual ? (unsigned)epi->ld_residual : 0;
    p.flags |= (unsigned)epi->bias_axis << 2 | (epi->act == HIDET_ACT_RELU ? 16u : 0u);
  }
  p.flags |= (unsigned)c.slices << 8;
  p.slice = c.slice;
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
