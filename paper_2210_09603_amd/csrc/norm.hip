// Root-mean-square norm of rows, y = h / sqrt(mean(h^2) + eps) * (offset + weight) with h = x + residual, and its gradients.
//
// Memory bound: a row is read once, stays in the registers of the lanes that share it -- in its storage type, as it was rounded for the
// residual stream -- and leaves them normalised, in its type or in blocks of 32 with a scale.  The scale of a block is the maximum over 4 (16-bit
// types) or 8 neighbouring lanes.  Scales lie [block][row]: a workgroup that takes several rows collects theirs in LDS and writes
// words of 4 or 2.
//
// Squares are added in fp64, whose rate here is that of fp32: 1 / sqrt(mean) is the nearest fp32 however long the row and large its values, and
// the elements of y are then rounded to 8 bits on the same side by whoever works them out in this order.
#include <math.h>

#include <algorithm>

#include "mx.hpp"

using namespace hidet;
using namespace hidet::mx;

namespace {

constexpr long long kMaxCols = 32768;
constexpr long long kMaxLd = (1LL << 32) - 1;

struct NormArgs {
  const void* x;
  const void* residual;  // may be null, as all below but the weight
  const void* weight;
  void* sum;
  void* y;
  unsigned char* values;
  unsigned char* scales;
  float* rstd;
  unsigned ldx, ldr, lds, ldy;               // elements
  unsigned stride_values, stride_scales;     // bytes
  int rows, cols;
  int format;
  float eps, offset;
};
static_assert(sizeof(NormArgs) <= 112, "a launch with more takes longer");

// N weights from column `col` on, offset added; 0 beyond the row
template <typename TW, int N>
__device__ __forceinline__ void load_weights(const TW* w, int col, int cols, float offset, float (&v)[N]) {
  constexpr int PER = Chunk<TW>::N;
  if constexpr (PER == N) {
    float t[PER];
    unpack<TW>(load_chunk(w + col, cols - col), t);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = t[e] + offset;
  } else {  // (fp32 weights of a row in 16 bits: two chunks)
#pragma unroll
    for (int i = 0; i < N / PER; ++i) {
      float t[PER];
      unpack<TW>(load_chunk(w + col + i * PER, cols - col - i * PER), t);
#pragma unroll
      for (int e = 0; e < PER; ++e) v[i * PER + e] = t[e] + offset;
    }
  }
}

// A sum over 16 or 64 lanes, the same bits in all of them (a + b and b + a are), without the LDS that shuffles go through: neighbours, pairs, then the
// lanes of 8 and of 16 mirrored, then rows of 16 and halves exchanged.
template <int CONTROL>
__device__ __forceinline__ unsigned lanes_moved(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, 0xf, 0xf, true);
}
template <int CONTROL>
__device__ __forceinline__ float moved(float v) {
  return __builtin_bit_cast(float, lanes_moved<CONTROL>(__builtin_bit_cast(unsigned, v)));
}
template <int CONTROL>
__device__ __forceinline__ double moved(double v) {
  const u32x2 u = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(double, u32x2{lanes_moved<CONTROL>(u[0]), lanes_moved<CONTROL>(u[1])});
}
template <bool HALVES>
__device__ __forceinline__ void exchanged(unsigned u, unsigned& a, unsigned& b) {
  if constexpr (HALVES) {
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    a = (unsigned)r[0], b = (unsigned)r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    a = (unsigned)r[0], b = (unsigned)r[1];
  }
}
template <bool HALVES>
__device__ __forceinline__ float sum_exchanged(float v) {
  unsigned a, b;
  exchanged<HALVES>(__builtin_bit_cast(unsigned, v), a, b);
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
template <bool HALVES>
__device__ __forceinline__ double sum_exchanged(double v) {
  const u32x2 u = __builtin_bit_cast(u32x2, v);
  unsigned a[2], b[2];
  exchanged<HALVES>(u[0], a[0], b[0]);
  exchanged<HALVES>(u[1], a[1], b[1]);
  return __builtin_bit_cast(double, u32x2{a[0], a[1]}) + __builtin_bit_cast(double, u32x2{b[0], b[1]});
}
template <int LANES, typename S>
__device__ __forceinline__ S lane_sum(S v) {
  static_assert(LANES == 16 || LANES >= 64, "a row of lanes, or whole wavefronts");
  v += moved<0xb1>(v);   // quad_perm 1 0 3 2
  v += moved<0x4e>(v);   // quad_perm 2 3 0 1
  v += moved<0x141>(v);  // row_half_mirror
  v += moved<0x140>(v);  // row_mirror
  if constexpr (LANES >= 64) {
    v = sum_exchanged<false>(v);
    v = sum_exchanged<true>(v);
  }
  return v;
}
// Sum over the LANES threads of a row, the same bits in all of them.  LANES > 64: `room`, the row's own, holds a sum of each of its wavefronts;
// contains a barrier of the workgroup.
template <int LANES, typename S>
__device__ __forceinline__ S row_sum(S v, S* room) {
  v = lane_sum<LANES>(v);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) room[threadIdx.x % LANES >> 6] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (int i = 1; i < LANES / 64; ++i) v += room[i];
  }
  return v;
}

// LANES threads a row, CHUNKS chunks of 16 bytes a thread; 256 threads, or as many as a row has.  STREAM: x, residual and what is written pass
// the caches by.  16384 x 8192 in bf16, x + residual into the stream and 8 bits: 165 us for 944 MB, 5.7 TB/s (a copy: 6.1), into 4 bits 162;
// 16384 x 4096 in fp32, into the stream and fp32 174 us for 1074 MB, 6.2 TB/s, and 8 bits 147; 4 x 4096: 2.4 us in the
// kernel, a launch and one trip to memory: with one chunk a thread the weight is asked for with x (333 x 4096 into 8 bits and the product behind it
// 22.65 us together, 22.86 with the weight behind the sum).
template <typename T, typename TW, int LANES, int CHUNKS, bool STREAM>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_kernel(const NormArgs p) {
  static_assert(LANES >= 256 || 256 % LANES == 0, "whole rows");
  constexpr int N = Chunk<T>::N, ROWS = LANES > 256 ? 1 : 256 / LANES, BLOCKS = LANES * CHUNKS * N / kBlock;
  __shared__ double room[LANES > 64 ? ROWS : 1][LANES > 64 ? LANES / 64 : 1];
  __shared__ __attribute__((aligned(16))) unsigned char codes[ROWS > 1 ? BLOCKS * ROWS : 4];
  const int tid = threadIdx.x, lane = tid % LANES, mine = tid / LANES;
  const int row0 = blockIdx.x * ROWS, row = row0 + mine;
  const bool active = row < p.rows;
  const long long at = active ? row : p.rows - 1;  // (a thread without a row reads the last one and writes nothing)
  const T* x = reinterpret_cast<const T*>(p.x) + at * p.ldx;

  u32x4 h[CHUNKS];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int col = (i * LANES + lane) * N;
    h[i] = load_chunk<T, STREAM>(x + col, p.cols - col);
  }
  const TW* weight = reinterpret_cast<const TW*>(p.weight);
  constexpr bool EARLY = CHUNKS == 1;
  float early[N];
  if (EARLY) load_weights<TW, N>(weight, lane * N, p.cols, p.offset, early);
  if (p.residual) {
    const T* r = reinterpret_cast<const T*>(p.residual) + at * p.ldr;
    u32x4 other[CHUNKS];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int col = (i * LANES + lane) * N;
      other[i] = load_chunk<T, STREAM>(r + col, p.cols - col);
    }
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      float a[N], b[N];
      unpack<T>(h[i], a);
      unpack<T>(other[i], b);
#pragma unroll
      for (int e = 0; e < N; ++e) a[e] += b[e];
      h[i] = pack<T>(a);
    }
  }
  if (p.sum && active) {
    T* s = reinterpret_cast<T*>(p.sum) + at * p.lds;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int col = (i * LANES + lane) * N;
      store_chunk<T, STREAM>(s + col, p.cols - col, h[i]);
    }
  }
  double squares = 0.0;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    float v[N];
    unpack<T>(h[i], v);
#pragma unroll
    for (int e = 0; e < N; ++e) squares = __builtin_fma((double)v[e], (double)v[e], squares);
  }
  squares = row_sum<LANES>(squares, room[LANES > 64 ? mine : 0]);
  const float rstd = (float)(1.0 / sqrt(squares / p.cols + (double)p.eps));
  if (p.rstd && active && lane == 0) p.rstd[row] = rstd;

  T* y = p.y ? reinterpret_cast<T*>(p.y) + at * p.ldy : nullptr;
  unsigned char* values = p.values ? p.values + at * p.stride_values : nullptr;
  const int filled = (p.cols + kBlock - 1) / kBlock * kBlock;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int col = (i * LANES + lane) * N;
    float v[N], w[N];
    unpack<T>(h[i], v);
    if (!EARLY) load_weights<TW, N>(weight, col, p.cols, p.offset, w);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = v[e] * rstd * (EARLY ? early[e] : w[e]);
    if (y && active) store_chunk<T, STREAM>(y + col, p.cols - col, pack<T>(v));
    if (values) {  // (the same for all lanes)
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (col + e >= p.cols) v[e] = 0.0f;  // (0 * NaN of a row's statistics, were they left)
      const int code = scale_code(largest_of_block<N>(largest_of(v)), p.format), block = col / kBlock;
      if (col < filled) {
        if (active) store_elements<N, STREAM>(values, col, p.format, v, code);
        if (col % kBlock == 0) {
          if constexpr (ROWS > 1)
            codes[block * ROWS + mine] = (unsigned char)code;
          else
            p.scales[(long long)block * p.stride_scales + row] = (unsigned char)code;
        }
      }
    }
  }
  if constexpr (ROWS > 1) {
    if (!p.values) return;
    __syncthreads();
    using Word = typename std::conditional<ROWS % 4 == 0, unsigned, unsigned short>::type;
    constexpr int EACH = (int)sizeof(Word), WORDS = ROWS / EACH;
    for (int i = tid; i < filled / kBlock * WORDS; i += 256) {
      const int block = i / WORDS, first = i % WORDS * EACH;
      unsigned char* to = p.scales + (long long)block * p.stride_scales + row0 + first;
      const unsigned char* from = codes + block * ROWS + first;
      if (row0 + first + EACH <= p.rows)
        *reinterpret_cast<Word*>(to) = *reinterpret_cast<const Word*>(from);
      else
        for (int r = 0; row0 + first + r < p.rows; ++r) to[r] = from[r];
    }
  }
}

template <typename T, typename TW, int LANES, int CHUNKS>
hipError_t launch_norm(const NormArgs& p, bool far, hipStream_t stream) {
  constexpr int ROWS = LANES > 256 ? 1 : 256 / LANES;
  const dim3 grid((unsigned)((p.rows + ROWS - 1) / ROWS)), block(LANES > 256 ? LANES : 256);
  if ((unsigned long long)grid.x * block.x >= 1ull << 32) return hipErrorInvalidValue;  // (a launch has fewer work items)
  if (far)
    hipLaunchKernelGGL((norm_kernel<T, TW, LANES, CHUNKS, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((norm_kernel<T, TW, LANES, CHUNKS, false>), grid, block, 0, stream, p);
  return hipGetLastError();
}
// How many lanes share a row: two or three chunks each (bf16, x + residual into y and the stream: 16384 x 4096 by 256 lanes 87.7 us, 6.1 TB/s, by 128
// 91.1, by 64 94.4; 32768 x 2048 by 128 88.3, by 64 91.0, by 512 111; 16384 x 8192 into 8 bits by 512 166 us, by 256 172, by 1024 191).  Few
// rows: one chunk, since the row's latency is all there is.
template <typename T, typename TW>
hipError_t dispatch_norm(const NormArgs& p, bool far, hipStream_t stream) {
  const int chunks = (int)(blocks_of(p.cols) * kBlock / Chunk<T>::N);
  if (chunks <= 16) return launch_norm<T, TW, 16, 1>(p, far, stream);
  if (chunks <= 64) return launch_norm<T, TW, 64, 1>(p, far, stream);
  if (p.rows < 1024) {
    if (chunks <= 256) return launch_norm<T, TW, 256, 1>(p, far, stream);
    if (chunks <= 512) return launch_norm<T, TW, 512, 1>(p, far, stream);
    if (chunks <= 1024) return launch_norm<T, TW, 1024, 1>(p, far, stream);
  }
  if (chunks <= 128) return launch_norm<T, TW, 64, 2>(p, far, stream);
  if (chunks <= 192) return launch_norm<T, TW, 64, 3>(p, far, stream);
  if (chunks <= 256) return launch_norm<T, TW, 128, 2>(p, far, stream);
  if (chunks <= 384) return launch_norm<T, TW, 128, 3>(p, far, stream);
  if (chunks <= 512) return launch_norm<T, TW, 256, 2>(p, far, stream);
  if (chunks <= 768) return launch_norm<T, TW, 256, 3>(p, far, stream);
  if (chunks <= 1024) return launch_norm<T, TW, 512, 2>(p, far, stream);
  if (chunks <= 1536) return launch_norm<T, TW, 512, 3>(p, far, stream);
  if (chunks <= 2048) return launch_norm<T, TW, 1024, 2>(p, far, stream);
  if constexpr (Chunk<T>::N == 4)
    if (chunks > 4096) return launch_norm<T, TW, 1024, 8>(p, far, stream);
  return launch_norm<T, TW, 1024, 4>(p, far, stream);
}

// ---- gradients ------------------------------------------------------------------------------------------------------------
struct GradArgs {
  const void* grad_y;
  const void* h;
  const float* rstd;
  const void* weight;
  const void* grad_sum;  // may be null
  void* grad_h;
  float* part;           // [workgroup][cols]; null: no gradient of the weight
  unsigned ldg, ldh, lds, ldo;
  int rows, cols;
  float offset;
};
static_assert(sizeof(GradArgs) <= 112, "a launch with more takes longer");

// A workgroup takes every gridDim-th group of rows and keeps its part of the weight's gradient in registers: lanes hold the same columns of
// every row.  AHEAD: the loads of the next rows are on their way while one group is worked on, and the weight
// stays in registers; without, it and the residual's gradient are read where they are needed.  8192 x 5120 in bf16 with the residual's gradient:
// 60.9 us for 336 MB, 5.5 TB/s, of which the parts of the weight's gradient, written and added, are 4.
template <typename T, typename TW, int LANES, int CHUNKS, bool AHEAD, bool STREAM>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void grad_kernel(const GradArgs p) {
  constexpr int N = Chunk<T>::N, THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES, COLS = LANES * CHUNKS * N;
  __shared__ float room[2][ROWS][LANES > 64 ? LANES / 64 : 1];
  __shared__ float meet[ROWS > 1 ? (ROWS - 1) * COLS : 1];
  const int tid = threadIdx.x, lane = tid % LANES, mine = tid / LANES;
  const TW* weight = reinterpret_cast<const TW*>(p.weight);
  float w[AHEAD ? CHUNKS : 1][N], total[CHUNKS][N];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    if (AHEAD) load_weights<TW, N>(weight, (i * LANES + lane) * N, p.cols, p.offset, w[i]);
#pragma unroll
    for (int e = 0; e < N; ++e) total[i][e] = 0.0f;
  }
  const int groups = (p.rows + ROWS - 1) / ROWS;
  u32x4 next_g[CHUNKS], next_h[CHUNKS], next_s[AHEAD ? CHUNKS : 1];
  float next_rstd;
  auto load = [&](int group) {
    const long long at = min(group * ROWS + mine, p.rows - 1);  // (a thread without a row reads the last one, and nothing comes of it)
    const T* gy = reinterpret_cast<const T*>(p.grad_y) + at * p.ldg;
    const T* hh = reinterpret_cast<const T*>(p.h) + at * p.ldh;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int col = (i * LANES + lane) * N;
      next_g[i] = load_chunk<T, STREAM>(gy + col, p.cols - col);
      next_h[i] = load_chunk<T, STREAM>(hh + col, p.cols - col);
    }
    if (AHEAD) {
      const T* gs = reinterpret_cast<const T*>(p.grad_sum) + at * p.lds;
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int col = (i * LANES + lane) * N;
        next_s[i] = p.grad_sum ? load_chunk<T, STREAM>(gs + col, p.cols - col) : u32x4{0, 0, 0, 0};
      }
    }
    next_rstd = p.rstd[at];
  };
  if (AHEAD) load(blockIdx.x);
  int turn = 0;
  for (int group = blockIdx.x; group < groups; group += gridDim.x, turn ^= 1) {
    const int row = group * ROWS + mine;
    const bool active = row < p.rows;
    if (!AHEAD) load(group);
    u32x4 rg[CHUNKS], rh[CHUNKS], rs[AHEAD ? CHUNKS : 1];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      rg[i] = next_g[i];
      rh[i] = next_h[i];
      if (AHEAD) rs[i] = next_s[i];
    }
    const float rstd = next_rstd;
    if (AHEAD && group + (int)gridDim.x < groups) load(group + gridDim.x);
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      float g[N], h[N];
      unpack<T>(rg[i], g);
      unpack<T>(rh[i], h);
      if (!AHEAD) load_weights<TW, N>(weight, (i * LANES + lane) * N, p.cols, p.offset, w[0]);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float xhat = h[e] * rstd;
        dot += g[e] * w[AHEAD ? i : 0][e] * xhat;
        if (active) total[i][e] += g[e] * xhat;
      }
    }
    // (two rooms in turn: a wavefront may be a row ahead of one that still reads)
    const float mean = row_sum<LANES>(dot, room[turn][mine]) / (float)p.cols;
    if (!active) continue;
    T* out = reinterpret_cast<T*>(p.grad_h) + (long long)row * p.ldo;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int col = (i * LANES + lane) * N;
      float g[N], h[N], s[N];
      unpack<T>(rg[i], g);
      unpack<T>(rh[i], h);
      if (!AHEAD) {
        const T* gs = reinterpret_cast<const T*>(p.grad_sum) + (long long)row * p.lds;
        rs[0] = p.grad_sum ? load_chunk<T, STREAM>(gs + col, p.cols - col) : u32x4{0, 0, 0, 0};
        load_weights<TW, N>(weight, col, p.cols, p.offset, w[0]);
      }
      unpack<T>(rs[AHEAD ? i : 0], s);
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] = rstd * (g[e] * w[AHEAD ? i : 0][e] - h[e] * rstd * mean) + s[e];
      store_chunk<T, STREAM>(out + col, p.cols - col, pack<T>(g));
    }
  }
  if (!p.part) return;
  if constexpr (ROWS > 1) {
    if (mine > 0) {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) meet[(mine - 1) * COLS + (i * N + e) * LANES + lane] = total[i][e];
    }
    __syncthreads();
    if (mine > 0) return;
    for (int r = 0; r < ROWS - 1; ++r)
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) total[i][e] += meet[r * COLS + (i * N + e) * LANES + lane];
  }
  float* part = p.part + (long long)blockIdx.x * p.cols;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int col = (i * LANES + lane) * N;
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (col + e < p.cols) part[col + e] = total[i][e];
  }
}

// The parts of 64 columns: 16 threads add every 16th of them, and one adds what they have, in order.
template <typename TW>
__global__ __launch_bounds__(1024) void join_kernel(const float* part, TW* out, int parts, int cols) {
  __shared__ float meet[16][64];
  const int lane = threadIdx.x % 64, mine = threadIdx.x / 64, col = blockIdx.x * 64 + lane;
  float v = 0.0f;
  if (col < cols) {
#pragma unroll 8
    for (int i = mine; i < parts; i += 16) v += part[(long long)i * cols + col];
  }
  meet[mine][lane] = v;
  __syncthreads();
  if (mine > 0 || col >= cols) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) v += meet[i][lane];
  out[col] = from_f32<TW>(v);
}

// Lanes and chunks of a row's gradient, by its chunks; `most` workgroups, as many as the units hold at once by their registers.  One chunk a lane where a
// workgroup can have as many (bf16: 512 x 5120 by 768 lanes 12.2 us, by 256 of three chunks 18.1; 16384 x 5120 89 and 92, by 384 of two 127; 16384 x 8192 by
// 1024 lanes 142, by 512 of two 161; fp32, 16384 x 5120, by 512 lanes of three chunks 163, by 768 of two 183), then as many as 512
// lanes have registers for (bf16, 4096 x 16384 by 512 lanes of four chunks 86, by 1024, whose registers do not hold two rows, 395); no more workgroups than one
// to a unit, or two of 256 lanes (2048 x 2048: 512 workgroups 12.8, 1024 17.7), since each is a row to add up.  Workgroups are rows of the
// workspace: they follow from the sizes alone.  Where a row and the sums over rows are more than the registers of its lanes, some of it lies in scratch memory: 8 or
// 16 bytes a lane in 16 bits above 16384 columns, 12 in bf16 with fp32 weights from 12289 on, 408 in fp32 above 16384 (4096 x 32768: 630 us, 2.6 TB/s).
struct GradCut {
  int chunks, lanes, each, most;
};
constexpr GradCut kGradCuts[] = {{16, 16, 1, 512},   {64, 64, 1, 512},    {128, 64, 2, 512},    {256, 256, 1, 512},   {512, 512, 1, 256},
                                 {768, 768, 1, 256}, {1024, 1024, 1, 256}, {1536, 512, 3, 256}, {2048, 512, 4, 256},
                                 {4096, 512, 8, 256}, {8192, 512, 16, 256}};
constexpr GradCut kWideCut = {4096, 1024, 4, 256};  // of fp32 (4096 x 16384: 152 us, by 512 lanes 172; half the sums to a chunk)
int cut_of(long long cols, int per_chunk) {
  const long long chunks = (cols + per_chunk - 1) / per_chunk;
  int i = 0;
  while (kGradCuts[i].chunks < chunks) ++i;  // (kMaxCols of 4 a chunk are 8192)
  return i;
}
int parts_of(long long rows, long long cols, int per_chunk) {
  const GradCut& c = kGradCuts[cut_of(cols, per_chunk)];
  const int beside = c.lanes < 256 ? 256 / c.lanes : 1;
  return (int)std::min<long long>((rows + beside - 1) / beside, c.most);
}

template <typename T, typename TW, int CUT>
hipError_t launch_grad(const GradArgs& p, bool far, void* grad_weight, hipStream_t stream) {
  constexpr GradCut c = Chunk<T>::N == 4 && kGradCuts[CUT].chunks == kWideCut.chunks ? kWideCut : kGradCuts[CUT];
  constexpr bool AHEAD = c.each <= (c.lanes > 768 ? 1 : 4);  // (512 lanes have 256 registers each, 1024 have 128)
  const int parts = parts_of(p.rows, p.cols, Chunk<T>::N);
  const dim3 grid((unsigned)parts), block(c.lanes > 256 ? c.lanes : 256);
  if (far)
    hipLaunchKernelGGL((grad_kernel<T, TW, c.lanes, c.each, AHEAD, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((grad_kernel<T, TW, c.lanes, c.each, AHEAD, false>), grid, block, 0, stream, p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || !p.part) return e;
  hipLaunchKernelGGL((join_kernel<TW>), dim3((unsigned)((p.cols + 63) / 64)), dim3(1024), 0, stream, (const float*)p.part,
                     reinterpret_cast<TW*>(grad_weight), parts, p.cols);
  return hipGetLastError();
}
template <typename T, typename TW, int CUT = 0>
hipError_t dispatch_grad(int cut, const GradArgs& p, bool far, void* grad_weight, hipStream_t stream) {
  if constexpr (CUT + 1 < (int)(sizeof(kGradCuts) / sizeof(kGradCuts[0])) && kGradCuts[CUT].chunks * Chunk<T>::N < kMaxCols)
    if (cut > CUT) return dispatch_grad<T, TW, CUT + 1>(cut, p, far, grad_weight, stream);
  return launch_grad<T, TW, CUT>(p, far, grad_weight, stream);
}

hidet_status_t check_norm(int dtype, int weight_dtype, long long rows, long long cols) {
  if (dtype < 0 || dtype > 2 || weight_dtype < 0 || weight_dtype > 2 || rows < 0 || cols < 0) return HIDET_ERR_INVALID_ARG;
  if (weight_dtype != dtype && weight_dtype != HIDET_F32) return HIDET_ERR_UNSUPPORTED;
  if (rows >= kMaxSide || cols > kMaxCols) return HIDET_ERR_UNSUPPORTED;
  return HIDET_OK;
}
// check_rows, and distances that the kernels hold in 32 bits
hidet_status_t check_norm_rows(const void* data, int dtype, long long rows, long long cols, long long ld) {
  if (hidet_status_t st = check_rows(data, dtype, rows, cols, ld); st != HIDET_OK) return st;
  return ld > kMaxLd ? HIDET_ERR_UNSUPPORTED : HIDET_OK;
}
// `out` may be `in` itself, with the same rows
bool in_place_ok(const void* out, long long ld_out, const void* in, long long ld_in, long long rows) {
  return !out || out != in || rows <= 1 || ld_out == ld_in;
}

template <template <typename, typename> class Call, class... A>
hipError_t by_types(int dtype, int weight_dtype, A&&... a) {
  if (dtype == HIDET_F32) return Call<float, float>::run(a...);
  if (dtype == HIDET_F16) return weight_dtype == HIDET_F32 ? Call<f16, float>::run(a...) : Call<f16, f16>::run(a...);
  return weight_dtype == HIDET_F32 ? Call<bf16, float>::run(a...) : Call<bf16, bf16>::run(a...);
}
template <typename T, typename TW>
struct Norm {
  static hipError_t run(const NormArgs& p, bool far, hipStream_t s) { return dispatch_norm<T, TW>(p, far, s); }
};
template <typename T, typename TW>
struct Grad {
  static hipError_t run(const GradArgs& p, bool far, void* grad_weight, hipStream_t s) {
    return dispatch_grad<T, TW>(cut_of(p.cols, Chunk<T>::N), p, far, grad_weight, s);
  }
};

template <typename TW>
__global__ __launch_bounds__(256) void zero_kernel(TW* out, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) out[i] = TW(0.0f);
}

}  // namespace

extern "C" {

hidet_status_t hidet_rms_norm(int32_t dtype, int32_t weight_dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx,
                              const void* residual, int64_t ld_residual, const void* weight, float eps, float offset, void* sum,
                              int64_t ld_sum, void* y, int64_t ldy, const hidet_mx_t* quantized, float* rstd, void* stream) {
  hidet_status_t st = check_norm(dtype, weight_dtype, rows, cols);
  if (st != HIDET_OK) return st;
  if (!(eps >= 0.0f) || !std::isfinite(eps) || !std::isfinite(offset)) return HIDET_ERR_INVALID_ARG;
  if (!y && !quantized) return HIDET_ERR_INVALID_ARG;
  if (quantized)
    if (st = check_mx(quantized, rows, cols); st != HIDET_OK) return st;
  if (rows == 0 || cols == 0) return HIDET_OK;
  if (!weight) return HIDET_ERR_INVALID_ARG;
  if (st = check_norm_rows(x, dtype, rows, cols, ldx); st != HIDET_OK) return st;
  if (residual)
    if (st = check_norm_rows(residual, dtype, rows, cols, ld_residual); st != HIDET_OK) return st;
  if (sum)
    if (st = check_norm_rows(sum, dtype, rows, cols, ld_sum); st != HIDET_OK) return st;
  if (y)
    if (st = check_norm_rows(y, dtype, rows, cols, ldy); st != HIDET_OK) return st;
  if (!is_aligned(weight, size_of(weight_dtype)) || !is_aligned(rstd, 4)) return HIDET_ERR_ALIGNMENT;
  if (!in_place_ok(sum, ld_sum, x, ldx, rows) || !in_place_ok(sum, ld_sum, residual, ld_residual, rows) ||
      !in_place_ok(y, ldy, x, ldx, rows) || !in_place_ok(y, ldy, residual, ld_residual, rows) || (sum && sum == y))
    return HIDET_ERR_INVALID_ARG;
  NormArgs p{};
  p.x = x;
  p.residual = residual;
  p.weight = weight;
  p.sum = sum;
  p.y = y;
  p.rstd = rstd;
  p.ldx = (unsigned)ldx;
  p.ldr = residual ? (unsigned)ld_residual : 0;
  p.lds = sum ? (unsigned)ld_sum : 0;
  p.ldy = y ? (unsigned)ldy : 0;
  p.rows = (int)rows;
  p.cols = (int)cols;
  p.eps = eps;
  p.offset = offset;
  if (quantized) {
    p.values = reinterpret_cast<unsigned char*>(quantized->values);
    p.scales = reinterpret_cast<unsigned char*>(quantized->scales);
    p.stride_values = (unsigned)quantized->stride_values;
    p.stride_scales = (unsigned)quantized->stride_scales;
    p.format = quantized->format;
  }
  const bool far = rows * cols * (long long)size_of(dtype) * (1 + (residual ? 1 : 0) + (sum ? 1 : 0) + (y ? 1 : 0)) > 2 * kFarBytes;
  const hipError_t e = by_types<Norm>(dtype, weight_dtype, p, far, (hipStream_t)stream);
  return e == hipSuccess ? HIDET_OK : e == hipErrorInvalidValue ? HIDET_ERR_UNSUPPORTED : HIDET_ERR_LAUNCH;
}

int64_t hidet_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || rows >= kMaxSide || cols > kMaxCols) return 0;
  return 4LL * cols * std::max(parts_of(rows, cols, 4), parts_of(rows, cols, 8));  // (of rows in 32 bits, and in 16)
}

hidet_status_t hidet_rms_norm_backward(int32_t dtype, int32_t weight_dtype, int64_t rows, int64_t cols, const void* grad_y, int64_t ld_grad_y,
                                       const void* h, int64_t ldh, const float* rstd, const void* weight, float offset,
                                       const void* grad_sum, int64_t ld_grad_sum, void* grad_h, int64_t ld_grad_h, void* grad_weight,
                                       void* workspace, int64_t workspace_bytes, void* stream) {
  hidet_status_t st = check_norm(dtype, weight_dtype, rows, cols);
  if (st != HIDET_OK) return st;
  if (!std::isfinite(offset) || workspace_bytes < 0) return HIDET_ERR_INVALID_ARG;
  if (!is_aligned(grad_weight, size_of(weight_dtype))) return HIDET_ERR_ALIGNMENT;
  const hipStream_t s = (hipStream_t)stream;
  if (cols == 0) return HIDET_OK;
  if (rows == 0) {
    if (!grad_weight) return HIDET_OK;
    const dim3 grid((unsigned)((cols + 255) / 256));
    if (weight_dtype == HIDET_F32)
      hipLaunchKernelGGL((zero_kernel<float>), grid, dim3(256), 0, s, reinterpret_cast<float*>(grad_weight), (int)cols);
    else  // (the zeros of both types are alike)
      hipLaunchKernelGGL((zero_kernel<f16>), grid, dim3(256), 0, s, reinterpret_cast<f16*>(grad_weight), (int)cols);
    return hipGetLastError() == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
  }
  if (!weight || !rstd) return HIDET_ERR_INVALID_ARG;
  if (st = check_norm_rows(grad_y, dtype, rows, cols, ld_grad_y); st != HIDET_OK) return st;
  if (st = check_norm_rows(h, dtype, rows, cols, ldh); st != HIDET_OK) return st;
  if (grad_sum)
    if (st = check_norm_rows(grad_sum, dtype, rows, cols, ld_grad_sum); st != HIDET_OK) return st;
  if (st = check_norm_rows(grad_h, dtype, rows, cols, ld_grad_h); st != HIDET_OK) return st;
  if (!is_aligned(weight, size_of(weight_dtype)) || !is_aligned(rstd, 4)) return HIDET_ERR_ALIGNMENT;
  if (!in_place_ok(grad_h, ld_grad_h, grad_y, ld_grad_y, rows) || !in_place_ok(grad_h, ld_grad_h, grad_sum, ld_grad_sum, rows) || grad_h == h)
    return HIDET_ERR_INVALID_ARG;
  if (grad_weight) {
    if (!workspace || workspace_bytes < hidet_rms_norm_backward_workspace_bytes(rows, cols)) return HIDET_ERR_INVALID_ARG;
    if (!is_aligned(workspace, 16)) return HIDET_ERR_ALIGNMENT;
  }
  GradArgs p{};
  p.grad_y = grad_y;
  p.h = h;
  p.rstd = rstd;
  p.weight = weight;
  p.grad_sum = grad_sum;
  p.grad_h = grad_h;
  p.part = grad_weight ? reinterpret_cast<float*>(workspace) : nullptr;
  p.ldg = (unsigned)ld_grad_y;
  p.ldh = (unsigned)ldh;
  p.lds = grad_sum ? (unsigned)ld_grad_sum : 0;
  p.ldo = (unsigned)ld_grad_h;
  p.rows = (int)rows;
  p.cols = (int)cols;
  p.offset = offset;
  const bool far = rows * cols * (long long)size_of(dtype) * (grad_sum ? 4 : 3) > 2 * kFarBytes;  // (more than the last cache holds)
  const hipError_t e = by_types<Grad>(dtype, weight_dtype, p, far, grad_weight, s);
  return e == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

}  // extern "C"
