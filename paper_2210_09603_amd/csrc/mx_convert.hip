// Numbers into blocks of 32 that share a power of two, along rows, columns or both, and back.
//
// Memory bound: x is read once.  Along rows the lanes of a block (4, or 8 in fp32) find their maximum among themselves.  Along columns a tile
// of 128 x 128 goes through LDS, where a thread takes 32 rows of two neighbouring columns; both outputs come from the same tile.  Scales lie
// [block][row]: a tile collects those of its rows in LDS and writes words of 4.
#include <algorithm>

#include "mx.hpp"

using namespace hidet;
using namespace hidet::mx;

namespace {

constexpr int kCols = 128;                       // of a tile
constexpr long long kMaxTiles = (1LL << 24) - 1; // of 256 threads: below 2^32 work items

struct Side {
  unsigned char* values;  // null: not wanted
  unsigned char* scales;
  long long stride_values, stride_scales;
  int format;
};
struct QuantizeArgs {
  const void* x;
  long long ldx;
  int rows, cols, col_tiles;
  Side by_rows, by_columns;
};

// What the threads of a tile share while they go through its rows: 16 of them (32 in fp32) hold 128 columns of a row.
template <typename T>
struct Walk {
  static constexpr int N = Chunk<T>::N, LANES = kCols / N, ROWS = 256 / LANES;  // rows a pass
};

// One pass of blocks along rows: row r of the tile, `v` its values from column `col` on.
template <typename T, int TILE_ROWS>
__device__ __forceinline__ void rows_pass(const QuantizeArgs& p, u32x4 raw, int row, int r, int col, int filled, unsigned char* codes) {
  constexpr int N = Chunk<T>::N;
  float v[N];
  unpack<T>(raw, v);
  const int code = scale_code(largest_of_block<N>(v), p.by_rows.format);
  if (row < p.rows && col < filled) store_elements<N>(p.by_rows.values + (long long)row * p.by_rows.stride_values, col, p.by_rows.format, v, code);
  if (col % kBlock == 0) codes[col % kCols / kBlock * TILE_ROWS + r] = (unsigned char)code;
}
// The codes [block][row] of a tile into the scales.
template <int TILE_ROWS>
__device__ __forceinline__ void write_codes(const Side& s, const unsigned char* codes, int row0, int rows, int block0, int blocks) {
  constexpr int WORDS = TILE_ROWS / 4;
  for (int i = threadIdx.x; i < kCols / kBlock * WORDS; i += 256) {
    const int b = i / WORDS, first = i % WORDS * 4;
    if (block0 + b >= blocks) continue;
    unsigned char* to = s.scales + (long long)(block0 + b) * s.stride_scales + row0 + first;
    const unsigned char* from = codes + b * TILE_ROWS + first;
    if (row0 + first + 4 <= rows)
      *reinterpret_cast<unsigned*>(to) = *reinterpret_cast<const unsigned*>(from);
    else
      for (int r = 0; row0 + first + r < rows; ++r) to[r] = from[r];
  }
}

template <typename T, int PASSES>
__global__ __launch_bounds__(256) void rows_kernel(const QuantizeArgs p) {
  using W = Walk<T>;
  constexpr int TILE_ROWS = W::ROWS * PASSES;
  __shared__ __attribute__((aligned(4))) unsigned char codes[kCols / kBlock * TILE_ROWS];
  const int tile_row = blockIdx.x / p.col_tiles, tile_col = blockIdx.x - tile_row * p.col_tiles;
  const int row0 = tile_row * TILE_ROWS, lane = threadIdx.x % W::LANES, first = threadIdx.x / W::LANES;
  const int col = tile_col * kCols + lane * W::N, filled = (p.cols + kBlock - 1) / kBlock * kBlock;
  u32x4 raw[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = row0 + i * W::ROWS + first;
    raw[i] = load_chunk(reinterpret_cast<const T*>(p.x) + (long long)row * p.ldx + col, row < p.rows ? p.cols - col : 0);
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) rows_pass<T, TILE_ROWS>(p, raw[i], row0 + i * W::ROWS + first, i * W::ROWS + first, col, filled, codes);
  __syncthreads();
  write_codes<TILE_ROWS>(p.by_rows, codes, row0, p.rows, tile_col * (kCols / kBlock), filled / kBlock);
}

template <typename T>
struct Two {
  T a, b;
};
// 32 values of a column into its row of the transposed matrix
__device__ __forceinline__ void store_column(const Side& s, long long column, int block, const float (&v)[kBlock], int code) {
  unsigned char* to = s.values + column * s.stride_values + (long long)block * (s.format == HIDET_MX_E2M1 ? 16 : 32);
  unsigned words[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float part[8];
    unsigned two[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) part[e] = v[8 * i + e];
    encode<8>(part, scale_inverse(code), s.format, two);
    words[2 * i] = two[0];
    words[2 * i + 1] = two[1];
  }
  if (s.format == HIDET_MX_E2M1) {
    *reinterpret_cast<u32x4*>(to) = u32x4{words[0], words[2], words[4], words[6]};
  } else {
    *reinterpret_cast<u32x4*>(to) = u32x4{words[0], words[1], words[2], words[3]};
    *reinterpret_cast<u32x4*>(to + 16) = u32x4{words[4], words[5], words[6], words[7]};
  }
}

template <typename T>
__global__ __launch_bounds__(256) void columns_kernel(const QuantizeArgs p) {
  using W = Walk<T>;
  constexpr int TILE_ROWS = 128, PASSES = TILE_ROWS / W::ROWS;
  __shared__ __attribute__((aligned(16))) T tile[TILE_ROWS * kCols];
  __shared__ __attribute__((aligned(4))) unsigned char codes[kCols / kBlock * TILE_ROWS];
  const int tile_row = blockIdx.x / p.col_tiles, tile_col = blockIdx.x - tile_row * p.col_tiles;
  const int row0 = tile_row * TILE_ROWS, lane = threadIdx.x % W::LANES, first = threadIdx.x / W::LANES;
  const int col = tile_col * kCols + lane * W::N, filled = (p.cols + kBlock - 1) / kBlock * kBlock;
  u32x4 raw[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = row0 + i * W::ROWS + first;
    raw[i] = load_chunk(reinterpret_cast<const T*>(p.x) + (long long)row * p.ldx + col, row < p.rows ? p.cols - col : 0);
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) *reinterpret_cast<u32x4*>(tile + (i * W::ROWS + first) * kCols + lane * W::N) = raw[i];
  if (p.by_rows.values) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) rows_pass<T, TILE_ROWS>(p, raw[i], row0 + i * W::ROWS + first, i * W::ROWS + first, col, filled, codes);
  }
  __syncthreads();
  if (p.by_rows.values) write_codes<TILE_ROWS>(p.by_rows, codes, row0, p.rows, tile_col * (kCols / kBlock), filled / kBlock);

  const int pair = threadIdx.x % 64 * 2, block = threadIdx.x / 64;
  const long long column = (long long)tile_col * kCols + pair;
  if (column >= p.cols || row0 + block * kBlock >= p.rows) return;
  float a[kBlock], b[kBlock];
  unsigned top_a = 0, top_b = 0;
#pragma unroll
  for (int r = 0; r < kBlock; ++r) {
    const Two<T> two = *reinterpret_cast<const Two<T>*>(tile + (block * kBlock + r) * kCols + pair);
    a[r] = to_f32(two.a);
    b[r] = to_f32(two.b);
    top_a = max(top_a, magnitude(a[r]));
    top_b = max(top_b, magnitude(b[r]));
  }
  const Side& s = p.by_columns;
  const int code_a = scale_code(top_a, s.format), code_b = scale_code(top_b, s.format), at = row0 / kBlock + block;
  unsigned char* scales = s.scales + (long long)at * s.stride_scales + column;
  store_column(s, column, at, a, code_a);
  if (column + 1 < p.cols) {
    store_column(s, column + 1, at, b, code_b);
    *reinterpret_cast<unsigned short*>(scales) = (unsigned short)(code_a | code_b << 8);
  } else {
    *scales = (unsigned char)code_a;
  }
}

template <typename T>
hipError_t launch_quantize(QuantizeArgs p, hipStream_t stream) {
  const long long col_tiles = (p.cols + kCols - 1) / kCols;
  p.col_tiles = (int)col_tiles;
  if (p.by_columns.values) {
    const long long tiles = ((p.rows + 127LL) / 128) * col_tiles;
    if (tiles > kMaxTiles) return hipErrorInvalidValue;
    hipLaunchKernelGGL((columns_kernel<T>), dim3((unsigned)tiles), dim3(256), 0, stream, p);
  } else {
    constexpr int PASSES = 4, TILE_ROWS = Walk<T>::ROWS * PASSES;
    const long long tiles = ((p.rows + (long long)TILE_ROWS - 1) / TILE_ROWS) * col_tiles;
    if (tiles > kMaxTiles) return hipErrorInvalidValue;
    hipLaunchKernelGGL((rows_kernel<T, PASSES>), dim3((unsigned)tiles), dim3(256), 0, stream, p);
  }
  return hipGetLastError();
}

struct DequantizeArgs {
  const unsigned char* values;
  const unsigned char* scales;
  void* y;
  long long stride_values, stride_scales, ldy;
  int rows, cols, col_tiles, format;
};
// 16 threads hold 128 columns of a row, 8 each.
template <typename T, int PASSES>
__global__ __launch_bounds__(256) void dequantize_kernel(const DequantizeArgs p) {
  const int tile_row = blockIdx.x / p.col_tiles, tile_col = blockIdx.x - tile_row * p.col_tiles;
  const int row0 = tile_row * (16 * PASSES) + threadIdx.x / 16, col = tile_col * kCols + threadIdx.x % 16 * 8;
  if (col >= p.cols) return;
  const unsigned char* scales = p.scales + (long long)(col / kBlock) * p.stride_scales;
  unsigned words[PASSES][2];
  int codes[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = min(row0 + i * 16, p.rows - 1);
    const unsigned char* from = p.values + (long long)row * p.stride_values;
    if (p.format == HIDET_MX_E2M1) {
      words[i][0] = *reinterpret_cast<const unsigned*>(from + col / 2);
      words[i][1] = 0;
    } else {
      const u32x2 two = *reinterpret_cast<const u32x2*>(from + col);
      words[i][0] = two[0];
      words[i][1] = two[1];
    }
    codes[i] = scales[row];
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = row0 + i * 16;
    if (row >= p.rows) return;
    float v[8];
    decode(words[i], p.format, v);
    const float scale = scale_value(codes[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= scale;
    T* y = reinterpret_cast<T*>(p.y) + (long long)row * p.ldy + col;
    constexpr int N = Chunk<T>::N;
#pragma unroll
    for (int c = 0; c < 8 / N; ++c) {
      float part[N];
#pragma unroll
      for (int e = 0; e < N; ++e) part[e] = v[c * N + e];
      store_chunk<T>(y + c * N, p.cols - col - c * N, pack<T>(part));
    }
  }
}
template <typename T>
hipError_t launch_dequantize(DequantizeArgs p, hipStream_t stream) {
  constexpr int PASSES = 4;
  const long long col_tiles = (p.cols + kCols - 1) / kCols, tiles = ((p.rows + 16LL * PASSES - 1) / (16 * PASSES)) * col_tiles;
  if (tiles > kMaxTiles) return hipErrorInvalidValue;
  p.col_tiles = (int)col_tiles;
  hipLaunchKernelGGL((dequantize_kernel<T, PASSES>), dim3((unsigned)tiles), dim3(256), 0, stream, p);
  return hipGetLastError();
}

Side side_of(const hidet_mx_t* m) {
  if (!m) return Side{};
  return Side{reinterpret_cast<unsigned char*>(m->values), reinterpret_cast<unsigned char*>(m->scales), m->stride_values, m->stride_scales, m->format};
}
hidet_status_t status_of(hipError_t e) { return e == hipSuccess ? HIDET_OK : e == hipErrorInvalidValue ? HIDET_ERR_UNSUPPORTED : HIDET_ERR_LAUNCH; }
hidet_status_t check_sides(int dtype, long long rows, long long cols) {
  if (dtype < 0 || dtype > 2 || rows < 0 || cols < 0) return HIDET_ERR_INVALID_ARG;
  return rows >= kMaxSide || cols >= kMaxSide ? HIDET_ERR_UNSUPPORTED : HIDET_OK;
}

}  // namespace

extern "C" {

hidet_status_t hidet_mx_quantize(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, const hidet_mx_t* by_rows,
                                 const hidet_mx_t* by_columns, void* stream) {
  hidet_status_t st = check_sides(dtype, rows, cols);
  if (st != HIDET_OK) return st;
  if (!by_rows && !by_columns) return HIDET_ERR_INVALID_ARG;
  if (by_rows)
    if (st = check_mx(by_rows, rows, cols); st != HIDET_OK) return st;
  if (by_columns)
    if (st = check_mx(by_columns, cols, rows); st != HIDET_OK) return st;
  if (rows == 0 || cols == 0) return HIDET_OK;
  if (st = check_rows(x, dtype, rows, cols, ldx); st != HIDET_OK) return st;
  QuantizeArgs p{};
  p.x = x;
  p.ldx = ldx;
  p.rows = (int)rows;
  p.cols = (int)cols;
  p.by_rows = side_of(by_rows);
  p.by_columns = side_of(by_columns);
  const hipStream_t s = (hipStream_t)stream;
  return status_of(dtype == HIDET_F32   ? launch_quantize<float>(p, s)
                   : dtype == HIDET_F16 ? launch_quantize<f16>(p, s)
                                        : launch_quantize<bf16>(p, s));
}

hidet_status_t hidet_mx_dequantize(int64_t rows, int64_t cols, const hidet_mx_t* x, int32_t dtype, void* y, int64_t ldy, void* stream) {
  hidet_status_t st = check_sides(dtype, rows, cols);
  if (st != HIDET_OK) return st;
  if (st = check_mx(x, rows, cols); st != HIDET_OK) return st;
  if (rows == 0 || cols == 0) return HIDET_OK;
  if (st = check_rows(y, dtype, rows, cols, ldy); st != HIDET_OK) return st;
  DequantizeArgs p{};
  p.values = reinterpret_cast<const unsigned char*>(x->values);
  p.scales = reinterpret_cast<const unsigned char*>(x->scales);
  p.y = y;
  p.stride_values = x->stride_values;
  p.stride_scales = x->stride_scales;
  p.ldy = ldy;
  p.rows = (int)rows;
  p.cols = (int)cols;
  p.format = x->format;
  const hipStream_t s = (hipStream_t)stream;
  return status_of(dtype == HIDET_F32   ? launch_dequantize<float>(p, s)
                   : dtype == HIDET_F16 ? launch_dequantize<f16>(p, s)
                                        : launch_dequantize<bf16>(p, s));
}

}  // extern "C"
