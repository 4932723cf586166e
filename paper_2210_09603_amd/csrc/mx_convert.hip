// Numbers into blocks of 32 that share a power of two, along rows, columns or both, and back.
//
// Memory bound: x is read once.  Along rows the lanes of a block (4, or 8 in fp32) find their maximum among themselves.  Along columns a tile
// of 128 x 128 goes through LDS, where two lanes take 32 rows of two neighbouring columns; both outputs come from the same tile.  Scales lie
// [block][row]: a tile collects those of its rows in LDS and writes words of 4.
#include <algorithm>

#include "mx.hpp"

using namespace hidet;
using namespace hidet::mx;

namespace {

// The most workgroups of a launch: it has fewer than 2^32 work items.
constexpr long long most_tiles(int threads) { return ((1LL << 32) - 1) / threads; }

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

// How THREADS threads go through a tile of COLS columns: LANES of them hold a row, ROWS rows are a pass.
template <typename T, int COLS, int THREADS = 256>
struct Walk {
  static constexpr int N = Chunk<T>::N, LANES = COLS / N, ROWS = THREADS / LANES;
};

// One pass of blocks along rows: row r of the tile, `v` its values from column `col` on.
template <typename T, int COLS, int TILE_ROWS, bool STREAM>
__device__ __forceinline__ void rows_pass(const QuantizeArgs& p, u32x4 raw, int row, int r, int col, int filled, unsigned char* codes) {
  constexpr int N = Chunk<T>::N;
  float v[N];
  unpack<T>(raw, v);
  const int code = scale_code(largest_of_block<N>(largest_of_chunk<T>(raw)), p.by_rows.format);
  if (row < p.rows && col < filled) store_elements<N, STREAM>(p.by_rows.values + (long long)row * p.by_rows.stride_values, col, p.by_rows.format, v, code);
  if (col % kBlock == 0) codes[col % COLS / kBlock * TILE_ROWS + r] = (unsigned char)code;
}
// The codes [block][row] of a tile into the scales.
template <int COLS, int TILE_ROWS>
__device__ __forceinline__ void write_codes(const Side& s, const unsigned char* codes, int row0, int rows, int block0, int blocks) {
  constexpr int WORDS = TILE_ROWS / 4;
  for (int i = threadIdx.x; i < COLS / kBlock * WORDS; i += blockDim.x) {
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

template <typename T, int COLS, int PASSES, bool STREAM>
__global__ __launch_bounds__(256) void rows_kernel(const QuantizeArgs p) {
  using W = Walk<T, COLS>;
  constexpr int TILE_ROWS = W::ROWS * PASSES;
  __shared__ __attribute__((aligned(4))) unsigned char codes[COLS / kBlock * TILE_ROWS];
  const int tile_row = blockIdx.x / p.col_tiles, tile_col = blockIdx.x - tile_row * p.col_tiles;
  const int row0 = tile_row * TILE_ROWS, lane = threadIdx.x % W::LANES, first = threadIdx.x / W::LANES;
  const int col = tile_col * COLS + lane * W::N, filled = (p.cols + kBlock - 1) / kBlock * kBlock;
  u32x4 raw[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = row0 + i * W::ROWS + first;
    raw[i] = load_chunk<T, STREAM>(reinterpret_cast<const T*>(p.x) + (long long)row * p.ldx + col, row < p.rows ? p.cols - col : 0);
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) rows_pass<T, COLS, TILE_ROWS, STREAM>(p, raw[i], row0 + i * W::ROWS + first, i * W::ROWS + first, col, filled, codes);
  __syncthreads();
  write_codes<COLS, TILE_ROWS>(p.by_rows, codes, row0, p.rows, tile_col * (COLS / kBlock), filled / kBlock);
}

// 16 rows, half a block, of two neighbouring columns of a tile in LDS.
template <typename T>
struct Pair {
  static constexpr int ROWS = kBlock / 2;
  unsigned raw[ROWS * (int)sizeof(T) / 2];
  // the larger magnitude of either column
  __device__ __forceinline__ void largest(unsigned (&top)[2]) const {
    if constexpr (sizeof(T) == 4) {
      top[0] = top[1] = 0;
#pragma unroll
      for (int i = 0; i < 2 * ROWS; ++i) top[i & 1] = max(top[i & 1], raw[i] & 0x7fffffffu);
    } else {
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < ROWS; ++i) m = larger_pair(m, raw[i]);
      top[0] = widened<T>(m & 0xffffu);
      top[1] = widened<T>(m >> 16);
    }
  }
  __device__ __forceinline__ float value(int row, int column) const {
    if constexpr (sizeof(T) == 4)
      return __builtin_bit_cast(float, raw[2 * row + column]);
    else
      return to_f32(__builtin_bit_cast(T, (unsigned short)(column ? raw[row] >> 16 : raw[row] & 0xffffu)));
  }
};
// The elements of a column of them, 8 or 16 bytes of LDS
template <typename T>
__device__ __forceinline__ void put_half(unsigned char* to, int format, const Pair<T>& two, int column, int code) {
  unsigned words[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float part[8];
    unsigned out[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) part[e] = two.value(8 * i + e, column);
    encode<8>(part, scale_inverse(code), format, out);
    words[2 * i] = out[0];
    words[2 * i + 1] = out[1];
  }
  if (format == HIDET_MX_E2M1)
    *reinterpret_cast<u32x2*>(to) = u32x2{words[0], words[2]};
  else
    *reinterpret_cast<u32x4*>(to) = u32x4{words[0], words[1], words[2], words[3]};
}

// 4096 x 4096 in bf16 into 8 bits along both axes: 16.4 us, 4.2 TB/s; 4099 x 1003 in fp16 8.5; 16384 x 8192 110 (4.9 TB/s).  Four phases with a barrier between
// them: four workgroups of 512 threads a compute unit hide one behind another's.  (256 threads, each with whole blocks: 18.1, 11.1 and 111.)
template <typename T, bool STREAM>
__global__ __launch_bounds__(512) void columns_kernel(const QuantizeArgs p) {
  constexpr int COLS = 128, TILE_ROWS = 128, THREADS = 512;  // (lanes l and l + 32 for two columns of a block)
  using W = Walk<T, COLS, THREADS>;
  constexpr int PASSES = TILE_ROWS / W::ROWS;
  __shared__ __attribute__((aligned(16))) T tile[TILE_ROWS * COLS];
  __shared__ __attribute__((aligned(4))) unsigned char codes[COLS / kBlock * TILE_ROWS];
  const int tile_row = blockIdx.x / p.col_tiles, tile_col = blockIdx.x - tile_row * p.col_tiles;
  const int row0 = tile_row * TILE_ROWS, lane = threadIdx.x % W::LANES, first = threadIdx.x / W::LANES;
  const int col = tile_col * COLS + lane * W::N, filled = (p.cols + kBlock - 1) / kBlock * kBlock;
  u32x4 raw[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = row0 + i * W::ROWS + first;
    raw[i] = load_chunk<T, STREAM>(reinterpret_cast<const T*>(p.x) + (long long)row * p.ldx + col, row < p.rows ? p.cols - col : 0);
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) *reinterpret_cast<u32x4*>(tile + (i * W::ROWS + first) * COLS + lane * W::N) = raw[i];
  if (p.by_rows.values) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) rows_pass<T, COLS, TILE_ROWS, STREAM>(p, raw[i], row0 + i * W::ROWS + first, i * W::ROWS + first, col, filled, codes);
  }
  __syncthreads();
  if (p.by_rows.values) write_codes<COLS, TILE_ROWS>(p.by_rows, codes, row0, p.rows, tile_col * (COLS / kBlock), filled / kBlock);

  // columns: their elements back into LDS, from where they leave as whole rows of the transposed matrix
  constexpr int PITCH = TILE_ROWS + 16;
  static_assert(COLS * PITCH <= (int)sizeof(tile), "the elements take the tile's place");
  const Side& s = p.by_columns;
  const int wave = threadIdx.x / 64, half = threadIdx.x / 32 % 2, pair = (wave % 2 * 32 + threadIdx.x % 32) * 2, block = wave / 2;
  const int each = s.format == HIDET_MX_E2M1 ? 16 : 32;
  const long long column = (long long)tile_col * COLS + pair;
  Pair<T> two;
#pragma unroll
  for (int r = 0; r < Pair<T>::ROWS; ++r)
    __builtin_memcpy(two.raw + r * (int)sizeof(T) / 2, tile + (block * kBlock + half * Pair<T>::ROWS + r) * COLS + pair, 2 * sizeof(T));
  unsigned top[2];
  two.largest(top);
#pragma unroll
  for (int c = 0; c < 2; ++c) top[c] = max(top[c], (unsigned)__shfl_xor((int)top[c], 32));
  const int code_a = scale_code(top[0], s.format), code_b = scale_code(top[1], s.format);
  if (half == 0 && column < p.cols && row0 + block * kBlock < p.rows) {
    unsigned char* scales = s.scales + (long long)(row0 / kBlock + block) * s.stride_scales + column;
    if (column + 1 < p.cols)
      *reinterpret_cast<unsigned short*>(scales) = (unsigned short)(code_a | code_b << 8);
    else
      *scales = (unsigned char)code_a;
  }
  __syncthreads();  // (the tile is read)
  unsigned char* out = reinterpret_cast<unsigned char*>(tile);
  put_half(out + pair * PITCH + block * each + half * each / 2, s.format, two, 0, code_a);
  put_half(out + (pair + 1) * PITCH + block * each + half * each / 2, s.format, two, 1, code_b);
  __syncthreads();
  const int chunks = TILE_ROWS / kBlock * each / 16;  // of a row of the transposed matrix
  for (int i = threadIdx.x; i < COLS * chunks; i += THREADS) {
    const int r = i / chunks, c = i - r * chunks;
    if (tile_col * COLS + r >= p.cols || row0 + c * 16 / each * kBlock >= p.rows) continue;
    unsigned char* to = s.values + (long long)(tile_col * COLS + r) * s.stride_values + (long long)row0 / kBlock * each + c * 16;
    *reinterpret_cast<u32x4*>(to) = *reinterpret_cast<const u32x4*>(out + r * PITCH + c * 16);
  }
}

template <typename T>
hipError_t launch_quantize(QuantizeArgs p, hipStream_t stream) {
  const bool far = (long long)p.rows * p.cols * (int)sizeof(T) >= kFarBytes;
  auto grid = [&](int rows, int cols) {
    const long long col_tiles = (p.cols + (long long)cols - 1) / cols, tiles = (p.rows + (long long)rows - 1) / rows * col_tiles;
    p.col_tiles = (int)col_tiles;
    return tiles;
  };
  if (p.by_columns.values) {
    constexpr int THREADS = 512;
    const long long tiles = grid(128, 128);
    if (tiles > most_tiles(THREADS)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((far ? columns_kernel<T, true> : columns_kernel<T, false>), dim3((unsigned)tiles), dim3(THREADS), 0, stream, p);
    return hipGetLastError();
  }
  // Rows of 1 KB or more of a tile, four loads a thread in flight: 16384 x 4096 in bf16 into 4 bits 28.8 us (5.8 TB/s); 128 columns 32.1, two
  // loads 30.4, all through the caches 36.2.  Few tiles of these: smaller ones.  (us into 8 bits, large and small tiles, by large ones: bf16, 4096 columns,
  // 256 tiles 4.1 and 3.3, 1000 7.3 and 6.9, 1024 7.3 and 6.9, 1504 9.1 and 8.6, 2048 10.2 and 10.4; fp32, 512 4.0 and 3.7, 1024 6.4 and 6.2, 2048
  // 8.9 and 9.2, 8192 28.9 and 33.2: from 1024 to some 2000 tiles the small ones would still take up to 8 % less.)
  constexpr int FAR_ROWS = Walk<T, 512>::ROWS * 4, NEAR_ROWS = Walk<T, 128>::ROWS;
  constexpr int THREADS = 256;
  if (const long long tiles = grid(FAR_ROWS, 512); tiles >= 1024) {
    if (tiles > most_tiles(THREADS)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((far ? rows_kernel<T, 512, 4, true> : rows_kernel<T, 512, 4, false>), dim3((unsigned)tiles), dim3(THREADS), 0, stream, p);
  } else {
    hipLaunchKernelGGL((rows_kernel<T, 128, 1, false>), dim3((unsigned)grid(NEAR_ROWS, 128)), dim3(THREADS), 0, stream, p);
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
// Tiles of 16 x 128: 16 threads hold the columns of a row, 8 each.
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void dequantize_kernel(const DequantizeArgs p) {
  const int tile_row = blockIdx.x / p.col_tiles, tile_col = blockIdx.x - tile_row * p.col_tiles;
  const int row = tile_row * 16 + threadIdx.x / 16, col = tile_col * 128 + threadIdx.x % 16 * 8;
  if (col >= p.cols || row >= p.rows) return;
  const unsigned char* from = p.values + (long long)row * p.stride_values;
  unsigned words[2] = {0, 0};
  if (p.format == HIDET_MX_E2M1) {
    words[0] = load_word<STREAM>(reinterpret_cast<const unsigned*>(from + col / 2));
  } else {
    const u32x2 two = load_word<STREAM>(reinterpret_cast<const u32x2*>(from + col));
    words[0] = two[0];
    words[1] = two[1];
  }
  const float scale = scale_value(p.scales[(long long)(col / kBlock) * p.stride_scales + row]);
  float v[8];
  decode(words, p.format, v);
  T* y = reinterpret_cast<T*>(p.y) + (long long)row * p.ldy + col;
  constexpr int N = Chunk<T>::N;
#pragma unroll
  for (int c = 0; c < 8 / N; ++c) {
    float part[N];
#pragma unroll
    for (int e = 0; e < N; ++e) part[e] = v[c * N + e] * scale;
    store_chunk<T, STREAM>(y + c * N, p.cols - col - c * N, pack<T>(part));
  }
}
template <typename T>
hipError_t launch_dequantize(DequantizeArgs p, hipStream_t stream) {
  // (16384 x 4096 from 4 bits into bf16: 33.4 us, 5.0 TB/s, four fifths of it written; with two rows a thread 36.2, with four 39.7, all through the
  // caches 40.8)
  const long long col_tiles = (p.cols + 127LL) / 128, tiles = (p.rows + 15LL) / 16 * col_tiles;
  constexpr int THREADS = 256;
  if (tiles > most_tiles(THREADS)) return hipErrorInvalidValue;
  p.col_tiles = (int)col_tiles;
  const bool far = (long long)p.rows * p.cols * (int)sizeof(T) >= kFarBytes;
  hipLaunchKernelGGL((far ? dequantize_kernel<T, true> : dequantize_kernel<T, false>), dim3((unsigned)tiles), dim3(THREADS), 0, stream, p);
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
  if (by_rows && by_columns && (by_rows->values == by_columns->values || by_rows->scales == by_columns->scales)) return HIDET_ERR_INVALID_ARG;
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
