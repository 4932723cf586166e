// Rotary positions: pairs (a, b) of a vector turn by the angle position * frequency, a' = f (a cos - b sin), b' = f (b cos + a sin).
//
// Memory bound: every element is read and written once.  The angles are shared by all heads of a token, so a workgroup takes a
// few tokens with all their heads (or, where there are few tokens, some of the heads), works out sine and cosine of its tokens once
// into LDS, and then streams 16-byte chunks.  A thread holds both elements of its pairs, so that a tensor can be turned in place.
//
// Angles of far positions: position * frequency passes 10^5 rad, where fp32 steps are 0.01 rad.  The product is taken in
// turns and in fp64, its whole turns are dropped there, and sine and cosine are taken in fp32 of what is left.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "attention_host.hpp"

using namespace hidet;
using namespace hidet::attn;

namespace {

constexpr int kThreads = 256;
constexpr int kTableBytes = 32 * 1024;

struct RopeArgs {
  const void* x;
  void* y;
  Strides xs, ys;
  const double* frequencies;
  const int* positions;
  long long positions_stride, first_position;
  int heads, seq, dim, rotary;
  int tokens;  // batch * seq
  int block_tokens, block_heads, head_blocks;
  int turn_items, copy_items;  // of a row
  FastDiv d_seq, d_items, d_heads;
  int inverse;
  float amplitude;
};

template <typename T>
struct Vec {
  static constexpr int N = 16 / (int)sizeof(T);
  struct __attribute__((packed, aligned(sizeof(T)))) Raw {
    u32x4 v;
  };
  typedef u32x4 Streamed __attribute__((aligned(2)));  // (the same, for an access with a hint)
};
// up to N elements, element by element where fewer are left
template <typename T, bool STREAM>
__device__ __forceinline__ void load_vec(const T* at, int count, float (&v)[Vec<T>::N]) {
  T t[Vec<T>::N];
  if (count >= Vec<T>::N) {
    u32x4 raw;
    if constexpr (STREAM)
      raw = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T>::Streamed*>(at));
    else
      raw = reinterpret_cast<const typename Vec<T>::Raw*>(at)->v;
    __builtin_memcpy(t, &raw, 16);
  } else {
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) t[e] = at[e < count ? e : 0];
  }
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) v[e] = to_f32(t[e]);
}
template <typename T, bool STREAM>
__device__ __forceinline__ void store_vec(T* at, int count, const float (&v)[Vec<T>::N]) {
  T t[Vec<T>::N];
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) t[e] = from_f32<T>(v[e]);
  if (count >= Vec<T>::N) {
    u32x4 raw;
    __builtin_memcpy(&raw, t, 16);
    if constexpr (STREAM)
      __builtin_nontemporal_store(raw, reinterpret_cast<typename Vec<T>::Streamed*>(at));
    else
      reinterpret_cast<typename Vec<T>::Raw*>(at)->v = raw;
  } else {
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e)
      if (e < count) at[e] = t[e];
  }
}

// STREAM: what is read and written passes the caches by.
template <typename T, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeArgs p) {
  constexpr int N = Vec<T>::N;
  extern __shared__ float2 table[];  // [token][pair]: cosine, sine, times the amplitude
  const int tid = threadIdx.x, pairs = p.rotary / 2;
  const int token0 = (int)(blockIdx.x / p.head_blocks) * p.block_tokens;
  const int head0 = (int)(blockIdx.x % p.head_blocks) * p.block_heads;
  const int tokens = min(p.block_tokens, p.tokens - token0), heads = min(p.block_heads, p.heads - head0);

  for (int i = tid; i < tokens * pairs; i += kThreads) {
    const int t = i / pairs, j = i - t * pairs;
    const int b = p.d_seq.div(token0 + t), s = token0 + t - b * p.seq;
    const double position = p.positions ? (double)p.positions[b * p.positions_stride + s] : (double)(p.first_position + s);
    double turns = position * (p.frequencies[j] * 0.15915494309189533577);  // 1 / 2 pi
    turns -= rint(turns);
    float sine, cosine;
    sincospif((float)(2.0 * turns), &sine, &cosine);
    table[i] = float2{cosine * p.amplitude, (p.inverse ? -sine : sine) * p.amplitude};
  }
  __syncthreads();

  const int items = p.turn_items + p.copy_items, all = tokens * heads * items;
  for (int i = tid; i < all; i += kThreads) {
    const int row = p.d_items.div(i), item = i - row * items;
    const int t = heads == p.block_heads ? p.d_heads.div(row) : row / heads, h = head0 + row - t * heads;
    const int b = p.d_seq.div(token0 + t), s = token0 + t - b * p.seq;
    const T* x = reinterpret_cast<const T*>(p.x) + b * p.xs.batch + h * p.xs.head + s * p.xs.row;
    T* y = reinterpret_cast<T*>(p.y) + b * p.ys.batch + h * p.ys.head + s * p.ys.row;
    if (item >= p.turn_items) {  // past the rotary part
      const int d = p.rotary + (item - p.turn_items) * N;
      float v[N];
      load_vec<T, STREAM>(x + d, p.dim - d, v);
      store_vec<T, STREAM>(y + d, p.dim - d, v);
    } else if constexpr (INTERLEAVED) {
      const int d = item * N, count = p.rotary - d;
      const float2* turn = table + t * pairs + d / 2;
      float v[N], r[N];
      load_vec<T, STREAM>(x + d, count, v);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const float2 c = turn[e < count ? e / 2 : 0];
        r[e] = v[e] * c.x - v[e + 1] * c.y;
        r[e + 1] = v[e + 1] * c.x + v[e] * c.y;
      }
      store_vec<T, STREAM>(y + d, count, r);
    } else {
      const int d = item * N, count = pairs - d;
      const float2* turn = table + t * pairs + d;
      float a[N], b2[N], ra[N], rb[N];
      load_vec<T, STREAM>(x + d, count, a);
      load_vec<T, STREAM>(x + pairs + d, count, b2);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 c = turn[e < count ? e : 0];
        ra[e] = a[e] * c.x - b2[e] * c.y;
        rb[e] = b2[e] * c.x + a[e] * c.y;
      }
      store_vec<T, STREAM>(y + d, count, ra);
      store_vec<T, STREAM>(y + pairs + d, count, rb);
    }
  }
}

template <typename T>
hipError_t launch(const RopeArgs& p, bool interleaved, unsigned blocks, hipStream_t stream) {
  const size_t lds = (size_t)p.block_tokens * (p.rotary / 2) * sizeof(float2);
  // (tensors that the 256 MB of the last cache hold are found there by what comes next: 25 MB in fp32 8.0 us without the hint, 8.8 with it)
  const bool far = (long long)p.tokens * p.heads * p.dim * (int)sizeof(T) > kFarBytes;
  if (interleaved)
    hipLaunchKernelGGL((far ? rope_kernel<T, true, true> : rope_kernel<T, true, false>), dim3(blocks), dim3(kThreads), lds, stream, p);
  else
    hipLaunchKernelGGL((far ? rope_kernel<T, false, true> : rope_kernel<T, false, false>), dim3(blocks), dim3(kThreads), lds, stream, p);
  return hipGetLastError();
}

}  // namespace

extern "C" {

hidet_status_t hidet_rope(int32_t dtype, int64_t batch, int64_t heads, int64_t seq, int64_t head_dim, int64_t rotary_dim,
                          const hidet_heads_t* x, const hidet_heads_t* y, const double* frequencies, const int32_t* positions,
                          int64_t positions_stride, int64_t first_position, int32_t interleaved, int32_t inverse, float amplitude,
                          void* stream) {
  if (dtype < 0 || dtype > 2) return HIDET_ERR_INVALID_ARG;
  if (batch < 0 || heads < 0 || seq < 0 || head_dim <= 0 || rotary_dim <= 0 || rotary_dim > head_dim || rotary_dim % 2 != 0 ||
      positions_stride < 0 || interleaved < 0 || interleaved > 1 || inverse < 0 || inverse > 1)
    return HIDET_ERR_INVALID_ARG;
  if (batch == 0 || heads == 0 || seq == 0) return HIDET_OK;
  if (!x || !y || !frequencies) return HIDET_ERR_INVALID_ARG;
  if (head_dim > 4096 || batch >= kMaxRows || heads >= (1LL << 20) || seq >= kMaxRows || batch * seq >= kMaxRows) return HIDET_ERR_UNSUPPORTED;
  if (first_position < -(1LL << 31) || first_position > (1LL << 31)) return HIDET_ERR_UNSUPPORTED;
  if (positions && batch > 1 && positions_stride > kMaxSpan / batch) return HIDET_ERR_UNSUPPORTED;
  const size_t es = dtype == HIDET_F32 ? 4 : 2;
  if (hidet_status_t st = check_heads(x, batch, heads, seq, head_dim, false); st != HIDET_OK) return st;
  if (hidet_status_t st = check_heads(y, batch, heads, seq, head_dim, true); st != HIDET_OK) return st;
  if (!is_aligned(x->data, es) || !is_aligned(y->data, es) || !is_aligned(frequencies, 8) || !is_aligned(positions, 4)) return HIDET_ERR_ALIGNMENT;
  const bool in_place = x->data == y->data;
  if (in_place)  // (every element is written where it was read, and what is not turned is left)
    if ((batch > 1 && x->stride_batch != y->stride_batch) || (heads > 1 && x->stride_head != y->stride_head) || (seq > 1 && x->stride_row != y->stride_row))
      return HIDET_ERR_INVALID_ARG;
  RopeArgs p{};
  p.x = x->data;
  p.y = y->data;
  p.xs = strides_of(x);
  p.ys = strides_of(y);
  p.frequencies = frequencies;
  p.positions = positions;
  p.positions_stride = positions_stride;
  p.first_position = first_position;
  p.heads = (int)heads;
  p.seq = (int)seq;
  p.dim = (int)head_dim;
  p.rotary = (int)rotary_dim;
  p.tokens = (int)(batch * seq);
  const int vec = 16 / (int)es, pairs = p.rotary / 2;
  p.turn_items = ((interleaved ? p.rotary : pairs) + vec - 1) / vec;
  p.copy_items = in_place ? 0 : (p.dim - p.rotary + vec - 1) / vec;
  p.inverse = inverse;
  p.amplitude = amplitude;
  // A chunk or two a thread: the workgroups that a compute unit holds hide each other's latencies, and there are many rounds of them, so
  // that the last one's gaps are short (16384 tokens of 40 heads of 128 dimensions in bf16: 57 us; 68 with 4 chunks a thread, 73 with 8,
  // 71 with two chunks of a thread in flight at once, whose registers leave room for fewer workgroups).  Fewer tokens, then fewer
  // heads, where that leaves compute units without work.
  const long long items = p.turn_items + p.copy_items, per_token = items * heads;
  long long block_tokens = std::max(1LL, 512 / per_token);
  block_tokens = std::min(block_tokens, std::max(1LL, (long long)p.tokens / 1024));
  block_tokens = std::min(block_tokens, (long long)kTableBytes / (pairs * 8));
  const long long token_blocks = (p.tokens + block_tokens - 1) / block_tokens;
  long long block_heads = heads;
  if (token_blocks < 1024) {
    const long long least = std::max(1LL, kThreads / items);  // a chunk for every thread
    block_heads = std::min<long long>(heads, std::max(least, (heads * token_blocks + 1023) / 1024));
  }
  p.block_tokens = (int)block_tokens;
  p.block_heads = (int)block_heads;
  p.head_blocks = (int)((heads + block_heads - 1) / block_heads);
  const long long blocks = token_blocks * p.head_blocks;
  if (blocks > kMaxBlocks || block_tokens * block_heads * items >= (1LL << 31)) return HIDET_ERR_UNSUPPORTED;
  p.d_seq = make_fastdiv(seq);
  p.d_items = make_fastdiv(items);
  p.d_heads = make_fastdiv(block_heads);
  const hipStream_t s = (hipStream_t)stream;
  const hipError_t e = dtype == HIDET_F32   ? launch<float>(p, interleaved, (unsigned)blocks, s)
                       : dtype == HIDET_F16 ? launch<f16>(p, interleaved, (unsigned)blocks, s)
                                            : launch<bf16>(p, interleaved, (unsigned)blocks, s);
  return e == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

hidet_status_t hidet_rope_frequencies(int64_t rotary_dim, double base, int32_t scaling, double factor, double low_turns,
                                      double high_turns, double original_length, double* frequencies) {
  if (rotary_dim <= 0 || rotary_dim % 2 != 0 || !(base > 0) || scaling < 0 || scaling > 3 || !frequencies) return HIDET_ERR_INVALID_ARG;
  if (scaling != HIDET_ROPE_PLAIN && !(factor > 0)) return HIDET_ERR_INVALID_ARG;
  if (scaling == HIDET_ROPE_BASE && rotary_dim < 4) return HIDET_ERR_INVALID_ARG;
  if (scaling == HIDET_ROPE_BANDS && !(low_turns < high_turns && original_length > 0)) return HIDET_ERR_INVALID_ARG;
  if (scaling == HIDET_ROPE_BASE) base *= pow(factor, (double)rotary_dim / (double)(rotary_dim - 2));
  for (int64_t j = 0; j < rotary_dim / 2; ++j) {
    double f = pow(base, -2.0 * (double)j / (double)rotary_dim);
    if (scaling == HIDET_ROPE_LINEAR) f /= factor;
    if (scaling == HIDET_ROPE_BANDS) {
      const double turns = original_length * f / 6.283185307179586477;
      const double keep = std::min(1.0, std::max(0.0, (turns - low_turns) / (high_turns - low_turns)));
      f = keep * f + (1.0 - keep) * f / factor;
    }
    frequencies[j] = f;
  }
  return HIDET_OK;
}

}  // extern "C"
