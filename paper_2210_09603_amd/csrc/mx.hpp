// Matrices whose blocks of 32 share a power of two: the formats, their conversions, and the checks of what a caller describes.
//
// value = element * 2^(code - 127).  The code follows from the largest magnitude m of a block alone: floor(log2 m) is the exponent field of
// m, so that code = field - emax, 0 at least, where 2^emax is the largest power of two of the format.  Elements are x * 2^(127 - code), an
// exact product (what falls below the numbers of fp32 there is far below half a step of any format), cut to the largest value and
// rounded by the conversion instructions, which round to nearest even (compared with the definition for every kind of tie and both
// neighbours of it).  A NaN would be lost in a maximum of floats: magnitudes are compared as whole numbers, where it is the largest.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hidet_mi355x.h"
#include "types.hpp"

namespace hidet {
namespace mx {

constexpr int kBlock = 32;
constexpr long long kMaxSide = 1LL << 29;          // rows and columns of a matrix
constexpr long long kMaxSpan = 1LL << 47;          // elements that a matrix spans
constexpr long long kMaxValueStride = 1LL << 23;   // bytes: 256 rows are reached by 32-bit offsets
constexpr long long kFarBytes = 128LL << 20;       // matrices of more are streamed past the caches
constexpr long long kMaxScaleStride = 1LL << 29;   // bytes: 8 blocks likewise

inline bool is_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline long long blocks_of(long long cols) { return (cols + kBlock - 1) / kBlock; }
inline int block_bytes(int format) { return format == HIDET_MX_E2M1 ? 16 : 32; }
inline size_t size_of(int dtype) { return dtype == HIDET_F32 ? 4 : 2; }

// a row-major matrix of `rows` rows that lie ld elements apart
inline hidet_status_t check_rows(const void* data, int dtype, long long rows, long long cols, long long ld) {
  if (!data || ld < cols) return HIDET_ERR_INVALID_ARG;
  if (ld > kMaxSpan || (rows > 1 && ld > kMaxSpan / rows)) return HIDET_ERR_UNSUPPORTED;
  return is_aligned(data, size_of(dtype)) ? HIDET_OK : HIDET_ERR_ALIGNMENT;
}
inline hidet_status_t check_mx(const hidet_mx_t* m, long long rows, long long cols) {
  if (!m || m->struct_size != sizeof(hidet_mx_t) || m->format < 0 || m->format > HIDET_MX_E2M1) return HIDET_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return HIDET_OK;
  if (!m->values || !m->scales || m->stride_values < 0 || m->stride_scales < 0) return HIDET_ERR_INVALID_ARG;
  if (!is_aligned(m->values, 16) || m->stride_values % 16 != 0 || !is_aligned(m->scales, 4) || m->stride_scales % 4 != 0)
    return HIDET_ERR_ALIGNMENT;
  if (m->stride_values >= kMaxValueStride || m->stride_scales >= kMaxScaleStride) return HIDET_ERR_UNSUPPORTED;
  // (of one row, and of one block, the distance does not matter)
  if (rows > 1 && m->stride_values < blocks_of(cols) * block_bytes(m->format)) return HIDET_ERR_INVALID_ARG;
  if (cols > kBlock && m->stride_scales < (rows + 3) / 4 * 4) return HIDET_ERR_INVALID_ARG;
  return HIDET_OK;
}

#if defined(__HIPCC__)
typedef float f32x2 __attribute__((ext_vector_type(2)));

__host__ __device__ constexpr int largest_power(int format) { return format == HIDET_MX_E4M3 ? 8 : format == HIDET_MX_E5M2 ? 15 : 2; }
__host__ __device__ constexpr float largest_value(int format) { return format == HIDET_MX_E4M3 ? 448.0f : format == HIDET_MX_E5M2 ? 57344.0f : 6.0f; }

__device__ __forceinline__ unsigned magnitude(float v) { return __builtin_bit_cast(unsigned, v) & 0x7fffffffu; }
// from the largest magnitude of a block; 255 where it is no finite number
__device__ __forceinline__ int scale_code(unsigned largest, int format) {
  const int field = (int)(largest >> 23);
  return field == 255 ? 255 : max(field - largest_power(format), 0);
}
// 2^(127 - code); 0 for a block without finite scale, whose elements are 0
__device__ __forceinline__ float scale_inverse(int code) { return __builtin_bit_cast(float, code == 255 ? 0u : (unsigned)(254 - code) << 23); }
__device__ __forceinline__ float scale_value(int code) {
  return __builtin_bit_cast(float, code == 0 ? 0x00400000u : code == 255 ? 0x7fc00000u : (unsigned)code << 23);
}

// N (4 or 8) values of a block as elements of the format, first in the lowest bits: N / 4 words of 8 bits, one of 4
template <int N>
__device__ __forceinline__ void encode(const float (&v)[N], float inverse, int format, unsigned (&out)[N / 4]) {
  static_assert(N == 4 || N == 8, "a chunk of 16 bytes");
  float q[N];
  const float top = largest_value(format);
#pragma unroll
  for (int w = 0; w < N / 4; ++w) out[w] = 0;
  if (inverse == 0.0f) return;  // (no finite scale)
#pragma unroll
  for (int e = 0; e < N; ++e) q[e] = __builtin_amdgcn_fmed3f(v[e] * inverse, -top, top);
  if (format == HIDET_MX_E4M3) {
#pragma unroll
    for (int w = 0; w < N / 4; ++w) {
      int o = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * w], q[4 * w + 1], 0, false);
      out[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * w + 2], q[4 * w + 3], o, true);
    }
  } else if (format == HIDET_MX_E5M2) {
#pragma unroll
    for (int w = 0; w < N / 4; ++w) {
      int o = __builtin_amdgcn_cvt_pk_bf8_f32(q[4 * w], q[4 * w + 1], 0, false);
      out[w] = (unsigned)__builtin_amdgcn_cvt_pk_bf8_f32(q[4 * w + 2], q[4 * w + 3], o, true);
    }
  } else {
    unsigned o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, q[0], q[1], 1.0f, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, q[2], q[3], 1.0f, 1);
    if constexpr (N == 8) {
      o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, q[4], q[5], 1.0f, 2);
      o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, q[6], q[7], 1.0f, 3);
    }
    out[0] = o;
  }
}
// the numbers of 8 elements
__device__ __forceinline__ void decode(const unsigned (&in)[2], int format, float (&v)[8]) {
  if (format == HIDET_MX_E2M1) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.0f, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.0f, 3);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
    return;
  }
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const f32x2 a = format == HIDET_MX_E4M3 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)in[w], false) : __builtin_amdgcn_cvt_pk_f32_bf8((int)in[w], false);
    const f32x2 b = format == HIDET_MX_E4M3 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)in[w], true) : __builtin_amdgcn_cvt_pk_f32_bf8((int)in[w], true);
    v[4 * w] = a[0], v[4 * w + 1] = a[1], v[4 * w + 2] = b[0], v[4 * w + 3] = b[1];
  }
}

// ---- rows in chunks of 16 bytes, at element alignment ---------------------------------------------------------------------
template <typename T>
struct Chunk {
  static constexpr int N = 16 / (int)sizeof(T);
  struct __attribute__((packed, aligned(sizeof(T)))) Raw {
    u32x4 v;
  };
  typedef u32x4 Streamed __attribute__((aligned(2)));  // (the same, for an access with a hint)
};
// STREAM: past the caches
template <bool STREAM, typename W>
__device__ __forceinline__ W load_word(const W* at) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load(at);
  else
    return *at;
}
template <bool STREAM, typename W>
__device__ __forceinline__ void store_word(W* at, W v) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, at);
  else
    *at = v;
}
// `left` elements are there, any number: the others are 0.  STREAM: passes the caches by.
template <typename T, bool STREAM = false>
__device__ __forceinline__ u32x4 load_chunk(const T* at, int left) {
  constexpr int N = Chunk<T>::N;
  if (left >= N) {
    if constexpr (STREAM)
      return __builtin_nontemporal_load(reinterpret_cast<const typename Chunk<T>::Streamed*>(at));
    else
      return reinterpret_cast<const typename Chunk<T>::Raw*>(at)->v;
  }
  T t[N];
#pragma unroll
  for (int e = 0; e < N; ++e) t[e] = e < left ? at[e] : T(0.0f);
  u32x4 raw;
  __builtin_memcpy(&raw, t, 16);
  return raw;
}
template <typename T, bool STREAM = false>
__device__ __forceinline__ void store_chunk(T* at, int left, u32x4 raw) {
  constexpr int N = Chunk<T>::N;
  if (left >= N) {
    if constexpr (STREAM)
      __builtin_nontemporal_store(raw, reinterpret_cast<typename Chunk<T>::Streamed*>(at));
    else
      reinterpret_cast<typename Chunk<T>::Raw*>(at)->v = raw;
    return;
  }
  T t[N];
  __builtin_memcpy(t, &raw, 16);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < left) at[e] = t[e];
}
template <typename T>
__device__ __forceinline__ void unpack(u32x4 raw, float (&v)[Chunk<T>::N]) {
  T t[Chunk<T>::N];
  __builtin_memcpy(t, &raw, 16);
#pragma unroll
  for (int e = 0; e < Chunk<T>::N; ++e) v[e] = to_f32(t[e]);
}
template <typename T>
__device__ __forceinline__ u32x4 pack(const float (&v)[Chunk<T>::N]) {
  T t[Chunk<T>::N];
#pragma unroll
  for (int e = 0; e < Chunk<T>::N; ++e) t[e] = from_f32<T>(v[e]);
  u32x4 raw;
  __builtin_memcpy(&raw, t, 16);
  return raw;
}
// Magnitudes as whole numbers, two of a 16-bit type in a word: they are ordered as the numbers are, infinity and NaN above.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned larger_pair(unsigned a, unsigned b) {
  return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b & 0x7fff7fffu)));
}
// The number that 16 bits of T are, as the bits of its magnitude in fp32.
template <typename T>
__device__ __forceinline__ unsigned widened(unsigned bits) {
  return magnitude(to_f32(__builtin_bit_cast(T, (unsigned short)bits)));
}
// The largest magnitude of a chunk
template <typename T>
__device__ __forceinline__ unsigned largest_of_chunk(u32x4 raw) {
  if constexpr (sizeof(T) == 4) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, raw[i] & 0x7fffffffu);
    return m;
  } else {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = larger_pair(m, raw[i]);
    return widened<T>(max(m & 0xffffu, m >> 16));
  }
}
template <int N>
__device__ __forceinline__ unsigned largest_of(const float (&v)[N]) {
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) m = max(m, magnitude(v[e]));
  return m;
}
// The same of a block, from those of the 32 / N consecutive lanes that hold it.
template <int N>
__device__ __forceinline__ unsigned largest_of_block(unsigned m) {
#pragma unroll
  for (int d = 1; d < kBlock / N; d <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, d));
  return m;
}
// Encodes and stores N values of which the first has index `at` in its row of values; the block's lanes hold the same code.
template <int N, bool STREAM = false>
__device__ __forceinline__ void store_elements(unsigned char* row, int at, int format, const float (&v)[N], int code) {
  unsigned words[N / 4];
  encode<N>(v, scale_inverse(code), format, words);
  if (format == HIDET_MX_E2M1) {
    if constexpr (N == 8)
      store_word<STREAM>(reinterpret_cast<unsigned*>(row + at / 2), words[0]);
    else
      store_word<STREAM>(reinterpret_cast<unsigned short*>(row + at / 2), (unsigned short)words[0]);
  } else {
    if constexpr (N == 8)
      store_word<STREAM>(reinterpret_cast<u32x2*>(row + at), u32x2{words[0], words[1]});
    else
      store_word<STREAM>(reinterpret_cast<unsigned*>(row + at), words[0]);
  }
}
#endif

}  // namespace mx
}  // namespace hidet
