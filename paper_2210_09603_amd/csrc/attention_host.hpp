// Host side of the attention entry points: checks of what a caller describes, and how work is cut.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/hidet_mi355x.h"
#include "attention.hpp"

namespace hidet {
namespace attn {

constexpr long long kMaxRows = 1LL << 29;    // of a kv head's queries, and of keys: positions and their differences stay in 32 bits
constexpr long long kMaxSpan = 1LL << 47;    // elements that a tensor spans
constexpr long long kMaxStride = 1LL << 23;  // between keys: 64 rows of them are reached by a 32-bit byte offset
constexpr long long kMaxBlocks = 1LL << 24;  // of 512 threads: below 2^32 work items

constexpr long long kFarBytes = 128LL << 20;  // tensors beyond are streamed past the caches

inline bool is_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// strides >= 0 and (n0 - 1) * s0 + (n1 - 1) * s1 + (n2 - 1) * s2 + dim < 2^47
inline hidet_status_t check_span(const long long (&n)[3], const long long (&s)[3], long long dim) {
  long long span = dim;
  for (int i = 0; i < 3; ++i) {
    if (s[i] < 0) return HIDET_ERR_INVALID_ARG;
    if (n[i] > 1 && s[i] > kMaxSpan / (n[i] - 1)) return HIDET_ERR_UNSUPPORTED;
    if (n[i] > 1) span += (n[i] - 1) * s[i];
    if (span >= kMaxSpan) return HIDET_ERR_UNSUPPORTED;
  }
  return HIDET_OK;
}
// A tensor of vectors of 2-byte elements; `written`: no two elements of it may be the same.
inline hidet_status_t check_heads(const hidet_heads_t* t, long long batch, long long heads, long long rows, long long dim, bool written) {
  if (!t || !t->data) return HIDET_ERR_INVALID_ARG;
  const long long n[3] = {batch, heads, rows}, s[3] = {t->stride_batch, t->stride_head, t->stride_row};
  if (hidet_status_t st = check_span(n, s, dim); st != HIDET_OK) return st;
  if (written)
    for (int i = 0; i < 3; ++i)
      if (n[i] > 1 && s[i] < dim) return HIDET_ERR_INVALID_ARG;
  return is_aligned(t->data, 2) ? HIDET_OK : HIDET_ERR_ALIGNMENT;
}
inline Strides strides_of(const hidet_heads_t* t) { return Strides{t->stride_batch, t->stride_head, t->stride_row}; }

inline hidet_status_t check_options(const hidet_attention_options_t* o) {
  if (!o || o->struct_size != sizeof(hidet_attention_options_t)) return HIDET_ERR_INVALID_ARG;
  if (!std::isfinite(o->scale) || !std::isfinite(o->softcap) || o->softcap < 0 || o->window < 0 || o->causal < 0 || o->causal > 1)
    return HIDET_ERR_INVALID_ARG;
  if (o->ranges && (o->causal || o->window)) return HIDET_ERR_INVALID_ARG;
  // (factors of a product, as Score takes them)
  const float factor = 2.0f * kLog2e * o->scale;
  if (!std::isfinite(factor) || (o->softcap > 0 && !std::isfinite(factor / o->softcap))) return HIDET_ERR_UNSUPPORTED;
  if (!is_aligned(o->slopes, 4) || !is_aligned(o->ranges, 4)) return HIDET_ERR_ALIGNMENT;
  return HIDET_OK;
}
// (a window of 2^30 hides nothing of 2^29 positions)
inline int window_of(long long window) { return window >= (1LL << 30) ? 0 : (int)window; }
// (scores that are no positive multiple of the products take the form with a score of their own: a slope of 0 where there is none)
inline int form_of(const hidet_attention_options_t* o) {
  if (o->softcap > kWideCap) return FORM_WIDE;
  return (o->softcap > 0 ? FORM_CAP : 0) | (o->slopes || (o->softcap == 0 && !(o->scale > 0)) ? FORM_BIAS : 0);
}

// How the work of `entries` (batch entries x kv heads) of `rows` rows each over up to `keys` keys is cut.
struct Cut {
  bool stream;  // the kernel of few rows
  bool pairs;   // that of many with two wavefronts for 32 rows
  int row_tiles, splits, share;
};
// What cut_work and its like may be asked: with 2^24 entries of 2^29 rows the bytes of a partial result, 520 a row at most, stay
// below 2^63.  (More entries are more workgroups than a launch has.)
inline bool fits_cut(long long outer, long long kv_heads, long long rows, long long keys) {
  return outer <= kMaxBlocks && kv_heads <= kMaxBlocks && outer * kv_heads <= kMaxBlocks && rows < kMaxRows && keys < (1LL << 31);
}
inline long long split_bytes(long long entries, long long rows, int dp) { return entries * rows * (dp + 2) * 4; }
Cut cut_work(long long entries, long long rows, long long keys, int dp, long long room, bool ragged);

inline int padded_dim(long long dim) { return dim <= 64 ? 64 : 128; }

template <typename T, int DP, bool PAGED, int FORM>
hipError_t launch_forward(const Args& p, const Cut& c, hipStream_t stream) {
  const long long blocks = (long long)p.batch * p.kv_heads * c.row_tiles * c.splits;
  if constexpr (PAGED)
    if (p.flat) {
      hipLaunchKernelGGL((flat_kernel<T, DP, FORM>), dim3((unsigned)(p.flat * p.kv_heads)), dim3(64 * kStreamWaves), 0, stream, p);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      hipLaunchKernelGGL((join_flat_kernel<T, DP>), dim3((unsigned)(p.batch * p.kv_heads * p.seq_q * p.group)), dim3(256), 0, stream, p);
      return hipGetLastError();
    }
  if (c.stream)
    hipLaunchKernelGGL((stream_kernel<T, DP, PAGED, FORM>), dim3((unsigned)blocks), dim3(64 * kStreamWaves), 0, stream, p);
  else if (!PAGED && c.pairs)
    hipLaunchKernelGGL((tile_kernel<T, DP, PAGED, FORM, PAGED ? 1 : 2>), dim3((unsigned)blocks), dim3(512), 0, stream, p);
  else
    hipLaunchKernelGGL((tile_kernel<T, DP, PAGED, FORM, 1>), dim3((unsigned)blocks), dim3(256), 0, stream, p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || c.splits == 1) return e;
  const long long rows = (long long)p.batch * p.kv_heads * p.seq_q * p.group;
  if (c.splits > 16)
    hipLaunchKernelGGL((join_many_kernel<T, DP, PAGED>), dim3((unsigned)rows), dim3(256), 0, stream, p);
  else
    hipLaunchKernelGGL((join_kernel<T, DP, PAGED>), dim3((unsigned)((rows + 1024 / DP - 1) / (1024 / DP))), dim3(256), 0, stream, p);
  return hipGetLastError();
}
template <typename T, int DP, bool PAGED>
hipError_t dispatch_form(int form, const Args& p, const Cut& c, hipStream_t stream) {
  switch (form) {
    case FORM_PLAIN: return launch_forward<T, DP, PAGED, FORM_PLAIN>(p, c, stream);
    case FORM_BIAS: return launch_forward<T, DP, PAGED, FORM_BIAS>(p, c, stream);
    case FORM_CAP: return launch_forward<T, DP, PAGED, FORM_CAP>(p, c, stream);
    case FORM_WIDE: return launch_forward<T, DP, PAGED, FORM_WIDE>(p, c, stream);
    default: return launch_forward<T, DP, PAGED, FORM_CAP | FORM_BIAS>(p, c, stream);
  }
}
template <bool PAGED>
hipError_t dispatch_forward(int dtype, int form, const Args& p, const Cut& c, hipStream_t stream) {
  const bool wide = padded_dim(p.dim) == 128;
  if (dtype == HIDET_F16) return wide ? dispatch_form<f16, 128, PAGED>(form, p, c, stream) : dispatch_form<f16, 64, PAGED>(form, p, c, stream);
  return wide ? dispatch_form<bf16, 128, PAGED>(form, p, c, stream) : dispatch_form<bf16, 64, PAGED>(form, p, c, stream);
}

}  // namespace attn
}  // namespace hidet
