// Fused attention over dense keys: entry points, and the ranges that document, prefix and window masks come to.
#include "attention_host.hpp"

using namespace hidet;
using namespace hidet::attn;

namespace hidet {
namespace attn {

// Rows beyond 32 run in tiles of 128.  Splits: as many as give every compute unit its workgroups, as long as each keeps some
// tiles of keys.
Cut cut_work(long long entries, long long rows, long long keys, int dp, long long room) {
  Cut c;
  c.stream = rows <= 32;
  const long long tile = c.stream ? 32 : 128;
  c.row_tiles = (int)((rows + tile - 1) / tile);
  const long long blocks = entries * c.row_tiles, wanted = 512;
  const long long least = c.stream ? 2 * kStreamWaves * kStreamKeys : 4 * kTileKeys;  // keys of a split
  long long splits = blocks >= wanted ? 1 : std::min((wanted + blocks - 1) / blocks, (keys + least - 1) / least);
  splits = std::min(splits, room / split_bytes(entries, rows, dp));
  c.splits = (int)std::max(1LL, splits);
  return c;
}

namespace {

// What a query may see of its document, from the run of equal document numbers around it.  One workgroup a batch entry walks over
// its positions: every thread owns a contiguous piece, knows the runs within it, and gets the start of its first run from the
// pieces before it and the end of its last run from those behind it (maxima and minima over the 1024 pieces in LDS).
constexpr int kRangeThreads = 1024;
__global__ __launch_bounds__(kRangeThreads) void ranges_kernel(const int* documents, const int* prefix, int* ranges, int seq_q, int seq_k,
                                                               int causal, int window) {
  __shared__ int starts[kRangeThreads], ends[kRangeThreads];
  const int tid = threadIdx.x, b = blockIdx.x;
  const int piece = (seq_k + kRangeThreads - 1) / kRangeThreads;
  const int first = min(tid * piece, seq_k), last = min(first + piece, seq_k);
  const int* doc = documents ? documents + (long long)b * seq_k : nullptr;
  const int skipped = seq_k - seq_q;
  int* out = ranges + (long long)b * seq_q * 2;
  const int pre = prefix ? max(prefix[b], 0) : 0;
  auto put = [&](int at, int start, int end, int number) {
    const int i = at - skipped;
    if (i < 0) return;
    int lo = start, hi = end;
    if (causal) {
      hi = min(hi, at + 1);
      if (pre) hi = max(hi, min(end, pre < end - start ? start + pre : end));
    }
    if (window) {
      lo = max(lo, at - window + 1);
      if (!causal) hi = window < hi - at ? at + window : hi;
    }
    if (number < 0) lo = hi = 0;
    out[2 * i] = lo;
    out[2 * i + 1] = hi;
  };
  if (doc) {
    // the last position in the piece that begins a run, the first that ends one (the position behind it)
    int start = -1, end = 0x7fffffff;
    for (int at = first; at < last; ++at)
      if (at == 0 || doc[at] != doc[at - 1]) {
        start = at;
        if (end == 0x7fffffff && at > first) end = at;
      }
    if (first < last && end == 0x7fffffff && (last == seq_k || doc[last] != doc[last - 1])) end = last;
    starts[tid] = start;
    ends[tid] = end;
    __syncthreads();
    for (int step = 1; step < kRangeThreads; step <<= 1) {
      const int s = tid >= step ? starts[tid - step] : -1, t = tid + step < kRangeThreads ? ends[tid + step] : 0x7fffffff;
      __syncthreads();
      starts[tid] = max(starts[tid], s);
      ends[tid] = min(ends[tid], t);
      __syncthreads();
    }
    // runs of the piece in turn; `end` is found ahead of the run's positions
    int run = tid > 0 ? starts[tid - 1] : 0;
    for (int at = first; at < last;) {
      const int number = doc[at];
      if (at == 0 || number != doc[at - 1]) run = at;
      int stop = at + 1;
      while (stop < last && doc[stop] == number) ++stop;
      int finish = stop;
      if (stop == last && last < seq_k && doc[last] == number) finish = ends[tid + 1];
      for (; at < stop; ++at) put(at, run, finish, number);
    }
  } else {
    for (int at = tid; at < seq_k; at += kRangeThreads) put(at, 0, seq_k, 0);
  }
  // queries before the first key's position
  for (int i = tid; i < -skipped; i += kRangeThreads) out[2 * i] = out[2 * i + 1] = 0;
}

}  // namespace
}  // namespace attn
}  // namespace hidet

extern "C" {

int64_t hidet_attention_workspace_bytes(int64_t batch, int64_t heads, int64_t kv_heads, int64_t seq_q, int64_t seq_k, int64_t head_dim) {
  if (batch <= 0 || kv_heads <= 0 || heads <= 0 || heads % kv_heads != 0 || seq_q <= 0 || seq_k <= 0 || head_dim <= 0 || head_dim > 128) return 0;
  const long long group = heads / kv_heads;
  if (group > kMaxRows || seq_q >= kMaxRows || seq_q * group >= kMaxRows || batch > kMaxBlocks || kv_heads > kMaxBlocks) return 0;
  const int dp = padded_dim(head_dim);
  const Cut c = cut_work(batch * kv_heads, seq_q * group, seq_k, dp, 1LL << 62);
  return c.splits > 1 ? c.splits * split_bytes(batch * kv_heads, seq_q * group, dp) : 0;
}

hidet_status_t hidet_attention(int32_t dtype, int64_t batch, int64_t heads, int64_t kv_heads, int64_t seq_q, int64_t seq_k,
                               int64_t head_dim, const hidet_heads_t* q, const hidet_heads_t* k, const hidet_heads_t* v,
                               const hidet_heads_t* out, float* lse, const hidet_attention_options_t* options, void* workspace,
                               int64_t workspace_bytes, void* stream) {
  if (dtype < 0 || dtype > 2) return HIDET_ERR_INVALID_ARG;
  if (dtype == HIDET_F32) return HIDET_ERR_UNSUPPORTED;
  if (batch < 0 || heads < 0 || kv_heads < 0 || seq_q < 0 || seq_k < 0 || head_dim <= 0 || workspace_bytes < 0) return HIDET_ERR_INVALID_ARG;
  if (hidet_status_t st = check_options(options); st != HIDET_OK) return st;
  if (batch == 0 || heads == 0 || seq_q == 0) return HIDET_OK;
  if (kv_heads == 0 || heads % kv_heads != 0) return HIDET_ERR_INVALID_ARG;
  if (head_dim > 128 || head_dim % 8 != 0) return HIDET_ERR_UNSUPPORTED;
  const long long group = heads / kv_heads;
  if (group >= kMaxRows || seq_q >= kMaxRows || seq_k >= kMaxRows || seq_q * group >= kMaxRows) return HIDET_ERR_UNSUPPORTED;
  if (hidet_status_t st = check_heads(q, batch, heads, seq_q, head_dim, false); st != HIDET_OK) return st;
  if (hidet_status_t st = check_heads(out, batch, heads, seq_q, head_dim, true); st != HIDET_OK) return st;
  if (seq_k > 0)
    for (const hidet_heads_t* t : {k, v}) {
      if (hidet_status_t st = check_heads(t, batch, kv_heads, seq_k, head_dim, false); st != HIDET_OK) return st;
      if (t->stride_row >= kMaxStride) return HIDET_ERR_UNSUPPORTED;
    }
  if (!is_aligned(lse, 4) || !is_aligned(workspace, 16)) return HIDET_ERR_ALIGNMENT;
  if (batch > kMaxBlocks || kv_heads > kMaxBlocks) return HIDET_ERR_UNSUPPORTED;
  Args p{};
  p.q = q->data;
  p.k = seq_k > 0 ? k->data : nullptr;
  p.v = seq_k > 0 ? v->data : nullptr;
  p.out = out->data;
  p.lse = lse;
  p.slopes = options->slopes;
  p.ranges = options->ranges;
  p.part = static_cast<float*>(workspace);
  p.qs = strides_of(q);
  if (seq_k > 0) {
    p.ks = strides_of(k);
    p.vs = strides_of(v);
  }
  p.os = strides_of(out);
  p.d_group = make_fastdiv(group);
  p.batch = (int)batch;
  p.heads = (int)heads;
  p.kv_heads = (int)kv_heads;
  p.group = (int)group;
  p.seq_q = (int)seq_q;
  p.seq_k = (int)seq_k;
  p.dim = (int)head_dim;
  p.causal = options->causal;
  p.window = window_of(options->window);
  p.scale = options->scale;
  p.softcap = options->softcap;
  const Cut c = cut_work(batch * kv_heads, seq_q * group, seq_k, padded_dim(head_dim), workspace ? workspace_bytes : 0);
  if (batch * kv_heads * c.row_tiles > kMaxBlocks) return HIDET_ERR_UNSUPPORTED;
  p.row_tiles = c.row_tiles;
  p.splits = c.splits;
  return dispatch_forward<false>(dtype, is_extra(options), p, c, (hipStream_t)stream) == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

hidet_status_t hidet_attention_ranges(int64_t batch, int64_t seq_q, int64_t seq_k, const int32_t* documents, const int32_t* prefix,
                                      int32_t causal, int64_t window, int32_t* ranges, void* stream) {
  if (batch < 0 || seq_q < 0 || seq_k < 0 || causal < 0 || causal > 1 || window < 0 || (prefix && window)) return HIDET_ERR_INVALID_ARG;
  if (batch == 0 || seq_q == 0) return HIDET_OK;
  if (!ranges) return HIDET_ERR_INVALID_ARG;
  if (seq_q >= kMaxRows || seq_k >= kMaxRows || batch > (1LL << 21)) return HIDET_ERR_UNSUPPORTED;
  if (!is_aligned(documents, 4) || !is_aligned(prefix, 4) || !is_aligned(ranges, 4)) return HIDET_ERR_ALIGNMENT;
  hipLaunchKernelGGL(ranges_kernel, dim3((unsigned)batch), dim3(kRangeThreads), 0, (hipStream_t)stream, documents, prefix, ranges, (int)seq_q,
                     (int)seq_k, causal, window_of(window));
  return hipGetLastError() == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

}  // extern "C"
