// Fused attention over dense keys: entry points, and the ranges that document, prefix and window masks come to.
#include "attention_host.hpp"

using namespace hidet;
using namespace hidet::attn;

namespace hidet {
namespace attn {

// Which kernel: up to 32 rows, or little work on keys that more than one wavefront can share, runs in pieces of 32 rows, where 4
// wavefronts share the keys; the rest in tiles of 128 rows.  Microseconds in pieces and in tiles, heads of 64 dimensions with as many
// causal keys as rows: 12 heads of 128 5.8 and 6.1, of 512 8.5 and 11.1, of 1024 17.7 and 16.5; 48 heads of 128 5.9 and 6.1, of 256 8.0 and
// 7.9; one head of 64 rows 5.5 and 4.7.
//
// Splits: one is a fixed number of tiles of keys, so that the sequences of a ragged batch give pieces of equal length.
//   Few rows: 512 workgroups fill the device, which is worth a partial result for 16 tiles of 32 keys (one sequence of 131000 keys, 2 kv
//   heads: 39 us with 16, 40 with 32, 56 with 64); up to 2048 even out a ragged batch, as long as 64 tiles remain (64 sequences of 100 to
//   8000 keys, 8 kv heads: 220 us; 231 with 1024 workgroups, 225 with 4096 of 16 tiles).
//   Tiles of 128 rows: while they are no more than the 8 wavefronts that the device takes at once, they run in pairs of wavefronts (256
//   compute units; two of them each at 64 dimensions, whose tiles are half as large), and in as many splits as leave a compute unit for
//   each (more would be a second round: 210 tiles of 2068 keys 52 us whole, 69 in halves) of at least 4 tiles of 128 keys.  n heads of as
//   many rows as keys, us with plain wavefronts, with pairs, and with pairs and splits: 128 dimensions, 4 heads of 4096 97, 69, 50; 8 of
//   2048 52, 40, 34; 32 of 1024, 256 tiles, 31 and 27; 36 of 1024, 288 tiles, 41 and 51; 64 dimensions, 4 of 4096 59, 45, 33; 12 of 1024
//   18.7, 17.0, 16.9; 12 of 512 13.1 and 12.9.
//   Of a ragged batch's tiles some have no rows: 1024 workgroups of at least 8 tiles of 64 keys (chunks of 4 prompts of 37 to 512 tokens
//   over 4096 keys: 157 us, 192 with 256).
Cut cut_work(long long entries, long long rows, long long keys, int dp, long long room, bool ragged) {
  Cut c;
  const long long pieces = entries * ((rows + 31) / 32);
  c.stream = rows <= 32 || (keys > kTileKeys && pieces <= 256 && pieces * ((keys + 31) / 32) <= 4096);
  const long long tile = c.stream ? 32 : 128;
  c.row_tiles = (int)((rows + tile - 1) / tile);
  const long long blocks = entries * c.row_tiles;
  c.pairs = !c.stream && !ragged && (dp == 64 ? blocks < 512 : blocks <= 256) && keys > kTileKeys;
  const long long tile_keys = c.stream ? kStreamKeys : c.pairs ? 2 * kTileKeys : kTileKeys;
  const long long tiles = std::max(1LL, (keys + tile_keys - 1) / tile_keys);
  const auto wish = [&](long long workgroups, long long least) { return std::min((workgroups + blocks - 1) / blocks, tiles / least); };
  long long splits = c.stream ? std::max(wish(512, 8), wish(2048, 64)) : ragged ? wish(1024, 8) : c.pairs ? std::min(256 / blocks, tiles / 4) : 1;
  splits = std::max(1LL, std::min(splits, room / split_bytes(entries, rows, dp)));
  const long long share = (tiles + splits - 1) / splits;
  c.share = (int)share;
  c.splits = (int)((tiles + share - 1) / share);
  return c;
}

namespace {

// What a query may see of its document: the run of equal document numbers around it.  A workgroup has 1024 positions; it looks for
// the last run that begins before them and the first that ends behind them in the whole row (coalesced, all loads independent: a row
// of 4096 takes the time of one), and within them every thread finds the borders around its position in its wavefront's bit mask, or
// in those of the other wavefronts.
constexpr int kRangeThreads = 1024, kRangeWaves = kRangeThreads / 64;
__global__ __launch_bounds__(kRangeThreads) void ranges_kernel(const int* documents, const int* prefix, int* ranges, int seq_q, int seq_k,
                                                               int causal, int window) {
  __shared__ unsigned long long masks[kRangeWaves + 1];
  __shared__ int outer[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.y;
  const int first = blockIdx.x * kRangeThreads, at = first + tid;
  const int* doc = documents ? documents + (long long)b * seq_k : nullptr;
  const int skipped = seq_k - seq_q;
  int* out = ranges + (long long)b * seq_q * 2;
  int start = 0, end = seq_k, number = 0;
  if (doc) {
    if (tid < 2) outer[tid] = tid ? seq_k : 0;
    __syncthreads();
    const int last = min(first + kRangeThreads, seq_k);
    int before = 0, behind = seq_k;
#pragma unroll 4
    for (int i = tid; i < seq_k; i += kRangeThreads) {
      const bool border = i == 0 || doc[i] != doc[i - 1];  // (a run begins here)
      if (border && i <= first) before = max(before, i);
      if (border && i >= last) behind = min(behind, i);
    }
    if (before > 0) atomicMax(&outer[0], before);  // (whole numbers: the order changes nothing)
    if (behind < seq_k) atomicMin(&outer[1], behind);
    const bool border = at < seq_k && (at == 0 || doc[at] != doc[at - 1]);
    number = at < seq_k ? doc[at] : 0;
    const unsigned long long mask = __ballot(border);
    if (lane == 0) masks[wave] = mask;
    __syncthreads();
    start = outer[0];
    end = outer[1];
    const unsigned long long up_to = mask & (~0ull >> (63 - lane)), beyond = lane < 63 ? mask >> (lane + 1) : 0;
    if (up_to) {
      start = first + wave * 64 + 63 - __builtin_clzll(up_to);
    } else {
      for (int i = wave - 1; i >= 0; --i)
        if (masks[i]) {
          start = first + i * 64 + 63 - __builtin_clzll(masks[i]);
          break;
        }
    }
    if (beyond) {
      end = at + 1 + __builtin_ctzll(beyond);
    } else {
      for (int i = wave + 1; i < kRangeWaves; ++i)
        if (masks[i]) {
          end = first + i * 64 + __builtin_ctzll(masks[i]);
          break;
        }
    }
  }
  if (at < seq_k && at >= skipped) {
    const int pre = prefix ? max(prefix[b], 0) : 0;
    int lo = start, hi = end;
    if (causal) {
      hi = min(hi, at + 1);
      if (pre) hi = max(hi, pre < end - start ? start + pre : end);
    }
    if (window) {
      lo = max(lo, at - window + 1);
      if (!causal && window < hi - at) hi = at + window;
    }
    if (number < 0) lo = hi = 0;
    out[2 * (at - skipped)] = lo;
    out[2 * (at - skipped) + 1] = hi;
  }
  // queries before the first key
  for (int i = at; i < -skipped; i += gridDim.x * kRangeThreads) out[2 * i] = out[2 * i + 1] = 0;
}

}  // namespace
}  // namespace attn
}  // namespace hidet

extern "C" {

int64_t hidet_attention_workspace_bytes(int64_t batch, int64_t heads, int64_t kv_heads, int64_t seq_q, int64_t seq_k, int64_t head_dim) {
  if (batch <= 0 || kv_heads <= 0 || heads <= 0 || heads % kv_heads != 0 || seq_q <= 0 || seq_k <= 0 || head_dim <= 0 || head_dim > 128) return 0;
  const long long group = heads / kv_heads;
  if (group >= kMaxRows || seq_q >= kMaxRows || seq_k >= kMaxRows || !fits_cut(batch, kv_heads, seq_q * group, seq_k)) return 0;
  const int dp = padded_dim(head_dim);
  const Cut c = cut_work(batch * kv_heads, seq_q * group, seq_k, dp, 1LL << 62, false);
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
  if (!fits_cut(batch, kv_heads, seq_q * group, seq_k)) return HIDET_ERR_UNSUPPORTED;
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
  // (a window leaves the 128 rows of a tile no more keys than this)
  const long long keys = options->window > 0 ? std::min<long long>(seq_k, 2LL * std::min<long long>(options->window, kMaxRows) + 128) : seq_k;
  const Cut c = cut_work(batch * kv_heads, seq_q * group, keys, padded_dim(head_dim), workspace ? workspace_bytes : 0, false);
  if (batch * kv_heads * c.row_tiles > kMaxBlocks) return HIDET_ERR_UNSUPPORTED;
  p.row_tiles = c.row_tiles;
  p.splits = c.splits;
  p.share = c.share;
  return dispatch_forward<false>(dtype, form_of(options), p, c, (hipStream_t)stream) == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

hidet_status_t hidet_attention_ranges(int64_t batch, int64_t seq_q, int64_t seq_k, const int32_t* documents, const int32_t* prefix,
                                      int32_t causal, int64_t window, int32_t* ranges, void* stream) {
  if (batch < 0 || seq_q < 0 || seq_k < 0 || causal < 0 || causal > 1 || window < 0 || (prefix && window)) return HIDET_ERR_INVALID_ARG;
  if (batch == 0 || seq_q == 0) return HIDET_OK;
  if (!ranges) return HIDET_ERR_INVALID_ARG;
  if (seq_q >= kMaxRows || seq_k >= kMaxRows || batch >= (1LL << 16) || batch * (seq_k + kRangeThreads) > (1LL << 31)) return HIDET_ERR_UNSUPPORTED;
  if (!is_aligned(documents, 4) || !is_aligned(prefix, 4) || !is_aligned(ranges, 4)) return HIDET_ERR_ALIGNMENT;
  const unsigned pieces = (unsigned)((std::max(seq_k, (int64_t)1) + kRangeThreads - 1) / kRangeThreads);
  hipLaunchKernelGGL(ranges_kernel, dim3(pieces, (unsigned)batch), dim3(kRangeThreads), 0, (hipStream_t)stream, documents, prefix, ranges, (int)seq_q,
                     (int)seq_k, causal, window_of(window));
  return hipGetLastError() == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

}  // extern "C"
