// A paged cache of keys and values: new tokens into its pages, and the attention of a ragged batch's newest tokens over them.
#include "attention_host.hpp"

using namespace hidet;
using namespace hidet::attn;

namespace {

// ---- append -----------------------------------------------------------------------------------------------------------
// Memory bound: every element of the new keys and values is read and written once, in 16-byte chunks.  A workgroup takes
// consecutive tokens of the batch, finds where each of them goes (one thread a token), and then streams.
constexpr int kThreads = 256;
constexpr int kMaxTokens = 64;  // of a workgroup

struct AppendArgs {
  const void* from[2];  // keys, values
  void* to[2];
  long long token_stride[2], head_stride[2];              // bytes
  long long page_stride, slot_stride, cache_head_stride;  // bytes
  const int* starts;
  const int* lengths;
  const int* tables;
  long long table_stride;
  int table_width, num_pages, page_size, seqs, tokens, max_new, block_tokens;
  int chunks, per_tensor;  // 16-byte chunks of a vector, of a token's heads
  FastDiv d_page, d_chunks, d_token;
};

struct __attribute__((packed, aligned(2))) Bytes16 {
  u32x4 v;
};
typedef u32x4 Streamed __attribute__((aligned(2)));  // (the same, for a store with a hint)

template <bool STREAM>
__global__ __launch_bounds__(kThreads) void append_kernel(const AppendArgs p) {
  __shared__ long long place[kMaxTokens];  // -1: goes nowhere
  __shared__ int before;
  const int tid = threadIdx.x, token0 = blockIdx.x * p.block_tokens;
  const int tokens = min(p.block_tokens, p.tokens - token0);
  // the sequences that end before the first token
  if (tid == 0) before = 0;
  __syncthreads();
  int ended = 0;
  // (starts are cut to the rows that there are, as the attention cuts them: a sequence's new tokens are those that are left)
  const auto start = [&](int s) { return min(max(p.starts[s], 0), p.tokens); };
  for (int s = tid; s < p.seqs; s += kThreads) ended += start(s + 1) <= token0;
#pragma unroll
  for (int m = 32; m; m >>= 1) ended += __shfl_xor(ended, m);
  if ((tid & 63) == 0 && ended) atomicAdd(&before, ended);  // (whole numbers: the order changes nothing)
  __syncthreads();
  if (tid < tokens) {
    const int token = token0 + tid;
    int s = before;
    while (s < p.seqs && start(s + 1) <= token) ++s;
    long long at = -1;
    if (s < p.seqs) {
      const int first = start(s), count = start(s + 1) - first, i = token - first;
      const long long position = (long long)p.lengths[s] - count + i;
      if (i >= 0 && i < p.max_new && position >= 0 && position < (long long)p.table_width * p.page_size) {
        const int page_at = p.d_page.div((int)position);
        const int page = p.tables[(long long)s * p.table_stride + page_at];
        if ((unsigned)page < (unsigned)p.num_pages)
          at = (long long)page * p.page_stride + (position - (long long)page_at * p.page_size) * p.slot_stride;
      }
    }
    place[tid] = at;
  }
  __syncthreads();
  const int per_token = 2 * p.per_tensor, all = tokens * per_token;
  constexpr int U = 4;
  for (int i0 = tid; i0 < all; i0 += U * kThreads) {
    u32x4 v[U];
    char* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kThreads;
      to[u] = nullptr;
      if (i < all) {
        const int t = p.d_token.div(i);
        int rest = i - t * per_token;
        const int which = rest >= p.per_tensor;
        rest -= which * p.per_tensor;
        const int h = p.d_chunks.div(rest), c = rest - h * p.chunks;
        const long long at = place[t];
        if (at >= 0) {
          const char* from = static_cast<const char*>(p.from[which]) + (long long)(token0 + t) * p.token_stride[which] +
                             h * p.head_stride[which] + c * 16;
          if constexpr (STREAM)
            v[u] = __builtin_nontemporal_load(reinterpret_cast<const Streamed*>(from));
          else
            v[u] = reinterpret_cast<const Bytes16*>(from)->v;
          to[u] = static_cast<char*>(p.to[which]) + at + h * p.cache_head_stride + c * 16;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) {
        if constexpr (STREAM)
          __builtin_nontemporal_store(v[u], reinterpret_cast<Streamed*>(to[u]));
        else
          reinterpret_cast<Bytes16*>(to[u])->v = v[u];
      }
  }
}

hidet_status_t check_cache(const hidet_cache_t* c, size_t& es) {
  if (!c || c->struct_size != sizeof(hidet_cache_t) || c->dtype < 0 || c->dtype > 2) return HIDET_ERR_INVALID_ARG;
  if (c->num_pages < 0 || c->page_size <= 0 || c->heads < 0 || c->head_dim <= 0 || c->table_width < 0 || c->seqs < 0 ||
      c->table_stride < 0)
    return HIDET_ERR_INVALID_ARG;
  es = c->dtype == HIDET_F32 ? 4 : 2;
  if (c->seqs == 0 || c->heads == 0) return HIDET_OK;
  if (c->head_dim % 8 != 0 || c->head_dim > 4096 || c->num_pages >= (1LL << 31) || c->page_size >= (1LL << 31) || c->table_width >= (1LL << 31) ||
      c->seqs > kMaxBlocks || c->heads > kMaxBlocks)
    return HIDET_ERR_UNSUPPORTED;
  if (!c->lengths || (c->table_width > 0 && !c->tables)) return HIDET_ERR_INVALID_ARG;
  if (c->num_pages > 0 && (!c->k || !c->v)) return HIDET_ERR_INVALID_ARG;
  const long long n[3] = {c->num_pages, c->heads, c->page_size}, s[3] = {c->stride_page, c->stride_head, c->stride_slot};
  if (hidet_status_t st = check_span(n, s, c->head_dim); st != HIDET_OK) return st;
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && s[i] < c->head_dim) return HIDET_ERR_INVALID_ARG;
  if (c->table_stride > kMaxSpan / c->seqs || (c->seqs > 1 && c->table_stride < c->table_width)) return HIDET_ERR_INVALID_ARG;
  if (!is_aligned(c->k, es) || !is_aligned(c->v, es) || !is_aligned(c->tables, 4) || !is_aligned(c->lengths, 4)) return HIDET_ERR_ALIGNMENT;
  return HIDET_OK;
}

// what a query may be up to away from the keys that it sees: a window shortens them
long long keys_at_most(const hidet_cache_t* c, long long max_new, long long window) {
  long long keys = std::min<long long>(c->table_width * c->page_size, (1LL << 31) - 1);
  if (window > 0) keys = std::min(keys, std::min<long long>(window, 1LL << 31) + max_new);
  return std::max(keys, 1LL);
}
// The pieces of flat_kernel for a kv head, or 0: splits.  Lengths are known on the device alone, and splits are cut for as many keys as the
// tables have room for: where that is far more than the sequences hold, one split has all of a sequence.  64 sequences, 8 kv heads,
// splits and pieces, us: room for 131000, lengths 100 to 8000 244 and 204, 100 to 163 27.6 and 23.1, one of 120000 beside 63 of 200 546
// and 154; room for 8000 and lengths 100 to 8000 222 and 217; room for 2000 and lengths 100 to 163 12.3 and 23, where splits stay:
// the pieces' second kernel, and the ends of two sequences one after the other.  Fewer than 256 entries (sequences x kv heads) keep splits,
// though pieces would be the faster in most tables that are too wide.  Room for 131000, 8 kv heads, splits and pieces, us: one sequence
// of 2000 tokens 34.6 and 19.5, of 120000 102 and 104; 8 of 2000 34.7 and 27.2, of 8000 57.5 and 55.1; 16 of 8000 126 and 108; 31 of 8000
// 184 and 192, of 100 to 7600 124 and 102.
int flat_pieces(const hidet_cache_t* c, long long rows, long long keys) {
  if (rows > 32 || c->seqs > kFlatSeqs || c->seqs * c->heads < 256 || keys < 16384 || (keys / kStreamKeys + 1) * c->seqs >= (1LL << 30)) return 0;
  if (c->seqs * c->heads * rows > kMaxBlocks) return 0;  // (the second kernel has a workgroup for each)
  return (int)std::max(1LL, 512 / (long long)c->heads);
}
long long flat_bytes(const hidet_cache_t* c, long long rows, int pieces, int dp) {
  return (kFlatSeqs + 4 + 2LL * pieces * c->heads * rows * (dp + 2)) * 4;
}

}  // namespace

extern "C" {

hidet_status_t hidet_cache_append(const hidet_cache_t* cache, int64_t tokens, int64_t max_new, const hidet_heads_t* k,
                                  const hidet_heads_t* v, const int32_t* starts, void* stream) {
  size_t es = 0;
  if (hidet_status_t st = check_cache(cache, es); st != HIDET_OK) return st;
  if (tokens < 0 || max_new < 0) return HIDET_ERR_INVALID_ARG;
  if (tokens == 0 || max_new == 0 || cache->seqs == 0 || cache->heads == 0 || cache->num_pages == 0) return HIDET_OK;
  if (tokens >= kMaxRows) return HIDET_ERR_UNSUPPORTED;
  if (!starts) return HIDET_ERR_INVALID_ARG;
  for (const hidet_heads_t* t : {k, v}) {
    if (hidet_status_t st = check_heads(t, 1, cache->heads, tokens, cache->head_dim, false); st != HIDET_OK) return st;
    if (!is_aligned(t->data, es)) return HIDET_ERR_ALIGNMENT;
  }
  if (!is_aligned(starts, 4)) return HIDET_ERR_ALIGNMENT;
  AppendArgs p{};
  p.from[0] = k->data;
  p.from[1] = v->data;
  p.to[0] = cache->k;
  p.to[1] = cache->v;
  const long long e = (long long)es;
  p.token_stride[0] = k->stride_row * e;
  p.token_stride[1] = v->stride_row * e;
  p.head_stride[0] = k->stride_head * e;
  p.head_stride[1] = v->stride_head * e;
  p.page_stride = cache->stride_page * e;
  p.slot_stride = cache->stride_slot * e;
  p.cache_head_stride = cache->stride_head * e;
  p.starts = starts;
  p.lengths = cache->lengths;
  p.tables = cache->tables;
  p.table_stride = cache->table_stride;
  p.table_width = (int)cache->table_width;
  p.num_pages = (int)cache->num_pages;
  p.page_size = (int)cache->page_size;
  p.seqs = (int)cache->seqs;
  p.tokens = (int)tokens;
  p.max_new = (int)std::min(max_new, (int64_t)kMaxRows);
  const long long chunks = cache->head_dim * e / 16, per_tensor = chunks * cache->heads;
  // 4 chunks a thread, which are in flight together, fewer where that leaves compute units without work (48000 tokens of 12 heads of 64
  // dimensions: 61 us; 84 with 2, where finding the tokens' places weighs more, 63 with 8)
  long long block_tokens = std::min((long long)kMaxTokens, std::max(1LL, 4 * kThreads / (2 * per_tensor)));
  block_tokens = std::min(block_tokens, std::max(1LL, (long long)tokens / 1024));
  const long long blocks = (tokens + block_tokens - 1) / block_tokens;
  if (blocks > kMaxBlocks || block_tokens * 2 * per_tensor >= (1LL << 30)) return HIDET_ERR_UNSUPPORTED;
  p.block_tokens = (int)block_tokens;
  p.chunks = (int)chunks;
  p.per_tensor = (int)per_tensor;
  p.d_page = make_fastdiv(cache->page_size);
  p.d_chunks = make_fastdiv(chunks);
  p.d_token = make_fastdiv(2 * per_tensor);
  const bool far = tokens * 2 * per_tensor * 16 > kFarBytes / 2;
  hipLaunchKernelGGL(far ? append_kernel<true> : append_kernel<false>, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, p);
  return hipGetLastError() == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

int64_t hidet_cache_attention_workspace_bytes(const hidet_cache_t* cache, int64_t heads, int64_t max_new, int64_t window) {
  size_t es = 0;
  if (check_cache(cache, es) != HIDET_OK || cache->seqs == 0 || cache->heads == 0 || heads <= 0 || heads % cache->heads != 0 || max_new <= 0 ||
      cache->head_dim > 128 || window < 0)
    return 0;
  const long long group = heads / cache->heads;
  if (max_new >= kMaxRows || group >= kMaxRows) return 0;
  const int dp = padded_dim(cache->head_dim);
  const long long entries = cache->seqs * cache->heads, rows = max_new * group;
  const long long keys = keys_at_most(cache, max_new, window);
  if (!fits_cut(cache->seqs, cache->heads, rows, keys)) return 0;
  if (const int pieces = flat_pieces(cache, rows, keys)) return flat_bytes(cache, rows, pieces, dp);
  const Cut c = cut_work(entries, rows, keys, dp, 1LL << 62, true);
  return c.splits > 1 ? c.splits * split_bytes(entries, rows, dp) : 0;
}

hidet_status_t hidet_cache_attention(const hidet_cache_t* cache, int64_t heads, int64_t tokens, int64_t max_new, const hidet_heads_t* q,
                                     const hidet_heads_t* out, float* lse, const int32_t* starts,
                                     const hidet_attention_options_t* options, void* workspace, int64_t workspace_bytes, void* stream) {
  size_t es = 0;
  if (hidet_status_t st = check_cache(cache, es); st != HIDET_OK) return st;
  if (hidet_status_t st = check_options(options); st != HIDET_OK) return st;
  if (cache->dtype == HIDET_F32 || cache->head_dim > 128) return HIDET_ERR_UNSUPPORTED;
  if (heads < 0 || tokens < 0 || max_new < 0 || workspace_bytes < 0 || !options->causal) return HIDET_ERR_INVALID_ARG;
  if (heads == 0 || tokens == 0 || max_new == 0 || cache->seqs == 0) return HIDET_OK;
  if (cache->heads == 0 || heads % cache->heads != 0 || !starts) return HIDET_ERR_INVALID_ARG;
  const long long group = heads / cache->heads;
  if (group >= kMaxRows || tokens >= kMaxRows || max_new >= kMaxRows || max_new * group >= kMaxRows) return HIDET_ERR_UNSUPPORTED;
  if (hidet_status_t st = check_heads(q, 1, heads, tokens, cache->head_dim, false); st != HIDET_OK) return st;
  if (hidet_status_t st = check_heads(out, 1, heads, tokens, cache->head_dim, true); st != HIDET_OK) return st;
  if (!is_aligned(lse, 4) || !is_aligned(starts, 4) || !is_aligned(workspace, 16)) return HIDET_ERR_ALIGNMENT;
  Args p{};
  p.q = q->data;
  p.k = cache->k;
  p.v = cache->v;
  p.out = out->data;
  p.lse = lse;
  p.slopes = options->slopes;
  p.part = static_cast<float*>(workspace);
  p.qs = strides_of(q);
  p.os = strides_of(out);
  p.ks = p.vs = Strides{cache->stride_page, cache->stride_head, cache->stride_slot};
  p.starts = starts;
  p.lengths = cache->lengths;
  p.tables = cache->tables;
  p.table_stride = cache->table_stride;
  // (a cache without pages has no keys)
  p.table_width = cache->num_pages > 0 ? (int)cache->table_width : 0;
  p.num_pages = (int)cache->num_pages;
  p.page_size = (int)cache->page_size;
  p.tokens = (int)tokens;
  p.d_page = make_fastdiv(cache->page_size);
  p.d_group = make_fastdiv(group);
  p.batch = (int)cache->seqs;
  p.heads = (int)heads;
  p.kv_heads = (int)cache->heads;
  p.group = (int)group;
  p.seq_q = (int)max_new;
  p.dim = (int)cache->head_dim;
  p.causal = 1;
  p.window = window_of(options->window);
  p.scale = options->scale;
  p.softcap = options->softcap;
  const long long entries = cache->seqs * cache->heads, rows = max_new * group;
  const long long keys = keys_at_most(cache, max_new, options->window);
  if (!fits_cut(cache->seqs, cache->heads, rows, keys)) return HIDET_ERR_UNSUPPORTED;
  const int dp = padded_dim(cache->head_dim), pieces = flat_pieces(cache, rows, keys);
  if (pieces && workspace && workspace_bytes >= flat_bytes(cache, rows, pieces, dp)) p.flat = pieces;
  const Cut c = cut_work(entries, rows, keys, dp, workspace ? workspace_bytes : 0, true);
  if (entries * c.row_tiles > kMaxBlocks) return HIDET_ERR_UNSUPPORTED;
  p.row_tiles = c.row_tiles;
  p.splits = c.splits;
  p.share = c.share;
  return dispatch_forward<true>(cache->dtype, form_of(options), p, c, (hipStream_t)stream) == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

}  // extern "C"
