// Fused attention, backward.  With P = exp(x - lse), t the capped score's tanh and D_i = sum_d dout_id out_id,
//
//   dP = dout . V^T     dS = P (dP - D) (1 - t^2)     dQ = scale dS . K     dK = scale dS^T . Q     dV = P^T . dout
//
// P is computed again from the products and the saved lse.  Two kernels, so that every output is summed by one workgroup in a
// fixed order, without atomics: the first walks over the keys of 128 rows (dQ, and D on the way), the second over the rows of
// 128 keys (dK, dV).  Scores are computed in both: 7 products instead of 5, against an fp32 dQ that all key tiles would add to.
// Rows are packed as in the forward pass, so that the heads that share keys are summed into dK and dV by the same loop.
//
// The operands lie so that P and dS never leave their lanes: the first kernel computes S^T and dP^T (lane = query) and multiplies
// K^T by dS^T, the second S and dP (lane = key) and multiplies dout^T by P and Q^T by dS.
//
// P is at most 1 and mostly far below; as an operand it is taken times 2^10, which keeps it out of fp16's subnormals down to
// 2^-24, and divided out at the end.  dS is rounded as it is: its size follows the caller's gradients.
#include "attention_host.hpp"

using namespace hidet;
using namespace hidet::attn;

namespace {

struct BackArgs {
  Args f;  // f.lse: of the forward pass; f.out: its output
  const void* dout;
  void* dq;
  void* dk;
  void* dv;
  Strides dos, dqs, dks, dvs;
  float* delta;   // [batch][heads][seq_q]
  int4* seen;     // [batch][row_groups]: of 32 rows, the first and last + 1 of the keys that any of them sees; that all of them see
  int row_groups;
  int key_tiles;
};

constexpr float kLift = 1024.0f, kLiftBits = 10.0f;

__device__ __forceinline__ float lse_to_base_2(float lse) { return lse == kNoMax ? __builtin_huge_valf() : lse * kLog2e; }

// Rows that come out not finite, again: only what a query sees takes part (see the forward pass).
template <typename T, int DP>
__device__ __forceinline__ void dq_by_definition(const BackArgs& b, const Entry& e, int r, float delta) {
  constexpr int E = DP / 64;
  const Args& p = b.f;
  const int lane = threadIdx.x & 63;
  const Row w = make_row<false>(p, e, r);
  const Score score(p, p.slopes ? p.slopes[w.head] : 0.0f);
  const T* q = reinterpret_cast<const T*>(p.q) + query_offset<false>(p, e, p.qs, w);
  const T* g = reinterpret_cast<const T*>(b.dout) + query_offset<false>(p, e, b.dos, w);
  const T* k = keys_of<T, false>(p, e, p.k, p.ks);
  const T* v = keys_of<T, false>(p, e, p.v, p.vs);
  const float lse = lse_to_base_2(p.lse[lse_offset<false>(p, e, w)]);
  float mq[E], mg[E], acc[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int d = lane * E + i;
    mq[i] = d < p.dim ? to_f32(q[d]) : 0.0f;
    mg[i] = d < p.dim ? to_f32(g[d]) : 0.0f;
    acc[i] = 0.0f;
  }
  for (int j = w.lo; j < w.hi; ++j) {
    float dot = 0.0f, dp = 0.0f, mk[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int d = lane * E + i;
      mk[i] = d < p.dim ? to_f32(k[(long long)j * p.ks.row + d]) : 0.0f;
      const float mv = d < p.dim ? to_f32(v[(long long)j * p.vs.row + d]) : 0.0f;
      dot = __builtin_fmaf(mq[i], mk[i], dot);
      dp = __builtin_fmaf(mg[i], mv, dp);
    }
    dot = wave_sum(dot);
    dp = wave_sum(dp);
    const float prob = exp2_fast(score(dot, w.token + e.shift - j) - lse);
    if (prob == 0.0f) continue;
    float ds = prob * (dp - delta);
    if (p.softcap > 0) {
      const float t = score.tanh_of(dot);
      ds *= 1.0f - t * t;
    }
    bool finite = false;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      acc[i] += ds * mk[i];
      finite |= acc[i] == acc[i];
    }
    if (!__any(finite)) break;
  }
  T* to = reinterpret_cast<T*>(b.dq) + query_offset<false>(p, e, b.dqs, w);
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (lane * E + i < p.dim) to[lane * E + i] = from_f32<T>(acc[i] * p.scale);
}

template <typename T, int DP>
__device__ __forceinline__ void dkv_by_definition(const BackArgs& b, const Entry& e, int j) {
  constexpr int E = DP / 64;
  const Args& p = b.f;
  const int lane = threadIdx.x & 63;
  const T* k = keys_of<T, false>(p, e, p.k, p.ks) + (long long)j * p.ks.row;
  const T* v = keys_of<T, false>(p, e, p.v, p.vs) + (long long)j * p.vs.row;
  float mk[E], mv[E], dk[E], dv[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int d = lane * E + i;
    mk[i] = d < p.dim ? to_f32(k[d]) : 0.0f;
    mv[i] = d < p.dim ? to_f32(v[d]) : 0.0f;
    dk[i] = dv[i] = 0.0f;
  }
  for (int r = 0; r < e.tokens * p.group; ++r) {
    const Row w = make_row<false>(p, e, r);
    if (j < w.lo || j >= w.hi) continue;
    const Score score(p, p.slopes ? p.slopes[w.head] : 0.0f);
    const T* q = reinterpret_cast<const T*>(p.q) + query_offset<false>(p, e, p.qs, w);
    const T* g = reinterpret_cast<const T*>(b.dout) + query_offset<false>(p, e, b.dos, w);
    float dot = 0.0f, dp = 0.0f, mq[E], mg[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int d = lane * E + i;
      mq[i] = d < p.dim ? to_f32(q[d]) : 0.0f;
      mg[i] = d < p.dim ? to_f32(g[d]) : 0.0f;
      dot = __builtin_fmaf(mq[i], mk[i], dot);
      dp = __builtin_fmaf(mg[i], mv[i], dp);
    }
    dot = wave_sum(dot);
    dp = wave_sum(dp);
    const long long at = lse_offset<false>(p, e, w);
    const float prob = exp2_fast(score(dot, w.token + e.shift - j) - lse_to_base_2(p.lse[at]));
    if (prob == 0.0f) continue;
    float ds = prob * (dp - b.delta[at]);
    if (p.softcap > 0) {
      const float t = score.tanh_of(dot);
      ds *= 1.0f - t * t;
    }
    bool finite = false;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      dk[i] += ds * mq[i];
      dv[i] += prob * mg[i];
      finite |= dk[i] == dk[i] || dv[i] == dv[i];
    }
    if (!__any(finite)) break;
  }
  T* to_k = reinterpret_cast<T*>(b.dk) + (long long)e.b * b.dks.batch + (long long)e.kv * b.dks.head + (long long)j * b.dks.row;
  T* to_v = reinterpret_cast<T*>(b.dv) + (long long)e.b * b.dvs.batch + (long long)e.kv * b.dvs.head + (long long)j * b.dvs.row;
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (lane * E + i < p.dim) {
      to_k[lane * E + i] = from_f32<T>(dk[i] * p.scale);
      to_v[lane * E + i] = from_f32<T>(dv[i]);
    }
}

// A transposed accumulator (lane = vector, registers = its dimensions) to the vector's memory, times `by`.
template <typename T, int DT>
__device__ __forceinline__ void store_columns(T* to, const f32x16 (&acc)[DT], int half, int dim, float by) {
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * t + 8 * g + 4 * half;
      T four[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) four[i] = from_f32<T>(acc[t][4 * g + i] * by);
      if (d < dim) __builtin_memcpy(reinterpret_cast<Chunk8*>(to + d), four, 8);
    }
}
template <int DT>
__device__ __forceinline__ bool all_finite(const f32x16 (&acc)[DT]) {
  bool finite = true;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) finite &= __builtin_fabsf(acc[t][i]) < __builtin_huge_valf();
  return finite;
}

// ---- dQ ---------------------------------------------------------------------------------------------------------------
// The forward kernel's walk, with dout and out beside q.
template <typename T, int DP, bool EXTRA>
__global__ __launch_bounds__(256, 2) void dq_kernel(const BackArgs b) {
  constexpr int CPR = DP / 8, STAGE = kTileKeys * CPR * 16, NL = kTileKeys * CPR / 256, RPP = 256 / CPR, KS = DP / 16, DT = DP / 32;
  using Frag = typename Frag8<T>::type;
  __shared__ __attribute__((aligned(16))) unsigned char smem[4 * STAGE];
  __shared__ int bounds[4][2];
  const Args& p = b.f;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int id = xcd_run(blockIdx.x, gridDim.x);
  const int tile = p.row_tiles - 1 - id % p.row_tiles;
  id /= p.row_tiles;
  const Entry e = make_entry<false>(p, id / p.kv_heads, id % p.kv_heads);
  const int rows = e.tokens * p.group, r0 = tile * 128 + wave * 32;

  const Row w = make_row<false>(p, e, min(r0 + (lane & 31), rows - 1));
  const int at = w.token + e.shift;
  const bool sees = w.lo < w.hi;
  const int wave_lo = wave_min(sees ? w.lo : 0x7fffffff), wave_hi = wave_max(w.hi);
  const int full_lo = wave_max(w.lo), full_hi = wave_min(w.hi);
  if (lane == 0) {
    bounds[wave][0] = wave_lo;
    bounds[wave][1] = wave_hi;
    if (e.kv == 0 && r0 < rows) b.seen[(long long)e.b * b.row_groups + (r0 >> 5)] = int4{wave_lo, wave_hi, full_lo, full_hi};
  }
  Frag q[KS], g[KS];
  load_row_frags<T, DP>(reinterpret_cast<const T*>(p.q) + query_offset<false>(p, e, p.qs, w), half, p.dim, q);
  load_row_frags<T, DP>(reinterpret_cast<const T*>(b.dout) + query_offset<false>(p, e, b.dos, w), half, p.dim, g);
  float delta = 0.0f;
  {
    Frag o[KS];
    load_row_frags<T, DP>(reinterpret_cast<const T*>(p.out) + query_offset<false>(p, e, p.os, w), half, p.dim, o);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < 8; ++i) delta = __builtin_fmaf(to_f32(g[ks][i]), to_f32(o[ks][i]), delta);
  }
  delta = sum_of_halves(delta);
  const long long stat = lse_offset<false>(p, e, w);
  const float lse = lse_to_base_2(p.lse[stat]);
  if (half == 0 && r0 + lane < rows) b.delta[stat] = delta;
  const Score score(p, p.slopes ? p.slopes[w.head] : 0.0f);
  if (p.dim < DP)
    for (int i = tid; i < 4 * STAGE / 16; i += 256) reinterpret_cast<u32x4*>(smem)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
  int begin = 0x7fffffff, end = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    begin = min(begin, bounds[i][0]);
    end = max(end, bounds[i][1]);
  }
  begin = __builtin_amdgcn_readfirstlane(begin);
  end = __builtin_amdgcn_readfirstlane(end);
  if (begin >= end) begin = end = 0;
  const int tiles = (end - begin + kTileKeys - 1) / kTileKeys;

  const T* kbase = keys_of<T, false>(p, e, p.k, p.ks);
  const T* vbase = keys_of<T, false>(p, e, p.v, p.vs);
  const int load_row = tid / CPR, load_chunk = (tid % CPR) ^ swz<CPR>(load_row);
  const bool loads = load_chunk * 8 < p.dim;
  const unsigned lds = lds_address(smem) + wave * 1024;
  auto request = [&](int t) {
    const unsigned to = lds + (t & 1) * STAGE;
    const int first = begin + t * kTileKeys, last = end - 1 - first;
    const T* kt = kbase + (long long)first * p.ks.row;
    const T* vt = vbase + (long long)first * p.vs.row;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = min(i * RPP + load_row, last);
      const unsigned ko = ((unsigned)row * (unsigned)p.ks.row + load_chunk * 8) * 2;
      const unsigned vo = ((unsigned)row * (unsigned)p.vs.row + load_chunk * 8) * 2;
      if (loads) {
        DirectLoad::at(kt, ko, to + i * 4096);
        DirectLoad::at(vt, vo, to + 2 * STAGE + i * 4096);
      }
    }
  };
  f32x16 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.0f;
  if (tiles > 0) request(0);
  for (int t = 0; t < tiles; ++t) {
    wait_all_and_meet();
    if (t + 1 < tiles) request(t + 1);
    const int first = begin + t * kTileKeys;
    if (first >= wave_hi || first + kTileKeys <= wave_lo) continue;
    const unsigned char* keys = smem + (t & 1) * STAGE;
    const unsigned char* values = keys + 2 * STAGE;
    const bool masked = first < full_lo || first + kTileKeys > full_hi;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s = mfma_op(row_frag<T, CPR>(keys, lane, c * 32, ks), q[ks], s);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) dp = mfma_op(row_frag<T, CPR>(values, lane, c * 32, ks), g[ks], dp);
      const int base = first + c * 32 + 4 * half;
      Frag ds[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = base + 8 * (r >> 2) + (r & 3);
        float x = EXTRA ? score(s[r], at - j) - lse : __builtin_fmaf(s[r], score.factor, -lse);
        float d = exp2_fast(x) * (dp[r] - delta);
        if (EXTRA && score.cap > 0) {
          const float th = score.tanh_of(s[r]);
          d *= 1.0f - th * th;
        }
        if (masked) d = (unsigned)(j - w.lo) < (unsigned)(w.hi - w.lo) ? d : 0.0f;
        ds[r >> 3][r & 7] = from_f32<T>(d);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = mfma_op(col_frag<T, CPR>(keys, lane, c * 32 + h * 16, d), ds[h], acc[d]);
    }
  }
  const unsigned long long odd = __ballot(!all_finite(acc));
  unsigned again = (unsigned)odd | (unsigned)(odd >> 32);
  if (r0 + (lane & 31) < rows && !((again >> (lane & 31)) & 1))
    store_columns<T, DT>(reinterpret_cast<T*>(b.dq) + query_offset<false>(p, e, b.dqs, w), acc, half, p.dim, p.scale);
  again = __builtin_amdgcn_readfirstlane(again);
  while (again) {
    const int i = __builtin_ctz(again);
    again &= again - 1;
    const float its = __shfl(delta, i);
    if (r0 + i < rows) dq_by_definition<T, DP>(b, e, r0 + i, its);
  }
}

// ---- dK, dV -------------------------------------------------------------------------------------------------------------
// A workgroup of 4 wavefronts keeps 128 keys and values, 32 a wavefront, in registers with their two sums (192 registers at 128
// dimensions) and walks over the rows that see one of them in tiles of 64 rows of q and dout, one tile ahead of it in LDS.
constexpr int kTileRows = 64;

template <typename T, int DP, bool EXTRA>
__global__ __launch_bounds__(256, DP == 64 ? 2 : 1) void dkv_kernel(const BackArgs b) {
  constexpr int CPR = DP / 8, STAGE = kTileRows * CPR * 16, NL = kTileRows * CPR / 256, RPP = 256 / CPR, KS = DP / 16, DT = DP / 32;
  using Frag = typename Frag8<T>::type;
  __shared__ __attribute__((aligned(16))) unsigned char smem[4 * STAGE];  // q of two stages, dout of two
  __shared__ __attribute__((aligned(16))) float row_lse[2][kTileRows], row_delta[2][kTileRows], row_slope[2][kTileRows];
  __shared__ __attribute__((aligned(16))) int row_lo[2][kTileRows], row_count[2][kTileRows], row_at[2][kTileRows];
  __shared__ int4 tile_seen[2][2];
  __shared__ int bounds[4][2];
  const Args& p = b.f;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int id = xcd_run(blockIdx.x, gridDim.x);
  const int tile = id % b.key_tiles;  // (causal: the longest first)
  id /= b.key_tiles;
  const Entry e = make_entry<false>(p, id / p.kv_heads, id % p.kv_heads);
  const int rows = e.tokens * p.group;
  const int block_key = tile * 128, key0 = block_key + wave * 32, key = key0 + (lane & 31);
  const int block_end = min(block_key + 128, e.keys);

  // the first and last groups of 32 rows that see a key of the block
  const int groups = (rows + 31) >> 5;
  const int4* seen = b.seen + (long long)e.b * b.row_groups;
  int from = 0x7fffffff, to = 0;
  for (int i = tid; i < groups; i += 256)
    if (seen[i].x < block_end && seen[i].y > block_key) {
      from = min(from, i);
      to = i + 1;
    }
  from = wave_min(from);
  to = wave_max(to);
  if (lane == 0) {
    bounds[wave][0] = from;
    bounds[wave][1] = to;
  }
  Frag kf[KS], vf[KS];
  const int mine = min(key, e.keys - 1);
  load_row_frags<T, DP>(keys_of<T, false>(p, e, p.k, p.ks) + (long long)mine * p.ks.row, half, p.dim, kf);
  load_row_frags<T, DP>(keys_of<T, false>(p, e, p.v, p.vs) + (long long)mine * p.vs.row, half, p.dim, vf);
  if (p.dim < DP)
    for (int i = tid; i < 4 * STAGE / 16; i += 256) reinterpret_cast<u32x4*>(smem)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    from = min(from, bounds[i][0]);
    to = max(to, bounds[i][1]);
  }
  from = __builtin_amdgcn_readfirstlane(from);
  to = __builtin_amdgcn_readfirstlane(to);
  const int t0 = from < to ? from >> 1 : 0, t1 = from < to ? (to + 1) >> 1 : 0;  // tiles of 64 rows

  const int load_row = tid / CPR, load_chunk = (tid % CPR) ^ swz<CPR>(load_row);
  const bool loads = load_chunk * 8 < p.dim;
  const unsigned lds = lds_address(smem) + wave * 1024;
  auto request = [&](int t) {
    const unsigned dst = lds + (t & 1) * STAGE;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = min(t * kTileRows + i * RPP + load_row, rows - 1);  // (rows past the last: the last again, seen by nobody)
      const int token = p.d_group.div(r), head = e.kv * p.group + (r - token * p.group);
      const T* qr = reinterpret_cast<const T*>(p.q) + (long long)e.b * p.qs.batch + (long long)head * p.qs.head + (long long)token * p.qs.row;
      const T* gr = reinterpret_cast<const T*>(b.dout) + (long long)e.b * b.dos.batch + (long long)head * b.dos.head + (long long)token * b.dos.row;
      if (loads) {
        DirectLoad::at(qr + load_chunk * 8, dst + i * 4096);
        DirectLoad::at(gr + load_chunk * 8, dst + 2 * STAGE + i * 4096);
      }
    }
  };
  // what thread i < 64 knows of row i of a tile
  float next_lse = 0, next_delta = 0, next_slope = 0;
  int next_lo = 0, next_count = 0, next_at = 0;
  int4 next_seen = {0, 0, 0, 0};
  auto look_up = [&](int t) {
    if (tid < kTileRows) {
      const int r = t * kTileRows + tid;
      const Row w = make_row<false>(p, e, min(r, rows - 1));
      const long long stat = lse_offset<false>(p, e, w);
      next_lse = lse_to_base_2(p.lse[stat]);
      next_delta = b.delta[stat];
      next_lo = w.lo;
      next_count = r < rows ? w.hi - w.lo : 0;
      next_at = w.token + e.shift;
      if (EXTRA) next_slope = p.slopes ? p.slopes[w.head] * kLog2e : 0.0f;
      if (tid < 2) {
        const int i = 2 * t + tid;
        next_seen = seen[min(i, groups - 1)];
        if (i >= groups || (i + 1) * 32 > rows) next_seen.z = 0x7fffffff;  // (rows past the last: never seen by all)
        if (i >= groups) next_seen.y = 0;
      }
    }
  };
  auto put = [&](int t) {
    const int s = t & 1;
    if (tid < kTileRows) {
      row_lse[s][tid] = next_lse - kLiftBits;
      row_delta[s][tid] = next_delta * (1.0f / kLift);
      row_lo[s][tid] = next_lo;
      row_count[s][tid] = next_count;
      row_at[s][tid] = next_at;
      if (EXTRA) row_slope[s][tid] = next_slope;
      if (tid < 2) tile_seen[s][tid] = next_seen;
    }
  };

  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[d][r] = dv[d][r] = 0.0f;
  Score score(p, 0.0f);
  if (t0 < t1) {
    request(t0);
    look_up(t0);
    put(t0);
  }
  for (int t = t0; t < t1; ++t) {
    wait_all_and_meet();
    if (t + 1 < t1) {
      request(t + 1);
      look_up(t + 1);
    }
    const unsigned char* qs = smem + (t & 1) * STAGE;
    const unsigned char* gs = qs + 2 * STAGE;
    const int st = t & 1;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int4 group = tile_seen[st][c];
      if (__builtin_amdgcn_readfirstlane(group.x) >= key0 + 32 || __builtin_amdgcn_readfirstlane(group.y) <= key0) continue;
      const bool masked = __builtin_amdgcn_readfirstlane(group.z) > key0 || __builtin_amdgcn_readfirstlane(group.w) < key0 + 32;
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s = mfma_op(row_frag<T, CPR>(qs, lane, c * 32, ks), kf[ks], s);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) dp = mfma_op(row_frag<T, CPR>(gs, lane, c * 32, ks), vf[ks], dp);
      Frag pf[2], ds[2];
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        const int i = c * 32 + 8 * gq + 4 * half;
        const f32x4 lse = *reinterpret_cast<const f32x4*>(&row_lse[st][i]);
        const f32x4 delta = *reinterpret_cast<const f32x4*>(&row_delta[st][i]);
        float prob[4], d[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float dot = s[4 * gq + u];
          float deriv = 1.0f;
          if constexpr (EXTRA) {
            float x = dot * score.factor;
            if (score.cap > 0) {
              const float th = score.tanh_of(dot);
              x = score.cap * th;
              deriv = 1.0f - th * th;
            }
            x -= row_slope[st][i + u] * (float)abs(row_at[st][i + u] - key);
            prob[u] = exp2_fast(x - lse[u]);
          } else {
            prob[u] = exp2_fast(__builtin_fmaf(dot, score.factor, -lse[u]));
          }
          d[u] = prob[u] * __builtin_fmaf(dp[4 * gq + u], 1.0f / kLift, -delta[u]);
          if (EXTRA) d[u] *= deriv;
        }
        if (masked) {
          const int4 first = *reinterpret_cast<const int4*>(&row_lo[st][i]), count = *reinterpret_cast<const int4*>(&row_count[st][i]);
          const int f4[4] = {first.x, first.y, first.z, first.w}, c4[4] = {count.x, count.y, count.z, count.w};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const bool in = (unsigned)(key - f4[u]) < (unsigned)c4[u];
            prob[u] = in ? prob[u] : 0.0f;
            d[u] = in ? d[u] : 0.0f;
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          pf[gq >> 1][4 * (gq & 1) + u] = from_f32<T>(prob[u]);
          ds[gq >> 1][4 * (gq & 1) + u] = from_f32<T>(d[u]);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          dv[d] = mfma_op(col_frag<T, CPR>(gs, lane, c * 32 + h * 16, d), pf[h], dv[d]);
          dk[d] = mfma_op(col_frag<T, CPR>(qs, lane, c * 32 + h * 16, d), ds[h], dk[d]);
        }
    }
    if (t + 1 < t1) put(t + 1);
  }
  const unsigned long long odd = __ballot(!(all_finite(dk) && all_finite(dv)));
  unsigned again = (unsigned)odd | (unsigned)(odd >> 32);
  if (key < e.keys && !((again >> (lane & 31)) & 1)) {
    store_columns<T, DT>(reinterpret_cast<T*>(b.dk) + (long long)e.b * b.dks.batch + (long long)e.kv * b.dks.head + (long long)key * b.dks.row, dk,
                         half, p.dim, p.scale);
    store_columns<T, DT>(reinterpret_cast<T*>(b.dv) + (long long)e.b * b.dvs.batch + (long long)e.kv * b.dvs.head + (long long)key * b.dvs.row, dv,
                         half, p.dim, 1.0f / kLift);
  }
  again = __builtin_amdgcn_readfirstlane(again);
  while (again) {
    const int i = __builtin_ctz(again);
    again &= again - 1;
    if (key0 + i < e.keys) dkv_by_definition<T, DP>(b, e, key0 + i);
  }
}

template <typename T, int DP, bool EXTRA>
hipError_t launch(const BackArgs& b, hipStream_t stream) {
  const Args& p = b.f;
  const long long entries = (long long)p.batch * p.kv_heads;
  if (p.seq_q > 0) {
    hipLaunchKernelGGL((dq_kernel<T, DP, EXTRA>), dim3((unsigned)(entries * p.row_tiles)), dim3(256), 0, stream, b);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (p.seq_k > 0) {
    hipLaunchKernelGGL((dkv_kernel<T, DP, EXTRA>), dim3((unsigned)(entries * b.key_tiles)), dim3(256), 0, stream, b);
    return hipGetLastError();
  }
  return hipSuccess;
}
template <typename T>
hipError_t dispatch(bool extra, const BackArgs& b, hipStream_t stream) {
  if (padded_dim(b.f.dim) == 128) return extra ? launch<T, 128, true>(b, stream) : launch<T, 128, false>(b, stream);
  return extra ? launch<T, 64, true>(b, stream) : launch<T, 64, false>(b, stream);
}

long long row_groups_of(long long rows) { return (rows + 31) / 32; }
long long delta_bytes(long long batch, long long heads, long long seq_q) { return (batch * heads * seq_q * 4 + 15) / 16 * 16; }

}  // namespace

extern "C" {

int64_t hidet_attention_backward_workspace_bytes(int64_t batch, int64_t heads, int64_t kv_heads, int64_t seq_q, int64_t seq_k,
                                                 int64_t head_dim) {
  (void)seq_k;
  (void)head_dim;
  if (batch <= 0 || kv_heads <= 0 || heads <= 0 || heads % kv_heads != 0 || seq_q <= 0) return 0;
  const long long group = heads / kv_heads;
  if (group >= kMaxRows || seq_q >= kMaxRows || seq_q * group >= kMaxRows || batch > kMaxBlocks || kv_heads > kMaxBlocks) return 0;
  return delta_bytes(batch, heads, seq_q) + batch * row_groups_of(seq_q * group) * 16;
}

hidet_status_t hidet_attention_backward(int32_t dtype, int64_t batch, int64_t heads, int64_t kv_heads, int64_t seq_q, int64_t seq_k,
                                        int64_t head_dim, const hidet_heads_t* grad_out, const hidet_heads_t* q, const hidet_heads_t* k,
                                        const hidet_heads_t* v, const hidet_heads_t* out, const float* lse, const hidet_heads_t* grad_q,
                                        const hidet_heads_t* grad_k, const hidet_heads_t* grad_v,
                                        const hidet_attention_options_t* options, void* workspace, int64_t workspace_bytes, void* stream) {
  if (dtype < 0 || dtype > 2) return HIDET_ERR_INVALID_ARG;
  if (dtype == HIDET_F32) return HIDET_ERR_UNSUPPORTED;
  if (batch < 0 || heads < 0 || kv_heads < 0 || seq_q < 0 || seq_k < 0 || head_dim <= 0 || workspace_bytes < 0) return HIDET_ERR_INVALID_ARG;
  if (hidet_status_t st = check_options(options); st != HIDET_OK) return st;
  if (batch == 0 || heads == 0 || (seq_q == 0 && seq_k == 0)) return HIDET_OK;
  if (kv_heads == 0 || heads % kv_heads != 0) return HIDET_ERR_INVALID_ARG;
  if (head_dim > 128 || head_dim % 8 != 0) return HIDET_ERR_UNSUPPORTED;
  const long long group = heads / kv_heads;
  if (group >= kMaxRows || seq_q >= kMaxRows || seq_k >= kMaxRows || seq_q * group >= kMaxRows) return HIDET_ERR_UNSUPPORTED;
  if (batch > kMaxBlocks || kv_heads > kMaxBlocks) return HIDET_ERR_UNSUPPORTED;
  if (seq_q > 0) {
    for (const hidet_heads_t* t : {grad_out, q, out})
      if (hidet_status_t st = check_heads(t, batch, heads, seq_q, head_dim, false); st != HIDET_OK) return st;
    if (hidet_status_t st = check_heads(grad_q, batch, heads, seq_q, head_dim, true); st != HIDET_OK) return st;
    if (!lse || !workspace) return HIDET_ERR_INVALID_ARG;
    if (workspace_bytes < hidet_attention_backward_workspace_bytes(batch, heads, kv_heads, seq_q, seq_k, head_dim)) return HIDET_ERR_INVALID_ARG;
  }
  if (seq_k > 0) {
    for (const hidet_heads_t* t : {k, v}) {
      if (hidet_status_t st = check_heads(t, batch, kv_heads, seq_k, head_dim, false); st != HIDET_OK) return st;
      if (t->stride_row >= kMaxStride) return HIDET_ERR_UNSUPPORTED;
    }
    for (const hidet_heads_t* t : {grad_k, grad_v})
      if (hidet_status_t st = check_heads(t, batch, kv_heads, seq_k, head_dim, true); st != HIDET_OK) return st;
  }
  if (!is_aligned(lse, 4) || !is_aligned(workspace, 16)) return HIDET_ERR_ALIGNMENT;
  BackArgs b{};
  Args& p = b.f;
  if (seq_q > 0) {
    p.q = q->data;
    p.out = out->data;
    p.lse = const_cast<float*>(lse);
    p.qs = strides_of(q);
    p.os = strides_of(out);
    b.dout = grad_out->data;
    b.dos = strides_of(grad_out);
    b.dq = grad_q->data;
    b.dqs = strides_of(grad_q);
    b.delta = static_cast<float*>(workspace);
    b.seen = reinterpret_cast<int4*>(static_cast<char*>(workspace) + delta_bytes(batch, heads, seq_q));
  }
  if (seq_k > 0) {
    p.k = k->data;
    p.v = v->data;
    p.ks = strides_of(k);
    p.vs = strides_of(v);
    b.dk = grad_k->data;
    b.dv = grad_v->data;
    b.dks = strides_of(grad_k);
    b.dvs = strides_of(grad_v);
  }
  p.slopes = options->slopes;
  p.ranges = options->ranges;
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
  p.splits = 1;
  p.row_tiles = (int)((seq_q * group + 127) / 128);
  b.row_groups = (int)row_groups_of(seq_q * group);
  b.key_tiles = (int)((seq_k + 127) / 128);
  if (batch * kv_heads * std::max(p.row_tiles, b.key_tiles) > kMaxBlocks) return HIDET_ERR_UNSUPPORTED;
  const bool extra = is_extra(options);
  const hipStream_t s = (hipStream_t)stream;
  const hipError_t e = dtype == HIDET_F16 ? dispatch<f16>(extra, b, s) : dispatch<bf16>(extra, b, s);
  return e == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

}  // extern "C"
