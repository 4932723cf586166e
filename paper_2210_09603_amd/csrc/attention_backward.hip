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
// 2^-24, and divided out at the end.  dS follows the caller's gradients and values in size: an fp16 operand takes it times a power of
// two that follows it, see Lift.  (As it is, dS of gradients of 1e-3 over 4096 keys is four steps of fp16's subnormals.)  bf16 has
// the range of fp32.
#include "attention_host.hpp"

using namespace hidet;
using namespace hidet::attn;

namespace {

constexpr float kLift = 1024.0f, kLiftBits = 10.0f;

struct BackArgs {
  Args f;  // f.lse: of the forward pass; f.out: its output
  const void* dout;
  void* dq;
  void* dk;
  void* dv;
  Strides dos, dqs, dks, dvs;
  float* info;    // of every row of a kv head, see row_info
  float* peak;    // [entry][row_groups]: of 32 rows, the largest of what their dS are likely to be, see Lift (fp16)
  int4* seen;     // [batch][row_groups]: of 32 rows, the first and last + 1 of the keys that any of them sees; that all of them see
  int* order;     // [batch][key_tiles]: the blocks of keys, the longest first; null: as they lie
  float* part;    // partial sums of the splits: dQ's [split][kv row][DP], then dK's and dV's [split][entry][key][2][DP]
  int row_groups;
  int key_tiles;
  int dq_pairs;               // two wavefronts for 32 rows
  int dq_splits, dq_share;    // share: tiles of keys of a split
  int dkv_splits, dkv_share;  // share: tiles of rows
  int regular;    // 32 rows hold whole tokens, and offsets within them fit 32 bits
};

// What the second kernel needs to know of a row, as the first leaves it: for 4 rows each in turn, so that a lane reads those of its 4
// rows at once, and padded to whole tiles by rows that nobody is seen by.
//   0  lse to base 2, less the lift     1  D, divided by the lift     2, 3  first key seen, their number
//   4  position, 5  slope to base 2 (with a bias only: 8 fields, else 4)
// (positions are whole numbers, as their differences to a key's are taken: from 2^24 on fp32 does not hold them)
template <int FORM>
__device__ __forceinline__ float* row_info(const BackArgs& b, const Entry& e, int r, int field) {
  constexpr int FIELDS = FORM & FORM_BIAS ? 8 : 4;
  const long long rows = (long long)b.f.row_tiles * 128, entry = (long long)e.b * b.f.kv_heads + e.kv;
  return b.info + (entry * rows + (r & ~3)) * FIELDS + field * 4 + (r & 3);
}

// The weight of a query's only key is 1 whatever the score: dS = P (dP - D) is 0, of which the two sums D and dP, in their different
// orders, would leave a rounding.  (Times 0, so that what is not finite stays so.)
__device__ __forceinline__ float unless_alone(int keys) { return keys == 1 ? 0.0f : 1.0f; }

__device__ __forceinline__ float lse_to_base_2(float lse) { return lse == kNoMax ? __builtin_huge_valf() : lse * kLog2e; }

// The power of two by which dS is taken as an fp16 operand.  A query's dS = P (dP - D) are about as large as the product of its largest
// |dout| and its largest |out| (`peak`), times the root of the dimensions: out is the sum of P v, and P v alone is not much larger.  For
// dK it is the largest of the rows that see a block of keys.  `by` brings that to between 2^4 and 2^5: dS may be 2^11 times as large, and
// steps of fp16's subnormals are 2^-29 of it.  Where dS passes fp16 all the same (large values that cancel in out) the sums come out not
// finite, and are taken again: dQ with 2^-12 of it as often as that takes, dK with a look at every tile.
struct Lift {
  float by;
  __device__ __forceinline__ explicit Lift(float peak) {
    by = peak > 0.0f ? __builtin_ldexpf(1.0f, 5 - __builtin_amdgcn_frexp_expf(peak)) : 1.0f;
  }
  // ds: the numbers of a tile, already times `by`, acc: the sum so far, both of them lowered where ds would pass fp16
  template <int DT>
  __device__ __forceinline__ void fit(f32x16& ds, f32x16 (&acc)[DT]) {
    float top = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, __builtin_fabsf(ds[r]));
    top = max_of_halves(top);
    if (!__any(top > 32768.0f)) return;
    const float f = top > 32768.0f && top < __builtin_huge_valf() ? __builtin_ldexpf(1.0f, 10 - __builtin_amdgcn_frexp_expf(top)) : 1.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) ds[r] *= f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][r] *= f;
    by *= f;
  }
};

// What comes out not finite, as in the forward pass: a second walk without what is not finite of the operands of the last products -- zeros
// for such keys for dQ, for such elements of q and dout for dK and dV --, which gives the bits that there are without.  A query whose
// log-sum or D is not finite has dS that are not, in its own row and for all keys that it sees, from those two numbers alone; and where a
// key is seen by a gradient of the output that is not finite, one pass over such rows puts it into dV.  (4096 rows and keys, 16 heads of 128
// dimensions, causal, 570 us: with one infinite gradient 1170, one in every row 4400; 620 ms when such rows were computed one by one.)

// dQ of a query that sees keys that are not finite and has a finite log-sum all the same (their scores are -inf, their weights 0), where zeros
// in their place have weights that pass fp32: a log-sum below -88.  Over its keys from `from` on and before `to`; by all lanes of a
// wavefront.
template <typename T, int DP, int FORM>
__device__ __forceinline__ void dq_by_definition(const BackArgs& b, const Entry& e, int r, int from, int to, float delta, float (&acc)[DP / 64]) {
  constexpr int E = DP / 64;
  const Args& p = b.f;
  const int lane = threadIdx.x & 63;
  const Row w = make_row<false>(p, e, r);
  const Score<FORM> score(p, p.slopes ? p.slopes[w.head] : 0.0f);
  const T* q = reinterpret_cast<const T*>(p.q) + query_offset<false>(p, e, p.qs, w);
  const T* g = reinterpret_cast<const T*>(b.dout) + query_offset<false>(p, e, b.dos, w);
  const T* k = keys_of<T, false>(p, e, p.k, p.ks);
  const T* v = keys_of<T, false>(p, e, p.v, p.vs);
  const float lse = lse_to_base_2(p.lse[lse_offset<false>(p, e, w)]);
  float mq[E], mg[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int d = lane * E + i;
    mq[i] = d < p.dim ? to_f32(q[d]) : 0.0f;
    mg[i] = d < p.dim ? to_f32(g[d]) : 0.0f;
    acc[i] = 0.0f;
  }
  from = max(from, w.lo);
  to = min(to, w.hi);
  for (int j = from; j < to; ++j) {
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
    float derivative;
    const float prob = exp2_fast(score(dot, (float)(w.token + e.shift - j), derivative) - lse);
    if (prob == 0.0f) continue;
    const float ds = prob * (dp - delta) * derivative * unless_alone(w.hi - w.lo);
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] += ds * mk[i];
  }
}

// What is not finite of the gradients of the output of rows from `from` on and before `to`, for the lane's key: the sum of those that see it.
template <typename T, int DP, int FORM>
__device__ __forceinline__ OddSums<DP> odd_gradients(const BackArgs& b, const Entry& e, int key, int from, int to, bool ask) {
  constexpr int E = DP / 64, U = 8;
  struct __attribute__((packed, aligned(2))) Own {
    T x[E];
  };
  const Args& p = b.f;
  const int lane = worked_out_here(threadIdx.x & 63);
  const bool has = lane * E < p.dim;
  const T* base = reinterpret_cast<const T*>(b.dout) + (long long)e.b * b.dos.batch + (long long)e.kv * p.group * b.dos.head + (has ? lane * E : 0);
  OddSums<DP> sums;
  sums.clear();
#pragma unroll 1
  for (int r0 = from; r0 < to; r0 += 64) {
    // (a row whose own log-sum is not finite has weights that are 0 or NaN already)
    const int r = min(r0 + lane, to - 1);
    const bool odd = r0 + lane < to && !(__builtin_fabsf(*row_info<FORM>(b, e, r, 1)) < __builtin_huge_valf()) &&
                     __builtin_fabsf(*row_info<FORM>(b, e, r, 0)) < __builtin_huge_valf();
    const unsigned long long rows = __ballot(odd);
    if (!rows) continue;
    const int lo = *reinterpret_cast<int*>(row_info<FORM>(b, e, r, 2)), count = *reinterpret_cast<int*>(row_info<FORM>(b, e, r, 3));
#pragma unroll 1
    for (int c = 0; c < 64; c += U) {
      if (!((rows >> c) & ((1u << U) - 1))) continue;
      Own g[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = min(r0 + c + u, to - 1), token = p.d_group.div(row), head = row - token * p.group;
        g[u] = *reinterpret_cast<const Own*>(base + (long long)head * b.dos.head + (long long)token * b.dos.row);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if ((rows >> (c + u)) & 1) {
          float x[E];
#pragma unroll
          for (int i = 0; i < E; ++i) x[i] = has ? to_f32(g[u].x[i]) : 0.0f;
          sums.add(x, ask && (unsigned)(key - __builtin_amdgcn_readlane(lo, c + u)) < (unsigned)__builtin_amdgcn_readlane(count, c + u));
        }
      if (!__any(ask && any_but_nan(sums, p.dim))) return sums;
    }
  }
  return sums;
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
__device__ __forceinline__ void store_part(float* to, const f32x16 (&acc)[DT], int half) {
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(to + 32 * t + 8 * g + 4 * half) = f32x4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]};
}
template <int DP>
__device__ __forceinline__ float* dq_part(const BackArgs& b, int z, const Entry& e, int r) {
  const long long per_entry = (long long)b.f.seq_q * b.f.group;
  return b.part + (((long long)z * b.f.batch * b.f.kv_heads + (long long)e.b * b.f.kv_heads + e.kv) * per_entry + r) * DP;
}
template <int DP>
__device__ __forceinline__ float* dkv_part(const BackArgs& b, int z, const Entry& e, int key) {
  return b.part + (((long long)z * b.f.batch * b.f.kv_heads + (long long)e.b * b.f.kv_heads + e.kv) * b.f.seq_k + key) * (2 * DP);
}

// ---- the order of the second kernel's work -------------------------------------------------------------------------------------
// Ranges may give blocks of keys work in any order, and what begins last should be short.  One workgroup of the first kernel ranks the
// blocks, 256 at a time, by how many groups of 32 rows see one of their keys: a sum over the differences at the first block of a group
// and behind its last.  What a group sees is estimated by its first and last rows; of equal blocks the first comes first, so that
// every block has one place, whatever the ranges are.  (Packed documents of 146 to 1024 tokens, 8 entries of 64 blocks: dK and dV 172 us
// as they lie, 138 in order, with the ranking at the start of every workgroup; a group of workgroups that begin at once needs none.)
constexpr int kTileRows = 128, kBlockKeys = 64, kDkvThreads = 512;
constexpr int kOrdered = 256;
template <int THREADS>
__device__ __forceinline__ void write_order(const BackArgs& b, int batch, int* edges, int* work) {
  const Args& p = b.f;
  const int rows = p.seq_q * p.group;
  const int* ranges = p.ranges + (long long)batch * p.seq_q * 2;
  int* order = b.order + (long long)batch * b.key_tiles;
  for (int base = 0; base < b.key_tiles; base += kOrdered) {
    const int count = min(b.key_tiles - base, kOrdered);
    for (int i = threadIdx.x; i < kOrdered; i += THREADS) edges[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < b.row_groups; i += THREADS) {
      const int first = 2 * p.d_group.div(i * 32), last = 2 * p.d_group.div(min(i * 32 + 31, rows - 1));
      const int lo = max(min(ranges[first], ranges[last]), 0), hi = min(max(ranges[first + 1], ranges[last + 1]), p.seq_k);
      const int from = max(lo / kBlockKeys - base, 0), to = (hi + kBlockKeys - 1) / kBlockKeys - base;
      if (lo >= hi || from >= count || to <= 0) continue;
      atomicAdd(&edges[from], 1);
      if (to < count) atomicAdd(&edges[to], -1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += THREADS) {
      int sum = 0;
      for (int j = 0; j <= i; ++j) sum += edges[j];
      work[i] = sum;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += THREADS) {
      int rank = 0;
      for (int j = 0; j < count; ++j) rank += work[j] > work[i] || (work[j] == work[i] && j < i);
      order[base + rank] = base + i;
    }
    __syncthreads();
  }
}

constexpr int kFewKeys = 32;

// ---- dQ ---------------------------------------------------------------------------------------------------------------
// The forward kernel's walk, with dout and out beside q, and its pairs of wavefronts.
template <typename T, int DP, int FORM, int PAIRS>
__global__ __launch_bounds__(256 * PAIRS, 2) void dq_kernel(const BackArgs b) {
  constexpr int THREADS = 256 * PAIRS, TILE = kTileKeys * PAIRS;  // keys of a tile
  constexpr int CPR = DP / 8, STAGE = TILE * CPR * 16, NL = TILE * CPR / THREADS, RPP = THREADS / CPR, KS = DP / 16, DT = DP / 32;
  using Frag = typename Frag8<T>::type;
  __shared__ __attribute__((aligned(16))) unsigned char smem[4 * STAGE];
  __shared__ int bounds[4][2], few_bounds[4][2], spoilt;
  __shared__ unsigned odd_keys[TILE / 32];
  __shared__ float halves[8][32];
  const Args& p = b.f;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int own = (wave >> 2) * kTileKeys;  // the first of its 64 keys of a tile

  const Place place = place_of(blockIdx.x, p.batch * p.kv_heads, p.row_tiles * b.dq_splits);
  const int z = place.piece % b.dq_splits, tile = p.row_tiles - 1 - place.piece / b.dq_splits;
  const Entry e = make_entry<false>(p, place.entry / p.kv_heads, place.entry % p.kv_heads);
  const int rows = e.tokens * p.group, r0 = tile * 128 + (wave & 3) * 32;
  if (b.order && e.kv == 0 && z == 0 && tile == p.row_tiles / 2)
    write_order<THREADS>(b, e.b, reinterpret_cast<int*>(smem), reinterpret_cast<int*>(smem) + kOrdered);

  const Row w = make_row<false>(p, e, min(r0 + (lane & 31), rows - 1));
  const int at = w.token + e.shift;
  const Seen mine = seen_by<false>(p, e, w, min(r0, rows - 1), min(r0 + 31, rows - 1));
  // the keys that rows of few keys see
  const bool few = w.hi - w.lo > 1 && w.hi - w.lo <= kFewKeys;
  const int few_lo = wave_min(few ? w.lo : 0x7fffffff), few_hi = wave_max(few ? w.hi : 0);
  if (lane == 0 && wave < 4) {
    few_bounds[wave][0] = few_lo;
    few_bounds[wave][1] = few_hi;
  }
  int begin, end;  // of the workgroup
  if (p.ranges) {
    if (lane == 0 && wave < 4) {
      bounds[wave][0] = mine.lo;
      bounds[wave][1] = mine.hi;
    }
  } else {
    const Seen all = seen_by<false>(p, e, w, tile * 128, min(tile * 128 + 127, rows - 1));
    begin = all.lo;
    end = all.hi;
  }
  if (lane == 0 && wave < 4 && e.kv == 0 && z == 0 && r0 < rows) b.seen[(long long)e.b * b.row_groups + (r0 >> 5)] = int4{mine.lo, mine.hi, mine.full_lo, mine.full_hi};
  Frag q[KS], g[KS];
  load_row_frags<T, DP>(reinterpret_cast<const T*>(p.q) + query_offset<false>(p, e, p.qs, w), half, p.dim, q);
  load_row_frags<T, DP>(reinterpret_cast<const T*>(b.dout) + query_offset<false>(p, e, b.dos, w), half, p.dim, g);
  constexpr bool LIFTS = !std::is_same<T, bf16>::value;
  float delta = 0.0f, peak = 0.0f;
  {
    Frag o[KS];
    float g_peak = 0.0f, o_peak = 0.0f;
    load_row_frags<T, DP>(reinterpret_cast<const T*>(p.out) + query_offset<false>(p, e, p.os, w), half, p.dim, o);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float its = to_f32(g[ks][i]), out = to_f32(o[ks][i]);
        delta = __builtin_fmaf(its, out, delta);
        if constexpr (LIFTS) {
          g_peak = fmaxf(g_peak, __builtin_fabsf(its) < __builtin_huge_valf() ? __builtin_fabsf(its) : 0.0f);
          o_peak = fmaxf(o_peak, __builtin_fabsf(out) < __builtin_huge_valf() ? __builtin_fabsf(out) : 0.0f);
        }
      }
    if constexpr (LIFTS) {
      peak = max_of_halves(g_peak) * max_of_halves(o_peak);
      // (numbers that are not negative compare as whole numbers)
      const int of_rows = wave_max(__builtin_bit_cast(int, peak));
      if (lane == 0 && wave < 4 && z == 0 && r0 < rows)
        b.peak[((long long)e.b * p.kv_heads + e.kv) * b.row_groups + (r0 >> 5)] = __builtin_bit_cast(float, of_rows);
    }
  }
  delta = sum_of_halves(delta);
  const long long stat = lse_offset<false>(p, e, w);
  const float lse = lse_to_base_2(p.lse[stat]);
  if (half == 0 && wave < 4 && z == 0) {
    const int r = r0 + lane;
    const bool is = r < rows;
    *row_info<FORM>(b, e, r, 0) = (is ? lse : __builtin_huge_valf()) - kLiftBits;
    *reinterpret_cast<int*>(row_info<FORM>(b, e, r, 2)) = w.lo;
    *reinterpret_cast<int*>(row_info<FORM>(b, e, r, 3)) = is ? w.hi - w.lo : 0;
    if constexpr (FORM & FORM_BIAS) {
      *reinterpret_cast<int*>(row_info<FORM>(b, e, r, 4)) = at;
      *row_info<FORM>(b, e, r, 5) = p.slopes ? p.slopes[w.head] * kLog2e : 0.0f;
    }
  }
  const Score<FORM> score(p, p.slopes ? p.slopes[w.head] : 0.0f);
  if (tid == 0) spoilt = 0;
  if (p.dim < DP)
    for (int i = tid; i < 4 * STAGE / 16; i += THREADS) reinterpret_cast<u32x4*>(smem)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
  if (p.ranges) {
    begin = min(min(bounds[0][0], bounds[1][0]), min(bounds[2][0], bounds[3][0]));
    end = max(max(bounds[0][1], bounds[1][1]), max(bounds[2][1], bounds[3][1]));
    begin = __builtin_amdgcn_readfirstlane(begin);
    end = __builtin_amdgcn_readfirstlane(end);
  }
  if (begin >= end) begin = end = 0;
  const int all = (end - begin + TILE - 1) / TILE;
  const int t0 = min(all, z * b.dq_share), t1 = z + 1 < b.dq_splits ? min(all, t0 + b.dq_share) : all;

  const T* kbase = keys_of<T, false>(p, e, p.k, p.ks);
  const T* vbase = keys_of<T, false>(p, e, p.v, p.vs);
  const int load_row = tid / CPR, load_chunk = (tid % CPR) ^ swz<CPR>(load_row);
  const bool loads = load_chunk * 8 < p.dim;
  const unsigned lds0 = lds_address(smem), lds = lds0 + wave * 1024;
  const ReadMap<DP> map(lane);
  auto request = [&](int begin, int end, int t) {  // tile t of the keys begin..end - 1
    const unsigned to = lds + (t & 1) * STAGE;
    const int first = begin + t * TILE, last = end - 1 - first;
    const T* kt = kbase + (long long)first * p.ks.row;
    const T* vt = vbase + (long long)first * p.vs.row;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = min(i * RPP + load_row, last);
      const unsigned ko = ((unsigned)row * (unsigned)p.ks.row + load_chunk * 8) * 2;
      const unsigned vo = ((unsigned)row * (unsigned)p.vs.row + load_chunk * 8) * 2;
      if (loads) {
        DirectLoad::at(kt, ko, to + i * (THREADS * 16));
        DirectLoad::at(vt, vo, to + 2 * STAGE + i * (THREADS * 16));
      }
    }
  };
  int few_begin = min(min(few_bounds[0][0], few_bounds[1][0]), min(few_bounds[2][0], few_bounds[3][0]));
  int few_end = max(max(few_bounds[0][1], few_bounds[1][1]), max(few_bounds[2][1], few_bounds[3][1]));
  few_begin = __builtin_amdgcn_readfirstlane(few_begin);
  few_end = __builtin_amdgcn_readfirstlane(few_end);
  settle();
  // D of a query that sees few keys, from what it sees: D = sum P dP, of which dout . out has the rounding of out.  That is half a step of
  // D, and dS = P (dP - D) may be far smaller than D where a few keys have all the weight; among many it is not.  (Scores of 5 keys that
  // spread by 4: dQ in bf16 13 times as far off without.  Windows of 32 keys over 4096 positions, 36 heads: a pass 154 us, 146 without.)
  // Every split of the tile works it out, over the tiles that such rows see.
  if (few_begin < few_end) {
    const int tiles = tiles_of<TILE>(few_begin, few_end);
    float rest = 0.0f;
    request(few_begin, few_end, 0);
    for (int t = 0; t < tiles; ++t) {
      wait_all_and_meet();
      if (t + 1 < tiles) request(few_begin, few_end, t + 1);
      const int first = few_begin + t * TILE + own;
      if (first >= few_hi || first + kTileKeys <= few_lo) continue;
      const unsigned keys = lds0 + (t & 1) * STAGE + own * (DP * 2), values = keys + 2 * STAGE;
#pragma unroll 1
      for (int c = 0; c < 2; ++c) {
        f32x16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mfma_op(row_frag<T, DP>(map, keys, c * 32, ks), q[ks], s);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mfma_op(row_frag<T, DP>(map, values, c * 32, ks), g[ks], dp);
        const int base = first + c * 32 + 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = base + 8 * (r >> 2) + (r & 3);
          float derivative;
          const float d = exp2_fast(score(s[r], (float)(at - j), derivative) - lse) * (dp[r] - delta);
          rest += (unsigned)(j - w.lo) < (unsigned)(w.hi - w.lo) ? d : 0.0f;
        }
      }
    }
    rest = sum_of_halves(rest);
    if constexpr (PAIRS == 2) {
      if (half == 0) halves[wave][lane] = rest;
      __syncthreads();
      rest += halves[wave ^ 4][lane & 31];
    }
    // (D that is not finite says so already)
    if (few && __builtin_fabsf(rest) < __builtin_huge_valf()) delta += rest;
    __syncthreads();
  }
  if (half == 0 && wave < 4 && z == 0) *row_info<FORM>(b, e, r0 + lane, 1) = r0 + lane < rows ? delta * (1.0f / kLift) : 0.0f;
  // Zeros for the keys of tile t that are not finite.  A row that sees such a one, and has a finite log-sum all the same, has a score of -inf
  // for it and no weight: with a key of zeros its weight is another, but what it adds is 0.
  auto drop_odd_keys = [&](int t) {
    const int thread = worked_out_here(threadIdx.x);
    if (thread < TILE / 32) odd_keys[thread] = 0;
    __syncthreads();
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
#pragma unroll 1
      for (int i = 0; i < NL; ++i) {
        u32x4* at = reinterpret_cast<u32x4*>(smem + (t & 1) * STAGE + (i * THREADS + thread) * 16);
        const u32x4 was = *at, is = finite_ones<T>(was);
        const int row = i * RPP + thread / CPR;
        if (turn) {
          if ((odd_keys[row / 32] >> (row % 32)) & 1) *at = u32x4{0, 0, 0, 0};
        } else if (was[0] != is[0] || was[1] != is[1] || was[2] != is[2] || was[3] != is[3]) {
          atomicOr(&odd_keys[row / 32], 1u << (row % 32));
        }
      }
      __syncthreads();
    }
  };
  auto sees_one_of = [&](int t) {
    const Row seen = make_row<false>(p, e, worked_out_here(min(r0 + (lane & 31), rows - 1)));
    bool sees = false;
#pragma unroll 1
    for (int i = 0; i < TILE; ++i) {
      const int j = begin + t * TILE + i;
      sees |= ((odd_keys[i / 32] >> (i % 32)) & 1) && j >= seen.lo && j < seen.hi;
    }
    return sees;
  };
  f32x16 acc[DT];
  Lift lift(peak);
  bool sees_odd = false, odd = false;
  int pass = 0;  // from 1 on without keys that are not finite
  for (;; ++pass) {
    const float lifted = delta * lift.by;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] = 0.0f;
    if (t0 < t1) request(begin, end, t0);
    for (int t = t0; t < t1; ++t) {
      wait_all_and_meet();
      if (__builtin_expect(pass != 0, 0)) {
        drop_odd_keys(t);
        sees_odd |= sees_one_of(t);
      }
      if (t + 1 < t1) request(begin, end, t + 1);
      const int first = begin + t * TILE + own;
      if (first >= mine.hi || first + kTileKeys <= mine.lo) continue;
      const unsigned keys = lds0 + (t & 1) * STAGE + own * (DP * 2), values = keys + 2 * STAGE;
      const bool masked = first < mine.full_lo || first + kTileKeys > mine.full_hi;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        f32x16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mfma_op(row_frag<T, DP>(map, keys, c * 32, ks), q[ks], s);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mfma_op(row_frag<T, DP>(map, values, c * 32, ks), g[ks], dp);
        const int base = first + c * 32 + 4 * half;
        const float distance = (float)(at - base);
        Frag ds[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = base + 8 * (r >> 2) + (r & 3);
          float derivative = 1.0f, x;
          if constexpr (FORM == FORM_PLAIN)
            x = __builtin_fmaf(s[r], score.factor, -lse);
          else
            x = score(s[r], distance - (float)(8 * (r >> 2) + (r & 3)), derivative) - lse;
          float d = exp2_fast(x) * (LIFTS ? __builtin_fmaf(dp[r], lift.by, -lifted) : dp[r] - delta) * derivative;
          if (masked) d = (unsigned)(j - w.lo) < (unsigned)(w.hi - w.lo) ? d : 0.0f;
          ds[r >> 3][r & 7] = from_f32<T>(d);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[d] = mfma_op(col_frag<T, DP>(map, keys, c * 32 + h * 16, d), ds[h], acc[d]);
      }
    }
    odd = !all_finite(acc) && __builtin_fabsf(delta) < __builtin_huge_valf() && __builtin_fabsf(lse) < __builtin_huge_valf();
    if (__any(odd) && lane == 0) spoilt = pass + 1;
    __syncthreads();
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(spoilt) <= pass, 1) || pass == (LIFTS ? 6 : 1)) break;
    if (pass > 0) {  // (finite numbers whose dS fp16 does not hold)
      const unsigned long long lanes = __ballot(odd);
      if ((((unsigned)lanes | (unsigned)(lanes >> 32)) >> (lane & 31)) & 1) lift.by *= 0x1p-12f;
    }
  }
  const bool again = pass != 0;
  if (lse == __builtin_huge_valf()) {  // (nothing was seen, or scores of -inf alone)
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] = 0.0f;
  }
  const float by = unless_alone(w.hi - w.lo) / lift.by;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] *= by;
  if constexpr (PAIRS == 2) {
    __syncthreads();
    float* meet = reinterpret_cast<float*>(smem) + (wave & 3) * (DT * 16 * 64) + lane;
    if (wave >= 4) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) meet[(d * 16 + r) * 64] = acc[d][r];
    }
    __syncthreads();
    if (wave >= 4) return;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] += meet[(d * 16 + r) * 64];
  }
  const unsigned long long lanes = __ballot(odd && sees_odd);
  const bool alone_again = again && ((((unsigned)lanes | (unsigned)(lanes >> 32)) >> (lane & 31)) & 1);
  const bool real = r0 + (lane & 31) < rows;
  if (real && !alone_again) {
    if (b.dq_splits > 1)
      store_part<DT>(dq_part<DP>(b, z, e, r0 + (lane & 31)), acc, half);
    else
      store_columns<T, DT>(reinterpret_cast<T*>(b.dq) + query_offset<false>(p, e, b.dqs, place_of_row(p, e, worked_out_here(r0 + (lane & 31)))), acc, half,
                           p.dim, p.scale);
  }
  if (__builtin_expect(!again, 1)) return;
  unsigned left = __builtin_amdgcn_readfirstlane((unsigned)__ballot(real && alone_again));  // (the same in both halves)
  while (left) {
    constexpr int E = DP / 64;
    const int i = __builtin_ctz(left);
    left &= left - 1;
    float row[E];
    dq_by_definition<T, DP, FORM>(b, e, r0 + i, key_at<TILE>(begin, t0, 0, end), key_at<TILE>(begin, t1, 0, end), __shfl(delta, i), row);
    const Row its = make_row<false>(p, e, r0 + i);
    T* to = reinterpret_cast<T*>(b.dq) + query_offset<false>(p, e, b.dqs, its);
    float* part = b.dq_splits > 1 ? dq_part<DP>(b, z, e, r0 + i) : nullptr;
#pragma unroll
    for (int u = 0; u < E; ++u) {
      const int d = lane * E + u;
      if (part)
        part[d] = row[u];
      else if (d < p.dim)
        to[d] = from_f32<T>(row[u] * p.scale);
    }
  }
}

// The splits of a query's sum, in ascending order; one wavefront a query.
template <typename T, int DP>
__global__ __launch_bounds__(256) void dq_join_kernel(const BackArgs b) {
  constexpr int E = DP / 64;
  const Args& p = b.f;
  const int lane = threadIdx.x & 63, per_entry = p.seq_q * p.group;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= (long long)p.batch * p.kv_heads * per_entry) return;
  const int entry = (int)(row / per_entry), r = (int)(row - (long long)entry * per_entry);
  const Entry e = make_entry<false>(p, entry / p.kv_heads, entry % p.kv_heads);
  float acc[E];
#pragma unroll
  for (int i = 0; i < E; ++i) acc[i] = 0.0f;
#pragma unroll 4
  for (int z = 0; z < b.dq_splits; ++z) {
    const float* from = dq_part<DP>(b, z, e, r) + lane * E;
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] += from[i];
  }
  const Row w = place_of_row(p, e, r);
  T* to = reinterpret_cast<T*>(b.dq) + query_offset<false>(p, e, b.dqs, w);
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (lane * E + i < p.dim) to[lane * E + i] = from_f32<T>(acc[i] * p.scale);
}

// ---- dK, dV -------------------------------------------------------------------------------------------------------------
// A workgroup of 8 wavefronts works on 64 keys and walks over the rows that see one of them in tiles of 128 rows of q and dout,
// which arrive in LDS one tile ahead.  4 wavefronts share 32 keys and meet in LDS at the end.  Up to 64 dimensions each of them takes
// 32 of the tile's rows and sums dK and dV.  Beyond, two sum dK and two dV, each of 64 rows: the scores are computed for either sum
// (5 products for 4), which halves what a wavefront keeps -- a sum, its keys and values, 128 registers at 128 dimensions -- so that two
// wavefronts fit a SIMD, one of each kind.
// Microseconds for 2 x 4096 positions of 16 heads on 4, 128 dimensions, no mask: 800; both sums in a wavefront, one a SIMD, waiting for
// LDS half of the time, 1237; the same with the values in LDS, two a SIMD and 44 registers spilled, 1200.  For 3 x 1021 positions of 12
// heads, 64 dimensions: both sums in a wavefront 48, apart 53.

template <typename T, int DP, int FORM>
__global__ __launch_bounds__(kDkvThreads, 2) void dkv_kernel(const BackArgs b) {
  constexpr int CPR = DP / 8, STAGE = kTileRows * CPR * 16, NL = kTileRows * CPR / kDkvThreads, RPP = kDkvThreads / CPR, KS = DP / 16, DT = DP / 32;
  constexpr bool BOTH = DP == 64;
  constexpr int GROUPS = BOTH ? 1 : 2, SUMS = BOTH ? 2 : 1;
  constexpr int FIELDS = FORM & FORM_BIAS ? 8 : 4, INFO = kTileRows * FIELDS * 4;  // bytes of a tile's row_info
  using Frag = typename Frag8<T>::type;
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * STAGE];  // q of two stages, dout of two
  __shared__ __attribute__((aligned(16))) unsigned char info[2 * INFO];
  __shared__ int bounds[8][3], spoilt;
  constexpr bool LIFTS = !std::is_same<T, bf16>::value;
  const Args& p = b.f;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool for_dv = !BOTH && wave >= 4;
  const int part = BOTH ? wave >> 1 : ((wave >> 1) & 1) * 2;  // the first of its GROUPS groups of 32 rows

  const Place place = place_of(blockIdx.x, p.batch * p.kv_heads, b.key_tiles * b.dkv_splits);
  const int z = place.piece % b.dkv_splits, turn = place.piece / b.dkv_splits;
  const Entry e = make_entry<false>(p, place.entry / p.kv_heads, place.entry % p.kv_heads);
  const int tile = b.order ? b.order[(long long)e.b * b.key_tiles + turn] : turn;  // (causal: the longest first)
  const int rows = e.tokens * p.group;
  const int block_key = tile * kBlockKeys, key0 = block_key + (wave & 1) * 32, key = key0 + (lane & 31);
  const int block_end = min(block_key + kBlockKeys, e.keys);

  // the first and last groups of 32 rows that see a key of the block, and the largest peak of such groups (as a whole number)
  const int groups = (rows + 31) >> 5;
  const int4* seen = b.seen + (long long)e.b * b.row_groups;
  const float* peaks = b.peak + ((long long)e.b * p.kv_heads + e.kv) * b.row_groups;
  int from = 0x7fffffff, to = 0, peak = 0;
  for (int i = tid; i < groups; i += kDkvThreads)
    if (seen[i].x < block_end && seen[i].y > block_key) {
      from = min(from, i);
      to = i + 1;
      if constexpr (LIFTS) peak = max(peak, __builtin_bit_cast(int, peaks[i]));
    }
  from = wave_min(from);
  to = wave_max(to);
  if constexpr (LIFTS) peak = wave_max(peak);
  if (lane == 0) {
    bounds[wave][0] = from;
    bounds[wave][1] = to;
    bounds[wave][2] = peak;
  }
  Frag kf[KS], vf[KS];
  const int mine = min(key, e.keys - 1);
  load_row_frags<T, DP>(keys_of<T, false>(p, e, p.k, p.ks) + (long long)mine * p.ks.row, half, p.dim, kf);
  load_row_frags<T, DP>(keys_of<T, false>(p, e, p.v, p.vs) + (long long)mine * p.vs.row, half, p.dim, vf);
  if (tid == 0) spoilt = 0;
  if (p.dim < DP)
    for (int i = tid; i < 4 * STAGE / 16; i += kDkvThreads) reinterpret_cast<u32x4*>(smem)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    from = min(from, bounds[i][0]);
    to = max(to, bounds[i][1]);
    if constexpr (LIFTS) peak = max(peak, bounds[i][2]);
  }
  Lift lift(LIFTS ? __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(peak)) : 0.0f);
  from = __builtin_amdgcn_readfirstlane(from);
  to = __builtin_amdgcn_readfirstlane(to);
  const int first_tile = from < to ? from >> 2 : 0, last_tile = from < to ? (to + 3) >> 2 : 0;
  const int t0 = min(last_tile, first_tile + z * b.dkv_share), t1 = z + 1 < b.dkv_splits ? min(last_tile, t0 + b.dkv_share) : last_tile;

  const int load_row = tid / CPR, load_chunk = (tid % CPR) ^ swz<CPR>(load_row);
  const bool loads = load_chunk * 8 < p.dim;
  const unsigned lds0 = lds_address(smem), lds = lds0 + wave * 1024, info0 = lds_address(info);
  const ReadMap<DP> map(lane);
  const T* qbase = reinterpret_cast<const T*>(p.q) + (long long)e.b * p.qs.batch + (long long)e.kv * p.group * p.qs.head;
  const T* gbase = reinterpret_cast<const T*>(b.dout) + (long long)e.b * b.dos.batch + (long long)e.kv * p.group * b.dos.head;
  // regular: RPP rows lie alike everywhere
  const int load_token = p.d_group.div(load_row), load_head = load_row - load_token * p.group, step_tokens = p.d_group.div(RPP);
  const unsigned qoff = ((unsigned)load_token * (unsigned)p.qs.row + (unsigned)load_head * (unsigned)p.qs.head + load_chunk * 8) * 2;
  const unsigned goff = ((unsigned)load_token * (unsigned)b.dos.row + (unsigned)load_head * (unsigned)b.dos.head + load_chunk * 8) * 2;
  const float* rinfo = row_info<FORM>(b, e, 0, 0);
  auto request = [&](int t) {
    const unsigned dst = lds + (t & 1) * STAGE;
    if (wave * 1024 < INFO) DirectLoad::at(rinfo + (long long)t * (INFO / 4), tid * 16, info0 + (t & 1) * INFO + wave * 1024);
    if (b.regular && (t + 1) * kTileRows <= rows) {
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (loads) {
          const long long token = (long long)(t * NL + i) * step_tokens;
          DirectLoad::at(qbase + token * p.qs.row, qoff, dst + i * (kDkvThreads * 16));
          DirectLoad::at(gbase + token * b.dos.row, goff, dst + 2 * STAGE + i * (kDkvThreads * 16));
        }
      return;
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = min(t * kTileRows + i * RPP + load_row, rows - 1);  // (rows past the last: the last again, seen by nobody)
      const int token = p.d_group.div(r), head = r - token * p.group;
      const T* qr = qbase + (long long)head * p.qs.head + (long long)token * p.qs.row;
      const T* gr = gbase + (long long)head * b.dos.head + (long long)token * b.dos.row;
      if (loads) {
        DirectLoad::at(qr + load_chunk * 8, dst + i * (kDkvThreads * 16));
        DirectLoad::at(gr + load_chunk * 8, dst + 2 * STAGE + i * (kDkvThreads * 16));
      }
    }
  };

  const Score<FORM> all_scores(p, 0.0f);
  // (which groups of 32 rows take part: asked for a tile ahead, and in scalar registers before the next tile's loads are under way, for
  // which the compiler would otherwise wait)
  const auto in_scalars = [](const int4& v) {
    return int4{__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z),
                __builtin_amdgcn_readfirstlane(v.w)};
  };
  f32x16 acc[SUMS][DT];  // dK, dV or both, transposed: lane = key
  bool again = false;
  for (;;) {
#pragma unroll
    for (int i = 0; i < SUMS; ++i)
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][d][r] = 0.0f;
    int4 next0 = {0, 0, 0, 0}, next1 = next0;
    if (t0 < t1) {  // (without queries there is no list of them)
      next0 = seen[min(4 * t0 + part, groups - 1)];
      next1 = seen[min(4 * t0 + part + GROUPS - 1, groups - 1)];
    }
    settle();
    if (t0 < t1) request(t0);
    for (int t = t0; t < t1; ++t) {
      wait_all_and_meet();
      if (__builtin_expect(again, 0)) {
        keep_finite<T, kDkvThreads, NL>(smem + (t & 1) * STAGE);
        keep_finite<T, kDkvThreads, NL>(smem + (t & 1) * STAGE + 2 * STAGE);
        __syncthreads();
      }
      const int4 seen0 = in_scalars(next0), seen1 = in_scalars(next1);
      if (t + 1 < t1) {
        request(t + 1);
        next0 = seen[min(4 * t + 4 + part, groups - 1)];
        next1 = seen[min(4 * t + 4 + part + GROUPS - 1, groups - 1)];
      }
      const unsigned qs = lds0 + (t & 1) * STAGE, gs = qs + 2 * STAGE;
      const float* of_rows = reinterpret_cast<const float*>(info + (t & 1) * INFO);
#pragma unroll 1
      for (int c = 0; c < GROUPS; ++c) {
        const int row = (part + c) * 32, behind = t * kTileRows + row + 32;
        if ((c ? seen1.x : seen0.x) >= key0 + 32 || (c ? seen1.y : seen0.y) <= key0 || behind - 32 >= rows) continue;
        const bool masked = (c ? seen1.z : seen0.z) > key0 || (c ? seen1.w : seen0.w) < key0 + 32 || behind > rows;
        f32x16 s, dp;
        Frag gcol[BOTH ? 4 : 1], qcol[BOTH ? 4 : 1];
        if constexpr (BOTH) {
          // (one workgroup to a compute unit: what a wavefront reads from LDS is asked for well before its products, which the scheduler
          // does not do of itself; 24 heads over 1449 keys 89 to 84 us)
          Frag a[KS], g[KS];
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) a[ks] = row_frag<T, DP>(map, qs, row, ks);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) g[ks] = row_frag<T, DP>(map, gs, row, ks);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) s = mfma_op(a[ks], kf[ks], s);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) dp = mfma_op(g[ks], vf[ks], dp);
#pragma unroll
          for (int i = 0; i < 4; ++i) qcol[i] = col_frag<T, DP>(map, qs, row + (i / DT) * 16, i % DT);
#pragma unroll
          for (int i = 0; i < 4; ++i) gcol[i] = col_frag<T, DP>(map, gs, row + (i / DT) * 16, i % DT);
          __builtin_amdgcn_sched_barrier(0);
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) s = mfma_op(row_frag<T, DP>(map, qs, row, ks), kf[ks], s);
          if (!for_dv) {
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) dp = mfma_op(row_frag<T, DP>(map, gs, row, ks), vf[ks], dp);
          }
        }
        Score<FORM> score = all_scores;
        float derivative[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {  // P
          const float* quad = of_rows + (row / 4 + 2 * g + half) * (FIELDS * 4);
          const f32x4 lse = *reinterpret_cast<const f32x4*>(quad);
          f32x4 slope = {0, 0, 0, 0};
          int4 at = {0, 0, 0, 0};
          if constexpr (FORM & FORM_BIAS) {
            at = *reinterpret_cast<const int4*>(quad + 16);
            slope = *reinterpret_cast<const f32x4*>(quad + 20);
          }
          const int at4[4] = {at.x, at.y, at.z, at.w};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int r = 4 * g + u;
            if constexpr (FORM == FORM_PLAIN) {
              s[r] = exp2_fast(__builtin_fmaf(s[r], score.factor, -lse[u]));
            } else {
              score.slope = slope[u];
              s[r] = exp2_fast(score(s[r], (float)(at4[u] - key), derivative[r]) - lse[u]);
            }
          }
        }
        if (!for_dv) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {  // dS
            const f32x4 delta = *reinterpret_cast<const f32x4*>(of_rows + (row / 4 + 2 * g + half) * (FIELDS * 4) + 4);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const int r = 4 * g + u;
              dp[r] = __builtin_fmaf(dp[r], 1.0f / kLift, -delta[u]);
              if constexpr (LIFTS) dp[r] *= lift.by;
              dp[r] *= s[r];
              if constexpr (FORM & FORM_CAP) dp[r] *= derivative[r];
            }
          }
        }
        if (!BOTH && !for_dv) s = dp;
        if (masked) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float* quad = of_rows + (row / 4 + 2 * g + half) * (FIELDS * 4);
            const int4 first = *reinterpret_cast<const int4*>(quad + 8), count = *reinterpret_cast<const int4*>(quad + 12);
            const int f4[4] = {first.x, first.y, first.z, first.w}, c4[4] = {count.x, count.y, count.z, count.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const bool in = (unsigned)(key - f4[u]) < (unsigned)c4[u];
              // (a row that sees one key has no whole tile, and comes by here)
              const float by = for_dv ? 1.0f : unless_alone(c4[u]);
              s[4 * g + u] = in ? (BOTH ? s[4 * g + u] : s[4 * g + u] * by) : 0.0f;
              if constexpr (BOTH) dp[4 * g + u] = in ? dp[4 * g + u] * by : 0.0f;
            }
          }
        }
        if constexpr (LIFTS)
          if (__builtin_expect(again, 0) && !for_dv) lift.fit(BOTH ? dp : s, acc[0]);
        Frag w[SUMS][2];  // both: dS, P
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          w[0][r >> 3][r & 7] = from_f32<T>(BOTH ? dp[r] : s[r]);
          if constexpr (BOTH) w[SUMS - 1][r >> 3][r & 7] = from_f32<T>(s[r]);
        }
        const unsigned from_rows = for_dv ? gs : qs;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            if constexpr (BOTH) {
              acc[0][d] = mfma_op(qcol[h * DT + d], w[0][h], acc[0][d]);
              acc[SUMS - 1][d] = mfma_op(gcol[h * DT + d], w[SUMS - 1][h], acc[SUMS - 1][d]);
            } else {
              acc[0][d] = mfma_op(col_frag<T, DP>(map, from_rows, row + h * 16, d), w[0][h], acc[0][d]);
            }
          }
      }
    }
    if (again) break;
    bool finite = all_finite(acc[0]);
    if constexpr (BOTH) finite &= all_finite(acc[SUMS - 1]);
    if (!__all(finite) && lane == 0) spoilt = 1;
    __syncthreads();
    again = __builtin_amdgcn_readfirstlane(spoilt);
    if (__builtin_expect(!again, 1)) break;
  }
  if (LIFTS && !for_dv) {
    const float by = 1.0f / lift.by;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[0][d][r] *= by;
  }
  // the wavefronts of a sum meet: four (two of them onto two, one onto one), or two
  const int lead = BOTH ? 0 : wave & 4;  // the first wavefront of the kind
#pragma unroll
  for (int step = BOTH ? 4 : 2; step >= 2; step >>= 1) {
    __syncthreads();
    const int mate = wave - lead;
    f32x4* meet = reinterpret_cast<f32x4*>(smem) + ((mate & (step - 1)) + lead / 2) * (SUMS * DT * 4 * 64) + lane;
    if (mate >= step && mate < 2 * step) {
#pragma unroll
      for (int i = 0; i < SUMS; ++i)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            meet[((i * DT + d) * 4 + g) * 64] = f32x4{acc[i][d][4 * g], acc[i][d][4 * g + 1], acc[i][d][4 * g + 2], acc[i][d][4 * g + 3]};
    }
    __syncthreads();
    if (mate < step) {
#pragma unroll
      for (int i = 0; i < SUMS; ++i)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 other = meet[((i * DT + d) * 4 + g) * 64];
#pragma unroll
            for (int u = 0; u < 4; ++u) acc[i][d][4 * g + u] += other[u];
          }
    }
  }
  if (part) return;
#pragma unroll
  for (int i = 0; i < SUMS; ++i) {
    const bool is_dv = for_dv || i == 1;
    if (__builtin_expect(again && is_dv, 0)) {
      // (a key that is not finite has a weight of 0 here, or all its rows are NaN)
      bool odd_key = false;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int u = 0; u < 8; ++u) odd_key |= !(__builtin_fabsf(to_f32(kf[ks][u])) < __builtin_huge_valf());
      odd_key |= __shfl_xor((int)odd_key, 32);
      settle_odd<DP>(acc[i], odd_gradients<T, DP, FORM>(b, e, key, t0 * kTileRows, min(t1 * kTileRows, rows), key < e.keys && !odd_key), half);
    }
    if (key >= e.keys) continue;
    if (b.dkv_splits > 1) {
      store_part<DT>(dkv_part<DP>(b, z, e, key) + (is_dv ? DP : 0), acc[i], half);
    } else {
      const Strides& to_s = is_dv ? b.dvs : b.dks;
      T* out = reinterpret_cast<T*>(is_dv ? b.dv : b.dk) + (long long)e.b * to_s.batch + (long long)e.kv * to_s.head + (long long)key * to_s.row;
      store_columns<T, DT>(out, acc[i], half, p.dim, is_dv ? 1.0f / kLift : p.scale);
    }
  }
}

// The splits of a key's two sums, in ascending order; one wavefront a key.
template <typename T, int DP>
__global__ __launch_bounds__(256) void dkv_join_kernel(const BackArgs b) {
  constexpr int E = DP / 64;
  const Args& p = b.f;
  const int lane = threadIdx.x & 63;
  const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= (long long)p.batch * p.kv_heads * p.seq_k) return;
  const int entry = (int)(at / p.seq_k), key = (int)(at - (long long)entry * p.seq_k);
  const Entry e = make_entry<false>(p, entry / p.kv_heads, entry % p.kv_heads);
  float dk[E], dv[E];
#pragma unroll
  for (int i = 0; i < E; ++i) dk[i] = dv[i] = 0.0f;
#pragma unroll 4
  for (int z = 0; z < b.dkv_splits; ++z) {
    const float* from = dkv_part<DP>(b, z, e, key) + lane * E;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      dk[i] += from[i];
      dv[i] += from[DP + i];
    }
  }
  T* to_k = reinterpret_cast<T*>(b.dk) + (long long)e.b * b.dks.batch + (long long)e.kv * b.dks.head + (long long)key * b.dks.row;
  T* to_v = reinterpret_cast<T*>(b.dv) + (long long)e.b * b.dvs.batch + (long long)e.kv * b.dvs.head + (long long)key * b.dvs.row;
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (lane * E + i < p.dim) {
      to_k[lane * E + i] = from_f32<T>(dk[i] * p.scale);
      to_v[lane * E + i] = from_f32<T>(dv[i] * (1.0f / kLift));
    }
}

template <typename T, int DP, int FORM>
hipError_t launch(const BackArgs& b, hipStream_t stream) {
  const Args& p = b.f;
  const long long entries = (long long)p.batch * p.kv_heads;
  if (p.seq_q > 0) {
    const dim3 grid((unsigned)(entries * p.row_tiles * b.dq_splits));
    if (b.dq_pairs)
      hipLaunchKernelGGL((dq_kernel<T, DP, FORM, 2>), grid, dim3(512), 0, stream, b);
    else
      hipLaunchKernelGGL((dq_kernel<T, DP, FORM, 1>), grid, dim3(256), 0, stream, b);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (b.dq_splits > 1) {
      const long long rows = entries * p.seq_q * p.group;
      hipLaunchKernelGGL((dq_join_kernel<T, DP>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, b);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
  }
  if (p.seq_k > 0) {
    hipLaunchKernelGGL((dkv_kernel<T, DP, FORM>), dim3((unsigned)(entries * b.key_tiles * b.dkv_splits)), dim3(kDkvThreads), 0, stream, b);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (b.dkv_splits > 1) {
      hipLaunchKernelGGL((dkv_join_kernel<T, DP>), dim3((unsigned)((entries * p.seq_k + 3) / 4)), dim3(256), 0, stream, b);
      return hipGetLastError();
    }
  }
  return hipSuccess;
}
template <typename T, int DP>
hipError_t dispatch_form(int form, const BackArgs& b, hipStream_t stream) {
  switch (form) {
    case FORM_PLAIN: return launch<T, DP, FORM_PLAIN>(b, stream);
    case FORM_BIAS: return launch<T, DP, FORM_BIAS>(b, stream);
    case FORM_CAP: return launch<T, DP, FORM_CAP>(b, stream);
    case FORM_WIDE: return launch<T, DP, FORM_WIDE>(b, stream);
    default: return launch<T, DP, FORM_CAP | FORM_BIAS>(b, stream);
  }
}
template <typename T>
hipError_t dispatch(int form, const BackArgs& b, hipStream_t stream) {
  return padded_dim(b.f.dim) == 128 ? dispatch_form<T, 128>(form, b, stream) : dispatch_form<T, 64>(form, b, stream);
}

long long row_groups_of(long long rows) { return (rows + 31) / 32; }
long long order_bytes(long long batch, long long key_tiles) { return (batch * key_tiles * 4 + 15) / 16 * 16; }
long long peak_bytes(long long entries, long long row_groups) { return (entries * row_groups * 4 + 15) / 16 * 16; }
// (of all forms: with a bias twice the fields)
long long info_bytes(long long entries, long long rows) { return entries * ((rows + 127) / 128 * 128) * 8 * 4; }

// How the two kernels' work is cut.
//   dQ: tiles of 128 rows, in pairs of wavefronts while a compute unit each takes them (its registers leave room for one such workgroup, at 64
//   dimensions too, where the tail of up to 320 is short enough: heads of 1021 rows, pairs and without, us: 288 tiles 46 and 47, 320 47 and
//   48, 416 56 and 49, 496 57 and 49), and then as many splits of at least 4 tiles of 128 keys as find a compute unit each.  A whole pass
//   (forward, dQ, dK and dV) without and with pairs, us: 6 entries of 3146 rows of 96 dimensions 170 and 152, 9 of 3332 at 128 470 and 429;
//   36 of 1024 at 128, 288 tiles, 202 and 227, and so without; one fits worse, 4 entries of 1472 rows over 184 keys 47 and 50.
//   dK and dV: tiles of 64 keys, and where they leave compute units without work splits of at least 2 tiles of 128 rows: 256 workgroups
//   (512 at 64 dimensions: 24 heads over 1449 keys 199 us for 211).  With 512 of at least 4 everywhere: the first of the passes above 220 for 190,
//   the second 486 for 449, and 285 for 271 of 2 entries of 6599 rows.
struct BackCut {
  int row_tiles, key_tiles, dq_splits, dq_share, dkv_splits, dkv_share;
  bool dq_pairs;
  long long part_bytes;
};
void split(long long tiles, long long n, int& splits, int& share) {
  n = std::max(1LL, n);
  share = (int)std::max(1LL, (tiles + n - 1) / n);
  splits = (int)std::max(1LL, (tiles + share - 1) / share);
}
BackCut cut_backward(long long entries, long long rows, long long keys, int dp) {
  BackCut c;
  c.row_tiles = (int)((rows + 127) / 128);
  c.key_tiles = (int)((keys + kBlockKeys - 1) / kBlockKeys);
  const long long row_blocks = std::max(1LL, entries * c.row_tiles), key_blocks = std::max(1LL, entries * c.key_tiles);
  c.dq_pairs = row_blocks <= (dp == 64 ? 320 : 256) && keys > kTileKeys;
  const long long tile_keys = c.dq_pairs ? 2 * kTileKeys : kTileKeys;
  const long long tiles = std::max(1LL, (keys + tile_keys - 1) / tile_keys), row_tiles = std::max(1LL, (rows + kTileRows - 1) / kTileRows);
  split(tiles, c.dq_pairs ? std::min(256 / row_blocks, tiles / 4) : 1, c.dq_splits, c.dq_share);
  const long long wanted = dp == 64 ? 512 : 256;
  split(row_tiles, std::min((wanted + key_blocks - 1) / key_blocks, row_tiles / 2), c.dkv_splits, c.dkv_share);
  const long long dq = c.dq_splits > 1 ? c.dq_splits * entries * rows * dp * 4 : 0;
  const long long dkv = c.dkv_splits > 1 ? c.dkv_splits * entries * keys * dp * 8 : 0;
  c.part_bytes = std::max(dq, dkv);
  return c;
}

}  // namespace

extern "C" {

int64_t hidet_attention_backward_workspace_bytes(int64_t batch, int64_t heads, int64_t kv_heads, int64_t seq_q, int64_t seq_k,
                                                 int64_t head_dim) {
  if (batch <= 0 || kv_heads <= 0 || heads <= 0 || heads % kv_heads != 0 || seq_q <= 0 || seq_k < 0 || head_dim <= 0 || head_dim > 128) return 0;
  const long long group = heads / kv_heads;
  if (group >= kMaxRows || seq_q >= kMaxRows || seq_k >= kMaxRows || !fits_cut(batch, kv_heads, seq_q * group, seq_k)) return 0;
  const BackCut c = cut_backward(batch * kv_heads, seq_q * group, seq_k, padded_dim(head_dim));
  const long long row_groups = row_groups_of(seq_q * group);
  return info_bytes(batch * kv_heads, seq_q * group) + peak_bytes(batch * kv_heads, row_groups) + batch * row_groups * 16 +
         order_bytes(batch, c.key_tiles) + c.part_bytes;
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
  if (!fits_cut(batch, kv_heads, seq_q * group, seq_k)) return HIDET_ERR_UNSUPPORTED;
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
    b.info = static_cast<float*>(workspace);
    char* peak = static_cast<char*>(workspace) + info_bytes(batch * kv_heads, seq_q * group);
    b.peak = reinterpret_cast<float*>(peak);
    b.seen = reinterpret_cast<int4*>(peak + peak_bytes(batch * kv_heads, row_groups_of(seq_q * group)));
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
  const BackCut c = cut_backward(batch * kv_heads, seq_q * group, seq_k, padded_dim(head_dim));
  p.row_tiles = c.row_tiles;
  b.row_groups = (int)row_groups_of(seq_q * group);
  b.key_tiles = c.key_tiles;
  b.dq_pairs = c.dq_pairs;
  b.dq_splits = c.dq_splits;
  b.dq_share = c.dq_share;
  // (without queries there is no workspace, and nothing to add up)
  b.dkv_splits = seq_q > 0 ? c.dkv_splits : 1;
  b.dkv_share = c.dkv_share;
  if (seq_q > 0) {
    char* order = reinterpret_cast<char*>(b.seen) + batch * b.row_groups * 16;
    // (more workgroups than begin at once)
    if (options->ranges && batch * kv_heads * c.key_tiles * c.dkv_splits > 256) b.order = reinterpret_cast<int*>(order);
    b.part = reinterpret_cast<float*>(order + order_bytes(batch, c.key_tiles));
  }
  const auto near = [&](const Strides& s) { return s.row < (1LL << 23) && s.head < (1LL << 23); };
  b.regular = group <= 32 && 32 % group == 0 && near(p.qs) && near(b.dos);
  if (batch * kv_heads * std::max((long long)c.row_tiles * c.dq_splits, (long long)c.key_tiles * c.dkv_splits) > kMaxBlocks) return HIDET_ERR_UNSUPPORTED;
  const int form = form_of(options);
  const hipStream_t s = (hipStream_t)stream;
  const hipError_t e = dtype == HIDET_F16 ? dispatch<f16>(form, b, s) : dispatch<bf16>(form, b, s);
  return e == hipSuccess ? HIDET_OK : HIDET_ERR_LAUNCH;
}

}  // extern "C"
