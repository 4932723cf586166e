// What the kernels of fused attention share: tiles in LDS that are read as rows and as columns, direct loads into them, the
// interval of keys that a query sees, and the forward kernels over dense and over paged keys.
//
// A score is x = scale * q.k, capped to cap * tanh(x / cap) where a cap is asked for, minus slope * |distance|; a query's
// output is softmax(x) . v over the keys that it sees.  Every mask that the entry points offer leaves a query one interval of
// keys, so that a mask costs two numbers a query, and tiles outside of every interval are not visited at all.
//
// Scores are computed transposed, S^T = K . Q^T on 32x32x16 matrix instructions: the column of the result that a lane holds is
// one query, so that maximum and sum of the softmax stay within a lane and its partner 32 lanes away, and the 4 consecutive
// keys that a lane holds of every 8 are, in this order, the operand that O^T = V^T . P^T wants when the columns of V come
// from the transposing LDS read in the same order.  P never leaves the registers.
//
// The heads that share keys (heads / kv_heads of them) are rows of the same tile: row r is token r / group, head r % group.
// Keys and values are then read once for all of them, and a decoding step of a group of 8 fills 8 columns instead of 1.
//
// Arithmetic is fp32; exponentials are taken to base 2.  P is rounded to the storage type for the second product (the matrix
// cores take no other), the sum of P is not.
#pragma once

#include "types.hpp"

namespace hidet {
namespace attn {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNoMax = -__builtin_huge_valf();
constexpr int kTileKeys = 64;
// A running maximum is replaced only by one that is 2^8 times as large: P then stays below 2^8, which both storage types
// hold, and most tiles leave the output's registers alone.
constexpr float kSlack = 8.0f;

struct Strides {
  long long batch, head, row;  // elements
};

struct Args {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;             // [batch][heads][seq_q] (paged: [tokens][heads]); may be null
  const float* slopes;    // [heads]; may be null
  const int* ranges;      // [batch][seq_q][2]; may be null
  float* part;            // splits > 1: [split][kv row][DP] sums, then [split][kv row][2] maxima and sums
  Strides qs, ks, vs, os;  // paged: k and v [page][head][slot]
  const int* starts;      // paged: [seqs + 1]
  const int* lengths;     // paged: [seqs]
  const int* tables;      // paged: [seqs][table_stride]
  long long table_stride;
  int table_width, num_pages, page_size, tokens;
  FastDiv d_page, d_group;
  int batch, heads, kv_heads, group, seq_q, seq_k, dim;
  int causal, window;     // window 0: none
  int row_tiles, splits;
  float scale, softcap;   // softcap 0: none
};

// ---- tiles in LDS -------------------------------------------------------------------------------------------------
// Rows of CPR 16-byte chunks without padding, chunk c of row r at position c ^ swz(r).  The same tile is read in two ways:
// a row per lane (32 consecutive rows, one chunk column) and, transposing, 4 rows x 32 bytes a group of 16 lanes, two
// neighbouring groups side by side.  swz keeps 16 consecutive rows apart for the first and, for the second, gives 4 consecutive
// rows pairs of chunks that stay apart from their neighbours' (0, 3, 5, 6 against 1, 2, 4, 7 where a row covers all banks).
template <int CPR>
__device__ __forceinline__ constexpr int swz(int row) {
  if constexpr (CPR == 16)
    return ((0xCA60 >> (4 * (row & 3))) & 15) ^ (((row >> 2) & 1) << 1) ^ ((row >> 3) & 1);
  else
    return (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
}

template <typename T>
struct Frag8;
template <>
struct Frag8<f16> {
  using type = f16x8;
};
template <>
struct Frag8<bf16> {
  using type = bf16x8;
};

// Rows first..first+31 as the operand with a row per lane: chunk column 2 * step + lane / 32.
template <typename T, int CPR>
__device__ __forceinline__ typename Frag8<T>::type row_frag(const unsigned char* tile, int lane, int first, int step) {
  const int row = lane & 31;
  const int c = (2 * step + (lane >> 5)) ^ swz<CPR>(row);
  return __builtin_bit_cast(typename Frag8<T>::type, *reinterpret_cast<const u32x4*>(tile + ((first + row) * CPR + c) * 16));
}

// Columns 32 * dt..+31 as the operand with a column per lane; its 8 values are rows first + {0..3, 8..11} + 4 * (lane / 32).
template <typename T, int CPR>
__device__ __forceinline__ typename Frag8<T>::type col_frag(const unsigned char* tile, int lane, int first, int dt) {
  const int s = lane & 15, h = lane >> 5;
  const int chunk = dt * 4 + 2 * ((lane >> 4) & 1) + ((s & 3) >> 1);
  u32x2 part[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 8 * i + 4 * h + (s >> 2);
    const unsigned char* at = tile + ((first + row) * CPR + (chunk ^ swz<CPR>(row))) * 16 + (s & 1) * 8;
    part[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                            (__attribute__((address_space(3))) i16x4*)(const_cast<unsigned char*>(at))));
  }
  const u32x4 v = {part[0][0], part[0][1], part[1][0], part[1][1]};
  return __builtin_bit_cast(typename Frag8<T>::type, v);
}

// ---- direct loads into LDS ----------------------------------------------------------------------------------------
// Lane l of a wavefront fills the 16 bytes at lds + 16 * l; lanes that are switched off fill nothing.  The loads write no
// register, so that nothing has to stay reserved while they run; they are waited for by wait_all_and_meet or wait_loads.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
struct DirectLoad {
  // from `offset` bytes behind `base`, which the scalar unit copies (a load may read a scalar register that a vector instruction has
  // written five wait states later at the earliest)
  static __device__ __forceinline__ void at(const void* base, unsigned offset, unsigned lds) {
    const void* copy;
    asm volatile(
        "s_mov_b32 m0, %3\n\t"
        "s_mov_b64 %0, %2\n\t"
        "global_load_lds_dwordx4 %1, %0"
        : "=&s"(copy)
        : "v"(offset), "s"(base), "s"(lds)
        : "memory", "m0");
  }
  // from an address of the lane's own
  static __device__ __forceinline__ void at(const void* address, unsigned lds) {
    asm volatile(
        "s_mov_b32 m0, %1\n\t"
        "s_nop 3\n\t"
        "global_load_lds_dwordx4 %0, off"
        :
        : "v"(address), "s"(lds)
        : "memory", "m0");
  }
};
#pragma clang diagnostic pop
// All loads of this wavefront have arrived and all its LDS reads are back; then the workgroup meets.
__device__ __forceinline__ void wait_all_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ unsigned lds_address(const void* p) {
  return (unsigned)(size_t)(__attribute__((address_space(3))) const void*)p;
}

// ---- lanes and their partners ---------------------------------------------------------------------------------------
// lane l and lane l + 32 hold the two halves of a query's keys
__device__ __forceinline__ float max_of_halves(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v = min(v, __shfl_xor(v, m));
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max(int v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v = max(v, __shfl_xor(v, m));
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// ---- scores -----------------------------------------------------------------------------------------------------------
// The score to base 2 of a product: scale and cap as they stand in Args, slope for the query's head.
struct Score {
  float factor;       // to base 2; with a cap: 2 log2(e) scale / cap, so that exp2 of it is e^2y
  float cap;          // cap * log2(e); 0: none
  float slope;        // slope * log2(e)
  __device__ __forceinline__ Score(const Args& p, float slope_of_head) {
    factor = p.softcap > 0 ? 2.0f * kLog2e * p.scale / p.softcap : p.scale * kLog2e;
    cap = p.softcap * kLog2e;
    slope = slope_of_head * kLog2e;
  }
  // tanh(y) = 1 - 2 / (e^2y + 1): off by some 2^-23, which is what the score's own rounding to fp32 is off for scores near
  // the cap
  __device__ __forceinline__ float tanh_of(float dot) const {
    return 1.0f - 2.0f * __builtin_amdgcn_rcpf(exp2_fast(dot * factor) + 1.0f);
  }
  __device__ __forceinline__ float operator()(float dot, int distance) const {
    float x = cap > 0 ? cap * tanh_of(dot) : dot * factor;
    // (no slope: a distance of any size adds nothing, not even to an infinite score)
    return x - slope * (float)(distance < 0 ? -distance : distance);
  }
};

// ---- rows -------------------------------------------------------------------------------------------------------------
// The batch entry (or sequence) that a workgroup works on.
struct Entry {
  int b, kv;        // batch entry, kv head
  int tokens;       // queries of the entry
  int first_token;  // paged: of the entry in q and out
  int keys;         // keys of the entry
  int shift;        // position of query t: t + shift
  const int* table;
};
template <bool PAGED>
__device__ __forceinline__ Entry make_entry(const Args& p, int b, int kv) {
  Entry e;
  e.b = b;
  e.kv = kv;
  if constexpr (PAGED) {
    // (whatever the three lists hold, no index leaves its tensor)
    const int s0 = min(max(p.starts[b], 0), p.tokens), s1 = min(max(p.starts[b + 1], 0), p.tokens);
    e.first_token = s0;
    const int new_tokens = s1 > s0 ? s1 - s0 : 0;
    const long long room = (long long)p.table_width * p.page_size;
    const int length = max(p.lengths[b], 0);
    e.keys = (long long)length < room ? length : (int)room;
    e.shift = length - new_tokens;
    e.tokens = min(new_tokens, p.seq_q);
    e.table = p.tables + (long long)b * p.table_stride;
  } else {
    e.first_token = 0;
    e.tokens = p.seq_q;
    e.keys = p.seq_k;
    e.shift = p.seq_k - p.seq_q;
    e.table = nullptr;
  }
  return e;
}

struct Row {
  int token, head;  // head: of all heads
  int lo, hi;       // keys that it sees: lo <= j < hi; none: 0, 0
};
template <bool PAGED>
__device__ __forceinline__ Row make_row(const Args& p, const Entry& e, int r) {
  Row w;
  w.token = p.d_group.div(r);
  w.head = e.kv * p.group + (r - w.token * p.group);
  const int at = w.token + e.shift;
  if (!PAGED && p.ranges) {
    const int* range = p.ranges + ((long long)e.b * p.seq_q + w.token) * 2;
    w.lo = range[0];
    w.hi = range[1];
  } else {
    // (at + window may pass 32 bits)
    w.lo = p.window ? at - p.window + 1 : 0;
    if (PAGED || p.causal)
      w.hi = at + 1;
    else
      w.hi = p.window && p.window < e.keys - at ? at + p.window : e.keys;
  }
  w.lo = max(w.lo, 0);
  w.hi = min(w.hi, e.keys);
  if (w.lo >= w.hi) w.lo = w.hi = 0;
  return w;
}

template <bool PAGED>
__device__ __forceinline__ long long query_offset(const Args& p, const Entry& e, const Strides& s, const Row& w) {
  if constexpr (PAGED)
    return (long long)(e.first_token + w.token) * s.row + (long long)w.head * s.head;
  else
    return (long long)e.b * s.batch + (long long)w.head * s.head + (long long)w.token * s.row;
}
template <bool PAGED>
__device__ __forceinline__ long long lse_offset(const Args& p, const Entry& e, const Row& w) {
  if constexpr (PAGED)
    return (long long)(e.first_token + w.token) * p.heads + w.head;
  else
    return ((long long)e.b * p.heads + w.head) * p.seq_q + w.token;
}

// Where a key is: its offset from the entry's keys, in elements; `there` says whether its page is one of the cache's.
template <bool PAGED>
__device__ __forceinline__ long long key_offset(const Args& p, const Entry& e, const Strides& s, int j, bool& there) {
  if constexpr (PAGED) {
    const int at = p.d_page.div(j), slot = j - at * p.page_size;
    const int page = e.table[at];
    there = (unsigned)page < (unsigned)p.num_pages;
    return (long long)(there ? page : 0) * s.batch + (long long)slot * s.row;
  } else {
    there = true;
    return (long long)j * s.row;
  }
}
template <typename T, bool PAGED>
__device__ __forceinline__ const T* keys_of(const Args& p, const Entry& e, const void* base, const Strides& s) {
  return reinterpret_cast<const T*>(base) + (PAGED ? 0 : (long long)e.b * s.batch) + (long long)e.kv * s.head;
}

// 16 bytes at element alignment
struct __attribute__((packed, aligned(2))) Chunk16 {
  u32x4 v;
};
struct __attribute__((packed, aligned(2))) Chunk8 {
  u32x2 v;
};

// The 8 * DP / 128 pieces of a query's row that a lane feeds to the scores; zeros past the head's dimension.
template <typename T, int DP>
__device__ __forceinline__ void load_row_frags(const T* row, int half, int dim, typename Frag8<T>::type (&f)[DP / 16]) {
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) {
    const int d = ks * 16 + half * 8;
    u32x4 raw = {0, 0, 0, 0};
    if (d < dim) raw = reinterpret_cast<const Chunk16*>(row + d)->v;
    f[ks] = __builtin_bit_cast(typename Frag8<T>::type, raw);
  }
}

// ---- the state of 32 queries in a wavefront ------------------------------------------------------------------------------
template <typename T, int DP>
struct State {
  static constexpr int DT = DP / 32;
  using Frag = typename Frag8<T>::type;
  Frag q[DP / 16];
  f32x16 o[DT];  // O^T: lane = query, register r of tile t: dimension 32 t + 8 (r / 4) + 4 (lane / 32) + r % 4
  float top;     // running maximum, to base 2; of the products themselves where scores are a positive multiple of them
  float shift;   // what is taken from a score: top * factor, 0 while nothing was seen
  float sum;     // of this lane's half of the keys

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
    top = kNoMax;
    shift = 0.0f;
    sum = 0.0f;
  }
  // A larger maximum: what was summed so far shrinks.
  __device__ __forceinline__ void raise(float tile_top, float factor) {
    const float now = fmaxf(top, tile_top);
    const float next = now == kNoMax ? 0.0f : now * factor;
    const float shrink = top == kNoMax ? 0.0f : exp2_fast(shift - next);  // (nothing was summed: 0 stays 0)
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] *= shrink;
    sum *= shrink;
    top = now;
    shift = next;
  }
};

// A tile of 32 * KT keys: s holds the products with the queries.  P goes to p (the operand of the second product), its sum and
// maximum to the state.  `first`: key of register 0 of lane 0; MASKED: some query does not see some of the keys.
// `there`: bit j: key j of the tile is on a page of the cache (only looked at where MASKED).
template <typename T, int DP, bool EXTRA, int KT>
__device__ __forceinline__ void softmax_tile(State<T, DP>& st, f32x16 (&s)[KT], typename Frag8<T>::type (&p)[2 * KT], const Score& score,
                                             int first, int lo, int hi, int at, int half, bool masked, unsigned long long there) {
  if constexpr (EXTRA) {
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = score(s[t][r], at - (first + 4 * half + 32 * t + 8 * (r >> 2) + (r & 3)));
  }
  if (masked) {
    const int from = lo - first - 4 * half;
    const unsigned count = (unsigned)(hi - lo);
    const unsigned long long mine = there >> (4 * half);
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = 32 * t + 8 * (r >> 2) + (r & 3);
        s[t][r] = (unsigned)(j - from) < count && ((mine >> j) & 1) ? s[t][r] : kNoMax;
      }
  }
  float top = s[0][0];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
  top = max_of_halves(top);
  const float factor = EXTRA ? 1.0f : score.factor;
  // (a first maximum is larger than none by any measure)
  if (__any((top - st.top) * factor > kSlack || (st.top == kNoMax && top != kNoMax))) st.raise(top, factor);
  float sum = 0.0f;
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float e = EXTRA ? exp2_fast(s[t][r] - st.shift) : exp2_fast(__builtin_fmaf(s[t][r], factor, -st.shift));
      sum += e;
      p[2 * t + (r >> 3)][r & 7] = from_f32<T>(e);
    }
  st.sum += sum;
}

// ---- results --------------------------------------------------------------------------------------------------------------
// Where the partial results of a row of split z are.
struct Part {
  float* sums;  // DP of them
  float* stat;  // maximum (to base 2) and sum
};
template <int DP>
__device__ __forceinline__ Part part_of(const Args& p, int b, int kv, int z, int r) {
  const long long per_split = (long long)p.batch * p.kv_heads * p.seq_q * p.group;
  const long long row = (long long)z * per_split + ((long long)b * p.kv_heads + kv) * ((long long)p.seq_q * p.group) + r;
  return Part{p.part + row * DP, p.part + p.splits * per_split * DP + row * 2};
}

// One query again, by all lanes of a wavefront: only the keys that it sees take part, each with its own multiplication.  Where
// a masked key or value is infinite or NaN the tiled products multiply it by a zero and their sums become NaN; the rows that
// come out not finite are computed by this definition instead.  Rare, and slow: a few hundred cycles a key.
template <typename T, int DP, bool PAGED>
__device__ __forceinline__ void row_by_definition(const Args& p, const Entry& e, int r, int from, int to, int z) {
  constexpr int E = DP / 64;
  const int lane = threadIdx.x & 63;
  const Row w = make_row<PAGED>(p, e, r);
  const Score score(p, p.slopes ? p.slopes[w.head] : 0.0f);
  const T* q = reinterpret_cast<const T*>(p.q) + query_offset<PAGED>(p, e, p.qs, w);
  const T* k = keys_of<T, PAGED>(p, e, p.k, p.ks);
  const T* v = keys_of<T, PAGED>(p, e, p.v, p.vs);
  float mine[E], acc[E], top = kNoMax, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int d = lane * E + i;
    mine[i] = d < p.dim ? to_f32(q[d]) : 0.0f;
    acc[i] = 0.0f;
  }
  from = max(from, w.lo);
  to = min(to, w.hi);
  for (int j = from; j < to; ++j) {
    bool there;
    const long long ko = key_offset<PAGED>(p, e, p.ks, j, there);
    if (!there) continue;
    const long long vo = key_offset<PAGED>(p, e, p.vs, j, there);
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (lane * E + i < p.dim) dot = __builtin_fmaf(mine[i], to_f32(k[ko + lane * E + i]), dot);
    const float x = score(wave_sum(dot), w.token + e.shift - j);
    if (x == kNoMax) continue;  // (weight 0: as a masked key)
    if (!(x <= top)) {
      const float shrink = top == kNoMax ? 0.0f : exp2_fast(top - x);
      sum *= shrink;
#pragma unroll
      for (int i = 0; i < E; ++i) acc[i] = top == kNoMax ? 0.0f : acc[i] * shrink;
      top = x;
    }
    const float weight = exp2_fast(x - top);
    sum += weight;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (lane * E + i < p.dim) acc[i] += weight * to_f32(v[vo + lane * E + i]);
    if (sum != sum) break;  // (NaN stays NaN)
  }
  const bool none = top == kNoMax;
  if (sum != sum) {
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = sum;
    top = sum;
  }
  if (p.splits > 1) {
    const Part part = part_of<DP>(p, e.b, e.kv, z, r);
#pragma unroll
    for (int i = 0; i < E; ++i) part.sums[lane * E + i] = acc[i];
    if (lane == 0) {
      part.stat[0] = top;
      part.stat[1] = sum;
    }
    return;
  }
  T* out = reinterpret_cast<T*>(p.out) + query_offset<PAGED>(p, e, p.os, w);
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (lane * E + i < p.dim) out[lane * E + i] = from_f32<T>(none ? 0.0f : acc[i] / sum);
  if (lane == 0 && p.lse) p.lse[lse_offset<PAGED>(p, e, w)] = none ? kNoMax : (top + __builtin_log2f(sum)) * kLn2;
}

// Stores a wavefront's 32 rows: the finished output, or the sums of a split.  `r0`: its first row.
template <typename T, int DP, bool PAGED>
__device__ __forceinline__ void finish(const Args& p, const Entry& e, State<T, DP>& st, int r0, int rows, const Row& w, int from, int to, int z) {
  const int lane = threadIdx.x & 63, half = lane >> 5, r = r0 + (lane & 31);
  const float sum = sum_of_halves(st.sum);
  bool finite = true;
#pragma unroll
  for (int t = 0; t < State<T, DP>::DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) finite &= __builtin_fabsf(st.o[t][i]) < __builtin_huge_valf();
  finite &= __builtin_fabsf(sum) < __builtin_huge_valf();
  const unsigned long long odd = __ballot(!finite);
  unsigned again = (unsigned)odd | (unsigned)(odd >> 32);
  const bool mine = r < rows && !((again >> (lane & 31)) & 1);
  if (p.splits > 1) {
    if (mine) {
      const Part part = part_of<DP>(p, e.b, e.kv, z, r);
#pragma unroll
      for (int t = 0; t < State<T, DP>::DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 v = {st.o[t][4 * g], st.o[t][4 * g + 1], st.o[t][4 * g + 2], st.o[t][4 * g + 3]};
          *reinterpret_cast<f32x4*>(part.sums + 32 * t + 8 * g + 4 * half) = v;
        }
      if (half == 0) {
        part.stat[0] = sum > 0.0f ? st.shift : kNoMax;
        part.stat[1] = sum;
      }
    }
  } else if (mine) {
    const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
    T* out = reinterpret_cast<T*>(p.out) + query_offset<PAGED>(p, e, p.os, w);
#pragma unroll
    for (int t = 0; t < State<T, DP>::DT; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 32 * t + 8 * g + 4 * half;
        T four[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) four[i] = from_f32<T>(st.o[t][4 * g + i] * by);
        if (d < p.dim) __builtin_memcpy(reinterpret_cast<Chunk8*>(out + d), four, 8);
      }
    if (half == 0 && p.lse) p.lse[lse_offset<PAGED>(p, e, w)] = sum > 0.0f ? (st.shift + __builtin_log2f(sum)) * kLn2 : kNoMax;
  }
  again = __builtin_amdgcn_readfirstlane(again);
  while (again) {
    const int i = __builtin_ctz(again);
    again &= again - 1;
    if (r0 + i < rows) row_by_definition<T, DP, PAGED>(p, e, r0 + i, from, to, z);
  }
}

// ---- the kernel of many rows ------------------------------------------------------------------------------------------------
// A workgroup of 4 wavefronts works on 128 rows, 32 a wavefront, and walks over the keys that one of them sees in tiles of 64,
// which arrive in LDS by direct loads one tile ahead (2 stages of 16 KB of keys and of values at 128 dimensions: two workgroups a
// compute unit, so that one's products run beside the other's exponentials).
template <int DP>
constexpr int tile_lds_bytes() {
  return 2 * 2 * kTileKeys * DP * 2;
}

// Workgroups are dealt to the 8 XCDs in turn, each with an L2 of its own: every XCD gets a contiguous run of the work, so that
// the row tiles of a kv head read its keys from the same L2.
__device__ __forceinline__ int xcd_run(int w, int n) {
  const int x = w & 7, each = n >> 3, rest = n & 7;
  return x * each + min(x, rest) + (w >> 3);
}

template <typename T, int DP, bool PAGED, bool EXTRA>
__global__ __launch_bounds__(256, 2) void tile_kernel(const Args p) {
  constexpr int CPR = DP / 8, STAGE = kTileKeys * CPR * 16, NL = kTileKeys * CPR / 256, RPP = 256 / CPR, KS = DP / 16, DT = DP / 32;
  using Frag = typename Frag8<T>::type;
  __shared__ __attribute__((aligned(16))) unsigned char smem[4 * STAGE];  // keys of two stages, values of two
  __shared__ int bounds[4][2];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int id = xcd_run(blockIdx.x, gridDim.x);
  const int z = id % p.splits;
  id /= p.splits;
  const int tile = p.row_tiles - 1 - id % p.row_tiles;  // (causal: the longest first)
  id /= p.row_tiles;
  const Entry e = make_entry<PAGED>(p, id / p.kv_heads, id % p.kv_heads);
  const int rows = e.tokens * p.group, r0 = tile * 128 + wave * 32;
  if (tile * 128 >= rows) return;  // (the whole workgroup)

  // (rows past the last are the last again, and not stored)
  const Row w = make_row<PAGED>(p, e, min(r0 + (lane & 31), rows - 1));
  const int at = w.token + e.shift;
  const bool sees = w.lo < w.hi;
  const int wave_lo = wave_min(sees ? w.lo : 0x7fffffff), wave_hi = wave_max(w.hi);
  const int full_lo = wave_max(w.lo), full_hi = wave_min(w.hi);
  if (lane == 0) {
    bounds[wave][0] = wave_lo;
    bounds[wave][1] = wave_hi;
  }
  State<T, DP> st;
  st.clear();
  load_row_frags<T, DP>(reinterpret_cast<const T*>(p.q) + query_offset<PAGED>(p, e, p.qs, w), half, p.dim, st.q);
  const Score score(p, p.slopes ? p.slopes[w.head] : 0.0f);
  const bool narrow = p.dim < DP;
  if (narrow)  // the chunks past the head's dimension, which no load fills
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
  // this split's share of the tiles, the first of which begins with the first key that anyone sees
  const int all = (end - begin + kTileKeys - 1) / kTileKeys, share = (all + p.splits - 1) / p.splits;
  const int t0 = min(all, z * share), t1 = min(all, t0 + share);

  const T* kbase = keys_of<T, PAGED>(p, e, p.k, p.ks);
  const T* vbase = keys_of<T, PAGED>(p, e, p.v, p.vs);
  const int load_row = tid / CPR, load_chunk = (tid % CPR) ^ swz<CPR>(load_row);
  const bool loads = load_chunk * 8 < p.dim;
  const unsigned lds = lds_address(smem) + wave * 1024;
  unsigned koff[NL], voff[NL];
  if constexpr (!PAGED) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      koff[i] = ((unsigned)(i * RPP + load_row) * (unsigned)p.ks.row + load_chunk * 8) * 2;
      voff[i] = ((unsigned)(i * RPP + load_row) * (unsigned)p.vs.row + load_chunk * 8) * 2;
    }
  }
  // paged: where lane l's key of the tile after the next is
  long long ahead = 0;
  unsigned long long there_next = ~0ull, there_now = ~0ull;
  auto look_up = [&](int t) {
    if constexpr (PAGED) {
      bool there;
      ahead = key_offset<PAGED>(p, e, p.ks, min(begin + t * kTileKeys + lane, end - 1), there);
      there_next = __ballot(there);
    }
  };
  auto request = [&](int t) {
    const unsigned to = lds + (t & 1) * STAGE;
    const int first = begin + t * kTileKeys;
    if constexpr (PAGED) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int from = i * RPP + load_row;
        const unsigned low = __shfl((int)(unsigned)ahead, from), high = __shfl((int)(unsigned)(ahead >> 32), from);
        const long long off = (long long)(((unsigned long long)high << 32) | low) + load_chunk * 8;
        if (loads) {
          DirectLoad::at(kbase + off, to + i * 4096);
          DirectLoad::at(vbase + off, to + 2 * STAGE + i * 4096);
        }
      }
    } else {
      const T* kt = kbase + (long long)first * p.ks.row;
      const T* vt = vbase + (long long)first * p.vs.row;
      const int last = end - 1 - first;  // (keys past the last that anyone sees are that one again)
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        unsigned ko = koff[i], vo = voff[i];
        if (last < kTileKeys - 1) {
          const int row = min(i * RPP + load_row, last);
          ko = ((unsigned)row * (unsigned)p.ks.row + load_chunk * 8) * 2;
          vo = ((unsigned)row * (unsigned)p.vs.row + load_chunk * 8) * 2;
        }
        if (loads) {
          DirectLoad::at(kt, ko, to + i * 4096);
          DirectLoad::at(vt, vo, to + 2 * STAGE + i * 4096);
        }
      }
    }
  };

  if (t0 < t1) {
    look_up(t0);
    there_now = there_next;
    request(t0);
    if (t0 + 1 < t1) look_up(t0 + 1);
  }
  for (int t = t0; t < t1; ++t) {
    wait_all_and_meet();
    const unsigned long long there = there_now;
    if (t + 1 < t1) {
      there_now = there_next;
      request(t + 1);
      if (t + 2 < t1) look_up(t + 2);
    }
    const int first = begin + t * kTileKeys;
    if (first >= wave_hi || first + kTileKeys <= wave_lo) continue;
    const unsigned char* keys = smem + (t & 1) * STAGE;
    const unsigned char* values = keys + 2 * STAGE;
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[i][r] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[i] = mfma_op(row_frag<T, CPR>(keys, lane, i * 32, ks), st.q[ks], s[i]);
    }
    const bool masked = first < full_lo || first + kTileKeys > full_hi || (PAGED && ~there != 0);
    Frag pf[4];
    softmax_tile<T, DP, EXTRA, 2>(st, s, pf, score, first, w.lo, w.hi, at, half, masked, there);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int d = 0; d < DT; ++d) st.o[d] = mfma_op(col_frag<T, CPR>(values, lane, c * 16, d), pf[c], st.o[d]);
  }
  finish<T, DP, PAGED>(p, e, st, r0, rows, w, begin + t0 * kTileKeys, min(end, begin + t1 * kTileKeys), z);
}

// ---- the kernel of few rows ---------------------------------------------------------------------------------------------------
// At most 32 rows, over many keys: memory bound, so that what counts are the bytes in flight.  A wavefront of the 8 in a workgroup
// streams tiles of 32 keys of its own, without meeting the others before the end: keys straight into the registers that the
// products want, values through registers into 8 KB of LDS of its own (they are read as columns), both asked for one tile ahead:
// 16 KB a wavefront, 128 KB a compute unit at 128 dimensions.
constexpr int kStreamWaves = 8, kStreamKeys = 32;

template <typename T, int DP, bool PAGED, bool EXTRA>
__global__ __launch_bounds__(64 * kStreamWaves, 2) void stream_kernel(const Args p) {
  constexpr int CPR = DP / 8, NV = kStreamKeys * CPR / 64, RPP = 64 / CPR, KS = DP / 16, DT = DP / 32;
  constexpr int TILE = kStreamKeys * CPR * 16;
  constexpr int JOIN = 32 * (DP + 4) * 4;  // fp32 sums of 32 rows
  using Frag = typename Frag8<T>::type;
  __shared__ __attribute__((aligned(16))) unsigned char smem[kStreamWaves * TILE > kStreamWaves / 2 * JOIN ? kStreamWaves * TILE : kStreamWaves / 2 * JOIN];
  __shared__ float stat[kStreamWaves][32][2];
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  int id = xcd_run(blockIdx.x, gridDim.x);
  const int z = id % p.splits;
  id /= p.splits;
  const int tile = id % p.row_tiles;
  id /= p.row_tiles;
  const Entry e = make_entry<PAGED>(p, id / p.kv_heads, id % p.kv_heads);
  const int rows = e.tokens * p.group, r0 = tile * 32;
  if (r0 >= rows) return;

  const Row w = make_row<PAGED>(p, e, min(r0 + (lane & 31), rows - 1));
  const int at = w.token + e.shift;
  const bool sees = w.lo < w.hi;
  int begin = wave_min(sees ? w.lo : 0x7fffffff);
  const int end = wave_max(w.hi);
  const int full_lo = wave_max(w.lo), full_hi = wave_min(w.hi);
  if (begin >= end) begin = end;
  State<T, DP> st;
  st.clear();
  load_row_frags<T, DP>(reinterpret_cast<const T*>(p.q) + query_offset<PAGED>(p, e, p.qs, w), half, p.dim, st.q);
  const Score score(p, p.slopes ? p.slopes[w.head] : 0.0f);

  const int all = (end - begin + kStreamKeys - 1) / kStreamKeys, share = (all + p.splits - 1) / p.splits;
  const int t0 = min(all, z * share), t1 = min(all, t0 + share);
  const T* kbase = keys_of<T, PAGED>(p, e, p.k, p.ks);
  const T* vbase = keys_of<T, PAGED>(p, e, p.v, p.vs);
  unsigned char* mine = smem + wave * TILE;
  const int v_row = lane / CPR, v_chunk = lane % CPR;

  u32x4 kr[KS], vr[NV];
  long long ko_next = 0, vo_next = 0;
  bool there_next = true;
  auto look_up = [&](int t) {  // lane's key, lane % 32 of tile t
    const int j = min(begin + t * kStreamKeys + (lane & 31), end - 1);
    bool there;
    ko_next = key_offset<PAGED>(p, e, p.ks, j, there);
    vo_next = PAGED ? ko_next : key_offset<PAGED>(p, e, p.vs, j, there);
    there_next = there;
  };
  auto request = [&]() {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int d = ks * 16 + half * 8;
      kr[ks] = u32x4{0, 0, 0, 0};
      if (d < p.dim) kr[ks] = reinterpret_cast<const Chunk16*>(kbase + ko_next + d)->v;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int from = i * RPP + v_row;
      const unsigned low = __shfl((int)(unsigned)vo_next, from), high = __shfl((int)(unsigned)(vo_next >> 32), from);
      const long long off = (long long)(((unsigned long long)high << 32) | low) + v_chunk * 8;
      vr[i] = u32x4{0, 0, 0, 0};
      if (v_chunk * 8 < p.dim) vr[i] = reinterpret_cast<const Chunk16*>(vbase + off)->v;
    }
  };

  int t = t0 + wave;
  unsigned long long there_now = ~0ull;
  if (t < t1) {
    look_up(t);
    there_now = __ballot(there_next);
    request();
    if (t + kStreamWaves < t1) look_up(t + kStreamWaves);
  }
  for (; t < t1; t += kStreamWaves) {
    const int first = begin + t * kStreamKeys;
    f32x16 s[1];
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[0] = mfma_op(__builtin_bit_cast(Frag, kr[ks]), st.q[ks], s[0]);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int row = i * RPP + v_row;
      *reinterpret_cast<u32x4*>(mine + (row * CPR + (v_chunk ^ swz<CPR>(row))) * 16) = vr[i];
    }
    const unsigned long long there = there_now & 0xffffffffull;
    if (t + kStreamWaves < t1) {
      there_now = __ballot(there_next);
      request();
      if (t + 2 * kStreamWaves < t1) look_up(t + 2 * kStreamWaves);
    }
    const bool masked = first < full_lo || first + kStreamKeys > full_hi || (PAGED && there != 0xffffffffull);
    Frag pf[2];
    softmax_tile<T, DP, EXTRA, 1>(st, s, pf, score, first, w.lo, w.hi, at, half, masked, there);
    asm volatile("" ::: "memory");  // (a wavefront's LDS accesses run in order: its writes, then its reads)
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int d = 0; d < DT; ++d) st.o[d] = mfma_op(col_frag<T, CPR>(mine, lane, c * 16, d), pf[c], st.o[d]);
    asm volatile("" ::: "memory");
  }

  // the wavefronts' sums meet: all to one maximum, then halves of them into LDS and onto the others
  st.sum = sum_of_halves(st.sum);
  if (half == 0) {
    stat[wave][lane][0] = st.top == kNoMax ? kNoMax : st.shift;
    stat[wave][lane][1] = st.sum;
  }
  __syncthreads();
  float top = kNoMax;
#pragma unroll
  for (int i = 0; i < kStreamWaves; ++i) top = fmaxf(top, stat[i][lane & 31][0]);
  const float next = top == kNoMax ? 0.0f : top;
  const float shrink = st.top == kNoMax ? 0.0f : exp2_fast(st.shift - next);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kStreamWaves; ++i) {
    const float m = stat[i][lane & 31][0];
    sum += m == kNoMax ? 0.0f : stat[i][lane & 31][1] * exp2_fast(m - next);
  }
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.o[d][r] *= shrink;
#pragma unroll
  for (int step = kStreamWaves / 2; step >= 1; step >>= 1) {
    if (wave >= step && wave < 2 * step) {
      float* to = reinterpret_cast<float*>(smem) + (wave - step) * (JOIN / 4) + (lane & 31) * (DP + 4) + 4 * half;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4*>(to + 32 * d + 8 * g) = f32x4{st.o[d][4 * g], st.o[d][4 * g + 1], st.o[d][4 * g + 2], st.o[d][4 * g + 3]};
    }
    __syncthreads();
    if (wave < step) {
      const float* from = reinterpret_cast<const float*>(smem) + wave * (JOIN / 4) + (lane & 31) * (DP + 4) + 4 * half;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(from + 32 * d + 8 * g);
#pragma unroll
          for (int i = 0; i < 4; ++i) st.o[d][4 * g + i] += v[i];
        }
    }
    __syncthreads();
  }
  if (wave != 0) return;
  st.top = top;
  st.shift = next;
  st.sum = half == 0 ? sum : 0.0f;
  finish<T, DP, PAGED>(p, e, st, r0, rows, w, begin + t0 * kStreamKeys, min(end, begin + t1 * kStreamKeys), z);
}

// ---- joining the splits -----------------------------------------------------------------------------------------------------
// One wavefront a row: the splits' sums to one maximum, in ascending order.
template <typename T, int DP, bool PAGED>
__global__ __launch_bounds__(256) void join_kernel(const Args p) {
  constexpr int E = DP / 64;
  const int lane = threadIdx.x & 63, per_entry = p.seq_q * p.group;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= (long long)p.batch * p.kv_heads * per_entry) return;
  const int entry = (int)(row / per_entry), r = (int)(row - (long long)entry * per_entry);
  const Entry e = make_entry<PAGED>(p, entry / p.kv_heads, entry % p.kv_heads);
  if (r >= e.tokens * p.group) return;
  const Row w = make_row<PAGED>(p, e, r);
  float top = kNoMax;
  bool nan = false;
  for (int z = 0; z < p.splits; ++z) {
    const float m = part_of<DP>(p, e.b, e.kv, z, r).stat[0];
    nan |= m != m;
    top = fmaxf(top, m);
  }
  const float next = top == kNoMax ? 0.0f : top;
  float sum = 0.0f, acc[E];
#pragma unroll
  for (int i = 0; i < E; ++i) acc[i] = 0.0f;
  for (int z = 0; z < p.splits; ++z) {
    const Part part = part_of<DP>(p, e.b, e.kv, z, r);
    const float m = part.stat[0];
    if (m == kNoMax) continue;
    const float weight = exp2_fast(m - next);
    sum += weight * part.stat[1];
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] += weight * part.sums[lane * E + i];
  }
  if (nan) sum = __builtin_nanf("");
  T* out = reinterpret_cast<T*>(p.out) + query_offset<PAGED>(p, e, p.os, w);
  const bool none = top == kNoMax && !nan;
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (lane * E + i < p.dim) out[lane * E + i] = from_f32<T>(none ? 0.0f : acc[i] / sum);
  if (lane == 0 && p.lse) p.lse[lse_offset<PAGED>(p, e, w)] = none ? kNoMax : (next + __builtin_log2f(sum)) * kLn2;
}

}  // namespace attn
}  // namespace hidet
