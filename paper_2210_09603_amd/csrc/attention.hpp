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
// bf16 holds values as large as fp32: P is kept below 1 by taking 2^8 more from every score, which costs it nothing.  (fp16 has bits for
// neither.)
template <typename T>
constexpr float kAbove = std::is_same<T, bf16>::value ? kSlack : 0.0f;

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
  int share;              // tiles of keys of a split
  int flat;               // pieces of a ragged batch, see flat_kernel; 0: splits
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

// Where a lane reads, as byte offsets from a tile: worked out once, so that a read costs an addition at most.
template <int DP>
struct ReadMap {
  static constexpr int CPR = DP / 8, KS = DP / 16, DT = DP / 32;
  unsigned row[KS];     // as a row: chunk column 2 * step + lane / 32 of row lane % 32
  unsigned col[DT][2];  // as a column: 4 rows of the group's 16 lanes, and those 8 below
  __device__ __forceinline__ explicit ReadMap(int lane) {
    const int r = lane & 31, s = lane & 15, h = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) row[ks] = (r * CPR + ((2 * ks + h) ^ swz<CPR>(r))) * 16;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int chunk = d * 4 + 2 * ((lane >> 4) & 1) + ((s & 3) >> 1), c = 8 * i + 4 * h + (s >> 2);
        col[d][i] = (c * CPR + (chunk ^ swz<CPR>(c))) * 16 + (s & 1) * 8;
      }
  }
};
typedef __attribute__((address_space(3))) const u32x4 LdsChunk;
typedef __attribute__((address_space(3))) i16x4 LdsQuad;

// Rows first..first+31 of the tile at LDS address `tile` as the operand with a row per lane.
template <typename T, int DP>
__device__ __forceinline__ typename Frag8<T>::type row_frag(const ReadMap<DP>& m, unsigned tile, int first, int step) {
  return __builtin_bit_cast(typename Frag8<T>::type, *(LdsChunk*)(__UINTPTR_TYPE__)(tile + m.row[step] + first * DP * 2));
}
// Columns 32 * dt..+31 as the operand with a column per lane; its 8 values are rows first + {0..3, 8..11} + 4 * (lane / 32).
template <typename T, int DP>
__device__ __forceinline__ typename Frag8<T>::type col_frag(const ReadMap<DP>& m, unsigned tile, int first, int dt) {
  u32x2 part[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    part[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad*)(__UINTPTR_TYPE__)(tile + m.col[dt][i] + first * DP * 2)));
  const u32x4 v = {part[0][0], part[0][1], part[1][0], part[1][1]};
  return __builtin_bit_cast(typename Frag8<T>::type, v);
}

// ---- direct loads into LDS ----------------------------------------------------------------------------------------
// Lane l of a wavefront fills the 16 bytes at lds + 16 * l; lanes that are switched off fill nothing.  The loads write no
// register, so that nothing has to stay reserved while they run; they are waited for by wait_all_and_meet or wait_loads.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// (the same in all lanes, which the compiler does not always see)
__device__ __forceinline__ unsigned in_scalar(unsigned v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const void* in_scalar(const void* v) {
  const unsigned long long bits = (unsigned long long)v;
  return (const void*)(((unsigned long long)in_scalar((unsigned)(bits >> 32)) << 32) | in_scalar((unsigned)bits));
}
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
        : "v"(offset), "s"(in_scalar(base)), "s"(in_scalar(lds))
        : "memory", "m0");
  }
  // from an address of the lane's own
  static __device__ __forceinline__ void at(const void* address, unsigned lds) {
    asm volatile(
        "s_mov_b32 m0, %1\n\t"
        "s_nop 3\n\t"
        "global_load_lds_dwordx4 %0, off"
        :
        : "v"(address), "s"(in_scalar(lds))
        : "memory", "m0");
  }
};
#pragma clang diagnostic pop
// All loads of this wavefront have arrived and all its LDS reads are back; then the workgroup meets.
__device__ __forceinline__ void wait_all_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Nothing is outstanding, and the compiler knows it: where a register that it loaded was first used inside a loop, it would wait
// there for all loads in flight, the direct ones among them, in every round (a capped prompt of 4096 x 32 heads: 240 us).
__device__ __forceinline__ void settle() { __builtin_amdgcn_s_waitcnt(0); }

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
// What a score is besides scale * q.k, a template parameter of the kernels: an exponential and a reciprocal an element for the cap
// (half of such a kernel's vector time), two instructions for the bias.
enum : int { FORM_PLAIN = 0, FORM_BIAS = 1, FORM_CAP = 2, FORM_WIDE = 7 };  // PLAIN: scale > 0 and nothing else; WIDE: both, see Score

// The score to base 2 of a product: scale and cap as they stand in Args, slope for the query's head.
//
// cap tanh(y) = cap - 2 cap / (e^2y + 1) is off by some 2^-23 of the cap (2^-22 if every rounding falls the same way), whatever the
// score is: up to kWideCap that is 8e-6, as much as scores of the cap's size are off anyhow.  Under larger caps (WIDE) scores below a
// quarter of them are taken by tanh(y) = y (1 - y^2/3 + 2 y^4/15 - 17 y^6/315 + 62 y^8/2835 - ...), off by 4e-8 of itself at y = 1/4,
// times cap / y, so that a cap that no score comes near leaves them as they are.  (A cap of 1e4, scores of 1 to 3: off by 1e-3 in the
// first form.)  A form of its own: as a branch in the kernels of usual caps it took 25 registers of theirs.
constexpr float kWideCap = 64.0f;
template <int FORM>
struct Score {
  float factor;  // to base 2; with a cap: 2 log2(e) scale / cap, so that exp2 of it is e^2y
  float cap;     // cap * log2(e)
  float slope;   // slope * log2(e)
  float small, ratio;  // WIDE: without the cap, to base 2; y of a product
  __device__ __forceinline__ Score(const Args& p, float slope_of_head) {
    factor = FORM & FORM_CAP ? 2.0f * kLog2e * p.scale / p.softcap : p.scale * kLog2e;
    cap = p.softcap * kLog2e;
    slope = slope_of_head * kLog2e;
    small = p.scale * kLog2e;
    ratio = p.scale / p.softcap;
  }
  // 1 / (e^2y + 1), of which tanh(y) is 1 - 2 r and its derivative 4 r (1 - r)
  __device__ __forceinline__ float share(float dot) const { return __builtin_amdgcn_rcpf(exp2_fast(dot * factor) + 1.0f); }
  // (distances beyond 2^24 are rounded to fp32, 2^-24 of themselves)
  __device__ __forceinline__ float biased(float x, float distance) const {
    if constexpr (FORM & FORM_BIAS) return __builtin_fmaf(-slope, __builtin_fabsf(distance), x);
    return x;
  }
  __device__ __forceinline__ float operator()(float dot, float distance) const {
    float derivative;
    return (*this)(dot, distance, derivative);
  }
  // the same with its derivative to the uncapped score
  __device__ __forceinline__ float operator()(float dot, float distance, float& derivative) const {
    derivative = 1.0f;
    if constexpr (!(FORM & FORM_CAP)) return biased(dot * factor, distance);
    const float r = share(dot);
    float x = __builtin_fmaf(-2.0f * cap, r, cap);
    derivative = 4.0f * r * (1.0f - r);
    if constexpr (FORM == FORM_WIDE) {
      const float y = dot * ratio, y2 = y * y;
      const float to_y = __builtin_fmaf(
          y2, __builtin_fmaf(y2, __builtin_fmaf(y2, __builtin_fmaf(y2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
      const bool flat = __builtin_fabsf(y) < 0.25f;
      x = flat ? dot * small * to_y : x;
      derivative = flat ? __builtin_fmaf(-(y * to_y), y * to_y, 1.0f) : derivative;
    }
    return biased(x, distance);
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
// The keys from lo to hi that the query at position `at` sees where there are no ranges; lo and hi never fall from a query to the next.
// None: lo >= hi.
template <bool PAGED>
__device__ __forceinline__ void seen_from(const Args& p, const Entry& e, int at, int& lo, int& hi) {
  lo = max(p.window ? at - p.window + 1 : 0, 0);
  if (PAGED || p.causal)
    hi = at + 1;
  else
    hi = p.window && p.window < e.keys - at ? at + p.window : e.keys;  // (at + window may pass 32 bits)
  hi = min(hi, e.keys);
}
__device__ __forceinline__ Row place_of_row(const Args& p, const Entry& e, int r) {
  const int token = p.d_group.div(r);
  return Row{token, e.kv * p.group + (r - token * p.group), 0, 0};
}
template <bool PAGED>
__device__ __forceinline__ Row make_row(const Args& p, const Entry& e, int r) {
  Row w = place_of_row(p, e, r);
  if (!PAGED && p.ranges) {
    const int* range = p.ranges + ((long long)e.b * p.seq_q + w.token) * 2;
    w.lo = max(range[0], 0);
    w.hi = min(range[1], e.keys);
  } else {
    seen_from<PAGED>(p, e, w.token + e.shift, w.lo, w.hi);
  }
  if (w.lo >= w.hi) w.lo = w.hi = 0;
  return w;
}

// Of the rows first..last: from the first to the last key + 1 that any of them sees, and the keys that all of them see.
struct Seen {
  int lo, hi, full_lo, full_hi;
};
// `w`: one of the rows in each half of a wavefront, all of them in its 32 lanes
template <bool PAGED>
__device__ __forceinline__ Seen seen_by(const Args& p, const Entry& e, const Row& w, int first, int last) {
  Seen s;
  if (!PAGED && p.ranges) {
    s.lo = wave_min(w.lo < w.hi ? w.lo : 0x7fffffff);
    s.hi = wave_max(w.hi);
    s.full_lo = wave_max(w.lo);
    s.full_hi = wave_min(w.hi);
  } else {
    seen_from<PAGED>(p, e, p.d_group.div(first) + e.shift, s.lo, s.full_hi);
    seen_from<PAGED>(p, e, p.d_group.div(last) + e.shift, s.full_lo, s.hi);
  }
  return s;
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

// Tiles of TILE keys from `begin` on: how many there are up to `end`, and key i of tile t, `end` at the farthest.  A cache's keys may
// end at 2^31 - 1, and what lies a tile behind them passes 32 bits with a sign.
template <int TILE>
__device__ __forceinline__ int tiles_of(int begin, int end) {
  return (int)(((unsigned)(end - begin) + TILE - 1) / TILE);
}
template <int TILE>
__device__ __forceinline__ int key_at(int begin, int t, int i, int end) {
  return (int)min((unsigned)begin + (unsigned)t * TILE + (unsigned)i, (unsigned)end);
}

// Where a key is.  What is asked of the table and what is made of it are apart: a loop asks one tile ahead of the keys' own loads, and
// using the answer at once would wait for every load in flight.
struct KeyPlace {
  int page, row;  // row: slot of the page, or the key where there are no pages
};
template <bool PAGED>
__device__ __forceinline__ KeyPlace find_key(const Args& p, const Entry& e, int j) {
  if constexpr (PAGED) {
    const int at = p.d_page.div(j);
    return KeyPlace{e.table[at], j - at * p.page_size};
  } else {
    return KeyPlace{0, j};
  }
}
template <bool PAGED>
__device__ __forceinline__ bool is_there(const Args& p, const KeyPlace& k) {  // (its page is one of the cache's)
  return !PAGED || (unsigned)k.page < (unsigned)p.num_pages;
}
// its offset from the entry's keys, in elements; of no page: some page's
template <bool PAGED>
__device__ __forceinline__ long long key_offset(const Args& p, const Strides& s, const KeyPlace& k) {
  return (PAGED ? (long long)(is_there<PAGED>(p, k) ? k.page : 0) * s.batch : 0) + (long long)k.row * s.row;
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
    const float next = now == kNoMax ? 0.0f : now * factor + kAbove<T>;
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
template <typename T, int DP, int FORM, int KT>
__device__ __forceinline__ void softmax_tile(State<T, DP>& st, f32x16 (&s)[KT], typename Frag8<T>::type (&p)[2 * KT], const Score<FORM>& score,
                                             int first, int lo, int hi, int at, int half, bool masked, unsigned long long there) {
  if constexpr (FORM != FORM_PLAIN) {
    const float distance = (float)(at - first - 4 * half);
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = score(s[t][r], distance - (float)(32 * t + 8 * (r >> 2) + (r & 3)));
  }
  if (masked) {
    const unsigned from = (unsigned)lo - (unsigned)first - 4u * half;
    const unsigned count = (unsigned)(hi - lo);
    const unsigned long long mine = there >> (4 * half);
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = 32 * t + 8 * (r >> 2) + (r & 3);
        s[t][r] = (unsigned)j - from < count && ((mine >> j) & 1) ? s[t][r] : kNoMax;
      }
  }
  float top = s[0][0];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
  top = max_of_halves(top);
  const float factor = FORM != FORM_PLAIN ? 1.0f : score.factor;
  // (a first maximum is larger than none by any measure)
  if (__any((top - st.top) * factor > kSlack || (st.top == kNoMax && top != kNoMax))) st.raise(top, factor);
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float e = FORM != FORM_PLAIN ? exp2_fast(s[t][r] - st.shift) : exp2_fast(__builtin_fmaf(s[t][r], factor, -st.shift));
      sum[r & 3] += e;
      p[2 * t + (r >> 3)][r & 7] = from_f32<T>(e);
    }
  st.sum += (sum[0] + sum[1]) + (sum[2] + sum[3]);
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

// ---- what comes out not finite -------------------------------------------------------------------------------------------------
// A tile multiplies the values of keys that a query does not see by weights of 0, and where such a value is infinite or NaN the sum
// becomes NaN.  What comes out finite was not touched by any.  Of the rest:
//   - A score that is NaN or +inf makes the row's sum of weights NaN, and the row is NaN, whatever else it saw.
//   - Otherwise the workgroup goes over its keys a second time, with 0 for what is not finite of the values: that gives every row what it
//     would have been without (the same bits).  One pass over the values of keys that are seen then finds those that are not finite: in a
//     dimension in which a row sees one, that is its result -- infinite, or NaN if it sees both infinities or a NaN.
// So infinities and NaN cost a call a few times its time, whichever they are, and what they do not reach keeps its bits.  (A causal prompt of
// 4096, 16 heads of 128 dimensions, 120 us: with one infinite value 590, one in each key 1200, all of them NaN 260; of the last key alone
// 38 ms when such rows were computed one by one.)

// A lane's number that the compiler knows nothing of: what follows from it is worked out behind this, and not before the tiles, whose loop
// has no registers to keep it in.
__device__ __forceinline__ int worked_out_here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Sets of a vector's dimensions, as ballots of lanes that hold DP / 64 each give them: dimension (DP / 64) lane + u is bit `lane` of set u.
template <int DP>
struct Dims {
  static constexpr int E = DP / 64;
  unsigned long long of[E];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int u = 0; u < E; ++u) of[u] = 0;
  }
  // A transposed accumulator has dimension 32 t + 8 g + 4 half + i in register 4 g + i of tile t: of set i % E the bit below, counted from
  // the first of the half.
  static __device__ __forceinline__ constexpr int bit(int t, int r) { return (32 * t + 8 * (r >> 2) + (r & 3)) / E; }
  static __device__ __forceinline__ int first(int half) { return 4 / E * half; }
};
// Sums of what is not finite: which dimensions hold +inf, -inf, NaN.
template <int DP>
struct OddSums {
  Dims<DP> plus, minus, nan;
  __device__ __forceinline__ void clear() {
    plus.clear();
    minus.clear();
    nan.clear();
  }
  // v: of a vector, dimensions (DP / 64) lane + u, the same vector in all lanes; adds it where `to` says so
  __device__ __forceinline__ void add(const float (&v)[DP / 64], bool to) {
#pragma unroll
    for (int u = 0; u < DP / 64; ++u) {
      const unsigned long long p = __ballot(v[u] == __builtin_huge_valf()), m = __ballot(v[u] == -__builtin_huge_valf()), n = __ballot(v[u] != v[u]);
      plus.of[u] |= to ? p : 0;
      minus.of[u] |= to ? m : 0;
      nan.of[u] |= to ? n : 0;
    }
  }
  __device__ __forceinline__ void add_nan() {
#pragma unroll
    for (int u = 0; u < DP / 64; ++u) nan.of[u] = ~0ull;
  }
};
template <int DT>
__device__ __forceinline__ bool all_finite(const f32x16 (&acc)[DT]) {
  bool finite = true;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) finite &= __builtin_fabsf(acc[t][i]) < __builtin_huge_valf();
  return finite;
}
// Whether more of them may change anything.
template <int DP>
__device__ __forceinline__ bool any_but_nan(const OddSums<DP>& sums, int dim) {
  bool any = false;
#pragma unroll
  for (int u = 0; u < DP / 64; ++u) any |= (~sums.nan.of[u] & ~0ull >> (64 - dim / (DP / 64))) != 0;
  return any;
}
// Puts the sums in their places.
template <int DP>
__device__ __forceinline__ void settle_odd(f32x16 (&acc)[DP / 32], const OddSums<DP>& sums, int half) {
  const float inf = __builtin_huge_valf();
#pragma unroll
  for (int u = 0; u < Dims<DP>::E; ++u) {
    const unsigned long long plus = sums.plus.of[u] >> Dims<DP>::first(half), minus = sums.minus.of[u] >> Dims<DP>::first(half);
    const unsigned long long nan = sums.nan.of[u] >> Dims<DP>::first(half) | (plus & minus);
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int r = u; r < 16; r += Dims<DP>::E) {
        float x = acc[t][r];
        const unsigned long long bit = 1ull << Dims<DP>::bit(t, r);
        x = plus & bit ? inf : x;
        x = minus & bit ? -inf : x;
        x = nan & bit ? __builtin_nanf("") : x;
        acc[t][r] = x;
      }
  }
}

// What lane's row, if it asks, sees of values that are not finite, of keys from `from` on and before `to`, which the workgroup went over.
template <typename T, int DP, bool PAGED>
__device__ __forceinline__ OddSums<DP> odd_values(const Args& p, const Entry& e, const Row& w, int from, int to, bool ask) {
  constexpr int E = DP / 64, U = 8;
  struct __attribute__((packed, aligned(2))) Own {
    T x[E];
  };
  const int lane = worked_out_here(threadIdx.x & 63);
  const bool has = lane * E < p.dim;
  const T* k = keys_of<T, PAGED>(p, e, p.k, p.ks) + (has ? lane * E : 0);
  const T* v = keys_of<T, PAGED>(p, e, p.v, p.vs) + (has ? lane * E : 0);
  OddSums<DP> sums;
  sums.clear();
  const int first = max(from, wave_min(ask ? w.lo : to)), last = min(to, wave_max(ask ? w.hi : from));
  const unsigned count = last > first ? last - first : 0;
#pragma unroll 1
  for (unsigned i = 0; i < count; i += U) {
    Own key[U], value[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      KeyPlace place = find_key<PAGED>(p, e, first + (int)min(i + u, count - 1));
      if constexpr (PAGED) place.page = __builtin_amdgcn_readfirstlane(place.page);
      key[u] = *reinterpret_cast<const Own*>(k + key_offset<PAGED>(p, p.ks, place));
      value[u] = *reinterpret_cast<const Own*>(v + key_offset<PAGED>(p, p.vs, place));
      there[u] = is_there<PAGED>(p, place);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[E];
      bool odd_key = false, odd = false;
#pragma unroll
      for (int c = 0; c < E; ++c) {
        x[c] = has ? to_f32(value[u].x[c]) : 0.0f;
        odd |= !(__builtin_fabsf(x[c]) < __builtin_huge_valf());
        odd_key |= !(__builtin_fabsf(has ? to_f32(key[u].x[c]) : 0.0f) < __builtin_huge_valf());
      }
      // (a key that is not finite has a score of -inf here, and no weight: with any other the row were NaN)
      if (__any(odd) && !__any(odd_key)) {
        const int j = first + (int)min(i + u, count - 1);
        sums.add(x, ask && there[u] && j >= w.lo && j < w.hi);
      }
    }
    if (!__any(ask && any_but_nan(sums, p.dim))) break;
  }
  return sums;
}

// 16-bit numbers, 8 of them, with 0 for what is not finite.
template <typename T>
__device__ __forceinline__ u32x4 finite_ones(u32x4 v) {
  constexpr unsigned EXPONENT = std::is_same<T, bf16>::value ? 0x7f80 : 0x7c00;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((v[i] & EXPONENT) == EXPONENT) v[i] &= 0xffff0000u;
    if ((v[i] & (EXPONENT << 16)) == EXPONENT << 16) v[i] &= 0xffffu;
  }
  return v;
}
// The chunks of a tile that this thread's loads filled, of N threads.
template <typename T, int N, int NL>
__device__ __forceinline__ void keep_finite(unsigned char* tile) {
  const unsigned first = worked_out_here(threadIdx.x) * 16;
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    u32x4* at = reinterpret_cast<u32x4*>(tile + i * N * 16 + first);
    *at = finite_ones<T>(*at);
  }
}

// ---- results of a wavefront's 32 rows ---------------------------------------------------------------------------------------
// Stores the finished output, or the sums of a split, from `to_rows` of row 0 on.  `r0`: the first row; `again`: the sums are those of
// finite values alone, of keys from `from` on and before `to`.
template <typename T, int DP, bool PAGED, int FORM>
__device__ __forceinline__ void finish(const Args& p, const Entry& e, State<T, DP>& st, int r0, int rows, int from, int to, const Part& to_rows,
                                       bool partial, bool again) {
  const int lane = worked_out_here(threadIdx.x & 63), half = lane >> 5, r = r0 + (lane & 31);
  const float sum = sum_of_halves(st.sum);
  if (__builtin_expect(again, 0)) {
    const Row w = make_row<PAGED>(p, e, min(r, rows - 1));
    settle_odd<DP>(st.o, odd_values<T, DP, PAGED>(p, e, w, from, to, sum > 0.0f), half);
  }
  if (r >= rows) return;
  if (partial) {
    const Part part = {to_rows.sums + (long long)r * DP, to_rows.stat + r * 2LL};
    if (sum > 0.0f)  // (the sums of nothing are not read)
#pragma unroll
      for (int t = 0; t < State<T, DP>::DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 v = {st.o[t][4 * g], st.o[t][4 * g + 1], st.o[t][4 * g + 2], st.o[t][4 * g + 3]};
          *reinterpret_cast<f32x4*>(part.sums + 32 * t + 8 * g + 4 * half) = v;
        }
    if (half == 0) {
      part.stat[0] = sum > 0.0f ? st.shift : sum == 0.0f ? kNoMax : sum;
      part.stat[1] = again ? -sum : sum;  // (see Joined)
    }
    return;
  }
  const float by = sum > 0.0f ? 1.0f / sum : sum;  // (0: nothing was seen; NaN: so is the row)
  const Row w = place_of_row(p, e, r);
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
  if (half == 0 && p.lse) p.lse[lse_offset<PAGED>(p, e, w)] = sum > 0.0f ? (st.shift + __builtin_log2f(sum)) * kLn2 : sum == 0.0f ? kNoMax : sum;
}

// ---- the kernel of many rows ------------------------------------------------------------------------------------------------
// A workgroup of 4 wavefronts works on 128 rows, 32 a wavefront, and walks over the keys that one of them sees in tiles of 64,
// which arrive in LDS by direct loads one tile ahead (2 stages of 16 KB of keys and of values at 128 dimensions: two workgroups a
// compute unit, so that one's products run beside the other's exponentials).  Where there is not a second workgroup for every compute
// unit, 8 wavefronts (PAIRS 2): two of them share 32 rows and take the halves of tiles of 128 keys, and meet at the end.
// Workgroups are dealt to the 8 XCDs in turn, each with an L2 of its own: the pieces of an entry (a batch entry's or sequence's kv head)
// go to one XCD, one entry after the other, so that they read its keys from the same L2; every eighth entry, so that the heads of a
// long sequence are spread.  What is left of the entries is cut into contiguous runs.  (Chunks of 4 prompts of 37 to 512 tokens, 8 kv
// heads: 206 us with runs of all of them, which gave two XCDs the longest prompt.)
struct Place {
  int entry, piece;
};
__device__ __forceinline__ Place place_of(int w, int entries, int pieces) {
  const int whole = (entries & ~7) * pieces;
  if (w < whole) {
    const int j = w >> 3, turn = j / pieces;
    return Place{turn * 8 + (w & 7), j - turn * pieces};
  }
  const int n = (entries & 7) * pieces, v = w - whole, x = v & 7, each = n >> 3, rest = n & 7;
  const int at = x * each + min(x, rest) + (v >> 3), turn = at / pieces;
  return Place{(entries & ~7) + turn, at - turn * pieces};
}

// (wavefronts to a SIMD: 64 dimensions fit 128 registers, but for a bias and a cap over pages, and caps of the WIDE form)
template <typename T, int DP, bool PAGED, int FORM, int PAIRS>
__global__ __launch_bounds__(256 * PAIRS, DP == 128 ? 2 : FORM < 3 || (FORM == 3 && !PAGED) ? 4 : 3) void tile_kernel(const Args p) {
  static_assert(PAIRS == 1 || !PAGED, "a wavefront looks up 64 keys");
  constexpr int THREADS = 256 * PAIRS, TILE = kTileKeys * PAIRS;  // keys of a tile
  constexpr int CPR = DP / 8, STAGE = TILE * CPR * 16, NL = TILE * CPR / THREADS, RPP = THREADS / CPR, KS = DP / 16, DT = DP / 32;
  using Frag = typename Frag8<T>::type;
  __shared__ __attribute__((aligned(16))) unsigned char smem[4 * STAGE];  // keys of two stages, values of two
  __shared__ int bounds[4][2], spoilt;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int own = (wave >> 2) * kTileKeys;  // the first of its 64 keys of a tile

  const Place place = place_of(blockIdx.x, p.batch * p.kv_heads, p.row_tiles * p.splits);
  const int z = place.piece % p.splits, tile = p.row_tiles - 1 - place.piece / p.splits;  // (causal: the longest first)
  const Entry e = make_entry<PAGED>(p, place.entry / p.kv_heads, place.entry % p.kv_heads);
  const int rows = e.tokens * p.group, r0 = tile * 128 + (wave & 3) * 32;
  if (tile * 128 >= rows) return;  // (the whole workgroup)

  // (rows past the last are the last again, and not stored)
  const Row w = make_row<PAGED>(p, e, min(r0 + (lane & 31), rows - 1));
  const int at = w.token + e.shift;
  const Seen mine = seen_by<PAGED>(p, e, w, min(r0, rows - 1), min(r0 + 31, rows - 1));
  int begin, end;  // of the workgroup
  if (!PAGED && p.ranges) {
    if (lane == 0 && wave < 4) {
      bounds[wave][0] = mine.lo;
      bounds[wave][1] = mine.hi;
    }
  } else {
    const Seen all = seen_by<PAGED>(p, e, w, tile * 128, min(tile * 128 + 127, rows - 1));
    begin = all.lo;
    end = all.hi;
  }
  State<T, DP> st;
  load_row_frags<T, DP>(reinterpret_cast<const T*>(p.q) + query_offset<PAGED>(p, e, p.qs, w), half, p.dim, st.q);
  const Score<FORM> score(p, p.slopes ? p.slopes[w.head] : 0.0f);
  if (tid == 0) spoilt = 0;
  const bool narrow = p.dim < DP;
  if (narrow)  // the chunks past the head's dimension, which no load fills
    for (int i = tid; i < 4 * STAGE / 16; i += THREADS) reinterpret_cast<u32x4*>(smem)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
  if (!PAGED && p.ranges) {
    begin = min(min(bounds[0][0], bounds[1][0]), min(bounds[2][0], bounds[3][0]));
    end = max(max(bounds[0][1], bounds[1][1]), max(bounds[2][1], bounds[3][1]));
    begin = __builtin_amdgcn_readfirstlane(begin);
    end = __builtin_amdgcn_readfirstlane(end);
  }
  if (begin >= end) begin = end = 0;
  // this split's share of the tiles, the first of which begins with the first key that anyone sees
  const int all = tiles_of<TILE>(begin, end);
  const int t0 = min(all, z * p.share), t1 = z + 1 < p.splits ? min(all, t0 + p.share) : all;

  const T* kbase = keys_of<T, PAGED>(p, e, p.k, p.ks);
  const T* vbase = keys_of<T, PAGED>(p, e, p.v, p.vs);
  const int load_row = tid / CPR, load_chunk = (tid % CPR) ^ swz<CPR>(load_row);
  const bool loads = load_chunk * 8 < p.dim;
  const unsigned lds0 = lds_address(smem), lds = lds0 + wave * 1024;
  const ReadMap<DP> map(lane);
  unsigned koff[NL], voff[NL];
  if constexpr (!PAGED) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      koff[i] = ((unsigned)(i * RPP + load_row) * (unsigned)p.ks.row + load_chunk * 8) * 2;
      voff[i] = ((unsigned)(i * RPP + load_row) * (unsigned)p.vs.row + load_chunk * 8) * 2;
    }
  }
  KeyPlace next = {0, 0};  // paged: where lane l's key of the tile after the next is
  unsigned long long there = ~0ull, there_next = ~0ull;
  auto look_up = [&](int t) {
    if constexpr (PAGED) next = find_key<PAGED>(p, e, key_at<TILE>(begin, t, lane, end - 1));
  };
  auto request = [&](int t) {
    const unsigned to = lds + (t & 1) * STAGE;
    const int first = begin + t * TILE;
    if constexpr (PAGED) {
      there_next = __ballot(is_there<PAGED>(p, next));
      const long long mine_at = key_offset<PAGED>(p, p.ks, next);
      long long off[NL];
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int from = i * RPP + load_row;
        const unsigned low = __shfl((int)(unsigned)mine_at, from), high = __shfl((int)(unsigned)(mine_at >> 32), from);
        off[i] = (long long)(((unsigned long long)high << 32) | low) + load_chunk * 8;
      }
      if (t + 1 < t1) look_up(t + 1);
      if (loads) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          DirectLoad::at(kbase + off[i], to + i * (THREADS * 16));
          DirectLoad::at(vbase + off[i], to + 2 * STAGE + i * (THREADS * 16));
        }
      }
    } else {
      const T* kt = kbase + (long long)first * p.ks.row;
      const T* vt = vbase + (long long)first * p.vs.row;
      const int last = end - 1 - first;
      if (!loads) return;
      if (last >= TILE - 1) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          DirectLoad::at(kt, koff[i], to + i * (THREADS * 16));
          DirectLoad::at(vt, voff[i], to + 2 * STAGE + i * (THREADS * 16));
        }
      } else {  // (keys past the last that anyone sees are that one again)
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const unsigned row = min(i * RPP + load_row, last);
          DirectLoad::at(kt, (row * (unsigned)p.ks.row + load_chunk * 8) * 2, to + i * (THREADS * 16));
          DirectLoad::at(vt, (row * (unsigned)p.vs.row + load_chunk * 8) * 2, to + 2 * STAGE + i * (THREADS * 16));
        }
      }
    }
  };

  settle();
  bool again = false;
  for (;;) {
    st.clear();
    if (t0 < t1) {
      look_up(t0);
      request(t0);
    }
    for (int t = t0; t < t1; ++t) {
      wait_all_and_meet();
      if (__builtin_expect(again, 0)) {
        keep_finite<T, THREADS, NL>(smem + 2 * STAGE + (t & 1) * STAGE);
        __syncthreads();
      }
      there = there_next;
      if (t + 1 < t1) request(t + 1);
      const int first = begin + t * TILE + own;
      if (first >= mine.hi || first <= mine.lo - kTileKeys) continue;
      const unsigned keys = lds0 + (t & 1) * STAGE + own * (DP * 2), values = keys + 2 * STAGE;
      f32x16 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[i][r] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s[i] = mfma_op(row_frag<T, DP>(map, keys, i * 32, ks), st.q[ks], s[i]);
      }
      const bool masked = first < mine.full_lo || first > mine.full_hi - kTileKeys || (PAGED && ~there != 0);
      Frag pf[4];
      softmax_tile<T, DP, FORM, 2>(st, s, pf, score, first, w.lo, w.hi, at, half, masked, there);
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int d = 0; d < DT; ++d) st.o[d] = mfma_op(col_frag<T, DP>(map, values, c * 16, d), pf[c], st.o[d]);
    }
    if (again) break;
    if (__any(!all_finite(st.o) && st.sum < __builtin_huge_valf()) && lane == 0) spoilt = 1;
    __syncthreads();
    again = __builtin_amdgcn_readfirstlane(spoilt);
    if (__builtin_expect(!again, 1)) break;
  }
  if constexpr (PAIRS == 2) {
    __syncthreads();
    float* meet = reinterpret_cast<float*>(smem) + (wave & 3) * (DT * 16 + 2) * 64 + lane;
    if (wave >= 4) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) meet[(d * 16 + r) * 64] = st.o[d][r];
      meet[DT * 16 * 64] = st.top == kNoMax ? kNoMax : st.shift;
      meet[(DT * 16 + 1) * 64] = st.sum;
    }
    __syncthreads();
    if (wave >= 4) return;
    const float other = meet[DT * 16 * 64], own_level = st.top == kNoMax ? kNoMax : st.shift;
    const float top = fmaxf(own_level, other), level = top == kNoMax ? 0.0f : top;
    const float by = own_level == kNoMax ? 0.0f : exp2_fast(own_level - level), by_other = other == kNoMax ? 0.0f : exp2_fast(other - level);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[d][r] = st.o[d][r] * by + meet[(d * 16 + r) * 64] * by_other;
    st.sum = st.sum * by + meet[(DT * 16 + 1) * 64] * by_other;
    st.shift = level;
  }
  finish<T, DP, PAGED, FORM>(p, e, st, r0, rows, key_at<TILE>(begin, t0, 0, end), key_at<TILE>(begin, t1, 0, end),
                                part_of<DP>(p, e.b, e.kv, z, 0), p.splits > 1, again);
}

// ---- the kernel of few rows ---------------------------------------------------------------------------------------------------
// At most 32 rows, over many keys: memory bound, so that what counts are the bytes in flight.  A wavefront streams tiles of 32 keys of
// its own, without meeting the others before the end: whole rows through registers, asked for one tile ahead (16 KB a wavefront, 128 KB
// a compute unit at 128 dimensions), into 16 KB of LDS of its own, where the products read them as rows and as columns.  Workgroups
// of 4 wavefronts, so that one begins and ends beside another.
constexpr int kStreamWaves = 4, kStreamKeys = 32;

// What the wavefronts of a workgroup have for themselves, and to meet in.
template <int DP>
struct StreamLds {
  static constexpr int TILE = kStreamKeys * DP * 2, JOIN = 32 * (DP + 4) * 4;  // JOIN: fp32 sums of 32 rows
  static constexpr int BYTES = kStreamWaves * 2 * TILE > kStreamWaves / 2 * JOIN ? kStreamWaves * 2 * TILE : kStreamWaves / 2 * JOIN;
  __attribute__((aligned(16))) unsigned char smem[BYTES];
  float stat[kStreamWaves][32][2];
  int spoilt[kStreamWaves];
};
// Rows r0.. of an entry over tiles t0..t1 - 1 of the keys that they see.
template <typename T, int DP, bool PAGED, int FORM>
__device__ __forceinline__ void stream_tiles(const Args& p, StreamLds<DP>& lds, const Entry& e, int r0, int t0, int t1, const Part& to_rows,
                                             bool partial) {
  constexpr int CPR = DP / 8, NL = kStreamKeys * CPR / 64, RPP = 64 / CPR, KS = DP / 16, DT = DP / 32;
  constexpr int TILE = StreamLds<DP>::TILE, JOIN = StreamLds<DP>::JOIN;
  using Frag = typename Frag8<T>::type;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = e.tokens * p.group;
  unsigned char* smem = lds.smem;
  auto& stat = lds.stat;
  const Row w = make_row<PAGED>(p, e, min(r0 + (lane & 31), rows - 1));
  const int at = w.token + e.shift;
  const Seen seen = seen_by<PAGED>(p, e, w, r0, min(r0 + 31, rows - 1));
  const int end = seen.hi, begin = min(seen.lo, end);
  const int all = tiles_of<kStreamKeys>(begin, end);
  t0 = min(t0, all);
  t1 = min(t1, all);
  const T* kbase = keys_of<T, PAGED>(p, e, p.k, p.ks);
  const T* vbase = keys_of<T, PAGED>(p, e, p.v, p.vs);
  unsigned char* mine = smem + wave * 2 * TILE;
  const unsigned keys = lds_address(mine), values = keys + TILE;
  const int load_row = lane / CPR, load_chunk = lane % CPR;
  const bool loads = load_chunk * 8 < p.dim;

  u32x4 kr[NL], vr[NL];
  KeyPlace next = {0, 0};  // of lane's key, lane % 32 of the tile after the next
  unsigned long long there_next = ~0ull;
  auto look_up = [&](int t) { next = find_key<PAGED>(p, e, key_at<kStreamKeys>(begin, t, lane & 31, end - 1)); };
  auto from_lane = [&](long long v, int lane_of_row) {
    const unsigned low = __shfl((int)(unsigned)v, lane_of_row), high = __shfl((int)(unsigned)(v >> 32), lane_of_row);
    return (long long)(((unsigned long long)high << 32) | low) + load_chunk * 8;
  };
  auto request = [&](int t) {
    there_next = __ballot(is_there<PAGED>(p, next));
    const long long ko = key_offset<PAGED>(p, p.ks, next), vo = PAGED ? ko : key_offset<PAGED>(p, p.vs, next);
    if (t + kStreamWaves < t1) look_up(t + kStreamWaves);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const long long k_at = from_lane(ko, i * RPP + load_row), v_at = PAGED ? k_at : from_lane(vo, i * RPP + load_row);
      kr[i] = vr[i] = u32x4{0, 0, 0, 0};
      if (loads) {
        kr[i] = reinterpret_cast<const Chunk16*>(kbase + k_at)->v;
        vr[i] = reinterpret_cast<const Chunk16*>(vbase + v_at)->v;
      }
    }
  };

  int t = t0 + wave;
  if (t < t1) {
    look_up(t);
    request(t);
  }
  State<T, DP> st;
  load_row_frags<T, DP>(reinterpret_cast<const T*>(p.q) + query_offset<PAGED>(p, e, p.qs, w), half, p.dim, st.q);
  const Score<FORM> score(p, p.slopes ? p.slopes[w.head] : 0.0f);
  const ReadMap<DP> map(lane);
  bool again = false;
  for (;;) {
    st.clear();
    for (; t < t1; t += kStreamWaves) {
      const int first = begin + t * kStreamKeys;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int row = i * RPP + load_row, to = (row * CPR + (load_chunk ^ swz<CPR>(row))) * 16;
        *reinterpret_cast<u32x4*>(mine + to) = kr[i];
        *reinterpret_cast<u32x4*>(mine + TILE + to) = vr[i];
      }
      asm volatile("" ::: "memory");  // (a wavefront's LDS accesses run in order: its writes, then its reads)
      if (__builtin_expect(again, 0)) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          u32x4* at = reinterpret_cast<u32x4*>(mine + TILE + (i * 64 + lane) * 16);
          *at = finite_ones<T>(*at);
        }
        asm volatile("" ::: "memory");
      }
      const unsigned long long there = there_next & 0xffffffffull;
      if (t + kStreamWaves < t1) request(t + kStreamWaves);
      f32x16 s[1];
#pragma unroll
      for (int r = 0; r < 16; ++r) s[0][r] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[0] = mfma_op(row_frag<T, DP>(map, keys, 0, ks), st.q[ks], s[0]);
      const bool masked = first < seen.full_lo || first > seen.full_hi - kStreamKeys || (PAGED && there != 0xffffffffull);
      Frag pf[2];
      softmax_tile<T, DP, FORM, 1>(st, s, pf, score, first, w.lo, w.hi, at, half, masked, there);
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int d = 0; d < DT; ++d) st.o[d] = mfma_op(col_frag<T, DP>(map, values, c * 16, d), pf[c], st.o[d]);
      asm volatile("" ::: "memory");
    }
    // the wavefronts' sums meet: all to one maximum, then halves of them into LDS and onto the others
    const int spoilt = !again && __any(!all_finite(st.o) && st.sum < __builtin_huge_valf());
    st.sum = sum_of_halves(st.sum);
    if (half == 0) {
      stat[wave][lane][0] = st.sum == 0.0f ? kNoMax : st.shift;  // (a sum that is NaN counts, though its scores make no maximum)
      stat[wave][lane][1] = st.sum;
    }
    if (lane == 0) lds.spoilt[wave] = spoilt;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int i = 0; i < kStreamWaves; ++i) any |= lds.spoilt[i];
    if (__builtin_expect(!__builtin_amdgcn_readfirstlane(any), 1)) break;
    again = true;
    __syncthreads();  // (what was read above is written again)
    t = t0 + wave;
    if (t < t1) {
      look_up(t);
      request(t);
    }
  }
  float top = kNoMax;
#pragma unroll
  for (int i = 0; i < kStreamWaves; ++i) top = fmaxf(top, stat[i][lane & 31][0]);
  const float level = top == kNoMax ? 0.0f : top;
  const float shrink = st.top == kNoMax ? 0.0f : exp2_fast(st.shift - level);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kStreamWaves; ++i) {
    const float m = stat[i][lane & 31][0];
    sum += m == kNoMax ? 0.0f : stat[i][lane & 31][1] * exp2_fast(m - level);
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
  st.shift = level;
  st.sum = half == 0 ? sum : 0.0f;
  finish<T, DP, PAGED, FORM>(p, e, st, r0, rows, key_at<kStreamKeys>(begin, t0, 0, end), key_at<kStreamKeys>(begin, t1, 0, end), to_rows,
                              partial, again);
}

template <typename T, int DP, bool PAGED, int FORM>
__global__ __launch_bounds__(64 * kStreamWaves, DP == 128 ? 2 : 3) void stream_kernel(const Args p) {
  __shared__ StreamLds<DP> lds;
  // (workgroups share no keys; dealt to the XCDs in turn by kv head and sequence, so that each gets its part of every sequence, the first
  // splits of all before the second ones, which only long sequences have)
  int id = blockIdx.x;
  const int tile = id % p.row_tiles;
  id /= p.row_tiles;
  const int entries = p.batch * p.kv_heads, z = id / entries;
  id -= z * entries;
  const Entry e = make_entry<PAGED>(p, id / p.kv_heads, id % p.kv_heads);
  if (tile * 32 >= e.tokens * p.group) return;
  stream_tiles<T, DP, PAGED, FORM>(p, lds, e, tile * 32, z * p.share, z + 1 < p.splits ? (z + 1) * p.share : 0x7fffffff,
                                   part_of<DP>(p, e.b, e.kv, z, 0), p.splits > 1);
}

// ---- a ragged batch in equal pieces ------------------------------------------------------------------------------------------------
// The sequences' tiles of 32 keys one behind the other, once for every kv head, cut into as many equal pieces as the device takes workgroups:
// one may end one sequence and begin others.  What lies in one piece whole is finished there; of the others each piece
// leaves its sums, and join_flat_kernel adds them in the order of the pieces.  Where the tiles of a sequence begin is worked out by each
// workgroup (lengths are known on the device alone), and left for the second kernel by one of them.
constexpr int kFlatSeqs = 1024;
// (a sequence with new tokens has a tile at least, so that what sees nothing is written as well)
__device__ __forceinline__ int flat_tiles(const Args& p, int s) {
  const Entry e = make_entry<true>(p, s, 0);
  if (e.tokens == 0) return 0;
  int lo, first_hi, last_lo, hi;
  seen_from<true>(p, e, e.shift, lo, first_hi);
  seen_from<true>(p, e, e.tokens - 1 + e.shift, last_lo, hi);
  return max(tiles_of<kStreamKeys>(min(lo, hi), hi), 1);
}
__device__ __forceinline__ int flat_share(const Args& p, int total) { return max((total + p.flat - 1) / p.flat, 1); }
// sums of a piece's part of a sequence: `begins` if the sequence begins in it
template <int DP>
__device__ __forceinline__ Part flat_part(const Args& p, int piece, bool begins, int kv) {
  const long long rows = (long long)p.seq_q * p.group, slot = ((long long)piece * 2 + begins) * p.kv_heads + kv;
  float* part = p.part + (kFlatSeqs + 4);
  return Part{part + slot * rows * DP, part + 2LL * p.flat * p.kv_heads * rows * DP + slot * rows * 2};
}

template <typename T, int DP, int FORM>
__global__ __launch_bounds__(64 * kStreamWaves, DP == 128 ? 2 : 3) void flat_kernel(const Args p) {
  constexpr int THREADS = 64 * kStreamWaves;
  __shared__ StreamLds<DP> lds;
  __shared__ int begins[kFlatSeqs + 1], sums[kStreamWaves], found;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kv = blockIdx.x % p.kv_heads, piece = blockIdx.x / p.kv_heads;
  int total = 0;
  for (int s0 = 0; s0 < p.batch; s0 += THREADS) {
    const int s = s0 + tid;
    int upto = s < p.batch ? flat_tiles(p, s) : 0;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int other = __shfl_up(upto, m);
      if (lane >= m) upto += other;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int before = total;
#pragma unroll
    for (int i = 0; i < kStreamWaves; ++i) {
      if (i < wave) before += sums[i];
      total += sums[i];
    }
    if (s < p.batch) begins[s + 1] = before + upto;
    __syncthreads();
  }
  if (tid == 0) begins[0] = 0;
  total = __builtin_amdgcn_readfirstlane(total);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int s = tid; s <= p.batch; s += THREADS) reinterpret_cast<int*>(p.part)[s] = begins[s];
  const int share = flat_share(p, total);
  if ((long long)piece * share >= total) return;
  int from = piece * share;
  const int till = min(total - from, share) + from;
  for (int s = tid; s < p.batch; s += THREADS)
    if (begins[s] <= from && from < begins[s + 1]) found = s;
  __syncthreads();
  for (int s = __builtin_amdgcn_readfirstlane(found); from < till; ++s) {
    const int first = __builtin_amdgcn_readfirstlane(begins[s]), last = __builtin_amdgcn_readfirstlane(begins[s + 1]);
    if (first == last) continue;
    const int t0 = from - first, t1 = min(last, till) - first;
    stream_tiles<T, DP, true, FORM>(p, lds, make_entry<true>(p, s, kv), 0, t0, t1, flat_part<DP>(p, piece, t0 == 0, kv),
                                    t0 > 0 || t1 < last - first);
    __syncthreads();
    from = first + t1;
  }
}

// A row's sums, of parts that are added to them.  Where fp32 has no weight for a part or for the sums before it, it is 2^-149 if they may not
// be finite, so that they stay so; such a part has left a sum of its weights that is negative.
struct Joined {
  float top = kNoMax, sum = 0.0f;
  f32x4 acc = {0, 0, 0, 0};
  bool odd = false;
  static __device__ __forceinline__ float weight(float x, bool odd) {
    const float w = exp2_fast(x);
    return odd && w == 0.0f ? __builtin_bit_cast(float, 1u) : w;
  }
  __device__ __forceinline__ void add(float m, float its, const f32x4& v) {
    const float next = m > top || m != m ? m : top;
    const float old = top == kNoMax ? 0.0f : weight(top - next, odd), now = weight(m - next, its < 0.0f);
    sum = sum * old + now * __builtin_fabsf(its);
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] = acc[c] * old + now * v[c];
    top = next;
    odd |= its < 0.0f;
  }
};

// One row of a sequence that lies in several pieces, by groups of lanes that take a piece each in turn.
template <typename T, int DP>
__global__ __launch_bounds__(256) void join_flat_kernel(const Args p) {
  constexpr int LANES = DP / 4, GROUPS = 256 / LANES;
  __shared__ __attribute__((aligned(16))) float meet[GROUPS][DP];
  __shared__ float stat[GROUPS][2];
  const int rows = p.seq_q * p.group, r = blockIdx.x % rows, entry = blockIdx.x / rows, s = entry / p.kv_heads, kv = entry - s * p.kv_heads;
  const int* begins = reinterpret_cast<const int*>(p.part);
  const int first = begins[s], last = begins[s + 1], share = flat_share(p, begins[p.batch]);
  if (first == last) return;
  const int from = first / share, to = (last - 1) / share;
  if (from == to) return;  // (finished)
  const Entry e = make_entry<true>(p, s, kv);
  if (r >= e.tokens * p.group) return;
  const int group = threadIdx.x / LANES, d = threadIdx.x % LANES * 4;
  Joined all;
  for (int piece = from + group; piece <= to; piece += GROUPS) {
    const Part part = flat_part<DP>(p, piece, piece == from, kv);
    const float m = part.stat[r * 2];
    if (m != kNoMax) all.add(m, part.stat[r * 2 + 1], *reinterpret_cast<const f32x4*>(part.sums + (long long)r * DP + d));
  }
  *reinterpret_cast<f32x4*>(&meet[group][d]) = all.acc;
  if (d == 0) {
    stat[group][0] = all.top;
    stat[group][1] = all.odd ? -all.sum : all.sum;
  }
  __syncthreads();
  if (group != 0) return;
  for (int g = 1; g < GROUPS; ++g)
    if (stat[g][0] != kNoMax) all.add(stat[g][0], stat[g][1], *reinterpret_cast<const f32x4*>(&meet[g][d]));
  const Row w = place_of_row(p, e, r);
  const bool none = all.top == kNoMax;
  if (d < p.dim) {
    T four[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) four[c] = from_f32<T>(none ? 0.0f : all.acc[c] / all.sum);
    __builtin_memcpy(reinterpret_cast<Chunk8*>(reinterpret_cast<T*>(p.out) + query_offset<true>(p, e, p.os, w) + d), four, 8);
  }
  if (d == 0 && p.lse) p.lse[lse_offset<true>(p, e, w)] = none ? kNoMax : (all.top + __builtin_log2f(all.sum)) * kLn2;
}

// ---- joining the splits -----------------------------------------------------------------------------------------------------
// The order of additions depends on the number of splits alone.  A few splits: DP / 4 lanes a row, whose splits' sums and maxima are
// all asked for at once.
template <typename T, int DP, bool PAGED>
__global__ __launch_bounds__(256) void join_kernel(const Args p) {
  constexpr int LANES = DP / 4, ROWS = 256 / LANES, U = 4;
  const int per_entry = p.seq_q * p.group, d = (threadIdx.x % LANES) * 4;
  const long long row = (long long)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (row >= (long long)p.batch * p.kv_heads * per_entry) return;
  const int entry = (int)(row / per_entry), r = (int)(row - (long long)entry * per_entry);
  const Entry e = make_entry<PAGED>(p, entry / p.kv_heads, entry % p.kv_heads);
  if (r >= e.tokens * p.group) return;
  Joined all;
  for (int z0 = 0; z0 < p.splits; z0 += U) {
    f32x4 v[U];
    float m[U], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const Part part = part_of<DP>(p, e.b, e.kv, min(z0 + u, p.splits - 1), r);
      m[u] = z0 + u < p.splits ? part.stat[0] : kNoMax;
      s[u] = part.stat[1];
      v[u] = *reinterpret_cast<const f32x4*>(part.sums + d);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (m[u] != kNoMax) all.add(m[u], s[u], v[u]);  // (nothing was seen otherwise, and no sums were written)
  }
  const Row w = place_of_row(p, e, r);
  const bool none = all.top == kNoMax;
  if (d < p.dim) {
    T four[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) four[c] = from_f32<T>(none ? 0.0f : all.acc[c] / all.sum);
    __builtin_memcpy(reinterpret_cast<Chunk8*>(reinterpret_cast<T*>(p.out) + query_offset<PAGED>(p, e, p.os, w) + d), four, 8);
  }
  if (d == 0 && p.lse) p.lse[lse_offset<PAGED>(p, e, w)] = none ? kNoMax : (all.top + __builtin_log2f(all.sum)) * kLn2;
}
// Many: a workgroup a row, four splits of it in flight in each half or quarter of a wavefront.
template <typename T, int DP, bool PAGED>
__global__ __launch_bounds__(256) void join_many_kernel(const Args p) {
  constexpr int WAVES = 4, LANES = DP / 4, GROUPS = 64 / LANES;
  __shared__ __attribute__((aligned(16))) float meet[WAVES][DP + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per_entry = p.seq_q * p.group;
  const int entry = blockIdx.x / per_entry, r = blockIdx.x - entry * per_entry;
  const Entry e = make_entry<PAGED>(p, entry / p.kv_heads, entry % p.kv_heads);
  const int d = (lane % LANES) * 4, group = lane / LANES;
  float top = kNoMax, sum = 0.0f;
  f32x4 acc = {0, 0, 0, 0};
  bool nan = false;
  // (the maximum over all splits, by every wavefront)
  for (int z = lane; z < p.splits; z += 64) {
    const float m = part_of<DP>(p, e.b, e.kv, z, r).stat[0];
    nan |= m != m;
    top = fmaxf(top, m);
  }
#pragma unroll
  for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
  nan = __any(nan);
  if (r >= e.tokens * p.group) return;  // (asked behind the first loads: it takes loads of its own)
  const float level = top == kNoMax ? 0.0f : top;
  for (int z0 = wave * 64; z0 < p.splits; z0 += WAVES * 64) {
    float weight = 0.0f;  // (of a split in which nothing was seen, whose sums were not written)
    if (z0 + lane < p.splits) {
      const Part part = part_of<DP>(p, e.b, e.kv, z0 + lane, r);
      if (part.stat[0] != kNoMax) {
        weight = Joined::weight(part.stat[0] - level, part.stat[1] < 0.0f);
        sum += weight * __builtin_fabsf(part.stat[1]);
      }
    }
    const int count = min(64, p.splits - z0);
    for (int i = 0; i < count; i += 4 * GROUPS) {
      f32x4 v[4];
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int z = i + u * GROUPS + group;
        w[u] = __shfl(weight, z & 63);
        v[u] = f32x4{0, 0, 0, 0};
        if (z >= count) w[u] = 0.0f;
        if (w[u] != 0.0f) v[u] = *reinterpret_cast<const f32x4*>(part_of<DP>(p, e.b, e.kv, z0 + z, r).sums + d);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = __builtin_fmaf(w[u], v[u][c], acc[c]);
    }
  }
  sum = wave_sum(sum);
#pragma unroll
  for (int m = 32; m >= LANES; m >>= 1)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] += __shfl_xor(acc[c], m);
  if (group == 0) *reinterpret_cast<f32x4*>(&meet[wave][d]) = acc;
  if (lane == 0) meet[wave][DP] = sum;
  __syncthreads();
  if (wave != 0) return;
  acc = f32x4{0, 0, 0, 0};
  sum = 0.0f;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    acc += *reinterpret_cast<const f32x4*>(&meet[i][d]);
    sum += meet[i][DP];
  }
  if (nan) sum = __builtin_nanf("");
  const Row w = place_of_row(p, e, r);
  const bool none = top == kNoMax && !nan;
  if (group == 0 && d < p.dim) {
    T four[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) four[c] = from_f32<T>(none ? 0.0f : acc[c] / sum);
    __builtin_memcpy(reinterpret_cast<Chunk8*>(reinterpret_cast<T*>(p.out) + query_offset<PAGED>(p, e, p.os, w) + d), four, 8);
  }
  if (lane == 0 && p.lse) p.lse[lse_offset<PAGED>(p, e, w)] = none ? kNoMax : (level + __builtin_log2f(sum)) * kLn2;
}

}  // namespace attn
}  // namespace hidet
