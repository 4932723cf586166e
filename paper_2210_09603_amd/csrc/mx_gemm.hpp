// The product of two matrices in blocks of 32 that share a power of two, C = epilogue(A . B^T), on the scaled matrix instruction
// v_mfma_scale_f32_16x16x128_f8f6f4.
//
// What the instruction takes, per operand: lane l holds row l % 16.  In 8 bits its first 16 bytes are k = 16 (l / 16) + 0..15, the last 16 the
// same + 64; in 4 bits its 16 bytes are k = 32 (l / 16) + 0..31.  So a lane takes chunk l / 16 of the row's 128 k, and in 8 bits chunk 4 + l / 16
// too.  The scale of block l / 16 of the row comes from one byte of a register, chosen by the instruction.
//
// Rows are taken in groups of 64 as four fragments f = 0..3 of the rows 4 r + f, r = 0..15.  The scales of rows 4 r .. 4 r + 3 for one
// block are then one 32-bit word of a matrix whose scales lie [block][row], and serve four instructions; and the four columns 4 c .. 4 c + 3
// of C that a lane holds are neighbours: its stores are 8 or 16 bytes wide, 16 lanes fill 128 bytes or more of a row, and nothing is transposed.
//
// K beyond the last block is 0: chunks there are not read, and their scales are those of the last block, so that a NaN among them is one that
// the row has anyhow.  Rows beyond the matrix repeat its last one and are not stored.
#pragma once

#include <utility>

#include "mx.hpp"

namespace hidet {
namespace mx {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// At most 112 bytes: a launch with more takes longer.
struct GemmArgs {
  const unsigned char* a;
  const unsigned char* b;
  const unsigned char* scales_a;
  const unsigned char* scales_b;
  void* c;  // slices > 1: fp32 sums [slice][M][N]
  const void* bias;
  const void* residual;
  unsigned lda, ldb, ld_scales_a, ld_scales_b;  // bytes
  unsigned ldc, ldr;                            // elements
  int M, N, blocks;                             // blocks: of K
  float alpha;
  unsigned flags;  // bits 0-1 dtype of C, 2-3 bias axis, 4 ReLU, 5 rows of C and residual are aligned to 4 elements, 8.. slices
  int slice;       // K steps of 128 of a slice
};
static_assert(sizeof(GemmArgs) <= 112, "a launch with more takes longer");

__host__ __device__ __forceinline__ int slices_of(const GemmArgs& p) { return (int)(p.flags >> 8); }

__host__ __device__ constexpr int hardware_format(int format) { return format == HIDET_MX_E2M1 ? 4 : format; }
__host__ __device__ constexpr bool is_wide(int format) { return format != HIDET_MX_E2M1; }  // 8 bits
__host__ __device__ constexpr int step_bytes(int format) { return is_wide(format) ? 128 : 64; }  // of a row, per step of 128 k

template <class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
// f(0) .. f(N - 1) with the numbers as constants: the instruction's choice of a byte is one
template <int N, class F>
__device__ __forceinline__ void each(F f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}

template <int FORMAT>
struct Fragment {
  u32x4 v[is_wide(FORMAT) ? 2 : 1];
  __device__ __forceinline__ i32x8 operand() const {
    if constexpr (is_wide(FORMAT))
      return i32x8{(int)v[0][0], (int)v[0][1], (int)v[0][2], (int)v[0][3], (int)v[1][0], (int)v[1][1], (int)v[1][2], (int)v[1][3]};
    else
      return i32x8{(int)v[0][0], (int)v[0][1], (int)v[0][2], (int)v[0][3], 0, 0, 0, 0};
  }
};
template <int FA, int FB, int BYTE_A, int BYTE_B>
__device__ __forceinline__ f32x4 multiply(const Fragment<FA>& a, const Fragment<FB>& b, f32x4 c, unsigned scale_a, unsigned scale_b) {
  constexpr int CODE_A = hardware_format(FA), CODE_B = hardware_format(FB);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.operand(), b.operand(), c, CODE_A, CODE_B, BYTE_A, (int)scale_a, BYTE_B, (int)scale_b);
}

// ---- epilogue -----------------------------------------------------------------------------------------------------------
// Columns n .. n + 3 of row m, as the other products finish theirs: alpha, bias, residual, ReLU, one rounding.
template <typename TO>
__device__ __forceinline__ void finish4(const GemmArgs& p, int m, int n, const float (&sum)[4]) {
  struct __attribute__((aligned(4 * sizeof(TO)))) Quad {
    TO e[4];
  };
  const int left = p.N - n;
  if (m >= p.M || left <= 0) return;
  const int axis = (p.flags >> 2) & 3;
  const bool whole = (p.flags & 32) != 0 && left >= 4;
  const TO* bias = reinterpret_cast<const TO*>(p.bias);
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = p.alpha * sum[e];
  if (axis == HIDET_BIAS_PER_ROW) {
    const float b = to_f32(bias[m]);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += b;
  } else if (axis == HIDET_BIAS_PER_COL) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += to_f32(bias[n + (e < left ? e : 0)]);
  }
  if (p.residual) {
    const TO* r = reinterpret_cast<const TO*>(p.residual) + (long long)m * p.ldr + n;
    TO t[4];
    if (whole) {
      *reinterpret_cast<Quad*>(t) = *reinterpret_cast<const Quad*>(r);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = r[e < left ? e : 0];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += to_f32(t[e]);
  }
  TO o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = from_f32<TO>((p.flags & 16) != 0 && v[e] < 0.0f ? 0.0f : v[e]);
  TO* c = reinterpret_cast<TO*>(p.c) + (long long)m * p.ldc + n;
  if (whole) {
    *reinterpret_cast<Quad*>(c) = *reinterpret_cast<const Quad*>(o);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) c[e] = o[e];
  }
}
// f(a value of the type of C)
template <class F>
__device__ __forceinline__ void with_out_type(const GemmArgs& p, F f) {
  const int dtype = p.flags & 3;
  if (dtype == HIDET_F32)
    f(0.0f);
  else if (dtype == HIDET_F16)
    f(f16(0.0f));
  else
    f(bf16(0.0f));
}
// The same columns as raw sums of a slice.
__device__ __forceinline__ void keep4(const GemmArgs& p, int slice, int m, int n, const float (&sum)[4]) {
  const int left = p.N - n;
  if (m >= p.M || left <= 0) return;
  float* c = reinterpret_cast<float*>(p.c) + ((long long)slice * p.M + m) * p.N + n;
  if (left >= 4 && p.N % 4 == 0) {
    *reinterpret_cast<f32x4*>(c) = f32x4{sum[0], sum[1], sum[2], sum[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) c[e] = sum[e];
  }
}

// ---- direct loads into LDS ------------------------------------------------------------------------------------------------
// Lane l fills the 16 (4) bytes at lds + 16 l (4 l); lanes that are switched off fill nothing.  The scalar unit copies the base: a load may
// read a scalar register that a vector instruction has written five wait states later at the earliest.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ unsigned in_scalar(unsigned v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const unsigned char* in_scalar(const unsigned char* v) {
  const unsigned long long bits = (unsigned long long)v;
  return (const unsigned char*)(((unsigned long long)in_scalar((unsigned)(bits >> 32)) << 32) | in_scalar((unsigned)bits));
}
struct DirectLoad {
  static __device__ __forceinline__ void chunks(const unsigned char* base, unsigned offset, unsigned lds) {
    const void* copy;
    asm volatile(
        "s_mov_b32 m0, %3\n\t"
        "s_mov_b64 %0, %2\n\t"
        "global_load_lds_dwordx4 %1, %0"
        : "=&s"(copy)
        : "v"(offset), "s"(in_scalar(base)), "s"(in_scalar(lds))
        : "memory", "m0");
  }
  static __device__ __forceinline__ void words(const unsigned char* base, unsigned offset, unsigned lds) {
    const void* copy;
    asm volatile(
        "s_mov_b32 m0, %3\n\t"
        "s_mov_b64 %0, %2\n\t"
        "global_load_lds_dword %1, %0"
        : "=&s"(copy)
        : "v"(offset), "s"(in_scalar(base)), "s"(in_scalar(lds))
        : "memory", "m0");
  }
};
#pragma clang diagnostic pop
// All loads of this wavefront have arrived and all its LDS accesses are done; then the workgroup meets.
__device__ __forceinline__ void wait_all_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ unsigned lds_address(const void* p) {
  return (unsigned)(size_t)(__attribute__((address_space(3))) const void*)p;
}

// One operand of a tile in LDS: ROWS rows of a step of 128 k, and their scales.  Row 64 g + 4 r + f lies in place 64 g + 16 f + r, so that a
// fragment's rows are neighbours; the chunks of a place are permuted (swz_kc) so that the reads of a fragment spread over the banks.
template <int FORMAT, int ROWS, int WAVES>
struct Panel {
  static constexpr int CHUNKS = step_bytes(FORMAT) / 16, BYTES = ROWS * CHUNKS * 16, SCALE_BYTES = ROWS * 4;
  static constexpr int LOADS = ROWS * CHUNKS / 64 / WAVES;  // 1 KB each, of a wavefront
  static constexpr int SCALE_LOADS = ROWS / 64;             // 256 bytes each, of the workgroup
  static_assert(LOADS * 64 * WAVES == ROWS * CHUNKS, "whole loads");
  const unsigned char* base;    // of the tile's first row
  const unsigned char* scales;  // of block 0
  unsigned ld_scales;
  int chunks, blocks;           // of a whole row
  unsigned offset[LOADS];       // of the lane's chunk of every load
  int chunk[LOADS];
  unsigned scale_word;          // 4 times the word of scales that the lane loads, in its block
  int scale_block;

  // `part`: which of the workgroup's loads of scales this wavefront makes (any number beyond SCALE_LOADS: none)
  __device__ __forceinline__ void init(const unsigned char* values, const unsigned char* s, unsigned ld, unsigned ld_s, int row0, int rows,
                                       int blocks_in_row, int wave, int lane, int part) {
    base = values + (long long)row0 * ld;
    scales = s;
    ld_scales = ld_s;
    blocks = blocks_in_row;
    chunks = blocks_in_row * (is_wide(FORMAT) ? 2 : 1);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int q = (wave * LOADS + i) * 64 + lane, place = q / CHUNKS;
      const int row = (place & ~63) + 4 * (place & 15) + ((place >> 4) & 3);
      chunk[i] = (q % CHUNKS) ^ swz_kc<CHUNKS, 16>(place);
      offset[i] = (unsigned)min(row, rows - 1 - row0) * ld + chunk[i] * 16;
    }
    const int q = part * 64 + lane;
    scale_block = q / (ROWS / 4);
    scale_word = 4u * (unsigned)min(row0 / 4 + q % (ROWS / 4), (rows + 3) / 4 - 1);
  }
  // The loads of step `step` into a stage at `at` in LDS (scales at `scales_at`).
  template <bool SCALES>
  __device__ __forceinline__ void request(int step, unsigned at, unsigned scales_at, unsigned char* smem, int wave, int lane, int part) const {
    const unsigned char* from = base + (long long)step * (CHUNKS * 16);
    if ((step + 1) * CHUNKS <= chunks) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) DirectLoad::chunks(from, offset[i], at + (wave * LOADS + i) * 1024);
    } else {  // the last step: what lies beyond K is 0
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        if (step * CHUNKS + chunk[i] < chunks)
          DirectLoad::chunks(from, offset[i], at + (wave * LOADS + i) * 1024);
        else
          *reinterpret_cast<u32x4*>(smem + (wave * LOADS + i) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
      }
    }
    if (SCALES && part < SCALE_LOADS) {
      const int block = min(step * 4 + scale_block, blocks - 1);
      DirectLoad::words(scales + (long long)step * 4 * ld_scales, (unsigned)(block - step * 4) * ld_scales + scale_word, scales_at + part * 256);
    }
  }
  // Fragment f of group g, and the word of scales of group g.
  static __device__ __forceinline__ Fragment<FORMAT> fragment(const unsigned char* stage, int g, int f, int lane) {
    const int place = 64 * g + 16 * f + lane % 16, swz = swz_kc<CHUNKS, 16>(lane % 16);
    const unsigned char* row = stage + place * (CHUNKS * 16);
    Fragment<FORMAT> x;
    x.v[0] = *reinterpret_cast<const u32x4*>(row + ((lane / 16) ^ swz) * 16);
    if constexpr (is_wide(FORMAT)) x.v[1] = *reinterpret_cast<const u32x4*>(row + ((4 + lane / 16) ^ swz) * 16);
    return x;
  }
  static __device__ __forceinline__ unsigned scale(const unsigned char* stage_scales, int g, int lane) {
    return *reinterpret_cast<const unsigned*>(stage_scales + (lane / 16) * ROWS + 64 * g + 4 * (lane % 16));
  }
};

// Which tile a workgroup takes: workgroups are handed to the 8 dies in turn; each die, which has an L2 of its own, gets one run of tiles, walked
// 4 tile rows at a time.
__device__ __forceinline__ void tile_of(int tiles_m, int tiles_n, int& i, int& j) {
  const unsigned total = (unsigned)tiles_m * (unsigned)tiles_n, xcd = blockIdx.x % 8u, slot = blockIdx.x / 8u;
  const unsigned each = total / 8u, extra = total % 8u;
  const unsigned w = xcd * each + (xcd < extra ? xcd : extra) + slot;
  const unsigned panel = w / (4u * tiles_n), first = panel * 4u, rows = min(4u, (unsigned)tiles_m - first), within = w - first * tiles_n;
  i = (int)(first + within % rows);
  j = (int)(within / rows);
}

// Tiles from LDS: WM x WN wavefronts of 64 GM x 64 GN each, two stages of 128 k.
template <int FA, int FB, int GM, int GN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(const GemmArgs p) {
  constexpr int WAVES = WM * WN, BM = 64 * GM * WM, BN = 64 * GN * WN;
  using A = Panel<FA, BM, WAVES>;
  using B = Panel<FB, BN, WAVES>;
  constexpr int VALUES = A::BYTES + B::BYTES, STAGE = VALUES + A::SCALE_BYTES + B::SCALE_BYTES;
  static_assert(A::SCALE_LOADS + B::SCALE_LOADS <= WAVES, "a wavefront loads scales once a stage");
  __shared__ __attribute__((aligned(16))) unsigned char smem[2 * STAGE];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  int ti, tj;
  tile_of((p.M + BM - 1) / BM, (p.N + BN - 1) / BN, ti, tj);
  const int m0 = ti * BM, n0 = tj * BN, gm = wave / WN * GM, gn = wave % WN * GN;

  A a;
  B b;
  const int part_b = wave < A::SCALE_LOADS ? WAVES : wave - A::SCALE_LOADS;
  a.init(p.a, p.scales_a, p.lda, p.ld_scales_a, m0, p.M, p.blocks, wave, lane, wave);
  b.init(p.b, p.scales_b, p.ldb, p.ld_scales_b, n0, p.N, p.blocks, wave, lane, part_b);
  f32x4 acc[4 * GM][4 * GN];
#pragma unroll
  for (int i = 0; i < 4 * GM; ++i)
#pragma unroll
    for (int j = 0; j < 4 * GN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const unsigned lds = lds_address(smem);
  auto request = [&](int step) {
    const unsigned at = (step & 1) * STAGE;
    a.template request<true>(step, lds + at, lds + at + VALUES, smem + at, wave, lane, wave);
    b.template request<true>(step, lds + at + A::BYTES, lds + at + VALUES + A::SCALE_BYTES, smem + at + A::BYTES, wave, lane, part_b);
  };
  const int steps = (p.blocks + 3) / 4;
  if (steps > 0) request(0);
  for (int step = 0; step < steps; ++step) {
    wait_all_and_meet();  // (the stage has arrived, and nobody reads the other one any more)
    if (step + 1 < steps) request(step + 1);
    const unsigned char* stage = smem + (step & 1) * STAGE;
    Fragment<FB> fb[4 * GN];
    unsigned sb[GN];
#pragma unroll
    for (int g = 0; g < GN; ++g) {
      sb[g] = B::scale(stage + VALUES + A::SCALE_BYTES, gn + g, lane);
#pragma unroll
      for (int f = 0; f < 4; ++f) fb[4 * g + f] = B::fragment(stage + A::BYTES, gn + g, f, lane);
    }
#pragma unroll
    for (int g = 0; g < GM; ++g) {
      const unsigned sa = A::scale(stage + VALUES, gm + g, lane);
      each<4>([&](auto f) {
        constexpr int F = decltype(f)::value;
        const Fragment<FA> fa = A::fragment(stage, gm + g, F, lane);
#pragma unroll
        for (int h = 0; h < GN; ++h)
          each<4>([&](auto e) {
            constexpr int E = decltype(e)::value;
            acc[4 * g + F][4 * h + E] = multiply<FA, FB, F, E>(fa, fb[4 * h + E], acc[4 * g + F][4 * h + E], sa, sb[h]);
          });
      });
    }
  }
  with_out_type(p, [&](auto type) {
    using TO = decltype(type);
#pragma unroll
    for (int g = 0; g < GM; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
          for (int h = 0; h < GN; ++h) {
            const float v[4] = {acc[4 * g + f][4 * h][i], acc[4 * g + f][4 * h + 1][i], acc[4 * g + f][4 * h + 2][i], acc[4 * g + f][4 * h + 3][i]};
            finish4<TO>(p, m0 + 64 * (gm + g) + 16 * (lane / 16) + 4 * i + f, n0 + 64 * (gn + h) + 4 * (lane % 16), v);
          }
  });
}

// ---- few rows -------------------------------------------------------------------------------------------------------------
// One operand read from memory by every wavefront for itself: GROUP ? a group of 64 rows as four fragments : 16 rows as one.
template <int FORMAT, bool GROUP>
struct Rows {
  static constexpr int F = GROUP ? 4 : 1;
  const unsigned char* row[F];
  const unsigned char* scales;  // of the lane's rows, block 0
  unsigned ld_scales;
  int blocks, shift;
  __device__ __forceinline__ void init(const unsigned char* values, const unsigned char* s, unsigned ld, unsigned ld_s, int row0, int rows,
                                       int blocks_in_row, int lane) {
    const int r = lane % 16;
#pragma unroll
    for (int f = 0; f < F; ++f) row[f] = values + (long long)min(row0 + (GROUP ? 4 * r + f : r), rows - 1) * ld;
    // (a single fragment has the scale of its one row of the word: moved to the lowest byte)
    const int word = min((row0 + (GROUP ? 4 * r : r)) / 4, (rows + 3) / 4 - 1);
    scales = s + 4LL * word;
    shift = GROUP ? 0 : 8 * (min(row0 + r, rows - 1) & 3);
    ld_scales = ld_s;
    blocks = blocks_in_row;
  }
  __device__ __forceinline__ void load(int step, int lane, Fragment<FORMAT> (&x)[F], unsigned& scale) const {
    const int g = lane / 16, last = blocks - 1;
    const int first = step * step_bytes(FORMAT) + g * 16;
    const int end = blocks * (is_wide(FORMAT) ? 32 : 16);
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const u32x4 none = {0, 0, 0, 0};
      x[f].v[0] = first < end ? *reinterpret_cast<const u32x4*>(row[f] + first) : none;
      if constexpr (is_wide(FORMAT)) x[f].v[1] = first + 64 < end ? *reinterpret_cast<const u32x4*>(row[f] + first + 64) : none;
    }
    scale = *reinterpret_cast<const unsigned*>(scales + (long long)min(step * 4 + g, last) * ld_scales) >> shift;
  }
};

// A workgroup takes 64 or 16 rows x 64 or 16 columns; its wavefronts take the steps of K in turn and add their sums in LDS, in order.
template <int FA, int FB, bool GROUP_M, bool GROUP_N, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void stream_kernel(const GemmArgs p) {
  constexpr int FM = GROUP_M ? 4 : 1, FN = GROUP_N ? 4 : 1, BM = 16 * FM, BN = 16 * FN;
  __shared__ f32x4 meet[WAVES][FM * FN][64];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN, slices = slices_of(p);
  const int tile = blockIdx.x / slices, slice = blockIdx.x - tile * slices;
  const int m0 = tile % tiles_m * BM, n0 = tile / tiles_m * BN;
  (void)tiles_n;
  Rows<FA, GROUP_M> a;
  Rows<FB, GROUP_N> b;
  a.init(p.a, p.scales_a, p.lda, p.ld_scales_a, m0, p.M, p.blocks, lane);
  b.init(p.b, p.scales_b, p.ldb, p.ld_scales_b, n0, p.N, p.blocks, lane);
  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int steps = min((p.blocks + 3) / 4, (slice + 1) * p.slice);
#pragma unroll 4
  for (int step = slice * p.slice + wave; step < steps; step += WAVES) {
    Fragment<FA> fa[FM];
    Fragment<FB> fb[FN];
    unsigned sa, sb;
    a.load(step, lane, fa, sa);
    b.load(step, lane, fb, sb);
    each<FM>([&](auto f) {
      each<FN>([&](auto e) {
        constexpr int F = decltype(f)::value, E = decltype(e)::value;
        acc[F][E] = multiply<FA, FB, F, E>(fa[F], fb[E], acc[F][E], sa, sb);
      });
    });
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) meet[wave][i * FN + j][lane] = acc[i][j];
  __syncthreads();
  // every wavefront finishes some of the rows: those of fragment i, or (16 rows) the first does all
  for (int i = wave; i < FM; i += WAVES) {
    f32x4 sum[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      sum[j] = meet[0][i * FN + j][lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) sum[j] += meet[w][i * FN + j][lane];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = m0 + (GROUP_M ? 16 * (lane / 16) + 4 * e + i : 4 * (lane / 16) + e);
      if constexpr (GROUP_N) {
        const float v[4] = {sum[0][e], sum[1][e], sum[2][e], sum[3][e]};
        const int col = n0 + 4 * (lane % 16);
        if (slices > 1)
          keep4(p, slice, row, col, v);
        else
          with_out_type(p, [&](auto type) { finish4<decltype(type)>(p, row, col, v); });
      } else {  // a column a lane: four lanes' make the four that are finished together
        float v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = __shfl(sum[0][e], (lane & ~3) + c);
        const int col = n0 + (lane % 16);
        if (lane % 4 == 0) {
          if (slices > 1)
            keep4(p, slice, row, col, v);
          else
            with_out_type(p, [&](auto type) { finish4<decltype(type)>(p, row, col, v); });
        }
      }
    }
  }
}

// The sums of the slices, in ascending order, and the epilogue: a thread for 4 columns of a row.  `workspace`: [slice][M][N].
template <typename TO>
__global__ __launch_bounds__(256) void join_slices_kernel(const GemmArgs p, const float* workspace) {
  const int quads = (p.N + 3) / 4, slices = slices_of(p);
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(i / quads), n = (int)(i - (long long)m * quads) * 4;
  if (m >= p.M) return;
  const float* from = workspace + (long long)m * p.N + n;
  const long long each = (long long)p.M * p.N;
  const bool whole = p.N % 4 == 0;
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < slices; ++s) {
    if (whole) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(from + s * each);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += t[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += from[s * each + (n + e < p.N ? e : 0)];
    }
  }
  finish4<TO>(p, m, n, v);
}

// Which kernel serves a product, and how it is cut.
enum : int { KERNEL_TILE_128 = 0, KERNEL_STREAM_16 = 1, KERNEL_STREAM_64 = 2 };
struct GemmCut {
  int kernel;
  int slices;
  long long blocks;  // workgroups
};
// the kernels of A's format (mx_kernels.hip, once for each)
template <int FA>
hipError_t launch_gemm(int format_b, const GemmCut& cut, const GemmArgs& p, hipStream_t stream);

}  // namespace mx
}  // namespace hidet
