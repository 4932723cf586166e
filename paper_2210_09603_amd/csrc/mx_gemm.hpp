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
// What it adds: the products of 8 neighbouring k, of which an element has 8 bits, are cut to 13 bits below the largest of their exponents before they
// are added; sums of eights are added in fp32.  That is fewer bits than the accumulators', a choice: no other instruction takes these formats with
// their scales, and products of operands widened to bf16, exact and added in fp32, run at 1.2 to 1.5 PFLOP/s (8192 x 8192 x 8192 by the library) for 2.6 here.
// 1.5e-5 of a result from normally distributed operands, a hundredth of half a step of bf16; 4 bits by 4 lose nothing (no product lies 13 bits
// below another).
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
  unsigned flags;  // bits 0-1 dtype of C, 2-3 bias axis, 4 ReLU, 8.. slices
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
// R rows of four neighbouring columns, as the other products finish theirs: alpha, bias, residual, ReLU, one rounding.  All that is read
// is asked for before anything is written, so that a thread waits once for all of it.
template <typename TO>
struct ColumnBias {
  float v[4];  // 0 if there is none
  __device__ __forceinline__ ColumnBias(const GemmArgs& p, int col) {
    const bool any = ((p.flags >> 2) & 3) == HIDET_BIAS_PER_COL;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = any ? to_f32(reinterpret_cast<const TO*>(p.bias)[min(col + e, p.N - 1)]) : 0.0f;
  }
};
template <typename TO, int R>
__device__ __forceinline__ void finish(const GemmArgs& p, const int (&row)[R], int col, const ColumnBias<TO>& bias, const float (&sum)[R][4]) {
  struct __attribute__((packed, aligned(sizeof(TO)))) Quad {  // (one access, at element alignment)
    TO e[4];
  };
  float of_row[R];
  Quad other[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    of_row[r] = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) other[r].e[e] = TO(0.0f);
  }
  if (((p.flags >> 2) & 3) == HIDET_BIAS_PER_ROW) {
#pragma unroll
    for (int r = 0; r < R; ++r) of_row[r] = to_f32(reinterpret_cast<const TO*>(p.bias)[min(row[r], p.M - 1)]);
  }
  if (p.residual) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int left = row[r] < p.M ? p.N - col : 0;
      const TO* from = reinterpret_cast<const TO*>(p.residual) + (long long)row[r] * p.ldr + col;
      if (left >= 4) {
        other[r] = *reinterpret_cast<const Quad*>(from);
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (e < left) other[r].e[e] = from[e];
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    Quad o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v = p.alpha * sum[r][e] + of_row[r] + bias.v[e] + to_f32(other[r].e[e]);
      o.e[e] = from_f32<TO>((p.flags & 16) != 0 && v < 0.0f ? 0.0f : v);
    }
    const int left = row[r] < p.M ? p.N - col : 0;
    TO* c = reinterpret_cast<TO*>(p.c) + (long long)row[r] * p.ldc + col;
    if (left >= 4) {
      *reinterpret_cast<Quad*>(c) = o;
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) c[e] = o.e[e];
    }
  }
}
template <typename TO>
__device__ __forceinline__ void finish4(const GemmArgs& p, int m, int n, const float (&sum)[4]) {
  const int row[1] = {m};
  const float v[1][4] = {{sum[0], sum[1], sum[2], sum[3]}};
  finish<TO, 1>(p, row, n, ColumnBias<TO>(p, n), v);
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
  struct __attribute__((packed, aligned(4))) Quad {
    f32x4 v;
  };
  if (left >= 4) {
    reinterpret_cast<Quad*>(c)->v = f32x4{sum[0], sum[1], sum[2], sum[3]};
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

// One operand of a tile in LDS: ROWS rows of STEPS steps of 128 k, and their scales.  Row 64 g + 4 r + f lies in place 64 g + 16 f + r, so that
// a fragment's rows are neighbours; the chunks of a place are permuted (swz_kc) so that the reads of a fragment spread over the banks.
template <int FORMAT, int ROWS, int STEPS, int WAVES>
struct Panel {
  static constexpr int CHUNKS = STEPS * step_bytes(FORMAT) / 16, BYTES = ROWS * CHUNKS * 16, SCALE_BYTES = ROWS * 4 * STEPS;
  static constexpr int LOADS = ROWS * CHUNKS / 64 / WAVES;  // 1 KB each, of a wavefront
  static constexpr int PARTS = ROWS / 64;                   // loads of scales a step, 256 bytes each, of the workgroup
  static_assert(LOADS * 64 * WAVES == ROWS * CHUNKS, "whole loads");
  const unsigned char* base;    // of the tile's first row
  const unsigned char* scales;  // of the tile's first row, block 0
  unsigned ld_scales;
  int last_word;                // word of scales, from the tile's first row, that the matrix ends with
  int blocks;                   // of a row
  unsigned offset[LOADS];       // of the lane's chunk of every load, in bytes from the tile's first row: below 2^31

  __device__ __forceinline__ Panel(const unsigned char* values, const unsigned char* s, unsigned ld, unsigned ld_s, int row0, int rows, int first_block,
                                   int blocks_in_row, int wave, int lane)
      : base(values + (long long)row0 * ld + (long long)first_block * (is_wide(FORMAT) ? 32 : 16)),
        scales(s + (long long)first_block * ld_s + row0), ld_scales(ld_s), last_word((rows + 3) / 4 - 1 - row0 / 4), blocks(blocks_in_row) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int place = place_of(i, wave, lane), row = (place & ~63) + 4 * (place & 15) + ((place >> 4) & 3);
      offset[i] = (unsigned)min(row, rows - 1 - row0) * ld + chunk_of(i, wave, lane) * 16;
    }
  }
  static __device__ __forceinline__ int place_of(int load, int wave, int lane) { return ((wave * LOADS + load) * 64 + lane) / CHUNKS; }
  static __device__ __forceinline__ int chunk_of(int load, int wave, int lane) { return lane % CHUNKS ^ swz_kc<CHUNKS, 16>(place_of(load, wave, lane)); }
  // The loads of a whole stage to `at` in LDS.
  __device__ __forceinline__ void request(int stage, unsigned at, int wave) const {
    const unsigned char* from = base + (long long)stage * (CHUNKS * 16);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) DirectLoad::chunks(from, offset[i], at + (wave * LOADS + i) * 1024);
  }
  // The same of the last stage, which K ends in: what lies beyond is 0.  `smem`: `at` as an address.
  __device__ __forceinline__ void request_end(int stage, unsigned at, unsigned char* smem, int wave, int lane) const {
    const unsigned char* from = base + (long long)stage * (CHUNKS * 16);
    const int left = blocks * (is_wide(FORMAT) ? 2 : 1) - stage * CHUNKS;  // chunks
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      if (chunk_of(i, wave, lane) < left)
        DirectLoad::chunks(from, offset[i], at + (wave * LOADS + i) * 1024);
      else
        *reinterpret_cast<u32x4*>(smem + (wave * LOADS + i) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
    }
  }
  // Part `part` of the scales of step s of a stage.  (Blocks beyond K: the last one.)
  __device__ __forceinline__ void request_scales(int stage, int s, unsigned at, int part, int lane) const {
    const int first = min((stage * STEPS + s) * 4, blocks - 1), q = part * 64 + lane;
    const int block = min(q / (ROWS / 4), blocks - 1 - first), word = min(q % (ROWS / 4), last_word);
    DirectLoad::words(scales + (long long)first * ld_scales, (unsigned)block * ld_scales + 4u * (unsigned)word, at + (s * PARTS + part) * 256);
  }
  // Fragment f of group g for step s of the stage, and the word of scales of group g.
  static __device__ __forceinline__ Fragment<FORMAT> fragment(const unsigned char* stage, int s, int g, int f, int lane) {
    const int place = 64 * g + 16 * f + lane % 16, swz = swz_kc<CHUNKS, 16>(lane % 16);
    const unsigned char* row = stage + place * (CHUNKS * 16);
    Fragment<FORMAT> x;
    x.v[0] = *reinterpret_cast<const u32x4*>(row + ((s * (step_bytes(FORMAT) / 16) + lane / 16) ^ swz) * 16);
    if constexpr (is_wide(FORMAT)) x.v[1] = *reinterpret_cast<const u32x4*>(row + ((s * 8 + 4 + lane / 16) ^ swz) * 16);
    return x;
  }
  static __device__ __forceinline__ unsigned scale(const unsigned char* stage_scales, int s, int g, int lane) {
    return *reinterpret_cast<const unsigned*>(stage_scales + (s * 4 + lane / 16) * ROWS + 64 * g + 4 * (lane % 16));
  }
};

// Workgroups are handed to the 8 dies in turn; each die, which has an L2 of its own, gets one run of `total` places.
__device__ __forceinline__ unsigned place_of(unsigned at, unsigned total) {
  const unsigned xcd = at % 8u, each = total / 8u, extra = total % 8u;
  return xcd * each + (xcd < extra ? xcd : extra) + at / 8u;
}
// Which tile a workgroup takes: runs of tiles, walked 4 tile rows at a time.
__device__ __forceinline__ void tile_of(unsigned at, int tiles_m, int tiles_n, int& i, int& j) {
  const unsigned w = place_of(at, (unsigned)tiles_m * (unsigned)tiles_n);
  const unsigned panel = w / (4u * tiles_n), first = panel * 4u, rows = min(4u, (unsigned)tiles_m - first), within = w - first * tiles_n;
  i = (int)(first + within % rows);
  j = (int)(within / rows);
}

// What a wavefront has summed: 64 x 64 from row m and column n on.
__device__ __forceinline__ void finish_tile(const GemmArgs& p, int slice, int m, int n, int lane, const f32x4 (&acc)[4][4]) {
  const int col = n + 4 * (lane % 16);
  auto rows = [&](auto done) {  // four at a time
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      int row[4];
      float v[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        row[i] = m + 16 * (lane / 16) + 4 * i + f;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = acc[f][e][i];
      }
      done(row, v);
    }
  };
  if (slices_of(p) > 1)
    rows([&](const int (&row)[4], const float (&v)[4][4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) keep4(p, slice, row[i], col, v[i]);
    });
  else
    with_out_type(p, [&](auto type) {
      using TO = decltype(type);
      const ColumnBias<TO> bias(p, col);
      rows([&](const int (&row)[4], const float (&v)[4][4]) { finish<TO, 4>(p, row, col, bias, v); });
    });
}

constexpr int PLACES = 2;  // of stages in LDS
// (256 x 256 tiles of 8 by 4 bits need all of their 128 registers: with the first request written out in place of its loop they do not suffice, and
// 4096 x 4096 x 4096 takes 129 us for 52.)
// Bytes of a stage, and of the LDS of tile_kernel.
template <int FA, int FB, int WM, int WN, int GROUPS>
struct TileShape {
  // steps of 128 k: of a wavefront, and of a stage.  (Rows of 128 bytes, a line, in a stage: with 64 every line is fetched twice.)
  static constexpr int EACH = !is_wide(FA) && !is_wide(FB) && GROUPS == 1 ? 2 : 1, STEPS = EACH * GROUPS;
  static constexpr int WAVES = WM * WN * GROUPS, BM = 64 * WM, BN = 64 * WN;
  using A = Panel<FA, BM, STEPS, WAVES>;
  using B = Panel<FB, BN, STEPS, WAVES>;
  static constexpr int VALUES = A::BYTES + B::BYTES, STAGE = VALUES + A::SCALE_BYTES + B::SCALE_BYTES;
  static constexpr int SUMS = (GROUPS - 1) * WM * WN * 16384, LDS = PLACES * STAGE > SUMS ? PLACES * STAGE : SUMS;
};

// Tiles from LDS: WM x WN wavefronts of 64 x 64 each, two stages, one of them on its way.  GROUPS such sets of wavefronts take a part of
// every stage's k each, and add their sums in LDS, in order.
//
// 8192 x 8192 x 8192 into bf16 on 256 x 256 tiles: 4 bits by 4 264 us (4.2 PFLOP/s), 8 by 8 430 (2.6), 8 by 4 375 (2.9).  Of these the matrix
// instructions alone, at the clock that the board's power leaves them, are 157, 260 and 250; the loads into LDS alone 151, 270 and 261; products
// with their reads of LDS and no loads 209, 361 and 310: no one of the three bounds it, but they do not overlap wholly, since a compute
// unit has room for one workgroup of two stages.  128 x 128 tiles of 4 wavefronts: 296, 514, 442 (half the products per byte loaded); 3 or 4
// smaller stages, 8 wavefronts of 128 x 64 and wavefronts that only load: no shorter.
//
// 333 x 5120 x 4096 on 64 x 128 tiles, one to a compute unit, 8 bits by 4: 17.9 us; its loads alone 16.1, reads of LDS and products without loads
// 11.9, products alone 9.9, each with launch and stores: a stage's loads are waited for, then a SIMD's one wavefront reads, then it multiplies.  With a
// third stage on its way the loads alone take 12.2, the whole 17.2.
template <int FA, int FB, int WM, int WN, int GROUPS>
__global__ __launch_bounds__(64 * WM * WN * GROUPS) void tile_kernel(const GemmArgs p) {
  using S = TileShape<FA, FB, WM, WN, GROUPS>;
  using A = typename S::A;
  using B = typename S::B;
  constexpr int SET = WM * WN, PARTS = A::PARTS + B::PARTS;
  static_assert(PARTS <= S::WAVES, "a load of scales a wavefront");
  // The loads of another stage are handed over behind a quarter of a wavefront's products, not before them: it is held up there for long
  // enough that the matrix cores should have work by then.  (Two operands of 8 bits have no registers left for it.)
  constexpr bool LATE = !(is_wide(FA) && is_wide(FB));
  __shared__ __attribute__((aligned(16))) unsigned char smem[S::LDS];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int group = wave / SET, member = wave % SET;
  const int slices = slices_of(p), slice = blockIdx.x % slices, first_block = slice * p.slice * 4;
  const int blocks = min(p.blocks - first_block, p.slice * 4);  // of this slice
  int ti, tj;
  tile_of(blockIdx.x / slices, (p.M + S::BM - 1) / S::BM, (p.N + S::BN - 1) / S::BN, ti, tj);
  const int m0 = ti * S::BM, n0 = tj * S::BN, gm = member / WN, gn = member % WN;
  const A a(p.a, p.scales_a, p.lda, p.ld_scales_a, m0, p.M, first_block, blocks, wave, lane);
  const B b(p.b, p.scales_b, p.ldb, p.ld_scales_b, n0, p.N, first_block, blocks, wave, lane);
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const unsigned lds = lds_address(smem);
  // whole stages; what K ends in comes before them, in the first place
  const int stages = blocks / (4 * S::STEPS), ahead = blocks % (4 * S::STEPS) != 0;
  auto request_scales = [&](int s, unsigned at) {
    const int part = wave % PARTS;  // (some may be loaded twice: all wavefronts have as many in flight)
#pragma unroll
    for (int u = 0; u < S::STEPS; ++u) {
      if (part < A::PARTS)
        a.request_scales(s, u, at + S::VALUES, part, lane);
      else
        b.request_scales(s, u, at + S::VALUES + A::SCALE_BYTES, part - A::PARTS, lane);
    }
  };
  auto request = [&](int s, int place) {
    const unsigned at = lds + place * S::STAGE;
    a.request(s, at, wave);
    b.request(s, at + A::BYTES, wave);
    request_scales(s, at);
  };
  // `between`: called behind the first quarter of the products
  auto work = [&](int place, auto between) {
    const unsigned char* stage = smem + place * S::STAGE;
#pragma unroll
    for (int i = 0; i < S::EACH; ++i) {
      const int u = group * S::EACH + i;
      Fragment<FA> fa[4];
      Fragment<FB> fb[4];
      const unsigned sb = B::scale(stage + S::VALUES + A::SCALE_BYTES, u, gn, lane);
#pragma unroll
      for (int f = 0; f < 4; ++f) fb[f] = B::fragment(stage + A::BYTES, u, gn, f, lane);
      const unsigned sa = A::scale(stage + S::VALUES, u, gm, lane);
#pragma unroll
      for (int f = 0; f < 4; ++f) fa[f] = A::fragment(stage, u, gm, f, lane);
      each<4>([&](auto f) {
        constexpr int F = decltype(f)::value;
        if (i == 0 && F == 1) between();
        each<4>([&](auto e) {
          constexpr int E = decltype(e)::value;
          acc[F][E] = multiply<FA, FB, F, E>(fa[F], fb[E], acc[F][E], sa, sb);
        });
      });
    }
  };
  if (ahead) {
    a.request_end(stages, lds, smem, wave, lane);
    b.request_end(stages, lds + A::BYTES, smem + A::BYTES, wave, lane);
    request_scales(stages, lds);
  }
#pragma unroll
  for (int s = 0; s < PLACES - 1; ++s)
    if (s < stages) request(s, (s + ahead) % PLACES);
  if (ahead) {
    wait_all_and_meet();
    work(0, [] {});
  }
  int place = ahead, next = (PLACES - 1 + ahead) % PLACES;  // of this stage, and of the one that is requested
  for (int s = 0; s < stages; ++s) {
    __builtin_amdgcn_sched_barrier(0);
    wait_all_and_meet();  // the stage has arrived, and nobody reads the one before any more
    __builtin_amdgcn_sched_barrier(0);
    const bool more = s + PLACES - 1 < stages;
    if (!LATE && more) request(s + PLACES - 1, next);
    work(place, [&] {
      if constexpr (LATE) {
        __builtin_amdgcn_sched_barrier(0);
        if (more) request(s + PLACES - 1, next);
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    place = place + 1 == PLACES ? 0 : place + 1;
    next = next + 1 == PLACES ? 0 : next + 1;
  }
  if constexpr (GROUPS > 1) {
    f32x4* meet = reinterpret_cast<f32x4*>(smem) + lane;
    __syncthreads();  // (the stages are read)
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) meet[(((group - 1) * SET + member) * 16 + i * 4 + j) * 64] = acc[i][j];
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 0; k < GROUPS - 1; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += meet[((k * SET + member) * 16 + i * 4 + j) * 64];
  }
  finish_tile(p, slice, m0 + 64 * gm, n0 + 64 * gn, lane, acc);
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
  // Whole steps, and one that K ends in.
  __device__ __forceinline__ void load(int step, int lane, Fragment<FORMAT> (&x)[F], unsigned& scale) const {
    const long long first = (long long)step * step_bytes(FORMAT) + lane / 16 * 16;
#pragma unroll
    for (int f = 0; f < F; ++f) {
      x[f].v[0] = *reinterpret_cast<const u32x4*>(row[f] + first);
      if constexpr (is_wide(FORMAT)) x[f].v[1] = *reinterpret_cast<const u32x4*>(row[f] + first + 64);
    }
    scale = *reinterpret_cast<const unsigned*>(scales + (long long)(step * 4 + lane / 16) * ld_scales) >> shift;
  }
  __device__ __forceinline__ void load_end(int step, int lane, Fragment<FORMAT> (&x)[F], unsigned& scale) const {
    const int g = lane / 16, first = step * step_bytes(FORMAT) + g * 16, end = blocks * (is_wide(FORMAT) ? 32 : 16);
    const u32x4 none = {0, 0, 0, 0};
#pragma unroll
    for (int f = 0; f < F; ++f) {
      x[f].v[0] = first < end ? *reinterpret_cast<const u32x4*>(row[f] + first) : none;
      if constexpr (is_wide(FORMAT)) x[f].v[1] = first + 64 < end ? *reinterpret_cast<const u32x4*>(row[f] + first + 64) : none;
    }
    scale = *reinterpret_cast<const unsigned*>(scales + (long long)min(step * 4 + g, blocks - 1) * ld_scales) >> shift;
  }
};

// A workgroup takes 16 rows x 64 (GROUP) or 16 columns; its 8 wavefronts take a run of K's steps each and add their sums in LDS, in order.
//
// Bound by memory's latency: B is read once, and with 8 wavefronts on 4 steps each all of K = 4096 is asked for at once.  4 x 8192 x 4096, 8 bits
// by 4, with a residual: 7.1 us for 17.9 MB, which a stream reads in 2.8 behind a launch of 1.5.  (8.7 with the steps dealt to the wavefronts in turn,
// tiles to the dies in turn, and rows finished one behind the other.)
template <int FA, int FB, bool GROUP>
__global__ __launch_bounds__(512) void stream_kernel(const GemmArgs p) {
  constexpr int WAVES = 8, FN = GROUP ? 4 : 1;
  constexpr int AT_ONCE = GROUP ? 2 : 4;  // steps whose loads are in flight
  __shared__ f32x4 meet[WAVES][FN][64];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int tiles_m = (p.M + 15) / 16, slices = slices_of(p);
  // (neighbouring tiles of columns share lines of scales)
  const int place = (int)place_of(blockIdx.x, gridDim.x), tile = place / slices, slice = place - tile * slices;
  const int m0 = tile % tiles_m * 16, n0 = tile / tiles_m * 16 * FN;
  Rows<FA, false> a;
  Rows<FB, GROUP> b;
  a.init(p.a, p.scales_a, p.lda, p.ld_scales_a, m0, p.M, p.blocks, lane);
  b.init(p.b, p.scales_b, p.ldb, p.ld_scales_b, n0, p.N, p.blocks, lane);
  // (the residual is asked for before all else, so that it is at hand when the sums are)
  unsigned near = 0;
  if (p.residual && slices == 1 && wave == 0) {
    const int size = (p.flags & 3) == HIDET_F32 ? 4 : 2, col = n0 + (GROUP ? 4 : 1) * (lane % 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = m0 + 4 * (lane / 16) + e;
      if (row < p.M && col < p.N) near |= *reinterpret_cast<const unsigned short*>(reinterpret_cast<const unsigned char*>(p.residual) + ((long long)row * p.ldr + col) * size);
    }
  }
  f32x4 acc[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  Fragment<FA> fa[AT_ONCE][1];
  Fragment<FB> fb[AT_ONCE][FN];
  unsigned sa[AT_ONCE], sb[AT_ONCE];
  auto product = [&](int u) {
    each<FN>([&](auto e) {
      constexpr int E = decltype(e)::value;
      acc[E] = multiply<FA, FB, 0, E>(fa[u][0], fb[u][E], acc[E], sa[u], sb[u]);
    });
  };
  // a run of steps for every wavefront, so that it takes whole lines of 4-bit rows; its last may be the one that K ends in
  const int begin = slice * p.slice, end = min((p.blocks + 3) / 4, begin + p.slice), each_wave = (end - begin + WAVES - 1) / WAVES;
  int step = begin + wave * each_wave;
  const int last = min(step + each_wave, end), whole = min(last, p.blocks / 4);
  for (; step + AT_ONCE <= whole; step += AT_ONCE) {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      a.load(step + u, lane, fa[u], sa[u]);
      b.load(step + u, lane, fb[u], sb[u]);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) product(u);
  }
#pragma unroll
  for (int u = 0; u < AT_ONCE; ++u)
    if (step + u < whole) {
      a.load(step + u, lane, fa[u], sa[u]);
      b.load(step + u, lane, fb[u], sb[u]);
    } else if (step + u < last) {
      a.load_end(step + u, lane, fa[u], sa[u]);
      b.load_end(step + u, lane, fb[u], sb[u]);
    }
#pragma unroll
  for (int u = 0; u < AT_ONCE; ++u)
    if (step + u < last) product(u);
  asm volatile("" ::"v"(near));
#pragma unroll
  for (int j = 0; j < FN; ++j) meet[wave][j][lane] = acc[j];
  __syncthreads();
  if (wave > 0) return;  // (the first finishes all rows)
  f32x4 sum[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    sum[j] = meet[0][j][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum[j] += meet[w][j][lane];
  }
  if constexpr (GROUP) {
    const int col = n0 + 4 * (lane % 16);
    int row[4];
    float v[4][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      row[e] = m0 + 4 * (lane / 16) + e;
#pragma unroll
      for (int c = 0; c < 4; ++c) v[e][c] = sum[c][e];
    }
    if (slices > 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) keep4(p, slice, row[e], col, v[e]);
    } else {
      with_out_type(p, [&](auto type) {
        using TO = decltype(type);
        finish<TO, 4>(p, row, col, ColumnBias<TO>(p, col), v);
      });
    }
  } else {  // a column a lane, four rows: of four lanes, each takes the four columns of one row
    float v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float t[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = __shfl(sum[0][e], (lane & ~3) + c);
      v[c] = lane & 2 ? (lane & 1 ? t[3] : t[2]) : (lane & 1 ? t[1] : t[0]);
    }
    const int row = m0 + 4 * (lane / 16) + lane % 4, col = n0 + lane % 16 / 4 * 4;
    if (slices > 1)
      keep4(p, slice, row, col, v);
    else
      with_out_type(p, [&](auto type) { finish4<decltype(type)>(p, row, col, v); });
  }
}

// The sums of the slices, in ascending order, and the epilogue: a thread for 4 columns of a row.  A launch and two loads one behind the other: 3 to 4 us.  `workspace`: [slice][M][N].
template <typename TO>
__global__ __launch_bounds__(256) void join_slices_kernel(const GemmArgs p, const float* workspace) {
  const int quads = (p.N + 3) / 4, slices = slices_of(p);
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(i / quads), n = (int)(i - (long long)m * quads) * 4;
  if (m >= p.M) return;
  const float* from = workspace + (long long)m * p.N + n;
  const long long each = (long long)p.M * p.N;
  struct __attribute__((packed, aligned(4))) Quad {
    f32x4 v;
  };
  const bool whole = n + 4 <= p.N;
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < slices; ++s) {
    if (whole) {
      const f32x4 t = reinterpret_cast<const Quad*>(from + s * each)->v;
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
enum : int { KERNEL_TILE_256 = 0, KERNEL_TILE_128, KERNEL_TILE_64X128, KERNEL_TILE_64, KERNEL_STREAM_16, KERNEL_STREAM_16X64 };
struct GemmCut {
  int kernel;
  int slices, slice;  // slice: steps of 128 k of each
  long long blocks;   // workgroups
};
// the kernels of A's format (mx_kernels.hip, once for each)
template <int FA>
hipError_t launch_gemm(int format_b, const GemmCut& cut, const GemmArgs& p, hipStream_t stream);

}  // namespace mx
}  // namespace hidet
