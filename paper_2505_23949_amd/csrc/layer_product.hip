// tsenor_product: out = a b^T of two matrices in 8-bit floating point with a power of two for each row and 128 columns.
//
// Everything goes through the scaled matrix instructions (v_mfma_scale_f32_*_f8f6f4), which apply the powers of two of both rows
// on the way, so the scales cost no vector instruction.  b (weights) is their first operand: a lane then holds neighbouring
// columns of the result.  The order of the columns in the sum is free as long as both operands agree on it.
#include <algorithm>
#include <type_traits>

#include "layer.hpp"
#include "layer_plan.hpp"

namespace {

using namespace tsenor_dev;

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

struct ProductArgs {
  tsenor_scaled a, b;
  uint16_t* out;
  const uint8_t* mask;
  int64_t out_ld, mask_ld;
  int m, n, blocks;      // blocks of 128 columns
  int tiles_m, tiles_n;  // of the tile kernel
  int splits;            // workgroups that share the columns of a tile: each leaves its sums in `parts`
  floatx4* parts;
};

// keeps the instructions around it in the order written
#define TSENOR_IN_ORDER() __builtin_amdgcn_sched_barrier(0)

// ---- few rows of a -------------------------------------------------------------------------------------------------------
// One token or a few: the weights are read once, straight into registers, by a workgroup of eight waves for each 16 of their rows.
// The waves share the columns, every wave takes each eighth block, four of them at a time, and their sums meet in LDS.
// Lane l holds 32 of the 128 columns of row l % 16: the 16 bytes at 16 (l / 16) and those 64 further on, so that the four lanes
// of a row read 64 bytes in a row.
constexpr int kWaves = 8;
__device__ __forceinline__ intx8 load_operand(const uint8_t* row) {
  const int4 lo = *reinterpret_cast<const int4*>(row), hi = *reinterpret_cast<const int4*>(row + 64);
  return intx8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
}

// results of row i, columns j to j + 3
__device__ __forceinline__ void write4(const ProductArgs& a, int i, int j, float (&v)[4]) {
  if (i >= a.m || j >= a.n) return;
  if (a.mask) {
    const uint8_t* m = a.mask + i * a.mask_ld + j;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j + k < a.n && !m[k]) v[k] = 0.0f;
  }
  uint16_t* out = a.out + (int64_t)i * a.out_ld + j;
  const uint32_t w[2] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  if (j + 4 <= a.n) {
    __builtin_memcpy(out, w, 8);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j + k < a.n) out[k] = (uint16_t)(w[k / 2] >> (k % 2 * 16));
  }
}

__global__ __launch_bounds__(kWaves* kWave) void few_rows_kernel(ProductArgs p) {
  __shared__ float sums[kWaves][kWave][4];
  const int lane = (int)threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int n0 = (int)blockIdx.x * 16;
  const int row_b = min(n0 + lane % 16, p.n - 1), row_a = min(lane % 16, p.m - 1);  // (rows past the last are not written)
  const uint8_t* const b = p.b.values + row_b * p.b.ld + lane / 16 * 16;
  const uint8_t* const a = p.a.values + row_a * p.a.ld + lane / 16 * 16;
  floatx4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  const auto take = [&](int k0, auto count) {  // blocks k0, k0 + kWaves, ...
    constexpr int kCount = decltype(count)::value;
    intx8 x[kCount], y[kCount];
    int x_scale[kCount], y_scale[kCount];
#pragma unroll
    for (int u = 0; u < kCount; ++u) {
      const int k = k0 + u * kWaves;
      x[u] = load_operand(b + (int64_t)k * kBlock);
      x_scale[u] = p.b.scales[k * p.b.scale_ld + row_b];
      y[u] = load_operand(a + (int64_t)k * kBlock);
      y_scale[u] = p.a.scales[k * p.a.scale_ld + row_a];
    }
    TSENOR_IN_ORDER();  // (all of them are asked for before the first is waited for)
#pragma unroll
    for (int u = 0; u < kCount; ++u)
      sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[u], y[u], sum, 0, 0, 0, x_scale[u], 0, y_scale[u]);
  };
  int k0 = wave;
  for (; k0 + 3 * kWaves < p.blocks; k0 += 4 * kWaves) take(k0, std::integral_constant<int, 4>());
  if (k0 + kWaves < p.blocks) take(k0, std::integral_constant<int, 2>()), k0 += 2 * kWaves;
  if (k0 < p.blocks) take(k0, std::integral_constant<int, 1>());
#pragma unroll
  for (int k = 0; k < 4; ++k) sums[wave][lane][k] = sum[k];
  __syncthreads();
  if (wave == 0) {
    float v[4] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += sums[w][lane][k];
    write4(p, lane % 16, n0 + lane / 16 * 4, v);
  }
}

// ---- tiles ---------------------------------------------------------------------------------------------------------------
// A workgroup of four waves, two by two, takes 64 TN rows of b and 64 TM rows of a; a wave 32 TN x 32 TM results in accumulators.
// Blocks of 128 columns come into a ring of BUFFERS in LDS by loads that go there directly.
//
//   Rows: tile t of a wave holds rows T r + t (r = 0..31) of its 32 T, so that one read fetches the scale bytes of all its tiles (the
//   instruction picks the byte), and a lane ends up with 4 TN neighbouring columns of the result.  In LDS they stand at 32 t + r.
//   Rows past the last are read as the last one and not written.
//   16-byte pieces: piece c of row r stands at place c ^ (r / 2 % 8), so that the 16 lanes that LDS serves at a time (other rows, the
//   same piece) take all banks.  The loads write LDS in order, so it is the lanes' addresses in memory that are permuted.
//   Loads are spread evenly: those of a block over the second half of a step and, with more than two buffers, the first of the next
//   (all in one half: 5-10 % slower).
//   Waits: by the middle of a step every wave has the rest of the current block in registers; after a barrier there its buffer is
//   loaded anew, and the second half of the step reads the beginning of the next block.
//
// 256 x 256 is bound by the matrix cores under the card's power: 2500-2970 TFLOP/s for random operands at 8192^3, 3840 for zeros, where
// the instruction alone reaches 4040 and 4940.  A wave of 128 x 128 reads 16 bytes of LDS for 4096 multiplications; one of
// 64 x 128 a half more.  It takes all 256 accumulators of a wave, one wave to a SIMD, so what hides latency is the order of the
// instructions.  The 32 x 32 x 64 instruction is 5 % faster than 16 x 16 x 128 here (fewer operands read for a multiplication).
// Blocks of 64 columns with twice as many barriers were 8-25 % slower, all loads of a block asked for at once 4 %.
template <int TN, int TM>
struct TileShape {
  static constexpr int kRowsB = 64 * TN, kRowsA = 64 * TM;
  static constexpr int kValues = (kRowsB + kRowsA) * kBlock;   // bytes of a block's values; b's rows first
  static constexpr int kBuffer = kValues + 512;                // and of its scales, 256 for either operand
  static constexpr int kPieces = 2 * TN + 2 * TM + 1;          // loads that a wave makes for a block
};

struct Resource {
  uint64_t base;
  uint32_t bytes, format;
};
__device__ __forceinline__ intx4 resource_of(const void* base, int64_t bytes) {
  return __builtin_bit_cast(intx4, Resource{(uint64_t)base, (uint32_t)bytes, 0x00020000u});
}
// 16 (or 4) bytes per lane from memory into LDS, in the order of the lanes from byte `to` on.  (The compiler would wait for loads into
// LDS that it knows of before any read of LDS; here the waits stand in the code.  A scalar write of m0 needs one other
// instruction before such a load.)
__device__ __forceinline__ void load_to_lds(uint32_t to, int lane_offset, const intx4& from, int offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(lane_offset), "s"(from), "s"(offset)
               : "memory", "m0");
}
__device__ __forceinline__ void load_dword_to_lds(uint32_t to, int lane_offset, const intx4& from, int offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(lane_offset), "s"(from), "s"(offset)
               : "memory", "m0");
}
// waits for what this wave has asked of LDS (with LDS), and of memory but for the last PENDING loads, then for the other waves
template <int PENDING, bool LDS = true>
__device__ __forceinline__ void meet() {
  static_assert(PENDING < 64);
  __builtin_amdgcn_s_waitcnt((LDS ? 0x0070 : 0x0F70) | (PENDING & 15) | (PENDING >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");  // (neither of the two keeps a read of LDS behind it)
  TSENOR_IN_ORDER();
}
constexpr int kAnyPending = 63;

// Which tile a workgroup takes: the ones that run on an XCD at a time (workgroups go round the eight) are neighbours, four rows of
// tiles high, and share its L2.  (14336 x 4096 x 8192: 374 us; 2 high 390, 8 high 376, 16 high 379, without XCDs 385-400.)
constexpr int kXcds = 8, kTilesHigh = 4;
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int& tile_m, int& tile_n) {
  const int total = tiles_m * tiles_n, per = total / kXcds, rest = total % kXcds, xcd = id % kXcds;
  id = xcd * per + min(xcd, rest) + id / kXcds;
  const int first = id / (kTilesHigh * tiles_n) * kTilesHigh, high = min(kTilesHigh, tiles_m - first), at = id - first * tiles_n;
  tile_m = first + at % high, tile_n = at / high;
}

// what a wave needs to load its quarter of the rows of one operand into LDS: piece j (0..2 T - 1) is 8 rows of LDS
template <int T>
struct Loader {
  intx4 from;
  uint32_t to;      // LDS address of its rows in the first buffer
  int lane[2 * T];  // offset of the lane in memory, for every piece

  __device__ __forceinline__ Loader(const uint8_t* values, int64_t ld, int first, int rows, int lane_id, int wave, uint32_t lds) {
    from = resource_of(values + first * ld, min(64 * T, rows - first) * ld);
    to = lds + wave * 16 * T * kBlock;
#pragma unroll
    for (int j = 0; j < 2 * T; ++j) {
      const int at = wave * 16 * T + 8 * j + lane_id / 8;                             // row of LDS
      const int row = at / (32 * T) * (32 * T) + at % 32 * T + at % (32 * T) / 32;    // row of the tile
      lane[j] = min(row, rows - 1 - first) * (int)ld + (lane_id % 8 ^ at / 2 % 8) * 16;
    }
  }
  __device__ __forceinline__ void load(int buffer, int j, int column) const { load_to_lds(to + buffer + j * 1024, lane[j], from, column); }
};

// scale bytes of T neighbouring rows
template <int T>
__device__ __forceinline__ int load_scales(const uint8_t* p) {
  if constexpr (T == 4)
    return *reinterpret_cast<const int*>(p);
  else if constexpr (T == 2)
    return *reinterpret_cast<const uint16_t*>(p);
  else
    return *p;
}

// the lane's 4 T results of row `row` from column `col` on, in pairs
template <int T>
__device__ __forceinline__ void write_results(const ProductArgs& p, int64_t row, int col, uint32_t (&w)[2 * T]) {
  if (row >= p.m) return;
  const bool whole = col + 4 * T <= p.n;
  if (p.mask) {
    const uint8_t* mask = p.mask + row * p.mask_ld + col;
    uint8_t keep[4 * T];
    if (whole) {
      __builtin_memcpy(keep, mask, 4 * T);
    } else {
#pragma unroll
      for (int e = 0; e < 4 * T; ++e) keep[e] = col + e < p.n ? mask[e] : 0;
    }
#pragma unroll
    for (int e = 0; e < 2 * T; ++e) w[e] &= (keep[2 * e] ? 0xFFFFu : 0u) | (keep[2 * e + 1] ? 0xFFFF0000u : 0u);
  }
  uint16_t* out = p.out + row * p.out_ld + col;
  if (whole) {
    __builtin_memcpy(out, w, 8 * T);
  } else {
#pragma unroll
    for (int e = 0; e < 4 * T; ++e)
      if (col + e < p.n) out[e] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
  }
}
// Piece g of what a lane holds of tile j of a goes out: element 4 g + e of its 16 is row 8 g + 4 q + e of its tile of b, which is row
// TN (8 g + 4 q + e) + tile of its wave.
template <int TN, int TM>
__device__ __forceinline__ void write_piece(const ProductArgs& p, int m0, int n0, int j, int g, const floatx4 (&v)[TN]) {
  const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave, r = lane % 32, q = lane / 32;
  uint32_t w[2 * TN];
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int t = 0; t < TN; t += 2) w[(e * TN + t) / 2] = pack_bf16(v[t][e], v[t + 1][e]);
  write_results<TN>(p, m0 + (wave / 2 * 32 + r) * TM + j, n0 + (wave % 2 * 32 + 8 * g + 4 * q) * TN, w);
}

// SPLIT: p.splits workgroups share the columns of a tile, and each leaves its sums in p.parts, piece by piece.
template <int TN, int TM, int BUFFERS>
constexpr int kGroupsPerCu = BUFFERS * TileShape<TN, TM>::kBuffer <= 80 * 1024 ? 2 : 1;
template <int TN, int TM, int BUFFERS, bool SPLIT>
__global__ __launch_bounds__(256, (kGroupsPerCu<TN, TM, BUFFERS>)) void tile_kernel(ProductArgs p) {
  using Shape = TileShape<TN, TM>;
  __shared__ __align__(1024) uint8_t lds[BUFFERS * Shape::kBuffer];
  const int lane = (int)threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int wave_n = wave % 2, wave_m = wave / 2, r = lane % 32, q = lane / 32;
  int tile_m, tile_n;
  const int tiles = p.tiles_m * p.tiles_n, split = SPLIT ? (int)blockIdx.x / tiles : 0;
  tile_of((int)blockIdx.x - split * tiles, p.tiles_m, p.tiles_n, tile_m, tile_n);
  const int first = SPLIT ? (int)((int64_t)p.blocks * split / p.splits) : 0;
  const int last = (SPLIT ? (int)((int64_t)p.blocks * (split + 1) / p.splits) : p.blocks) - 1;
  const int m0 = tile_m * Shape::kRowsA, n0 = tile_n * Shape::kRowsB;

  const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  const Loader<TN> of_b(p.b.values, p.b.ld, n0, p.n, lane, wave, lds_at);
  const Loader<TM> of_a(p.a.values, p.a.ld, m0, p.m, lane, wave, lds_at + Shape::kRowsB * kBlock);
  // scales of the tile's rows, four to a lane, of b to the even waves and of a to the odd ones
  const int scale_rows = wave % 2 ? p.m - m0 : p.n - n0, scale_ld = (int)(wave % 2 ? p.a.scale_ld : p.b.scale_ld);
  const intx4 of_scales = resource_of(wave % 2 ? p.a.scales + m0 : p.b.scales + n0, (int64_t)p.blocks * scale_ld);
  const int scale_lane = 4 * lane < scale_rows ? 4 * lane : 0;
  const auto load = [&](int buffer, int piece, int block) {
    if (piece < 2 * TN)
      of_b.load(buffer, piece, block * kBlock);
    else if (piece < 2 * TN + 2 * TM)
      of_a.load(buffer, piece - 2 * TN, block * kBlock);
    else
      load_dword_to_lds(lds_at + buffer + Shape::kValues + wave % 2 * 256, scale_lane, of_scales, block * scale_ld);
  };

  // pieces 4 h + 2 q and 4 h + 2 q + 1 of row r: half h of the columns changes bit 6 of the place
  const int place[2] = {r * kBlock + ((2 * q) ^ (r / 2 % 8)) * 16, r * kBlock + ((2 * q + 1) ^ (r / 2 % 8)) * 16};
  const uint8_t* const rows_b = lds + wave_n * 32 * TN * kBlock;
  const uint8_t* const rows_a = lds + (Shape::kRowsB + wave_m * 32 * TM) * kBlock;
  const uint8_t* const scales_b = lds + Shape::kValues + (wave_n * 32 + r) * TN;
  const uint8_t* const scales_a = lds + Shape::kValues + 256 + (wave_m * 32 + r) * TM;
  intx8 b[TN][2], a[TM][2];  // tile, half of the columns
  const auto fetch = [&](const uint8_t* rows, int tile, int h) {
    const intx4 lo = *reinterpret_cast<const intx4*>(rows + tile * 32 * kBlock + (place[0] ^ h * 64));
    const intx4 hi = *reinterpret_cast<const intx4*>(rows + tile * 32 * kBlock + (place[1] ^ h * 64));
    return intx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  };

  floatx16 sum[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[i][j][e] = 0.0f;

  // With more than two buffers the loads of a block are spread over the second half of a step and the first of the next.
  // (A block past the last is the last one again, which nothing uses.)
  constexpr int kEarly = BUFFERS > 2 ? (Shape::kPieces + 1) / 2 : Shape::kPieces;  // loads of a block in the second half
#pragma unroll
  for (int k = 0; k < BUFFERS; ++k)
#pragma unroll
    for (int piece = 0; piece < (k == BUFFERS - 1 ? kEarly : Shape::kPieces); ++piece) load(k * Shape::kBuffer, piece, min(first + k, last));
  meet<(BUFFERS - 2) * Shape::kPieces + kEarly>();
  int scale_b = load_scales<TN>(scales_b), scale_a = load_scales<TM>(scales_a), next_b, next_a;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    b[0][h] = fetch(rows_b, 0, h), a[0][h] = fetch(rows_a, 0, h);
    if constexpr (TN == 4) b[1][h] = fetch(rows_b, 1, h);
    if constexpr (TN == 2 && TM == 4) a[1][h] = fetch(rows_a, 1, h);
  }

// The instructions of a step stand in the order in which they are issued: a matrix instruction takes 64 cycles, in which a few others
// can be issued, so reads of LDS, loads and multiplications are spread evenly.  (The statement behind each multiplication
// does nothing but keep it from being moved past the next.)
#define MULTIPLY(i, j, h)                                                                                                 \
  sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[i][h], a[j][h], sum[i][j], 0, 0, i, scale_b, j, scale_a);  \
  asm volatile("" : "+a"(sum[i][j]));                                                                                    \
  TSENOR_IN_ORDER();
#define FETCH_B(rows, t, h) b[t][h] = fetch(rows##_b, t, h); TSENOR_IN_ORDER();
#define FETCH_A(rows, t, h) a[t][h] = fetch(rows##_a, t, h); TSENOR_IN_ORDER();
#define LOAD(piece) if constexpr (piece < kEarly) { load(buffer, piece, ahead); TSENOR_IN_ORDER(); }
#define LATE(piece) if constexpr (piece >= kEarly) { load(old_buffer, piece, ahead_of_old); TSENOR_IN_ORDER(); }
#define FETCH_SCALES()                                                                                        \
  next_b = load_scales<TN>(scales_b + next_buffer), next_a = load_scales<TM>(scales_a + next_buffer);         \
  TSENOR_IN_ORDER();
  constexpr int kPending = (BUFFERS - 2) * Shape::kPieces;  // loads of the blocks after the next
  int buffer = 0, next_buffer = Shape::kBuffer, old_buffer = (BUFFERS - 1) * Shape::kBuffer;
  for (int block = first; block <= last; ++block) {
    const uint8_t *const this_b = rows_b + buffer, *const this_a = rows_a + buffer;
    const uint8_t *const next_rows_b = rows_b + next_buffer, *const next_rows_a = rows_a + next_buffer;
    const int ahead = min(block + BUFFERS, last), ahead_of_old = min(block + BUFFERS - 1, last);
    TSENOR_IN_ORDER();
    if constexpr (TN == 4 && TM == 4) {
      MULTIPLY(0, 0, 0) FETCH_A(this, 1, 0) MULTIPLY(1, 0, 0) FETCH_A(this, 1, 1) MULTIPLY(0, 0, 1) FETCH_A(this, 2, 0)
      MULTIPLY(1, 0, 1) FETCH_A(this, 2, 1) MULTIPLY(0, 1, 0) FETCH_A(this, 3, 0) MULTIPLY(1, 1, 0) FETCH_A(this, 3, 1)
      MULTIPLY(0, 1, 1) FETCH_B(this, 2, 0) MULTIPLY(1, 1, 1) FETCH_B(this, 2, 1) MULTIPLY(0, 2, 0) FETCH_B(this, 3, 0)
      MULTIPLY(1, 2, 0) FETCH_B(this, 3, 1) MULTIPLY(0, 2, 1) MULTIPLY(1, 2, 1)
      MULTIPLY(0, 3, 0) MULTIPLY(1, 3, 0) MULTIPLY(0, 3, 1) MULTIPLY(1, 3, 1)
      meet<kAnyPending>();
      MULTIPLY(2, 2, 0) LOAD(0) MULTIPLY(3, 2, 0) LOAD(1) MULTIPLY(2, 2, 1) LOAD(2) MULTIPLY(3, 2, 1) LOAD(3)
      MULTIPLY(2, 3, 0) LOAD(4) MULTIPLY(3, 3, 0) LOAD(5) MULTIPLY(2, 3, 1) LOAD(6) MULTIPLY(3, 3, 1) LOAD(7)
      // only here the next block has to have come: a quarter of a step more for its loads, which two buffers leave little time
      meet<8, false>();
      MULTIPLY(2, 0, 0) FETCH_B(next_rows, 0, 0) LOAD(8) MULTIPLY(3, 0, 0) FETCH_B(next_rows, 1, 0) LOAD(9)
      MULTIPLY(2, 0, 1) FETCH_B(next_rows, 0, 1) LOAD(10) MULTIPLY(3, 0, 1) FETCH_B(next_rows, 1, 1) LOAD(11)
      MULTIPLY(2, 1, 0) FETCH_A(next_rows, 0, 0) LOAD(12) MULTIPLY(3, 1, 0) FETCH_A(next_rows, 0, 1) LOAD(13)
      MULTIPLY(2, 1, 1) FETCH_SCALES() LOAD(14) MULTIPLY(3, 1, 1) LOAD(15) LOAD(16)
    } else if constexpr (TN == 2 && TM == 4) {
      MULTIPLY(0, 0, 0) FETCH_B(this, 1, 0) MULTIPLY(0, 1, 0) FETCH_B(this, 1, 1) LATE(7) MULTIPLY(0, 0, 1) FETCH_A(this, 2, 0) LATE(8)
      MULTIPLY(0, 1, 1) FETCH_A(this, 2, 1) LATE(9) MULTIPLY(1, 0, 0) FETCH_A(this, 3, 0) LATE(10) MULTIPLY(1, 1, 0) FETCH_A(this, 3, 1) LATE(11)
      MULTIPLY(1, 0, 1) LATE(12) MULTIPLY(1, 1, 1)
      meet<kPending>();
      MULTIPLY(0, 2, 0) LOAD(0) FETCH_A(next_rows, 0, 0) MULTIPLY(0, 3, 0) LOAD(1) MULTIPLY(0, 2, 1) LOAD(2) FETCH_A(next_rows, 0, 1)
      MULTIPLY(0, 3, 1) LOAD(3) FETCH_SCALES() MULTIPLY(1, 2, 0) LOAD(4) FETCH_B(next_rows, 0, 0)
      MULTIPLY(1, 3, 0) LOAD(5) FETCH_B(next_rows, 0, 1) MULTIPLY(1, 2, 1) LOAD(6) FETCH_A(next_rows, 1, 0) MULTIPLY(1, 3, 1) FETCH_A(next_rows, 1, 1)
    } else if constexpr (TN == 2 && TM == 2) {
      MULTIPLY(0, 0, 0) FETCH_A(this, 1, 0) FETCH_A(this, 1, 1) LATE(5) MULTIPLY(0, 0, 1) FETCH_B(this, 1, 0) FETCH_B(this, 1, 1) LATE(6)
      MULTIPLY(0, 1, 0) LATE(7) LATE(8) MULTIPLY(0, 1, 1)
      meet<kPending>();
      MULTIPLY(1, 0, 0) LOAD(0) LOAD(1) FETCH_B(next_rows, 0, 0) MULTIPLY(1, 0, 1) LOAD(2) LOAD(3) FETCH_B(next_rows, 0, 1) FETCH_SCALES()
      MULTIPLY(1, 1, 0) LOAD(4) LOAD(5) FETCH_A(next_rows, 0, 0) MULTIPLY(1, 1, 1) LOAD(6) LOAD(7) LOAD(8) FETCH_A(next_rows, 0, 1)
    } else {
      static_assert(TN == 2 && TM == 1);
      MULTIPLY(0, 0, 0) FETCH_B(this, 1, 0) FETCH_B(this, 1, 1) LATE(4) LATE(5) LATE(6) MULTIPLY(0, 0, 1)
      meet<kPending>();
      MULTIPLY(1, 0, 0) LOAD(0) LOAD(1) FETCH_B(next_rows, 0, 0) FETCH_B(next_rows, 0, 1) FETCH_SCALES()
      MULTIPLY(1, 0, 1) LOAD(2) LOAD(3) FETCH_A(next_rows, 0, 0) FETCH_A(next_rows, 0, 1)
    }
    scale_b = next_b, scale_a = next_a;
    old_buffer = buffer, buffer = next_buffer, next_buffer += Shape::kBuffer;
    if (next_buffer == BUFFERS * Shape::kBuffer) next_buffer = 0;
  }
#undef MULTIPLY
#undef FETCH_B
#undef FETCH_A
#undef LOAD
#undef LATE
#undef FETCH_SCALES
  meet<0>();  // (no load into LDS outlives the workgroup)

#pragma unroll
  for (int j = 0; j < TM; ++j)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      floatx4 v[TN];
#pragma unroll
      for (int t = 0; t < TN; ++t) {
        v[t] = floatx4{sum[t][j][4 * g], sum[t][j][4 * g + 1], sum[t][j][4 * g + 2], sum[t][j][4 * g + 3]};
        if (SPLIT) p.parts[((int64_t)blockIdx.x * (TM * 4 * TN) + (j * 4 + g) * TN + t) * 256 + threadIdx.x] = v[t];
      }
      if (!SPLIT) write_piece<TN, TM>(p, m0, n0, j, g, v);
    }
}

// adds what the workgroups that shared a tile left, in their order: a workgroup for each tile and piece
template <int TN, int TM>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs p) {
  using Shape = TileShape<TN, TM>;
  const int tiles = p.tiles_m * p.tiles_n, tile = (int)blockIdx.x / (4 * TM), piece = (int)blockIdx.x % (4 * TM);
  int tile_m, tile_n;
  tile_of(tile, p.tiles_m, p.tiles_n, tile_m, tile_n);
  const floatx4* part = p.parts + ((int64_t)tile * (TM * 4 * TN) + piece * TN) * 256 + threadIdx.x;
  const int64_t step = (int64_t)tiles * (TM * 4 * TN) * 256;
  floatx4 v[TN];
#pragma unroll
  for (int t = 0; t < TN; ++t) v[t] = part[t * 256];
#pragma unroll 4
  for (int k = 1; k < p.splits; ++k)
#pragma unroll
    for (int t = 0; t < TN; ++t) v[t] += part[k * step + t * 256];
  write_piece<TN, TM>(p, tile_m * Shape::kRowsA, tile_n * Shape::kRowsB, piece / 4, piece % 4, v);
}

// a sum over no columns
__global__ __launch_bounds__(256) void zero_kernel(ProductArgs p) {
  const int64_t total = (int64_t)p.m * p.n;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < total; k += (int64_t)gridDim.x * 256) p.out[k / p.n * p.out_ld + k % p.n] = 0;
}

// ---- host ------------------------------------------------------------------------------------------------------------------
constexpr int64_t kMaxProductLd = (int64_t)1 << 22;  // (offsets within the rows of a tile have 31 bits)

int check(const tsenor_product_problem* p) {
  if (!p || (p->a.rows != 0 && p->b.rows != 0 && !p->out)) return TSENOR_ERR_NULL;
  int rc = check_scaled(p->a);
  if (rc != TSENOR_OK) return rc;
  rc = check_scaled(p->b);
  if (rc != TSENOR_OK) return rc;
  if (p->a.cols != p->b.cols || p->b.rows > (int64_t)1 << 24 || !shape_ok(p->a.rows, p->b.rows) || !ld_ok(p->out_ld, p->a.rows, p->b.rows))
    return TSENOR_ERR_SHAPE;
  const int64_t blocks = blocks_of(p->a.cols);
  for (const tsenor_scaled* s : {&p->a, &p->b})
    if (s->ld > kMaxProductLd || s->scale_ld > INT32_MAX || blocks * s->scale_ld > INT32_MAX) return TSENOR_ERR_SHAPE;
  return aligned_to(p->out, 2) ? TSENOR_OK : TSENOR_ERR_ALIGN;
}

void launch(const tsenor_product_problem& p, const Part& part, void* workspace, hipStream_t s) {
  ProductArgs a = {};
  a.a = p.a, a.b = p.b, a.out = static_cast<uint16_t*>(p.out) + part.m0 * p.out_ld + part.n0, a.out_ld = p.out_ld;
  a.a.values += part.m0 * p.a.ld, a.a.scales += part.m0, a.b.values += part.n0 * p.b.ld, a.b.scales += part.n0;
  a.mask = p.mask ? p.mask + part.m0 * p.b.rows + part.n0 : nullptr, a.mask_ld = p.b.rows;
  a.m = (int)part.m, a.n = (int)part.n, a.blocks = (int)blocks_of(p.a.cols);
  a.tiles_m = part.tiles_m, a.tiles_n = part.tiles_n, a.splits = part.splits, a.parts = static_cast<floatx4*>(workspace);
  const unsigned tiles = (unsigned)(part.tiles_m * part.tiles_n), groups = tiles * (unsigned)part.splits;
  switch (part.kind) {
    case kNoColumns: zero_kernel<<<(unsigned)std::min<int64_t>(((int64_t)a.m * a.n + 255) / 256, 65536), 256, 0, s>>>(a); break;
    case kFewRows: few_rows_kernel<<<(unsigned)((a.n + 15) / 16), kWaves * kWave, 0, s>>>(a); break;
    case kSmallTile:
      if (part.splits > 1) {
        tile_kernel<2, 1, 6, true><<<groups, 256, 0, s>>>(a);
        join_kernel<2, 1><<<tiles * 4, 256, 0, s>>>(a);
      } else {
        tile_kernel<2, 1, 6, false><<<groups, 256, 0, s>>>(a);
      }
      break;
    case kTile: tile_kernel<2, 2, 4, false><<<groups, 256, 0, s>>>(a); break;
    case kTilePairs: tile_kernel<2, 2, 2, false><<<groups, 256, 0, s>>>(a); break;
    case kWideTile: tile_kernel<2, 4, 3, false><<<groups, 256, 0, s>>>(a); break;
    case kLargeTile: tile_kernel<4, 4, 2, false><<<groups, 256, 0, s>>>(a); break;
  }
}

}  // namespace

extern "C" size_t tsenor_product_workspace_bytes(const tsenor_product_problem* p) {
  return check(p) == TSENOR_OK ? plan_of(p->a.rows, p->b.rows, blocks_of(p->a.cols)).workspace : 0;
}

extern "C" int tsenor_product(const tsenor_product_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream) {
  const int rc = check(p);
  if (rc != TSENOR_OK) return rc;
  const Plan plan = plan_of(p->a.rows, p->b.rows, blocks_of(p->a.cols));
  if (plan.count == 0) return TSENOR_OK;
  if (plan.workspace && (!workspace || !aligned_to(workspace, 256) || workspace_bytes < plan.workspace)) return TSENOR_ERR_WORKSPACE;
  for (int k = 0; k < plan.count; ++k) launch(*p, plan.parts[k], workspace, static_cast<hipStream_t>(stream));
  return status_of_launches();
}
