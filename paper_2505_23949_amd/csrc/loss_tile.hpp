// The tile kernel of the losses' products, C[row][col] = sum_k a(row, k) b(col, k), in its three uses:
//   kLogits   a: states   (along the sum)    b: head (along)        z = h W^T, its rows' sums and exponentials
//   kLogitsInPlace                              the same, of a head whose rows end inside a line of 128 bytes
//   kLogitsCounted, kLogitsInPlaceCounted       the same, exponentials counted from c.refs
//   kStates   a: dz       (along)            b: head (across)       dh = dz W
//   kHead     a: dz       (across)           b: states (across)     dW = dz^T h
// "Along": a row of the operand lies along the sum in memory.  "Across": the sum goes from row to row of memory.
#pragma once
#include <algorithm>

#include "loss.hpp"

namespace tsenor_dev {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef int intx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

enum Use { kLogits, kLogitsInPlace, kLogitsCounted, kLogitsInPlaceCounted, kStates, kHead };
constexpr bool makes_logits(int use) { return use < kStates; }
constexpr bool is_counted(int use) { return use == kLogitsCounted || use == kLogitsInPlaceCounted; }
constexpr bool is_in_place(int use) { return use == kLogitsInPlace || use == kLogitsInPlaceCounted; }

// A workgroup of 2 WM waves, two side by side, takes 64 TN rows of b (columns of the result) and 32 TM WM rows of a; a wave 32 TN x 32 TM
// results in accumulators, of the 32 x 32 matrix instructions whose first operand is b: a lane holds four neighbouring columns of a row.
// 64 columns of the sum, 128 bytes of a row, are a block; blocks come into a ring of BUFFERS in LDS by loads that go there directly.
//   Along: 128 bytes of LDS to a row; piece c of 16 bytes of row r stands at place c ^ (r / 2 % 8), so that the lanes that LDS serves
//   at a time take all banks.
//   Across: a row of LDS holds one column of the sum for all rows of the operand, and reads that transpose 4 x 16 values on the way give a
//   lane four columns of the sum for its row; the 64-byte chunks of LDS rows k are exchanged by k % 4 (chunk c stands at c ^ (k % 4)),
//   so that the four rows of such a read take different banks.
//   The order of the columns in the sum is free as long as both operands agree on it: half q of a wave holds, of half h of a block, its
//   columns 32 h + 16 q to 32 h + 16 q + 15.
//
// Single precision: x = x1 + x2 + x3 exactly, with x1 the nearest (finite) bf16 value to x, x2 to x - x1 and x3 the rest, and of the nine products of
// two such sums six are made, x1 y1, x1 y2, x2 y1, x2 y2, x1 y3 and x3 y1; the others are below 2^-25 of x y.  bf16 products run 16 times as
// fast as those of fp32, so six of them take 0.4 of one in fp32.  Rows of the operands then hold three planes one behind the other, and the
// sum goes over six pairs of planes, as if it were six times as long.
//
// What bounds it: 256 x 256 is held by the card's power (8192 tokens x 128256 x 4096: 1.5-1.6 GHz, matrix cores busy 74-81 % of the cycles;
// the loss alone of 4096 x 128256 x 4096 3.22-3.37 ms, of operands that are all zeros 2.51).  dh of 8192 x 128256 x 4096, two rounds of 2004 blocks,
// 6.29 ms: 1.57 us a block of one tile on each CU, 1.37 PFLOP/s.  Logits of 1433 x 50257 x 1024, five rounds of 16 blocks, 164 us: 33 us a round, of
// which 8 are not its blocks.  Four rows of waves (WM) put two waves on a SIMD, of which one works while the other waits: with two, and twice the
// rows to a wave, dW of 1433 x 50257 x 1024 took 169 us (157 so); full rounds are about the same (dh of 4096 x 32768 x 4096 806 and 813).
template <int TN, int TM, int WM>
struct TileShape {
  static constexpr int kWaves = 2 * WM, kThreads = kWaves * kWave;
  static constexpr int kRowsB = 64 * TN, kRowsA = 32 * TM * WM;
  static constexpr int kBuffer = (kRowsB + kRowsA) * 128;                                // bytes of a block; b's rows first
  static constexpr int kPiecesB = kRowsB / 8 / kWaves, kPiecesA = kRowsA / 8 / kWaves;  // loads that a wave makes for a block
  static constexpr int kPieces = kPiecesB + kPiecesA;
};

// Which planes of a and b block `block` of the sum takes, and which of their `per` blocks.  The five pairs whose products are small come first
// (each 64 columns' in turn, so that their planes are still in L2), the large one last: the accumulators are rounded at their full size
// only as often as one product would.  (dW of 1000 x 5003 x 769: 1.6e-6 off with all six in turn, 7e-7 so; with each pair for the
// whole sum the same and 6 % slower.)
template <bool BF16>
struct Place {
  int plane_a, plane_b, at;
  __device__ __forceinline__ Place(int block, int per) {
    if constexpr (BF16) {
      plane_a = plane_b = 0, at = block;
    } else {
      if (block < 5 * per) {
        const int pair = block % 5;
        plane_a = 0x052 >> 2 * pair & 3, plane_b = 0x118 >> 2 * pair & 3, at = block / 5;  // 2 0 1 1 0 and 0 2 1 0 1
      } else {
        plane_a = plane_b = 0, at = block - 5 * per;
      }
    }
  }
};

// Loads a wave's share of ROWS rows of an operand, PIECES times 8; `plane_bytes`: from plane to plane of a row.
// PART: rows end inside a line: what follows them is read for its rest, and behind the last row something inside (the other operand has
// zeros there).  A kernel of its own, because the choice costs each load a branch: 10 % of the product.
// T > 1: row 32 t + r of each 32 T rows of LDS is row T r + t of memory, so that a lane gets T times as many neighbouring columns.
template <int ROWS, int PIECES, int T, bool PART>
struct LoaderAlong {
  intx4 from;
  uint32_t to, past;  // past: offset of the last 16 bytes
  int plane_bytes, whole, lane[PIECES];
  __device__ __forceinline__ LoaderAlong(const void* p, int64_t ld_bytes, int plane_bytes_, int row_bytes, int first, int rows, int lane_id, int wave,
                                         uint32_t lds) {
    const int count = min(ROWS, rows - first);
    past = (uint32_t)(count - 1) * (uint32_t)ld_bytes + row_bytes - 16;
    from = resource_of(static_cast<const char*>(p) + first * ld_bytes, (int64_t)past + 16);
#pragma unroll
    for (int k = 0; k < 4; ++k) from[k] = __builtin_amdgcn_readfirstlane(from[k]);  // (the same in all lanes: it has to be in scalar registers)
    to = lds + wave * PIECES * 1024;
    plane_bytes = plane_bytes_, whole = row_bytes / 128;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      const int at = (wave * PIECES + j) * 8 + lane_id / 8;
      const int row = at / (32 * T) * (32 * T) + at % 32 * T + at % (32 * T) / 32;
      lane[j] = (int)((uint32_t)min(row, count - 1) * (uint32_t)ld_bytes + (lane_id % 8 ^ at / 2 % 8) * 16);  // (32 bits, unsigned)
    }
  }
  __device__ __forceinline__ void load(int buffer, int j, int plane, int at) const {
    if (!PART || at < whole)
      load_to_lds(to + buffer + j * 1024, lane[j], from, plane * plane_bytes + at * 128);
    else
      load_to_lds(to + buffer + j * 1024, (int)min((uint32_t)lane[j] + at * 128, past), from, 0);  // (rows of one plane)
  }
};

// `count` columns of the sum, `row_bytes` bytes of operand in each plane.  What lies past either end is read as something inside: past the
// last column the other operand is zero, and past the last row nothing is written.
template <int ROWS, int WAVES>
struct LoaderAcross {
  static constexpr int kRowBytes = 2 * ROWS, kAtOnce = 1024 / kRowBytes;
  static_assert(WAVES * kAtOnce % 4 == 0 && kRowBytes >= 128);
  const char* base;
  int64_t ld_bytes, past;  // past: offset of the last 16 bytes of a plane
  uint32_t to;
  int plane_bytes, lane, step;
  __device__ __forceinline__ LoaderAcross(const void* p, int64_t ld_bytes_, int row_bytes, int first, int count, int lane_id, int wave, uint32_t lds) {
    base = static_cast<const char*>(p), ld_bytes = ld_bytes_, plane_bytes = row_bytes, past = (count - 1) * ld_bytes + row_bytes - 16;
    to = lds + wave * 1024;
    const int k = wave * kAtOnce + lane_id * 16 / kRowBytes, at = lane_id * 16 % kRowBytes, swap = kRowBytes >= 256 ? k % 4 : k / 2 % 2;
    lane = k * (int)ld_bytes + min(first * 2 + (at ^ swap * 64), row_bytes - 16);
    step = WAVES * kAtOnce * (int)ld_bytes;
  }
  __device__ __forceinline__ void load(int buffer, int j, int plane, int at) const {
    const int64_t begin = at * (64 * ld_bytes);
    const int limit = (int)min(past - begin, (int64_t)INT32_MAX - 16), offset = min(j * step, limit);
    load_to_lds(to + buffer + j * WAVES * 1024, min(lane, limit - offset), resource_of(base + begin + plane * plane_bytes, (int64_t)limit + 16), offset);
  }
};

// Reads one of a wave's T tiles of 32 rows: half h of the sum's columns of a block.
template <int T, int ROWS, bool ALONG>
struct Reader {
  static constexpr int kRowBytes = 2 * ROWS;
  int place[ALONG ? 2 : T];
  __device__ __forceinline__ Reader(int lane, int wave) {  // wave: which 32 T of the ROWS rows
    const int r = lane % 32, q = lane / 32;
    if constexpr (ALONG) {
      place[0] = wave * 32 * T * 128 + r * 128 + ((2 * q) ^ (r / 2 % 8)) * 16;
      place[1] = wave * 32 * T * 128 + r * 128 + ((2 * q + 1) ^ (r / 2 % 8)) * 16;
    } else {
      const int i = lane % 16, k = 16 * q + i / 4, swap = kRowBytes >= 256 ? k % 4 : k / 2 % 2;
#pragma unroll
      for (int t = 0; t < T; ++t) place[t] = k * kRowBytes + ((wave * T + t) ^ swap) * 64 + lane / 16 % 2 * 32 + i % 4 * 8;
    }
  }
  __device__ __forceinline__ intx8 fetch(const uint8_t* rows, int t, int h) const {
    if constexpr (ALONG) {
      const intx4 lo = *reinterpret_cast<const intx4*>(rows + t * 4096 + (place[0] ^ h * 64));
      const intx4 hi = *reinterpret_cast<const intx4*>(rows + t * 4096 + (place[1] ^ h * 64));
      return intx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    } else {
      typedef __attribute__((address_space(3))) shortx4* Lds;
      intx2 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        v[u] = __builtin_bit_cast(intx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(rows + place[t] + (32 * h + 4 * u) * kRowBytes)));
      return intx8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
    }
  }
};

__device__ __forceinline__ floatx16 multiply(const intx8& b, const intx8& a, floatx16 sum) {
  const intx4 b0 = {b[0], b[1], b[2], b[3]}, b1 = {b[4], b[5], b[6], b[7]}, a0 = {a[0], a[1], a[2], a[3]}, a1 = {a[4], a[5], a[6], a[7]};
  sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b0), __builtin_bit_cast(bf16x8, a0), sum, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b1), __builtin_bit_cast(bf16x8, a1), sum, 0, 0, 0);
}

// columns col .. col + 3 of a row of n
__device__ __forceinline__ void store4(float* to, const floatx4& v, int col, int n) {
  if (col + 4 <= n) {
    __builtin_memcpy(to, &v, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < n) to[e] = v[e];
  }
}

// Adds columns col + 4 q .. (lo) and col + 8 + 4 q .. (hi) of a row of dW that begins at element `at` to the sums of the pieces before.
template <bool BF16>
__device__ __forceinline__ void add_gradient(const LossCall& c, int row, int64_t at, int col, floatx4 lo, floatx4 hi) {
  const int q = (int)threadIdx.x / 32 % 2, n = c.width;
  float* const sums = BF16 ? c.dweight_sum : static_cast<float*>(c.dweight);
  const auto add = [&](floatx4& v, int col) {
    if (row < 0) return;
    float* const to = sums + at + col;
    if (c.first > 0) {
      float old[4];
      if (col + 4 <= n) {
        __builtin_memcpy(old, to, 16);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) old[e] = col + e < n ? to[e] : 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += old[e];
    }
    if (!BF16 || !c.last) {
      store4(to, v, col, n);
    } else {
      uint16_t* const out = static_cast<uint16_t*>(c.dweight) + at + col;
      const uint32_t w[2] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
      if (col + 4 <= n) {
        __builtin_memcpy(out, w, 8);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (col + e < n) out[e] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
      }
    }
  };
  add(lo, col + 4 * q);
  add(hi, col + 8 + 4 * q);
}

// How many workgroups share the sum of each of `tiles` tiles: more than planned where tokens that are left out leave fewer of them.
__device__ __forceinline__ int splits_of(const LossCall& c, int tiles) { return min(c.groups / max(tiles, 1), kMaxSplits); }

template <int TN, int TM, int WM, int BUFFERS>
constexpr int kWavesPerSimd = BUFFERS * TileShape<TN, TM, WM>::kBuffer <= 80 * 1024 ? 2 : WM / 2;

// Gradients leave a wave 32 rows at a time, through LDS, so that a store writes whole lines: the lanes hold a few columns of 32 rows each.
// (1 x 116621 x 5083 in fp32, whose dW is 2.4 GB: 3584 -> 3397 us.  The exponentials, 32 to 64 bytes of a row to a lane, gain nothing by it.)
template <int TN, int SIZE>
struct Staged {
  static constexpr int kRowBytes = 32 * TN * SIZE, kStride = kRowBytes + 16;
};
// bytes of LDS of a workgroup: its buffers, or 32 rows of fp32 results for each wave
template <int TN, int TM, int WM, int BUFFERS>
constexpr int kLds = std::max(BUFFERS * TileShape<TN, TM, WM>::kBuffer, TileShape<TN, TM, WM>::kWaves * 32 * Staged<TN, 4>::kStride);
// row_at(row): where a row's columns go, NULL for none; `valid`: bytes of a row that there are
template <int TN, int SIZE, class RowAt>
__device__ __forceinline__ void store_staged(const uint8_t* staged, int valid, RowAt row_at) {
  using S = Staged<TN, SIZE>;
  constexpr int kPieces = S::kRowBytes / 16;
  const int lane = (int)threadIdx.x % kWave, piece = lane % kPieces;
#pragma unroll
  for (int i = 0; i < 32 * kPieces / kWave; ++i) {
    const int row = i * (kWave / kPieces) + lane / kPieces;
    const intx4 v = *reinterpret_cast<const intx4*>(staged + row * S::kStride + piece * 16);
    char* const to = row_at(row);
    if (!to) continue;
    if (piece * 16 + 16 <= valid) {
      __builtin_memcpy(to + piece * 16, &v, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 16 / SIZE; ++e)
        if (piece * 16 + (e + 1) * SIZE <= valid) {
          if constexpr (SIZE == 2)
            reinterpret_cast<uint16_t*>(to)[piece * 8 + e] = (uint16_t)(v[e / 2] >> (e % 2 * 16));
          else
            reinterpret_cast<int*>(to)[piece * 4 + e] = v[e];
        }
    }
  }
}

// Exponentials of a row counted from one number: a lane's sums up to here are taken (2^22 of them stay far inside single precision, and what they
// are divided by, times a weight, inside its other end).  Nothing can be counted from minus infinity, either.
constexpr float kMostOverRef = 0x1p59f;

// What becomes of a tile of logits.
template <bool BF16, bool COUNTED, int TN, int TM>
__device__ __forceinline__ void finish_logits(const LossCall& c, floatx16 (&sum)[TN][TM], int m, int n, int m0, int n0, uint8_t* lds) {
  const int lane = (int)threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int wave_n = wave % 2, wave_m = wave / 2, r = lane % 32, q = lane / 32;
  uint8_t* const staged = lds + wave * 32 * Staged<TN, 4>::kStride;  // the wave's own
  // a lane holds, of row 32 j + r of its wave's rows of a, columns TN (8 g + 4 q + e) + t of its wave's rows of b.  The sums of a row are
  // of those 32 TN columns: no wave waits for another.
  const int wave_col = n0 + wave_n * 32 * TN, col0 = wave_col + 4 * TN * q;
  constexpr float kBits = exp_bits(BF16, COUNTED);
  // Entries: a wave puts 32 rows into LDS, where their entries' columns can be picked.  (distill 4096 x 128256 x 4096 with 128 entries:
  // read again, their rows of the head would be 4 GB, 1 ms)
  const bool only = c.k == 1;
  uint32_t entries[TM];  // of the only one of a row, its column among the wave's; of several, where they begin and end
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    const int row = m0 + (wave_m * TM + j) * 32 + r;
    entries[j] = only ? UINT32_MAX : 0;
    if (row < m && wave_col < n) {
      if (only)
        entries[j] = (uint32_t)((TM > 1 ? c.words[row] : word_of(c, row)) - wave_col);
      else if (TM > 1 || c.sorted)
        __builtin_memcpy(&entries[j], c.begins + (int64_t)row * (c.tiles + 1) + wave_col / (32 * TN), 4);
    }
  }
  // several entries that nothing has put in order (direct calls, which have small tiles): the wave looks at all of its rows'.  use(row of the 32, entry, column)
  const auto look = [&](auto use) {
    const int rows = min(m - (m0 + wave_m * 32), 32);
    for (int i = lane; i < rows * c.k; i += kWave) {
      const int row = i / c.k;
      const int64_t id = c.ids[(int64_t)(c.first + m0 + wave_m * 32 + row) * c.ids_ld + (i - row * c.k)];
      if (id >= wave_col && id < min(wave_col + 32 * TN, n)) use(row, i - row * c.k, (int)id - wave_col);
    }
  };
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    const int row = m0 + (wave_m * TM + j) * 32 + r;
    const int64_t at = (int64_t)row * c.dz_ld;
    TSENOR_IN_ORDER();
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int k = j; k < TM; ++k) asm volatile("" : "+a"(sum[t][k]));  // (accumulators stay what they are until their turn)
    if (wave_col + 32 * TN > n) {
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (col0 + TN * (e / 4 * 8 + e % 4) + t >= n) sum[t][j][e] = -__builtin_inff();
    }
    const bool apart = only && __any(entries[j] < 32 * TN);  // the exponential of one among them
    bool some = (entries[j] & 0xFFFFu) != entries[j] >> 16;
    if constexpr (TM == 1)
      if (!only && !c.sorted) look([&](int, int, int) { some = true; });
    if (apart || (!only && __any(some))) {
      float* const logits = reinterpret_cast<float*>(staged + r * Staged<TN, 4>::kStride);
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; e += 4 / TN) {
          floatx4 v;
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = sum[k % TN][j][4 * g + e + k / TN];
          *reinterpret_cast<floatx4*>(logits + TN * (8 * g + 4 * q + e)) = v;
        }
      if (only) {
        if (q == 0 && entries[j] < 32 * TN) c.dots[row] = logits[entries[j]];
      } else if (TM == 1 && !c.sorted) {
        look([&](int k, int i, int col) {
          c.dots[(int64_t)(m0 + wave_m * 32 + k) * c.k + i] = reinterpret_cast<const float*>(staged + k * Staged<TN, 4>::kStride)[col];
        });
      } else {
        for (int i = (int)(entries[j] & 0xFFFFu) + q; i < (int)(entries[j] >> 16); i += 2) {
          const uint32_t key = c.sorted[(int64_t)row * c.k + i];
          c.dots[(int64_t)row * c.k + (key & 255)] = logits[(int)(key >> 8) - wave_col];
        }
      }
    }
    float largest = -__builtin_inff();
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) largest = fmaxf(largest, sum[t][j][e]);
    largest = fmaxf(largest, lane_xor<32>(largest));
    if (COUNTED && row < m) largest = c.refs[row];
    const float base = largest == -__builtin_inff() ? 0.0f : largest;
    float v = 0.0f, of_group[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float x[4 * TN];
      of_group[g] = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < TN; ++t) {
          x[e * TN + t] = exp_from(sum[t][j][4 * g + e], base, c.scale, kBits);
          of_group[g] += x[e * TN + t];
        }
      const int col = col0 + 8 * TN * g;
      if (c.exps && row < m && col < c.dz_ld) {
        if constexpr (BF16) {
          uint32_t w[2 * TN];
#pragma unroll
          for (int k = 0; k < 2 * TN; ++k)
            w[k] = COUNTED ? pack_bf16(x[2 * k], x[2 * k + 1]) : __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{x[2 * k], x[2 * k + 1]}, halfx2));
          __builtin_memcpy(__builtin_assume_aligned(static_cast<uint16_t*>(c.exps) + at + col, 16), w, 8 * TN);
        } else {
          __builtin_memcpy(__builtin_assume_aligned(static_cast<float*>(c.exps) + at + col, 16), x, 16 * TN);
        }
      }
    }
    if constexpr (COUNTED) {
      v = (of_group[0] + of_group[1]) + (of_group[2] + of_group[3]);
      if (row < m && (v > kMostOverRef || largest == -__builtin_inff())) *c.again = 1;  // (whoever finds one writes the same)
    }
    if (apart) {  // a row's only entry: the group that it is in once more, without it, rather than a comparison with each word
      const int target = (int)min(entries[j], (uint32_t)(32 * TN - 1)), group = target / (4 * TN);  // (of other rows, the last: not used)
      const float* const logits = reinterpret_cast<const float*>(staged + r * Staged<TN, 4>::kStride) + group * 4 * TN;
      float rest = 0.0f;
#pragma unroll
      for (int e = 0; e < 4 * TN; ++e) {
        const float x = exp_from(logits[e], base, c.scale, kBits);
        rest += e == target % (4 * TN) ? 0.0f : x;
      }
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (entries[j] < 32 * TN && group == 2 * g + q) of_group[g] = rest;
    }
    v = (of_group[0] + of_group[1]) + (of_group[2] + of_group[3]);
    v += lane_xor<32>(v);
    if (q == 0 && row < m && wave_col < n) c.sums[(int64_t)row * c.tiles + wave_col / (32 * TN)] = make_float2(largest, v);
  }
}

// SPLIT: several workgroups share the sum of a tile, and each leaves its part in c.parts.  kMaybe: where c.groups says so.
enum Split { kNever, kAlways, kMaybe };
template <bool BF16, int USE, int TN, int TM, int WM, int BUFFERS, int SPLIT>
__device__ __forceinline__ void tile(const LossCall& c, const int id, uint8_t* lds) {
  using Shape = TileShape<TN, TM, WM>;
  constexpr int kPlanes = BF16 ? 1 : 3;
  constexpr bool kAlongB = makes_logits(USE), kAlongA = USE != kHead;
  const int lane = (int)threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int wave_n = wave % 2, wave_m = wave / 2, r = lane % 32, q = lane / 32;
  const int piece = __builtin_amdgcn_readfirstlane(rows_of(c));
  const int m = USE == kHead ? c.head_rows : piece, n = makes_logits(USE) ? c.vocab : c.width;
  const int tiles_m = (m + Shape::kRowsA - 1) / Shape::kRowsA, tiles_n = (n + Shape::kRowsB - 1) / Shape::kRowsB;
  const int tiles = tiles_m * tiles_n;
  const bool shared = SPLIT == kAlways || (SPLIT == kMaybe && c.groups > 0);
  const int splits = shared ? splits_of(c, tiles) : 1;
  if (id >= tiles * splits) return;  // (of a piece without tokens that count, all of them)
  const int split = shared ? id / tiles : 0;
  const int per = makes_logits(USE) ? c.states_ld / 64 : USE == kStates ? c.dz_ld / 64 : (piece + 63) / 64, all_blocks = per * (BF16 ? 1 : kPairs);
  if (USE == kHead && all_blocks == 0 && c.first > 0 && !c.last) return;
  int tile_m, tile_n;
  tile_of(id - split * tiles, tiles_m, tiles_n, tile_m, tile_n);
  const int first = shared ? (int)((int64_t)all_blocks * split / splits) : 0;
  const int last = (shared ? (int)((int64_t)all_blocks * (split + 1) / splits) : all_blocks) - 1;
  const int m0 = tile_m * Shape::kRowsA, n0 = tile_n * Shape::kRowsB;
  const int first_row = USE == kHead ? c.head_first : 0;

  floatx16 sum[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[i][j][e] = 0.0f;

  const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  const int states = c.states_ld * 2, dz = c.dz_ld * 2;  // bytes of a row of a plane (of the head: as of the states)
  const auto of_b = [&] {
    if constexpr (makes_logits(USE))
      return LoaderAlong<Shape::kRowsB, Shape::kPiecesB, TN, is_in_place(USE)>(c.head, c.head_ld * 2, states, c.head_bytes * kPlanes, n0, n, lane, wave, lds_at);
    else if constexpr (USE == kStates)
      return LoaderAcross<Shape::kRowsB, Shape::kWaves>(c.head, c.head_ld * 2, c.head_bytes, n0, c.vocab, lane, wave, lds_at);
    else
      return LoaderAcross<Shape::kRowsB, Shape::kWaves>(c.states, (int64_t)states * kPlanes, states, n0, (piece + 63) / 64 * 64, lane, wave, lds_at);
  }();
  const uint32_t lds_a = lds_at + Shape::kRowsB * 128;
  const auto of_a = [&] {
    if constexpr (makes_logits(USE))
      return LoaderAlong<Shape::kRowsA, Shape::kPiecesA, 1, false>(c.states, c.states_row * 2, states, states * kPlanes, m0, m, lane, wave, lds_a);
    else if constexpr (USE == kStates)
      return LoaderAlong<Shape::kRowsA, Shape::kPiecesA, 1, false>(c.dz, (int64_t)dz * kPlanes, dz, dz * kPlanes, m0, m, lane, wave, lds_a);
    else
      return LoaderAcross<Shape::kRowsA, Shape::kWaves>(c.dz, (int64_t)dz * kPlanes, dz, first_row + m0, piece, lane, wave, lds_a);
  }();
  const auto load = [&](int buffer, int k, const Place<BF16>& place) {
    if (k < Shape::kPiecesB)
      of_b.load(buffer, k, place.plane_b, place.at);
    else
      of_a.load(buffer, k - Shape::kPiecesB, place.plane_a, place.at);
  };
  const Reader<TN, Shape::kRowsB, kAlongB> read_b(lane, wave_n);
  const Reader<TM, Shape::kRowsA, kAlongA> read_a(lane, wave_m);
  const uint8_t *const rows_b = lds, *const rows_a = lds + Shape::kRowsB * 128;

  // With more than two buffers the loads of a block are spread over the second half of a step and the first of the next.
  // (A block past the last is the last one again, which nothing uses.)
  constexpr int kEarly = BUFFERS > 2 ? Shape::kPieces / 2 : Shape::kPieces;  // loads of a block in the second half
  intx8 b[TN][2], a[TM][2];                                                   // tile, half of the columns
  if (first <= last) {
#pragma unroll
    for (int k = 0; k < BUFFERS; ++k)
#pragma unroll
      for (int at = 0; at < (k == BUFFERS - 1 ? kEarly : Shape::kPieces); ++at) load(k * Shape::kBuffer, at, Place<BF16>(min(first + k, last), per));
    meet<(BUFFERS - 2) * Shape::kPieces + kEarly>();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      b[0][h] = read_b.fetch(rows_b, 0, h), a[0][h] = read_a.fetch(rows_a, 0, h);
      if constexpr (TN == 4) b[1][h] = read_b.fetch(rows_b, 1, h);
    }
  }

// The instructions of a step stand in the order in which they are issued: reads of LDS, loads and multiplications are spread evenly.
// (The statement behind each multiplication does nothing but keep it from being moved past the next.)
#define MULTIPLY(i, j, h)                               \
  sum[i][j] = multiply(b[i][h], a[j][h], sum[i][j]); \
  asm volatile("" : "+a"(sum[i][j]));                   \
  TSENOR_IN_ORDER();
#define FETCH_B(buffer, t, h) b[t][h] = read_b.fetch(rows_b + buffer, t, h); TSENOR_IN_ORDER();
#define FETCH_A(buffer, t, h) a[t][h] = read_a.fetch(rows_a + buffer, t, h); TSENOR_IN_ORDER();
#define LOAD(k) if constexpr (k < kEarly && k < Shape::kPieces) { load(buffer, k, ahead); TSENOR_IN_ORDER(); }
#define LATE(k) if constexpr (k >= kEarly && k < Shape::kPieces) { load(old_buffer, k, ahead_of_old); TSENOR_IN_ORDER(); }
  constexpr int kPending = (BUFFERS - 2) * Shape::kPieces;  // loads of the blocks after the next
  int buffer = 0, next_buffer = Shape::kBuffer, old_buffer = (BUFFERS - 1) * Shape::kBuffer;
  for (int block = first; block <= last; ++block) {
    const Place<BF16> ahead(min(block + BUFFERS, last), per), ahead_of_old(min(block + BUFFERS - 1, last), per);
    TSENOR_IN_ORDER();
    if constexpr (TN == 4 && TM == 2) {
      MULTIPLY(0, 0, 0) FETCH_A(buffer, 1, 0) MULTIPLY(1, 0, 0) FETCH_A(buffer, 1, 1) MULTIPLY(0, 0, 1) FETCH_B(buffer, 2, 0)
      MULTIPLY(1, 0, 1) FETCH_B(buffer, 2, 1) MULTIPLY(0, 1, 0) FETCH_B(buffer, 3, 0) MULTIPLY(1, 1, 0) FETCH_B(buffer, 3, 1)
      MULTIPLY(0, 1, 1) MULTIPLY(1, 1, 1)
      meet<kAnyPending>();
      MULTIPLY(2, 0, 0) LOAD(0) MULTIPLY(3, 0, 0) LOAD(1) MULTIPLY(2, 0, 1) LOAD(2) MULTIPLY(3, 0, 1) LOAD(3)
      meet<4, false>();
      MULTIPLY(2, 1, 0) FETCH_B(next_buffer, 0, 0) LOAD(4) MULTIPLY(3, 1, 0) FETCH_B(next_buffer, 0, 1) LOAD(5) FETCH_B(next_buffer, 1, 0)
      MULTIPLY(2, 1, 1) FETCH_B(next_buffer, 1, 1) LOAD(6) FETCH_A(next_buffer, 0, 0) MULTIPLY(3, 1, 1) LOAD(7) FETCH_A(next_buffer, 0, 1)
    } else if constexpr (TN == 2 && TM == 2) {
      MULTIPLY(0, 0, 0) FETCH_A(buffer, 1, 0) FETCH_A(buffer, 1, 1) LATE(3) LATE(4) MULTIPLY(0, 0, 1) FETCH_B(buffer, 1, 0) FETCH_B(buffer, 1, 1) LATE(5)
      MULTIPLY(0, 1, 0) LATE(6) LATE(7) MULTIPLY(0, 1, 1)
      meet<kPending>();
      MULTIPLY(1, 0, 0) LOAD(0) LOAD(1) FETCH_B(next_buffer, 0, 0) MULTIPLY(1, 0, 1) LOAD(2) LOAD(3) FETCH_B(next_buffer, 0, 1)
      MULTIPLY(1, 1, 0) LOAD(4) LOAD(5) FETCH_A(next_buffer, 0, 0) MULTIPLY(1, 1, 1) LOAD(6) LOAD(7) FETCH_A(next_buffer, 0, 1)
    } else {
      static_assert(TN == 2 && TM == 1);
      MULTIPLY(0, 0, 0) FETCH_B(buffer, 1, 0) FETCH_B(buffer, 1, 1) LATE(2) LATE(3) LATE(4) LATE(5) MULTIPLY(0, 0, 1)
      meet<kPending>();
      MULTIPLY(1, 0, 0) LOAD(0) LOAD(1) FETCH_B(next_buffer, 0, 0) LOAD(2) FETCH_B(next_buffer, 0, 1) LOAD(3)
      MULTIPLY(1, 0, 1) LOAD(4) LOAD(5) FETCH_A(next_buffer, 0, 0) FETCH_A(next_buffer, 0, 1)
    }
    old_buffer = buffer, buffer = next_buffer, next_buffer += Shape::kBuffer;
    if (next_buffer == BUFFERS * Shape::kBuffer) next_buffer = 0;
  }
#undef MULTIPLY
#undef FETCH_B
#undef FETCH_A
#undef LOAD
#undef LATE
  meet<0>();  // (no load into LDS outlives the workgroup)

  if constexpr (makes_logits(USE) && SPLIT == kNever) {
    finish_logits<BF16, is_counted(USE), TN, TM>(c, sum, m, n, m0, n0, lds);
  } else {
    if (shared) {
#pragma unroll
      for (int j = 0; j < TM; ++j)
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            c.parts[((int64_t)id * (TM * TN * 4) + (j * TN + t) * 4 + g) * Shape::kThreads + threadIdx.x] =
                floatx4{sum[t][j][4 * g], sum[t][j][4 * g + 1], sum[t][j][4 * g + 2], sum[t][j][4 * g + 3]};
      return;
    }
    if constexpr (makes_logits(USE)) return;
    const float scale = c.largest_weight[1];
    constexpr int kSize = BF16 ? 2 : 4;
    using Rows = Staged<TN, kSize>;
    uint8_t* const staged = lds + wave * 32 * Rows::kStride;
    const int wave_col = n0 + wave_n * 32 * TN;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int row = m0 + (wave_m * TM + j) * 32 + r;
      TSENOR_IN_ORDER();
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int k = j; k < TM; ++k) asm volatile("" : "+a"(sum[t][k]));  // (accumulators stay what they are until their turn)
      if (USE == kHead && (c.first > 0 || !c.last)) {  // sums of several pieces
        const int64_t at = (int64_t)(row >= m ? 0 : first_row + row) * c.width;
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            floatx4 lo, hi;
#pragma unroll
            for (int e = 0; e < 4; ++e) lo[e] = sum[t][j][8 * p + e] * scale, hi[e] = sum[t][j][8 * p + 4 + e] * scale;
            add_gradient<BF16>(c, row < m ? row : -1, at, wave_col + t * 32 + 16 * p, lo, hi);
          }
        continue;
      }
      const float2 factors = USE == kStates && c.row_scale ? c.row_scale[min(row, m - 1)] : make_float2(1.0f, 1.0f);
      const float of_row = factors.y * scale;
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = sum[t][j][4 * g + e] * factors.x * of_row;
          uint8_t* const to = staged + r * Rows::kStride + (32 * t + 8 * g + 4 * q) * kSize;
          if constexpr (BF16) {
            const uint32_t w[2] = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
            __builtin_memcpy(__builtin_assume_aligned(to, 8), w, 8);
          } else {
            __builtin_memcpy(__builtin_assume_aligned(to, 16), x, 16);
          }
        }
      // (kStates: lanes 0 to 31 know which token each row is of)
      const int token = USE == kStates ? c.order[c.first + min(row, m - 1)] : 0;
      char* const out = static_cast<char*>(USE == kStates ? c.dh : c.dweight) + (int64_t)wave_col * kSize;
      store_staged<TN, kSize>(staged, (n - wave_col) * kSize, [&](int k) -> char* {
        const int to = USE == kStates ? __shfl(token, k) : first_row + m0 + (wave_m * TM + j) * 32 + k;
        return m0 + (wave_m * TM + j) * 32 + k < m ? out + (int64_t)to * n * kSize : nullptr;
      });
    }
  }
}

template <bool BF16, int USE, int TN, int TM, int WM, int BUFFERS, int SPLIT>
__global__ __launch_bounds__((TileShape<TN, TM, WM>::kThreads), (kWavesPerSimd<TN, TM, WM, BUFFERS>)) void tile_kernel(LossCall c) {
  __shared__ __align__(1024) uint8_t lds[kLds<TN, TM, WM, BUFFERS>];
  tile<BF16, USE, TN, TM, WM, BUFFERS, SPLIT>(c, (int)blockIdx.x, lds);
}

// all of them once more, should that be needed, by as many workgroups as run at a time
template <int USE>
__global__ __launch_bounds__((TileShape<4, 2, 4>::kThreads)) void logits_again_kernel(LossCall c, int tiles) {
  __shared__ __align__(1024) uint8_t lds[kLds<4, 2, 4, 2>];
  if (!*c.again) return;
  for (int id = (int)blockIdx.x; id < tiles; id += (int)gridDim.x) {
    tile<true, USE, 4, 2, 4, 2, kNever>(c, id, lds);
    __syncthreads();
  }
}

// adds the parts of a tile in their order: a workgroup for each tile and 4 TN TM-th of it
template <bool BF16, int USE, int TN, int TM, int WM>
__device__ __forceinline__ void join(const LossCall& c, const int id) {
  using Shape = TileShape<TN, TM, WM>;
  const int piece = rows_of(c), m = USE == kHead ? c.head_rows : piece;
  const int tiles_m = (m + Shape::kRowsA - 1) / Shape::kRowsA, tiles_n = (c.width + Shape::kRowsB - 1) / Shape::kRowsB, tiles = tiles_m * tiles_n;
  const int tile = id / (TN * TM * 4), at_j = id / (4 * TN) % TM, t = id / 4 % TN, g = id % 4;
  if (tile >= tiles || (USE == kHead && piece == 0 && c.first > 0 && !c.last)) return;
  int tile_m, tile_n;
  tile_of(tile, tiles_m, tiles_n, tile_m, tile_n);
  const floatx4* part = c.parts + ((int64_t)tile * (TM * TN * 4) + (at_j * TN + t) * 4 + g) * Shape::kThreads + threadIdx.x;
  const int64_t step = (int64_t)tiles * (TM * TN * 4) * Shape::kThreads;
  const int splits = splits_of(c, tiles);
  floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  int k = 0;
  for (; k + 8 <= splits; k += 8) {
    floatx4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = part[(k + u) * step];
#pragma unroll
    for (int u = 0; u < 8; ++u) v += x[u];
  }
  for (; k < splits; ++k) v += part[k * step];
  const int wave = (int)threadIdx.x / kWave, row = tile_m * Shape::kRowsA + (wave / 2 * TM + at_j) * 32 + (int)threadIdx.x % 32;
  if (row >= m) return;
  const int col = tile_n * Shape::kRowsB + (wave % 2 * TN + t) * 32 + 8 * g + 4 * ((int)threadIdx.x / 32 % 2), n = c.width;
  const int64_t at = (int64_t)(USE == kStates ? c.order[c.first + row] : c.head_first + row) * n + col;
  const float2 factors = USE == kStates && c.row_scale ? c.row_scale[row] : make_float2(1.0f, 1.0f);
  const float of_row = factors.y * c.largest_weight[1];
  float x[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = v[e] * factors.x * of_row;
  if constexpr (USE == kHead) {
    float* const sums = (BF16 ? c.dweight_sum : static_cast<float*>(c.dweight)) + at;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c.first > 0 && col + e < n) x[e] += sums[e];
    if (BF16 && !c.last) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < n) sums[e] = x[e];
      return;
    }
  }
  void* const out = USE == kStates ? c.dh : c.dweight;
  if constexpr (BF16) {
    const uint32_t w[2] = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    uint16_t* const to = static_cast<uint16_t*>(out) + at;
    if (col + 4 <= n) {
      __builtin_memcpy(to, w, 8);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < n) to[e] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
    }
  } else {
    store4(static_cast<float*>(out) + at, floatx4{x[0], x[1], x[2], x[3]}, col, n);
  }
}

template <bool BF16, int USE, int TN, int TM, int WM>
__global__ __launch_bounds__((TileShape<TN, TM, WM>::kThreads)) void join_kernel(LossCall c) {
  join<BF16, USE, TN, TM, WM>(c, (int)blockIdx.x);
}

// Both gradients of a small call in one launch: the first `groups` workgroups make dh, the others dW.
template <bool BF16, int TN, int TM, int WM, int BUFFERS>
__global__ __launch_bounds__((TileShape<TN, TM, WM>::kThreads), (kWavesPerSimd<TN, TM, WM, BUFFERS>)) void both_kernel(LossCall dh, LossCall head, int groups) {
  __shared__ __align__(1024) uint8_t lds[kLds<TN, TM, WM, BUFFERS>];
  if ((int)blockIdx.x < groups)
    tile<BF16, kStates, TN, TM, WM, BUFFERS, kMaybe>(dh, (int)blockIdx.x, lds);
  else
    tile<BF16, kHead, TN, TM, WM, BUFFERS, kMaybe>(head, (int)blockIdx.x - groups, lds);
}
template <bool BF16, int TN, int TM, int WM>
__global__ __launch_bounds__((TileShape<TN, TM, WM>::kThreads)) void join_both_kernel(LossCall dh, LossCall head, int groups) {
  if ((int)blockIdx.x < groups)
    join<BF16, kStates, TN, TM, WM>(dh, (int)blockIdx.x);
  else
    join<BF16, kHead, TN, TM, WM>(head, (int)blockIdx.x - groups);
}
template <bool BF16, int TN, int TM, int WM, int BUFFERS>
void launch_both(const LossCall& c, const BothPlan& plan, hipStream_t s) {
  const int tiles_dh = plan.dh.tiles_m * plan.dh.tiles_n, tiles_head = plan.dweight.tiles_m * plan.dweight.tiles_n;
  LossCall dh = c, head = c;
  dh.groups = plan.dh.splits > 1 ? tiles_dh * plan.dh.splits : 0, head.groups = plan.dweight.splits > 1 ? tiles_head * plan.dweight.splits : 0;
  head.parts = c.parts + plan.dh.workspace / sizeof(floatx4);
  const int groups = tiles_dh * plan.dh.splits;
  both_kernel<BF16, TN, TM, WM, BUFFERS><<<(unsigned)(groups + tiles_head * plan.dweight.splits), TileShape<TN, TM, WM>::kThreads, 0, s>>>(dh, head, groups);
  const int join_dh = dh.groups ? tiles_dh * TN * TM * 4 : 0, join_head = head.groups ? tiles_head * TN * TM * 4 : 0;
  if (join_dh + join_head) join_both_kernel<BF16, TN, TM, WM><<<(unsigned)(join_dh + join_head), TileShape<TN, TM, WM>::kThreads, 0, s>>>(dh, head, join_dh);
}

// the same of logits: a workgroup to a tile, which takes the place of its first
template <bool BF16, int TN, int TM, int WM>
__global__ __launch_bounds__((TileShape<TN, TM, WM>::kThreads)) void join_logits_kernel(LossCall c) {
  using Shape = TileShape<TN, TM, WM>;
  __shared__ __align__(16) uint8_t lds[TileShape<TN, TM, WM>::kWaves * 32 * Staged<TN, 4>::kStride];
  const int m = rows_of(c), n = c.vocab;
  const int tiles_m = (m + Shape::kRowsA - 1) / Shape::kRowsA, tiles_n = (n + Shape::kRowsB - 1) / Shape::kRowsB, tiles = tiles_m * tiles_n;
  if ((int)blockIdx.x >= tiles) return;
  int tile_m, tile_n;
  tile_of((int)blockIdx.x, tiles_m, tiles_n, tile_m, tile_n);
  const floatx4* const part = c.parts + (int64_t)blockIdx.x * (TM * TN * 4) * Shape::kThreads + threadIdx.x;
  const int64_t step = (int64_t)tiles * (TM * TN * 4) * Shape::kThreads;
  floatx4 v[TM * TN * 4] = {};
  const int splits = splits_of(c, tiles);
  for (int k = 0; k < splits; ++k) {
#pragma unroll
    for (int at = 0; at < TM * TN * 4; ++at) v[at] += part[k * step + at * Shape::kThreads];
  }
  floatx16 sum[TN][TM];
#pragma unroll
  for (int j = 0; j < TM; ++j)
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[t][j][e] = v[(j * TN + t) * 4 + e / 4][e % 4];
  finish_logits<BF16, false, TN, TM>(c, sum, m, n, tile_m * Shape::kRowsA, tile_n * Shape::kRowsB, lds);
}

// the kernel with the tiles of a plan
template <bool BF16, int USE, int TN, int TM, int WM, int BUFFERS>
void launch_tiles(const LossCall& c, const ProductPlan& plan, hipStream_t s) {
  const unsigned tiles = (unsigned)(plan.tiles_m * plan.tiles_n);
  if constexpr (!makes_logits(USE) || (TM == 1 && WM == 2)) {
    if (plan.splits > 1) {
      LossCall shared = c;
      shared.groups = (int)tiles * plan.splits;
      tile_kernel<BF16, USE, TN, TM, WM, BUFFERS, kAlways><<<tiles * (unsigned)plan.splits, TileShape<TN, TM, WM>::kThreads, 0, s>>>(shared);
      if constexpr (makes_logits(USE))
        join_logits_kernel<BF16, TN, TM, WM><<<tiles, TileShape<TN, TM, WM>::kThreads, 0, s>>>(shared);
      else
        join_kernel<BF16, USE, TN, TM, WM><<<tiles * TN * TM * 4, TileShape<TN, TM, WM>::kThreads, 0, s>>>(shared);
      return;
    }
  }
  tile_kernel<BF16, USE, TN, TM, WM, BUFFERS, kNever><<<tiles, TileShape<TN, TM, WM>::kThreads, 0, s>>>(c);
}
template <bool BF16, int USE>
void launch_tiles(const LossCall& c, const ProductPlan& plan, hipStream_t s) {
  switch (plan.kind) {
    case kLargeTile: launch_tiles<BF16, USE, 4, 2, 4, 2>(c, plan, s); break;
    case kWideTile: launch_tiles<BF16, USE, 2, 2, 4, 3>(c, plan, s); break;
    case kTile: launch_tiles<BF16, USE, 2, 1, 4, 4>(c, plan, s); break;
    case kTilePairs: launch_tiles<BF16, USE, 2, 2, 2, 2>(c, plan, s); break;
    default: launch_tiles<BF16, USE, 2, 1, 2, 6>(c, plan, s); break;
  }
}

}  // namespace tsenor_dev
