// tsenor_quantize: a matrix into 8-bit floating point with a power of two per 128 values, along the rows, along the columns
// (the transposed matrix) or both, entries that a mask drops being 0.
//
// A workgroup takes a tile of 128 x 128: a block of either direction lies within it, so x is read once whatever is wanted.  A
// thread holds 4 x 8 of it: the row maxima are found over 16 lanes, the column maxima over 4 rows, 4 lanes and 8 waves,
// the tile's over all.  Its 4 rows of a column are one 4-byte piece of the transposed tile, which goes through LDS so that both
// results leave in whole 128-byte rows.  Bound by memory: 28672 x 8192 in single precision with a mask, both ways, 317 us
// (5.2 TB/s), bf16 4096 x 14336 both ways 51 us (4.6); one tile to a CU, 1024 x 4096, 6.8 us, 7.2 where
// the loads of a row wait for those of the one before; the 4-byte writes of the transposed tile conflict four ways in LDS.
// (8 x 8 to a thread, half as many waves, took 2, 12 and 43 % more.)
#include "layer.hpp"

namespace {

using namespace tsenor_dev;

struct QuantizeArgs {
  const void* x;
  const uint8_t* mask;
  int64_t ld;
  int rows, cols, tiles_across;
  tsenor_scaled out, out_t;
};

constexpr int kTileStride = kBlock + 8;  // bytes between columns of the transposed tile in LDS

constexpr int kRows = 4, kThreads = kBlock / kRows * (kBlock / 8), kWaves = kThreads / kWave;
template <bool BF16, bool SQUARE>
__global__ __launch_bounds__(kThreads) void quantize_kernel(QuantizeArgs a) {
  __shared__ __align__(16) uint8_t tile[kBlock * kTileStride];
  __shared__ uint32_t largest[kWaves][kBlock];
  const int t = (int)threadIdx.x, lane_col = t % 16 * 8, lane_row = t / 16 * kRows;
  const int tile_row = (int)(blockIdx.x / (unsigned)a.tiles_across), tile_col = (int)(blockIdx.x % (unsigned)a.tiles_across);
  const int64_t row0 = (int64_t)tile_row * kBlock + lane_row;
  const int col0 = tile_col * kBlock + lane_col;

  // All loads of a thread are asked for before the first is waited for: those of rows past the last read the last one.
  Raw8<BF16> raw[kRows];
  uint64_t keep[kRows];
  const auto row_of = [&](int r) { return min(row0 + r, (int64_t)a.rows - 1); };
  const int before = max(col0 + 8 - a.cols, 0);  // columns before col0 that the last 8 of a row begin with
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const char* const row = static_cast<const char*>(a.x) + row_of(r) * a.ld * (BF16 ? 2 : 4);
    if (a.cols >= 8)  // (without a condition of each thread's own: 1072 x 2928 6.6 us, with one 7.3)
      __builtin_memcpy(raw[r].w, row + (int64_t)(col0 - before) * (BF16 ? 2 : 4), sizeof(raw[r].w));
    else
      raw[r] = load_raw8<BF16>(row, col0, a.cols);
  }
  if (a.mask) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const uint8_t* const mask = a.mask + row_of(r) * a.cols;
      if (a.cols >= 8) {
        __builtin_memcpy(&keep[r], mask + (col0 - before), 8);
      } else {
        keep[r] = 0u;
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (col0 + c < a.cols) keep[r] |= (uint64_t)mask[col0 + c] << (c * 8);
      }
    }
  }
  __builtin_amdgcn_sched_barrier(0);

  float x[kRows][8];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    widen8<BF16>(raw[r], col0, a.cols, x[r]);
    if (row0 + r >= a.rows || col0 >= a.cols) {
#pragma unroll
      for (int c = 0; c < 8; ++c) x[r][c] = 0.0f;
    }
  }
  if (a.mask) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (a.cols >= 8) keep[r] >>= before % 8 * 8;  // (past the last column x is 0 whatever it says)
#pragma unroll
      for (int c = 0; c < 8; ++c) x[r][c] = (keep[r] >> (c * 8) & 0xFFu) ? x[r][c] : 0.0f;
    }
  }

  uint32_t of_row[kRows], of_col[8];
#pragma unroll
  for (int r = 0; r < kRows; ++r) of_row[r] = 0u;
#pragma unroll
  for (int c = 0; c < 8; ++c) of_col[c] = 0u;
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t u = finite_size(x[r][c]);
      of_row[r] = max(of_row[r], u), of_col[c] = max(of_col[c], u);
    }

  // largest of a column over the workgroup (of the tile, where all columns hold the same)
  const auto over_waves = [&](int column) {
    uint32_t m = largest[0][column];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = max(m, largest[w][column]);
    return m;
  };
  uint32_t square_byte = 0;
  if constexpr (SQUARE) {
    uint32_t m = 0;
#pragma unroll
    for (int r = 0; r < kRows; ++r) m = max(m, of_row[r]);
    m = row16_max(m);
    m = max(m, (uint32_t)lane_xor_i32<16>((int)m));
    m = max(m, (uint32_t)lane_xor_i32<32>((int)m));
    if (t % kWave == 0) largest[t / kWave][0] = m;
    __syncthreads();
    square_byte = scale_byte(over_waves(0));
  }

  if (a.out.values) {
    uint32_t bytes[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      bytes[r] = SQUARE ? square_byte : scale_byte(row16_max(of_row[r]));
      if (row0 + r < a.rows)
        *reinterpret_cast<uint2*>(a.out.values + (row0 + r) * a.out.ld + col0) = to_8bit(x[r], inverse_of_scale(bytes[r]));
    }
    if (lane_col == 0) {
      uint8_t* s = a.out.scales + (int64_t)tile_col * a.out.scale_ld + row0;
      if (row0 + kRows <= a.rows) {
        *reinterpret_cast<uint32_t*>(s) = bytes[0] | bytes[1] << 8 | bytes[2] << 16 | bytes[3] << 24;
      } else {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
          if (row0 + r < a.rows) s[r] = (uint8_t)bytes[r];
      }
    }
  }

  if (a.out_t.values) {
    uint32_t byte[8];
    if constexpr (SQUARE) {
#pragma unroll
      for (int c = 0; c < 8; ++c) byte[c] = square_byte;
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        uint32_t m = of_col[c];
        m = max(m, (uint32_t)lane_xor_i32<16>((int)m));
        m = max(m, (uint32_t)lane_xor_i32<32>((int)m));
        if (t % kWave < 16) largest[t / kWave][lane_col + c] = m;
      }
      __syncthreads();
#pragma unroll
      for (int c = 0; c < 8; ++c) byte[c] = scale_byte(over_waves(lane_col + c));
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      *reinterpret_cast<uint32_t*>(tile + (lane_col + c) * kTileStride + lane_row) =
          to_8bit(x[0][c], x[1][c], x[2][c], x[3][c], inverse_of_scale(byte[c]));
    }
    if (lane_row == 0) {
      uint8_t* s = a.out_t.scales + (int64_t)tile_row * a.out_t.scale_ld + col0;
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (col0 + c < a.cols) s[c] = (uint8_t)byte[c];
    }
    __syncthreads();
#pragma unroll
    for (int piece = t; piece < kBlock * 8; piece += kThreads) {
      const int column = piece / 8, at = piece % 8 * 16;
      const uint2 lo = *reinterpret_cast<const uint2*>(tile + column * kTileStride + at);
      const uint2 hi = *reinterpret_cast<const uint2*>(tile + column * kTileStride + at + 8);
      const int64_t row = (int64_t)tile_col * kBlock + column;
      if (row < a.cols)
        *reinterpret_cast<uint4*>(a.out_t.values + row * a.out_t.ld + (int64_t)tile_row * kBlock + at) =
            make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  }
}

int check(const tsenor_quantize_problem* p) {
  if (!p) return TSENOR_ERR_NULL;
  if (p->rows != 0 && p->cols != 0 && (!p->x || (!p->out.values && !p->out_t.values))) return TSENOR_ERR_NULL;
  if (!known(p->dtype) || (p->square != 0 && p->square != 1)) return TSENOR_ERR_UNSUPPORTED;
  if (!shape_ok(p->rows, p->cols) || !ld_ok(p->ld, p->rows, p->cols)) return TSENOR_ERR_SHAPE;
  if (p->out_t.values && p->rows > (int64_t)1 << 24) return TSENOR_ERR_SHAPE;
  if (!aligned_to(p->x, size_of(p->dtype))) return TSENOR_ERR_ALIGN;
  if (p->out.values) {
    if (p->out.rows != p->rows || p->out.cols != p->cols) return TSENOR_ERR_SHAPE;
    const int rc = check_scaled(p->out);
    if (rc != TSENOR_OK) return rc;
  }
  if (p->out_t.values) {
    if (p->out_t.rows != p->cols || p->out_t.cols != p->rows) return TSENOR_ERR_SHAPE;
    const int rc = check_scaled(p->out_t);
    if (rc != TSENOR_OK) return rc;
  }
  return TSENOR_OK;
}

void launch(const QuantizeArgs& a, bool bf16, bool square, dim3 grid, hipStream_t s) {
  if (bf16)
    square ? quantize_kernel<true, true><<<grid, kThreads, 0, s>>>(a) : quantize_kernel<true, false><<<grid, kThreads, 0, s>>>(a);
  else
    square ? quantize_kernel<false, true><<<grid, kThreads, 0, s>>>(a) : quantize_kernel<false, false><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace

extern "C" int tsenor_quantize(const tsenor_quantize_problem* p, tsenor_stream_t stream) {
  const int rc = check(p);
  if (rc != TSENOR_OK) return rc;
  if (p->rows == 0 || p->cols == 0) return TSENOR_OK;  // no entry, no block
  QuantizeArgs a = {};
  a.x = p->x, a.mask = p->mask, a.ld = p->ld;
  a.rows = (int)p->rows, a.cols = (int)p->cols, a.tiles_across = (int)blocks_of(p->cols);
  a.out = p->out, a.out_t = p->out_t;
  const dim3 grid((unsigned)(blocks_of(p->rows) * blocks_of(p->cols)));
  hipStream_t s = static_cast<hipStream_t>(stream);
  launch(a, p->dtype == TSENOR_BF16, p->square != 0, grid, s);
  return status_of_launches();
}
