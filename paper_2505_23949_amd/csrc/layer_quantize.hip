// tsenor_quantize: a matrix into 8-bit floating point with a power of two per 128 values, along the rows, along the columns
// (the transposed matrix) or both, entries that a mask drops being 0.
//
// A workgroup takes a tile of 128 x 128: a block of either direction lies within it, so x is read once whatever is wanted.  A
// thread holds 8 x 8 of it: the row maxima are found over 16 lanes, the column maxima over 8 rows, 4 lanes and 4 waves,
// the tile's over all.  Its 8 rows of a column are one 8-byte piece of the transposed tile, which goes through LDS so that both
// results leave in whole 128-byte rows.  Bound by memory.
#include "layer.hpp"

namespace {

using namespace tsenor_dev;

struct QuantizeArgs {
  const void* x;
  const uint8_t* mask;
  int64_t ld;
  int rows, cols, tiles_across;
  tsenor_scaled out, out_t;
  bool vec, mask_vec;  // rows of x begin at multiples of 16 bytes, rows of the mask at multiples of 8
};

constexpr int kThreads = 256;
constexpr int kTileStride = kBlock + 8;  // bytes between columns of the transposed tile in LDS

template <bool BF16, bool SQUARE>
__global__ __launch_bounds__(kThreads) void quantize_kernel(QuantizeArgs a) {
  __shared__ __align__(16) uint8_t tile[kBlock * kTileStride];
  __shared__ uint32_t largest[kThreads / kWave][kBlock];
  const int t = (int)threadIdx.x, lane_col = t % 16 * 8, lane_row = t / 16 * 8;
  const int tile_row = (int)(blockIdx.x / (unsigned)a.tiles_across), tile_col = (int)(blockIdx.x % (unsigned)a.tiles_across);
  const int64_t row0 = (int64_t)tile_row * kBlock + lane_row;
  const int col0 = tile_col * kBlock + lane_col;

  float x[8][8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const bool inside = row0 + r < a.rows;
    const char* row = static_cast<const char*>(a.x) + (inside ? row0 + r : 0) * a.ld * (BF16 ? 2 : 4);
    load_row8<BF16>(row, col0, inside ? a.cols : 0, a.vec, x[r]);
  }
  if (a.mask) {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      if (row0 + r >= a.rows) continue;
      const uint8_t* m = a.mask + (row0 + r) * a.cols;
      if (a.mask_vec && col0 + 8 <= a.cols) {
        const uint2 w = *reinterpret_cast<const uint2*>(m + col0);
#pragma unroll
        for (int c = 0; c < 8; ++c) x[r][c] = ((c < 4 ? w.x : w.y) >> (c % 4 * 8) & 0xFFu) ? x[r][c] : 0.0f;
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (col0 + c < a.cols && !m[col0 + c]) x[r][c] = 0.0f;
      }
    }
  }

  uint32_t of_row[8], of_col[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) of_row[k] = of_col[k] = 0u;
#pragma unroll
  for (int r = 0; r < 8; ++r)
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t u = finite_size(x[r][c]);
      of_row[r] = max(of_row[r], u), of_col[c] = max(of_col[c], u);
    }

  uint32_t square_byte = 0;
  if constexpr (SQUARE) {
    uint32_t m = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) m = max(m, of_row[r]);
    m = row16_max(m);
    m = max(m, (uint32_t)lane_xor_i32<16>((int)m));
    m = max(m, (uint32_t)lane_xor_i32<32>((int)m));
    if (t % kWave == 0) largest[t / kWave][0] = m;
    __syncthreads();
    square_byte = scale_byte(max(max(largest[0][0], largest[1][0]), max(largest[2][0], largest[3][0])));
  }

  if (a.out.values) {
    uint32_t bytes[2] = {0u, 0u};
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const uint32_t b = SQUARE ? square_byte : scale_byte(row16_max(of_row[r]));
      bytes[r / 4] |= b << (r % 4 * 8);
      if (row0 + r < a.rows)
        *reinterpret_cast<uint2*>(a.out.values + (row0 + r) * a.out.ld + col0) = to_8bit(x[r], inverse_of_scale(b));
    }
    if (lane_col == 0) {
      uint8_t* s = a.out.scales + (int64_t)tile_col * a.out.scale_ld + row0;
      if (row0 + 8 <= a.rows) {
        *reinterpret_cast<uint2*>(s) = make_uint2(bytes[0], bytes[1]);
      } else {
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (row0 + r < a.rows) s[r] = (uint8_t)(bytes[r / 4] >> (r % 4 * 8));
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
      for (int c = 0; c < 8; ++c) {
        const int k = lane_col + c;
        byte[c] = scale_byte(max(max(largest[0][k], largest[1][k]), max(largest[2][k], largest[3][k])));
      }
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const float column[8] = {x[0][c], x[1][c], x[2][c], x[3][c], x[4][c], x[5][c], x[6][c], x[7][c]};
      *reinterpret_cast<uint2*>(tile + (lane_col + c) * kTileStride + lane_row) = to_8bit(column, inverse_of_scale(byte[c]));
    }
    if (lane_row == 0) {
      uint8_t* s = a.out_t.scales + (int64_t)tile_row * a.out_t.scale_ld + col0;
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (col0 + c < a.cols) s[c] = (uint8_t)byte[c];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int piece = t + k * kThreads, column = piece / 8, at = piece % 8 * 16;
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
  if (!shape_ok(p->rows, p->cols) || !ld_ok(p->ld, p->cols)) return TSENOR_ERR_SHAPE;
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

}  // namespace

extern "C" int tsenor_quantize(const tsenor_quantize_problem* p, tsenor_stream_t stream) {
  const int rc = check(p);
  if (rc != TSENOR_OK) return rc;
  if (p->rows == 0 || p->cols == 0) return TSENOR_OK;  // no entry, no block
  QuantizeArgs a = {};
  a.x = p->x, a.mask = p->mask, a.ld = p->ld;
  a.rows = (int)p->rows, a.cols = (int)p->cols, a.tiles_across = (int)blocks_of(p->cols);
  a.out = p->out, a.out_t = p->out_t;
  a.vec = rows_of_vectors(p->x, p->ld, size_of(p->dtype));
  a.mask_vec = aligned_to(p->mask, 8) && p->cols % 8 == 0;
  const dim3 grid((unsigned)(blocks_of(p->rows) * blocks_of(p->cols)));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p->dtype == TSENOR_BF16)
    p->square ? quantize_kernel<true, true><<<grid, kThreads, 0, s>>>(a) : quantize_kernel<true, false><<<grid, kThreads, 0, s>>>(a);
  else
    p->square ? quantize_kernel<false, true><<<grid, kThreads, 0, s>>>(a) : quantize_kernel<false, false><<<grid, kThreads, 0, s>>>(a);
  return status_of_launches();
}
