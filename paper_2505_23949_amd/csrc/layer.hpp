// What the layer operators (tsenor_layer.h) share: loads and stores of rows, the 8-bit format with its scales, checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lanes.hpp"
#include "tsenor.h"
#include "tsenor_layer.h"

namespace tsenor_dev {

// TSENOR_OK or TSENOR_ERR_HIP for the launches since the last call (tsenor.hip)
int status_of_launches();

constexpr int kBlock = TSENOR_SCALE_BLOCK;
constexpr uint32_t kInfinityBits = 0x7F800000u;

// ---- host: checks ----------------------------------------------------------------------------------------------------
inline bool aligned_to(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline size_t size_of(int dtype) { return dtype == TSENOR_BF16 ? 2 : 4; }
inline bool known(int dtype) { return dtype == TSENOR_F32 || dtype == TSENOR_BF16; }
inline int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }
// (rows: the last row of a tile of 256 still has a 32-bit number; tiles: a grid counts fewer than 2^32 threads, and takes
// 512 for each tile to quantise it, 256 for each half of one in a product)
constexpr int64_t kMaxRows = INT32_MAX - 255;
inline bool shape_ok(int64_t rows, int64_t cols) {
  return rows >= 0 && rows <= kMaxRows && cols >= 0 && cols <= (int64_t)1 << 24 && blocks_of(rows) * blocks_of(cols) < (int64_t)1 << 23;
}
// (the offset of every row, in elements, is below 2^60: bytes have 63 bits)
constexpr int64_t kMaxLd = (int64_t)1 << 40, kMaxElements = (int64_t)1 << 60;
inline bool ld_ok(int64_t ld, int64_t rows, int64_t cols) { return ld >= cols && ld <= kMaxLd && (rows == 0 || ld <= kMaxElements / rows); }
inline int check_scaled(const tsenor_scaled& s) {
  if (s.rows != 0 && s.cols != 0 && (!s.values || !s.scales)) return TSENOR_ERR_NULL;
  if (!shape_ok(s.rows, s.cols) || !ld_ok(s.ld, s.rows, s.cols) || !ld_ok(s.scale_ld, blocks_of(s.cols), s.rows)) return TSENOR_ERR_SHAPE;
  if (s.ld < blocks_of(s.cols) * kBlock) return TSENOR_ERR_SHAPE;
  if (!aligned_to(s.values, 16) || !aligned_to(s.scales, 16) || s.ld % kBlock || s.scale_ld % 16) return TSENOR_ERR_ALIGN;
  return TSENOR_OK;
}

// ---- device: rows ----------------------------------------------------------------------------------------------------
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
// two values rounded to bf16 (nearest, ties to even), the first in the low half
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, bf16x2));
}

// 8 elements of a row from column `c` on, as floats; 0 past the last column.  Rows may begin anywhere: a load of 16 bytes needs no
// alignment here, and an 8192 x 8192 bf16 matrix with rows of 8195 elements is quantised in 58 us, with loads of 2 bytes in 125.
template <bool BF16>
struct Raw8 {
  uint32_t w[BF16 ? 4 : 8];
};
// As it stands in memory, so that nothing waits for it yet: the last elements of a row, where fewer than 8 are left, come as the last 8
// of it, and are put in place when they are used.  (With loads of single elements, which have to be waited for and joined, the norm's
// backward pass of bf16 1973 x 3844 took 32.5 us, 25.4 so, and 2377 x 14111 96, 82.)
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> load_raw8(const void* row, int c, int cols) {
  Raw8<BF16> raw = {};
  if (c + 8 <= cols) {
    __builtin_memcpy(raw.w, static_cast<const char*>(row) + c * (BF16 ? 2 : 4), sizeof(raw.w));
  } else if (cols >= 8) {
    if (c < cols) __builtin_memcpy(raw.w, static_cast<const char*>(row) + (cols - 8) * (BF16 ? 2 : 4), sizeof(raw.w));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c + k < cols) {
        if constexpr (BF16)
          raw.w[k / 2] |= (uint32_t)static_cast<const uint16_t*>(row)[c + k] << (k % 2 * 16);
        else
          raw.w[k] = static_cast<const uint32_t*>(row)[c + k];
      }
  }
  return raw;
}
template <bool BF16>
__device__ __forceinline__ void widen8(const Raw8<BF16>& raw, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if constexpr (BF16)
      x[k] = __uint_as_float(k % 2 ? raw.w[k / 2] & 0xFFFF0000u : raw.w[k / 2] << 16);
    else
      x[k] = __uint_as_float(raw.w[k]);
  }
}
template <bool BF16>
__device__ __forceinline__ void widen8(const Raw8<BF16>& raw, int c, int cols, float (&x)[8]) {
  widen8<BF16>(raw, x);
  if (c + 8 <= cols || cols < 8) return;
  const int past = c + 8 - cols;  // the first `past` of them belong to columns before c (and all are 0 from cols on)
#pragma unroll
  for (int step = 4; step > 0; step /= 2)
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = past & step ? (k + step < 8 ? x[k + step] : 0.0f) : x[k];
}
template <bool BF16>
__device__ __forceinline__ void load_row8(const void* row, int c, int cols, float (&x)[8]) {
  widen8<BF16>(load_raw8<BF16>(row, c, cols), c, cols, x);
}

// the same way back, rounded once
template <bool BF16>
__device__ __forceinline__ void store_row8(void* row, int c, int cols, const float (&x)[8]) {
  if constexpr (BF16) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = pack_bf16(x[2 * k], x[2 * k + 1]);
    if (c + 8 <= cols) {
      __builtin_memcpy(static_cast<uint16_t*>(row) + c, w, 16);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < cols) static_cast<uint16_t*>(row)[c + k] = (uint16_t)(w[k / 2] >> (k % 2 * 16));
    }
  } else {
    if (c + 8 <= cols) {
      __builtin_memcpy(static_cast<float*>(row) + c, x, 32);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < cols) static_cast<float*>(row)[c + k] = x[k];
    }
  }
}

// ---- device: the 8-bit format ------------------------------------------------------------------------------------------
// |x| as bits that compare like it; 0 for infinities and NaN, which no scale is made for
__device__ __forceinline__ uint32_t finite_size(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < kInfinityBits ? u : 0u;
}
// Byte of the smallest power of two s with largest <= 448 s: 448 = 1.75 * 2^8, so the exponent of `largest` goes down by 8, and up
// by one where its fraction is above 1.75, which a carry does.  At least 2^-126: its reciprocal is finite, and so is that of
// the largest one, 2^120.
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest) {
  const int e = (int)((largest + 0x1FFFFFu) >> 23) - 8;
  return largest == 0u ? 127u : (uint32_t)max(e, 1);
}
__device__ __forceinline__ float inverse_of_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// values times a power of two (exact but for results below 2^-126, which are 0 in 8 bits) to the nearest 8-bit ones, ties to even
__device__ __forceinline__ uint32_t to_8bit(float a, float b, float c, float d, float inverse) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, low, true);
}
__device__ __forceinline__ uint2 to_8bit(const float (&x)[8], float inverse) {
  return make_uint2(to_8bit(x[0], x[1], x[2], x[3], inverse), to_8bit(x[4], x[5], x[6], x[7], inverse));
}

// largest over the 16 lanes of a DPP row, in all of them
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
  v = max(v, (uint32_t)lane_xor_i32<1>((int)v));
  v = max(v, (uint32_t)lane_xor_i32<2>((int)v));
  v = max(v, (uint32_t)lane_xor_i32<7>((int)v));
  return max(v, (uint32_t)lane_xor_i32<15>((int)v));
}

// sum over the wave, in all lanes, the same bits in each
__device__ __forceinline__ float wave_sum(float v) {
  v += lane_xor<1>(v);
  v += lane_xor<2>(v);
  v += lane_xor<7>(v);
  v += lane_xor<15>(v);
  v += lane_xor<16>(v);
  return v + lane_xor<32>(v);
}

}  // namespace tsenor_dev
