// Logits of up to 16 tokens: the head is read once, straight into registers, whatever its rows begin at.
//
// A workgroup of eight waves takes 16 words.  The waves share the width, 32 columns at a time, and their sums meet in LDS.  A lane holds
// columns 8 (l / 16) to 8 (l / 16) + 7 of row l % 16, of a word and of a token; the words are the first operand of the matrix instruction,
// so that it ends up with four neighbouring words of a token.  Single precision takes the fp32 instruction: 16 rows are too few for its
// rate to matter (8 operations a byte).
// Against tiles of 64 x 128, which need operands in whole lines, and where few of them fill the GPU (us of the kernel): 2 x 534 x 6848
// 31, 12 so.
#include "loss.hpp"

namespace {

using namespace tsenor_dev;

constexpr int kWaves = 8, kAtOnce = 4;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));

template <bool BF16>
__device__ __forceinline__ floatx4 multiply(const Raw8<BF16>& b, const Raw8<BF16>& a, floatx4 sum) {
  if constexpr (BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), sum, 0, 0, 0);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.w[u]), __uint_as_float(a.w[u]), sum, 0, 0, 0);
    return sum;
  }
}

template <bool BF16>
__device__ __forceinline__ Raw8<BF16> load_whole(const char* row, int k) {
  Raw8<BF16> raw;
  __builtin_memcpy(raw.w, row + k * (BF16 ? 2 : 4), sizeof(raw.w));
  return raw;
}
// the same where the row may end
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> load_end(const char* row, int k, int width) {
  float x[8];
  load_row8<BF16>(row, k, width, x);
  Raw8<BF16> raw;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (!BF16)
      raw.w[e] = __float_as_uint(x[e]);
    else if (e % 2)
      raw.w[e / 2] = __float_as_uint(x[e - 1]) >> 16 | (__float_as_uint(x[e]) & 0xFFFF0000u);
  }
  return raw;
}

template <bool BF16>
__global__ __launch_bounds__(kWaves* kWave) void few_logits_kernel(LossCall c) {
  __shared__ floatx4 parts[kWaves][kWave];
  constexpr int kSize = BF16 ? 2 : 4;
  const int lane = (int)threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int rows = rows_of(c), first = (int)blockIdx.x * kFewWords;
  if (rows == 0) return;
  const int row = min(lane % 16, rows - 1), word = min(first + lane % 16, c.vocab - 1), at = lane / 16 * 8;  // (what lies past the last is not written)
  const char* const h = static_cast<const char*>(c.h) + (int64_t)(c.count ? c.order[c.first + row] : c.first + row) * c.h_ld * kSize;
  const char* const w = static_cast<const char*>(c.weight) + (int64_t)word * c.weight_ld * kSize;
  floatx4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  const int whole = c.width / 32;
  int k = wave;
  for (; k + (kAtOnce - 1) * kWaves < whole; k += kAtOnce * kWaves) {
    Raw8<BF16> x[kAtOnce], y[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) x[u] = load_whole<BF16>(w, (k + u * kWaves) * 32 + at), y[u] = load_whole<BF16>(h, (k + u * kWaves) * 32 + at);
    TSENOR_IN_ORDER();  // (all of them are asked for before the first is waited for)
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) sum = multiply<BF16>(x[u], y[u], sum);
  }
  for (; k < whole; k += kWaves) sum = multiply<BF16>(load_whole<BF16>(w, k * 32 + at), load_whole<BF16>(h, k * 32 + at), sum);
  if (k == whole && whole * 32 < c.width)  // (one of the waves)
    sum = multiply<BF16>(load_end<BF16>(w, whole * 32 + at, c.width), load_end<BF16>(h, whole * 32 + at, c.width), sum);
  parts[wave][lane] = sum;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int k = 1; k < kWaves; ++k) sum += parts[k][lane];

  // token lane % 16, words first + 4 (lane / 16) to + 3
  const int col = first + lane / 16 * 4, token = lane % 16;
  float largest = -__builtin_inff();
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (col + e >= c.vocab) sum[e] = -__builtin_inff();
    largest = fmaxf(largest, sum[e]);
  }
  largest = fmaxf(largest, lane_xor<16>(largest));
  largest = fmaxf(largest, lane_xor<32>(largest)) * c.scale - kExpBits;
  const float base = largest == -__builtin_inff() ? 0.0f : largest;
  float x[4], total = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = __builtin_amdgcn_exp2f(fmaf(sum[e], c.scale, -base));
    total += x[e];
  }
  total += lane_xor<16>(total);
  total += lane_xor<32>(total);
  if (token >= rows) return;
  if (lane < 16) c.sums[(int64_t)token * c.tiles + blockIdx.x] = make_float2(largest, total);
  if (!c.exps || col >= c.dz_ld) return;
  if constexpr (BF16) {
    const uint32_t w[2] = {__builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{x[0], x[1]}, halfx2)),
                           __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{x[2], x[3]}, halfx2))};
    __builtin_memcpy(__builtin_assume_aligned(static_cast<uint16_t*>(c.exps) + (int64_t)token * c.dz_ld + col, 8), w, 8);
  } else {
    __builtin_memcpy(__builtin_assume_aligned(static_cast<float*>(c.exps) + (int64_t)token * c.dz_ld + col, 16), x, 16);
  }
}

}  // namespace

void tsenor_dev::launch_few_logits(const LossCall& c, bool bf16, hipStream_t s) {
  const unsigned groups = (unsigned)((c.vocab + kFewWords - 1) / kFewWords);
  bf16 ? few_logits_kernel<true><<<groups, kWaves * kWave, 0, s>>>(c) : few_logits_kernel<false><<<groups, kWaves * kWave, 0, s>>>(c);
}
