// The products of the losses for heads whose rows begin anywhere.
#include "loss_tile.hpp"

namespace {

using namespace tsenor_dev;

constexpr int kTile = 128, kStep = 32, kThreads = 256;

template <bool BF16>
struct Format {
  using Element = float;
  static constexpr int kLd = kStep + 4;
};
template <>
struct Format<true> {
  using Element = uint16_t;
  static constexpr int kLd = kStep + 8;
};

// 128 x 32 of an operand into LDS, a row of it to a row of LDS.  ALONG: its rows lie along the sum in memory; otherwise they lie across.
template <bool BF16, bool ALONG>
__device__ __forceinline__ void fill(typename Format<BF16>::Element* to, const void* from, int64_t ld, int row0, int rows, int k0, int k_end) {
  using F = Format<BF16>;
  constexpr int kSize = BF16 ? 2 : 4;
  const char* base = static_cast<const char*>(from);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float x[8] = {};
    int r, k;
    if constexpr (ALONG) {
      r = (int)threadIdx.x / 4 + 64 * i, k = (int)threadIdx.x % 4 * 8;
      if (row0 + r < rows && k0 + k < k_end) load_row8<BF16>(base + (int64_t)(row0 + r) * ld * kSize, k0 + k, k_end, x);
    } else {
      k = (int)threadIdx.x / 16 + 16 * i, r = (int)threadIdx.x % 16 * 8;
      if (k0 + k < k_end && row0 + r < rows) load_row8<BF16>(base + (int64_t)(k0 + k) * ld * kSize, row0 + r, rows, x);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      typename F::Element* at = to + (ALONG ? r * F::kLd + k + e : (r + e) * F::kLd + k);
      if constexpr (BF16)
        *at = (uint16_t)(__float_as_uint(x[e]) >> 16);
      else
        *at = x[e];
    }
  }
}

template <bool BF16>
__device__ __forceinline__ floatx4 multiply(const typename Format<BF16>::Element* b, const typename Format<BF16>::Element* a, floatx4 sum) {
  if constexpr (BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(b), *reinterpret_cast<const bf16x8*>(a), sum, 0, 0, 0);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(b[u], a[u], sum, 0, 0, 0);
    return sum;
  }
}

template <bool BF16, int USE>
__global__ __launch_bounds__(kThreads) void any_kernel(LossCall c) {
  using F = Format<BF16>;
  __shared__ __align__(16) typename F::Element rows_a[kTile * F::kLd], rows_b[kTile * F::kLd];
  const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave, r = lane % 16, q = lane / 16;
  const int piece = rows_of(c);
  const int m = USE == kHead ? c.vocab : piece, n = USE == kLogits ? c.vocab : c.width;
  const int k_end = USE == kLogits ? c.width : USE == kStates ? c.vocab : piece;
  const int tiles_n = (n + kTile - 1) / kTile;
  const int m0 = (int)(blockIdx.x / (unsigned)tiles_n) * kTile, n0 = (int)(blockIdx.x % (unsigned)tiles_n) * kTile;
  if (m0 >= m || (USE == kHead && piece == 0 && c.first > 0 && !c.last)) return;
  floatx4 sum[4][4] = {};
  for (int k0 = 0; k0 < k_end; k0 += kStep) {
    if constexpr (USE == kLogits) {
      fill<BF16, true>(rows_a, c.states, c.states_ld, m0, m, k0, k_end);
      fill<BF16, true>(rows_b, c.weight, c.weight_ld, n0, n, k0, k_end);
    } else if constexpr (USE == kStates) {
      fill<BF16, true>(rows_a, c.dz, c.dz_ld, m0, m, k0, k_end);
      fill<BF16, false>(rows_b, c.weight, c.weight_ld, n0, n, k0, k_end);
    } else {
      fill<BF16, false>(rows_a, c.dz, c.dz_ld, m0, m, k0, k_end);
      fill<BF16, false>(rows_b, c.states, c.states_ld, n0, n, k0, k_end);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        sum[i][j] = multiply<BF16>(rows_b + (wave % 2 * 64 + i * 16 + r) * F::kLd + q * 8, rows_a + (wave / 2 * 64 + j * 16 + r) * F::kLd + q * 8, sum[i][j]);
    __syncthreads();
  }
  // a lane holds row 16 j + r of its wave's 64 of a, of tile i columns 4 q to 4 q + 3
  const int col0 = n0 + wave % 2 * 64 + q * 4, row0 = m0 + wave / 2 * 64 + r;
  if constexpr (USE == kLogits) {
    __shared__ float part[2][kTile];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[i][j][e] = col0 + 16 * i + e < n ? sum[i][j][e] : -__builtin_inff();
    float largest[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v = fmaxf(v, sum[i][j][e]);
      v = fmaxf(v, lane_xor<16>(v));
      v = fmaxf(v, lane_xor<32>(v));
      if (q == 0) part[wave % 2][wave / 2 * 64 + j * 16 + r] = v;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) largest[j] = fmaxf(part[0][wave / 2 * 64 + j * 16 + r], part[1][wave / 2 * 64 + j * 16 + r]) * c.scale - kExpBits;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float base = largest[j] == -__builtin_inff() ? 0.0f : largest[j];
      float v = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sum[i][j][e] = __builtin_amdgcn_exp2f(fmaf(sum[i][j][e], c.scale, -base));
          v += sum[i][j][e];
        }
      v += lane_xor<16>(v);
      v += lane_xor<32>(v);
      if (q == 0) part[wave % 2][wave / 2 * 64 + j * 16 + r] = v;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = row0 + 16 * j;
      if (row >= m) continue;
      if (q == 0 && wave % 2 == 0)
        c.sums[(int64_t)row * c.tiles + n0 / kTile] = make_float2(largest[j], part[0][row - m0] + part[1][row - m0]);
      if (!c.dz) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = col0 + 16 * i + e;
          if (col >= c.dz_ld) continue;
          if constexpr (BF16)
            static_cast<_Float16*>(c.dz)[(int64_t)row * c.dz_ld + col] = (_Float16)sum[i][j][e];
          else
            static_cast<float*>(c.dz)[(int64_t)row * c.dz_ld + col] = sum[i][j][e];
        }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = row0 + 16 * j;
      if (row >= m) continue;
      const int64_t at = (int64_t)(USE == kStates ? c.order[c.first + row] : row) * c.width;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = col0 + 16 * i + e;
          if (col >= n) continue;
          float v = sum[i][j][e] * c.largest_weight[1];
          if constexpr (USE == kHead) {
            float* const all = BF16 ? c.dweight_sum : static_cast<float*>(c.dweight);
            if (c.first > 0) v += all[at + col];
            if (!BF16 || !c.last) {
              all[at + col] = v;
              continue;
            }
          }
          void* const out = USE == kStates ? c.dh : c.dweight;
          if constexpr (BF16)
            static_cast<uint16_t*>(out)[at + col] = (uint16_t)pack_bf16(v, 0.0f);
          else
            static_cast<float*>(out)[at + col] = v;
        }
    }
  }
}

inline unsigned tiles_of(int m, int n) { return (unsigned)((m + kTile - 1) / kTile) * (unsigned)((n + kTile - 1) / kTile); }

}  // namespace

void tsenor_dev::launch_any_logits(const LossCall& c, bool bf16, hipStream_t s) {
  const unsigned tiles = tiles_of(c.rows, c.vocab);
  bf16 ? any_kernel<true, kLogits><<<tiles, kThreads, 0, s>>>(c) : any_kernel<false, kLogits><<<tiles, kThreads, 0, s>>>(c);
}
void tsenor_dev::launch_any_dh(const LossCall& c, bool bf16, hipStream_t s) {
  const unsigned tiles = tiles_of(c.rows, c.width);
  bf16 ? any_kernel<true, kStates><<<tiles, kThreads, 0, s>>>(c) : any_kernel<false, kStates><<<tiles, kThreads, 0, s>>>(c);
}
void tsenor_dev::launch_any_dweight(const LossCall& c, bool bf16, hipStream_t s) {
  const unsigned tiles = tiles_of(c.vocab, c.width);
  bf16 ? any_kernel<true, kHead><<<tiles, kThreads, 0, s>>>(c) : any_kernel<false, kHead><<<tiles, kThreads, 0, s>>>(c);
}
