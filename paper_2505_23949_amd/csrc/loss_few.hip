// Logits and dh of up to 16 tokens: the head is read once for each, straight into registers, whatever its rows begin at.
//
// Logits: a workgroup of eight waves takes 16 words.  The waves share the width, 32 columns at a time, and their sums meet in LDS.  A lane holds
// columns 8 (l / 16) to 8 (l / 16) + 7 of row l % 16, of a word and of a token; the words are the first operand of the matrix instruction,
// so that it ends up with four neighbouring words of a token.  Single precision takes the fp32 instruction: 16 rows are too few for its
// rate to matter (8 operations a byte).
// Of several entries to a token, all threads look for those among the workgroup's words, in logits that LDS holds.
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
  __shared__ __align__(16) float logits[kFewTokens][kFewWords];
  constexpr int kSize = BF16 ? 2 : 4;
  const int lane = (int)threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int rows = rows_of(c), first = (int)blockIdx.x * kFewWords;
  if (rows == 0) return;
  const int row = min(lane % 16, rows - 1), word = min(first + lane % 16, c.vocab - 1), at = lane / 16 * 8;  // (what lies past the last is not written)
  const char* const h = static_cast<const char*>(c.h) + (int64_t)(c.count ? c.order[c.first + row] : c.first + row) * c.h_ld * kSize;
  const char* const w = static_cast<const char*>(c.weight) + (int64_t)word * c.weight_ld * kSize;
  const int target = wave == 0 && c.k == 1 ? word_of(c, row) : -1;
  const int pairs = c.k > 1 ? rows * c.k : 0;
  const auto id_of = [&](int i) {
    const int of = i / c.k;
    return c.ids[(int64_t)(c.count ? c.order[c.first + of] : c.first + of) * c.ids_ld + (i - of * c.k)];
  };
  int64_t id = (int)threadIdx.x < pairs ? id_of((int)threadIdx.x) : -1;  // (asked for before the rows)
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
  if (wave == 0) {
#pragma unroll
    for (int k = 1; k < kWaves; ++k) sum += parts[k][lane];
    if (pairs) *reinterpret_cast<floatx4*>(&logits[lane % 16][lane / 16 * 4]) = sum;
  }
  if (pairs) {
    if (pairs > kWave) __syncthreads();  // (up to there only the first wave has any)
    for (int i = (int)threadIdx.x; i < pairs; i += kWaves * kWave) {
      if (i != (int)threadIdx.x) id = id_of(i);
      if (id >= first && id < min(first + kFewWords, c.vocab)) c.dots[i] = logits[i / c.k][(int)id - first];
    }
  }
  if (wave != 0) return;

  // token lane % 16, words first + 4 (lane / 16) to + 3
  const int col = first + lane / 16 * 4, token = lane % 16;
  float largest = -__builtin_inff();
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (col + e >= c.vocab) sum[e] = -__builtin_inff();
    largest = fmaxf(largest, sum[e]);
  }
  largest = fmaxf(largest, lane_xor<16>(largest));
  largest = fmaxf(largest, lane_xor<32>(largest));
  const float base = largest == -__builtin_inff() ? 0.0f : largest;
  float x[4], total = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = exp_from(sum[e], base, c.scale, exp_bits(BF16, false));
    if (col + e != target) total += x[e];
    else if (token < rows) c.dots[token] = sum[e];
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

// dh = dz W by the fp32 matrix instruction, 16 tokens x 4 words x 16 columns.  A wave takes 4 words and 128 columns at a time: 8 columns of a word to
// a lane, straight from memory, element e of all lanes being the second operand of the e-th of 8 instructions, so that a lane ends up with 8
// neighbouring columns of 4 tokens.  dz of 512 words at a time stands in LDS in fp32 (of single precision the sum of its three planes, which
// is exact).  The four waves of a workgroup take words in turn, and their sums meet in LDS; workgroups that share a block's words leave
// theirs to join_few_kernel.  Sums of all have a fixed order.
// Memory bounds it: 1 x 116621 x 5083 in fp32 566 us, 4.2 TB/s (a copy in planes 1072 and tiles 948), 16 x 60001 x 300 25 (30 and 38).  By the vector
// units, 16 tokens of 8 columns in a lane's registers, the latter took 101.
constexpr int kThreads = 256, kAhead = 4;
__device__ __forceinline__ float* part_of(const LossCall& c, int split, int row) {
  return reinterpret_cast<float*>(c.parts) + ((int64_t)split * c.tokens + row) * c.width;
}
template <bool BF16>
__device__ __forceinline__ void store_dh(const LossCall& c, int row, int col, float sum) {
  const int64_t at = (int64_t)c.order[c.first + row] * c.width + col;
  sum *= c.largest_weight[1];
  if constexpr (BF16)
    static_cast<uint16_t*>(c.dh)[at] = (uint16_t)pack_bf16(sum, 0.0f);
  else
    static_cast<float*>(c.dh)[at] = sum;
}

// WHOLE: all of the block's columns are there
template <bool BF16, bool WHOLE>
__device__ __forceinline__ void few_dh(const LossCall& c, float* lds, int rows, int first_col, int first, int last, floatx4 (&sum)[8]) {
  const int t = (int)threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave), q = lane / 16, col = first_col + lane % 16 * 8;
  for (int begin = first; begin < last; begin += kFewDhWords) {
    const int n = min(last - begin, kFewDhWords);
    __syncthreads();
    const int token = t % 16;
    for (int k = t / 16 * 8; k < n; k += kThreads / 16 * 8) {  // (dz has whole lines of 64 words, zeros behind the last)
      float x[8] = {};
      if (token < rows) {
        const uint16_t* const dz = static_cast<const uint16_t*>(c.dz) + (int64_t)token * c.dz_ld * (BF16 ? 1 : 3) + begin + k;
        load_row8<true>(dz, 0, 8, x);
        if constexpr (!BF16) {
          float mid[8], low[8];
          load_row8<true>(dz + c.dz_ld, 0, 8, mid);
          load_row8<true>(dz + 2 * c.dz_ld, 0, 8, low);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] += mid[e] + low[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) lds[(k + e) * 16 + token] = x[e];
    }
    __syncthreads();
    const auto load = [&](int k) {
      const char* const row = static_cast<const char*>(c.weight) + (int64_t)(begin + k + q) * c.weight_ld * (BF16 ? 2 : 4);
      if constexpr (WHOLE)
        return load_whole<BF16>(row, col);
      else
        return load_raw8<BF16>(row, col, c.width);
    };
    const auto add = [&](int k, const Raw8<BF16>& raw) {
      float x[8];
      if constexpr (WHOLE)
        widen8<BF16>(raw, x);
      else
        widen8<BF16>(raw, col, c.width, x);
      const float w = lds[(k + q) * 16 + lane % 16];
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(w, x[e], sum[e], 0, 0, 0);
    };
    constexpr int kStep = kThreads / kWave * 4;
    int k = wave * 4;
    for (; k + (kAhead - 1) * kStep + 4 <= n; k += kAhead * kStep) {
      Raw8<BF16> raw[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) raw[u] = load(k + u * kStep);
      TSENOR_IN_ORDER();  // (all of them are asked for before the first is waited for)
#pragma unroll
      for (int u = 0; u < kAhead; ++u) add(k + u * kStep, raw[u]);
    }
    for (; k < n; k += kStep) {  // (words behind the last are zeros on both sides: dz in LDS may end before them)
      Raw8<BF16> raw = {};
      if (k + q < n) raw = load(k);
      add(k, raw);
    }
  }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void few_dh_kernel(LossCall c, int words) {
  static_assert(kFewDhWords * 16 >= kThreads / kWave * 16 * kFewDhColumns);
  __shared__ __align__(16) float lds[kFewDhWords * 16];  // dz of a word and token; then sums of a wave, token and column
  const int rows = rows_of(c), first_col = (int)blockIdx.x * kFewDhColumns, first = (int)blockIdx.y * words, last = min(first + words, c.vocab);
  if (rows == 0) return;
  floatx4 sum[8] = {};
  if (first_col + kFewDhColumns <= c.width)
    few_dh<BF16, true>(c, lds, rows, first_col, first, last, sum);
  else
    few_dh<BF16, false>(c, lds, rows, first_col, first, last, sum);
  const int t = (int)threadIdx.x, lane = t % kWave, wave = t / kWave;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int half = 0; half < 2; ++half)
      *reinterpret_cast<floatx4*>(lds + (wave * 16 + lane / 16 * 4 + i) * kFewDhColumns + lane % 16 * 8 + 4 * half) =
          floatx4{sum[4 * half][i], sum[4 * half + 1][i], sum[4 * half + 2][i], sum[4 * half + 3][i]};
  __syncthreads();
  for (int at = t; at < rows * kFewDhColumns; at += kThreads) {
    const int row = at / kFewDhColumns, col = first_col + at % kFewDhColumns;
    if (col >= c.width) continue;
    float all = lds[at];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) all += lds[w * 16 * kFewDhColumns + at];
    if (gridDim.y > 1)
      part_of(c, (int)blockIdx.y, row)[col] = all;
    else
      store_dh<BF16>(c, row, col, all);
  }
}

// a wave to every fourth of the parts of 64 columns
template <bool BF16>
__global__ __launch_bounds__(kThreads) void join_few_kernel(LossCall c, int splits) {
  __shared__ float sums[kThreads / kWave][kWave];
  const int row = (int)blockIdx.y, lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave, col = (int)blockIdx.x * kWave + lane;
  if (row >= rows_of(c)) return;
  float sum = 0.0f;
  if (col < c.width) {
    constexpr int kWaves = kThreads / kWave;
    int k = wave;
    for (; k + 7 * kWaves < splits; k += 8 * kWaves) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = part_of(c, k + u * kWaves, row)[col];
#pragma unroll
      for (int u = 0; u < 8; ++u) sum += x[u];
    }
    for (; k < splits; k += kWaves) sum += part_of(c, k, row)[col];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || col >= c.width) return;
#pragma unroll
  for (int w = 1; w < kThreads / kWave; ++w) sum += sums[w][lane];
  store_dh<BF16>(c, row, col, sum);
}

template <bool BF16>
void launch_dh_of_few(const LossCall& c, const FewDhPlan& plan, hipStream_t s) {
  few_dh_kernel<BF16><<<dim3((unsigned)plan.blocks, (unsigned)plan.splits), kThreads, 0, s>>>(c, plan.words);
  if (plan.splits > 1)
    join_few_kernel<BF16><<<dim3((unsigned)((c.width + kWave - 1) / kWave), (unsigned)c.rows), kThreads, 0, s>>>(c, plan.splits);
}

}  // namespace

void tsenor_dev::launch_few_dh(const LossCall& c, const FewDhPlan& plan, bool bf16, hipStream_t s) {
  bf16 ? launch_dh_of_few<true>(c, plan, s) : launch_dh_of_few<false>(c, plan, s);
}
void tsenor_dev::launch_few_logits(const LossCall& c, bool bf16, hipStream_t s) {
  const unsigned groups = (unsigned)((c.vocab + kFewWords - 1) / kFewWords);
  bf16 ? few_logits_kernel<true><<<groups, kWaves * kWave, 0, s>>>(c) : few_logits_kernel<false><<<groups, kWaves * kWave, 0, s>>>(c);
}
