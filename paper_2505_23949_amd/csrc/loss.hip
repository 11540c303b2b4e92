// tsenor_cross_entropy, tsenor_distill: host side, and the kernels that go through tokens (the products: loss_tile.hpp).
#include <algorithm>
#include <type_traits>

#include "loss.hpp"

namespace {

using namespace tsenor_dev;

constexpr int kThreads = 256;
constexpr int kMaxEntries = TSENOR_LOSS_MAX_ENTRIES;

__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, lane_xor<1>(v)), v = fmaxf(v, lane_xor<2>(v)), v = fmaxf(v, lane_xor<7>(v));
  v = fmaxf(v, lane_xor<15>(v)), v = fmaxf(v, lane_xor<16>(v));
  return fmaxf(v, lane_xor<32>(v));
}

// logit of an entry by the teacher; -infinity where it takes no part
__device__ __forceinline__ float teacher_of(const LossCall& c, int64_t token, int i) {
  const int64_t id = c.ids[token * c.ids_ld + i];
  if (id < 0 || id >= c.vocab) return -__builtin_inff();
  const int64_t at = token * c.teacher_ld + i;
  return c.teacher_bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(c.teacher)[at] << 16) : static_cast<const float*>(c.teacher)[at];
}

// two values rounded to bf16, but the largest numbers of single precision, which would round up to infinity, to the largest of bf16
__device__ __forceinline__ uint32_t plane_of(float a, float b) {
  const auto near = [](float x) { return fabsf(x) < __builtin_inff() ? __builtin_amdgcn_fmed3f(x, -0x1.FEp127f, 0x1.FEp127f) : x; };
  return pack_bf16(near(a), near(b));
}
// what is left of x (infinities and NaN have nothing left)
__device__ __forceinline__ float remainder_of(float x, uint32_t rounded) {
  return (rounded & kInfinityBits) == kInfinityBits ? 0.0f : x - __uint_as_float(rounded);
}
// 8 elements of a row of an operand as the products read it: bf16, or three planes whose sum they are
template <bool BF16>
__device__ __forceinline__ void store_planes(void* row, int ld, int c, const float (&x)[8]) {
  if constexpr (BF16) {
    store_row8<true>(row, c, ld, x);
  } else {
    float rest[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) rest[k] = x[k];
#pragma unroll
    for (int plane = 0; plane < 3; ++plane) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[k] = plane == 0 ? plane_of(rest[2 * k], rest[2 * k + 1]) : pack_bf16(rest[2 * k], rest[2 * k + 1]);
        rest[2 * k] = remainder_of(rest[2 * k], w[k] << 16), rest[2 * k + 1] = remainder_of(rest[2 * k + 1], w[k] & 0xFFFF0000u);
      }
      __builtin_memcpy(static_cast<uint16_t*>(row) + plane * ld + c, w, 16);
    }
  }
}

// which tokens have an entry that takes part: a wave to a token
__global__ __launch_bounds__(kThreads) void counts_kernel(LossCall c) {
  const int token = (int)blockIdx.x * (kThreads / kWave) + (int)threadIdx.x / kWave, lane = (int)threadIdx.x % kWave;
  if (token >= c.tokens) return;
  bool any = false;
  for (int i = lane; i < c.k; i += kWave) any |= teacher_of(c, token, i) != -__builtin_inff();  // (NaN does)
  any = __any(any);
  if (lane == 0) c.counts[token] = any;
}

// one workgroup: a thread takes 8 tokens at a time
constexpr int kOrderThreads = 1024;
__global__ __launch_bounds__(kOrderThreads) void order_kernel(LossCall c) {
  __shared__ int before[kOrderThreads / kWave];
  __shared__ float weights[kOrderThreads / kWave];
  float weight = 0.0f;
  const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave;
  int done = 0;
  for (int t0 = 0; t0 < c.tokens; t0 += kOrderThreads * 8) {
    const int begin = t0 + (int)threadIdx.x * 8;
    unsigned bits = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = begin + e;
      if (t < c.tokens && (c.teacher ? c.counts[t] != 0 : c.ids[t] >= 0 && c.ids[t] < c.vocab)) {
        bits |= 1u << e;
        const float w = c.dloss ? fabsf(c.dloss[t]) : 1.0f;
        if (w < __builtin_inff()) weight = fmaxf(weight, w);
      }
    }
    int upto = __popc(bits);  // of the wave's threads up to this one
#pragma unroll
    for (int step = 1; step < kWave; step *= 2) {
      const int v = __shfl_up(upto, step);
      if (lane >= step) upto += v;
    }
    __syncthreads();
    if (lane == kWave - 1) before[wave] = upto;
    __syncthreads();
    int at = done + upto - __popc(bits), all = 0;
#pragma unroll
    for (int w = 0; w < kOrderThreads / kWave; ++w) {
      if (w < wave) at += before[w];
      all += before[w];
    }
    for (int e = 0; e < 8 && begin + e < c.tokens; ++e) {
      if (bits >> e & 1)
        c.order[at++] = begin + e;
      else
        c.order[c.tokens - 1 - (begin + e - at)] = begin + e;  // (as many as are not counted stand before it)
    }
    done += all;
  }
  weight = wave_max(weight);
  if (lane == 0) weights[wave] = weight;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kOrderThreads / kWave; ++w) weight = fmaxf(weight, weights[w]);
    *c.count = done, c.largest_weight[0] = weight, c.largest_weight[1] = weight * c.inverse_temperature;
  }
}

// The token that a row is of, by a workgroup on its own: the row-th of those that count, or, behind them, of those that do not.  A thread
// looks at 8 tokens.  `count` becomes how many count, `weight` the largest finite |dloss| of the thread's.
constexpr int kAloneTokens = 1024;
static_assert(kAloneTokens <= kThreads * 8);
__device__ __forceinline__ int token_alone(const LossCall& c, int row, int& count, float& weight) {
  __shared__ int before[kThreads / kWave], found;
  const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave, begin = (int)threadIdx.x * 8;
  unsigned bits = 0;
  weight = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int t = begin + e;
    if (t < c.tokens && (c.teacher ? c.counts[t] != 0 : c.ids[t] >= 0 && c.ids[t] < c.vocab)) {
      bits |= 1u << e;
      const float w = c.dloss && row == 0 ? fabsf(c.dloss[t]) : 1.0f;
      if (w < __builtin_inff()) weight = fmaxf(weight, w);
    }
  }
  int upto = __popc(bits);
#pragma unroll
  for (int step = 1; step < kWave; step *= 2) {
    const int v = __shfl_up(upto, step);
    if (lane >= step) upto += v;
  }
  if (lane == kWave - 1) before[wave] = upto;
  __syncthreads();
  int at = upto - __popc(bits);
  count = 0;
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) {
    if (w < wave) at += before[w];
    count += before[w];
  }
  const bool counts = row < count;
  int rank = counts ? at : begin - at;  // of the thread's first token of the kind
  for (int e = 0; e < 8 && begin + e < c.tokens; ++e)
    if ((bits >> e & 1) == counts && rank++ == (counts ? row : row - count)) found = begin + e;
  __syncthreads();
  return found;
}

// A workgroup to a row of the piece's states, and to one more for each that its last tile has.  ALONE: nothing has put the tokens in order
// before (up to kAloneTokens of them, in one piece: a launch less, 5 us).
template <bool BF16, bool ALONE>
__global__ __launch_bounds__(kThreads) void gather_kernel(LossCall c) {
  constexpr int kSize = BF16 ? 2 : 4;
  const int row = (int)blockIdx.x;
  int rows, token = 0;
  if constexpr (ALONE) {
    float weight;
    if (row < c.tokens || row == 0) token = token_alone(c, row, rows, weight);
    else rows = 0;
    if (row < c.tokens && threadIdx.x == 0) c.order[row] = token;
    if (row == 0) {
      __shared__ float weights[kThreads / kWave];
      weight = wave_max(weight);
      if (threadIdx.x % kWave == 0) weights[threadIdx.x / kWave] = weight;
      __syncthreads();
      weight = fmaxf(fmaxf(weights[0], weights[1]), fmaxf(weights[2], weights[3]));
      if (threadIdx.x == 0) *c.count = rows, c.largest_weight[0] = weight, c.largest_weight[1] = weight * c.inverse_temperature;
    }
  } else {
    rows = rows_of(c);
    if (row < c.rows) token = c.order[c.first + row];
  }
  uint16_t* const state = static_cast<uint16_t*>(c.states) + (int64_t)row * c.states_ld * (BF16 ? 1 : 3);
  float x[8] = {};
  if (row >= rows) {
    for (int k = (int)threadIdx.x * 8; k < c.states_ld; k += kThreads * 8) store_planes<BF16>(state, c.states_ld, k, x);
    if (row >= c.rows) return;
    if (threadIdx.x == 0) {
      c.loss[token] = 0.0f;
      if (c.lse) c.lse[token] = 0.0f;
    }
    if (c.dh)
      for (int k = (int)threadIdx.x * 8; k < c.width; k += kThreads * 8)
        store_row8<BF16>(static_cast<char*>(c.dh) + (int64_t)token * c.width * kSize, k, c.width, x);
    return;
  }
  const char* const h = static_cast<const char*>(c.h) + (int64_t)token * c.h_ld * kSize;
  for (int k = (int)threadIdx.x * 8; k < c.states_ld; k += kThreads * 8) {
    load_row8<BF16>(h, k, c.width, x);
    store_planes<BF16>(state, c.states_ld, k, x);
  }
  // a number that its exponentials can be counted from: the largest logit of up to four of its entries
  if (c.refs) {
    __shared__ float most[kThreads / kWave];
    const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave;
    float z = -__builtin_inff();
    for (int i = wave; i < c.k; i += kThreads / kWave) {
      const int64_t id = c.ids[(int64_t)token * c.ids_ld + i];
      if (id < 0 || id >= c.vocab) continue;
      const char* const w = static_cast<const char*>(c.weight) + id * c.weight_ld * kSize;
      float s = 0.0f;
      for (int k = lane * 8; k < c.width; k += kWave * 8) {
        float y[8];
        load_row8<BF16>(h, k, c.width, x);
        load_row8<BF16>(w, k, c.width, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
      }
      z = wave_sum(s);
      break;
    }
    if (lane == 0) most[wave] = z;
    __syncthreads();
    if (threadIdx.x == 0) {
      const float ref = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])), sum = most[0] + most[1] + most[2] + most[3];
      c.refs[row] = sum == sum ? ref : sum;  // (NaN if there is one: its row is NaN whatever it is counted from, and needs no other way)
      if (row == 0) *c.again = 0;
    }
  }
  if (c.words && threadIdx.x == 0) c.words[row] = (int)c.ids[token * c.ids_ld];  // (it counts: it has a word of the vocabulary)
  if (!c.sorted) return;

  // its entries by word, and where those of each part of a tile begin
  static_assert(kThreads == kMaxEntries);
  __shared__ uint32_t keys[kMaxEntries], sorted[kMaxEntries];
  const int i = (int)threadIdx.x;
  if (i < c.k) {
    const int64_t id = c.ids[(int64_t)token * c.ids_ld + i];
    keys[i] = id < 0 || id >= c.vocab ? UINT32_MAX - 255 + i : (uint32_t)id << 8 | i;
  }
  __syncthreads();
  if (i < c.k) {
    int rank = 0;
    for (int j = 0; j < c.k; ++j) rank += keys[j] < keys[i];
    sorted[rank] = keys[i];
    c.sorted[(int64_t)row * c.k + rank] = keys[i];
  }
  __syncthreads();
  for (int t = i; t <= c.tiles; t += kThreads) {
    const uint32_t first = (uint32_t)min(t * c.tile_n, c.vocab) << 8;
    int lo = 0, hi = c.k;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (sorted[mid] < first)
        lo = mid + 1;
      else
        hi = mid;
    }
    c.begins[(int64_t)row * (c.tiles + 1) + t] = (uint16_t)lo;
  }
}

// the head with rows of whole lines: a workgroup to a row, or to as many short ones as have 8 elements for each thread
template <bool BF16>
__global__ __launch_bounds__(kThreads) void head_kernel(LossCall c, uint16_t* head, int rows) {
  const int threads = kThreads / rows, of_group = (int)threadIdx.x / threads, row = (int)blockIdx.x * rows + of_group;
  if (of_group >= rows || row >= c.vocab) return;
  const char* const from = static_cast<const char*>(c.weight) + (int64_t)row * c.weight_ld * (BF16 ? 2 : 4);
  uint16_t* const to = head + (int64_t)row * c.head_ld;
  for (int k = (int)threadIdx.x % threads * 8; k < c.states_ld; k += threads * 8) {
    float x[8];
    load_row8<BF16>(from, k, c.width, x);
    store_planes<BF16>(to, c.states_ld, k, x);
  }
}

// A workgroup to a token: lse, loss; exponentials into dz.
// Exponents here are counted from `largest`, the teacher's from `top` (before the temperature, which may take either beyond single precision).
template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void rows_kernel(LossCall c) {
  constexpr int kSize = BF16 ? 2 : 4, kWaves = THREADS / kWave, kMine = 2;
  __shared__ float part[2][kWaves], dots[kMaxEntries], teacher[kMaxEntries], q[kMaxEntries], dentry[kMaxEntries];
  __shared__ int words[kMaxEntries];
  const int row = (int)blockIdx.x, lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave;
  if (row >= rows_of(c)) return;
  const int token = c.count ? c.order[c.first + row] : c.first + row;
  const float2* const sums = c.sums + (int64_t)row * c.tiles;
  const bool ready = c.refs && !*c.again;  // the exponentials are dz but for 1 / total and the weight
  const float bits = exp_bits(BF16, ready), one = __builtin_amdgcn_exp2f(-bits);

  // what has to be read, asked for at once
  float2 mine[kMine];
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    const int t = u * THREADS + (int)threadIdx.x;
    mine[u] = t < c.tiles ? sums[t] : make_float2(-__builtin_inff(), 0.0f);
  }
  float top = -__builtin_inff();
  bool any = false;
  for (int i = (int)threadIdx.x; i < c.k; i += THREADS) {
    const int64_t id = c.ids[(int64_t)token * c.ids_ld + i];
    const bool valid = id >= 0 && id < c.vocab;
    const float u = c.teacher ? teacher_of(c, token, i) : valid ? 0.0f : -__builtin_inff();
    words[i] = valid ? (int)id : -1, teacher[i] = u;
    dots[i] = valid ? c.dots[(int64_t)row * c.k + i] : 0.0f;
    top = fmaxf(top, u), any |= u != -__builtin_inff();  // (NaN takes part)
  }
  if (!c.count && !__syncthreads_or(any)) {  // nothing has left it out before
    if (threadIdx.x == 0) {
      c.loss[token] = 0.0f;
      if (c.lse) c.lse[token] = 0.0f;
    }
    return;
  }
  float largest = -__builtin_inff();
#pragma unroll
  for (int u = 0; u < kMine; ++u) largest = fmaxf(largest, mine[u].x);
  for (int t = kMine * THREADS + (int)threadIdx.x; t < c.tiles; t += THREADS) largest = fmaxf(largest, sums[t].x);
  largest = wave_max(largest), top = wave_max(top);
  if (lane == 0) part[0][wave] = largest, part[1][wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) largest = fmaxf(largest, part[0][w]), top = fmaxf(top, part[1][w]);

  float total = 0.0f, all = 0.0f;
#pragma unroll
  for (int u = 0; u < kMine; ++u)
    if (u * THREADS + (int)threadIdx.x < c.tiles) total += mine[u].y * exp_from(mine[u].x, largest, c.scale, 0.0f);
  for (int t = kMine * THREADS + (int)threadIdx.x; t < c.tiles; t += THREADS) total += sums[t].y * exp_from(sums[t].x, largest, c.scale, 0.0f);
  for (int i = (int)threadIdx.x; i < c.k; i += THREADS) all += expf((teacher[i] - top) * c.inverse_temperature);
  total = wave_sum(total), all = wave_sum(all);
  __syncthreads();
  if (lane == 0) part[0][wave] = total, part[1][wave] = all;
  __syncthreads();
  total = all = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) total += part[0][w], all += part[1][w];

  const float rest = total;  // (of several entries: of all words)
  if (c.k == 1) total += exp_from(dots[0], largest, c.scale, bits);
  const float log_total = logf(total * one), log_all = logf(all);
  const float unit = c.dz ? c.largest_weight[0] : 1.0f, weight = c.dloss ? (unit > 0.0f ? c.dloss[token] / unit : c.dloss[token]) : 1.0f;
  float loss = 0.0f;
  for (int i = (int)threadIdx.x; i < c.k; i += THREADS) {
    const float s = dots[i], u = (teacher[i] - top) * c.inverse_temperature, p = c.teacher ? expf(u) / all : 1.0f, own = exp_from(s, largest, c.scale, bits);
    const float off = fmaf(largest - s, c.inverse_temperature, log_total);  // lse - z
    q[i] = p, dentry[i] = own / total;
    if (c.k == 1)
      loss = p * (own > rest ? log1pf(rest / own) : off);  // (p is 1, or a teacher's NaN)
    else if (p != 0.0f)
      loss = fmaf(p, u - log_all + off, loss);
  }
  loss = wave_sum(loss);
  __syncthreads();
  if (lane == 0) part[0][wave] = loss;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kWaves; ++w) loss += part[0][w];
    c.loss[token] = loss;
    if (c.lse) c.lse[token] = fmaf(largest, c.inverse_temperature, log_total);
  }
  if (!c.dz) return;
  if (c.row_scale && threadIdx.x == 0) c.row_scale[row] = ready ? make_float2(1.0f / total, weight) : make_float2(1.0f, 1.0f);
  // (the same word twice: both write what belongs to both)
  for (int i = (int)threadIdx.x; i < c.k; i += THREADS) {
    float p = 0.0f;
    for (int j = 0; j < c.k; ++j)
      if (words[j] == words[i]) p += q[j];
    dentry[i] = (ready ? total : weight) * (c.k == 1 ? -(rest / total) * p : dentry[i] - p);
  }
  const float share = weight / total;
  uint16_t* const dz = static_cast<uint16_t*>(c.dz) + (int64_t)row * c.dz_ld * (BF16 ? 1 : 3);
  const char* const exps = static_cast<const char*>(c.exps) + (int64_t)row * c.dz_ld * kSize;
  constexpr int kAtOnce = 4;  // that a thread has asked for at a time
  for (int k0 = (int)threadIdx.x * 8; k0 < c.dz_ld && !ready; k0 += kAtOnce * THREADS * 8) {
    typedef typename std::conditional<BF16, _Float16, float>::type Exp;
    Exp y[kAtOnce][8];
    float scale[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int k = k0 + u * THREADS * 8;
      if (k >= c.dz_ld) continue;
      __builtin_memcpy(y[u], exps + k * kSize, 8 * kSize);
      scale[u] = sums[min(k / c.tile_n, c.tiles - 1)].x;
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int k = k0 + u * THREADS * 8;
      if (k >= c.dz_ld) continue;
      const float factor = share * exp_from(scale[u], largest, c.scale, 0.0f);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = k + e < c.vocab ? (float)y[u][e] * factor : 0.0f;
      store_planes<BF16>(dz, c.dz_ld, k, x);
    }
  }
  __syncthreads();
  for (int i = (int)threadIdx.x; i < c.k; i += THREADS) {
    if (words[i] < 0) continue;
    float rest = dentry[i];
    for (int plane = 0; plane < (BF16 ? 1 : 3); ++plane) {
      const uint32_t w = pack_bf16(rest, 0.0f);
      dz[plane * c.dz_ld + words[i]] = (uint16_t)w;
      rest = remainder_of(rest, w << 16);
    }
  }
}

template <bool BF16>
void launch_rows(const LossCall& c, int threads, hipStream_t s) {
  const unsigned rows = (unsigned)c.rows;
  if (threads == 1024)
    rows_kernel<BF16, 1024><<<rows, 1024, 0, s>>>(c);
  else if (threads == kWave)
    rows_kernel<BF16, kWave><<<rows, kWave, 0, s>>>(c);
  else
    rows_kernel<BF16, kThreads><<<rows, kThreads, 0, s>>>(c);
}
void launch_rows(const LossCall& c, int threads, bool bf16, hipStream_t s) { bf16 ? launch_rows<true>(c, threads, s) : launch_rows<false>(c, threads, s); }

// no token counts, or there is none: zeros
template <bool BF16>
__global__ __launch_bounds__(kThreads) void zero_kernel(void* out, int64_t count) {
  for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < count; k += (int64_t)gridDim.x * kThreads) {
    if constexpr (BF16)
      static_cast<uint16_t*>(out)[k] = 0;
    else
      static_cast<uint32_t*>(out)[k] = 0;
  }
}
void launch_zero(void* out, int64_t count, bool bf16, hipStream_t s) {
  const unsigned groups = (unsigned)std::min<int64_t>((count + kThreads - 1) / kThreads, 65536);
  if (count == 0) return;
  bf16 ? zero_kernel<true><<<groups, kThreads, 0, s>>>(out, count) : zero_kernel<false><<<groups, kThreads, 0, s>>>(out, count);
}

// ---- host ------------------------------------------------------------------------------------------------------------------
constexpr int64_t kMaxTokens = (int64_t)1 << 24, kMaxVocab = (int64_t)1 << 21, kMaxWidth = (int64_t)1 << 16;
constexpr int64_t kMaxTileLd = (int64_t)1 << 21;   // (the tile kernels' offsets within a tile have 31 bits)
constexpr double kLog2e = 1.4426950408889634;

int check(const tsenor_head& p) {
  if (p.tokens < 0 || p.tokens > kMaxTokens || p.vocab < 0 || p.vocab > kMaxVocab || p.width < 0 || p.width > kMaxWidth) return TSENOR_ERR_SHAPE;
  if (!known(p.dtype)) return TSENOR_ERR_UNSUPPORTED;
  if (p.tokens && (!p.loss_out || (p.width && !p.h))) return TSENOR_ERR_NULL;
  if (p.vocab && p.width && !p.weight) return TSENOR_ERR_NULL;
  if (!ld_ok(p.h_ld, p.tokens, p.width) || !ld_ok(p.weight_ld, p.vocab, p.width)) return TSENOR_ERR_SHAPE;
  for (const void* m : {p.h, p.weight, (const void*)p.dh_out, (const void*)p.dweight_out})
    if (!aligned_to(m, size_of(p.dtype))) return TSENOR_ERR_ALIGN;
  for (const float* v : {p.dloss, (const float*)p.loss_out, (const float*)p.lse_out})
    if (!aligned_to(v, sizeof(float))) return TSENOR_ERR_ALIGN;
  return TSENOR_OK;
}
int check(const tsenor_cross_entropy_problem* p) {
  if (!p) return TSENOR_ERR_NULL;
  const int rc = check(p->head);
  if (rc != TSENOR_OK) return rc;
  if (p->head.tokens && !p->targets) return TSENOR_ERR_NULL;
  return aligned_to(p->targets, sizeof(int64_t)) ? TSENOR_OK : TSENOR_ERR_ALIGN;
}
int check(const tsenor_distill_problem* p) {
  if (!p) return TSENOR_ERR_NULL;
  const int rc = check(p->head);
  if (rc != TSENOR_OK) return rc;
  if (p->k < 0 || p->k > kMaxEntries || !ld_ok(p->ids_ld, p->head.tokens, p->k) || !ld_ok(p->logits_ld, p->head.tokens, p->k)) return TSENOR_ERR_SHAPE;
  if (!known(p->logits_dtype)) return TSENOR_ERR_UNSUPPORTED;
  if (!(p->temperature >= 0x1p-20 && p->temperature <= 0x1p20)) return TSENOR_ERR_PARAM;
  if (p->head.tokens && p->k && (!p->ids || !p->logits)) return TSENOR_ERR_NULL;
  return aligned_to(p->ids, sizeof(int64_t)) && aligned_to(p->logits, size_of(p->logits_dtype)) ? TSENOR_OK : TSENOR_ERR_ALIGN;
}

inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// describes a call to the kernels; the workspace begins at `workspace` (which may be NULL to ask for its size alone)
size_t lay_out(const tsenor_head& p, char* workspace, LossCall& c, LossPlan& plan) {
  const bool bf16 = p.dtype == TSENOR_BF16, gradients = p.dh_out || p.dweight_out;
  const int64_t size = bf16 ? 2 : 4, planes = bf16 ? 1 : 3;
  // (a row's last line goes on into the next row, but not into what lies between the rows of a wider matrix)
  const bool in_place = bf16 && p.width && (p.width % 64 == 0 || (p.width % 8 == 0 && p.weight_ld == p.width)) && p.weight_ld % 8 == 0 &&
                        p.weight_ld <= kMaxTileLd && aligned_to(p.weight, 16);
  const bool states_too = p.width % 64 == 0 && p.h_ld % 8 == 0 && p.h_ld <= kMaxTileLd && aligned_to(p.h, 16);
  plan = loss_plan({p.tokens, p.vocab, p.width, bf16, p.dh_out != nullptr, p.dweight_out != nullptr, c.k, c.teacher != nullptr, in_place, states_too});
  c.h = p.h, c.weight = p.weight, c.h_ld = p.h_ld, c.weight_ld = p.weight_ld;
  c.dloss = p.dloss, c.loss = p.loss_out, c.lse = p.lse_out, c.dh = p.dh_out, c.dweight = p.dweight_out;
  c.tokens = (int)p.tokens, c.vocab = (int)p.vocab, c.width = (int)p.width, c.rows = (int)plan.rows;
  c.states_ld = (int)round_up(std::max<int64_t>(p.width, 1), 64), c.dz_ld = (int)round_up(p.vocab, 64);
  c.tile_n = plan.tile_n, c.tiles = plan.tiles;
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    char* const begin = workspace + at;
    at += (bytes + 255) / 256 * 256;
    return begin;
  };
  const size_t rows = (size_t)c.rows;
  c.sums = reinterpret_cast<float2*>(take(rows * c.tiles * sizeof(float2)));
  c.parts = reinterpret_cast<floatx4*>(take(std::max({plan.logits.workspace, plan.dh.workspace, plan.dweight.parts[0].workspace,
                                                      plan.dweight.parts[1].workspace, plan.both.dh.workspace + plan.both.dweight.workspace,
                                                      plan.dh_of_few.workspace})));
  c.dots = reinterpret_cast<float*>(take(rows * c.k * sizeof(float)));
  c.head = in_place || plan.direct || (plan.few && (!p.dh_out || plan.few_dh)) ? p.weight : take((size_t)p.vocab * c.states_ld * planes * 2);
  c.head_ld = in_place ? p.weight_ld : c.states_ld * planes;
  c.head_bytes = in_place ? (int)p.width * 2 : c.states_ld * 2;
  if (plan.direct) {
    c.states = const_cast<void*>(p.h), c.states_row = p.h_ld;
    return std::max<size_t>(at, 256);
  }
  c.count = reinterpret_cast<int*>(take(sizeof(int) + 2 * sizeof(float)));
  c.largest_weight = reinterpret_cast<float*>(c.count + 1);
  c.order = reinterpret_cast<int*>(take((size_t)p.tokens * sizeof(int)));
  c.counts = c.teacher ? reinterpret_cast<uint8_t*>(take((size_t)p.tokens)) : nullptr;
  c.states_row = c.states_ld * planes;
  c.states = take((size_t)round_up(c.rows, 64) * c.states_ld * planes * 2);
  if (c.k == 1) c.words = reinterpret_cast<int*>(take(rows * sizeof(int)));
  if (plan.picked) {
    c.sorted = reinterpret_cast<uint32_t*>(take(rows * c.k * sizeof(uint32_t)));
    c.begins = reinterpret_cast<uint16_t*>(take(rows * (c.tiles + 1) * sizeof(uint16_t)));
  }
  if (plan.counted) {
    c.refs = reinterpret_cast<float*>(take(rows * sizeof(float)));
    c.again = reinterpret_cast<int*>(take(sizeof(int)));
    c.row_scale = reinterpret_cast<float2*>(take(rows * sizeof(float2)));
  }
  c.dz = gradients ? take(rows * c.dz_ld * planes * 2) : nullptr;
  c.exps = gradients && !bf16 ? take(rows * c.dz_ld * 4) : c.dz;
  c.dweight_sum = bf16 && p.dweight_out && c.rows < p.tokens ? reinterpret_cast<float*>(take((size_t)p.vocab * p.width * sizeof(float))) : nullptr;
  return at;
}

int run(const tsenor_head& p, LossCall c, void* workspace, size_t workspace_bytes, hipStream_t s) {
  const bool bf16 = p.dtype == TSENOR_BF16;
  LossPlan plan;
  const size_t need = lay_out(p, nullptr, c, plan);
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < need) return TSENOR_ERR_WORKSPACE;
  lay_out(p, static_cast<char*>(workspace), c, plan);
  if (p.vocab == 0 || p.tokens == 0 || c.k == 0) {
    launch_zero(p.loss_out, p.tokens, false, s);
    if (p.lse_out) launch_zero(p.lse_out, p.tokens, false, s);
    if (p.dh_out) launch_zero(p.dh_out, p.tokens * p.width, bf16, s);
    if (p.dweight_out) launch_zero(p.dweight_out, p.vocab * p.width, bf16, s);
    return status_of_launches();
  }
  if (plan.direct) {
    for (c.first = 0; c.first < c.tokens; c.first += c.rows) {
      c.rows = std::min(c.rows, c.tokens - c.first);
      plan.few ? launch_few_logits(c, bf16, s) : launch_logits(c, plan.logits, bf16, s);
      launch_rows(c, plan.row_threads, bf16, s);
    }
    return status_of_launches();
  }
  if (c.teacher) counts_kernel<<<(unsigned)((c.tokens + 3) / 4), kThreads, 0, s>>>(c);
  const bool alone = c.tokens <= std::min(c.rows, kAloneTokens);
  if (!alone) order_kernel<<<1, kOrderThreads, 0, s>>>(c);
  if (c.head != c.weight) {
    uint16_t* const head = static_cast<uint16_t*>(const_cast<void*>(c.head));
    const int rows = std::max(1, std::min(kThreads / 8, kThreads * 8 / c.states_ld));  // (93469 x 76: one to a workgroup 30 us, 16 together 11)
    const unsigned groups = (unsigned)((c.vocab + rows - 1) / rows);
    bf16 ? head_kernel<true><<<groups, kThreads, 0, s>>>(c, head, rows) : head_kernel<false><<<groups, kThreads, 0, s>>>(c, head, rows);
  }
  for (c.first = 0; c.first < c.tokens; c.first += c.rows) {
    LossCall piece = c;
    piece.rows = std::min(c.rows, c.tokens - c.first), piece.last = c.first + piece.rows == c.tokens;
    const unsigned padded = (unsigned)round_up(piece.rows, 64);
    if (alone)
      bf16 ? gather_kernel<true, true><<<padded, kThreads, 0, s>>>(piece) : gather_kernel<false, true><<<padded, kThreads, 0, s>>>(piece);
    else
      bf16 ? gather_kernel<true, false><<<padded, kThreads, 0, s>>>(piece) : gather_kernel<false, false><<<padded, kThreads, 0, s>>>(piece);
    plan.few ? launch_few_logits(piece, bf16, s) : launch_logits(piece, plan.logits, bf16, s);
    launch_rows(piece, plan.row_threads, bf16, s);
    if (plan.both.use && c.width) {
      piece.head_first = 0, piece.head_rows = c.vocab;
      launch_both(piece, plan.both, bf16, s);
      continue;
    }
    if (c.dh && c.width) plan.few_dh ? launch_few_dh(piece, plan.dh_of_few, bf16, s) : launch_dh(piece, plan.dh, bf16, s);
    if (c.dweight && c.width)
      for (int k = 0; k < plan.dweight.count; ++k) {
        piece.head_first = k ? (int)plan.dweight.rows[0] : 0, piece.head_rows = (int)plan.dweight.rows[k];
        launch_dweight(piece, plan.dweight.parts[k], bf16, s);
      }
  }
  return status_of_launches();
}

LossCall call_of(const tsenor_cross_entropy_problem& p) {
  LossCall c = {};
  c.ids = p.targets, c.ids_ld = 1, c.k = 1, c.inverse_temperature = 1.0f, c.scale = (float)kLog2e;
  return c;
}
LossCall call_of(const tsenor_distill_problem& p) {
  LossCall c = {};
  c.ids = p.ids, c.ids_ld = p.ids_ld, c.teacher = p.logits, c.teacher_ld = p.logits_ld, c.teacher_bf16 = p.logits_dtype == TSENOR_BF16;
  c.k = p.k, c.inverse_temperature = (float)(1.0 / p.temperature), c.scale = (float)(kLog2e / p.temperature);
  return c;
}
template <class Problem>
size_t workspace_of(const Problem* p) {
  if (check(p) != TSENOR_OK) return 0;
  LossCall c = call_of(*p);
  LossPlan plan;
  return lay_out(p->head, nullptr, c, plan);
}
template <class Problem>
int run(const Problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream) {
  const int rc = check(p);
  return rc != TSENOR_OK ? rc : run(p->head, call_of(*p), workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" size_t tsenor_cross_entropy_workspace_bytes(const tsenor_cross_entropy_problem* p) { return workspace_of(p); }
extern "C" int tsenor_cross_entropy(const tsenor_cross_entropy_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream) {
  return run(p, workspace, workspace_bytes, stream);
}
extern "C" size_t tsenor_distill_workspace_bytes(const tsenor_distill_problem* p) { return workspace_of(p); }
extern "C" int tsenor_distill(const tsenor_distill_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream) {
  return run(p, workspace, workspace_bytes, stream);
}
