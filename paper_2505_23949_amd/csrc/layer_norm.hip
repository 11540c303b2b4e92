// tsenor_norm: residual addition, root-mean-square norm, 8-bit output with scales; tsenor_norm_backward: its gradients.
//
// Both need a sum over the row before the first result, and both keep the row in registers meanwhile, so that it is read once:
// THREADS threads to a row, VECTORS vectors of 8 to a thread, 128 columns on 16 neighbouring lanes, whose maximum is the scale's.
// Rows too long for that are read twice.  Bound by memory: bf16 4096 x 8192 with residual, sum, norm and its 8-bit form 57 us
// (5.3 TB/s), single precision 4096 x 4096 42 us (5.2); a single row by the launch (2.7 us).
#include <algorithm>
#include <cmath>

#include "layer.hpp"

namespace {

using namespace tsenor_dev;

struct NormArgs {
  const void *x, *residual, *gain;
  void *sum_out, *y_out;
  int64_t ld, residual_ld;
  int rows, cols;
  float eps;
  tsenor_scaled out;
  bool gain_bf16;
};

__host__ __device__ __forceinline__ const void* at_row(const void* p, int64_t row, int64_t ld, bool bf16) {
  return static_cast<const char*>(p) + row * ld * (bf16 ? 2 : 4);
}
__host__ __device__ __forceinline__ void* at_row(void* p, int64_t row, int64_t ld, bool bf16) {
  return static_cast<char*>(p) + row * ld * (bf16 ? 2 : 4);
}
__device__ __forceinline__ void load_gain8(const void* gain, bool bf16, int c, int cols, float (&g)[8]) {
  if (bf16)
    load_row8<true>(gain, c, cols, g);
  else
    load_row8<false>(gain, c, cols, g);
}

// x^-1/2 to within 0.51 units: the quotient's own error, and that of the root, taken off once more.  (A value whose error moves it over
// the middle between two 8-bit ones is 2^-4 off there, so each half unit less halves how many are.)
__device__ __forceinline__ float inverse_root(float x) {
  const float r = 1.0f / sqrtf(x);
  const float t = x * r, low = fmaf(x, r, -t), d = fmaf(-t, r, 1.0f) - low * r;
  return x > 0.0f && x < __builtin_inff() ? fmaf(0.5f * r, d, r) : r;
}

// h of 8 columns of a row: x, or its sum with the residual as it is stored
template <bool BF16>
__device__ __forceinline__ void load_sum8(const NormArgs& a, int64_t row, int c, float (&h)[8]) {
  const Raw8<BF16> x = load_raw8<BF16>(at_row(a.x, row, a.ld, BF16), c, a.cols);
  if (!a.residual) {
    widen8<BF16>(x, c, a.cols, h);
    return;
  }
  const Raw8<BF16> residual = load_raw8<BF16>(at_row(a.residual, row, a.residual_ld, BF16), c, a.cols);
  float r[8];
  widen8<BF16>(x, c, a.cols, h), widen8<BF16>(residual, c, a.cols, r);
#pragma unroll
  for (int k = 0; k < 8; ++k) h[k] = h[k] + r[k];
  if constexpr (BF16) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
      const uint32_t w = pack_bf16(h[k], h[k + 1]);
      h[k] = __uint_as_float(w << 16), h[k + 1] = __uint_as_float(w & 0xFFFF0000u);
    }
  }
}

// y of 8 columns from h, written as asked for.  h comes near 1 by a power of two first, so that its product with the gain is in range
// where y is; nothing is rounded then, and in bf16 not in that product either.
template <bool BF16>
__device__ __forceinline__ void write_norm8(const NormArgs& a, int64_t row, int c, float inverse, float (&h)[8]) {
  float g[8];
  load_gain8(a.gain, a.gain_bf16, c, a.cols, g);
  const bool ordinary = inverse > 0.0f && inverse < __builtin_inff();  // (not where the row has no norm)
  const uint32_t bits = __float_as_uint(inverse);
  const float power = ordinary ? __uint_as_float(bits & kInfinityBits) : 1.0f;
  const float rest = ordinary ? __uint_as_float((bits & ~kInfinityBits) | 0x3F800000u) : inverse;
#pragma unroll
  for (int k = 0; k < 8; ++k) h[k] = c + k < a.cols ? h[k] * power * g[k] * rest : 0.0f;
  if (a.y_out) store_row8<BF16>(at_row(a.y_out, row, a.cols, BF16), c, a.cols, h);
  if (a.out.values) {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) m = max(m, finite_size(h[k]));
    const uint32_t byte = scale_byte(row16_max(m));
    if (c / kBlock * kBlock < a.cols) {
      *reinterpret_cast<uint2*>(a.out.values + row * a.out.ld + c) = to_8bit(h, inverse_of_scale(byte));
      if (c % kBlock == 0) a.out.scales[(int64_t)(c / kBlock) * a.out.scale_ld + row] = (uint8_t)byte;
    }
  }
}

// sum over the THREADS threads of a row; `part` holds one float per wave, and may be used again after the next barrier
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = wave_sum(v);
  if constexpr (THREADS > kWave) {
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < THREADS / kWave; ++k) v += part[k];
  }
  return v;
}

constexpr int group_of(int threads) { return threads == kWave ? 256 : threads; }  // (four rows of a wave each)

template <bool BF16, int THREADS, int VECTORS>
__global__ __launch_bounds__(group_of(THREADS)) void norm_kernel(NormArgs a) {
  __shared__ float part[16];
  const int t = (int)threadIdx.x % THREADS;
  const int64_t row = (int64_t)blockIdx.x * (group_of(THREADS) / THREADS) + threadIdx.x / THREADS;
  if (THREADS == kWave && row >= a.rows) return;  // (whole waves, and no barrier follows)
  float h[VECTORS][8];
#pragma unroll
  for (int v = 0; v < VECTORS; ++v) load_sum8<BF16>(a, row, (v * THREADS + t) * 8, h[v]);
  float sum = 0.0f;
#pragma unroll
  for (int v = 0; v < VECTORS; ++v) {
    if (a.sum_out) store_row8<BF16>(at_row(a.sum_out, row, a.cols, BF16), (v * THREADS + t) * 8, a.cols, h[v]);
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fmaf(h[v][k], h[v][k], s);
    sum += s;
  }
  const float inverse = inverse_root(row_sum<THREADS>(sum, part) / (float)a.cols + a.eps);
#pragma unroll
  for (int v = 0; v < VECTORS; ++v) write_norm8<BF16>(a, row, (v * THREADS + t) * 8, inverse, h[v]);
}

// rows of any length, read twice: h comes back from sum_out where that is written (it may be x or the residual)
constexpr int kLongThreads = 1024;
template <bool BF16>
__global__ __launch_bounds__(kLongThreads) void norm_long_kernel(NormArgs a) {
  __shared__ float part[16];
  const int64_t row = blockIdx.x;
  const int step = kLongThreads * 8, end = (a.cols + kBlock - 1) / kBlock * kBlock;
  float sum = 0.0f;
  for (int c = (int)threadIdx.x * 8; c < a.cols; c += step) {
    float h[8], s = 0.0f;
    load_sum8<BF16>(a, row, c, h);
    if (a.sum_out) store_row8<BF16>(at_row(a.sum_out, row, a.cols, BF16), c, a.cols, h);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fmaf(h[k], h[k], s);
    sum += s;
  }
  const float inverse = inverse_root(row_sum<kLongThreads>(sum, part) / (float)a.cols + a.eps);
  // (whole groups of 16 lanes stay together: a step of 8192 columns is a multiple of 128, and so is `end`)
  for (int c = (int)threadIdx.x * 8; c < end; c += step) {
    float h[8];
    if (a.sum_out)
      load_row8<BF16>(at_row(a.sum_out, row, a.cols, BF16), c, a.cols, h);
    else
      load_sum8<BF16>(a, row, c, h);
    write_norm8<BF16>(a, row, c, inverse, h);
  }
}

// ---- backward ----------------------------------------------------------------------------------------------------------
struct BackwardArgs {
  const void *h, *gain, *dy, *dsum;
  void* dh;
  float* dgain;  // of each workgroup, `cols` apart; the result itself where there is one workgroup
  int64_t ld, dy_ld, dsum_ld;
  int rows, cols;
  float eps;
  bool gain_bf16;
};

// sums of two values over the THREADS threads of a row, in all of them
template <int THREADS>
__device__ __forceinline__ void row_sum2(float& u, float& v, float (*part)[2]) {
  u = wave_sum(u), v = wave_sum(v);
  if constexpr (THREADS > kWave) {
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave][0] = u, part[threadIdx.x / kWave][1] = v;
    __syncthreads();
    u = 0.0f, v = 0.0f;
#pragma unroll
    for (int k = 0; k < THREADS / kWave; ++k) u += part[k][0], v += part[k][1];
  }
}

// dh of 8 columns, and their part of dgain added to `dg`; d: the gradient that reaches h past the norm.  With u = h c, a row of mean
// square 1, the formula is dh = c (gain dy - u toward) + d, toward = mean(gain dy u): c^3 is not needed, which leaves the range of
// single precision for rows of 1e13 or 1e-13 where none of these does.
template <bool BF16>
__device__ __forceinline__ void write_backward8(const BackwardArgs& a, int64_t row, int c, float inverse, float toward, const float (&h)[8],
                                                const float (&dy)[8], const float (&g)[8], float (&d)[8], float (&dg)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float unit = h[k] * inverse;
    d[k] = fmaf(inverse, fmaf(-unit, toward, g[k] * dy[k]), d[k]);  // (d last: it may cancel what the norm gives)
    dg[k] = fmaf(dy[k], unit, dg[k]);
  }
  store_row8<BF16>(at_row(a.dh, row, a.cols, BF16), c, a.cols, d);
}

// what a thread reads of a row
template <bool BF16, int VECTORS>
struct BackwardRow {
  Raw8<BF16> h[VECTORS], dy[VECTORS], dsum[VECTORS];
};
template <bool BF16, int THREADS, bool AHEAD, int VECTORS>
__device__ __forceinline__ void load_backward(const BackwardArgs& a, int64_t row, BackwardRow<BF16, VECTORS>& x) {
  if (row >= a.rows) return;
#pragma unroll
  for (int v = 0; v < VECTORS; ++v) {
    const int c = (v * THREADS + (int)threadIdx.x) * 8;
    x.h[v] = load_raw8<BF16>(at_row(a.h, row, a.ld, BF16), c, a.cols);
    x.dy[v] = load_raw8<BF16>(at_row(a.dy, row, a.dy_ld, BF16), c, a.cols);
    if (AHEAD && a.dsum) x.dsum[v] = load_raw8<BF16>(at_row(a.dsum, row, a.dsum_ld, BF16), c, a.cols);
  }
}

// A workgroup takes every gridDim.x-th row, asks for the next before it works on one (AHEAD: where the registers hold both, which those
// of 1024 threads do for bf16 only), and keeps its sum of dgain in registers.  Bound by memory: 2047 x 4096 in single precision 31 us
// (4.3 TB/s), bf16 4096 x 4096 with dsum 33 (45 where each row was asked for when its turn came); single precision 2048 x 8192 55,
// with the next row asked for 55.6 and, where that spills, 2000 x 5001 53 for 47.
template <bool BF16, int THREADS, int VECTORS, bool AHEAD>
__global__ __launch_bounds__(THREADS) void norm_backward_kernel(BackwardArgs a) {
  __shared__ float part[2][16][2];
  const int t = (int)threadIdx.x;
  float g[VECTORS][8], dg[VECTORS][8] = {};
#pragma unroll
  for (int v = 0; v < VECTORS; ++v) load_gain8(a.gain, a.gain_bf16, (v * THREADS + t) * 8, a.cols, g[v]);
  const auto work = [&](int64_t row, const BackwardRow<BF16, VECTORS>& x, float (&sums)[16][2]) {
    float h[VECTORS][8], dy[VECTORS][8];
    float squares = 0.0f, along = 0.0f;
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
      const int c = (v * THREADS + t) * 8;
      widen8<BF16>(x.h[v], c, a.cols, h[v]), widen8<BF16>(x.dy[v], c, a.cols, dy[v]);
#pragma unroll
      for (int k = 0; k < 8; ++k) squares = fmaf(h[v][k], h[v][k], squares), along = fmaf(g[v][k] * dy[v][k], h[v][k], along);
    }
    row_sum2<THREADS>(squares, along, sums);
    const float inverse = inverse_root(squares / (float)a.cols + a.eps);
    const float toward = along * inverse / (float)a.cols;
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
      const int c = (v * THREADS + t) * 8;
      float d[8] = {};
      if (a.dsum) widen8<BF16>(AHEAD ? x.dsum[v] : load_raw8<BF16>(at_row(a.dsum, row, a.dsum_ld, BF16), c, a.cols), c, a.cols, d);
      write_backward8<BF16>(a, row, c, inverse, toward, h[v], dy[v], g[v], d, dg[v]);
    }
  };
  // (two places for the sums: one barrier a row)
  if constexpr (AHEAD) {
    BackwardRow<BF16, VECTORS> even = {}, odd = {};
    load_backward<BF16, THREADS, true>(a, blockIdx.x, even);
    for (int64_t row = blockIdx.x; row < a.rows; row += 2 * (int64_t)gridDim.x) {
      load_backward<BF16, THREADS, true>(a, row + gridDim.x, odd);
      work(row, even, part[0]);
      if (row + gridDim.x >= a.rows) break;
      load_backward<BF16, THREADS, true>(a, row + 2 * (int64_t)gridDim.x, even);
      work(row + gridDim.x, odd, part[1]);
    }
  } else {
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
      BackwardRow<BF16, VECTORS> x;
      load_backward<BF16, THREADS, false>(a, row, x);
      work(row, x, part[turn]);
    }
  }
  float* sums = a.dgain + (int64_t)blockIdx.x * a.cols;
#pragma unroll
  for (int v = 0; v < VECTORS; ++v) store_row8<false>(sums, (v * THREADS + t) * 8, a.cols, dg[v]);
}

// Rows too long for registers: their two numbers first,
template <bool BF16>
__global__ __launch_bounds__(kLongThreads) void backward_stats_kernel(BackwardArgs a, float2* stats) {
  __shared__ float part[16][2];
  const int64_t row = blockIdx.x;
  float squares = 0.0f, along = 0.0f;
  for (int c = (int)threadIdx.x * 8; c < a.cols; c += kLongThreads * 8) {
    float h[8], dy[8], g[8], s = 0.0f, l = 0.0f;
    load_row8<BF16>(at_row(a.h, row, a.ld, BF16), c, a.cols, h);
    load_row8<BF16>(at_row(a.dy, row, a.dy_ld, BF16), c, a.cols, dy);
    load_gain8(a.gain, a.gain_bf16, c, a.cols, g);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fmaf(h[k], h[k], s), l = fmaf(g[k] * dy[k], h[k], l);
    squares += s, along += l;
  }
  row_sum2<kLongThreads>(squares, along, part);
  const float inverse = inverse_root(squares / (float)a.cols + a.eps);
  if (threadIdx.x == 0) stats[row] = make_float2(inverse, along * inverse / (float)a.cols);
}
// then the gradients, 2048 columns and every gridDim.y-th row to a workgroup.
constexpr int kSlab = 2048;
template <bool BF16>
__global__ __launch_bounds__(256) void backward_apply_kernel(BackwardArgs a, const float2* stats) {
  const int c = (int)blockIdx.x * kSlab + (int)threadIdx.x * 8;
  float g[8], dg[8] = {};
  load_gain8(a.gain, a.gain_bf16, c, a.cols, g);
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    float h[8], dy[8];
    load_row8<BF16>(at_row(a.h, row, a.ld, BF16), c, a.cols, h);
    load_row8<BF16>(at_row(a.dy, row, a.dy_ld, BF16), c, a.cols, dy);
    const float2 s = stats[row];
    float d[8] = {};
    if (a.dsum) load_row8<BF16>(at_row(a.dsum, row, a.dsum_ld, BF16), c, a.cols, d);
    write_backward8<BF16>(a, row, c, s.x, s.y, h, dy, g, d, dg);
  }
  store_row8<false>(a.dgain + (int64_t)blockIdx.y * a.cols, c, a.cols, dg);
}

// dgain from what the `groups` workgroups left, in a fixed order: for 16 columns, 64 runs of workgroups, then the runs
__global__ __launch_bounds__(1024) void gather_dgain_kernel(const float* sums, int groups, int cols, float* dgain) {
  __shared__ float part[16][16];
  const int lane = (int)threadIdx.x % 16, run = (int)threadIdx.x / 16, wave = (int)threadIdx.x / kWave;
  const int64_t c = (int64_t)blockIdx.x * 16 + lane;
  const int per = (groups + 63) / 64, end = min(groups, (run + 1) * per);
  float s = 0.0f;
  if (c < cols)
#pragma unroll 8
    for (int k = run * per; k < end; ++k) s += sums[(int64_t)k * cols + c];
  s += lane_xor<16>(s);
  s += lane_xor<32>(s);
  if (threadIdx.x % kWave < 16) part[wave][lane] = s;
  __syncthreads();
  if (run == 0 && c < cols) {
#pragma unroll
    for (int k = 1; k < 16; ++k) s += part[k][lane];
    dgain[c] = s;
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------
int check(const tsenor_norm_problem* p) {
  if (!p) return TSENOR_ERR_NULL;
  if (p->rows != 0 && p->cols != 0 && (!p->x || !p->gain || (!p->sum_out && !p->y_out && !p->out.values))) return TSENOR_ERR_NULL;
  if (!known(p->dtype) || !known(p->gain_dtype)) return TSENOR_ERR_UNSUPPORTED;
  if (!shape_ok(p->rows, p->cols) || !ld_ok(p->ld, p->rows, p->cols) ||
      (p->residual && !ld_ok(p->residual_ld, p->rows, p->cols)))
    return TSENOR_ERR_SHAPE;
  if (!(p->eps >= 0.0) || !std::isfinite((float)p->eps)) return TSENOR_ERR_PARAM;
  const size_t e = size_of(p->dtype);
  if (!aligned_to(p->x, e) || !aligned_to(p->residual, e) || !aligned_to(p->sum_out, e) || !aligned_to(p->y_out, e) ||
      !aligned_to(p->gain, size_of(p->gain_dtype)))
    return TSENOR_ERR_ALIGN;
  if (!p->out.values) return TSENOR_OK;
  if (p->out.rows != p->rows || p->out.cols != p->cols) return TSENOR_ERR_SHAPE;
  return check_scaled(p->out);
}

int check(const tsenor_norm_backward_problem* p) {
  if (!p) return TSENOR_ERR_NULL;
  if (p->cols != 0 && (!p->gain || !p->dgain_out || (p->rows != 0 && (!p->h || !p->dy || !p->dh_out)))) return TSENOR_ERR_NULL;
  if (!known(p->dtype) || !known(p->gain_dtype)) return TSENOR_ERR_UNSUPPORTED;
  if (!shape_ok(p->rows, p->cols) || !ld_ok(p->ld, p->rows, p->cols) || !ld_ok(p->dy_ld, p->rows, p->cols) ||
      (p->dsum && !ld_ok(p->dsum_ld, p->rows, p->cols)))
    return TSENOR_ERR_SHAPE;
  if (!(p->eps >= 0.0) || !std::isfinite((float)p->eps)) return TSENOR_ERR_PARAM;
  const size_t e = size_of(p->dtype);
  if (!aligned_to(p->h, e) || !aligned_to(p->dy, e) || !aligned_to(p->dsum, e) || !aligned_to(p->dh_out, e) ||
      !aligned_to(p->gain, size_of(p->gain_dtype)) || !aligned_to(p->dgain_out, 4))
    return TSENOR_ERR_ALIGN;
  return TSENOR_OK;
}

constexpr int64_t kLaunchRows = 1 << 21;  // of up to 1024 threads: a grid counts fewer than 2^32 threads
constexpr int kLongRow = 16384;  // columns that the registers of 1024 threads hold, 16 to a thread
inline size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Workgroups that share the rows of a backward pass: each leaves a sum of dgain, which costs a write and a read of its columns; fewer than
// one to a CU leave the memory idle.  (bf16 4096 x 8192 256 of them 56.9 us, 512 64.0; 2000 x 14336 55.8, 63.7; 8000 x 512 with 2048
// 14.4, with 512 18.2.)
inline int64_t backward_groups(const tsenor_norm_backward_problem& p) {
  const int64_t most = p.cols <= kLongRow ? std::clamp<int64_t>(((int64_t)1 << 20) / std::max<int64_t>(p.cols, 1), 256, 2048)
                                          : std::max<int64_t>(1, 1024 / ((p.cols + kSlab - 1) / kSlab));
  return std::max<int64_t>(1, std::min({p.rows, most, std::max<int64_t>(256, p.rows / 4)}));
}
struct BackwardLayout {
  size_t stats, sums, total;
};
inline BackwardLayout layout_of(const tsenor_norm_backward_problem& p) {
  BackwardLayout l = {0, 0, 0};
  const int64_t groups = backward_groups(p);
  l.sums = p.cols > kLongRow ? padded((size_t)p.rows * sizeof(float2)) : 0;
  l.total = l.sums + (groups > 1 ? padded((size_t)(groups * p.cols) * sizeof(float)) : 0);
  return l;
}

// One vector to a thread as long as a workgroup can have that many: 16 x 8192 3.5 us where 256 threads with four take 5.4, 2048 x 8192
// 22.0 (22.6), 4096 x 4096 21.2 (512 with one) and 21.8 (256 with two).
template <bool BF16>
void launch_norm(const NormArgs& a, hipStream_t s) {
  const unsigned rows = (unsigned)a.rows;
  if (a.cols <= 512)
    norm_kernel<BF16, 64, 1><<<(rows + 3) / 4, 256, 0, s>>>(a);
  else if (a.cols <= 1024)
    norm_kernel<BF16, 128, 1><<<rows, 128, 0, s>>>(a);
  else if (a.cols <= 2048)
    norm_kernel<BF16, 256, 1><<<rows, 256, 0, s>>>(a);
  else if (a.cols <= 4096)
    norm_kernel<BF16, 512, 1><<<rows, 512, 0, s>>>(a);
  else if (a.cols <= 8192)
    norm_kernel<BF16, 1024, 1><<<rows, 1024, 0, s>>>(a);
  else if (a.cols <= kLongRow)
    norm_kernel<BF16, 1024, 2><<<rows, 1024, 0, s>>>(a);
  else
    norm_long_kernel<BF16><<<rows, kLongThreads, 0, s>>>(a);
}

template <bool BF16>
void launch_backward(const BackwardArgs& a, unsigned groups, float2* stats, hipStream_t s) {
  if (a.cols <= 512) {
    norm_backward_kernel<BF16, 64, 1, true><<<groups, 64, 0, s>>>(a);
  } else if (a.cols <= 1024) {
    norm_backward_kernel<BF16, 128, 1, true><<<groups, 128, 0, s>>>(a);
  } else if (a.cols <= 2048) {
    norm_backward_kernel<BF16, 256, 1, true><<<groups, 256, 0, s>>>(a);
  } else if (a.cols <= 4096) {
    norm_backward_kernel<BF16, 512, 1, true><<<groups, 512, 0, s>>>(a);
  } else if (a.cols <= 8192) {
    norm_backward_kernel<BF16, 1024, 1, BF16><<<groups, 1024, 0, s>>>(a);
  } else if (a.cols <= kLongRow) {
    norm_backward_kernel<BF16, 1024, 2, false><<<groups, 1024, 0, s>>>(a);
  } else {
    BackwardArgs part = a;
    for (int64_t row = 0; row < a.rows; row += kLaunchRows) {
      part.h = at_row(a.h, row, a.ld, BF16), part.dy = at_row(a.dy, row, a.dy_ld, BF16);
      backward_stats_kernel<BF16><<<(unsigned)std::min(a.rows - row, kLaunchRows), kLongThreads, 0, s>>>(part, stats + row);
    }
    backward_apply_kernel<BF16><<<dim3((unsigned)((a.cols + kSlab - 1) / kSlab), groups), 256, 0, s>>>(a, stats);
  }
}

}  // namespace

extern "C" int tsenor_norm(const tsenor_norm_problem* p, tsenor_stream_t stream) {
  const int rc = check(p);
  if (rc != TSENOR_OK) return rc;
  if (p->rows == 0 || p->cols == 0) return TSENOR_OK;
  NormArgs a = {};
  a.x = p->x, a.residual = p->residual, a.gain = p->gain, a.sum_out = p->sum_out, a.y_out = p->y_out;
  a.ld = p->ld, a.residual_ld = p->residual_ld, a.cols = (int)p->cols, a.eps = (float)p->eps;
  a.out = p->out;
  a.gain_bf16 = p->gain_dtype == TSENOR_BF16;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = p->dtype == TSENOR_BF16;
  for (int64_t row = 0; row < p->rows; row += kLaunchRows) {
    a.rows = (int)std::min(p->rows - row, kLaunchRows);
    bf16 ? launch_norm<true>(a, s) : launch_norm<false>(a, s);
    a.x = at_row(a.x, a.rows, a.ld, bf16);
    if (a.residual) a.residual = at_row(a.residual, a.rows, a.residual_ld, bf16);
    if (a.sum_out) a.sum_out = at_row(a.sum_out, a.rows, a.cols, bf16);
    if (a.y_out) a.y_out = at_row(a.y_out, a.rows, a.cols, bf16);
    if (a.out.values) a.out.values += a.rows * a.out.ld, a.out.scales += a.rows;
  }
  return status_of_launches();
}

extern "C" size_t tsenor_norm_backward_workspace_bytes(const tsenor_norm_backward_problem* p) {
  return check(p) == TSENOR_OK ? layout_of(*p).total : 0;
}

extern "C" int tsenor_norm_backward(const tsenor_norm_backward_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream) {
  const int rc = check(p);
  if (rc != TSENOR_OK) return rc;
  const BackwardLayout l = layout_of(*p);
  if (l.total && (!workspace || !aligned_to(workspace, 256) || workspace_bytes < l.total)) return TSENOR_ERR_WORKSPACE;
  if (p->cols == 0) return TSENOR_OK;
  const int groups = (int)backward_groups(*p);
  char* ws = static_cast<char*>(workspace);
  BackwardArgs a = {};
  a.h = p->h, a.gain = p->gain, a.dy = p->dy, a.dsum = p->dsum, a.dh = p->dh_out;
  a.dgain = groups > 1 ? reinterpret_cast<float*>(ws + l.sums) : p->dgain_out;
  a.ld = p->ld, a.dy_ld = p->dy_ld, a.dsum_ld = p->dsum_ld, a.rows = (int)p->rows, a.cols = (int)p->cols, a.eps = (float)p->eps;
  a.gain_bf16 = p->gain_dtype == TSENOR_BF16;
  hipStream_t s = static_cast<hipStream_t>(stream);
  float2* stats = reinterpret_cast<float2*>(ws);
  p->dtype == TSENOR_BF16 ? launch_backward<true>(a, (unsigned)groups, stats, s) : launch_backward<false>(a, (unsigned)groups, stats, s);
  if (groups > 1) gather_dgain_kernel<<<(unsigned)((p->cols + 15) / 16), 1024, 0, s>>>(a.dgain, groups, (int)p->cols, p->dgain_out);
  return status_of_launches();
}
