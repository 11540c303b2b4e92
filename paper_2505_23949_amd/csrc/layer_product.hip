// tsenor_product: out = a b^T of two matrices in 8-bit floating point with a power of two for each row and 128 columns.
//
// Everything goes through v_mfma_scale_f32_16x16x128_f8f6f4: 16 rows of either operand, one block of 128 columns, whose powers of
// two the instruction applies, so the scales cost no vector instruction.  b (weights) is its first operand: a lane then holds four
// neighbouring columns of the result.  The order of the 128 columns in the sum is free as long as both operands agree: lane l
// takes the 16 bytes at 16 (l / 16) and those 64 further on, so that four lanes read 64 bytes in a row.
#include "layer.hpp"

namespace {

using namespace tsenor_dev;

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

struct ProductArgs {
  tsenor_scaled a, b;
  uint16_t* out;
  const uint8_t* mask;
  int64_t out_ld;
  int m, n, blocks;  // blocks of 128 columns
  bool out_vec;      // four results from a multiple of 4 on can be written at once
};

// 16 rows of a scaled matrix, one block of columns: the operand of lane l holds part of row l % 16
__device__ __forceinline__ intx8 load_operand(const uint8_t* row) {
  const int4 lo = *reinterpret_cast<const int4*>(row), hi = *reinterpret_cast<const int4*>(row + 64);
  return intx8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
}
__device__ __forceinline__ floatx4 multiply(const intx8& x, const intx8& y, const floatx4& sum, int x_scale, int y_scale) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, sum, 0, 0, 0, x_scale, 0, y_scale);
}

// results of row i, columns j to j + 3
__device__ __forceinline__ void write4(const ProductArgs& a, int i, int j, float (&v)[4]) {
  if (i >= a.m || j >= a.n) return;
  if (a.mask) {
    const uint8_t* m = a.mask + (int64_t)i * a.n + j;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j + k < a.n && !m[k]) v[k] = 0.0f;
  }
  uint16_t* out = a.out + (int64_t)i * a.out_ld + j;
  const uint2 w = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  if (a.out_vec && j + 4 <= a.n) {
    *reinterpret_cast<uint2*>(out) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j + k < a.n) out[k] = (uint16_t)((k < 2 ? w.x : w.y) >> (k % 2 * 16));
  }
}

// Few rows of a: the weights are read once, straight into registers, by a workgroup of WAVES waves for each 16 of their rows, that
// share the columns: every wave takes each WAVES-th block.  Their sums meet in LDS.
constexpr int kWaves = 8;
template <int TILES>
__global__ __launch_bounds__(kWaves* kWave) void few_rows_kernel(ProductArgs p) {
  __shared__ float sums[kWaves][TILES][kWave][4];
  const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave;
  const int n0 = (int)blockIdx.x * 16, m0 = (int)blockIdx.y * TILES * 16;
  const int64_t row_b = min(n0 + lane % 16, p.n - 1);
  const uint8_t* b = p.b.values + row_b * p.b.ld + lane / 16 * 16;
  const uint8_t* a[TILES];
  int64_t row_a[TILES];
  floatx4 sum[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    row_a[t] = min(m0 + t * 16 + lane % 16, p.m - 1);
    a[t] = p.a.values + row_a[t] * p.a.ld + lane / 16 * 16;
    sum[t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  for (int k = wave; k < p.blocks; k += kWaves) {
    const intx8 x = load_operand(b + (int64_t)k * kBlock);
    const int x_scale = p.b.scales[k * p.b.scale_ld + row_b];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const intx8 y = load_operand(a[t] + (int64_t)k * kBlock);
      sum[t] = multiply(x, y, sum[t], x_scale, p.a.scales[k * p.a.scale_ld + row_a[t]]);
    }
  }
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[wave][t][lane][k] = sum[t][k];
  __syncthreads();
  for (int at = (int)threadIdx.x; at < TILES * kWave; at += kWaves * kWave) {
    const int t = at / kWave, l = at % kWave;
    float v[4] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += sums[w][t][l][k];
    write4(p, m0 + t * 16 + l % 16, n0 + l / 16 * 4, v);
  }
}

int check(const tsenor_product_problem* p) {
  if (!p || (p->a.rows != 0 && p->b.rows != 0 && !p->out)) return TSENOR_ERR_NULL;
  int rc = check_scaled(p->a);
  if (rc != TSENOR_OK) return rc;
  rc = check_scaled(p->b);
  if (rc != TSENOR_OK) return rc;
  if (p->a.cols != p->b.cols || p->b.rows > (int64_t)1 << 24 || !ld_ok(p->out_ld, p->b.rows) || !shape_ok(p->a.rows, p->b.rows))
    return TSENOR_ERR_SHAPE;
  return aligned_to(p->out, 2) ? TSENOR_OK : TSENOR_ERR_ALIGN;
}

}  // namespace

extern "C" size_t tsenor_product_workspace_bytes(const tsenor_product_problem* p) {
  (void)p;
  return 0;
}

extern "C" int tsenor_product(const tsenor_product_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream) {
  (void)workspace, (void)workspace_bytes;
  const int rc = check(p);
  if (rc != TSENOR_OK) return rc;
  if (p->a.rows == 0 || p->b.rows == 0) return TSENOR_OK;
  ProductArgs a = {};
  a.a = p->a, a.b = p->b, a.out = static_cast<uint16_t*>(p->out), a.mask = p->mask, a.out_ld = p->out_ld;
  a.m = (int)p->a.rows, a.n = (int)p->b.rows, a.blocks = (int)blocks_of(p->a.cols);
  a.out_vec = aligned_to(p->out, 8) && p->out_ld % 4 == 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned across = (unsigned)((a.n + 15) / 16);
  few_rows_kernel<4><<<dim3(across, (unsigned)((a.m + 63) / 64)), kWaves * kWave, 0, s>>>(a);
  return status_of_launches();
}
