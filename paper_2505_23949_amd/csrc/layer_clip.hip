// tsenor_clip: the norm of all gradients of a model, and the gradients scaled down to a largest norm.
//
// A tensor is cut into chunks; the chunks of up to kMaxTensors tensors share a launch, whose table is a kernel argument.  Each
// workgroup of the first pass leaves one sum of squares in double, and each of the second adds all of those in the same order
// before it scales: no atomics, nothing to clear, and no launch between the two.  Bound by memory.  The second pass goes
// through the chunks from the last to the first: what the first one read last is still in the cache of the memory side.
#include <algorithm>

#include "layer.hpp"

namespace {

using namespace tsenor_dev;

constexpr int kThreads = 256;
constexpr int kChunk = 8192;       // elements
constexpr int kMaxTensors = 100;   // of a launch
constexpr int kMaxGroups = 1024;   // workgroups of a launch, sums that it leaves

struct ClipTensor {
  const void* in;
  void* out;
  int64_t count;
};
struct ClipTable {
  int count;
  uint32_t first[kMaxTensors + 1];  // chunk that each tensor begins with
  uint8_t bf16[kMaxTensors];
  ClipTensor t[kMaxTensors];
};
static_assert(sizeof(ClipTable) <= 4000, "the table travels as a kernel argument");

// tensor that a chunk belongs to (those without elements have none)
__device__ __forceinline__ int tensor_of(const ClipTable& table, uint32_t chunk) {
  int lo = 0, hi = table.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (table.first[mid] <= chunk)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double square_of(float v) { return (double)v * (double)v; }

template <bool BF16>
__device__ __forceinline__ double squares_of_chunk(const void* in, int64_t begin, int64_t end) {
  double s = 0.0;
  if (end - begin == kChunk) {
#pragma unroll
    for (int k = 0; k < kChunk / (kThreads * 8); ++k) {
      float x[8];
      load_row8<BF16>(static_cast<const char*>(in) + begin * (BF16 ? 2 : 4), (k * kThreads + (int)threadIdx.x) * 8, kChunk, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fma((double)x[j], (double)x[j], s);
    }
  } else {
    for (int64_t i = begin + threadIdx.x; i < end; i += kThreads)
      s += square_of(BF16 ? widen(static_cast<const uint16_t*>(in)[i]) : static_cast<const float*>(in)[i]);
  }
  return s;
}

// sum over the workgroup, in thread 0
__device__ __forceinline__ double group_sum(double s) {
  __shared__ double part[kThreads / kWave];
  s += lane_xor<1>(s), s += lane_xor<2>(s), s += lane_xor<7>(s), s += lane_xor<15>(s), s += lane_xor<16>(s), s += lane_xor<32>(s);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = s;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

__global__ __launch_bounds__(kThreads) void squares_kernel(ClipTable table, double* sums) {
  double s = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < table.first[table.count]; chunk += gridDim.x) {
    const int k = tensor_of(table, chunk);
    const ClipTensor t = table.t[k];
    const int64_t begin = (int64_t)(chunk - table.first[k]) * kChunk, end = min(t.count, begin + kChunk);
    s += table.bf16[k] ? squares_of_chunk<true>(t.in, begin, end) : squares_of_chunk<false>(t.in, begin, end);
  }
  s = group_sum(s);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

template <bool BF16>
__device__ __forceinline__ void scale_chunk(const ClipTensor& t, int64_t begin, int64_t end, float factor) {
  if (end - begin == kChunk) {
#pragma unroll
    for (int k = 0; k < kChunk / (kThreads * 8); ++k) {
      const int c = (k * kThreads + (int)threadIdx.x) * 8;
      float x[8];
      load_row8<BF16>(static_cast<const char*>(t.in) + begin * (BF16 ? 2 : 4), c, kChunk, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= factor;
      store_row8<BF16>(static_cast<char*>(t.out) + begin * (BF16 ? 2 : 4), c, kChunk, x);
    }
  } else {
    for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) {
      if constexpr (BF16)
        static_cast<uint16_t*>(t.out)[i] = (uint16_t)pack_bf16(widen(static_cast<const uint16_t*>(t.in)[i]) * factor, 0.0f);
      else
        static_cast<float*>(t.out)[i] = static_cast<const float*>(t.in)[i] * factor;
    }
  }
}

__global__ __launch_bounds__(kThreads) void scale_kernel(ClipTable table, const double* sums, int count, double max_norm, float* norm_out) {
  double s = 0.0;
  for (int k = (int)threadIdx.x; k < count; k += kThreads) s += sums[k];
  const double norm = sqrt(group_sum(s));
  const float factor = norm > max_norm && norm <= 1.7976931348623157e308 ? (float)(max_norm / norm) : 1.0f;
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) norm_out[0] = (float)norm, norm_out[1] = factor;
  const uint32_t chunks = table.first[table.count];
  for (uint32_t back = blockIdx.x; back < chunks; back += gridDim.x) {
    const uint32_t chunk = chunks - 1 - back;
    const int k = tensor_of(table, chunk);
    const ClipTensor t = table.t[k];
    if (factor == 1.0f && t.in == t.out) continue;
    const int64_t begin = (int64_t)(chunk - table.first[k]) * kChunk, end = min(t.count, begin + kChunk);
    table.bf16[k] ? scale_chunk<true>(t, begin, end, factor) : scale_chunk<false>(t, begin, end, factor);
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------
constexpr int64_t kMaxCount = (int64_t)1 << 40;
constexpr int kMaxGradients = 1 << 20;
// (a launch counts its chunks in 32 bits)
constexpr int64_t kMaxChunks = (int64_t)1 << 31;
inline int64_t chunks_of(int64_t count) { return (count + kChunk - 1) / kChunk; }

int check(const tsenor_clip_problem* p) {
  if (!p || !p->norm_out || (p->count > 0 && !p->gradients)) return TSENOR_ERR_NULL;
  if (p->count < 0 || p->count > kMaxGradients) return TSENOR_ERR_SHAPE;
  if (!(p->max_norm >= 0.0)) return TSENOR_ERR_PARAM;
  if (!aligned_to(p->norm_out, 4)) return TSENOR_ERR_ALIGN;
  for (int k = 0; k < p->count; ++k) {
    const tsenor_gradient& g = p->gradients[k];
    if (!known(g.dtype)) return TSENOR_ERR_UNSUPPORTED;
    if (g.count < 0 || g.count > kMaxCount) return TSENOR_ERR_SHAPE;
    if (g.count > 0 && (!g.in || !g.out)) return TSENOR_ERR_NULL;
    if (!aligned_to(g.in, size_of(g.dtype)) || !aligned_to(g.out, size_of(g.dtype))) return TSENOR_ERR_ALIGN;
  }
  return TSENOR_OK;
}

// the table of the tensors from `k` on that share a launch; returns the one after them
int fill_table(const tsenor_clip_problem& p, int k, ClipTable& table) {
  table.count = 0;
  int64_t chunks = 0;
  for (; k < p.count && table.count < kMaxTensors; ++k) {
    const tsenor_gradient& g = p.gradients[k];
    if (g.count == 0) continue;
    if (chunks + chunks_of(g.count) > kMaxChunks) break;
    const int i = table.count++;
    table.first[i] = (uint32_t)chunks;
    table.bf16[i] = g.dtype == TSENOR_BF16;
    table.t[i] = {g.in, g.out, g.count};
    chunks += chunks_of(g.count);
  }
  table.first[table.count] = (uint32_t)chunks;
  return k;
}
inline unsigned groups_of(const ClipTable& table) { return std::min<unsigned>(table.first[table.count], kMaxGroups); }

}  // namespace

extern "C" size_t tsenor_clip_workspace_bytes(const tsenor_clip_problem* p) {
  if (check(p) != TSENOR_OK) return 0;
  // (as many launches as tensors at most, each with at least one tensor; 256 bytes where there is none)
  ClipTable table;
  size_t sums = 0;
  for (int k = 0; k < p->count;) {
    k = fill_table(*p, k, table);
    sums += groups_of(table);
  }
  return std::max<size_t>(256, (sums * sizeof(double) + 255) / 256 * 256);
}

extern "C" int tsenor_clip(const tsenor_clip_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream) {
  const int rc = check(p);
  if (rc != TSENOR_OK) return rc;
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < tsenor_clip_workspace_bytes(p)) return TSENOR_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  double* sums = static_cast<double*>(workspace);
  ClipTable table;
  int count = 0;
  for (int k = 0; k < p->count;) {
    k = fill_table(*p, k, table);
    const unsigned groups = groups_of(table);
    if (groups == 0) continue;
    squares_kernel<<<groups, kThreads, 0, s>>>(table, sums + count);
    count += (int)groups;
  }
  // norm and factor are written by the first launch of the second pass, which there is also without gradients
  float* norm_out = p->norm_out;
  for (int k = 0; k < p->count || norm_out;) {
    k = fill_table(*p, k, table);
    const unsigned groups = groups_of(table);
    if (groups == 0 && (!norm_out || k < p->count)) continue;
    scale_kernel<<<std::max(groups, 1u), kThreads, 0, s>>>(table, sums, count, p->max_norm, norm_out);
    norm_out = nullptr;
  }
  return status_of_launches();
}
