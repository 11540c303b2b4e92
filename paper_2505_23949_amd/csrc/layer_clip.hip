// tsenor_clip: the norm of all gradients of a model, and the gradients scaled down to a largest norm.
//
// A tensor is cut into chunks of 4096 elements; the chunks of up to kMaxTensors tensors share a launch, whose table is a kernel
// argument, and workgroups take every gridDim.x-th of them, so that what is read at a time lies together.  In the first pass each
// leaves one sum of squares in double, and each of the second adds all of those in the same order before it scales: no
// atomics, nothing to clear, and no launch between the two.  Workgroups of one number share a sum over all launches, so that what a
// workgroup adds does not grow with the tensors (4000 of 50 000 floats: 0.78 ms, 1.90 with sums of their own for each launch).
//
// Bound by memory.  The second pass goes through the chunks from the last to the first, what the first one read last being still
// in the cache of the memory side (2 % for a layer of 436 MB), and its accesses are marked as the last ones to what they touch, so
// that results do not drive out what is still to be read: the gradients of a layer of 4096 (218 M in bf16) 210-215 us, 243 without
// the mark.  (8 or 4 vectors in flight and half as many workgroups: 241, 227.)
#include <algorithm>

#include "layer.hpp"

namespace {

using namespace tsenor_dev;

constexpr int kThreads = 256;
constexpr int kVectors = 2;                      // of 8 elements, that a thread has in flight
constexpr int kChunk = kThreads * 8 * kVectors;  // elements
constexpr int kMaxTensors = 180;                 // of a launch
constexpr int kMaxGroups = 2048;                 // workgroups of a launch, sums that it leaves

struct ClipTable {
  int count;
  uint32_t first[kMaxTensors + 1];  // chunk that each tensor begins with
  uint16_t last[kMaxTensors];       // elements of its last chunk, and in the highest bit whether it is bf16
  const void* in[kMaxTensors];
  void* out[kMaxTensors];
};
static_assert(sizeof(ClipTable) <= 4032, "the table travels as a kernel argument");
static_assert(kChunk < 1 << 15);

// A chunk of a tensor: where it begins and how many elements it has
struct Chunk {
  const char* in;
  char* out;
  int size;
  bool bf16;
};
__device__ __forceinline__ Chunk chunk_of(const ClipTable& table, int k, uint32_t chunk) {
  const bool bf16 = table.last[k] >> 15;
  const int64_t at = (int64_t)(chunk - table.first[k]) * kChunk * (bf16 ? 2 : 4);
  return {static_cast<const char*>(table.in[k]) + at, static_cast<char*>(table.out[k]) + at,
          chunk + 1 < table.first[k + 1] ? kChunk : table.last[k] & 0x7FFF, bf16};
}

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

// element of a chunk that the thread's vector v begins with
__device__ __forceinline__ int element_of(int v) { return (v * kThreads + (int)threadIdx.x) * 8; }

// squares of `size` elements
template <bool BF16>
__device__ __forceinline__ double add_squares(const char* in, int size, double s) {
  float x[kVectors][8];
#pragma unroll
  for (int v = 0; v < kVectors; ++v) {
    if (size == kChunk) {
      Raw8<BF16> raw;
      __builtin_memcpy(raw.w, in + element_of(v) * (BF16 ? 2 : 4), sizeof(raw.w));
      widen8<BF16>(raw, x[v]);
    } else {
      load_row8<BF16>(in, element_of(v), size, x[v]);
    }
  }
#pragma unroll
  for (int v = 0; v < kVectors; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fma((double)x[v][j], (double)x[v][j], s);
  return s;
}

typedef uint32_t uintx4 __attribute__((ext_vector_type(4), aligned(2)));
// `size` elements times factor times `power`, a power of two
template <bool BF16>
__device__ __forceinline__ void scale(const char* in, char* out, int size, float factor, float power) {
  float x[kVectors][8];
#pragma unroll
  for (int v = 0; v < kVectors; ++v) {
    const int at = element_of(v);
    if (size != kChunk) {
      load_row8<BF16>(in, at, size, x[v]);
    } else if constexpr (BF16) {
      const uintx4 w = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(in + at * 2));
#pragma unroll
      for (int k = 0; k < 4; ++k) x[v][2 * k] = __uint_as_float(w[k] << 16), x[v][2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    } else {
      const uintx4 a = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(in + at * 4));
      const uintx4 b = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(in + at * 4 + 16));
#pragma unroll
      for (int k = 0; k < 4; ++k) x[v][k] = __uint_as_float(a[k]), x[v][4 + k] = __uint_as_float(b[k]);
    }
  }
#pragma unroll
  for (int v = 0; v < kVectors; ++v) {
    const int at = element_of(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[v][j] = x[v][j] * factor * power;
    if (size != kChunk) {
      store_row8<BF16>(out, at, size, x[v]);
    } else if constexpr (BF16) {
      const uintx4 w = {pack_bf16(x[v][0], x[v][1]), pack_bf16(x[v][2], x[v][3]), pack_bf16(x[v][4], x[v][5]), pack_bf16(x[v][6], x[v][7])};
      __builtin_nontemporal_store(w, reinterpret_cast<uintx4*>(out + at * 2));
    } else {
      uintx4 a, b;
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] = __float_as_uint(x[v][k]), b[k] = __float_as_uint(x[v][4 + k]);
      __builtin_nontemporal_store(a, reinterpret_cast<uintx4*>(out + at * 4));
      __builtin_nontemporal_store(b, reinterpret_cast<uintx4*>(out + at * 4 + 16));
    }
  }
}

// sum over the workgroup, in all threads
__device__ __forceinline__ double group_sum(double s) {
  __shared__ double part[kThreads / kWave];
  s += lane_xor<1>(s), s += lane_xor<2>(s), s += lane_xor<7>(s), s += lane_xor<15>(s), s += lane_xor<16>(s), s += lane_xor<32>(s);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = s;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

// (the first `begun` sums hold what earlier launches found)
__global__ __launch_bounds__(kThreads) void squares_kernel(ClipTable table, double* sums, unsigned begun) {
  double s = 0.0;
  const uint32_t chunks = table.first[table.count];
  int k = tensor_of(table, blockIdx.x);
  for (uint32_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
    while (table.first[k + 1] <= chunk) ++k;
    const Chunk c = chunk_of(table, k, chunk);
    // (a whole chunk's size is a constant: its loads have no conditions between them)
    if (c.size == kChunk)
      s = c.bf16 ? add_squares<true>(c.in, kChunk, s) : add_squares<false>(c.in, kChunk, s);
    else
      s = c.bf16 ? add_squares<true>(c.in, c.size, s) : add_squares<false>(c.in, c.size, s);
  }
  s = group_sum(s);
  if (threadIdx.x == 0) sums[blockIdx.x] = blockIdx.x < begun ? sums[blockIdx.x] + s : s;
}

__global__ __launch_bounds__(kThreads) void scale_kernel(ClipTable table, const double* sums, int count, double max_norm, float* norm_out) {
  double s = 0.0;
  for (int k = (int)threadIdx.x; k < count; k += kThreads) s += sums[k];
  const double norm = sqrt(group_sum(s));
  // (what is not finite goes by the norm as it is reported)
  const double exact = norm > max_norm && (float)norm < __builtin_inff() ? max_norm / norm : 1.0;
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) norm_out[0] = (float)norm, norm_out[1] = (float)exact;
  // (below 2^-126 a factor has fewer bits than its results: those of gradients of 1e38)
  const bool tiny = exact < 0x1p-126;
  const float factor = (float)(tiny ? exact * 0x1p126 : exact), power = tiny ? 0x1p-126f : 1.0f;
  const uint32_t chunks = table.first[table.count];
  if (blockIdx.x >= chunks) return;
  int k = tensor_of(table, chunks - 1 - blockIdx.x);
  for (uint32_t back = blockIdx.x; back < chunks; back += gridDim.x) {
    const uint32_t chunk = chunks - 1 - back;
    while (table.first[k] > chunk) --k;
    const Chunk c = chunk_of(table, k, chunk);
    if (factor == 1.0f && c.in == c.out) continue;
    if (c.size == kChunk)
      c.bf16 ? scale<true>(c.in, c.out, kChunk, factor, power) : scale<false>(c.in, c.out, kChunk, factor, power);
    else
      c.bf16 ? scale<true>(c.in, c.out, c.size, factor, power) : scale<false>(c.in, c.out, c.size, factor, power);
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
    table.last[i] = (uint16_t)(((g.count - 1) % kChunk + 1) | (g.dtype == TSENOR_BF16 ? 1 << 15 : 0));
    table.in[i] = g.in, table.out[i] = g.out;
    chunks += chunks_of(g.count);
  }
  table.first[table.count] = (uint32_t)chunks;
  return k;
}
inline unsigned groups_of(const ClipTable& table) { return std::min<unsigned>(table.first[table.count], kMaxGroups); }

}  // namespace

extern "C" size_t tsenor_clip_workspace_bytes(const tsenor_clip_problem* p) {
  if (check(p) != TSENOR_OK) return 0;
  // (a sum for each workgroup of the largest launch; 256 bytes where there is none)
  ClipTable table;
  size_t sums = 0;
  for (int k = 0; k < p->count;) {
    k = fill_table(*p, k, table);
    sums = std::max<size_t>(sums, groups_of(table));
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
  unsigned count = 0;
  for (int k = 0; k < p->count;) {
    k = fill_table(*p, k, table);
    const unsigned groups = groups_of(table);
    if (groups == 0) continue;
    squares_kernel<<<groups, kThreads, 0, s>>>(table, sums, count);
    count = std::max(count, groups);
  }
  // norm and factor are written by the first launch of the second pass, which there is also without gradients
  float* norm_out = p->norm_out;
  for (int k = 0; k < p->count || norm_out;) {
    k = fill_table(*p, k, table);
    const unsigned groups = groups_of(table);
    if (groups == 0 && (!norm_out || k < p->count)) continue;
    scale_kernel<<<std::max(groups, 1u), kThreads, 0, s>>>(table, sums, (int)count, p->max_norm, norm_out);
    norm_out = nullptr;
  }
  return status_of_launches();
}
