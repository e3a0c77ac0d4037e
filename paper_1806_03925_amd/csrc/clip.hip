// The global norm of a list of gradients and their clipping by it:
//
//   norm = sqrt(sum over tensors and elements of g^2),  c = min(1, max_norm / (norm + 1e-6)),  out = c g
//
// Two launches, whatever the number of tensors (one for a list of up to four chunks: us of two launches / one, 6273
// gradients in four tensors 6.8 / 4.4, 32768 in one 7.5 / 6.0, but 65536 7.5 / 9.1).  The list lies on the device as one
// entry per tensor; work is cut into chunks of kClipChunk elements that never cross a tensor, and a workgroup finds a
// chunk's tensor by bisection over the entries' first chunks.  The first launch leaves one fp64 sum per workgroup, the
// second adds these up in every workgroup (in the same order, so that all get the same factor) and scales.  Memory bound: all elements
// are read once for the norm, and read and written once more to be scaled, since the factor is not known before; the
// second pass walks its chunks backwards and finds in the cache what the first has read last.  400 M gradients (1.07 GB, bf16 and
// fp32) 681 us, 4.7 TB/s of the 3.2 GB; 704 forwards, 737 with results through the L2, 761 with neighbouring chunks to a workgroup.
#include "gear_internal.hpp"

#include <cmath>

namespace gear {
namespace {

struct GradEntry {
  const void *src;
  void *dst;
  int64_t n;
  int64_t first_chunk;
  int32_t dtype;
  int32_t pad;
};
static_assert(sizeof(GradEntry) == 40, "layout of the device list");

constexpr int kClipThreads = 256;
constexpr int64_t kClipChunk = 16384;    // elements
constexpr int kClipBlocks = 2048;    // workgroups, and partial sums

int clip_blocks(int64_t chunks) { return (int)(chunks < kClipBlocks ? chunks : kClipBlocks); }

// the entry that holds `chunk`: the last one whose first chunk is not beyond it (entries without elements have no chunk
// and share their first chunk with the entry after them)
__device__ __forceinline__ int entry_of(const GradEntry *__restrict__ list, int count, int64_t chunk) {
  int lo = 0, hi = count;   // first_chunk of lo is <= chunk
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (list[mid].first_chunk <= chunk)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kAtOnce = 4;   // pieces of a thread on their way together

// by kClipThreads threads, of which the caller is number t
template <typename T> __device__ __forceinline__ double square_sum(const T *__restrict__ p, int64_t n, int t) {
  constexpr int V = 16 / (int)sizeof(T);
  double sum = 0.0;
  auto add = [&](float v) { sum += (double)v * (double)v; };
  auto add_piece = [&](const u32x4 &w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4) {
        add(__uint_as_float(w[j]));
      } else {
        add(__uint_as_float(w[j] << 16));
        add(__uint_as_float(w[j] & 0xffff0000u));
      }
    }
  };
  // elements before the first 16-byte border, whole pieces, the rest
  const int head = (int)min(n, (int64_t)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T)));
  if (t < head) add(to_f32(p[t]));
  const int pieces = (int)(n - head) / V;
  const u32x4 *v = reinterpret_cast<const u32x4 *>(p + head);
  int i = t;
  for (; i + (kAtOnce - 1) * kClipThreads < pieces; i += kAtOnce * kClipThreads) {
    u32x4 w[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) w[k] = v[i + k * kClipThreads];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) add_piece(w[k]);
  }
  for (; i < pieces; i += kClipThreads) add_piece(v[i]);
  const int at = head + pieces * V + t;
  if (at < n) add(to_f32(p[at]));
  return sum;
}

template <int THREADS> __device__ __forceinline__ double block_sum(double v, double *s_sum) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, kWave);
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x / kWave] = v;
  __syncthreads();
  v = s_sum[0];
#pragma unroll
  for (int w = 1; w < THREADS / kWave; ++w) v += s_sum[w];
  return v;
}

// the sum of the squares of chunk c: a thread's share
__device__ __forceinline__ double chunk_squares(const GradEntry *__restrict__ list, int count, int64_t c, int t) {
  const GradEntry e = list[entry_of(list, count, c)];
  const int64_t first = (c - e.first_chunk) * kClipChunk, n = min(kClipChunk, e.n - first);
  return e.dtype == GEAR_BF16 ? square_sum(static_cast<const bf16_t *>(e.src) + first, n, t)
                              : square_sum(static_cast<const float *>(e.src) + first, n, t);
}

__global__ void __launch_bounds__(kClipThreads) k_grad_squares(const GradEntry *__restrict__ list, int count, int64_t chunks,
                                                               double *__restrict__ partial) {
  __shared__ double s_sum[kClipThreads / kWave];
  double sum = 0.0;
  for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) sum += chunk_squares(list, count, c, threadIdx.x);
  sum = block_sum<kClipThreads>(sum, s_sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <typename T> __device__ __forceinline__ u32x4 scale_piece(u32x4 w, float c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4)
      w[j] = __float_as_uint(__uint_as_float(w[j]) * c);
    else
      w[j] = pack_bf16(__uint_as_float(w[j] << 16) * c, __uint_as_float(w[j] & 0xffff0000u) * c);
  }
  return w;
}

template <typename T> __device__ __forceinline__ void scale_chunk(const T *src, T *dst, int64_t n, float c, int t) {
  constexpr int V = 16 / (int)sizeof(T);
  int head = (int)n;   // element by element where source and destination lie differently to 16 bytes
  if ((((uintptr_t)src ^ (uintptr_t)dst) & 15) == 0) head = (int)min(n, (int64_t)(((16 - ((uintptr_t)src & 15)) & 15) / sizeof(T)));
  for (int i = t; i < head; i += kClipThreads) dst[i] = from_f32<T>(to_f32(src[i]) * c);
  const int pieces = (int)(n - head) / V;
  const u32x4 *v = reinterpret_cast<const u32x4 *>(src + head);
  u32x4 *o = reinterpret_cast<u32x4 *>(dst + head);
  int i = t;
  for (; i + (kAtOnce - 1) * kClipThreads < pieces; i += kAtOnce * kClipThreads) {
    u32x4 w[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) w[k] = v[i + k * kClipThreads];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) __builtin_nontemporal_store(scale_piece<T>(w[k], c), o + i + k * kClipThreads);
  }
  for (; i < pieces; i += kClipThreads) __builtin_nontemporal_store(scale_piece<T>(v[i], c), o + i);
  const int at = head + pieces * V + t;
  if (at < n) dst[at] = from_f32<T>(to_f32(src[at]) * c);
}

// from the norm in fp64: fp32 may not hold that of gradients which are finite
__device__ __forceinline__ float clip_factor(double norm, float max_norm) {
  const double ratio = (double)max_norm / (norm + 1e-6);
  return ratio > 1.0 ? 1.0f : (float)ratio;   // NaN stays NaN
}

__device__ __forceinline__ void chunk_scale(const GradEntry *__restrict__ list, int count, int64_t k, float c, int t) {
  const GradEntry e = list[entry_of(list, count, k)];
  if (!e.dst || (c == 1.0f && e.src == e.dst)) return;
  const int64_t first = (k - e.first_chunk) * kClipChunk, n = min(kClipChunk, e.n - first);
  if (e.dtype == GEAR_BF16)
    scale_chunk(static_cast<const bf16_t *>(e.src) + first, static_cast<bf16_t *>(e.dst) + first, n, c, t);
  else
    scale_chunk(static_cast<const float *>(e.src) + first, static_cast<float *>(e.dst) + first, n, c, t);
}

// scale: 0, only the norm is wanted (one workgroup)
__global__ void __launch_bounds__(kClipThreads) k_grad_scale(const GradEntry *__restrict__ list, int count, int64_t chunks,
                                                             const double *__restrict__ partial, int n_partial, float max_norm,
                                                             int scale, float *__restrict__ norm_out) {
  __shared__ double s_sum[kClipThreads / kWave];
  double sum = 0.0;
  for (int i = threadIdx.x; i < n_partial; i += kClipThreads) sum += partial[i];
  const double norm = sqrt(block_sum<kClipThreads>(sum, s_sum));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  if (!scale) return;
  const float c = clip_factor(norm, max_norm);
  for (int64_t k = chunks - 1 - blockIdx.x; k >= 0; k -= gridDim.x) chunk_scale(list, count, k, c, threadIdx.x);
}

// Short lists, whose time is that of two launches and not of one workgroup's memory accesses: all of it by one
// workgroup, kClipThreads threads to a chunk.  All reads for the sum come before the barrier in block_sum, so gradients may be scaled in place.
constexpr int kShortChunks = 4, kShortThreads = kShortChunks * kClipThreads;
__global__ void __launch_bounds__(kShortThreads) k_grad_short(const GradEntry *__restrict__ list, int count, int chunks, float max_norm,
                                                              int scale, float *__restrict__ norm_out) {
  __shared__ double s_sum[kShortThreads / kWave];
  const int chunk = threadIdx.x / kClipThreads, t = threadIdx.x % kClipThreads;
  const double norm = sqrt(block_sum<kShortThreads>(chunk < chunks ? chunk_squares(list, count, chunk, t) : 0.0, s_sum));
  if (threadIdx.x == 0) *norm_out = (float)norm;
  if (scale && chunk < chunks) chunk_scale(list, count, chunk, clip_factor(norm, max_norm), t);
}

gear_status check(const void *list, int32_t count, int64_t chunks, const void *workspace, size_t bytes, const float *norm) {
  if (!list || count < 1 || chunks < 0 || !workspace || !norm || ((uintptr_t)list & 15) || ((uintptr_t)workspace & 255) ||
      ((uintptr_t)norm & 3))
    return GEAR_ERR_INVALID;
  return bytes < gear_grad_workspace_bytes(chunks) ? GEAR_ERR_CAPACITY : GEAR_OK;
}

gear_status run(const void *list, int32_t count, int64_t chunks, float max_norm, int scale, void *workspace, float *norm,
                hipStream_t s) {
  const GradEntry *entries = static_cast<const GradEntry *>(list);
  double *partial = static_cast<double *>(workspace);
  const int blocks = clip_blocks(chunks);
  if (chunks <= kShortChunks) {
    hipLaunchKernelGGL(k_grad_short, dim3(1), dim3(kShortThreads), 0, s, entries, count, (int)chunks, max_norm, scale, norm);
    return hipGetLastError() == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
  }
  hipLaunchKernelGGL(k_grad_squares, dim3(blocks), dim3(kClipThreads), 0, s, entries, count, chunks, partial);
  if (hipGetLastError() != hipSuccess) return GEAR_ERR_HIP;
  hipLaunchKernelGGL(k_grad_scale, dim3(scale ? blocks : 1), dim3(kClipThreads), 0, s, entries, count, chunks,
                     partial, blocks, max_norm, scale, norm);
  return hipGetLastError() == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

}  // namespace
}  // namespace gear

using namespace gear;

extern "C" size_t gear_grad_list_bytes(int32_t count) { return count > 0 ? (size_t)count * sizeof(GradEntry) : 0; }

extern "C" gear_status gear_grad_list_pack(const gear_grad_tensor *tensors, int32_t count, void *host_list, int64_t *chunks) {
  if (!tensors || count < 1 || !host_list || !chunks) return GEAR_ERR_INVALID;
  for (int32_t i = 0; i < count; ++i) {
    const gear_grad_tensor &t = tensors[i];
    if (t.n < 0 || t.n > ((int64_t)1 << 40) || (t.dtype != GEAR_F32 && t.dtype != GEAR_BF16)) return GEAR_ERR_INVALID;
    const uintptr_t to = dtype_bytes(t.dtype) - 1;
    if ((t.n > 0 && !t.src) || ((uintptr_t)t.src & to) || ((uintptr_t)t.dst & to)) return GEAR_ERR_INVALID;
  }
  GradEntry *e = static_cast<GradEntry *>(host_list);
  int64_t at = 0;
  for (int32_t i = 0; i < count; ++i) {
    const gear_grad_tensor &t = tensors[i];
    e[i] = GradEntry{t.src, t.dst, t.n, at, t.dtype, 0};
    at += (t.n + kClipChunk - 1) / kClipChunk;
  }
  *chunks = at;
  return GEAR_OK;
}

extern "C" size_t gear_grad_workspace_bytes(int64_t chunks) { return chunks < 0 ? 0 : (size_t)kClipBlocks * sizeof(double); }

extern "C" gear_status gear_grad_norm(const void *list, int32_t count, int64_t chunks, void *workspace, size_t workspace_bytes,
                                      float *norm, void *stream) {
  const gear_status ok = check(list, count, chunks, workspace, workspace_bytes, norm);
  return ok != GEAR_OK ? ok : run(list, count, chunks, 0.0f, 0, workspace, norm, (hipStream_t)stream);
}

extern "C" gear_status gear_clip_grads(const void *list, int32_t count, int64_t chunks, float max_norm, void *workspace,
                                       size_t workspace_bytes, float *norm, void *stream) {
  if (!(max_norm > 0.0f) || !std::isfinite(max_norm)) return GEAR_ERR_INVALID;
  const gear_status ok = check(list, count, chunks, workspace, workspace_bytes, norm);
  return ok != GEAR_OK ? ok : run(list, count, chunks, max_norm, 1, workspace, norm, (hipStream_t)stream);
}
