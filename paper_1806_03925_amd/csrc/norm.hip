// Root-mean-square norm of rows of features with the residual's addition, its output in 8 bits, and its backward pass:
//
//   h = x + residual,  s = (mean(h^2) + eps)^-1/2,  y = h s gain
//   a = dy gain,  u = h s,  dx = s (a - u s mean(a h)) + dsum,  dgain = sum over rows of dy u
//
// (dx: y_c depends on h_c directly, s a, and on all of h through s, whose derivative by h_c is -s^3 h_c / dim.  The cube of s
// leaves fp32's range where h is 1e13 or 1e-13 and is never formed.)
// Every call is one pass over its rows: a row stays in the registers of the threads that read it, from the sum of its
// squares to the last output, so what bounds these kernels is the memory they have to read and write (the norm in 8 bits: fp64,
// see there).  That holds up to 8192 columns (but for two registers of a bf16 row in 8 bits).  Wider rows are 1024 threads', which have 128
// registers each and keep part of a row in scratch memory; registers spilled up to 32768 columns / beyond, and TB/s of the bytes that a call
// has to move at 4096 x 16384 / 1024 x 65536:
//   backward bf16 45 / 265, 2.8 / 1.0; fp32 79 / 442, 3.6 / 1.5 (5.0 and 4.7 at 4096 x 8192)
//   8 bits   bf16 none / 36, 3.9 / 2.6; fp32 6 / 145, 4.7 / 2.3 (5.3 and 5.1)
//   norm     bf16 none, 6.7 / 5.8; fp32 none / 41, 4.2 / 3.7 (6.7 and 5.7)
#include "eight.hpp"

#include <cmath>
#include <type_traits>

namespace gear {
namespace {

// A row belongs to TPR threads with PER pieces of eight values each, piece i of thread t at columns 8 (t + TPR i): a
// wavefront's accesses are contiguous, and 16 neighbouring threads hold a block of 128 columns.
//
// KIND: what is made of a row, the norm itself, the norm in 8 bits, or the row in 8 bits.  The 8 bits of the norm are rounded once,
// from fp64: its fp32 value depends in the last bits on how the row was added up, and next to a tie they decide a whole step of the
// 8 bits, 2^-4 of the value.  10001 x 1152 bf16 with residual into sum, y and 8 bits: 21.7 us, the same reads and writes from fp32
// 18.9 us (5.4 TB/s): what is over is the arithmetic in fp64.  (h itself is fp32 where x is bf16: exact, unless one of both is 2^16
// times the other, and off by 2^-24 then.  With that sum in fp64, too, 20000 x 1152 without residual took 38.9 us for 34.3.)
enum NormKind { kNorm, kNorm8, kRows8 };

// Wavefronts a SIMD that the compiler has to leave room for, which takes fp64 pieces apart again rather than keeping them: 4, us without:
// 10001 x 1152 bf16 24.4 / 23.5, 15198 x 7664 158 / 140.  Not where pieces are 32 fp32 values: 20000 x 1152 86 with it, 72 without.
constexpr int simd_waves(NormKind kind, int tpr, int per, int size) { return kind == kNorm8 && tpr <= 256 && (per < 4 || size == 2) ? 4 : 1; }

template <typename T, int TPR, int PER, NormKind KIND>
__global__ void __launch_bounds__(TPR <= kWave ? 256 : TPR, simd_waves(KIND, TPR, PER, sizeof(T))) k_rmsnorm(gear_norm_args a) {
  using V = typename std::conditional<KIND == kNorm8, double, float>::type;
  constexpr int THREADS = TPR <= kWave ? 256 : TPR, ROWS = THREADS / TPR;
  __shared__ V s_part[TPR > kWave ? TPR / kWave : 1];
  const int t = threadIdx.x % TPR;
  // one pass for all but lists of more rows than a launch may have threads for
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; row < a.rows; row += (int64_t)gridDim.x * ROWS) {
    const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
    const T *res = KIND != kRows8 && a.residual ? static_cast<const T *>(a.residual) + row * a.ld_residual : nullptr;
    Raw8<T> xs[PER], rs[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = 8 * (t + TPR * i);
      xs[i].zero(), rs[i].zero();
      if (c < a.dim) {
        xs[i].load(x + c);
        if (res) rs[i].load(res + c);
      }
    }
    auto piece = [&](int i, V (&h)[8]) {
      float v[8], r[8];
      xs[i].get(v);
      rs[i].get(r);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = KIND == kRows8 ? (V)v[j] : sizeof(T) == 2 ? (V)(v[j] + r[j]) : (V)v[j] + (V)r[j];
    };
    V s = 1;
    if constexpr (KIND != kRows8) {
      V sq = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (i > 0 && 8 * TPR * i >= a.dim) break;
        V h[8];
        piece(i, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) sq += h[j] * h[j];
      }
      s = (V)1 / sqrt(row_sum<TPR>(sq, s_part) / (V)a.dim + (V)a.eps);
    }
    const int64_t ld8 = rows8_ld(a.dim), lds = scales8_ld(a.dim);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = 8 * (t + TPR * i);
      if (i > 0 && 8 * TPR * i >= a.dim) break;
      V h[8];
      float y[8];
      piece(i, h);
      if (KIND != kRows8 && c < a.dim) {
        float g[8];
        load8(a.gain + c, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (KIND == kNorm8)
            y[j] = round_odd(h[j] * s * (V)g[j]);
          else
            y[j] = h[j] * s * g[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = (float)h[j];
      }
      if constexpr (KIND != kNorm) {
        float top = top8(y);
#pragma unroll
        for (int o = 8; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
        const int e = exponent8(top);
        const uint2 q = pack8(y, unscale8(e));
        if (c < ld8) {
          *reinterpret_cast<uint2 *>(a.q8 + row * ld8 + c) = q;
          if (t % 16 == 0) a.scale[row * lds + c / kBlock8] = (uint8_t)(e + 127);
        }
        if constexpr (KIND == kNorm8) unpack8(q, scale8(e), y);
      }
      if (KIND == kRows8 || c >= a.dim) continue;
      if (a.sum) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)h[j];
        stream8(static_cast<T *>(a.sum) + row * a.ld_sum + c, v);
      }
      if (a.y) stream8(static_cast<T *>(a.y) + row * a.ld_y + c, y);
    }
    if (KIND != kNorm && t < lds - ld8 / kBlock8) a.scale[row * lds + ld8 / kBlock8 + t] = 0;   // behind the last block: not used
  }
}

// Backward pass.  A workgroup takes rows blockIdx.x * ROWS + threadIdx.x / TPR + k gridDim.x * ROWS and keeps its share of
// dgain in registers; what its rows sum to becomes one row of `partial`, added up by k_sum_rows in a fixed order.
template <typename T, int TPR, int PER>
__global__ void __launch_bounds__(TPR <= kWave ? 256 : TPR) k_rmsnorm_backward(gear_norm_backward_args a, float *__restrict__ partial) {
  constexpr int THREADS = TPR <= kWave ? 256 : TPR, ROWS = THREADS / TPR;
  __shared__ float s_part[TPR > kWave ? TPR / kWave : 1];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float dg[PER][8];
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = 0.0f;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + sub; row < a.rows; row += (int64_t)gridDim.x * ROWS) {
    const T *hp = static_cast<const T *>(a.h) + row * a.ld_h, *dyp = static_cast<const T *>(a.dy) + row * a.ld_dy;
    Raw8<T> h[PER], d[PER], more[PER];   // all of them on their way before the first sum
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = 8 * (t + TPR * i);
      h[i].zero(), d[i].zero(), more[i].zero();
      if (c < a.dim) {
        h[i].load(hp + c);
        d[i].load(dyp + c);
        if (a.dsum) more[i].load(static_cast<const T *>(a.dsum) + row * a.ld_dsum + c);
      }
    }
    float sq = 0.0f, dot = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = 8 * (t + TPR * i);
      if (c >= a.dim) continue;
      float g[8], hv[8], dv[8];
      load8(a.gain + c, g);
      h[i].get(hv);
      d[i].get(dv);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sq += hv[j] * hv[j];
        dot += dv[j] * g[j] * hv[j];
      }
    }
    sq = row_sum<TPR>(sq, s_part);
    dot = row_sum<TPR>(dot, s_part);
    const float s = 1.0f / sqrtf(sq / (float)a.dim + a.eps);
    const float along = s * (dot / (float)a.dim);   // mean(a u)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = 8 * (t + TPR * i);
      if (c >= a.dim) continue;
      float g[8], hv[8], dv[8], dx[8];
      load8(a.gain + c, g);
      h[i].get(hv);
      d[i].get(dv);
      more[i].get(dx);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = hv[j] * s;
        dx[j] = s * (dv[j] * g[j] - u * along) + dx[j];
        dg[i][j] += dv[j] * u;
      }
      stream8(static_cast<T *>(a.dx) + row * a.ld_dx + c, dx);
    }
  }
  if (!partial) return;
  if constexpr (ROWS > 1) {   // the wavefronts' shares, in ascending order
    __shared__ float s_dg[(ROWS - 1) * PER * 8 * TPR];
    if (sub > 0)
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s_dg[(((sub - 1) * PER + i) * 8 + j) * TPR + t] = dg[i][j];
    __syncthreads();
    if (sub > 0) return;
    for (int w = 0; w < ROWS - 1; ++w)
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[i][j] += s_dg[((w * PER + i) * 8 + j) * TPR + t];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = 8 * (t + TPR * i);
    if (c < a.dim) store8(partial + (size_t)blockIdx.x * a.dim + c, dg[i]);
  }
}

// out[c] = sum of partial[r][c], r < n, always in the same order.  A workgroup takes 32 columns, eight threads of four a row, 128
// rows at a time: few workgroups, so each has to have many rows on their way.  us of the whole backward pass of 16384 x 1024 bf16 (768 rows
// here) with 64 / 32 / 16 columns: 28.2 / 27.4 / 27.5; this launch with one column of a row to a thread, 16 rows at a time, 20 for 4.
constexpr int kSumCols = 32;
__global__ void __launch_bounds__(1024) k_sum_rows(const float *__restrict__ partial, int n, int dim, float *__restrict__ out) {
  constexpr int COLS = kSumCols, T = COLS / 4, ROWS = 1024 / T, PARTS = 1024 / COLS, EACH = ROWS / PARTS;   // threads to a row, rows at a time
  __shared__ __attribute__((aligned(16))) float s[ROWS][COLS];
  const int c = blockIdx.x * COLS + (threadIdx.x % T) * 4, r0 = threadIdx.x / T;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (c < dim) {
#pragma unroll 4
    for (int r = r0; r < n; r += ROWS) {
      const float4 p = *reinterpret_cast<const float4 *>(partial + (size_t)r * dim + c);
      v.x += p.x, v.y += p.y, v.z += p.z, v.w += p.w;
    }
  }
  *reinterpret_cast<float4 *>(&s[r0][(threadIdx.x % T) * 4]) = v;
  __syncthreads();
  const int col = threadIdx.x % COLS, q = threadIdx.x / COLS;
  float sum = 0.0f;
#pragma unroll
  for (int r = 0; r < EACH; ++r) sum += s[q * EACH + r][col];
  __syncthreads();
  s[q][col] = sum;
  __syncthreads();
  if (q == 0 && blockIdx.x * COLS + col < dim) {
#pragma unroll
    for (int r = 1; r < PARTS; ++r) sum += s[r][col];
    out[blockIdx.x * COLS + col] = sum;
  }
}

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool row_distance(int64_t ld, int64_t width) { return ld >= width && ld % 8 == 0 && ld < (1 << 20); }
bool matrix_ok(const void *p, int64_t ld, int64_t width) { return aligned(p, 16) && row_distance(ld, width); }
bool shape_ok(int64_t rows, int32_t dim, int32_t dtype) {
  return rows >= 0 && rows <= (1 << 30) && dim >= 8 && dim % 8 == 0 && dim <= GEAR_MAX_NORM_DIM &&
         (dtype == GEAR_F32 || dtype == GEAR_BF16);
}

// Threads of a row: a quarter or half of a wavefront for rows that a whole one would not fill (42115 x 144 fp32 backward 35.5 / 22.9 us), a
// wavefront up to 2048 columns, as many as hold the row in at most 32 values each beyond.  (bf16 in 8 bits up to 4096 with half as many, whose
// arithmetic is what counts: a wavefront computes whole pieces of 512 columns.  32126 x 2176 142 / 104, but fp32 10000 x 4096 126 / 131.)
template <typename T, NormKind KIND> hipError_t launch_norm(const gear_norm_args &a, hipStream_t s) {
  constexpr int64_t kMost = 1 << 21;   // workgroups: threads are counted in 32 bits
#define GEAR_NORM(TPR, PER)                                                                                            \
  do {                                                                                                                 \
    const int64_t blocks = TPR <= kWave ? (a.rows * TPR + 255) / 256 : a.rows;                                         \
    hipLaunchKernelGGL((k_rmsnorm<T, TPR, PER, KIND>), dim3((unsigned)(blocks < kMost ? blocks : kMost)),              \
                       dim3(TPR <= kWave ? 256 : TPR), 0, s, a);                                                       \
  } while (0)
  if (a.dim <= 128)
    GEAR_NORM(16, 1);
  else if (a.dim <= 256)
    GEAR_NORM(32, 1);
  else if (a.dim <= 512)
    GEAR_NORM(64, 1);
  else if (a.dim <= 1024)
    GEAR_NORM(64, 2);
  else if (a.dim <= 2048)
    GEAR_NORM(64, 4);
  else if (a.dim <= 4096) {
    if constexpr (KIND == kNorm8 && sizeof(T) == 2)
      GEAR_NORM(128, 4);
    else
      GEAR_NORM(256, 2);
  } else if (a.dim <= 8192)
    GEAR_NORM(256, 4);
  else if (a.dim <= 32768)
    GEAR_NORM(1024, 4);
  else
    GEAR_NORM(1024, 8);
#undef GEAR_NORM
  return hipGetLastError();
}

// Workgroups of the backward pass: rows are shared out to them, each leaves one row of partial sums.  768 in bf16 and 512 in fp32, which are
// those that are on the device at once for 1025 to 2048 and 4097 to 8192 columns, three and two for each CU (registers; others leave room for
// four and more, wider rows for one): us of 512 / 768 / 1024 for 65536 x 2048 bf16 178 / 160 / 197, 8192 x 8192 91 / 84 / 103, 16384 x 4096
// 93 / 80 / 81, 30000 x 1024 38 / 35 / 35, but 65536 x 512 46 / 41 / 37; fp32 65536 x 2048 309 / 347 / 308, 8192 x 8192 169 / 190 / 173, 16384 x
// 4096 160 / 156 / 162, 65536 x 512 67 / 70 / 70, but 100000 x 264 76 / 59 / 54: narrow rows could do with more of them.
// Few rows are one workgroup's, which leaves dgain itself: two launches / one, from Python, 32 x 512 bf16 (8 rounds of rows) 12.7 / 10.2, 16 x
// 1152 (4) 12.8 / 9.8, but 32 x 1152 (8) 12.9 / 15.4.
int back_blocks(int64_t rows, int32_t dim, int32_t dtype) {
  const int at_once = dim <= 128 ? 16 : dim <= 256 ? 8 : dim <= 2048 ? 4 : 1;   // rows of a workgroup
  const int64_t groups = (rows + at_once - 1) / at_once, most = dtype == GEAR_BF16 ? 768 : 512;
  if (groups <= (dim <= 512 ? 8 : 4)) return 1;
  return (int)(groups < most ? groups : most);
}

template <typename T> hipError_t launch_back(const gear_norm_backward_args &a, float *partial, hipStream_t s) {
  const dim3 grid(back_blocks(a.rows, a.dim, a.dtype));
#define GEAR_BACK(TPR, PER) \
  hipLaunchKernelGGL((k_rmsnorm_backward<T, TPR, PER>), grid, dim3(TPR <= kWave ? 256 : TPR), 0, s, a, partial)
  if (a.dim <= 128)
    GEAR_BACK(16, 1);
  else if (a.dim <= 256)
    GEAR_BACK(32, 1);
  else if (a.dim <= 512)
    GEAR_BACK(64, 1);
  else if (a.dim <= 1024)
    GEAR_BACK(64, 2);
  else if (a.dim <= 2048)
    GEAR_BACK(64, 4);
  else if (a.dim <= 4096)
    GEAR_BACK(256, 2);
  else if (a.dim <= 8192)
    GEAR_BACK(256, 4);
  else if (a.dim <= 32768)
    GEAR_BACK(1024, 4);
  else
    GEAR_BACK(1024, 8);
#undef GEAR_BACK
  return hipGetLastError();
}

}  // namespace
}  // namespace gear

using namespace gear;

extern "C" int64_t gear_rows8_ld(int32_t dim) { return dim > 0 ? rows8_ld(dim) : 0; }
extern "C" int64_t gear_scales8_ld(int32_t dim) { return dim > 0 ? scales8_ld(dim) : 0; }

extern "C" gear_status gear_rmsnorm(const gear_norm_args *a, void *stream) {
  if (!a || !shape_ok(a->rows, a->dim, a->dtype) || !(a->eps >= 0.0f) || !std::isfinite(a->eps)) return GEAR_ERR_INVALID;
  if (a->rows == 0) return GEAR_OK;
  if (!a->sum && !a->y && !a->q8) return GEAR_ERR_INVALID;
  if (!a->q8 != !a->scale) return GEAR_ERR_INVALID;
  if (!a->x || !a->gain || !aligned(a->gain, 16) || !matrix_ok(a->x, a->ld_x, a->dim)) return GEAR_ERR_INVALID;
  if (a->residual && !matrix_ok(a->residual, a->ld_residual, a->dim)) return GEAR_ERR_INVALID;
  if ((a->sum && !matrix_ok(a->sum, a->ld_sum, a->dim)) || (a->y && !matrix_ok(a->y, a->ld_y, a->dim))) return GEAR_ERR_INVALID;
  if (a->sum && a->sum == a->y) return GEAR_ERR_INVALID;
  if (!aligned(a->q8, 16) || !aligned(a->scale, 4)) return GEAR_ERR_INVALID;
  hipStream_t s = (hipStream_t)stream;
  const bool bf16 = a->dtype == GEAR_BF16;
  const hipError_t err = a->q8 ? bf16 ? launch_norm<bf16_t, kNorm8>(*a, s) : launch_norm<float, kNorm8>(*a, s)
                               : bf16 ? launch_norm<bf16_t, kNorm>(*a, s) : launch_norm<float, kNorm>(*a, s);
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

extern "C" gear_status gear_rows8(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t dim, uint8_t *q8,
                                  uint8_t *scale, void *stream) {
  if (!shape_ok(rows, dim, dtype)) return GEAR_ERR_INVALID;
  if (rows == 0) return GEAR_OK;
  if (!x || !q8 || !scale || !matrix_ok(x, ld_x, dim) || !aligned(q8, 16) || !aligned(scale, 4)) return GEAR_ERR_INVALID;
  gear_norm_args a = {};
  a.rows = rows, a.dim = dim, a.dtype = dtype, a.x = x, a.ld_x = ld_x, a.q8 = q8, a.scale = scale;
  hipStream_t s = (hipStream_t)stream;
  const hipError_t err = dtype == GEAR_BF16 ? launch_norm<bf16_t, kRows8>(a, s) : launch_norm<float, kRows8>(a, s);
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

extern "C" size_t gear_norm_backward_workspace_bytes(int64_t rows, int32_t dim) {
  if (!shape_ok(rows, dim, GEAR_F32)) return 0;
  const size_t bytes = (size_t)back_blocks(rows, dim, GEAR_BF16) * dim * sizeof(float);
  return bytes < 256 ? 256 : (bytes + 255) & ~(size_t)255;
}

extern "C" gear_status gear_rmsnorm_backward(const gear_norm_backward_args *a, void *workspace, size_t workspace_bytes,
                                             void *stream) {
  if (!a || !shape_ok(a->rows, a->dim, a->dtype) || !(a->eps >= 0.0f) || !std::isfinite(a->eps)) return GEAR_ERR_INVALID;
  if (!aligned(a->dgain, 16)) return GEAR_ERR_INVALID;
  hipStream_t s = (hipStream_t)stream;
  if (a->rows == 0) {
    if (a->dgain && launch_fill_zero(a->dgain, (size_t)a->dim * sizeof(float), s) != hipSuccess) return GEAR_ERR_HIP;
    return GEAR_OK;
  }
  if (!a->h || !a->dy || !a->gain || !a->dx || !aligned(a->gain, 16)) return GEAR_ERR_INVALID;
  if (!matrix_ok(a->h, a->ld_h, a->dim) || !matrix_ok(a->dy, a->ld_dy, a->dim) || !matrix_ok(a->dx, a->ld_dx, a->dim))
    return GEAR_ERR_INVALID;
  if (a->dsum && !matrix_ok(a->dsum, a->ld_dsum, a->dim)) return GEAR_ERR_INVALID;
  float *partial = nullptr;
  if (a->dgain) {
    if (!workspace || !aligned(workspace, 256)) return GEAR_ERR_INVALID;
    if (workspace_bytes < gear_norm_backward_workspace_bytes(a->rows, a->dim)) return GEAR_ERR_CAPACITY;
    partial = static_cast<float *>(workspace);
  }
  const bool alone = a->dgain && back_blocks(a->rows, a->dim, a->dtype) == 1;   // one workgroup's share is the sum
  if (alone) partial = a->dgain;
  const hipError_t err = a->dtype == GEAR_BF16 ? launch_back<bf16_t>(*a, partial, s) : launch_back<float>(*a, partial, s);
  if (err != hipSuccess) return GEAR_ERR_HIP;
  if (a->dgain && !alone) {
    hipLaunchKernelGGL(k_sum_rows, dim3((a->dim + kSumCols - 1) / kSumCols), dim3(1024), 0, s, partial, back_blocks(a->rows, a->dim, a->dtype), a->dim, a->dgain);
    if (hipGetLastError() != hipSuccess) return GEAR_ERR_HIP;
  }
  return GEAR_OK;
}
