// Rows on their way to experts and back (gear.h), in their own type or in 8-bit integers, and the gradients of both:
//
//   xs[place[r, j]] = x[r],   out[r] = residual[r] + sum_j w[r, j] y[place[r, j]]
//   dy[place[r, j]] = w[r, j] dout[r],   dw[r, j] = dout[r] . y[place[r, j]]
//
// Every one is a walk over the rows r, not over the places: what a row's k places share is read once, and what they add up to
// stays in registers.  Bound by memory; us and TB/s of what they have to move, bf16, 16384 x 1152 with k = 2 / 65536 x 2048 with k = 4 (a large copy: 4.75):
//   gather 21.0, 5.4 / 226, 5.9;  combine 28.4, 5.3 / 306, 5.3;  its gradients 32.2, 5.9 / 470, 5.1
//   combine of y in fp32 33.0, 6.9 and 491, 5.5 (y is half in the caches where it is small);
//   rows to integers 65536 x 4096 134, 6.0;  to four experts each 16384 x 1152 22.5, 5.0
// Sums and gradients leave past the L2, which then keeps more of what is read (us past it / through it: combine 26.9 / 29.7 and 280 / 328, its
// gradients 31.5 / 35.9 and 470 / 461); copies do not (250 / 228), and the next product reads them.
#include "eight.hpp"

#include <type_traits>

namespace gear {
namespace {

// the place of a pair, -1 where it has none within [0, places)
__device__ __forceinline__ int64_t place_of(const int32_t *__restrict__ place, int64_t pair, int64_t places) {
  const int p = place[pair];
  return p >= 0 && p < places ? p : -1;
}

// ---- one thread for eight values of a row -------------------------------------------------------------------------------
// Threads are numbered through all rows, so that no row's width leaves any of them idle (combine, 1152 columns: 28.4 us; a row by 256 threads 34.9).
constexpr int kPieceThreads = 256;
struct Piece {
  int64_t row;
  int c;
};
// the one of this thread in chunk number `chunk` of kPieceThreads pieces; row >= rows behind the last
__device__ __forceinline__ Piece piece_of(int64_t chunk, int pieces, float one_over) {
  const int64_t at = chunk * kPieceThreads, row0 = at / pieces;             // the same in all lanes
  const int local = (int)(at - row0 * pieces) + (int)threadIdx.x;          // below 2^13 + 2^8: the quotient below is exact
  const int down = (int)(((float)local + 0.5f) * one_over);
  return {row0 + down, 8 * (local - down * pieces)};
}

struct GatherArgs {
  int64_t rows, ld_x, ld_xs;
  int dim, k;
  float one_over;           // the row's pieces
  int64_t chunks;
  const void *x;
  const int32_t *place;
  void *xs;
};
template <typename T> __global__ void __launch_bounds__(kPieceThreads) k_gather(GatherArgs a) {
  for (int64_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const Piece t = piece_of(chunk, a.dim / 8, a.one_over);
    if (t.row >= a.rows) continue;
    constexpr int PIECES = 8 * (int)sizeof(T) / 16;
    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const T *>(a.x) + t.row * a.ld_x + t.c);
    const uint4 lo = src[0], hi = src[PIECES - 1];
    for (int j0 = 0; j0 < a.k; j0 += 4) {
      int64_t p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = j0 + j < a.k ? place_of(a.place, t.row * a.k + j0 + j, a.rows * a.k) : -1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (p[j] < 0) continue;
        uint4 *dst = reinterpret_cast<uint4 *>(static_cast<T *>(a.xs) + p[j] * a.ld_xs + t.c);
        dst[0] = lo;
        if constexpr (PIECES > 1) dst[1] = hi;
      }
    }
  }
}

struct CombineArgs {
  gear_expert_combine_args a;
  float one_over;
  int64_t chunks;
};
template <typename T, typename Y> __global__ void __launch_bounds__(kPieceThreads) k_combine(CombineArgs args) {   // Y: y's type
  const gear_expert_combine_args &a = args.a;
  for (int64_t chunk = blockIdx.x; chunk < args.chunks; chunk += gridDim.x) {
    const Piece t = piece_of(chunk, a.dim / 8, args.one_over);
    if (t.row >= a.rows) continue;
    Raw8<T> res;
    res.zero();
    if (a.residual) res.load(static_cast<const T *>(a.residual) + t.row * a.ld_residual + t.c);
    float sum[8];
    for (int j0 = 0; j0 < a.k; j0 += 4) {   // four places on their way at a time
      int64_t p[4];
      float w[4];
      Raw8<Y> y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t pair = t.row * a.k + j0 + j;
        const bool in = j0 + j < a.k;
        p[j] = in ? place_of(a.place, pair, a.rows * a.k) : -1;
        w[j] = !in ? 0.0f : a.weight ? a.weight[pair] : 1.0f;
        if (p[j] < 0 && w[j] == w[j]) w[j] = 0.0f;          // not an infinity times the zeros of no place; a NaN stays
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[j].zero();
        if (p[j] >= 0) y[j].load(static_cast<const Y *>(a.y) + p[j] * a.ld_y + t.c);
      }
      if (j0 == 0) res.get(sum);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v[8];
        y[j].get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = fmaf(w[j], v[i], sum[i]);
      }
    }
    stream8(static_cast<T *>(a.out) + t.row * a.ld_out + t.c, sum);
  }
}

// ---- one team for a row -----------------------------------------------------------------------------------------------
// A row belongs to TPR threads, with PER pieces of eight values each in registers: piece i of thread t at columns 8 (t + TPR i).
template <int TPR> struct Team {
  static constexpr int THREADS = TPR <= kWave ? 256 : TPR, ROWS = THREADS / TPR;
};

// dout stays in registers while the row's places go by, two at a time.
template <typename T, int TPR, int PER> __global__ void __launch_bounds__(Team<TPR>::THREADS) k_combine_back(gear_expert_combine_backward_args a) {
  __shared__ float s_part[TPR > kWave ? TPR / kWave : 1];
  constexpr int AHEAD = PER * sizeof(T) <= 8 ? 2 : 1;
  const int t = threadIdx.x % TPR;
  for (int64_t row0 = (int64_t)blockIdx.x * Team<TPR>::ROWS; row0 < a.rows; row0 += (int64_t)gridDim.x * Team<TPR>::ROWS) {
    const int64_t row = row0 + threadIdx.x / TPR;
    if (TPR <= kWave && row >= a.rows) continue;
    Raw8<T> d[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = 8 * (t + TPR * i);
      d[i].zero();
      if (c < a.dim) d[i].load(static_cast<const T *>(a.dout) + row * a.ld_dout + c);
    }
    for (int j0 = 0; j0 < a.k; j0 += AHEAD) {
      int64_t p[AHEAD];
      float w[AHEAD];
      Raw8<T> y[AHEAD][PER];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int64_t pair = row * a.k + j0 + j;
        const bool in = j0 + j < a.k;
        p[j] = in ? place_of(a.place, pair, a.rows * a.k) : -1;
        w[j] = in ? a.weight[pair] : 0.0f;
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int c = 8 * (t + TPR * i);
          y[j][i].zero();
          if (a.dweight && p[j] >= 0 && c < a.dim) y[j][i].load(static_cast<const T *>(a.y) + p[j] * a.ld_y + c);
        }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int c = 8 * (t + TPR * i);
          float dv[8], yv[8];
          d[i].get(dv);
          y[j][i].get(yv);
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = fmaf(dv[e], yv[e], dot);
          if (a.dy && p[j] >= 0 && c < a.dim) {
#pragma unroll
            for (int e = 0; e < 8; ++e) dv[e] *= w[j];
            stream8(static_cast<T *>(a.dy) + p[j] * a.ld_dy + c, dv);
          }
        }
        if (a.dweight) {
          dot = row_sum<TPR>(dot, s_part);
          if (t == 0 && j0 + j < a.k) a.dweight[row * a.k + j0 + j] = p[j] >= 0 ? dot : 0.0f;   // not 0 * NaN where there is no place
        }
      }
    }
  }
}

// ---- 8-bit integers -----------------------------------------------------------------------------------------------
// the integer nearest to 127 v / top, ties to even: the quotient in fp64 is never on the wrong side of a tie, as 127 v has at most 31 bits
// and top 24
__device__ __forceinline__ int nearest127(float v, float top) { return top > 0.0f ? (int)rint(127.0 * (double)v / (double)top) : 0; }

// the largest magnitude's bits: those of infinities and NaN are larger than all others'
__device__ __forceinline__ uint32_t top_bits(const float (&v)[8], uint32_t top) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  return top;
}
constexpr uint32_t kInfinite = 0x7f800000u;
__device__ __forceinline__ float scale127(uint32_t top) {   // of a row, from the bits of its largest magnitude
  return top >= kInfinite ? NAN : (float)((double)__uint_as_float(top) / 127.0);
}

// How a row's values become integers (65536 x 4096 bf16: 134 us; every quotient in fp64 270): v * factor in fp32, off by less than 127 2^-23, decides where that is not within kTie of a tie; else, or
// where the factor is no ordinary number, the quotient in fp64 does.
constexpr float kTie = 0x1p-15f;
struct Quantise {
  float top, factor;
  bool always;            // in fp64
};
__device__ __forceinline__ Quantise quantise_of(uint32_t top) {
  const float t = top >= kInfinite ? 0.0f : __uint_as_float(top);
  const bool small = t < 0x1p-100f;
  return {t, small ? 0.0f : 127.0f / t, small && t > 0.0f};
}
__device__ __forceinline__ uint2 pack_i8(const float (&v)[8], const Quantise &q) {
  constexpr float kWhole = 12582912.0f;   // 1.5 2^23: a sum with it is rounded to a whole number, whose last byte is the integer
  uint32_t m[8];
  float off = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float s = fmaf(v[i], q.factor, kWhole);
    m[i] = __float_as_uint(s);
    off = fmaxf(off, fabsf(fmaf(v[i], q.factor, kWhole - s)));
  }
  if (q.always || !(off < 0.5f - kTie)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = (uint32_t)nearest127(v[i], q.top);
  }
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {   // the last bytes of four words
    const uint32_t lo = __builtin_amdgcn_perm(m[4 * h + 1], m[4 * h], 0x0c0c0400u), hi = __builtin_amdgcn_perm(m[4 * h + 3], m[4 * h + 2], 0x0c0c0400u);
    w[h] = lo | hi << 16;
  }
  return make_uint2(w[0], w[1]);
}

template <int TPR> __device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *s_part) {
#pragma unroll
  for (int o = (TPR < kWave ? TPR : kWave) / 2; o; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, kWave));
  if constexpr (TPR > kWave) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x / kWave] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < TPR / kWave; ++w) v = max(v, s_part[w]);
  }
  return v;
}

struct RowsI8Args {
  int64_t rows, ld_x;
  int dim, k;
  const void *x;
  const int32_t *place;   // may be NULL: row r goes to r
  int8_t *q;
  float *scale;
};
template <typename T, int TPR, int PER> __global__ void __launch_bounds__(Team<TPR>::THREADS) k_rows_i8(RowsI8Args a) {
  __shared__ uint32_t s_part[TPR > kWave ? TPR / kWave : 1];
  const int t = threadIdx.x % TPR;
  const int64_t ld = rows8_ld(a.dim);
  for (int64_t row0 = (int64_t)blockIdx.x * Team<TPR>::ROWS; row0 < a.rows; row0 += (int64_t)gridDim.x * Team<TPR>::ROWS) {
    const int64_t row = row0 + threadIdx.x / TPR;
    if (TPR <= kWave && row >= a.rows) continue;
    const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
    Raw8<T> raw[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = 8 * (t + TPR * i);
      raw[i].zero();
      if (c < a.dim) raw[i].load(x + c);
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float v[8];
      raw[i].get(v);
      top = top_bits(v, top);
    }
    top = row_max<TPR>(top, s_part);
    const Quantise how = quantise_of(top);
    const bool broken = top >= kInfinite;
    uint2 q[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float v[8];
      raw[i].get(v);
      q[i] = broken ? make_uint2(0u, 0u) : pack_i8(v, how);
    }
    const float scale = scale127(top);
    for (int j = 0; j < a.k; ++j) {
      const int64_t p = a.place ? place_of(a.place, row * a.k + j, a.rows * a.k) : row;
      if (p < 0) continue;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int c = 8 * (t + TPR * i);
        if (c < ld) *reinterpret_cast<uint2 *>(a.q + p * ld + c) = q[i];
      }
      if (t == 0) a.scale[p] = scale;
    }
  }
}

// ---- weights in 8-bit integers ------------------------------------------------------------------------------------
// scales: an output's K weights are a wavefront's
template <typename S> __global__ void __launch_bounds__(256) k_scales_i8(const S *__restrict__ w, int64_t outputs, int K, float *__restrict__ scale) {
  for (int64_t n = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; n < outputs; n += (int64_t)gridDim.x * 4) {
    uint32_t top = 0u;
    for (int c = 8 * (threadIdx.x & 63); c < K; c += 8 * kWave) {
      float v[8];
      load8(w + n * K + c, v);
      top = top_bits(v, top);
    }
    top = row_max<kWave>(top, nullptr);
    if ((threadIdx.x & 63) == 0) scale[n] = __uint_as_float(top);    // the largest magnitude; k_finish_scales makes it the scale
  }
}

// packed [expert][32 outputs][k-block of 128][unit][lane] of 16 integers: output lane % 32, piece 2 unit + lane / 32 of the k-block; zeros
// beyond the matrix.  A wavefront takes a unit.  top NULL: w holds integers already.
template <typename S>
__global__ void __launch_bounds__(256) k_pack_i8(const S *__restrict__ w, int N, int K, const float *__restrict__ top, uint4 *__restrict__ packed) {
  const int nk = (K + 127) / 128, n32 = (N + 31) / 32;
  const int kb = blockIdx.x % nk, strip = blockIdx.x / nk % n32, e = blockIdx.x / nk / n32;
  const int lane = threadIdx.x & 63, unit = threadIdx.x >> 6;
  const int n = strip * 32 + (lane & 31), k = kb * 128 + (2 * unit + (lane >> 5)) * 16;
  uint2 half[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    half[h] = make_uint2(0u, 0u);
    if (n >= N || k + 8 * h >= K) continue;
    const int64_t at = ((int64_t)e * N + n) * K + k + 8 * h;
    if constexpr (sizeof(S) == 1) {
      half[h] = *reinterpret_cast<const uint2 *>(w + at);
    } else {
      float v[8];
      load8(w + at, v);
      const uint32_t t = __float_as_uint(top[(int64_t)e * N + n]);
      if (t < kInfinite) half[h] = pack_i8(v, quantise_of(t));
    }
  }
  packed[(int64_t)blockIdx.x * 256 + unit * 64 + lane] = make_uint4(half[0].x, half[0].y, half[1].x, half[1].y);
}
__global__ void __launch_bounds__(256) k_finish_scales(float *__restrict__ scale, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) scale[i] = scale127(__float_as_uint(scale[i]));
}

// call(TPR, PER) with the threads that a row of `dim` values has, and their pieces: a wavefront up to 4096 columns, which needs no
// barrier for its sum
template <typename F> hipError_t by_dim(int64_t dim, F &&call) {
  using std::integral_constant;
  const int64_t pieces = (dim + 7) / 8;
  if (pieces <= 16) return call(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (pieces <= 32) return call(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (pieces <= 64) return call(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (pieces <= 128) return call(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (pieces <= 192) return call(integral_constant<int, 64>{}, integral_constant<int, 3>{});
  if (pieces <= 256) return call(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  if (pieces <= 384) return call(integral_constant<int, 64>{}, integral_constant<int, 6>{});
  if (pieces <= 512) return call(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  if (pieces <= 1024) return call(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  if (pieces <= 2048) return call(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  if (pieces <= 4096) return call(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
  return call(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
}
template <int TPR> unsigned blocks_of(int64_t rows) {
  const int64_t blocks = (rows + Team<TPR>::ROWS - 1) / Team<TPR>::ROWS;
  return (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
}
int64_t chunks_of(int64_t rows, int dim) { return (rows * (dim / 8) + kPieceThreads - 1) / kPieceThreads; }
unsigned grid_of(int64_t chunks) { return (unsigned)(chunks < (1 << 22) ? chunks : (1 << 22)); }

bool dtype_ok(int32_t dtype) { return dtype == GEAR_F32 || dtype == GEAR_BF16; }
bool matrix_ok(const void *p, int64_t ld, int64_t dim) { return p && !((uintptr_t)p & 15) && ld >= dim && ld % 8 == 0 && ld < (1 << 20); }
bool sizes_ok(int64_t rows, int32_t dim, int32_t k) {
  return rows >= 0 && rows <= (1 << 30) && k >= 1 && k <= GEAR_MAX_CHOSEN && rows * k <= (1 << 30) && dim >= 8 && dim % 8 == 0 && dim <= GEAR_MAX_NORM_DIM;
}
bool words_ok(const void *p) { return p && !((uintptr_t)p & 3); }
bool i8_weights_ok(int32_t experts, int32_t N, int32_t K) {
  return experts >= 1 && experts <= GEAR_MAX_EXPERTS && N >= 8 && N % 8 == 0 && N < (1 << 20) && K >= 8 && K % 8 == 0 && K <= GEAR_MAX_NORM_DIM;
}

}  // namespace
}  // namespace gear

using namespace gear;

extern "C" gear_status gear_expert_gather(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t dim, const int32_t *place, int32_t k,
                                          void *xs, int64_t ld_xs, void *stream) {
  if (!sizes_ok(rows, dim, k) || !dtype_ok(dtype)) return GEAR_ERR_INVALID;
  if (rows == 0) return GEAR_OK;
  if (!matrix_ok(x, ld_x, dim) || !matrix_ok(xs, ld_xs, dim) || !words_ok(place)) return GEAR_ERR_INVALID;
  const GatherArgs a = {rows, ld_x, ld_xs, dim, k, 8.0f / (float)dim, chunks_of(rows, dim), x, place, xs};
  if (dtype == GEAR_F32)
    hipLaunchKernelGGL(k_gather<float>, dim3(grid_of(a.chunks)), dim3(kPieceThreads), 0, (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL(k_gather<bf16_t>, dim3(grid_of(a.chunks)), dim3(kPieceThreads), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

extern "C" gear_status gear_expert_combine(const gear_expert_combine_args *a, void *stream) {
  if (!a || !sizes_ok(a->rows, a->dim, a->k) || !dtype_ok(a->dtype)) return GEAR_ERR_INVALID;
  if (a->rows == 0) return GEAR_OK;
  if (!matrix_ok(a->y, a->ld_y, a->dim) || !matrix_ok(a->out, a->ld_out, a->dim) || !words_ok(a->place) || ((uintptr_t)a->weight & 3))
    return GEAR_ERR_INVALID;
  if (a->residual && !matrix_ok(a->residual, a->ld_residual, a->dim)) return GEAR_ERR_INVALID;
  const CombineArgs args = {*a, 8.0f / (float)a->dim, chunks_of(a->rows, a->dim)};
  const dim3 grid(grid_of(args.chunks)), block(kPieceThreads);
  if (a->dtype == GEAR_F32)
    hipLaunchKernelGGL((k_combine<float, float>), grid, block, 0, (hipStream_t)stream, args);
  else if (a->y_f32)
    hipLaunchKernelGGL((k_combine<bf16_t, float>), grid, block, 0, (hipStream_t)stream, args);
  else
    hipLaunchKernelGGL((k_combine<bf16_t, bf16_t>), grid, block, 0, (hipStream_t)stream, args);
  return hipGetLastError() == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

extern "C" gear_status gear_expert_combine_backward(const gear_expert_combine_backward_args *a, void *stream) {
  if (!a || !sizes_ok(a->rows, a->dim, a->k) || !dtype_ok(a->dtype)) return GEAR_ERR_INVALID;
  if (a->rows == 0) return GEAR_OK;
  if (!a->dy && !a->dweight) return GEAR_ERR_INVALID;
  if (!matrix_ok(a->dout, a->ld_dout, a->dim) || !words_ok(a->place) || !words_ok(a->weight) || ((uintptr_t)a->dweight & 3)) return GEAR_ERR_INVALID;
  if ((a->dweight && !matrix_ok(a->y, a->ld_y, a->dim)) || (a->dy && !matrix_ok(a->dy, a->ld_dy, a->dim))) return GEAR_ERR_INVALID;
  const hipError_t err = by_dim(a->dim, [&](auto tpr, auto per) {
    constexpr int TPR = decltype(tpr)::value, PER = decltype(per)::value;
    if (a->dtype == GEAR_F32)
      hipLaunchKernelGGL((k_combine_back<float, TPR, PER>), dim3(blocks_of<TPR>(a->rows)), dim3(Team<TPR>::THREADS), 0, (hipStream_t)stream, *a);
    else
      hipLaunchKernelGGL((k_combine_back<bf16_t, TPR, PER>), dim3(blocks_of<TPR>(a->rows)), dim3(Team<TPR>::THREADS), 0, (hipStream_t)stream, *a);
    return hipGetLastError();
  });
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

extern "C" gear_status gear_rows_i8(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t dim, const int32_t *place, int32_t k, int8_t *q,
                                    float *scale, void *stream) {
  if (!sizes_ok(rows, dim, k) || !dtype_ok(dtype) || (!place && k != 1)) return GEAR_ERR_INVALID;
  if (rows == 0) return GEAR_OK;
  if (!matrix_ok(x, ld_x, dim) || ((uintptr_t)place & 3) || !q || ((uintptr_t)q & 15) || !words_ok(scale)) return GEAR_ERR_INVALID;
  const RowsI8Args a = {rows, ld_x, dim, k, x, place, q, scale};
  const hipError_t err = by_dim(dim, [&](auto tpr, auto per) {
    constexpr int TPR = decltype(tpr)::value, PER = decltype(per)::value;
    if (dtype == GEAR_F32)
      hipLaunchKernelGGL((k_rows_i8<float, TPR, PER>), dim3(blocks_of<TPR>(rows)), dim3(Team<TPR>::THREADS), 0, (hipStream_t)stream, a);
    else
      hipLaunchKernelGGL((k_rows_i8<bf16_t, TPR, PER>), dim3(blocks_of<TPR>(rows)), dim3(Team<TPR>::THREADS), 0, (hipStream_t)stream, a);
    return hipGetLastError();
  });
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

extern "C" size_t gear_packed_i8_bytes(int32_t experts, int32_t N, int32_t K) {
  if (!i8_weights_ok(experts, N, K)) return 0;
  return (size_t)experts * ((N + 31) / 32) * ((K + 127) / 128) * 4096;
}

extern "C" gear_status gear_pack_weights_i8(const void *w, int32_t src_dtype, int32_t experts, int32_t N, int32_t K, int8_t *packed, float *scale,
                                            void *stream) {
  if (!i8_weights_ok(experts, N, K) || (!dtype_ok(src_dtype) && src_dtype != GEAR_I8)) return GEAR_ERR_INVALID;
  if (!w || ((uintptr_t)w & 15) || !packed || ((uintptr_t)packed & 15) || !scale || ((uintptr_t)scale & 15)) return GEAR_ERR_INVALID;
  const int64_t blocks = (int64_t)experts * ((N + 31) / 32) * ((K + 127) / 128), outputs = (int64_t)experts * N;
  if (blocks > (1 << 23)) return GEAR_ERR_INVALID;   // threads of a launch are counted in 32 bits
  hipStream_t s = (hipStream_t)stream;
  const int64_t each = (outputs + 3) / 4;
  const dim3 grid((unsigned)blocks), rows((unsigned)(each < (1 << 20) ? each : (1 << 20))), block(256);
  uint4 *to = reinterpret_cast<uint4 *>(packed);
  if (src_dtype == GEAR_I8) {
    hipLaunchKernelGGL(k_pack_i8<int8_t>, grid, block, 0, s, (const int8_t *)w, N, K, (const float *)nullptr, to);
  } else if (src_dtype == GEAR_BF16) {
    hipLaunchKernelGGL(k_scales_i8<bf16_t>, rows, block, 0, s, (const bf16_t *)w, outputs, K, scale);
    hipLaunchKernelGGL(k_pack_i8<bf16_t>, grid, block, 0, s, (const bf16_t *)w, N, K, (const float *)scale, to);
  } else {
    hipLaunchKernelGGL(k_scales_i8<float>, rows, block, 0, s, (const float *)w, outputs, K, scale);
    hipLaunchKernelGGL(k_pack_i8<float>, grid, block, 0, s, (const float *)w, N, K, (const float *)scale, to);
  }
  if (src_dtype != GEAR_I8) hipLaunchKernelGGL(k_finish_scales, dim3((rows.x + 63) / 64), block, 0, s, scale, outputs);
  return hipGetLastError() == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}
