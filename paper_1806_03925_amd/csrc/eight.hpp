// Eight values of a row in registers, and the 8-bit form of a row (gear.h): the pieces that the norm, the conversion of rows
// and the layout of weights share (gfx950 only).
#pragma once

#include "gear_internal.hpp"

namespace gear {

constexpr int kBlock8 = 128;   // columns that share a scale

__host__ __device__ __forceinline__ int64_t rows8_ld(int64_t dim) { return (dim + kBlock8 - 1) / kBlock8 * kBlock8; }
__host__ __device__ __forceinline__ int64_t scales8_ld(int64_t dim) { return ((dim + kBlock8 - 1) / kBlock8 + 3) / 4 * 4; }

namespace {

__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t *p, float (&v)[8]) {
  const uint4 a = *reinterpret_cast<const uint4 *>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
  *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&v)[8]) {
  *reinterpret_cast<uint4 *>(p) =
      make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// the same past the L2, for results that are larger than it and not read again soon
__device__ __forceinline__ void stream8(float *p, const float (&v)[8]) {
  typedef float f32x4_t __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(f32x4_t{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_t *>(p));
  __builtin_nontemporal_store(f32x4_t{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4_t *>(p) + 1);
}
__device__ __forceinline__ void stream8(bf16_t *p, const float (&v)[8]) {
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u32x4_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])},
                              reinterpret_cast<u32x4_t *>(p));
}

// eight values as they lie in memory: requested early, unpacked when they are needed
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float *p) { a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4); }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
};
template <> struct Raw8<bf16_t> {
  uint4 a;
  __device__ __forceinline__ void load(const bf16_t *p) { a = *reinterpret_cast<const uint4 *>(p); }
  __device__ __forceinline__ void zero() { a = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
};

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// the largest |v| of eight, those not finite left out
__device__ __forceinline__ float top8(const float (&v)[8]) {
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) t = fmaxf(t, finite(v[i]) ? fabsf(v[i]) : 0.0f);
  return t;
}

// smallest e >= -127 with top <= 448 2^e = 1.75 2^(8 + e), from the parts of top = (1 + frac / 2^23) 2^(E - 127)
__device__ __forceinline__ int exponent8(float top) {
  const uint32_t u = __float_as_uint(top);
  if (u == 0u) return 0;
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < -127 ? -127 : e;
}
// 2^-e, a normal number for every e that exponent8 gives (-127 .. 120), and 2^e, which is not at -127
__device__ __forceinline__ float unscale8(int e) { return __uint_as_float((uint32_t)(127 - e) << 23); }
__device__ __forceinline__ float scale8(int e) { return __uint_as_float(e == -127 ? 0x00400000u : (uint32_t)(127 + e) << 23); }

// v rounded to odd: towards zero, the last bit set if that lost anything.  What is rounded to fewer bits after that comes out as if v
// itself had been, and no v is taken for a border (448 2^e, a tie) that it is not on.
__device__ __forceinline__ float round_odd(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  uint32_t lo = (uint32_t)u;
  lo = (lo & 0xe0000000u) | ((lo & 0x1fffffffu) ? 0x20000000u : 0u);   // 23 of 52 fraction bits are left
  return (float)__longlong_as_double((long long)((u & 0xffffffff00000000ull) | lo));
}

// eight values times 2^-e as e4m3.  Scaled finite values are at most 448, so the conversion never saturates; infinities
// are turned into NaN first, for which e4m3 has a code.
__device__ __forceinline__ uint2 pack8(const float (&v)[8], float unscale) {
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = finite(v[i]) ? v[i] * unscale : __uint_as_float(0x7fc00000u);
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(z[4], z[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(z[6], z[7], hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}
__device__ __forceinline__ void unpack8(uint2 q, float scale, float (&v)[8]) {
  v[0] = __builtin_amdgcn_cvt_f32_fp8((int)q.x, 0) * scale;
  v[1] = __builtin_amdgcn_cvt_f32_fp8((int)q.x, 1) * scale;
  v[2] = __builtin_amdgcn_cvt_f32_fp8((int)q.x, 2) * scale;
  v[3] = __builtin_amdgcn_cvt_f32_fp8((int)q.x, 3) * scale;
  v[4] = __builtin_amdgcn_cvt_f32_fp8((int)q.y, 0) * scale;
  v[5] = __builtin_amdgcn_cvt_f32_fp8((int)q.y, 1) * scale;
  v[6] = __builtin_amdgcn_cvt_f32_fp8((int)q.y, 2) * scale;
  v[7] = __builtin_amdgcn_cvt_f32_fp8((int)q.y, 3) * scale;
}

// Sum over the TPR threads of a row, the same value in all of them: within a wavefront by exchange, between wavefronts
// through s_part [TPR / 64] in ascending order.  TPR > 64: every thread of the workgroup takes part.
template <int TPR, typename V> __device__ __forceinline__ V row_sum(V v, V *s_part) {
#pragma unroll
  for (int o = (TPR < kWave ? TPR : kWave) / 2; o; o >>= 1) v += __shfl_xor(v, o, kWave);
  if constexpr (TPR > kWave) {
    __syncthreads();   // the last sum has been read by everybody
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < TPR / kWave; ++w) v += s_part[w];
  }
  return v;
}

}  // namespace
}  // namespace gear
