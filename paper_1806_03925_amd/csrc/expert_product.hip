// Products of rows with the weights of their expert, out[r] = x[r] W_e^T, in fp32, bf16 and 8 bits, for training (forward,
// and dX on transposed weights) and for serving.  Off by row tiles that end with their expert, a layer is one expert.
//
// All three types are one kernel, because 128 bytes of a row are 32, 64 or 128 values of k: a k-block.  It is eight
// 16-byte pieces, and "unit" u of it is piece 2u for one half of a wavefront and piece 2u + 1 for the other.  A unit is
// four v_mfma_f32_32x32x2_f32, one v_mfma_f32_32x32x16_bf16, or half of a v_mfma_scale_f32_32x32x64_f8f6f4; which k a lane
// holds where does not matter, as long as both operands hold the same.  In 8 bits a k-block is also what shares a scale:
// the instruction multiplies by both operands' powers of two itself, so scales cost no vector instruction.
//
// Rows of x are copied global -> LDS by DMA, LDS rows of 128 bytes with their pieces XOR-ed by the row's number modulo 8
// (no bank conflicts); what lies beyond k or beyond the expert's rows is out of the buffer's range and becomes zeros.
// Weights come in operand order (k_pack) straight into registers and never pass LDS.
#include "eight.hpp"
#include "experts.hpp"

#include <type_traits>

namespace gear {
namespace {

typedef int i32x8_v __attribute__((ext_vector_type(8)));

constexpr int kKBlock = 128;           // bytes
constexpr int kPackedBlock = 32 * kKBlock;   // bytes of packed weights for 32 outputs and a k-block

__host__ __device__ constexpr int operand_bytes(int dtype) { return dtype == GEAR_E4M3 ? 1 : dtype == GEAR_BF16 ? 2 : 4; }

struct ProductArgs {
  const unsigned char *x;
  const uint8_t *x_scale;
  const unsigned char *packed;
  const uint8_t *w_scale;
  const int32_t *off;
  void *out;
  int64_t ld_x, ld_out;   // bytes, elements
  int rows, K, N, experts;
  int32_t *status;
};

// Tile shape: WAVES_M x WAVES_N wavefronts, each 32 WTM rows x 64 columns; STAGES k-blocks of x in LDS
template <int DT_, int WTM_, int WAVES_M_, int WAVES_N_, int STAGES_> struct ProductTile {
  static constexpr int DT = DT_, WTM = WTM_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, STAGES = STAGES_;
  static constexpr int WAVES = WAVES_M * WAVES_N, THREADS = WAVES * kWave;
  static constexpr int BM = 32 * WTM * WAVES_M, BN = WN * WAVES_N;
  static constexpr int STAGE_BYTES = BM * kKBlock, DMA = BM / 8 / WAVES;   // copies of a wavefront per stage, eight rows each
  static constexpr int PATCH_BYTES = WAVES * 32 * PATCH_LD * 2;
  static constexpr int LDS_BYTES = STAGES * STAGE_BYTES > PATCH_BYTES ? STAGES * STAGE_BYTES : PATCH_BYTES;
  static_assert(DMA * 8 * WAVES == BM, "a copy is eight rows");
};

// One unit pair (half a k-block): rows from LDS, weights b[unit][column tile] from registers.
template <typename C, int WHICH>
__device__ __forceinline__ void mma_half(f32x16_v (&acc)[C::WTM][TN], uint32_t addr, const u32x4_v (&b)[2][TN],
                                         const uint32_t (&sx)[C::WTM], uint32_t sw) {
  u32x4_v p[C::WTM], q[C::WTM];
  const uint32_t a0 = addr, a1 = addr ^ 32u;
  lds_read16<0>(p[0], a0);
  lds_read16<0>(q[0], a1);
  if constexpr (C::WTM > 1) {
    lds_read16<4096>(p[1], a0);
    lds_read16<4096>(q[1], a1);
  }
  if constexpr (C::WTM > 2) {
    lds_read16<8192>(p[2], a0);
    lds_read16<8192>(q[2], a1);
    lds_read16<12288>(p[3], a0);
    lds_read16<12288>(q[3], a1);
  }
#pragma unroll
  for (int i = 0; i < C::WTM; ++i) {
    if (i == 0) wait_lgkm<2 * (C::WTM - 1)>();
    if (i == 1) wait_lgkm<2 * (C::WTM > 1 ? C::WTM - 2 : 0)>();
    if (i == 2) wait_lgkm<2 * (C::WTM > 2 ? C::WTM - 3 : 0)>();
    if (i == 3) wait_lgkm<0>();
    landed(p[i]);
    landed(q[i]);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      if constexpr (C::DT == GEAR_E4M3) {
        const i32x8_v w = {(int)b[0][j].x, (int)b[0][j].y, (int)b[0][j].z, (int)b[0][j].w,
                           (int)b[1][j].x, (int)b[1][j].y, (int)b[1][j].z, (int)b[1][j].w};
        const i32x8_v r = {(int)p[i].x, (int)p[i].y, (int)p[i].z, (int)p[i].w, (int)q[i].x, (int)q[i].y, (int)q[i].z, (int)q[i].w};
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, r, acc[i][j], 0, 0, WHICH, (int)sw, WHICH, (int)sx[i]);
      } else if constexpr (C::DT == GEAR_BF16) {
        MFMA_BF16_T(acc[i][j], p[i], b[0][j]);
        MFMA_BF16_T(acc[i][j], q[i], b[1][j]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b[0][j][e]), __uint_as_float(p[i][e]), acc[i][j], 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b[1][j][e]), __uint_as_float(q[i][e]), acc[i][j], 0, 0, 0);
      }
    }
  }
}

// Results: a lane holds row lane % 32 of each 32 x 32 tile and four consecutive columns per four accumulator elements.
template <typename C, bool F32>
__device__ __forceinline__ void store_tile(const f32x16_v (&acc)[C::WTM][TN], bf16_t *patch, void *out, int64_t ld, int m0, int m_end,
                                           int n0, int N, int lane) {
  const int c = lane & 31, g = lane >> 5;
  if constexpr (F32) {
    float *o = static_cast<float *>(out);
#pragma unroll
    for (int i = 0; i < C::WTM; ++i) {
      const int m = m0 + i * 32 + c;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = n0 + j * 32 + 8 * q + 4 * g;
          if (m < m_end && n < N)
            *reinterpret_cast<float4 *>(o + m * ld + n) =
                make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        }
    }
  } else {   // through a patch of 32 rows x 64 columns, so that a lane stores 16 bytes and a row leaves as one 128-byte line
    bf16_t *o = static_cast<bf16_t *>(out);
    const int prow = lane >> 3, cv = (lane & 7) * 8;
#pragma unroll
    for (int i = 0; i < C::WTM; ++i) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<uint2 *>(patch + c * PATCH_LD + j * 32 + 8 * q + 4 * g) =
              make_uint2(pack_bf16(acc[i][j][4 * q], acc[i][j][4 * q + 1]), pack_bf16(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]));
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int row = it * 8 + prow, m = m0 + i * 32 + row;
        const uint4 v = *reinterpret_cast<const uint4 *>(patch + row * PATCH_LD + cv);
        if (m < m_end && n0 + cv < N)
          __builtin_nontemporal_store(u32x4_v{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4_v *>(o + m * ld + n0 + cv));
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

template <typename C, bool F32> __device__ __forceinline__ void product_tile(const ProductArgs &a, unsigned char *lds) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
  const int n_tiles = (a.N + C::BN - 1) / C::BN;
  const ExpertTile t = expert_tile(a.off, a.experts, a.rows, C::BM, n_tiles, blockIdx.x, lane);
  if (a.status && blockIdx.x == 0 && threadIdx.x == 0) *a.status = t.bad ? GEAR_ERR_RANGE : GEAR_OK;
  if (!t.have) return;
  const int m0 = t.m0, n0 = t.n_tile * C::BN, m_rows = min(C::BM, t.m_end - m0);
  const int row_bytes = a.K * operand_bytes(C::DT);
  const int nk = (row_bytes + kKBlock - 1) / kKBlock;

  // this lane's pieces of the rows it copies: LDS slot lane % 8 of row lane / 8 receives piece (lane % 8) ^ (row % 8)
  const int piece = (lane & 7) ^ (lane >> 3);
  const auto x_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.x) + (int64_t)m0 * a.ld_x, 0,
                                                        (int)((m_rows - 1) * a.ld_x) + nk * kKBlock, 0x00020000);
  // rows in 8 bits have zeros behind their end; others end inside a k-block, and what is beyond must not be read as k
  const int beyond = C::DT == GEAR_E4M3 ? nk * kKBlock : row_bytes;
  int x_at[C::DMA];
#pragma unroll
  for (int i = 0; i < C::DMA; ++i) {
    const int row = (i * C::WAVES + wave) * 8 + (lane >> 3);
    x_at[i] = row < m_rows ? row * (int)a.ld_x + piece * 16 : -(1 << 30);   // far out of range: zeros
  }
  auto copy = [&](int k) {
    const int kk = min(k, nk - 1);
    unsigned char *s = lds + (k % C::STAGES) * C::STAGE_BYTES;
    const bool in = kk * kKBlock + piece * 16 < beyond;
#pragma unroll
    for (int i = 0; i < C::DMA; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rsrc, (lds_ptr_t)(s + (i * C::WAVES + wave) * 1024), 16, in ? x_at[i] : -(1 << 30),
                                               kk * kKBlock, 0, 0);
    asm volatile("" ::: "memory");
  };
  // packed weights of this wavefront's 64 columns
  const int n32 = (a.N + 31) / 32, first32 = min(n0 / 32 + wn * 2, n32 - 1);
  const int64_t strip = (int64_t)nk * kPackedBlock;
  const auto w_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<unsigned char *>(a.packed) + ((int64_t)t.e * n32 + first32) * strip, 0, (int)(min(2, n32 - first32) * strip), 0x00020000);
  u32x4_v b[2][2][TN];
  auto load = [&](u32x4_v (&to)[2][TN], int k, int half) {
    const int at = min(k, nk - 1) * kPackedBlock + half * 2048;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        to[u][j] = __builtin_bit_cast(u32x4_v, __builtin_amdgcn_raw_buffer_load_b128(w_rsrc, j * (int)strip + lane * 16, at + u * 1024, 0));
    asm volatile("" ::: "memory");
  };
  // scale bytes of four k-blocks at a time: of this lane's rows, and of this wavefront's columns
  const int r = lane & 31, g = lane >> 5;
  constexpr bool E8 = C::DT == GEAR_E4M3;
  uint32_t sx[2][C::WTM], sw[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < C::WTM; ++i) sx[0][i] = sx[1][i] = 0u;
  const int64_t lds8 = scales8_ld(a.K);
  const uint8_t *xs = nullptr, *ws = nullptr;
  if constexpr (E8) {
    xs = a.x_scale + (int64_t)m0 * lds8;
    ws = a.w_scale + ((int64_t)t.e * ((a.N + kBlock8 - 1) / kBlock8) + min(n0 + wn * WN, a.N - 1) / kBlock8) * lds8;
  }
  auto scales = [&](int set, int k) {
    if constexpr (E8) {
      const int at = min(k, nk - 1) & ~3;
#pragma unroll
      for (int i = 0; i < C::WTM; ++i)
        sx[set][i] = *reinterpret_cast<const uint32_t *>(xs + (int64_t)min(wm * 32 * C::WTM + i * 32 + r, m_rows - 1) * lds8 + at);
      sw[set] = *reinterpret_cast<const uint32_t *>(ws + at);
    }
  };

  f32x16_v acc[C::WTM][TN];
#pragma unroll
  for (int i = 0; i < C::WTM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
  const uint32_t x_rel = lds_base + (uint32_t)(wm * C::WTM * 32 + r) * 128u + (uint32_t)((g ^ (r & 7)) << 4);

  scales(0, 0);
#pragma unroll
  for (int k = 0; k < C::STAGES - 1; ++k) copy(k);
  load(b[0], 0, 0);
  load(b[1], 0, 1);
  auto block = [&](int k, auto which) {
    constexpr int W = decltype(which)::value;
    if (k >= nk) return;
    // copies of k have landed once only what was issued after them is outstanding
    if (k == 0) wait_vm<0>(); else wait_vm<8>();
    block_barrier();
    copy(k + C::STAGES - 1);
    const uint32_t at = x_rel + (uint32_t)(k % C::STAGES) * C::STAGE_BYTES;
    mma_half<C, W>(acc, at, b[0], sx[0], sw[0]);
    load(b[0], k + 1, 0);
    mma_half<C, W>(acc, at ^ 64u, b[1], sx[0], sw[0]);
    load(b[1], k + 1, 1);
  };
  for (int k = 0; k < nk; k += 4) {
    scales(1, k + 4);
    block(k, std::integral_constant<int, 0>{});
    block(k + 1, std::integral_constant<int, 1>{});
    block(k + 2, std::integral_constant<int, 2>{});
    block(k + 3, std::integral_constant<int, 3>{});
#pragma unroll
    for (int i = 0; i < C::WTM; ++i) sx[0][i] = sx[1][i];
    sw[0] = sw[1];
  }
  wait_vm<0>();    // copies beyond the end have landed too: LDS becomes the patches
  __syncthreads();
  store_tile<C, F32>(acc, reinterpret_cast<bf16_t *>(lds) + wave * 32 * PATCH_LD, a.out, a.ld_out, m0 + wm * 32 * C::WTM, t.m_end,
                     n0 + wn * WN, a.N, lane);
}

template <typename C, bool F32> __global__ void __launch_bounds__(C::THREADS, 2) k_expert_product(ProductArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[C::LDS_BYTES];
  product_tile<C, F32>(a, lds);
}

// ---- weights in operand order -------------------------------------------------------------------------------------
// packed [expert][32 outputs][k-block][unit][lane] of 16 bytes: output lane % 32, piece 2 unit + lane / 32 of the k-block;
// zeros beyond the matrix.  A workgroup takes 64 x 64 weights through LDS, so that they are read once, in whole lines, for
// both layouts, and a wavefront stores 1 KB of either.  Bound by memory.
template <typename S, typename D>
__global__ void __launch_bounds__(256) k_pack(const S *__restrict__ w, int N, int K, uint4 *__restrict__ packed, uint4 *__restrict__ transposed) {
  constexpr int V = 16 / (int)sizeof(D), KB = kKBlock / (int)sizeof(D);
  constexpr int LD = 64 + 16 / (int)sizeof(D);   // rows 16 bytes apart in their banks
  __shared__ __attribute__((aligned(16))) D tile[64 * LD];
  const int k64 = (K + 63) / 64, n64 = (N + 63) / 64;
  const int kt = blockIdx.x % k64, nt = blockIdx.x / k64 % n64, e = blockIdx.x / k64 / n64;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int n = (threadIdx.x >> 3) + 32 * i, k = (threadIdx.x & 7) * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.0f;
    if (nt * 64 + n < N && kt * 64 + k < K) load8(w + ((int64_t)e * N + nt * 64 + n) * K + kt * 64 + k, v);
    store8(tile + n * LD + k, v);
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, c = lane & 31, wave = threadIdx.x >> 6;
  // 64 x 64 values are 2 strips of 32 outputs x (64 / KB) k-blocks x 4 units: 8 or 16 units, two or four for each wavefront
#pragma unroll
  for (int i = 0; i < 2 * (64 / KB); ++i) {
    const int id = i * 4 + wave, unit = id & 3, kb = (id >> 2) % (64 / KB), strip = (id >> 2) / (64 / KB);
    const int in = kb * KB + (2 * unit + (lane >> 5)) * V, out = strip * 32 + c;
    if (packed && nt * 2 + strip < (N + 31) / 32 && kt * (64 / KB) + kb < (K + KB - 1) / KB) {
      const int64_t blk = ((int64_t)e * ((N + 31) / 32) + nt * 2 + strip) * ((K + KB - 1) / KB) + kt * (64 / KB) + kb;
      packed[blk * 256 + unit * 64 + lane] = *reinterpret_cast<const uint4 *>(tile + out * LD + in);
    }
    if (transposed && kt * 2 + strip < (K + 31) / 32 && nt * (64 / KB) + kb < (N + KB - 1) / KB) {
      const int64_t blk = ((int64_t)e * ((K + 31) / 32) + kt * 2 + strip) * ((N + KB - 1) / KB) + nt * (64 / KB) + kb;
      union {
        D d[V];
        uint4 u;
      } p;
#pragma unroll
      for (int j = 0; j < V; ++j) p.d[j] = tile[(in + j) * LD + out];
      transposed[blk * 256 + unit * 64 + lane] = p.u;
    }
  }
}

// 8 bits: a workgroup takes 128 x 128 weights, finds their largest and stores them scaled
template <typename S>
__global__ void __launch_bounds__(256) k_pack8(const S *__restrict__ w, int N, int K, unsigned char *__restrict__ packed,
                                               uint8_t *__restrict__ scale) {
  __shared__ float s_top[4];
  const int nk = (K + kBlock8 - 1) / kBlock8, n128 = (N + kBlock8 - 1) / kBlock8, n32 = (N + 31) / 32;
  const int kb = blockIdx.x % nk, nb = blockIdx.x / nk % n128, e = blockIdx.x / nk / n128;
  // pieces of 16 values: thread t makes pieces t % 8 of rows t / 8 + 32 i
  const int piece = threadIdx.x & 7, k = kb * kBlock8 + piece * 16;
  float v[4][2][8];
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = nb * kBlock8 + i * 32 + (threadIdx.x >> 3);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][h][j] = 0.0f;
      if (n < N && k + 8 * h < K) load8(w + ((int64_t)e * N + n) * K + k + 8 * h, v[i][h]);
      top = fmaxf(top, top8(v[i][h]));
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
  if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
  const int ex = exponent8(top);
  const int64_t lds8 = scales8_ld(K);
  uint8_t *row = scale + ((int64_t)e * n128 + nb) * lds8;
  if (threadIdx.x == 0) row[kb] = (uint8_t)(ex + 127);
  if (kb == nk - 1 && (int)threadIdx.x < lds8 - nk) row[nk + threadIdx.x] = 0;
  const float unscale = unscale8(ex);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (nb * 4 + i >= n32) break;
    const uint2 lo = pack8(v[i][0], unscale), hi = pack8(v[i][1], unscale);
    const int lane = (threadIdx.x >> 3) + 32 * (piece & 1), unit = piece >> 1;
    unsigned char *dst = packed + (((int64_t)e * n32 + nb * 4 + i) * nk + kb) * kPackedBlock + (unit * 64 + lane) * 16;
    *reinterpret_cast<uint4 *>(dst) = make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
}

int64_t packed_blocks(int operand_dtype, int experts, int out, int in) {
  const int kb = kKBlock / operand_bytes(operand_dtype);
  return (int64_t)experts * ((out + 31) / 32) * ((in + kb - 1) / kb);
}

bool weights_ok(int operand_dtype, int experts, int N, int K, int transposed) {
  return (operand_dtype == GEAR_F32 || operand_dtype == GEAR_BF16 || (operand_dtype == GEAR_E4M3 && !transposed)) && experts >= 1 &&
         experts <= GEAR_MAX_EXPERTS && N >= 8 && N % 8 == 0 && K >= 8 && K % 8 == 0 && N < (1 << 20) && K < (1 << 20);
}

template <typename S, typename D>
hipError_t launch_pack(const void *w, int experts, int N, int K, void *packed, void *transposed, hipStream_t s) {
  const int64_t blocks = (int64_t)experts * ((N + 63) / 64) * ((K + 63) / 64);
  hipLaunchKernelGGL((k_pack<S, D>), dim3((unsigned)blocks), dim3(256), 0, s, (const S *)w, N, K, (uint4 *)packed, (uint4 *)transposed);
  return hipGetLastError();
}

template <int DT, int WTM, int WAVES_M, int WAVES_N, int STAGES>
hipError_t launch_tile(const ProductArgs &a, bool f32, hipStream_t s) {
  using C = ProductTile<DT, WTM, WAVES_M, WAVES_N, STAGES>;
  // as many row tiles as there can be (every expert may end inside one), one at least: it looks at the offsets
  const int64_t m_tiles = ((int64_t)a.rows + C::BM - 1) / C::BM + (a.off ? a.experts - 1 : 0);
  const dim3 grid((unsigned)(m_tiles > 0 ? m_tiles * ((a.N + C::BN - 1) / C::BN) : 1));
  if constexpr (DT == GEAR_F32) {
    hipLaunchKernelGGL((k_expert_product<C, true>), grid, dim3(C::THREADS), 0, s, a);
  } else {
    if (f32)
      hipLaunchKernelGGL((k_expert_product<C, true>), grid, dim3(C::THREADS), 0, s, a);
    else
      hipLaunchKernelGGL((k_expert_product<C, false>), grid, dim3(C::THREADS), 0, s, a);
  }
  return hipGetLastError();
}

template <int DT> hipError_t launch_product(const ProductArgs &a, bool f32, hipStream_t s) {
  return launch_tile<DT, 4, 1, 4, 2>(a, f32, s);
}

}  // namespace
}  // namespace gear

using namespace gear;

extern "C" size_t gear_packed_weights_bytes(int32_t operand_dtype, int32_t experts, int32_t N, int32_t K, int32_t transposed) {
  if (!weights_ok(operand_dtype, experts, N, K, transposed)) return 0;
  return (size_t)packed_blocks(operand_dtype, experts, transposed ? K : N, transposed ? N : K) * kPackedBlock;
}

extern "C" size_t gear_weight_scales_bytes(int32_t experts, int32_t N, int32_t K) {
  if (!weights_ok(GEAR_E4M3, experts, N, K, 0)) return 0;
  return (size_t)experts * ((N + kBlock8 - 1) / kBlock8) * scales8_ld(K);
}

extern "C" gear_status gear_pack_weights(const void *w, int32_t src_dtype, int32_t operand_dtype, int32_t experts, int32_t N,
                                         int32_t K, void *packed, void *packed_transposed, uint8_t *scale, void *stream) {
  if (!weights_ok(operand_dtype, experts, N, K, packed_transposed != nullptr) || (src_dtype != GEAR_F32 && src_dtype != GEAR_BF16))
    return GEAR_ERR_INVALID;
  if (!w || (!packed && !packed_transposed) || ((uintptr_t)w & 15) || ((uintptr_t)packed & 15) || ((uintptr_t)packed_transposed & 15))
    return GEAR_ERR_INVALID;
  if ((operand_dtype == GEAR_E4M3) != (scale != nullptr) || ((uintptr_t)scale & 3)) return GEAR_ERR_INVALID;
  if ((int64_t)experts * ((N + 63) / 64) * ((K + 63) / 64) > (1 << 23)) return GEAR_ERR_INVALID;   // blocks are counted in 32 bits
  hipStream_t s = (hipStream_t)stream;
  hipError_t err;
  if (operand_dtype == GEAR_E4M3) {
    const unsigned blocks = (unsigned)experts * ((N + kBlock8 - 1) / kBlock8) * ((K + kBlock8 - 1) / kBlock8);
    if (src_dtype == GEAR_BF16)
      hipLaunchKernelGGL(k_pack8<bf16_t>, dim3(blocks), dim3(256), 0, s, (const bf16_t *)w, N, K, (unsigned char *)packed, scale);
    else
      hipLaunchKernelGGL(k_pack8<float>, dim3(blocks), dim3(256), 0, s, (const float *)w, N, K, (unsigned char *)packed, scale);
    err = hipGetLastError();
  } else if (operand_dtype == GEAR_BF16) {
    err = src_dtype == GEAR_BF16 ? launch_pack<bf16_t, bf16_t>(w, experts, N, K, packed, packed_transposed, s)
                                 : launch_pack<float, bf16_t>(w, experts, N, K, packed, packed_transposed, s);
  } else {
    err = src_dtype == GEAR_BF16 ? launch_pack<bf16_t, float>(w, experts, N, K, packed, packed_transposed, s)
                                 : launch_pack<float, float>(w, experts, N, K, packed, packed_transposed, s);
  }
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

extern "C" gear_status gear_expert_product(const gear_expert_args *a, void *stream) {
  if (!a || !weights_ok(a->dtype, a->experts, a->N, a->K, 0) || a->rows < 0 || a->rows > (1 << 30)) return GEAR_ERR_INVALID;
  if (a->out_dtype != GEAR_F32 && (a->out_dtype != GEAR_BF16 || a->dtype == GEAR_F32)) return GEAR_ERR_INVALID;
  if (!a->packed || ((uintptr_t)a->packed & 15) || (a->off ? !a->status : a->experts != 1)) return GEAR_ERR_INVALID;
  // tiles are numbered, and their threads counted, in 32 bits: 2^23 tiles of 128 x 128 are more than memory holds
  if (((a->rows + 127) / 128 + a->experts) * ((a->N + 127) / 128) > (1 << 23)) return GEAR_ERR_INVALID;
  const bool e8 = a->dtype == GEAR_E4M3;
  const int size = operand_bytes(a->dtype);
  if (e8 && (!a->w_scale || ((uintptr_t)a->w_scale & 3))) return GEAR_ERR_INVALID;
  if (a->rows > 0) {
    if (!a->x || !a->out || ((uintptr_t)a->x & 15) || ((uintptr_t)a->out & 15)) return GEAR_ERR_INVALID;
    if (a->ld_x < (e8 ? rows8_ld(a->K) : a->K) || a->ld_x % (e8 ? 16 : 8) || a->ld_x >= (1 << 20)) return GEAR_ERR_INVALID;
    if (a->ld_out < a->N || a->ld_out % 8 || a->ld_out >= (1 << 20)) return GEAR_ERR_INVALID;
    if (e8 && (!a->x_scale || ((uintptr_t)a->x_scale & 3))) return GEAR_ERR_INVALID;
  }
  hipStream_t s = (hipStream_t)stream;
  if (a->rows == 0 && !a->off && !a->status) return GEAR_OK;
  const ProductArgs p = {static_cast<const unsigned char *>(a->x), a->x_scale, static_cast<const unsigned char *>(a->packed), a->w_scale,
                         a->off, a->out, a->ld_x * size, a->ld_out, (int)a->rows, a->K, a->N, a->experts, a->status};
  const bool f32 = a->out_dtype == GEAR_F32;
  const hipError_t err = a->dtype == GEAR_E4M3   ? launch_product<GEAR_E4M3>(p, f32, s)
                         : a->dtype == GEAR_BF16 ? launch_product<GEAR_BF16>(p, f32, s)
                                                 : launch_product<GEAR_F32>(p, f32, s);
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}
