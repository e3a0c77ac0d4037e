// Products of rows with the weights of their expert, out[r] = x[r] W_e^T, in fp32, bf16 and 8 bits, for training (forward,
// and dX on transposed weights) and for serving.  Off by row tiles that end with their expert, a layer is one expert.
//
// All three types are one kernel, because 128 bytes of a row are 32, 64 or 128 values of k: a k-block.  It is eight
// 16-byte pieces, and "unit" u of it is piece 2u for one half of a wavefront and piece 2u + 1 for the other.  A unit is
// four v_mfma_f32_32x32x2_f32, one v_mfma_f32_32x32x16_bf16, or half of a v_mfma_scale_f32_32x32x64_f8f6f4; which k a lane
// holds where does not matter, as long as both operands hold the same.  In 8 bits a k-block is also what shares a scale:
// the instruction multiplies by both operands' powers of two itself, so scales cost no vector instruction.
//
// Rows of x are copied global -> LDS by DMA, LDS rows of 128 bytes with their pieces XOR-ed by half the row's number modulo 8:
// the sixteen rows that are read at a time, two to the 256 bytes of all banks, then lie in sixteen different places; what lies
// beyond k or beyond the expert's rows is out of the buffer's range and becomes zeros.
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
  int keep_status;
};

// Tile shape: WAVES_M x WAVES_N wavefronts, each 32 WTM rows x 64 columns.  Both operands are requested a k-block before they are
// multiplied; more would take the registers that another workgroup on the CU needs, which hides more (us of two k-blocks / one: 64 x
// 256 4096 x 1024 x 1152 bf16 13.6 / 13.2, 128 x 128 35092 x 120 x 2840 by 4 in 8 bits 31.8 / 29.9, three / one: 32 x 128 1024 x 2048
// 17.8 / 17.1, fp32 64 x 128 2086 x 8064 x 80 by 61 87 / 74).
constexpr int kStages = 2;   // of x in LDS
template <int DT_, int WTM_, int WAVES_M_, int WAVES_N_> struct ProductTile {
  static constexpr int DT = DT_, WTM = WTM_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_;
  static constexpr int WAVES = WAVES_M * WAVES_N, THREADS = WAVES * kWave;
  static constexpr int BM = 32 * WTM * WAVES_M, BN = WN * WAVES_N;
  static constexpr bool HALVES = BM == 128 && BN == 256;
  static constexpr int STAGE_BYTES = BM * kKBlock, DMA = BM / 8 / WAVES;   // copies of a wavefront per stage, eight rows each
  static constexpr int PATCH_BYTES = WAVES * 32 * PATCH_LD * 2;
  static constexpr int LDS_BYTES = kStages * STAGE_BYTES > PATCH_BYTES ? kStages * STAGE_BYTES : PATCH_BYTES;
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
  } else {   // through a patch of 32 rows x 64 columns, so that a lane stores 16 bytes and a row leaves as 128 bytes
    bf16_t *o = static_cast<bf16_t *>(out);
    const int prow = lane >> 3, cv = (lane & 7) * 8;
    // Past the L2, which keeps the operands that other tiles share, where these are whole lines: us through it / past it, 65536 x
    // 1024 x 1152 in 8 bits 71.5 / 67.7, but 30000 x 4240 x 64, whose rows end inside lines that it puts together, 49.5 / 98.6.
    const bool lines = (ld & 63) == 0 && ((uintptr_t)out & 127) == 0;
    auto store = [&](int i, auto past) {
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int row = it * 8 + prow, m = m0 + i * 32 + row;
        const uint4 v = *reinterpret_cast<const uint4 *>(patch + row * PATCH_LD + cv);
        u32x4_v *dst = reinterpret_cast<u32x4_v *>(o + m * ld + n0 + cv);
        if (m < m_end && n0 + cv < N) {
          if constexpr (decltype(past)::value)
            __builtin_nontemporal_store(u32x4_v{v.x, v.y, v.z, v.w}, dst);
          else
            *dst = u32x4_v{v.x, v.y, v.z, v.w};
        }
      }
    };
#pragma unroll
    for (int i = 0; i < C::WTM; ++i) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<uint2 *>(patch + c * PATCH_LD + j * 32 + 8 * q + 4 * g) =
              make_uint2(pack_bf16(acc[i][j][4 * q], acc[i][j][4 * q + 1]), pack_bf16(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]));
      __builtin_amdgcn_wave_barrier();
      if (lines) {
        store(i, std::true_type{});
        asm volatile("" ::: "memory");   // the compiler would make one of both kinds of store, the plain one
      } else {
        store(i, std::false_type{});
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

template <typename C, bool F32> __device__ __forceinline__ void product_tile(const ProductArgs &a, const ExpertTile &t, unsigned char *lds) {
  const int m0 = t.m0 + max(t.part, 0) * C::BM;
  if (m0 >= t.m_end) return;   // the second half of a tile that has no more rows than the first
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
  const int n0 = t.n_tile * C::BN, m_rows = min(C::BM, t.m_end - m0);
  const int row_bytes = a.K * operand_bytes(C::DT);
  const int nk = (row_bytes + kKBlock - 1) / kKBlock;

  // this lane's pieces of the rows it copies: LDS slot lane % 8 of row lane / 8 receives piece (lane % 8) ^ (row / 2 % 8)
  static_assert(C::WAVES % 2 == 0, "a wavefront copies every second group of eight rows or all: its rows' XOR does not change");
  const int piece = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));
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
    unsigned char *s = lds + (k % kStages) * C::STAGE_BYTES;
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
  u32x4_v b[2][2][TN];   // [half][unit][column tile]
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
  const uint32_t x_rel = lds_base + (uint32_t)(wm * C::WTM * 32 + r) * 128u + (uint32_t)((g ^ (r >> 1 & 7)) << 4);

  scales(0, 0);
  copy(0);
  load(b[0], 0, 0);
  load(b[1], 0, 1);
  auto block = [&](int k, auto which) {
    constexpr int W = decltype(which)::value;
    if (k >= nk) return;
    wait_vm<8>();      // 8 loads were issued after the copies of k
    block_barrier();   // everybody's copies of k have landed, and everybody has read what copy() now overwrites
    copy(k + 1);
    const uint32_t at = x_rel + (uint32_t)(k % kStages) * C::STAGE_BYTES;
    mma_half<C, W>(acc, at, b[0], sx[0], sw[0]);
    load(b[0], k + 1, 0);
    mma_half<C, W>(acc, at ^ 64u, b[1], sx[0], sw[0]);
    load(b[1], k + 1, 1);
  };
  for (int k = 0; k < nk; k += 4) {   // four k-blocks share a word of scales
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

template <typename C> __device__ __forceinline__ ExpertTile look(const ProductArgs &a, bool halves) {
  const ExpertTile t = expert_tile(a.off, a.experts, a.rows, C::BM, (a.N + C::BN - 1) / C::BN, blockIdx.x, threadIdx.x & 63, halves);
  report(t.bad, a.status, a.keep_status);
  return t;
}

template <typename C, bool F32> __global__ void __launch_bounds__(C::THREADS, 2) k_expert_product(ProductArgs a) {
#ifdef __HIP_DEVICE_COMPILE__   // the host's pass does not know copies of 16 bytes into LDS
  using Half = ProductTile<C::DT, C::HALVES ? C::WTM / 2 : C::WTM, C::WAVES_M, C::WAVES_N>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[C::LDS_BYTES];
  const ExpertTile t = look<C>(a, C::HALVES);
  if (!t.have) return;
  if (C::HALVES && t.part >= 0)
    product_tile<Half, F32>(a, t, lds);
  else
    product_tile<C, F32>(a, t, lds);
#endif
}

// ---- few tiles ----------------------------------------------------------------------------------------------------
// A tile of 32 TM rows x 32 TN columns by WAVES wavefronts that take every WAVES-th k-block each and add their results up,
// in ascending order, through LDS.  Where there are too few tiles to fill the device a product is a walk through the
// weights, and what counts is that all of them are on their way at once: both operands go straight into registers, AHEAD
// k-blocks before they are multiplied, and nothing waits for anybody else before the end.
template <int DT_, int TM_, int TN_, int WAVES_, int AHEAD_> struct SplitTile {
  static constexpr int DT = DT_, TM = TM_, TN = TN_, WAVES = WAVES_, AHEAD = AHEAD_, THREADS = WAVES * kWave, BM = 32 * TM, BN = 32 * TN;
};

template <typename C> struct SplitBlock {   // operands of a k-block in registers
  u32x4_v x[C::TM][4], w[C::TN][4];
  int sx[C::TM], sw;
};

template <typename C, bool F32> __device__ __forceinline__ void split_tile(const ProductArgs &a, float *sums) {
  constexpr int DT = C::DT, TM_ = C::TM, TN_ = C::TN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ExpertTile t = look<C>(a, false);
  if (!t.have) return;
  const int m0 = t.m0, n0 = t.n_tile * C::BN, m_rows = min(C::BM, t.m_end - m0);
  const int row_bytes = a.K * operand_bytes(DT), nk = (row_bytes + kKBlock - 1) / kKBlock;
  const int beyond = DT == GEAR_E4M3 ? nk * kKBlock : row_bytes;
  const int r = lane & 31, g = lane >> 5;
  const auto x_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.x) + (int64_t)m0 * a.ld_x, 0,
                                                        (int)((m_rows - 1) * a.ld_x) + nk * kKBlock, 0x00020000);
  int x_at[TM_];
#pragma unroll
  for (int i = 0; i < TM_; ++i) x_at[i] = i * 32 + r < m_rows ? (i * 32 + r) * (int)a.ld_x + g * 16 : -(1 << 30);
  const int n32 = (a.N + 31) / 32, first32 = n0 / 32;
  const int64_t strip = (int64_t)nk * kPackedBlock;
  const auto w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.packed) + ((int64_t)t.e * n32 + first32) * strip, 0,
                                                        (int)(min(TN_, n32 - first32) * strip), 0x00020000);
  const int64_t lds8 = scales8_ld(a.K);
  const uint8_t *xs[TM_], *ws = nullptr;
  if constexpr (DT == GEAR_E4M3) {
#pragma unroll
    for (int i = 0; i < TM_; ++i) xs[i] = a.x_scale + (int64_t)(m0 + min(i * 32 + r, m_rows - 1)) * lds8;
    ws = a.w_scale + ((int64_t)t.e * ((a.N + kBlock8 - 1) / kBlock8) + n0 / kBlock8) * lds8;
  }
  f32x16_v acc[TM_][TN_];
#pragma unroll
  for (int i = 0; i < TM_; ++i)
#pragma unroll
    for (int j = 0; j < TN_; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;
  auto load = [&](SplitBlock<C> &b, int k) {   // past the end: the last block once more, which is not multiplied
    const int kk = min(k, nk - 1);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int j = 0; j < TN_; ++j)
        b.w[j][u] = __builtin_bit_cast(u32x4_v, __builtin_amdgcn_raw_buffer_load_b128(w_rsrc, j * (int)strip + lane * 16,
                                                                                      kk * kPackedBlock + u * 1024, 0));
      const bool in = kk * kKBlock + (2 * u + g) * 16 < beyond;
#pragma unroll
      for (int i = 0; i < TM_; ++i)
        b.x[i][u] = __builtin_bit_cast(u32x4_v, __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, in ? x_at[i] + u * 32 : -(1 << 30), kk * kKBlock, 0));
    }
    if constexpr (DT == GEAR_E4M3) {
#pragma unroll
      for (int i = 0; i < TM_; ++i) b.sx[i] = xs[i][kk];
      b.sw = ws[kk];
    }
  };
  auto mma = [&](const SplitBlock<C> &b) {
#pragma unroll
    for (int i = 0; i < TM_; ++i)
#pragma unroll
      for (int j = 0; j < TN_; ++j) {
        if constexpr (DT == GEAR_E4M3) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4_v &w0 = b.w[j][2 * h], &w1 = b.w[j][2 * h + 1], &x0 = b.x[i][2 * h], &x1 = b.x[i][2 * h + 1];
            const i32x8_v w = {(int)w0.x, (int)w0.y, (int)w0.z, (int)w0.w, (int)w1.x, (int)w1.y, (int)w1.z, (int)w1.w};
            const i32x8_v x = {(int)x0.x, (int)x0.y, (int)x0.z, (int)x0.w, (int)x1.x, (int)x1.y, (int)x1.z, (int)x1.w};
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, acc[i][j], 0, 0, 0, b.sw, 0, b.sx[i]);
          }
        } else if constexpr (DT == GEAR_BF16) {
#pragma unroll
          for (int u = 0; u < 4; ++u) MFMA_BF16_T(acc[i][j], b.x[i][u], b.w[j][u]);
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.w[j][u][e]), __uint_as_float(b.x[i][u][e]), acc[i][j], 0, 0, 0);
        }
      }
  };
  SplitBlock<C> b[C::AHEAD + 1];
#pragma unroll
  for (int p = 0; p < C::AHEAD; ++p) load(b[p], wave + p * C::WAVES);
  for (int k = wave; k < nk; k += (C::AHEAD + 1) * C::WAVES) {
#pragma unroll
    for (int p = 0; p <= C::AHEAD; ++p) {
      load(b[(p + C::AHEAD) % (C::AHEAD + 1)], k + (p + C::AHEAD) * C::WAVES);
      if (k + p * C::WAVES < nk) mma(b[p]);
    }
  }
  // [wavefront][tile][element / 4][lane] of four values each: four consecutive columns of row lane % 32
  constexpr int PARTS = TM_ * TN_ * 4;
#pragma unroll
  for (int i = 0; i < TM_; ++i)
#pragma unroll
    for (int j = 0; j < TN_; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4 *>(sums + (((wave * TM_ + i) * TN_ + j) * 256 + q * 64 + lane) * 4) =
            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
  __syncthreads();
  for (int part = wave; part < PARTS; part += C::WAVES) {
    const int q = part & 3, j = (part >> 2) % TN_, i = (part >> 2) / TN_;
    float4 v = *reinterpret_cast<const float4 *>(sums + (part * 64 + lane) * 4);
#pragma unroll
    for (int w = 1; w < C::WAVES; ++w) {
      const float4 o = *reinterpret_cast<const float4 *>(sums + ((w * PARTS + part) * 64 + lane) * 4);
      v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
    }
    const int m = i * 32 + r, n = n0 + j * 32 + 8 * q + 4 * g;
    if (m < m_rows && n < a.N) {
      if constexpr (F32)
        *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + (m0 + m) * a.ld_out + n) = v;
      else
        *reinterpret_cast<uint2 *>(static_cast<bf16_t *>(a.out) + (m0 + m) * a.ld_out + n) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    }
  }
}

template <typename C, bool F32> __global__ void __launch_bounds__(C::THREADS) k_expert_product_split(ProductArgs a) {
  __shared__ __attribute__((aligned(16))) float sums[C::WAVES * C::BM * C::BN];
  split_tile<C, F32>(a, sums);
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

template <int DT, int WTM, int WAVES_M, int WAVES_N>
hipError_t launch_tile(const ProductArgs &a, bool f32, hipStream_t s) {
  using C = ProductTile<DT, WTM, WAVES_M, WAVES_N>;
  // as many row tiles as there can be (every expert may end inside one), one at least: it looks at the offsets
  const int64_t m_tiles = ((int64_t)a.rows + C::BM - 1) / C::BM + (a.off ? a.experts - 1 : 0);
  const dim3 grid((unsigned)((m_tiles > 0 ? m_tiles * ((a.N + C::BN - 1) / C::BN) : 1) + (C::HALVES ? kHalved : 0)));
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

template <int DT, int TM, int TN, int WAVES, int AHEAD> hipError_t launch_split(const ProductArgs &a, bool f32, hipStream_t s) {
  using C = SplitTile<DT, TM, TN, WAVES, AHEAD>;
  const int64_t m_tiles = ((int64_t)a.rows + C::BM - 1) / C::BM + (a.off ? a.experts - 1 : 0);
  const dim3 grid((unsigned)(m_tiles > 0 ? m_tiles * ((a.N + C::BN - 1) / C::BN) : 1));
  if constexpr (DT == GEAR_F32) {
    hipLaunchKernelGGL((k_expert_product_split<C, true>), grid, dim3(C::THREADS), 0, s, a);
  } else {
    if (f32)
      hipLaunchKernelGGL((k_expert_product_split<C, true>), grid, dim3(C::THREADS), 0, s, a);
    else
      hipLaunchKernelGGL((k_expert_product_split<C, false>), grid, dim3(C::THREADS), 0, s, a);
  }
  return hipGetLastError();
}

// Which shape: the largest that still gives the device something to do, by the number of tiles (with experts, of about how
// many: half a tile more for each).  us measured, K = N where one is given, smaller / larger shape of each border:
//   few tiles, up to 256 of 32 x 32 (one for each CU), against 32 x 128: 256 x 1024 x 1152 bf16 7.3 / 7.6, 64 x 4096 8 bits 10.5 /
//     10.3; above, 512 x 1024 x 1152 bf16 11.9 / 7.8.  fp32, whose products are slow, up to 1024, against 64 x 128: 512 x 2048 53.5 /
//     70.0, 1024 x 2048 98.8 / 74.6
//   32 x 64 split over k by eight wavefronts where these are one for each CU at most and walk 48 k-blocks or more, against 32 x 128: 535 x
//     816 x 5568 bf16 22.9 / 32.1, 512 x 800 x 8192 8 bits 18.1 / 25.1, but half as far, 512 x 800 x 4096 8 bits, 11.3 / 10.5
//   32 x 128 up to 256 tiles, then 64 x 128 up to as many: 1024 x 1024 x 4096 bf16 25.2 / 27.1, 1024 x 2048 16.9 / 14.9, 256 x 8192
//     54.4 / 50.3; where experts have few rows only above 512: 1000 x 1024 by 32 15.9 / 18.2
//   64 x 256 above, against 32 x 128 and 64 x 128: 1500 x 2048 x 1024 bf16 12.0 / 13.6 / 14.2, 2000 x 2048 20.2 / 28.2 / 25.0, up to 512
//     tiles, against 128 x 256: 2048 x 2048 bf16 19.9 / 28.1, 4096 x 2048 34.4 / 33.8
//   fp32: 64 x 128 by four wavefronts: 16384 x 1024 x 1152 by 8 experts 308 / 405, but 65536 x 1024 x 576 577 / 557; 32 x 64 split over k,
//     which moves more, where rounds of one 64 x 128 for each CU would be less than three quarters full: 1441 x 1880 x 5736 by 2 (360
//     tiles) 295 / 340, 4000 x 512 x 576 by 8 (268) 33.7 / 40.5, 3000 x 1024 (376) 63.9 / 65.3, but 1600 x 2048 x 1024 (400) 71.4 / 66.9
//   up to 128 columns, and up to 384 where 256 are too few, of which wider tiles leave a quarter or more empty: 128 x 128, against 64 x 256:
//     65536 x 72 x 320 in 8 bits 9.2 / 11.3, 9000 x 264 x 2000 bf16 22.3 / 29.2
template <int DT> hipError_t launch_product(const ProductArgs &a, bool f32, hipStream_t s) {
  auto tiles = [&](int bm, int bn) { return ((int64_t)(a.rows + bm - 1) / bm + (a.off ? a.experts / 2 : 0)) * ((a.N + bn - 1) / bn); };
  if (tiles(32, 32) <= (DT == GEAR_F32 ? 1024 : 256)) return launch_split<DT, 1, 1, 4, 2>(a, f32, s);
  if constexpr (DT == GEAR_F32) {
    const int64_t count = tiles(64, 128), empty = (count + 255) / 256 * 256 - count;
    if (empty > count / 3) return launch_split<DT, 1, 2, 4, 1>(a, f32, s);
    return launch_tile<DT, 1, 2, 2>(a, f32, s);
  } else {
    if (tiles(32, 64) <= 256 && a.K * operand_bytes(DT) >= 48 * kKBlock) return launch_split<DT, 1, 2, 8, 1>(a, f32, s);
    const int64_t narrow = tiles(32, 128);
    if (narrow <= 256 || (narrow <= 512 && a.rows < 256 * (int64_t)a.experts)) return launch_tile<DT, 1, 1, 2>(a, f32, s);
    if (narrow <= 512) return launch_tile<DT, 1, 2, 2>(a, f32, s);
    if (a.N <= 128 || (a.N > 256 && a.N <= 384)) return launch_tile<DT, 2, 2, 2>(a, f32, s);
    if (tiles(64, 256) < 512) return launch_tile<DT, 2, 1, 4>(a, f32, s);
    return launch_tile<DT, 4, 1, 4>(a, f32, s);
  }
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
                         a->off, a->out, a->ld_x * size, a->ld_out, (int)a->rows, a->K, a->N, a->experts, a->status,
                         a->keep_status};
  const bool f32 = a->out_dtype == GEAR_F32;
  const hipError_t err = a->dtype == GEAR_E4M3   ? launch_product<GEAR_E4M3>(p, f32, s)
                         : a->dtype == GEAR_BF16 ? launch_product<GEAR_BF16>(p, f32, s)
                                                 : launch_product<GEAR_F32>(p, f32, s);
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}
