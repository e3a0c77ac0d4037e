// Weight gradients grouped by expert, dW_e = dy_e^T x_e over the rows of every expert: a contraction over the rows, whose
// number only the device knows.  A workgroup takes one tile of one expert's gradient and walks all of that expert's rows.
#include "experts.hpp"

namespace gear {
namespace {

struct WgradArgs {
  const void *dy, *x;
  const int32_t *off;
  float *dw;
  int64_t ld_dy, ld_x;   // elements
  int rows, K, N, experts;
  int32_t *status;
};

// Rows of both operands go global -> LDS as they are; operands are assembled from there as in tn_tile.hpp.
template <typename C> __global__ void __launch_bounds__(C::THREADS) k_expert_wgrad(WgradArgs a) {
  using T = typename C::T;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[C::STAGES * C::STAGE_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool ok = !a.off || offsets_ok(a.off, a.experts, a.rows, lane);
  if (a.status && blockIdx.x == 0 && threadIdx.x == 0) *a.status = ok ? GEAR_OK : GEAR_ERR_RANGE;
  if (!ok) return;
  const int n_tiles = (a.N + C::BM - 1) / C::BM, k_tiles = (a.K + C::BN - 1) / C::BN;
  const int work = xcd_remap(blockIdx.x, gridDim.x);
  const int e = work / (n_tiles * k_tiles), tile = work % (n_tiles * k_tiles);
  const int m0 = tile / k_tiles * C::BM, n0 = tile % k_tiles * C::BN;
  const int first = a.off ? a.off[e] : 0, last = a.off ? a.off[e + 1] : a.rows;

  const int wm = wave >> 1, wn = wave & 1;
  constexpr int VEC = 16 / (int)sizeof(T);
  const int krow = lane >> 4;
  const int piece = sizeof(T) == 2 ? (lane & 15) ^ (4 * krow) : (lane & 15);
  const T *a_src = static_cast<const T *>(a.dy) + min(m0 + piece * VEC, a.N - VEC);
  const T *b_src = static_cast<const T *>(a.x) + min(n0 + piece * VEC, a.K - VEC);
  const int nk = (last - first + C::KD - 1) / C::KD;
  const uint64_t zero = zero_address();
  auto issue = [&](int t, int stage) {
    unsigned char *da = lds + stage * C::STAGE_BYTES + wave * 1024, *db = da + C::OPERAND_BYTES;
#pragma unroll
    for (int i = 0; i < C::DMA; ++i) {
      const int64_t k = (int64_t)first + t * C::KD + (i * C::WAVES + wave) * C::ROWS_PER_DMA + krow;
      copy_piece_or_zero(a_src + k * a.ld_dy, k < last, zero, da + i * C::WAVES * 1024);
      copy_piece_or_zero(b_src + k * a.ld_x, k < last, zero, db + i * C::WAVES * 1024);
    }
  };
#pragma unroll
  for (int p = 0; p < C::STAGES - 1; ++p)
    if (p < nk) issue(p, p);

  f32x16_v acc[C::WTM][C::WTN];
#pragma unroll
  for (int i = 0; i < C::WTM; ++i)
#pragma unroll
    for (int j = 0; j < C::WTN; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
  uint32_t a_addr[C::WTM], b_addr[C::WTN];
  if constexpr (sizeof(T) == 4) {
    const uint32_t at = (uint32_t)(lane >> 5) * C::ROW + (uint32_t)(lane & 31) * 4u;
    a_addr[0] = lds_base + at + (uint32_t)wm * 128u;
    b_addr[0] = lds_base + C::OPERAND_BYTES + at + (uint32_t)wn * 128u;
  } else {
    const int j = lane & 15, h = (lane >> 4) & 1, g = lane >> 5;
    const uint32_t at = (uint32_t)(8 * g + (j >> 2)) * C::ROW + 32u * h + 8u * (j & 3);
#pragma unroll
    for (int i = 0; i < C::WTM; ++i) a_addr[i] = lds_base + at + (uint32_t)(((wm * C::WTM + i) ^ (j >> 2)) << 6);
#pragma unroll
    for (int i = 0; i < C::WTN; ++i)
      b_addr[i] = lds_base + C::OPERAND_BYTES + at + (uint32_t)(((wn * C::WTN + i) ^ (j >> 2)) << 6);
  }
  int stage = 0, fill = C::STAGES - 1;
  for (int t = 0; t < nk; ++t) {
    wait_stages<2 * C::DMA, C::STAGES - 2>(nk - 1 - t);
    block_barrier();
    if (t + C::STAGES - 1 < nk) issue(t + C::STAGES - 1, fill);
    mma_stage_rows<C>(acc, a_addr, b_addr, (uint32_t)stage * C::STAGE_BYTES);
    stage = stage + 1 == C::STAGES ? 0 : stage + 1;
    fill = fill + 1 == C::STAGES ? 0 : fill + 1;
  }
  float *dst = a.dw + (int64_t)e * a.N * a.K;
  const int c = lane & 31, g = lane >> 5;
#pragma unroll
  for (int i = 0; i < C::WTM; ++i)
#pragma unroll
    for (int j = 0; j < C::WTN; ++j) {
      const int n = n0 + (wn * C::WTN + j) * 32 + c;
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int m = m0 + (wm * C::WTM + i) * 32 + 8 * (q / 4) + 4 * g + (q % 4);
        if (m < a.N && n < a.K) dst[(int64_t)m * a.K + n] = acc[i][j][q];
      }
    }
}

// ---- bf16, many tiles: 256 x 256 by four wavefronts of 128 x 128 --------------------------------------------------
// Both operands pass LDS, so LDS bounds this product: of 32 rows a tile of 128 x 128 (four wavefronts of 64 x 64) moves 48 KB
// through it for 256 cycles of matrix instructions, this shape 96 KB for 1024.  With one wavefront per SIMD nobody else fills
// its waits, so operands are requested a k-step (16 rows, 512 cycles of products) ahead, also across the border of a stage.
struct WideTile {
  static constexpr int THREADS = 256, WAVES = 4, BM = 256, BN = 256, KD = 32, STAGES = 4;
  static constexpr int ROW = 512, OPERAND_BYTES = KD * ROW, STAGE_BYTES = 2 * OPERAND_BYTES;
  static constexpr int DMA = KD / 2 / WAVES;   // copies of a wavefront per operand and stage, two rows each
};

struct WideFrag {
  u32x2_v a[4][2], b[4][2];   // [32-column tile][rows +0..3 | +4..7 of the lane's eight]
  // even and odd column tiles: the rows' XOR by 64 (row % 4) makes neighbouring tiles trade places, not offsets
  __device__ __forceinline__ void fetch(const uint32_t (&at_a)[4], const uint32_t (&at_b)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lds_read_tr<0>(a[i][0], at_a[i]);
      lds_read_tr<4 * WideTile::ROW>(a[i][1], at_a[i]);
      lds_read_tr<0>(b[i][0], at_b[i]);
      lds_read_tr<4 * WideTile::ROW>(b[i][1], at_b[i]);
    }
  }
  __device__ __forceinline__ void wait() {
    wait_lgkm<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        landed(a[i][h]);
        landed(b[i][h]);
      }
  }
  __device__ __forceinline__ void mma(f32x16_v (&acc)[4][4]) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32x4_v av = {a[i][0].x, a[i][0].y, a[i][1].x, a[i][1].y};
        const u32x4_v bv = {b[j][0].x, b[j][0].y, b[j][1].x, b[j][1].y};
        MFMA_BF16(acc[i][j], av, bv);
      }
    __builtin_amdgcn_sched_barrier(0);
  }
};

__device__ __forceinline__ void wgrad_wide(const WgradArgs &a, unsigned char *lds) {
  using C = WideTile;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool ok = !a.off || offsets_ok(a.off, a.experts, a.rows, lane);
  if (a.status && blockIdx.x == 0 && threadIdx.x == 0) *a.status = ok ? GEAR_OK : GEAR_ERR_RANGE;
  if (!ok) return;
  const int n_tiles = (a.N + C::BM - 1) / C::BM, k_tiles = (a.K + C::BN - 1) / C::BN;
  const int work = xcd_remap(blockIdx.x, gridDim.x);
  const int e = work / (n_tiles * k_tiles), tile = work % (n_tiles * k_tiles);
  const int m0 = tile / k_tiles * C::BM, n0 = tile % k_tiles * C::BN;
  const int first = a.off ? a.off[e] : 0, last = a.off ? a.off[e + 1] : a.rows;
  const int wm = wave >> 1, wn = wave & 1;
  const int nk = (last - first + C::KD - 1) / C::KD;

  // A copy is two rows of 512 bytes; LDS slot lane % 32 of a row receives piece (lane % 32) ^ 4 (row % 4).  Rows beyond the
  // expert's and columns beyond the last row's end are out of the buffer's range and become zeros.
  const int ld_a = (int)a.ld_dy * 2, ld_b = (int)a.ld_x * 2;
  const int krow = lane >> 5, piece = (lane & 31) ^ (4 * (2 * (wave & 1) + krow));
  const unsigned char *pa = static_cast<const unsigned char *>(a.dy) + (int64_t)first * ld_a + m0 * 2;
  const unsigned char *pb = static_cast<const unsigned char *>(a.x) + (int64_t)first * ld_b + n0 * 2;
  const int width_a = min(C::BM, a.N - m0) * 2, width_b = min(C::BN, a.K - n0) * 2;
  auto issue = [&](int t, int stage) {
    const int rows = min(C::KD, last - first - t * C::KD);
    const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(pa) + (int64_t)t * C::KD * ld_a, 0,
                                                      (rows - 1) * ld_a + width_a, 0x00020000);
    const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(pb) + (int64_t)t * C::KD * ld_b, 0,
                                                      (rows - 1) * ld_b + width_b, 0x00020000);
    unsigned char *da = lds + stage * C::STAGE_BYTES + wave * 1024, *db = da + C::OPERAND_BYTES;
#pragma unroll
    for (int i = 0; i < C::DMA; ++i) {
      const int row = (i * C::WAVES + wave) * 2 + krow;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr_t)(da + i * C::WAVES * 1024), 16, row * ld_a + piece * 16, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr_t)(db + i * C::WAVES * 1024), 16, row * ld_b + piece * 16, 0, 0, 0);
    }
    asm volatile("" ::: "memory");
  };
#pragma unroll
  for (int p = 0; p < C::STAGES - 1; ++p)
    if (p < nk) issue(p, p);

  f32x16_v acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;
  uint32_t a_rel[4], b_rel[4];
  {
    const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    const int j = lane & 15, h = (lane >> 4) & 1, g = lane >> 5;
    const uint32_t at = lds_base + (uint32_t)(8 * g + (j >> 2)) * C::ROW + 32u * h + 8u * (j & 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a_rel[i] = at + (uint32_t)(((wm * 4 + i) ^ (j >> 2)) << 6);
      b_rel[i] = at + C::OPERAND_BYTES + (uint32_t)(((wn * 4 + i) ^ (j >> 2)) << 6);
    }
  }
  WideFrag f[2];
  auto fetch = [&](WideFrag &to, uint32_t so) {
    uint32_t at_a[4], at_b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) at_a[i] = a_rel[i] + so, at_b[i] = b_rel[i] + so;
    to.fetch(at_a, at_b);
  };
  if (nk > 0) {
    wait_stages<2 * C::DMA, C::STAGES - 2>(nk - 1);
    block_barrier();
    fetch(f[0], 0);
    f[0].wait();
    int stage = 0, fill = C::STAGES - 1;
    for (int t = 0; t < nk; ++t) {
      const int next = stage + 1 == C::STAGES ? 0 : stage + 1;
      fetch(f[1], (uint32_t)stage * C::STAGE_BYTES + 16u * C::ROW);
      f[0].mma(acc);
      f[1].wait();
      if (t + 1 < nk) {
        wait_stages<2 * C::DMA, C::STAGES - 3>(nk - 2 - t);   // this wave's share of stage t + 1 has landed
        block_barrier();                                      // everybody's has, and everybody has read stages t - 1 and t
        if (t + C::STAGES - 1 < nk) issue(t + C::STAGES - 1, fill);
        fetch(f[0], (uint32_t)next * C::STAGE_BYTES);
      }
      f[1].mma(acc);
      if (t + 1 < nk) f[0].wait();
      stage = next;
      fill = fill + 1 == C::STAGES ? 0 : fill + 1;
    }
  }
  float *dst = a.dw + (int64_t)e * a.N * a.K;
  const int c = lane & 31, g = lane >> 5;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + (wn * 4 + j) * 32 + c;
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int m = m0 + (wm * 4 + i) * 32 + 8 * (q / 4) + 4 * g + (q % 4);
        if (m < a.N && n < a.K) __builtin_nontemporal_store(acc[i][j][q], dst + (int64_t)m * a.K + n);
      }
    }
}

__global__ void __launch_bounds__(WideTile::THREADS, 1) k_expert_wgrad_wide(WgradArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[WideTile::STAGES * WideTile::STAGE_BYTES];
  wgrad_wide(a, lds);
}

template <typename C> hipError_t launch(const WgradArgs &a, hipStream_t s) {
  const int64_t tiles = (int64_t)a.experts * ((a.N + C::BM - 1) / C::BM) * ((a.K + C::BN - 1) / C::BN);
  hipLaunchKernelGGL(k_expert_wgrad<C>, dim3((unsigned)tiles), dim3(C::THREADS), 0, s, a);
  return hipGetLastError();
}

bool wgrad_ok(int dtype, int64_t rows, int experts, int N, int K) {
  return (dtype == GEAR_F32 || dtype == GEAR_BF16) && rows >= 0 && rows <= (1 << 30) && experts >= 1 && experts <= GEAR_MAX_EXPERTS &&
         N >= 8 && N % 8 == 0 && K >= 8 && K % 8 == 0 && N < (1 << 20) && K < (1 << 20) &&
         (int64_t)experts * ((N + 63) / 64) * ((K + 63) / 64) <= (1 << 23);   // tiles are counted in 32 bits
}

}  // namespace
}  // namespace gear

using namespace gear;

extern "C" size_t gear_expert_wgrad_workspace_bytes(int32_t dtype, int64_t rows, int32_t experts, int32_t N, int32_t K) {
  return wgrad_ok(dtype, rows, experts, N, K) ? 256 : 0;
}

extern "C" gear_status gear_expert_wgrad(const gear_expert_wgrad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  if (!a || !wgrad_ok(a->dtype, a->rows, a->experts, a->N, a->K)) return GEAR_ERR_INVALID;
  if (!a->dw || ((uintptr_t)a->dw & 15) || (a->off ? !a->status : a->experts != 1)) return GEAR_ERR_INVALID;
  if (a->rows > 0) {
    if (!a->dy || !a->x || ((uintptr_t)a->dy & 15) || ((uintptr_t)a->x & 15)) return GEAR_ERR_INVALID;
    if (a->ld_dy < a->N || a->ld_dy % 8 || a->ld_dy >= (1 << 20) || a->ld_x < a->K || a->ld_x % 8 || a->ld_x >= (1 << 20))
      return GEAR_ERR_INVALID;
  }
  if (!workspace || ((uintptr_t)workspace & 255)) return GEAR_ERR_INVALID;
  if (workspace_bytes < gear_expert_wgrad_workspace_bytes(a->dtype, a->rows, a->experts, a->N, a->K)) return GEAR_ERR_CAPACITY;
  const WgradArgs w = {a->dy, a->x, a->off, a->dw, a->ld_dy, a->ld_x, (int)a->rows, a->K, a->N, a->experts, a->status};
  hipStream_t s = (hipStream_t)stream;
  if (a->dtype == GEAR_BF16 && (int64_t)a->experts * ((a->N + 255) / 256) * ((a->K + 255) / 256) >= 128) {
    const int64_t tiles = (int64_t)a->experts * ((a->N + 255) / 256) * ((a->K + 255) / 256);
    hipLaunchKernelGGL(k_expert_wgrad_wide, dim3((unsigned)tiles), dim3(WideTile::THREADS), 0, s, w);
    return hipGetLastError() == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
  }
  const hipError_t err = a->dtype == GEAR_BF16 ? launch<TnTile<bf16_t, 2, 2, 3>>(w, s) : launch<TnTile<float, 1, 1, 4>>(w, s);
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}
