// Weight gradients grouped by expert, dW_e = dy_e^T x_e over the rows of every expert: a contraction over the rows, whose
// number only the device knows.  A workgroup takes one tile of one expert's gradient and walks that expert's rows, or a piece of
// them: long experts are cut, and what their pieces add up to is summed afterwards.
#include "experts.hpp"

#include <type_traits>

namespace gear {
namespace {

typedef float f32x4_v __attribute__((ext_vector_type(4)));

struct WgradArgs {
  const void *dy, *x;
  const int32_t *off;
  float *dw;
  int64_t ld_dy, ld_x;   // elements
  int rows, K, N, experts;
  int32_t *status;
  float *partial;        // [pieces of experts that are cut][N x K]
  int cut;               // rows of a piece
  int keep_status;
};

struct WgradTile {
  int m0, n0, first, last;
  float *dst;
  bool have, bad;
};

// An expert's rows are as many pieces as its rows need at `cut` rows each, all of them as long, in whole stages.
__device__ __forceinline__ int pieces_of(int rows, int cut) { return max((rows + cut - 1) / cut, 1); }   // no rows: zeros to write
__device__ __forceinline__ int piece_rows(int rows, int cut) {
  const int pieces = pieces_of(rows, cut);
  return ((rows + pieces - 1) / pieces + 31) / 32 * 32;
}

// partial results in front of those of expert e: the pieces of all experts before it that are cut
__device__ __forceinline__ int partials_before(const int32_t *__restrict__ off, int e, int cut, int lane) {
  int n = 0;
  for (int e0 = 0; e0 < e; e0 += kWave) {
    const int at = min(e0 + lane, e - 1), rows = off[at + 1] - off[at];
    n += e0 + lane < e && rows > cut ? pieces_of(rows, cut) : 0;
  }
  return wave_add(n);
}

// The tile of workgroup `block`, and the rows it adds up: an expert's rows are cut into pieces of `cut`, and what the pieces of
// one expert add up to is left in `partial` and summed by k_wgrad_sum (an expert of one piece needs neither).  Experts come
// in descending order of their rows (up to 64 experts, which one look at the offsets orders; with more of them chance does),
// so that the long tiles are not the last ones.  Workgroups are spread over the XCDs by their number modulo 8, whatever they
// cost: kSpread neighbouring tiles, which share rows of dy and x, go to one XCD, the next ones to the next.  us of 8 / 16 / 32: 65536 x
// 1024 x 1152 of one expert 180 / 171 / 170, 65536 x 2048 x 1024 of 64 392 / 392 / 421.
constexpr int kSpread = 16;
__device__ __forceinline__ WgradTile wgrad_tile(const WgradArgs &a, int bm, int bn, int block, int lane) {
  WgradTile r = {0, 0, 0, 0, nullptr, false, false};
  r.bad = a.off && !offsets_ok(a.off, a.experts, a.rows, lane);
  if (r.bad) return r;
  const int n_tiles = (a.N + bm - 1) / bm, k_tiles = (a.K + bn - 1) / bn;
  const int work = (block / kXcds / kSpread * kXcds + block % kXcds) * kSpread + block / kXcds % kSpread;
  const int want = work / (n_tiles * k_tiles), tile = work % (n_tiles * k_tiles);   // the want-th piece of all
  int e = -1, piece = 0;
  if (!a.off) {
    if (want < pieces_of(a.rows, a.cut)) e = 0, piece = want;
  } else if (a.experts <= kWave) {
    const int rows = lane < a.experts ? a.off[lane + 1] - a.off[lane] : -1, mine = lane < a.experts ? pieces_of(rows, a.cut) : 0;
    int before = 0;   // pieces of the experts with more rows
    for (int j = 0; j < a.experts; ++j) {
      const int other = __builtin_amdgcn_readlane(rows, j), pieces = __builtin_amdgcn_readlane(mine, j);
      before += other > rows || (other == rows && j < lane) ? pieces : 0;
    }
    const unsigned long long m = __ballot(want >= before && want < before + mine);
    if (m) e = __builtin_ctzll(m), piece = want - __shfl(before, e, kWave);
  } else {
    int before = 0;
    for (int e0 = 0; e0 < a.experts && e < 0; e0 += kWave) {
      const int at = min(e0 + lane, a.experts - 1), mine = e0 + lane < a.experts ? pieces_of(a.off[at + 1] - a.off[at], a.cut) : 0;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int v = __shfl_up(upto, o, kWave);
        if (lane >= o) upto += v;
      }
      const unsigned long long m = __ballot(want < before + upto);
      if (m) {
        const int l = __builtin_ctzll(m);
        e = e0 + l, piece = want - before - __shfl(upto - mine, l, kWave);
      }
      before += __shfl(upto, kWave - 1, kWave);
    }
  }
  e = __builtin_amdgcn_readfirstlane(e), piece = __builtin_amdgcn_readfirstlane(piece);
  if (e < 0) return r;
  const int first = a.off ? a.off[e] : 0, last = a.off ? a.off[e + 1] : a.rows;
  r.m0 = tile / k_tiles * bm, r.n0 = tile % k_tiles * bn, r.have = true;
  const int step = piece_rows(last - first, a.cut);
  r.first = min(last, first + piece * step), r.last = r.first + min(last - r.first, step);   // rounding up may leave the last piece nothing
  r.dst = a.dw + (int64_t)e * a.N * a.K;
  if (last - first > a.cut) {
    const int before = a.off ? __builtin_amdgcn_readfirstlane(partials_before(a.off, e, a.cut, lane)) : 0;
    r.dst = a.partial + (int64_t)(before + piece) * a.N * a.K;
  }
  return r;
}

// dw of the experts that were cut: their pieces in ascending order, in SHARES equal shares whose sums are added in that order, too
constexpr int kAtOnce = 8;
template <int SHARES> __global__ void __launch_bounds__(256) k_wgrad_sum(WgradArgs a) {
  constexpr int COLS = 256 / SHARES;
  __shared__ float4 s_sum[SHARES > 1 ? SHARES : 1][COLS];
  const int lane = threadIdx.x & 63, e = blockIdx.y;
  if (a.off && !offsets_ok(a.off, a.experts, a.rows, lane)) return;
  const int rows = a.off ? a.off[e + 1] - a.off[e] : a.rows;
  if (rows <= a.cut) return;
  const int before = a.off ? __builtin_amdgcn_readfirstlane(partials_before(a.off, e, a.cut, lane)) : 0, pieces = pieces_of(rows, a.cut);
  const int share = threadIdx.x / COLS, col = threadIdx.x % COLS, each = (pieces + SHARES - 1) / SHARES, last = min(pieces, (share + 1) * each);
  const int64_t vec = (int64_t)a.N * a.K / 4;
  const float4 *p = reinterpret_cast<const float4 *>(a.partial) + before * vec;
  float4 *o = reinterpret_cast<float4 *>(a.dw) + e * vec;
  for (int64_t i0 = (int64_t)blockIdx.x * COLS; i0 < vec; i0 += (int64_t)gridDim.x * COLS) {
    const int64_t i = i0 + col;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (i < vec) {
      for (int z = share * each; z < last; z += kAtOnce) {   // several on their way at a time, added in ascending order
        float4 w[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) w[k] = z + k < last ? p[(z + k) * vec + i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) v.x += w[k].x, v.y += w[k].y, v.z += w[k].z, v.w += w[k].w;
      }
    }
    if constexpr (SHARES > 1) {
      __syncthreads();   // the last sums have been read
      s_sum[share][col] = v;
      __syncthreads();
      if (share > 0) continue;
#pragma unroll
      for (int k = 1; k < SHARES; ++k) v.x += s_sum[k][col].x, v.y += s_sum[k][col].y, v.z += s_sum[k][col].z, v.w += s_sum[k][col].w;
    }
    if (i < vec) o[i] = v;
  }
}
// workgroups for `tiles` tiles: whole rounds of kSpread tiles on every XCD
inline unsigned wgrad_blocks(int64_t tiles) { return (unsigned)((tiles + kSpread * kXcds - 1) / (kSpread * kXcds) * (kSpread * kXcds)); }

// Rows of both operands go global -> LDS as they are; operands are assembled from there as in tn_tile.hpp.
template <typename C> __global__ void __launch_bounds__(C::THREADS) k_expert_wgrad(WgradArgs a) {
  using T = typename C::T;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[C::STAGES * C::STAGE_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const WgradTile t = wgrad_tile(a, C::BM, C::BN, blockIdx.x, lane);
  report(t.bad, a.status, a.keep_status);
  if (!t.have) return;
  const int m0 = t.m0, n0 = t.n0, first = t.first, last = t.last;

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
  for (int k = 0; k < nk; ++k) {
    wait_stages<2 * C::DMA, C::STAGES - 2>(nk - 1 - k);
    block_barrier();
    if (k + C::STAGES - 1 < nk) issue(k + C::STAGES - 1, fill);
    mma_stage_rows<C>(acc, a_addr, b_addr, (uint32_t)stage * C::STAGE_BYTES);
    stage = stage + 1 == C::STAGES ? 0 : stage + 1;
    fill = fill + 1 == C::STAGES ? 0 : fill + 1;
  }
  float *dst = t.dst;
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

// ---- bf16: 128 x 256 by four wavefronts of 64 x 128 ----------------------------------------------------------------
// Both operands pass LDS, whose 128 bytes a cycle bound the loop: of 32 rows a tile of 128 x 128 (four wavefronts of 64 x 64) moves 48 KB
// through it for 256 cycles of matrix instructions (these are busy 0.67 of the time at most), this one 72 KB for 512 (0.89).  Two workgroups share a CU, so that one stores
// its gradient (128 KB) while the other multiplies; and operands are requested a k-step (16 rows) ahead, also across the
// border of a stage.
template <int TM_, int TN_, int WAVES_M_, int WAVES_N_, int STAGES_> struct WideTile {
  static constexpr int TM = TM_, TN = TN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, STAGES = STAGES_, KD = 32;
  static constexpr int WAVES = WAVES_M * WAVES_N, THREADS = WAVES * kWave, BM = 32 * TM * WAVES_M, BN = 32 * TN * WAVES_N;
  static constexpr int ROW_A = BM * 2, ROW_B = BN * 2, A_BYTES = KD * ROW_A, STAGE_BYTES = A_BYTES + KD * ROW_B;
  static constexpr int DMA_A = A_BYTES / 1024 / WAVES, DMA_B = KD * ROW_B / 1024 / WAVES, DMA_ALL = DMA_A + DMA_B;   // copies of a wavefront
};

template <typename C> struct WideFrag {
  u32x2_v a[C::TM][2], b[C::TN][2];   // [32-column tile][rows +0..3 | +4..7 of the lane's eight]
  __device__ __forceinline__ void fetch(const uint32_t (&at_a)[C::TM], const uint32_t (&at_b)[C::TN], uint32_t so_a, uint32_t so_b) {
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
      lds_read_tr<0>(a[i][0], at_a[i] + so_a);
      lds_read_tr<4 * C::ROW_A>(a[i][1], at_a[i] + so_a);
    }
#pragma unroll
    for (int i = 0; i < C::TN; ++i) {
      lds_read_tr<0>(b[i][0], at_b[i] + so_b);
      lds_read_tr<4 * C::ROW_B>(b[i][1], at_b[i] + so_b);
    }
  }
  __device__ __forceinline__ void wait() {
    wait_lgkm<0>();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < C::TM; ++i) landed(a[i][h]);
#pragma unroll
      for (int i = 0; i < C::TN; ++i) landed(b[i][h]);
    }
  }
  __device__ __forceinline__ void mma(f32x16_v (&acc)[C::TM][C::TN]) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j) {
        const u32x4_v av = {a[i][0].x, a[i][0].y, a[i][1].x, a[i][1].y};
        const u32x4_v bv = {b[j][0].x, b[j][0].y, b[j][1].x, b[j][1].y};
        MFMA_BF16(acc[i][j], av, bv);
      }
    __builtin_amdgcn_sched_barrier(0);
  }
};

template <typename C> __device__ __forceinline__ void wgrad_wide(const WgradArgs &a, unsigned char *lds) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const WgradTile t = wgrad_tile(a, C::BM, C::BN, blockIdx.x, lane);
  report(t.bad, a.status, a.keep_status);
  if (!t.have) return;
  const int m0 = t.m0, n0 = t.n0, first = t.first, last = t.last;
  const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
  const int nk = (last - first + C::KD - 1) / C::KD;

  // A copy is four rows of dy (256 bytes) or two of x (512); the slot of a row's 16-byte piece is XOR-ed by 4 (row % 4), so that
  // the four rows that a transposing read touches lie in different quarters of the banks.  Rows beyond the expert's and columns
  // beyond the last row's end are out of the buffer's range and become zeros.
  const int ld_a = (int)a.ld_dy * 2, ld_b = (int)a.ld_x * 2;
  constexpr int PA = C::ROW_A / 16, PB = C::ROW_B / 16, RA = 64 / PA, RB = 64 / PB;   // pieces of a row, rows of a copy
  static_assert((PA == 16 || PA == 32) && (PB == 16 || PB == 32) && C::WAVES % 2 == 0, "copies of two rows or four");
  const int row_a = RA * wave + lane / PA, row_b = RB * wave + lane / PB;
  const int at_a = row_a * ld_a + ((lane % PA) ^ (4 * (row_a & 3))) * 16, at_b = row_b * ld_b + ((lane % PB) ^ (4 * (row_b & 3))) * 16;
  unsigned char *pa = static_cast<unsigned char *>(const_cast<void *>(a.dy)) + (int64_t)first * ld_a + m0 * 2;
  unsigned char *pb = static_cast<unsigned char *>(const_cast<void *>(a.x)) + (int64_t)first * ld_b + n0 * 2;
  const int width_a = min(C::BM, a.N - m0) * 2, width_b = min(C::BN, a.K - n0) * 2;
  auto issue = [&](int k, int stage) {
    const int rows = min(C::KD, last - first - k * C::KD);
    const auto ra = __builtin_amdgcn_make_buffer_rsrc(pa + (int64_t)k * C::KD * ld_a, 0, (rows - 1) * ld_a + width_a, 0x00020000);
    const auto rb = __builtin_amdgcn_make_buffer_rsrc(pb + (int64_t)k * C::KD * ld_b, 0, (rows - 1) * ld_b + width_b, 0x00020000);
    unsigned char *da = lds + stage * C::STAGE_BYTES + wave * 1024, *db = da + C::A_BYTES;
#pragma unroll
    for (int i = 0; i < C::DMA_A; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr_t)(da + i * C::WAVES * 1024), 16, at_a + i * RA * C::WAVES * ld_a, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < C::DMA_B; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr_t)(db + i * C::WAVES * 1024), 16, at_b + i * RB * C::WAVES * ld_b, 0, 0, 0);
    asm volatile("" ::: "memory");
  };
#pragma unroll
  for (int p = 0; p < C::STAGES - 1; ++p)
    if (p < nk) issue(p, p);

  f32x16_v acc[C::TM][C::TN];
#pragma unroll
  for (int i = 0; i < C::TM; ++i)
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;
  uint32_t a_rel[C::TM], b_rel[C::TN];
  {
    const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    const int j = lane & 15, h = (lane >> 4) & 1, g = lane >> 5;
    const uint32_t row = (uint32_t)(8 * g + (j >> 2)), in = 32u * h + 8u * (j & 3);
#pragma unroll
    for (int i = 0; i < C::TM; ++i) a_rel[i] = lds_base + row * C::ROW_A + in + (uint32_t)(((wm * C::TM + i) ^ (j >> 2)) << 6);
#pragma unroll
    for (int i = 0; i < C::TN; ++i) b_rel[i] = lds_base + C::A_BYTES + row * C::ROW_B + in + (uint32_t)(((wn * C::TN + i) ^ (j >> 2)) << 6);
  }
  if (nk > 0) {
    WideFrag<C> f[2];
    wait_stages<C::DMA_ALL, C::STAGES - 2>(nk - 1);
    block_barrier();
    f[0].fetch(a_rel, b_rel, 0, 0);
    f[0].wait();
    int stage = 0, fill = C::STAGES - 1;
    for (int k = 0; k < nk; ++k) {
      const int next = stage + 1 == C::STAGES ? 0 : stage + 1;
      const uint32_t so = (uint32_t)stage * C::STAGE_BYTES, sn = (uint32_t)next * C::STAGE_BYTES;
      if (k + C::STAGES - 1 < nk) issue(k + C::STAGES - 1, fill);   // everybody has read what was there: the barrier of k - 1
      f[1].fetch(a_rel, b_rel, so + 16u * C::ROW_A, so + 16u * C::ROW_B);
      f[0].mma(acc);
      f[1].wait();
      if (k + 1 < nk) {
        wait_stages<C::DMA_ALL, C::STAGES - 2>(nk - 2 - k);   // this wave's share of stage k + 1 has landed
        block_barrier();                                      // everybody's has, and everybody has read stage k
        f[0].fetch(a_rel, b_rel, sn, sn);
      }
      f[1].mma(acc);
      if (k + 1 < nk) f[0].wait();
      stage = next;
      fill = fill + 1 == C::STAGES ? 0 : fill + 1;
    }
  }
  // Results leave through a patch of 32 rows for each wavefront, so that a store instruction writes two rows of 512 bytes, past
  // the L2, which keeps the operands that other tiles share.  us of 9 experts, straight from the accumulators (128 bytes a row at a
  // time) / so: 9216 x 4576 x 1720, whose rows end inside lines, 216 / 165, x 4608 x 1792 170 / 158, 65536 x 2048 x 1024 by 64 387 / 371.
  // Short lists of rows share nothing, and the L2 puts their lines together: 144 x 4576 x 1720 past it 79, through it 53
  // (but 4608 x 4576 x 1720 111 and 141).
  static_assert(C::WAVES * 32 * C::TN * 32 * 4 <= C::STAGES * C::STAGE_BYTES && C::TN == 4, "patches fit, rows of 128 columns");
  wait_vm<0>();
  __syncthreads();   // all reads of the stages are done
  float *patch = reinterpret_cast<float *>(lds) + wave * 32 * 32 * C::TN;
  const int c = lane & 31, g = lane >> 5;
  const int n = n0 + wn * 32 * C::TN + 4 * c;
#pragma unroll
  for (int i = 0; i < C::TM; ++i) {
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) patch[(8 * (q / 4) + 4 * g + q % 4) * 128 + j * 32 + c] = acc[i][j][q];
    __builtin_amdgcn_wave_barrier();
    const int m = m0 + (wm * C::TM + i) * 32 + g;
    f32x4_v *dst = reinterpret_cast<f32x4_v *>(t.dst + (int64_t)m * a.K + n);
    auto store = [&](auto past) {
#pragma unroll
      for (int r = 0; r < 32; r += 2) {
        const f32x4_v v = *reinterpret_cast<const f32x4_v *>(patch + (r + g) * 128 + 4 * c);
        if (m + r < a.N && n < a.K) {
          if constexpr (decltype(past)::value)
            __builtin_nontemporal_store(v, dst + (int64_t)r * a.K / 4);
          else
            dst[(int64_t)r * a.K / 4] = v;
        }
      }
    };
    if (last - first > 128) {
      store(std::true_type{});
      asm volatile("" ::: "memory");   // the compiler would make one of both kinds of store, the plain one
    } else {
      store(std::false_type{});
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename C> __global__ void __launch_bounds__(C::THREADS, C::TM * C::TN > 8 ? 1 : 2) k_expert_wgrad_wide(WgradArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[C::STAGES * C::STAGE_BYTES];
  wgrad_wide<C>(a, lds);
}

// Tiles of a gradient: fp32 64 x 64, bf16 128 x 256, or 128 x 128 where half of those 256 would be empty
struct WgradShape {
  int bm, bn;
};
WgradShape wgrad_shape(int dtype, int K) { return dtype == GEAR_F32 ? WgradShape{64, 64} : K <= 128 ? WgradShape{128, 128} : WgradShape{128, 256}; }
int64_t wgrad_tiles(const WgradShape &t, int N, int K) { return (int64_t)((N + t.bm - 1) / t.bm) * ((K + t.bn - 1) / t.bn); }

// Rows of a piece.  Two workgroups fit on each CU: 512 at a time.  (More in fp32, whose two stages leave room for five, which is
// for short lists, all latency: 2086 x 80 x 8064 by 61 experts 170 us, with four stages 256; pieces for 1024 at a time gain
// nothing.)  Where all experts' tiles are fewer than two rounds of that, rows are cut so that one layer gives one whole
// round, and experts, whose sizes the host does not know, pieces of up to two fair shares (fp32 one and a half).  us, uncut / cut:
// 65536 x 1024 x 1152 by one expert 832 / 180, 16384 x 1024 x 1152 by 8 uneven ones 93 / 74, by 8 even ones 64 (one and a half
// fair shares: 72 and 94), fp32 16384 x 512 x 576 by 8 103 (two: 135).
int wgrad_cut(int dtype, int64_t rows, int experts, int N, int K) {
  constexpr int64_t slots = 512;
  const int64_t tiles = wgrad_tiles(wgrad_shape(dtype, K), N, K), whole = rows < 1 ? 1 : rows;
  if (experts * tiles >= 2 * slots) return (int)whole;
  const int64_t at_once = tiles < slots ? slots / tiles : 1;
  int64_t cut = experts == 1 ? (rows + at_once - 1) / at_once : rows * tiles * (dtype == GEAR_F32 ? 3 : 4) / (2 * slots);
  cut = (cut + 31) / 32 * 32;
  // What a piece adds and writes has to be worth it.  us with 128 / 256 / 512 rows at least, fp32: 1000 x 72 x 320 by 5 11 / 13 / 14,
  // 8000 x 64 x 64 by 16 12 / 14 / 19, 1000 x 72 x 320 by one 10 / 12 / 16; bf16: 2000 x 512 x 576 by 8 26 / 19 / 17, 1000 x 1024 x 1152
  // by one 25 / 22 / 21.
  const int64_t least = dtype == GEAR_F32 ? 128 : experts == 1 ? 256 : experts * tiles < slots ? 512 : 1024;
  if (cut < least) cut = least;
  return (int)(cut < whole ? cut : whole);
}
int64_t wgrad_partials(int64_t rows, int experts, int cut) {   // pieces of experts that are cut, at most
  const int64_t pieces = (rows + cut - 1) / cut;
  return pieces <= 1 ? 0 : experts == 1 ? pieces : 2 * (rows / cut);
}

template <typename C> hipError_t launch(const WgradArgs &a, unsigned blocks, hipStream_t s) {
  hipLaunchKernelGGL(k_expert_wgrad<C>, dim3(blocks), dim3(C::THREADS), 0, s, a);
  return hipGetLastError();
}

bool wgrad_ok(int dtype, int64_t rows, int experts, int N, int K) {
  return (dtype == GEAR_F32 || dtype == GEAR_BF16) && rows >= 0 && rows <= (1 << 30) && experts >= 1 && experts <= GEAR_MAX_EXPERTS &&
         N >= 8 && N % 8 == 0 && K >= 8 && K % 8 == 0 && N < (1 << 20) && K < (1 << 20) &&
         (int64_t)experts * ((N + 63) / 64) * ((K + 63) / 64) <= (1 << 23);   // tiles are counted in 32 bits (cut only below 1024)
}

}  // namespace
}  // namespace gear

using namespace gear;

extern "C" size_t gear_expert_wgrad_workspace_bytes(int32_t dtype, int64_t rows, int32_t experts, int32_t N, int32_t K) {
  if (!wgrad_ok(dtype, rows, experts, N, K)) return 0;
  const size_t bytes = (size_t)wgrad_partials(rows, experts, wgrad_cut(dtype, rows, experts, N, K)) * N * K * sizeof(float);
  return bytes < 256 ? 256 : (bytes + 255) & ~(size_t)255;
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
  const int cut = wgrad_cut(a->dtype, a->rows, a->experts, a->N, a->K);
  const WgradShape shape = wgrad_shape(a->dtype, a->K);
  const WgradArgs w = {a->dy, a->x, a->off, a->dw, a->ld_dy, a->ld_x, (int)a->rows, a->K, a->N, a->experts, a->status,
                       static_cast<float *>(workspace), cut, a->keep_status};
  hipStream_t s = (hipStream_t)stream;
  // rows that are not cut add no piece: the largest gradients have as many tiles as a launch may have threads for
  const int64_t pieces = a->off ? a->experts + (cut < a->rows ? a->rows / cut : 0) : (a->rows + cut - 1) / cut;
  const unsigned blocks = wgrad_blocks((pieces > 0 ? pieces : 1) * wgrad_tiles(shape, a->N, a->K));
  if (a->dtype == GEAR_F32) {
    if (launch<TnTile<float, 1, 1, 2>>(w, blocks, s) != hipSuccess) return GEAR_ERR_HIP;
  } else if (shape.bn == 128) {
    if (launch<TnTile<bf16_t, 2, 2, 3>>(w, blocks, s) != hipSuccess) return GEAR_ERR_HIP;
  } else {
    using Wide = WideTile<2, 4, 2, 2, 3>;
    hipLaunchKernelGGL(k_expert_wgrad_wide<Wide>, dim3(blocks), dim3(Wide::THREADS), 0, s, w);
    if (hipGetLastError() != hipSuccess) return GEAR_ERR_HIP;
  }
  if (wgrad_partials(a->rows, a->experts, cut) > 0) {
    const int64_t vec = (int64_t)a->N * a->K / 4;
    // few columns are few workgroups, each with a long walk: us by one share / 16, 65536 x 72 x 128 bf16 34 / 16, 9000 x 320 x 72 14 / 12, but
    // 30000 x 1024 x 128 by 4 28 / 36
    if (vec * a->experts <= 16384) {
      hipLaunchKernelGGL(k_wgrad_sum<16>, dim3((unsigned)((vec + 15) / 16), (unsigned)a->experts), dim3(256), 0, s, w);
    } else {
      // 4096 in all, as those of experts that are not cut have nothing to do: 16384 x 1024 x 1152 by 8 69 / 67
      const int64_t want = (vec + 255) / 256, most = 4096 / a->experts + 1;
      hipLaunchKernelGGL(k_wgrad_sum<1>, dim3((unsigned)(want < most ? want : most), (unsigned)a->experts), dim3(256), 0, s, w);
    }
    if (hipGetLastError() != hipSuccess) return GEAR_ERR_HIP;
  }
  return GEAR_OK;
}
