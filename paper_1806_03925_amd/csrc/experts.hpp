// What the products grouped by expert share: where an expert's rows are, and which tile is a workgroup's (gfx950 only).
#pragma once

#include "tn_tile.hpp"

namespace gear {
namespace {

// The tile of a workgroup: rows [m0, m_end) of expert e from m0 on, column tile n_tile; of its rows the first half (part 0), the second
// (1) or all (-1).  bad: off is not a CSR index.
struct ExpertTile {
  int e, m0, m_end, n_tile;
  bool have, bad;
  int part;
};

// Workgroups of the largest shape of tile that the device runs at a time, two for each CU.  If a few tiles are left for a last round,
// each of them is two workgroups' (`halves`: the shape allows it), at most one for each CU, so that it is over sooner.  us whole / in halves:
// 17408 x 1024 x 1152 bf16 (32 tiles left) 46.3 / 41.6, 20480 x 1024 x 1152 (128) 47.7 / 43.5, 9216 x 2048 x 4096 (64) 145 / 133; with
// about 150 left, 16384 x 1152 x 1024 by 8 experts, 44.7 / 47.5.
constexpr int kSlots = 512, kHalved = kSlots / 4;

__device__ __forceinline__ int wave_add(int v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// whether off is a CSR index into `rows` rows; every lane of a wavefront gets the answer
__device__ __forceinline__ bool offsets_ok(const int32_t *__restrict__ off, int experts, int rows, int lane) {
  bool bad = off[0] != 0;
  for (int e0 = 0; e0 < experts; e0 += kWave) {
    const int e = min(e0 + lane, experts - 1), a = off[e], b = off[e + 1];
    bad = bad || __any(a < 0 || b < a || b > rows);
  }
  return !bad;
}

// Offsets that are no CSR index are reported by one thread; those that are only where nobody shares the word (gear.h).
__device__ __forceinline__ void report(bool bad, int32_t *status, int keep) {
  if (status && blockIdx.x == 0 && threadIdx.x == 0 && (bad || !keep)) *status = bad ? GEAR_ERR_RANGE : GEAR_OK;
}

// Tile t of m_tiles x n_tiles: kGroupRows row tiles are walked down, column by column, before the next ones.  The 64 tiles
// that an XCD works on at a time then read 8 strips of rows and 8 of weights through its L2, not two and 32.
constexpr int kGroupRows = 8;
struct TileAt {
  int m, n;
};
__device__ __forceinline__ TileAt tile_at(int t, int m_tiles, int n_tiles) {
  const int first = t / (kGroupRows * n_tiles) * kGroupRows, in = t % (kGroupRows * n_tiles), rows = min(kGroupRows, m_tiles - first);
  return {first + in % rows, in / rows};
}

// Row tiles of `edge` rows are counted expert by expert; the workgroups' tiles are in the order of tile_at after
// neighbouring ones have been gathered on one XCD.  Every wavefront looks at all offsets, 64 at a time, so that all
// workgroups agree on whether they are a CSR index.
__device__ __forceinline__ ExpertTile expert_tile(const int32_t *__restrict__ off, int experts, int rows, int edge, int n_tiles,
                                                  int block, int lane, bool halves) {
  ExpertTile r = {0, 0, 0, 0, false, false, -1};
  auto tile_of = [&](int tiles) {   // the tile that `block` works on, or one beyond them
    const int whole = tiles / kSlots * kSlots, rest = tiles - whole;
    if (!halves || whole == 0 || rest > kHalved || block < whole) return block;
    if (block >= whole + 2 * rest) return tiles;
    r.part = block >= whole + rest;
    return block - r.part * rest;
  };
  if (!off) {
    const int m_tiles = (rows + edge - 1) / edge;
    const int tile = tile_of(m_tiles * n_tiles);
    if (tile >= m_tiles * n_tiles) return r;
    const TileAt t = tile_at(xcd_remap(tile, m_tiles * n_tiles), m_tiles, n_tiles);
    r.m0 = t.m * edge, r.m_end = rows, r.n_tile = t.n, r.have = true;
    return r;
  }
  int total = 0;
  bool bad = off[0] != 0;
  for (int e0 = 0; e0 < experts; e0 += kWave) {
    const int e = min(e0 + lane, experts - 1), a = off[e], b = off[e + 1];
    const bool wrong = a < 0 || b < a || b > rows;
    bad = bad || __any(wrong);
    total += wave_add(wrong || e0 + lane >= experts ? 0 : (b - a + edge - 1) / edge);
  }
  r.bad = bad;
  total = __builtin_amdgcn_readfirstlane(total);   // the same in all lanes: what follows from it is scalar
  const int tile = tile_of(total * n_tiles);
  if (bad || tile >= total * n_tiles) return r;
  const TileAt t = tile_at(xcd_remap(tile, total * n_tiles), total, n_tiles);
  const int want = t.m;
  int before = 0;
  for (int e0 = 0; e0 < experts; e0 += kWave) {
    const int e = min(e0 + lane, experts - 1), a = off[e], b = off[e + 1];
    const int mine = e0 + lane >= experts ? 0 : (b - a + edge - 1) / edge;
    int upto = mine;   // tiles of this and the lower lanes' experts
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int v = __shfl_up(upto, o, kWave);
      if (lane >= o) upto += v;
    }
    const unsigned long long m = __ballot(before + upto > want);
    if (m) {
      const int at = __builtin_ctzll(m);
      r.e = e0 + at;
      r.m0 = __shfl(a, at, kWave) + (want - before - __shfl(upto - mine, at, kWave)) * edge;
      r.m_end = __shfl(b, at, kWave);
      break;
    }
    before += __shfl(upto, kWave - 1, kWave);
  }
  r.e = __builtin_amdgcn_readfirstlane(r.e);
  r.m0 = __builtin_amdgcn_readfirstlane(r.m0);
  r.m_end = __builtin_amdgcn_readfirstlane(r.m_end);
  r.n_tile = t.n;
  r.have = true;
  return r;
}

}  // namespace
}  // namespace gear
