// Routing of rows to experts: scores, choice of k experts a row, weights, and the order of all (row, slot) pairs by expert; its
// gradient (gear.h has the definitions).
//
// A row is a team of LPR lanes' (8, 16, 32 or 64 of one wavefront), V logits a lane, all in registers from the one time they are
// read.  What decides the choice is score + bias, and two experts' sums lie closer together than fp32 resolves in one row of some
// hundred thousand.  So the choice is made twice at most: from fp32, with a bound on its error, and again by the definition, in
// fp64, by the wavefronts that have a row with two neighbours in its order closer than that.
//
// The choice from fp32.  A value becomes a whole number: how far it lies above a bound under the k-th, in 2^-23 of the way to the
// largest (2^-21 for 1024 experts), and behind that its expert's tag, so that one comparison moves both and equal ones come in the order of their experts.  The
// conversion keeps the order, if not every difference, so only neighbours with the same or (where scores are added up) too
// near numbers are in doubt.  A lane sorts its own by a network.  Where k is at most 8, teams then merge lists of 8 lane by lane,
// log2(LPR) times, and keep the best of what falls off; else k + 1 times the largest of the team's first ones is taken and its lane moves
// on.  Bound by these instructions: 65536 rows of 256 fp32 logits with a bias, k = 8, take 31.8 us, 1400 vector instructions for eight rows, which keep the
// vector pipes busy for three quarters of a wavefront's life; its 74 MB would take 15.7.  (k times the largest of all in fp64: 114 us; one by one from sorted
// numbers: 48.)  A row in doubt costs its wavefront 3 to 7 us, one in a thousand to ten thousand of random ones; with groups one such row is a
// quarter of a launch over 10001 rows (25.0 us; 20 without).
//
// The order of the pairs is a counting sort by expert.  A workgroup takes a run of rows and counts its experts; a second launch
// with the same runs finds from all counts where each run's pairs begin, ranks them (equal experts in a wavefront by ballots,
// wavefronts in order) and writes their places.  Batches of one run are both in one launch.  No atomic decides an order: those on
// counts in LDS only add.  65536 x 8 pairs 9.0 us: five steps one behind the other, each of them latency (without reading the counts, or
// without ranking, it takes as long within a tenth).
#include "lanes.hpp"

#include <cmath>
#include <type_traits>

namespace gear {
namespace {

constexpr int kMaxRuns = 256;        // one for each CU
// threads of a workgroup, at most: what its registers and, with groups, its LDS allow
constexpr int threads_of(int lpr, int v, bool grouped) { return grouped && lpr == kWave ? 256 : grouped || v > 16 ? 512 : 1024; }
constexpr int kMaxGroups = GEAR_MAX_GROUPS;

struct RouteArgs {
  int64_t rows, ld;
  int run;                           // rows of a workgroup
  int experts, k, softmax, groups, kept, best, renormalise;
  float scale;
  const void *logits;
  const float *bias;
  const int32_t *n;
  int32_t *expert;
  float *weight;
  int32_t *off, *place;
  void *count;                       // [experts x runs_ld] of 16 bits, of 32 where a run has more rows than that holds
};

__host__ __device__ constexpr int runs_ld(int runs) { return (runs + 7) / 8 * 8; }
__host__ __device__ constexpr bool narrow(int run) { return run <= 0xffff; }   // an expert is chosen once a row

// ---- over a team: every lane gets the result, and every lane of the wavefront takes part -------------------------------
template <int CTRL> __device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true); }
// The other half of a group of 2 << STEP lanes, in some order: what it holds is the same in all of its lanes.
template <int STEP> __device__ __forceinline__ int across(int v) {
  if constexpr (STEP == 0) return moved<0xb1>(v);         // lanes 1 0 3 2
  if constexpr (STEP == 1) return moved<0x4e>(v);         // lanes 2 3 0 1
  if constexpr (STEP == 2) return moved<0x141>(v);        // eight lanes backwards
  if constexpr (STEP == 3) return moved<0x140>(v);        // sixteen
  return __shfl_xor(v, 1 << STEP, kWave);
}
template <int STEP> __device__ __forceinline__ float across(float v) { return __int_as_float(across<STEP>(__float_as_int(v))); }
template <int STEP> __device__ __forceinline__ double across(double v) {
  return __hiloint2double(across<STEP>(__double2hiint(v)), across<STEP>(__double2loint(v)));
}
template <int LPR, int STEP = 0, typename V, typename F> __device__ __forceinline__ V team(V v, F &&f) {
  if constexpr ((1 << STEP) < LPR)
    return team<LPR, STEP + 1>(f(v, across<STEP>(v)), f);
  else
    return v;
}
template <int LPR> __device__ __forceinline__ float team_max(float v) {
  return team<LPR>(v, [](float x, float y) { return fmaxf(x, y); });
}
template <int LPR> __device__ __forceinline__ float team_min(float v) {
  return team<LPR>(v, [](float x, float y) { return fminf(x, y); });
}
template <int LPR> __device__ __forceinline__ int team_max(int v) {
  return team<LPR>(v, [](int x, int y) { return max(x, y); });
}
template <int LPR> __device__ __forceinline__ float team_add(float v) {
  return team<LPR>(v, [](float x, float y) { return x + y; });
}
template <int LPR> __device__ __forceinline__ uint64_t team_ballot(bool v) {   // of this lane's team, its first lane in bit 0
  const uint64_t m = __ballot(v);
  if constexpr (LPR == 64) return m;
  return m >> (threadIdx.x & 63 & ~(LPR - 1)) & ((1ull << LPR) - 1);
}
template <int LPR> __device__ __forceinline__ bool team_any(bool v) { return team_ballot<LPR>(v) != 0; }

// over a wavefront, in fp64: within 16 lanes, then the four
template <typename F> __device__ __forceinline__ double wave_of(double v, F &&f) {
  v = team<16>(v, f);
  double r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 16 * i), __builtin_amdgcn_readlane(__double2loint(v), 16 * i));
  return f(f(r[0], r[1]), f(r[2], r[3]));
}
// The largest of values [v][lane] and its number 64 v + lane, the lowest of equals; -1 where all are -inf.
struct Best {
  double value;
  int index;
};
template <int V> __device__ __forceinline__ Best wave_best(const double (&value)[V]) {
  double high = value[0];
#pragma unroll
  for (int v = 1; v < V; ++v) high = fmax(high, value[v]);
  Best b = {wave_of(high, [](double x, double y) { return fmax(x, y); }), -1};
  if (!(b.value > -INFINITY)) return b;
#pragma unroll
  for (int v = V - 1; v >= 0; --v) {
    const uint64_t m = __ballot(value[v] == b.value);
    if (m) b.index = v * kWave + __builtin_ctzll(m);
  }
  return b;
}

// ---- scores ---------------------------------------------------------------------------------------------------------
// in fp64, for the choice: softmax without its sum, or sigmoid
__device__ __forceinline__ double exact_score(float l, bool softmax, float top) {
  return softmax ? exp((double)l - (double)top) : 1.0 / (1.0 + exp(-(double)l));
}
__device__ __forceinline__ float quick_exp(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504f); }
// A chosen expert's share: its score up to a factor that is the same for all of its row where `relative`.  No sum of such scores
// vanishes then, however small they are, when `top` is the largest chosen logit.
__device__ __forceinline__ float share(float l, bool softmax, float top, bool relative) {
  if (softmax) return expf(l - top);
  if (l > 0.0f) return 1.0f / (1.0f + expf(-l));
  const float shift = relative ? fminf(top, 0.0f) : 0.0f;
  return expf(l - shift) / (1.0f + expf(l));
}

// ---- whole numbers that say whose they are ------------------------------------------------------------------------------
// TAG last bits are the expert's number turned round, so that the lower one of equal values' experts has the larger number; the others
// are 1 at the bound and STEPS + 1 at the largest value, 0 below the bound.
template <int TAG> struct Numbers {
  static constexpr int kLast = (1 << TAG) - 1, BITS = 31 - TAG < 23 ? 31 - TAG : 23;
  static constexpr float STEPS = (float)((1 << BITS) - 4);
  static __device__ __forceinline__ int of(float v, float bound, float steps, int expert) {   // v: -inf for who may not be chosen
    return (int)fmaxf(fmaf(v - bound, steps, 1.0f), 0.0f) << TAG | (kLast - expert);
  }
  static __device__ __forceinline__ bool is_somebody(int number) { return number > kLast; }
  static __device__ __forceinline__ int expert_of(int number) { return kLast - (number & kLast); }
  static __device__ __forceinline__ int height_of(int number) { return number >> TAG; }
};

// descending, by odd-even merges
template <int V> struct Sorter {
  template <int I, int J> static __device__ __forceinline__ void exchange(int (&k)[V]) {
    const int a = max(k[I], k[J]), b = min(k[I], k[J]);
    k[I] = a, k[J] = b;
  }
  template <int I, int END, int STEP, int R> static __device__ __forceinline__ void row(int (&k)[V]) {
    if constexpr (I + R < END) {
      exchange<I, I + R>(k);
      row<I + STEP, END, STEP, R>(k);
    }
  }
  template <int LO, int N, int R> static __device__ __forceinline__ void merge(int (&k)[V]) {
    if constexpr (2 * R < N) {
      merge<LO, N, 2 * R>(k);
      merge<LO + R, N, 2 * R>(k);
      row<LO + R, LO + N, 2 * R, R>(k);
    } else {
      exchange<LO, LO + R>(k);
    }
  }
  template <int LO = 0, int N = V> static __device__ __forceinline__ void sort(int (&k)[V]) {
    if constexpr (N > 1) {
      sort<LO, N / 2>(k);
      sort<LO + N / 2, N / 2>(k);
      merge<LO, N, 1>(k);
    }
  }
};

// The first eight of two lanes' lists of eight, and the largest of all that are in neither of their lists.
constexpr int kList = 8;
template <int STEP, int LPR> __device__ __forceinline__ void merge_lists(int (&mine)[kList], int &rest) {
  if constexpr ((1 << STEP) < LPR) {
    int all[kList];
    rest = max(rest, across<STEP>(rest));
#pragma unroll
    for (int i = 0; i < kList; ++i) {
      const int other = across<STEP>(mine[kList - 1 - i]);
      all[i] = max(mine[i], other);
      rest = max(rest, min(mine[i], other));
    }
#pragma unroll
    for (int apart = kList / 2; apart; apart /= 2)   // they fall, then rise: halves against each other
#pragma unroll
      for (int i = 0; i < kList; ++i)
        if (!(i & apart)) {
          const int a = max(all[i], all[i + apart]), b = min(all[i], all[i + apart]);
          all[i] = a, all[i + apart] = b;
        }
#pragma unroll
    for (int i = 0; i < kList; ++i) mine[i] = all[i];
    merge_lists<STEP + 1, LPR>(mine, rest);
  }
}

// ---- order of the pairs -------------------------------------------------------------------------------------------
// A wavefront's pairs, one behind the other, 64 at a time, four times 64 requested together; kept between counting and placing where these are all.
__host__ __device__ constexpr int rankers_of(int experts) { return experts <= 512 ? 16 : 8; }   // wavefronts that rank: their counts fit in LDS
__host__ __device__ constexpr int place_words(int experts) { return experts * (2 + rankers_of(experts)); }   // of LDS
struct Slice {
  static constexpr int AHEAD = 4, STEP = AHEAD * kWave;
  int64_t begin, end;
  int e[AHEAD];
  __device__ __forceinline__ Slice(const RouteArgs &a, int64_t first, int64_t last) {
    const unsigned wave = threadIdx.x / kWave, waves = min((int)blockDim.x / kWave, rankers_of(a.experts));
    const unsigned pairs = (unsigned)(last - first) * (unsigned)a.k, per = (pairs + waves - 1) / waves;   // at most 2^30 / 256 rows of 32
    begin = first * a.k + min(wave * per, pairs);
    end = wave < waves ? first * a.k + min((wave + 1) * per, pairs) : begin;
  }
  __device__ __forceinline__ void request(const RouteArgs &a, int64_t i0) {
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      const int64_t i = i0 + p * kWave + (threadIdx.x & 63);
      e[p] = i < end ? a.expert[i] : -1;
    }
  }
};

// Places of the pairs of rows [first, last), those of run number `run`; `slice`'s first pairs are requested.  On entry s_all[e] is the number of expert e's
// pairs in all runs and s_base[e] that in the runs before this one; s_wave [rankers x experts] is zero.
__device__ __forceinline__ void places(const RouteArgs &a, int run, Slice &slice, int32_t *s_base, int32_t *s_all, int32_t *s_wave) {
  const int threads = blockDim.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, E = a.experts, waves = min(threads / kWave, rankers_of(E));
  __syncthreads();
  if (wave == 0) {   // where each expert begins
    int begin = 0;
    for (int e0 = 0; e0 < E; e0 += kWave) {
      const int e = e0 + lane, mine = e < E ? s_all[e] : 0;
      const int upto = wave_scan(mine);
      if (e < E) {
        s_base[e] += begin + upto - mine;
        if (run == 0) a.off[e] = begin + upto - mine;
      }
      begin += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    if (run == 0 && lane == 0) a.off[E] = begin;
  }
  int32_t *mine = s_wave + min(wave, waves - 1) * E;
  for (int64_t i0 = slice.begin; i0 < slice.end; i0 += Slice::STEP) {
    if (i0 > slice.begin) slice.request(a, i0);
#pragma unroll
    for (int p = 0; p < Slice::AHEAD; ++p)
      if (slice.e[p] >= 0) atomicAdd(mine + slice.e[p], 1);
  }
  __syncthreads();
  for (int x = threadIdx.x; x < E; x += threads) {
    int c[16], at = s_base[x];
    static_assert(rankers_of(1) == 16, "all counts requested together");
#pragma unroll
    for (int w = 0; w < 16; ++w) c[w] = w < waves ? s_wave[w * E + x] : 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < waves) s_wave[w * E + x] = at;
      at += c[w];
    }
  }
  __syncthreads();
  int bits = 0;
  while ((1 << bits) < E) ++bits;
  for (int64_t i0 = slice.begin; i0 < slice.end; i0 += Slice::STEP) {
    if (slice.end - slice.begin > Slice::STEP) slice.request(a, i0);
#pragma unroll
    for (int p = 0; p < Slice::AHEAD; ++p) {
      const int64_t i = i0 + p * kWave + lane;
      if (i0 + p * kWave >= slice.end) break;
      const int e = slice.e[p];
      uint64_t same = __ballot(e >= 0);   // lanes of the same expert
      for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((e >> b) & 1);
        same &= (e >> b) & 1 ? set : ~set;
      }
      const int rank = __popcll(same & ((1ull << lane) - 1));
      int at = -1;
      if (e >= 0) at = mine[e] + rank;
      asm volatile("" ::: "memory");   // every lane has read before one adds
      if (e >= 0 && rank == 0) mine[e] += __popcll(same);
      if (i < slice.end) a.place[i] = at;
    }
  }
}

// The choice of one row by the definition, in fp64, by a whole wavefront: lane j gets the j-th expert, -1 where there is none.  The row is
// read again: its values in fp64 are few for 64 lanes, and nobody keeps registers for them who does not need them.  scratch: MAX_E doubles of LDS
// of this wavefront's, for groups.
template <typename T, int MAX_E, bool GROUPED> __device__ __forceinline__ int choose_exactly(const RouteArgs &a, int64_t row, float top, double *scratch) {
  constexpr int V = MAX_E / kWave;
  const double kNone = -INFINITY;
  const int lane = threadIdx.x & 63, E = a.experts;
  const T *x = static_cast<const T *>(a.logits) + row * a.ld;
  float lg[V];
  double order[V], sum = 1.0;
#pragma unroll
  for (int v = 0; v < V; ++v) lg[v] = v * kWave + lane < E ? to_f32(x[v * kWave + lane]) : -INFINITY;
  if (a.softmax && (a.bias || GROUPED)) {
    sum = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) sum += exact_score(lg[v], true, top);
    sum = wave_of(sum, [](double x, double y) { return x + y; });
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = v * kWave + lane;
    const float bias = a.bias && e < E ? a.bias[e] : 0.0f;
    order[v] = !(lg[v] > -INFINITY && bias > -INFINITY) ? kNone
               : a.bias || GROUPED                      ? exact_score(lg[v], a.softmax, top) / sum + (double)bias
                                                        : (double)lg[v];
  }
  if constexpr (GROUPED) {
    const int per = E / a.groups;
#pragma unroll
    for (int v = 0; v < V; ++v) scratch[v * kWave + lane] = order[v];
    asm volatile("" ::: "memory");   // LDS accesses of one wavefront come in order
    __builtin_amdgcn_wave_barrier();
    double worth[1] = {kNone};       // lane q: group q's value
    if (lane < a.groups) {
      double one = kNone, two = kNone;
#pragma unroll 4
      for (int c = 0; c < per; ++c) {
        const double v = scratch[lane * per + c];
        two = fmax(two, fmin(one, v));
        one = fmax(one, v);
      }
      worth[0] = a.best == 2 && two > kNone ? one + two : one;
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    uint64_t keep = 0;
    for (int j = 0; j < a.kept; ++j) {
      const Best b = wave_best(worth);
      if (b.index < 0) break;
      keep |= 1ull << b.index;
      if (lane == b.index) worth[0] = kNone;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = min(v * kWave + lane, E - 1);
      if (!(keep >> (e / per) & 1)) order[v] = kNone;
      if (order[v] > kNone && !a.bias) order[v] = (double)lg[v];
    }
  }
  int chosen = -1;
  for (int j = 0; j < a.k; ++j) {
    const Best b = wave_best(order);
    if (b.index < 0) break;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v * kWave + lane == b.index) order[v] = kNone;
    if (lane == j) chosen = b.index;
  }
  return chosen;
}

template <typename T, int LPR, int V, bool WIDE, bool GROUPED, bool FEW>   // FEW: k is at most kList
__global__ void __launch_bounds__(threads_of(LPR, V, GROUPED)) k_route(RouteArgs a) {
  constexpr int MAX_E = LPR * V, SLOTS = !FEW && LPR < GEAR_MAX_CHOSEN ? GEAR_MAX_CHOSEN / LPR : 1;   // of a lane
  static_assert(!WIDE || V % 4 == 0, "four neighbouring logits a load");
  static_assert(GEAR_MAX_EXPERTS <= 1024 && LPR >= kList, "a tag's bits; a lane for each of a list");
  constexpr int TAG = MAX_E <= 32 ? 5 : MAX_E <= 64 ? 6 : MAX_E <= 128 ? 7 : MAX_E <= 256 ? 8 : MAX_E <= 512 ? 9 : 10;
  static_assert(MAX_E <= 1 << TAG, "an expert's number fits");
  using Num = Numbers<TAG>;
  extern __shared__ int32_t s_words[];                          // [experts] counts, then what places() needs
  // a row's values for each team; a wavefront's are room for those of one row in 64 bits
  constexpr int TEAM_VALUES = LPR == kWave ? 2 * MAX_E : MAX_E, WAVE_VALUES = kWave / LPR * TEAM_VALUES;
  static_assert(WAVE_VALUES >= 2 * MAX_E, "doubles");
  __shared__ __attribute__((aligned(16))) float s_value[GROUPED ? threads_of(LPR, V, true) / kWave * WAVE_VALUES : 4];
  const int threads = blockDim.x, teams = threads / LPR;
  const int l = threadIdx.x % LPR, my_team = threadIdx.x / LPR, lane0_of_mine = threadIdx.x & 63 & ~(LPR - 1), E = a.experts;
  for (int e = threadIdx.x; e < E; e += threads) s_words[e] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * a.run, last = min(a.rows, first + a.run);
  const int64_t used = min(last, a.n ? (int64_t)max(*a.n, 0) : last);
  auto index = [&](int v) { return WIDE ? (v / 4) * (LPR * 4) + l * 4 + v % 4 : v * LPR + l; };
  float bias[V];                              // -inf where it may not be chosen
#pragma unroll
  for (int v = 0; v < V; ++v) {
    bias[v] = a.bias && index(v) < E ? a.bias[index(v)] : 0.0f;
    if (!(bias[v] > -INFINITY)) bias[v] = -INFINITY;
  }
  float most_bias = 0.0f;                     // of the finite ones' magnitudes
#pragma unroll
  for (int v = 0; v < V; ++v) most_bias = fmaxf(most_bias, fabsf(bias[v]) < INFINITY ? fabsf(bias[v]) : 0.0f);
  most_bias = team_max<LPR>(most_bias);
  const bool scores = a.bias || GROUPED;      // the choice looks at them

  float lg[V];
  auto load = [&](int64_t row) {
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    auto four = [&](int v) {
      if constexpr (sizeof(T) == 4) {
        const float4 f = *reinterpret_cast<const float4 *>(x + index(v));
        lg[v] = f.x, lg[v + 1] = f.y, lg[v + 2] = f.z, lg[v + 3] = f.w;
      } else {
        const uint2 f = *reinterpret_cast<const uint2 *>(x + index(v));
        lg[v] = __uint_as_float(f.x << 16), lg[v + 1] = __uint_as_float(f.x & 0xffff0000u);
        lg[v + 2] = __uint_as_float(f.y << 16), lg[v + 3] = __uint_as_float(f.y & 0xffff0000u);
      }
    };
    if (WIDE && E == MAX_E && __all(row < used)) {   // the whole wavefront: nothing to fill in
#pragma unroll
      for (int v = 0; v < V; v += 4) four(v);
      return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) lg[v] = -INFINITY;
    if (row >= used) return;
    if constexpr (WIDE) {
#pragma unroll
      for (int v = 0; v < V; v += 4)
        if (index(v) < E) four(v);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (index(v) < E) lg[v] = to_f32(x[index(v)]);
    }
  };
  load(first + my_team);
  for (int64_t row0 = first; row0 < last; row0 += teams) {
    const int64_t row = row0 + my_team;
    bool broken = false;
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; v += 2) broken |= __builtin_isunordered(lg[v], lg[v + 1]);   // either is NaN
#pragma unroll
    for (int v = 0; v < V; ++v) top = fmaxf(top, lg[v]);
    top = team_max<LPR>(top);
    broken = team_any<LPR>(broken) || (a.softmax && top == INFINITY);
    const bool empty = broken || top == -INFINITY;   // no expert for this row, whatever the biases
    const float from = empty ? 0.0f : top;
    float inv = 1.0f;                                // of the sum of exp(l - top)
    float value[V];
    if (scores || (a.softmax && !a.renormalise)) {
      if (a.softmax) {
        float sum[2] = {0.0f, 0.0f};   // half as many additions one behind the other
#pragma unroll
        for (int v = 0; v < V; ++v) {
          value[v] = quick_exp(lg[v] - from);
          sum[v & 1] += value[v];
        }
        inv = empty ? 0.0f : 1.0f / team_add<LPR>(sum[0] + sum[1]);
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) value[v] = __builtin_amdgcn_rcpf(1.0f + quick_exp(-lg[v]));
      }
#pragma unroll
      for (int v = 0; v < V; ++v) value[v] = fmaf(value[v], inv, bias[v]);
    }
    // How far apart two values of which one is v have to be, to be in their true order.  In units of 2^-23 of itself an exponential is off by 1.25 d + 1, d = top - l (its
    // argument, the factor log2 e, the instruction), the sum by half a unit for each of V / 2 + 7 additions and by what its terms are off by on their average, at most 7 (the mean of d is
    // below 4.5 whatever the scores of up to 1024 experts), the quotient and the product by 1 each: s (1.25 d + COEF), s at most |v| and the largest bias, and the
    // largest score, `inv` (all that counts beside a bias far beyond the scores, which parks its expert: else every row would be in doubt), s d at most 0.37 of `inv`.  A sigmoid is off by 2.1 2^-23 (an exponential's error times s (1 - s), an addition, the reciprocal).  And a sum with a bias is rounded.
    constexpr float COEF = 10.0f + 0.5f * (V / 2 + 7);
    auto apart = [&](float v) {
      return a.softmax ? 0x1p-22f * (COEF * fminf(inv, fabsf(v) + most_bias) + 0.5f * (inv + fabsf(v))) : 0x1.1p-21f + 0x1p-22f * fabsf(v);
    };
    bool unsure = false;
    uint64_t keep = ~0ull;
    if constexpr (GROUPED) {
      const int per = E / a.groups;
      float *mine = s_value + my_team * TEAM_VALUES;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (index(v) < E) mine[index(v)] = !empty && fminf(lg[v], bias[v]) > -INFINITY ? value[v] : -INFINITY;
      asm volatile("" ::: "memory");   // a team is part of one wavefront, whose LDS accesses come in order
      __builtin_amdgcn_wave_barrier();
      float worth[kMaxGroups / LPR], cancelled = 0.0f;   // what vanishes where two values of a group have different signs: half of it
#pragma unroll
      for (int i = 0; i < kMaxGroups / LPR; ++i) {
        const int q = l + i * LPR;
        worth[i] = -INFINITY;
        if (q < a.groups) {
          float one = -INFINITY, two = -INFINITY;
#pragma unroll 4
          for (int c = 0; c < per; ++c) {
            const float v = mine[q * per + c];
            two = fmaxf(two, fminf(one, v));
            one = fmaxf(one, v);
          }
          worth[i] = a.best == 2 && two > -INFINITY ? fmaxf(one + two, -0x1.fffffep127f) : one;   // below fp32's range is still eligible
          if (two > -INFINITY) cancelled = fmaxf(cancelled, fminf(one, -two));
        }
      }
      if (a.best == 2) cancelled = team_max<LPR>(cancelled);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
      keep = 0;
      float before = 0.0f;
      for (int j = 0; j <= a.kept; ++j) {
        float best = worth[0];
#pragma unroll
        for (int i = 1; i < kMaxGroups / LPR; ++i) best = fmaxf(best, worth[i]);
        const float mine_best = best;
        best = team_max<LPR>(best);
        if (!(best > -INFINITY)) continue;
        if (j == a.kept) {   // only between the last that is kept and the first that is not does the order matter; two scores and two biases make a sum,
                             // and each of them is rounded by itself before
          unsure = !(before - best > (a.best == 2 ? 3.0f * (apart(before) + apart(best)) + 0x1p-21f * cancelled : apart(before) + apart(best)) +
                                         0x1p-22f * (fabsf(before) + fabsf(best)));
          continue;
        }
        before = best;
        // one of the groups of that value: the others' turn comes next
        const bool is_mine = mine_best == best && (threadIdx.x & (LPR - 1)) == __builtin_ctzll(team_ballot<LPR>(mine_best == best) | 1ull << 63);
        int taken = -1;
#pragma unroll
        for (int i = kMaxGroups / LPR - 1; i >= 0; --i)
          if (is_mine && worth[i] == best) taken = l + i * LPR;
#pragma unroll
        for (int i = 0; i < kMaxGroups / LPR; ++i)
          if (l + i * LPR == taken) worth[i] = -INFINITY;
        keep |= 1ull << team_max<LPR>(taken);
      }
    }
    // what decides, -inf where it may not be chosen
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!a.bias)
        value[v] = lg[v];
      else if (!(lg[v] > -INFINITY))
        value[v] = -INFINITY;
      if constexpr (GROUPED)
        if (!(keep >> (min(index(v), E - 1) / (E / a.groups)) & 1)) value[v] = -INFINITY;
    }
    if (row0 + teams < last) load(row + teams);     // on their way while these are sorted
    // The least of the largest values of all lanes, or of all lanes' halves, is reached by LPR values, or twice as many: more than the k + 1 that a list of eight is
    // about.  Where there is no value in one of these, or k is larger, nobody eligible lies below the bound.
    constexpr int PART = LPR > kList ? V : V / 2;
    float high = -INFINITY, bound = INFINITY;
#pragma unroll
    for (int p = 0; p < V; p += PART) {
      float most = -INFINITY;
#pragma unroll
      for (int v = p; v < p + PART; ++v) most = fmaxf(most, value[v]);
      high = fmaxf(high, most);
      bound = fminf(bound, most);
    }
    bound = team_min<LPR>(bound);
    high = team_max<LPR>(high);
    if (!FEW || __any(!(bound > -INFINITY))) {
      asm volatile("" ::: "memory");   // a branch, not a choice of results
      float low = INFINITY;
#pragma unroll
      for (int v = 0; v < V; ++v) low = fminf(low, value[v] > -INFINITY ? value[v] : INFINITY);
      low = team_min<LPR>(low);
      if (!FEW || !(bound > -INFINITY)) bound = low;
    }
    const float range = high - bound, steps = fminf(Num::STEPS / range, 0x1p127f);   // range 0: those below are still below 1
    int number[V];
#pragma unroll
    for (int v = 0; v < V; ++v) number[v] = Num::of(value[v], bound, steps, index(v));
    Sorter<V>::sort(number);
    // x before y in the order, y somebody: is that in doubt?  Sums of scores and biases: if they are not `apart`, and three steps, which is what the
    // way to a number costs.  Logits: if their numbers are the same but they may not be.  All are where the range is none.  Of 16 bits, ones whose numbers
    // are the same are the same unless they are next to nothing, as they differ by 2^-8 of themselves, which is eight steps or more; but not where the range is so
    // small that `steps` is cut and has fewer of them.
    const bool uncut = range >= 0x1p-100f;
    auto doubt = [&](int x, int y) {
      const int ahead = Num::height_of(x) - Num::height_of(y);
      const float v = bound + (float)Num::height_of(x) * (range * (1.0f / Num::STEPS));
      if (a.bias) return ahead <= (int)fminf(apart(v) * steps, 0x1p24f) + 3;
      return ahead == 0 && range != 0.0f && !(sizeof(T) == 2 && uncut && fabsf(v) > range * 0x1p-10f);
    };
    unsure = !empty && (unsure || !(range < INFINITY));
    int chosen[SLOTS];
    if constexpr (FEW) {
      int list[kList], rest = V > kList ? number[V > kList ? kList : 0] : 0;
#pragma unroll
      for (int i = 0; i < kList; ++i) list[i] = i < V ? number[i < V ? i : 0] : 0;
      merge_lists<0, LPR>(list, rest);
      // lane l's: the l-th and the one behind it, by the bits of l
      auto pick = [&](int a0, int a1, int a2, int a3, int a4, int a5, int a6, int a7) {
        const int b0 = l & 1 ? a1 : a0, b1 = l & 1 ? a3 : a2, b2 = l & 1 ? a5 : a4, b3 = l & 1 ? a7 : a6;
        const int c0 = l & 2 ? b1 : b0, c1 = l & 2 ? b3 : b2;
        return l & 4 ? c1 : c0;
      };
      static_assert(kList == 8, "three bits");
      const int mine = pick(list[0], list[1], list[2], list[3], list[4], list[5], list[6], list[7]);
      const int next = pick(list[1], list[2], list[3], list[4], list[5], list[6], list[7], rest);
      const bool is = !empty && l < a.k && Num::is_somebody(mine);
      chosen[0] = is ? Num::expert_of(mine) : -1;
      if (is && Num::is_somebody(next) && doubt(mine, next)) unsure = true;
    } else {
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) chosen[s] = -1;
      int before = 0;
      for (int j = 0; j <= a.k; ++j) {        // one more, to see how far it is
        const int best = team_max<LPR>(number[0]);
        const bool hit = number[0] == best, is = !empty && Num::is_somebody(best);
        if (is && j > 0 && doubt(before, best)) unsure = true;
        before = best;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
          if (is && j < a.k && j == l + s * LPR) chosen[s] = Num::expert_of(best);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int stay = number[v], next = v + 1 < V ? number[v + 1] : 0;   // values: a choice of elements would become an array in scratch
          number[v] = hit ? next : stay;
        }
      }
    }
    for (uint64_t left = __ballot(unsure); left;) {   // by the definition, team by team
      const int lane0 = __builtin_ctzll(left) & ~(LPR - 1);
      left &= LPR == 64 ? 0 : ~(((1ull << (LPR & 63)) - 1) << lane0);
      const int pick = choose_exactly<T, (MAX_E < kWave ? kWave : MAX_E), GROUPED>(a, row + lane0 / LPR - lane0_of_mine / LPR, __shfl(top, lane0, kWave),
                                                                                           reinterpret_cast<double *>(s_value + (GROUPED ? threadIdx.x / kWave * WAVE_VALUES : 0)));
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        const int at = __shfl(pick, (l + s * LPR) & 63, kWave);
        if (lane0 == lane0_of_mine) chosen[s] = at;
      }
    }
    // weights
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    float logit[SLOTS], w[SLOTS], highest = top, total = 0.0f;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) logit[s] = chosen[s] >= 0 ? to_f32(x[chosen[s]]) : -INFINITY;
    if (a.renormalise) {
      highest = logit[0];
#pragma unroll
      for (int s = 1; s < SLOTS; ++s) highest = fmaxf(highest, logit[s]);
      highest = team_max<LPR>(highest);
    }
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      w[s] = chosen[s] >= 0 ? share(logit[s], a.softmax, highest, a.renormalise) : 0.0f;
      total += w[s];
    }
    total = a.renormalise ? team_add<LPR>(total) : 1.0f;
    const float factor = a.renormalise ? a.scale : a.scale * inv;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int j = l + s * LPR;
      if (row < last && j < a.k) {
        a.expert[row * a.k + j] = chosen[s];
        a.weight[row * a.k + j] = broken ? NAN : chosen[s] >= 0 ? w[s] / total * factor : 0.0f;   // not scale / total, which may be infinite
        if (chosen[s] >= 0) atomicAdd(&s_words[chosen[s]], 1);
      }
    }
  }
  if (!a.off) return;
  __syncthreads();
  if (gridDim.x > 1) {
    for (int e = threadIdx.x; e < E; e += threads) {
      const int at = e * runs_ld(gridDim.x) + blockIdx.x;
      if (narrow(a.run))
        static_cast<uint16_t *>(a.count)[at] = (uint16_t)s_words[e];
      else
        static_cast<int32_t *>(a.count)[at] = s_words[e];
    }
    return;
  }
  for (int e = threadIdx.x; e < E; e += threads) {
    s_words[E + e] = s_words[e];
    s_words[e] = 0;
  }
  for (int i = threadIdx.x; i < rankers_of(E) * E; i += threads) s_words[2 * E + i] = 0;
  Slice slice(a, first, last);
  slice.request(a, slice.begin);
  places(a, 0, slice, s_words, s_words + E, s_words + 2 * E);
}

// Sixteen bytes of an expert's counts a lane: LANES lanes have those of all runs, a wavefront takes 64 / LANES experts at a time.  Every workgroup
// reads all counts, 256 KB of 32 bits for 256 runs and experts, which is what 16 bits are for.
constexpr int kPlaceThreads = 1024;
template <typename T> __global__ void __launch_bounds__(kPlaceThreads) k_places(RouteArgs a) {
  extern __shared__ int32_t s_words[];
  constexpr int EACH = 16 / sizeof(T), LANES = kMaxRuns / EACH, AT_ONCE = kPlaceThreads / LANES, AHEAD = 8;
  static_assert(LANES == 32 || LANES == 64, "a part of a wavefront, or all of it");
  const int64_t first = (int64_t)blockIdx.x * a.run, last = min(a.rows, first + a.run);
  const int E = a.experts, runs = gridDim.x, run = blockIdx.x, l = threadIdx.x % LANES;
  Slice slice(a, first, last);
  slice.request(a, slice.begin);
  for (int i = threadIdx.x; i < rankers_of(E) * E; i += kPlaceThreads) s_words[2 * E + i] = 0;
  for (int e0 = 0; e0 < E; e0 += AT_ONCE * AHEAD) {
    uint4 c[AHEAD];
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      const int e = e0 + p * AT_ONCE + threadIdx.x / LANES;
      c[p] = make_uint4(0u, 0u, 0u, 0u);
      if (e < E && EACH * l < runs) c[p] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.count) + e * runs_ld(runs) + EACH * l);
    }
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      if (e0 + p * AT_ONCE >= E) break;
      const int e = e0 + p * AT_ONCE + threadIdx.x / LANES;
      const uint32_t w[4] = {c[p].x, c[p].y, c[p].z, c[p].w};
      int before = 0, all = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const int n = EACH == 4 ? (int)w[i & 3] : (int)(w[i / 2 & 3] >> (16 * (i & 1)) & 0xffffu);
        if (EACH * l + i < runs) all += n;
        if (EACH * l + i < run) before += n;
      }
      auto add = [](int x, int y) { return x + y; };
      all = team<LANES>(all, add);
      before = team<LANES>(before, add);
      if (l == 0 && e < E) s_words[e] = before, s_words[E + e] = all;
    }
  }
  places(a, run, slice, s_words, s_words + E, s_words + 2 * E);
}

// ---- gradient -----------------------------------------------------------------------------------------------------
// With f_j = dw_j at the chosen experts and zero elsewhere, and p = weight / scale where weights are divided by their sum, scale times
//   softmax             dl_i = s_i (f_i - sum_j s_j f_j)            every logit
//   softmax, divided    dl_j = p_j (f_j - sum_i p_i f_i)            the chosen ones' (the sum of the others cancels)
//   sigmoid             dl_j = s_j (1 - s_j) f_j
//   sigmoid, divided    dl_j = p_j (1 - s_j) (f_j - sum_i p_i f_i)
// Only the first reads more than the chosen experts' logits.  fp32: nothing is chosen here.  Bound by memory: 65536 x 256 fp32, softmax, 26.8 us for 138 MB (5.2 TB/s).
struct RouteBackArgs {
  int64_t rows, ld, ld_d;
  int experts, k, softmax, renormalise;
  float scale;
  const void *logits;
  const int32_t *expert;
  const float *weight, *dweight;
  void *dlogits;
};

template <typename T, int LPR, int V> __global__ void __launch_bounds__(256) k_route_back(RouteBackArgs a) {
  constexpr int TEAMS = 256 / LPR, MAX_E = LPR * V, SLOTS = LPR < GEAR_MAX_CHOSEN ? GEAR_MAX_CHOSEN / LPR : 1;
  __shared__ float s_flow[TEAMS * MAX_E];
  const int l = threadIdx.x % LPR, team = threadIdx.x / LPR, E = a.experts;
  float *flow = s_flow + team * MAX_E;
  const bool all = a.softmax && !a.renormalise;
  auto index = [&](int v) { return v * LPR + l; };
  for (int64_t row0 = (int64_t)blockIdx.x * TEAMS; row0 < a.rows; row0 += (int64_t)gridDim.x * TEAMS) {
    const int64_t row = row0 + team;
    const bool have = row < a.rows;
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
#pragma unroll
    for (int v = 0; v < V; ++v) flow[index(v)] = 0.0f;
    float lg[V];
    if (all) {
#pragma unroll
      for (int v = 0; v < V; ++v) lg[v] = have && index(v) < E ? to_f32(x[index(v)]) : -INFINITY;
    }
    int e[SLOTS];
    float f[SLOTS], p[SLOTS], inner = 0.0f;
    bool broken = false;
    int chosen = 0;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int j = l + s * LPR;
      const bool in = have && j < a.k;
      e[s] = in ? a.expert[row * a.k + j] : -1;
      const float w = in ? a.weight[row * a.k + j] : 0.0f;
      broken |= w != w;
      if (e[s] >= E) e[s] = -1;
      f[s] = e[s] >= 0 ? a.dweight[row * a.k + j] : 0.0f;
      p[s] = e[s] >= 0 ? w / a.scale : 0.0f;
      inner += p[s] * f[s];
      chosen += __popcll(team_ballot<LPR>(e[s] >= 0));
    }
    broken = team_any<LPR>(broken);
    const bool some = chosen > 0;    // else the row is padding, whatever its logits hold, or has no expert: zeros
    inner = team_add<LPR>(inner);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      if (e[s] < 0) continue;
      float d = f[s];
      if (!all) {
        if (a.renormalise) d = p[s] * (f[s] - (chosen == 1 ? f[s] : inner));   // an only one's p is 1: zero, whatever its weight was rounded to
        if (!a.softmax) {
          const float v = to_f32(x[e[s]]), t = expf(-fabsf(v)), big = 1.0f / (1.0f + t), small = t / (1.0f + t);   // of |v|: s and 1 - s
          d *= a.renormalise ? (v > 0.0f ? small : big) : big * small;
        }
        d *= a.scale;
      }
      flow[e[s]] = d;
    }
    __syncthreads();
    float d[V];
#pragma unroll
    for (int v = 0; v < V; ++v) d[v] = flow[index(v)];
    if (all) {
      float top = -INFINITY, sum = 0.0f, dot = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) top = fmaxf(top, lg[v]);
      top = team_max<LPR>(top);
      const bool none = top == -INFINITY;     // no logit: no score
#pragma unroll
      for (int v = 0; v < V; ++v) {
        lg[v] = none ? 0.0f : expf(lg[v] - top);
        sum += lg[v];
        dot += lg[v] * d[v];
      }
      sum = team_add<LPR>(sum);
      dot = team_add<LPR>(dot);
      const float inv = none ? 0.0f : 1.0f / sum, scaled = inv * a.scale;
#pragma unroll
      for (int v = 0; v < V; ++v) d[v] = lg[v] * scaled * (d[v] - dot * inv);
    }
    T *out = static_cast<T *>(a.dlogits) + row * a.ld_d;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (have && index(v) < E) out[index(v)] = from_f32<T>(broken ? NAN : some ? d[v] : 0.0f);
    __syncthreads();
  }
}

// Lanes of a row and logits of a lane.  Half as many lanes for twice as many logits where there are rows for all of them: what is done once for every
// four rows of a wavefront is then done for eight.  us with k = 8, eight lanes / sixteen: 65536 rows of 64 experts 19.5 / 23.9, of 160 with a bias 41 / 47,
// of 256 37.0 / 39.9 and with a bias 44.5 / 50.0; not for 65 to 128 experts, whose registers spill (35.3 / 33.8), nor for fewer rows (16384 of 64 12.5 / 12.5).
constexpr int kManyRows = 32768;
struct Shape {
  int lpr, v, threads, run, runs;
};
Shape shape_of(int64_t rows, int experts, int k, bool grouped) {
  Shape s;
  s.lpr = experts <= 256 ? 16 : experts <= 512 ? 32 : 64;
  if (!grouped && k <= kList && rows >= kManyRows && (experts <= 64 || (experts > 128 && experts <= 256))) s.lpr = 8;
  s.v = 4;
  while (s.lpr * s.v < experts) s.v *= 2;
  if (s.lpr > 16) s.v = 16;
  // runs of rows: as many as there are CUs at most, of whole passes of a workgroup over its rows; a batch that fits in one has no more threads than
  // its rows need (one row of 64 experts: 6.0 us by 64 threads, 9.1 by 1024)
  s.threads = threads_of(s.lpr, s.v, grouped);
  const int teams = s.threads / s.lpr;
  const int64_t passes = (rows + teams - 1) / teams, each = (passes + kMaxRuns - 1) / kMaxRuns, run = (each > 0 ? each : 1) * teams;
  s.run = (int)run;
  s.runs = (int)(rows > 0 ? (rows + run - 1) / run : 1);
  if (rows < teams) s.threads = rows > 0 ? (int)((rows * s.lpr + kWave - 1) / kWave * kWave) : kWave;
  return s;
}
// call(LPR, V) for a shape
template <typename F> hipError_t with_shape(const Shape &s, F &&call) {
  using std::integral_constant;
#define GEAR_SHAPE(L, W) \
  if (s.lpr == L && s.v == W) return call(integral_constant<int, L>{}, integral_constant<int, W>{});
  GEAR_SHAPE(8, 4) GEAR_SHAPE(8, 8) GEAR_SHAPE(8, 32)
  GEAR_SHAPE(16, 4) GEAR_SHAPE(16, 8) GEAR_SHAPE(16, 16) GEAR_SHAPE(32, 16) GEAR_SHAPE(64, 16)
#undef GEAR_SHAPE
  return hipErrorInvalidValue;
}

bool sizes_ok(int64_t rows, int32_t experts, int32_t k) {
  return rows >= 0 && rows <= (1 << 30) && experts >= 1 && experts <= GEAR_MAX_EXPERTS && k >= 1 && k <= GEAR_MAX_CHOSEN && k <= experts &&
         rows * k <= (1 << 30);
}

template <typename T, bool WIDE, bool GROUPED> hipError_t launch_route(const RouteArgs &a, const Shape &shape, hipStream_t s) {
  return with_shape(shape, [&](auto lpr, auto v) {
    constexpr int LPR = decltype(lpr)::value, V = decltype(v)::value;
    const size_t lds = (size_t)(shape.runs == 1 ? place_words(a.experts) : a.experts) * 4;
    const dim3 grid(shape.runs), block(shape.threads);
    if constexpr (LPR == 8 && GROUPED)
      return hipErrorInvalidValue;     // shape_of gives no such shape
    else if (a.k <= kList)
      hipLaunchKernelGGL((k_route<T, LPR, V, WIDE, GROUPED, true>), grid, block, lds, s, a);
    else if constexpr (LPR == 8)
      return hipErrorInvalidValue;
    else
      hipLaunchKernelGGL((k_route<T, LPR, V, WIDE, GROUPED, false>), grid, block, lds, s, a);
    return hipGetLastError();
  });
}

template <typename T> hipError_t launch_route_of(const RouteArgs &a, const Shape &shape, bool wide, hipStream_t s) {
  if (a.groups > 1) return wide ? launch_route<T, true, true>(a, shape, s) : launch_route<T, false, true>(a, shape, s);
  return wide ? launch_route<T, true, false>(a, shape, s) : launch_route<T, false, false>(a, shape, s);
}

template <typename T> hipError_t launch_back(const RouteBackArgs &a, hipStream_t s) {
  return with_shape(shape_of(1, a.experts, a.k, false), [&](auto lpr, auto v) {
    constexpr int LPR = decltype(lpr)::value, TEAMS = 256 / LPR;
    if constexpr (LPR == 8) {
      return hipErrorInvalidValue;     // not for one row
    } else {
      const int64_t blocks = (a.rows + TEAMS - 1) / TEAMS;
      hipLaunchKernelGGL((k_route_back<T, LPR, decltype(v)::value>), dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s, a);
      return hipGetLastError();
    }
  });
}

}  // namespace
}  // namespace gear

using namespace gear;

extern "C" size_t gear_route_workspace_bytes(int64_t rows, int32_t experts, int32_t k, int32_t groups) {
  if (!sizes_ok(rows, experts, k) || groups < 1) return 0;
  const Shape s = shape_of(rows, experts, k, groups > 1);
  return ((size_t)runs_ld(s.runs) * experts * (narrow(s.run) ? 2 : 4) + 255) / 256 * 256;
}

extern "C" gear_status gear_route(const gear_route_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  if (!a || !sizes_ok(a->rows, a->experts, a->k) || (a->dtype != GEAR_F32 && a->dtype != GEAR_BF16)) return GEAR_ERR_INVALID;
  if (a->score != GEAR_SCORE_SOFTMAX && a->score != GEAR_SCORE_SIGMOID) return GEAR_ERR_INVALID;
  if (a->groups < 1 || a->groups > kMaxGroups || a->experts % a->groups || a->groups_kept < 1 || a->groups_kept > a->groups ||
      a->k > a->experts / a->groups * a->groups_kept || (a->group_best != 1 && a->group_best != 2))
    return GEAR_ERR_INVALID;
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale)) return GEAR_ERR_INVALID;
  if ((a->off != nullptr) != (a->place != nullptr) && !(a->rows == 0 && a->off)) return GEAR_ERR_INVALID;
  const int size = (int)dtype_bytes(a->dtype);
  if (((uintptr_t)a->bias & 3) || ((uintptr_t)a->n & 3) || ((uintptr_t)a->expert & 3) || ((uintptr_t)a->weight & 3) || ((uintptr_t)a->off & 3) ||
      ((uintptr_t)a->place & 3))
    return GEAR_ERR_INVALID;
  if (a->rows > 0 && (!a->logits || ((uintptr_t)a->logits & (size - 1)) || !a->expert || !a->weight || a->ld_logits < a->experts ||
                      a->ld_logits >= (1 << 20)))
    return GEAR_ERR_INVALID;
  if (a->rows == 0 && !a->off) return GEAR_OK;
  const Shape shape = shape_of(a->rows, a->experts, a->k, a->groups > 1);
  if (a->off) {
    if (!workspace || ((uintptr_t)workspace & 255)) return GEAR_ERR_INVALID;
    if (workspace_bytes < gear_route_workspace_bytes(a->rows, a->experts, a->k, a->groups)) return GEAR_ERR_CAPACITY;
  }
  hipStream_t s = (hipStream_t)stream;
  const RouteArgs p = {a->rows, a->ld_logits, shape.run, a->experts, a->k, a->score == GEAR_SCORE_SOFTMAX, a->groups, a->groups_kept, a->group_best,
                       a->renormalise != 0, a->scale, a->logits, a->bias, a->n, a->expert, a->weight, a->off, a->place, workspace};
  const bool wide = a->experts % 4 == 0 && a->ld_logits % 4 == 0 && ((uintptr_t)a->logits & (4 * size - 1)) == 0;
  hipError_t err = a->dtype == GEAR_F32 ? launch_route_of<float>(p, shape, wide, s) : launch_route_of<bf16_t>(p, shape, wide, s);
  if (err == hipSuccess && a->off && shape.runs > 1) {
    const size_t lds = (size_t)place_words(a->experts) * 4;
    if (narrow(shape.run))
      hipLaunchKernelGGL(k_places<uint16_t>, dim3(shape.runs), dim3(kPlaceThreads), lds, s, p);
    else
      hipLaunchKernelGGL(k_places<int32_t>, dim3(shape.runs), dim3(kPlaceThreads), lds, s, p);
    err = hipGetLastError();
  }
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}

extern "C" gear_status gear_route_backward(const gear_route_backward_args *a, void *stream) {
  if (!a || !sizes_ok(a->rows, a->experts, a->k) || (a->dtype != GEAR_F32 && a->dtype != GEAR_BF16)) return GEAR_ERR_INVALID;
  if (a->score != GEAR_SCORE_SOFTMAX && a->score != GEAR_SCORE_SIGMOID) return GEAR_ERR_INVALID;
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale)) return GEAR_ERR_INVALID;
  if (a->rows == 0) return GEAR_OK;
  const int size = (int)dtype_bytes(a->dtype);
  if (!a->logits || !a->expert || !a->weight || !a->dweight || !a->dlogits || ((uintptr_t)a->logits & (size - 1)) ||
      ((uintptr_t)a->dlogits & (size - 1)) || ((uintptr_t)a->expert & 3) || ((uintptr_t)a->weight & 3) || ((uintptr_t)a->dweight & 3))
    return GEAR_ERR_INVALID;
  if (a->ld_logits < a->experts || a->ld_logits >= (1 << 20) || a->ld_dlogits < a->experts || a->ld_dlogits >= (1 << 20)) return GEAR_ERR_INVALID;
  const RouteBackArgs p = {a->rows, a->ld_logits, a->ld_dlogits, a->experts, a->k, a->score == GEAR_SCORE_SOFTMAX, a->renormalise != 0, a->scale,
                           a->logits, a->expert, a->weight, a->dweight, a->dlogits};
  const hipError_t err = a->dtype == GEAR_F32 ? launch_back<float>(p, (hipStream_t)stream) : launch_back<bf16_t>(p, (hipStream_t)stream);
  return err == hipSuccess ? GEAR_OK : GEAR_ERR_HIP;
}
