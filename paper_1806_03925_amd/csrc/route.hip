// Routing of rows to experts: scores, choice of k experts a row, weights, and the order of all (row, slot) pairs by expert; its
// gradient (gear.h has the definitions).
//
// A row is a team of LPR lanes' (16, 32 or 64 of one wavefront), V logits a lane, all in registers from the one time they are
// read.  Scores are fp64: what decides the choice is score + bias, and two experts' sums lie closer together than fp32 resolves
// in one row of some hundred thousand.  A choice is k times the largest over the team, ties to the lowest index.
//
// The order of the pairs is a counting sort by expert.  A workgroup takes a run of rows and counts its experts; a second launch
// with the same runs finds from all counts where each run's pairs begin, ranks them (equal experts in a wavefront by ballots,
// wavefronts in order) and writes their places.  Batches of one run are both in one launch.  No atomic decides an order: those on
// counts in LDS only add.
#include "gear_internal.hpp"

#include <cmath>
#include <type_traits>

namespace gear {
namespace {

constexpr int kMaxRuns = 256;        // one for each CU
constexpr int kRouteThreads = 1024, kGroupedThreads = 256;
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
  int32_t *off, *place, *count;      // count [runs x experts]
};

template <int LPR> __device__ __forceinline__ double team_add(double v) {
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}
template <int LPR> __device__ __forceinline__ float team_max(float v) {
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
  return v;
}
template <int LPR> __device__ __forceinline__ bool team_any(bool v) {
  int x = v;
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) x |= __shfl_xor(x, o, kWave);
  return x != 0;
}

// the largest of a team's (value, index), the lower index of equals; `with` goes along
struct Best {
  double value;
  int index;
  float with;
};
template <int LPR> __device__ __forceinline__ Best team_best(Best b) {
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) {
    const double v = __shfl_xor(b.value, o, kWave);
    const int i = __shfl_xor(b.index, o, kWave);
    const float w = __shfl_xor(b.with, o, kWave);
    if (v > b.value || (v == b.value && i < b.index)) b = {v, i, w};
  }
  return b;
}

// Sigmoid and softmax of a logit, up to a factor that is the same for all of `top`'s row where `relative`: no sum of such
// scores vanishes, however small they are.  Softmax: exp(l - top), relative or not.
__device__ __forceinline__ double score_of(float l, bool softmax, double top, bool relative) {
  const double v = (double)l;
  if (softmax) return exp(v - top);
  if (v > 0.0) return 1.0 / (1.0 + exp(-v));
  const double shift = relative && top < 0.0 ? top : 0.0;
  return exp(v - shift) / (1.0 + exp(v));
}

// ---- order of the pairs -------------------------------------------------------------------------------------------
// Places of the pairs of rows [first, last), those of run number `run`.  On entry s_wave[e] is the number of expert e's pairs in all
// runs and s_base[e] that in the runs before this one.  s_base, s_wave: experts and kRankers x experts words of LDS.
constexpr int kRankers = 8;          // wavefronts that rank pairs: as many as counts of 1024 experts fit in LDS
template <int THREADS> __device__ void places(const RouteArgs &a, int run, int64_t first, int64_t last, int32_t *s_base, int32_t *s_wave) {
  constexpr int WAVES = THREADS / kWave < kRankers ? THREADS / kWave : kRankers;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, E = a.experts;
  __syncthreads();
  if (wave == 0) {   // where each expert begins
    int begin = 0;
    for (int e0 = 0; e0 < E; e0 += kWave) {
      const int e = e0 + lane, mine = e < E ? s_wave[e] : 0;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int v = __shfl_up(upto, o, kWave);
        if (lane >= o) upto += v;
      }
      if (e < E) {
        s_base[e] += begin + upto - mine;
        if (run == 0) a.off[e] = begin + upto - mine;
      }
      begin += __shfl(upto, kWave - 1, kWave);
    }
    if (run == 0 && lane == 0) a.off[E] = begin;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < WAVES * E; i += THREADS) s_wave[i] = 0;
  __syncthreads();
  // a wavefront takes every pair from `from` on, 64 at a time: first it counts, then it places
  const int64_t pairs = (last - first) * a.k, per = (pairs + WAVES - 1) / WAVES;
  const int64_t begin = first * a.k + min(wave * per, pairs);
  const int64_t end = wave < WAVES ? first * a.k + min((wave + 1) * per, pairs) : begin;
  int32_t *mine = s_wave + min(wave, WAVES - 1) * E;
  int bits = 0;
  while ((1 << bits) < E) ++bits;
  auto walk = [&](auto &&then) {
    for (int64_t i0 = begin; i0 < end; i0 += kWave) {
      const int64_t i = i0 + lane;
      const int e = i < end ? a.expert[i] : -1;
      uint64_t same = __ballot(e >= 0);
      for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((e >> b) & 1);
        same &= (e >> b) & 1 ? set : ~set;
      }
      const int rank = __popcll(same & ((1ull << lane) - 1));
      then(i, e, rank, __popcll(same), i < end);
    }
  };
  walk([&](int64_t, int e, int rank, int all, bool) {
    if (e >= 0 && rank == 0) mine[e] += all;   // one lane for each expert
  });
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += THREADS) {
    int at = s_base[e];
    for (int w = 0; w < WAVES; ++w) {
      const int c = s_wave[w * E + e];
      s_wave[w * E + e] = at;
      at += c;
    }
  }
  __syncthreads();
  walk([&](int64_t i, int e, int rank, int all, bool in) {
    int at = -1;
    if (e >= 0) at = mine[e] + rank;
    asm volatile("" ::: "memory");   // every lane has read before one adds
    if (e >= 0 && rank == 0) mine[e] += all;
    if (in) a.place[i] = at;
  });
}

template <typename T, int LPR, int V, bool WIDE, bool GROUPED>
__global__ void __launch_bounds__(GROUPED ? kGroupedThreads : kRouteThreads) k_route(RouteArgs a) {
  constexpr int THREADS = GROUPED ? kGroupedThreads : kRouteThreads, TEAMS = THREADS / LPR, MAX_E = LPR * V;
  constexpr int SLOTS = LPR < GEAR_MAX_CHOSEN ? GEAR_MAX_CHOSEN / LPR : 1;   // of a lane
  static_assert(!WIDE || V % 4 == 0, "four neighbouring logits a load");
  extern __shared__ int32_t s_words[];                          // [experts] counts, then what places() needs
  __shared__ double s_value[GROUPED ? TEAMS * MAX_E : 1], s_group[GROUPED ? TEAMS * kMaxGroups : 1];
  const double kNone = -INFINITY;
  const int l = threadIdx.x % LPR, team = threadIdx.x / LPR, E = a.experts;
  for (int e = threadIdx.x; e < E; e += THREADS) s_words[e] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * a.run, last = min(a.rows, first + a.run);
  const int64_t used = a.n ? min(a.rows, (int64_t)max(*a.n, 0)) : a.rows;
  auto index = [&](int v) { return WIDE ? (v / 4) * (LPR * 4) + l * 4 + v % 4 : v * LPR + l; };
  float bias[V];
#pragma unroll
  for (int v = 0; v < V; ++v) bias[v] = a.bias && index(v) < E ? a.bias[index(v)] : 0.0f;

  for (int64_t row0 = first; row0 < last; row0 += TEAMS) {
    const int64_t row = row0 + team;
    const bool have = row < min(last, used);
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    float lg[V];
#pragma unroll
    for (int v = 0; v < V; ++v) lg[v] = -INFINITY;
    if (have) {
      if constexpr (WIDE) {
#pragma unroll
        for (int v = 0; v < V; v += 4)
          if (index(v) < E) {
            if constexpr (sizeof(T) == 4) {
              const float4 f = *reinterpret_cast<const float4 *>(x + index(v));
              lg[v] = f.x, lg[v + 1] = f.y, lg[v + 2] = f.z, lg[v + 3] = f.w;
            } else {
              const uint2 f = *reinterpret_cast<const uint2 *>(x + index(v));
              lg[v] = __uint_as_float(f.x << 16), lg[v + 1] = __uint_as_float(f.x & 0xffff0000u);
              lg[v + 2] = __uint_as_float(f.y << 16), lg[v + 3] = __uint_as_float(f.y & 0xffff0000u);
            }
          }
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (index(v) < E) lg[v] = to_f32(x[index(v)]);
      }
    }
    bool broken = false;
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      broken |= lg[v] != lg[v] || (a.softmax && lg[v] == INFINITY);
      top = fmaxf(top, lg[v]);
    }
    broken = team_any<LPR>(broken);
    top = team_max<LPR>(top);
    const bool empty = broken || top == -INFINITY;   // no expert for this row, whatever the biases
    double sum = 1.0;
    if (a.softmax && (a.bias || GROUPED || !a.renormalise)) {
      sum = 0.0;
#pragma unroll
      for (int v = 0; v < V; ++v) sum += empty ? 0.0 : score_of(lg[v], true, top, false);
      sum = team_add<LPR>(sum);
    }
    double order[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const bool ok = !empty && lg[v] > -INFINITY && bias[v] > -INFINITY;
      double value = (double)lg[v];
      if (GROUPED || a.bias) {
        value = score_of(lg[v], a.softmax, top, false) / sum + (double)bias[v];
        if (GROUPED && index(v) < E) s_value[team * MAX_E + index(v)] = ok ? value : kNone;
        if (!a.bias) value = (double)lg[v];
      }
      order[v] = ok ? value : kNone;
    }
    if constexpr (GROUPED) {
      __syncthreads();
      const int per = E / a.groups;
      for (int q = l; q < a.groups; q += LPR) {
        double one = kNone, two = kNone;
        for (int i = 0; i < per; ++i) {
          const double v = s_value[team * MAX_E + q * per + i];
          two = v > one ? one : fmax(two, v);
          one = fmax(one, v);
        }
        s_group[team * kMaxGroups + q] = a.best == 2 && two > kNone ? one + two : one;
      }
      __syncthreads();
      double mine[kMaxGroups / LPR];
#pragma unroll
      for (int i = 0; i < kMaxGroups / LPR; ++i) mine[i] = l + i * LPR < a.groups ? s_group[team * kMaxGroups + l + i * LPR] : kNone;
      uint64_t keep = 0;
      for (int j = 0; j < a.kept; ++j) {
        Best b = {kNone, kMaxGroups, 0.0f};
#pragma unroll
        for (int i = 0; i < kMaxGroups / LPR; ++i)
          if (mine[i] > b.value) b = {mine[i], l + i * LPR, 0.0f};
        b = team_best<LPR>(b);
        if (!(b.value > kNone)) break;
        keep |= 1ull << b.index;
#pragma unroll
        for (int i = 0; i < kMaxGroups / LPR; ++i)
          if (l + i * LPR == b.index) mine[i] = kNone;
      }
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (index(v) < E && !(keep >> (index(v) / per) & 1)) order[v] = kNone;
    }
    int chosen[SLOTS];
    float logit[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) chosen[s] = -1, logit[s] = -INFINITY;
    for (int j = 0; j < a.k; ++j) {
      Best b = {kNone, MAX_E, 0.0f};
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (order[v] > b.value) b = {order[v], index(v), lg[v]};
      b = team_best<LPR>(b);
      if (!(b.value > kNone)) break;     // the same for the whole team
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (index(v) == b.index) order[v] = kNone;
#pragma unroll
      for (int s = 0; s < SLOTS; ++s)
        if (j == l + s * LPR) chosen[s] = b.index, logit[s] = b.with;
    }
    // weights
    double highest = (double)top;
    if (a.renormalise) {
      float m = logit[0];
#pragma unroll
      for (int s = 1; s < SLOTS; ++s) m = fmaxf(m, logit[s]);
      highest = (double)team_max<LPR>(m);
    }
    double w[SLOTS], total = 0.0;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      w[s] = chosen[s] >= 0 ? score_of(logit[s], a.softmax, highest, a.renormalise) : 0.0;
      total += w[s];
    }
    total = a.renormalise ? team_add<LPR>(total) : sum;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int j = l + s * LPR;
      if (row < last && j < a.k) {
        a.expert[row * a.k + j] = chosen[s];
        a.weight[row * a.k + j] = broken ? NAN : chosen[s] >= 0 ? (float)((double)a.scale * w[s] / total) : 0.0f;
        if (chosen[s] >= 0) atomicAdd(&s_words[chosen[s]], 1);
      }
    }
    if constexpr (GROUPED) __syncthreads();   // s_value and s_group have been read
  }
  if (!a.off) return;
  __syncthreads();
  if (gridDim.x > 1) {
    for (int e = threadIdx.x; e < E; e += THREADS) a.count[(int64_t)blockIdx.x * E + e] = s_words[e];
    return;
  }
  for (int e = threadIdx.x; e < E; e += THREADS) {
    s_words[E + e] = s_words[e];
    s_words[e] = 0;
  }
  places<THREADS>(a, 0, first, last, s_words, s_words + E);
}

constexpr int kPlaceThreads = 512;
__global__ void __launch_bounds__(kPlaceThreads) k_places(RouteArgs a) {
  extern __shared__ int32_t s_words[];
  const int64_t first = (int64_t)blockIdx.x * a.run, last = min(a.rows, first + a.run);
  const int E = a.experts, runs = gridDim.x, run = blockIdx.x;
  for (int e = threadIdx.x; e < E; e += kPlaceThreads) {
    int before = 0, all = 0;
    for (int r = 0; r < runs; ++r) {
      const int c = a.count[r * E + e];
      all += c;
      before += r < run ? c : 0;
    }
    s_words[e] = before;
    s_words[E + e] = all;
  }
  places<kPlaceThreads>(a, run, first, last, s_words, s_words + E);
}

// ---- gradient -----------------------------------------------------------------------------------------------------
// With f_j = scale dw_j at the chosen experts and zero elsewhere, and p = weight / scale where weights are divided by their sum:
//   softmax             dl_i = s_i (f_i - sum_j s_j f_j)            every logit
//   softmax, divided    dl_j = p_j (f_j - sum_i p_i f_i)            the chosen ones' (the sum of the others cancels)
//   sigmoid             dl_j = s_j (1 - s_j) f_j
//   sigmoid, divided    dl_j = p_j (1 - s_j) (f_j - sum_i p_i f_i)
// Only the first reads more than the chosen experts' logits.  fp32: nothing is chosen here.
struct RouteBackArgs {
  int64_t rows, ld, ld_d;
  int experts, k, softmax, renormalise;
  float scale;
  const void *logits;
  const int32_t *expert;
  const float *weight, *dweight;
  void *dlogits;
};

template <int LPR> __device__ __forceinline__ float team_addf(float v) {
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

template <typename T, int LPR, int V, bool WIDE> __global__ void __launch_bounds__(256) k_route_back(RouteBackArgs a) {
  constexpr int TEAMS = 256 / LPR, MAX_E = LPR * V, SLOTS = LPR < GEAR_MAX_CHOSEN ? GEAR_MAX_CHOSEN / LPR : 1;
  __shared__ float s_flow[TEAMS * MAX_E];
  const int l = threadIdx.x % LPR, team = threadIdx.x / LPR, E = a.experts;
  float *flow = s_flow + team * MAX_E;
  const bool all = a.softmax && !a.renormalise;
  auto index = [&](int v) { return WIDE ? (v / 4) * (LPR * 4) + l * 4 + v % 4 : v * LPR + l; };
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
    bool broken = false, some = false;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int j = l + s * LPR;
      const bool in = have && j < a.k;
      e[s] = in ? a.expert[row * a.k + j] : -1;
      const float w = in ? a.weight[row * a.k + j] : 0.0f;
      broken |= w != w;
      if (e[s] >= E) e[s] = -1;
      f[s] = e[s] >= 0 ? a.scale * a.dweight[row * a.k + j] : 0.0f;
      p[s] = e[s] >= 0 ? w / a.scale : 0.0f;
      inner += p[s] * f[s];
      some |= e[s] >= 0;
    }
    broken = team_any<LPR>(broken);
    some = team_any<LPR>(some);      // else the row is padding, whatever its logits hold, or has no expert: zeros
    inner = team_addf<LPR>(inner);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      if (e[s] < 0) continue;
      float d = f[s];
      if (!all) {
        if (a.renormalise) d = p[s] * (f[s] - inner);
        if (!a.softmax) {
          const float v = to_f32(x[e[s]]), t = expf(-fabsf(v)), big = 1.0f / (1.0f + t), small = t / (1.0f + t);   // of |v|: s and 1 - s
          d *= a.renormalise ? (v > 0.0f ? small : big) : big * small;
        }
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
      sum = team_addf<LPR>(sum);
      dot = team_addf<LPR>(dot);
      const float inv = none ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int v = 0; v < V; ++v) d[v] = lg[v] * inv * (d[v] - dot * inv);
    }
    T *out = static_cast<T *>(a.dlogits) + row * a.ld_d;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (have && index(v) < E) out[index(v)] = from_f32<T>(broken ? NAN : some ? d[v] : 0.0f);
    __syncthreads();
  }
}

// lanes of a row and logits of a lane: call(LPR, V) for `experts`
template <typename F> hipError_t by_experts(int experts, F &&call) {
  using std::integral_constant;
  if (experts <= 64) return call(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (experts <= 128) return call(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  if (experts <= 256) return call(integral_constant<int, 16>{}, integral_constant<int, 16>{});
  if (experts <= 512) return call(integral_constant<int, 32>{}, integral_constant<int, 16>{});
  return call(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

struct Runs {
  int run, count;
};
// Runs of rows: as many as there are CUs, of whole passes of a workgroup over its rows.
Runs runs_of(int64_t rows, int experts, bool grouped) {
  const int lpr = experts <= 256 ? 16 : experts <= 512 ? 32 : 64, teams = (grouped ? kGroupedThreads : kRouteThreads) / lpr;
  const int64_t passes = (rows + teams - 1) / teams, each = (passes + kMaxRuns - 1) / kMaxRuns;
  const int64_t run = (each > 0 ? each : 1) * teams;
  return {(int)run, (int)(rows > 0 ? (rows + run - 1) / run : 1)};
}

bool sizes_ok(int64_t rows, int32_t experts, int32_t k) {
  return rows >= 0 && rows <= (1 << 30) && experts >= 1 && experts <= GEAR_MAX_EXPERTS && k >= 1 && k <= GEAR_MAX_CHOSEN && k <= experts &&
         rows * k <= (1 << 30);
}

template <typename T, bool WIDE, bool GROUPED> hipError_t launch_route(const RouteArgs &a, int runs, hipStream_t s) {
  return by_experts(a.experts, [&](auto lpr, auto v) {
    constexpr int THREADS = GROUPED ? kGroupedThreads : kRouteThreads;
    const size_t lds = (size_t)a.experts * (1 + (runs == 1 ? kRankers : 0)) * 4;
    hipLaunchKernelGGL((k_route<T, decltype(lpr)::value, decltype(v)::value, WIDE, GROUPED>), dim3(runs), dim3(THREADS), lds, s, a);
    return hipGetLastError();
  });
}

template <typename T> hipError_t launch_route_of(const RouteArgs &a, int runs, bool wide, hipStream_t s) {
  if (a.groups > 1) return wide ? launch_route<T, true, true>(a, runs, s) : launch_route<T, false, true>(a, runs, s);
  return wide ? launch_route<T, true, false>(a, runs, s) : launch_route<T, false, false>(a, runs, s);
}

template <typename T> hipError_t launch_back(const RouteBackArgs &a, hipStream_t s) {
  return by_experts(a.experts, [&](auto lpr, auto v) {
    constexpr int LPR = decltype(lpr)::value, TEAMS = 256 / LPR;
    const int64_t blocks = (a.rows + TEAMS - 1) / TEAMS;
    hipLaunchKernelGGL((k_route_back<T, LPR, decltype(v)::value, false>), dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

}  // namespace
}  // namespace gear

using namespace gear;

extern "C" size_t gear_route_workspace_bytes(int64_t rows, int32_t experts, int32_t k, int32_t groups) {
  if (!sizes_ok(rows, experts, k) || groups < 1) return 0;
  return ((size_t)runs_of(rows, experts, groups > 1).count * experts * 4 + 255) / 256 * 256;
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
  const Runs r = runs_of(a->rows, a->experts, a->groups > 1);
  if (a->off) {
    if (!workspace || ((uintptr_t)workspace & 255)) return GEAR_ERR_INVALID;
    if (workspace_bytes < gear_route_workspace_bytes(a->rows, a->experts, a->k, a->groups)) return GEAR_ERR_CAPACITY;
  }
  hipStream_t s = (hipStream_t)stream;
  const RouteArgs p = {a->rows, a->ld_logits, r.run, a->experts, a->k, a->score == GEAR_SCORE_SOFTMAX, a->groups, a->groups_kept, a->group_best,
                       a->renormalise != 0, a->scale, a->logits, a->bias, a->n, a->expert, a->weight, a->off, a->place, (int32_t *)workspace};
  const bool wide = a->experts % 4 == 0 && a->ld_logits % 4 == 0 && ((uintptr_t)a->logits & (4 * size - 1)) == 0;
  hipError_t err = a->dtype == GEAR_F32 ? launch_route_of<float>(p, r.count, wide, s) : launch_route_of<bf16_t>(p, r.count, wide, s);
  if (err == hipSuccess && a->off && r.count > 1) {
    hipLaunchKernelGGL(k_places, dim3(r.count), dim3(kPlaceThreads), (size_t)a->experts * (1 + kRankers) * 4, s, p);
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
