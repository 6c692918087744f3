// Beam search's selection.  A candidate is (beam i, token t) with total = score[i] + x[i, t] - log sum_t exp x[i, t]; within a beam totals are in the order of the logits, so a
// run of a row needs its `keep` largest logits and, for the sum, its maximum and the sum of exponentials behind it: one pass over the logits, which HBM bounds.  A second
// kernel puts a prompt's runs together and ranks their candidates by totals in 64 bits: of two beams' candidates the larger is wanted, however close they are.
//
// 64 prompts of eight beams over 131072 tokens in bf16, eight kept, 15 % of the beams ended, 114 MB: 30 us for the runs (3.8 TB/s; 26 without looking for candidates) and 8 for the ranks; one prompt of four over 49999 in fp32: 5.5 and 7.  What
// bounds the runs is vector work (250 instruction slots for 32 logits a lane, of which the exponentials are half) beside HBM, and that beams which ended leave some CUs with less than others; the
// ranks are latency: sums, their logarithm, the border, the candidates' entries.
#include <float.h>

#include "common.h"

namespace ac {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 512, kWaves = kThreads / kWave, kRoom = 128, kNoted = 320, kMostCandidates = 512;

struct BeamArgs {
  const void* logits; int64_t ld;
  const float* scores; const int32_t* ended;
  float* scores_out; int32_t *parent, *token, *ended_out;
  int beams, vocab, keep, end;
  int runs, steps;                    // runs of a row, and steps of a run
  Divisor of_beam, of_lists, of_keep; // runs, lists of a prompt, keep
  float* sums;                        // [rows][runs][2]: maximum, sum of exponentials
  float* value; int32_t* index;       // [rows][runs][keep], largest first; -inf where there are no more
};

typedef unsigned long long Key;
// (a, i) before (b, j): the larger total, of equal ones the lower key.  (Without a branch: one for each comparison takes 80 cycles of a candidate's count.)
__device__ __forceinline__ bool before(double a, Key i, double b, Key j) { return (a > b) | ((a == b) & (i < j)); }
// A logit and its index as one number: the larger comes first.  0: none.
__device__ __forceinline__ Key key_of(float v, int index) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.f);               // (one zero)
  return (Key)(u ^ ((int)u < 0 ? 0xffffffffu : 0x80000000u)) << 32 | ~(uint32_t)index;
}
__device__ __forceinline__ float value_of_key(Key k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __builtin_bit_cast(float, u ^ ((int)u < 0 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int index_of_key(Key k) { return (int)~(uint32_t)k; }

// Of equal totals the lower beam comes first, and of a beam's the larger logit (different ones may have one total: it has 53 bits, of a score that may be large), then the lower token: 6, 32 and
// 24 bits, lowest first.  Never 0, which stands before all of them.  An ended beam has one candidate.
constexpr int kTokenBits = 24;
__device__ __forceinline__ Key place_of(int beam, float v, int token) {
  return (Key)beam << (kTokenBits + 32) | (Key) ~(uint32_t)(key_of(v, 0) >> 32) << kTokenBits | (uint32_t)token;
}
__device__ __forceinline__ int beam_of_place(Key k) { return (int)(k >> (kTokenBits + 32)); }
__device__ __forceinline__ int token_of_place(Key k) { return (int)(k & ((1u << kTokenBits) - 1)); }

// The next number above a finite one.
__device__ __forceinline__ float above(float v) {
  const int i = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, v == 0.f ? 1 : i < 0 ? i - 1 : i + 1);
}

// Floats but NaN as integers in their order.
__device__ __forceinline__ int in_order(float v) {
  const int i = __builtin_bit_cast(int, v + 0.f);
  return i < 0 ? i ^ 0x7fffffff : i;
}
__device__ __forceinline__ float of_order(int i) { return __builtin_bit_cast(float, i < 0 ? i ^ 0x7fffffff : i); }

// 16 bytes that may begin at any element.
__device__ __forceinline__ void load_anywhere(const float* p, f32x4& v) {
  typedef f32x4 any_f32x4 __attribute__((aligned(4)));
  v = *reinterpret_cast<const any_f32x4*>(p);
}
__device__ __forceinline__ void load_anywhere(const bf16_t* p, bf16x8& v) {
  typedef bf16x8 any_bf16x8 __attribute__((aligned(2)));
  v = *reinterpret_cast<const any_bf16x8*>(p);
}
template <typename T> struct Vec;
template <> struct Vec<float> { typedef f32x4 type; };
template <> struct Vec<bf16_t> { typedef bf16x8 type; };

// A run's largest logits as they are found: more than are kept, and cut down to these where room runs out.
struct Largest { Key key[kRoom]; int vector[kNoted]; };
// Over the wave, by rotations within sixteen lanes.
__device__ __forceinline__ float max_of_wave(float v) {
  v = fmaxf(v, rotate_row<8>(v));
  v = fmaxf(v, rotate_row<4>(v));
  v = fmaxf(v, rotate_row<2>(v));
  v = fmaxf(v, rotate_row<1>(v));
  auto of = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); };
  return fmaxf(fmaxf(of(0), of(16)), fmaxf(of(32), of(48)));
}
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// One wave: a run of a row, `steps` steps of U vectors of 16 bytes a lane, the next step's on their way while a step's are used.  Vectors are counted from the row's begin,
// wherever that lies, so that equal rows give equal sums; one that would pass the row's end is the row's last one, without what the lanes before have of it.  A lane's exponents have its own
// maximum for reference.  A logit is a candidate if it reaches `least`, which lies above the keep-th largest of those that were there when they were last looked at: at first it is the
// keep-th largest of the maxima over groups of lanes, twice as many as are kept.  The block's waves, whose runs are of one row, share the highest of what they have: what lies below
// it has enough larger ones wherever they are, and after the first step hardly anything reaches it.  (Alone a wave finds a few new ones in each of its steps: 37 us where 64 prompts of eight
// beams over 131072 tokens took 34 then.)  Which candidates a run keeps then depends on time, but not which ones come out.
template <typename T, int U>
__global__ void __launch_bounds__(kThreads) beam_scan(BeamArgs g) {
  typedef typename Vec<T>::type V;
  constexpr int VEC = Elem<T>::kVec, STEP = kWave * VEC * U;
  __shared__ Largest all[kWaves];
  __shared__ int border_of_all;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), run = blockIdx.x * kWaves + wave;
  const int64_t row = (int64_t)blockIdx.z * g.beams + blockIdx.y, part = row * g.runs + run;
  if ((g.ended && g.ended[row] != 0) || !(g.scores[row] > -INFINITY)) return;                         // (no candidate of its logits)
  if (threadIdx.x == 0) border_of_all = in_order(-FLT_MAX);
  __syncthreads();
  if (run >= g.runs) return;
  Largest& found = all[wave];
  const T* const from = (const T*)g.logits + row * g.ld;
  const int begin = run * g.steps * STEP, left = g.vocab - begin, steps = left < g.steps * STEP ? (left + STEP - 1) / STEP : g.steps, last = g.vocab - VEC;
  auto place = [&](int step, int u) { return begin + step * STEP + (u * kWave + lane) * VEC; };
  auto load = [&](V (&x)[U], int step) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (last >= 0) {
        load_anywhere(from + min(place(step, u), last), x[u]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] = u == 0 && lane == 0 && e < g.vocab ? from[e] : (T)-INFINITY;
      }
    }
  };
  float top = -INFINITY, sum = 0.f, border = -INFINITY;
  int count = 0, noted = 0;
  auto share = [&](float v) {
    if (lane == 0) atomicMax(&border_of_all, in_order(v));
  };
  // keeps the `keep` largest, in order; the border is the last of them, if there are so many
  auto cut = [&]() __attribute__((always_inline)) {
    Key mine[2];
    int rank[2] = {0, 0};
    wave_fence();
#pragma unroll
    for (int h = 0; h < 2; ++h) mine[h] = lane + h * kWave < count ? found.key[lane + h * kWave] : 0;
    if (count <= kWave) {
#pragma unroll 4
      for (int j = 0; j < count; ++j) rank[0] += found.key[j] > mine[0];
    } else {
#pragma unroll 2
      for (int j = 0; j < count; ++j) {
        const Key k = found.key[j];
        rank[0] += k > mine[0];
        rank[1] += k > mine[1];
      }
    }
    wave_fence();
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (rank[h] < g.keep && mine[h] != 0) found.key[rank[h]] = mine[h];
    wave_fence();
    if (count >= g.keep) {
      count = g.keep;
      border = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, value_of_key(found.key[g.keep - 1]))));
      share(border);
    }
  };
  // The noted vectors' numbers once more, a lane one, those that reach `least` to the candidates.  (What was kept before lies before them: where it is cut meanwhile, equal ones may be among
  // both.)
  auto take = [&](float least) __attribute__((always_inline)) {
    if (noted == 0) return;
    wave_fence();
    for (int r = lane / VEC; r - lane / VEC < noted; r += kWave / VEC) {
      const int at = found.vector[min(r, noted - 1)], near = min(at, max(last, 0)) + lane % VEC;
      const float v = r < noted && near >= at && near < g.vocab ? (float)from[near] : -INFINITY;
      uint64_t which = __ballot(v >= least);
      if (which == 0) continue;
      if (count + __popcll(which) > kRoom) {
        cut();
        least = fmaxf(least, border);
        which = __ballot(v >= least);
      }
      if (which >> lane & 1) found.key[count + __popcll(which & ((1ull << lane) - 1))] = key_of(v, near);
      count += __popcll(which);
    }
    noted = 0;
    cut();
  };
  V next[U];
  load(next, 0);
  for (int step = 0; step < steps; ++step) {
    float x[U][VEC], big[U], largest = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[u][e] = (float)next[u][e];
    if (step + 1 < steps) load(next, step + 1);
    else if (begin + steps * STEP > g.vocab && last >= 0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int again = place(step, u) - last;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] = e < again ? -INFINITY : x[u][e];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      big[u] = x[u][0];
#pragma unroll
      for (int e = 1; e < VEC; ++e) big[u] = fmaxf(big[u], x[u][e]);        // (NaN is no maximum; it is in the sum)
      largest = fmaxf(largest, big[u]);
    }
    if (largest > top) {
      if (top > -INFINITY) sum *= __builtin_amdgcn_exp2f((top - largest) * kLog2e);
      top = largest;
    }
    // (the difference first: the maximum's own term is 1, and a row of one token has a logarithm of exactly 0)
    const float ref = top > -INFINITY ? top : 0.f;
    float part[4] = {sum, 0.f, 0.f, 0.f};                                 // (four sums: what comes next need not wait for each)
    if (!__any(top == INFINITY)) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) part[e % 4] += __builtin_amdgcn_exp2f((x[u][e] - ref) * kLog2e);
    } else {                                                          // infinities share the probability
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) part[e % 4] += x[u][e] == INFINITY ? 1.f : __builtin_amdgcn_exp2f((x[u][e] - ref) * kLog2e);
    }
    sum = (part[0] + part[1]) + (part[2] + part[3]);
    // (of equal ones the lower index comes first: what equals the border is a candidate if that may be of this step, and none if it is of one before)
    float least;
    if (step == 0) {
      const int group = g.keep <= 8 ? 4 : g.keep <= 16 ? 2 : 1;
      float m = largest;
      if (group >= 2) m = fmaxf(m, __shfl_xor(m, 1, kWave));
      if (group >= 4) m = fmaxf(m, __shfl_xor(m, 2, kWave));
      int larger = 0;
      for (int j = 0; j < kWave; j += group) larger += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, m), j)) > m;
      least = fmaxf(-max_of_wave(larger < g.keep ? -m : -INFINITY), -FLT_MAX);       // (the least of those with fewer than `keep` larger ones)
      share(least);
    } else {
      least = border > -INFINITY ? above(border) : -FLT_MAX;
    }
    least = fmaxf(least, of_order(__builtin_amdgcn_readfirstlane(__hip_atomic_load(&border_of_all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP))));
    if (!__any(largest >= least)) continue;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint64_t which = __ballot(big[u] >= least);
      if (which != 0) {
        if (which >> lane & 1) found.vector[noted + __popcll(which & ((1ull << lane) - 1))] = place(step, u);
        noted += __popcll(which);
      }
    }
    // (soon, for the border's sake: 30 us with 8 noted ones, of eight kept, 34 with one and with 32)
    if (step == 0 || noted >= max(8, g.keep)) take(least);
  }
  take(border > -INFINITY ? above(border) : -FLT_MAX);
  const int64_t list = part * g.keep;
  if (lane < g.keep) {
    g.value[list + lane] = lane < count ? value_of_key(found.key[lane]) : -INFINITY;
    if (lane < count) g.index[list + lane] = index_of_key(found.key[lane]);
  }
  const float of_all = max_of_wave(top);
  sum = group_sum<kWave>(top == of_all ? sum : sum * __builtin_amdgcn_exp2f((top - of_all) * kLog2e));
  if (lane == 0) {
    g.sums[part * 2] = of_all;
    g.sums[part * 2 + 1] = sum;
  }
}

// One block: a prompt.  What comes out is found among the entries that reach a border: the keep-th largest of the maxima over threads, or groups of them, of the lists' first
// `levels` entries, in 32 bits (as the entries compared with it are, which keeps their order).  Below these levels a list is followed as far as it reaches the border.  Each candidate then counts
// those before it.  Where more reach it than there is room for, all entries are looked at, and where they are too many still, as equal ones can be, the first are looked for one after another.
__global__ void __launch_bounds__(kThreads) beam_rank(BeamArgs g) {
  __shared__ double rest[64], done[64];     // of each beam its score minus the logarithm of its sum (behind the maximum); and the score of one that ended: -inf where there is none
  __shared__ float top[64];
  __shared__ __attribute__((aligned(16))) float largest[kThreads];
  __shared__ int border_at, count_at;
  __shared__ double value_of[kMostCandidates];
  __shared__ Key place_at[kMostCandidates];
  __shared__ double wave_value[kWaves];
  __shared__ Key wave_place[kWaves];
  const int tid = threadIdx.x, lane = tid % kWave, lists = g.beams * g.runs;
  const int64_t row0 = (int64_t)blockIdx.x * g.beams;
  const float* const value = g.value + row0 * g.runs * g.keep;
  const int32_t* const index = g.index + row0 * g.runs * g.keep;
  bool by_list = false;
  // an item: entry k of a list, all lists' first ones before all second ones; by_list: list by list, so that a list's entries are
  // different threads' (where one list has most of what comes out)
  auto list_of = [&](int item, int& k) {
    const int q = quotient(item, by_list ? g.of_keep : g.of_lists), r = item - q * (by_list ? g.keep : lists);
    k = by_list ? r : q;
    return by_list ? q : r;
  };
  int levels = min(g.keep, max(1, kThreads / lists)), k_ahead;
  const int list_ahead = list_of(tid, k_ahead);
  const float ahead = tid < lists * levels ? value[list_ahead * g.keep + k_ahead] : 0.f;       // (on its way while the sums are looked at)
  for (int i = tid / kWave; i < g.beams; i += kWaves) {
    const float* sums = g.sums + (row0 + i) * g.runs * 2;
    const float score = g.scores[row0 + i];
    const bool gone = g.ended && g.ended[row0 + i] != 0, dead = gone || !(score > -INFINITY);
    float m = -INFINITY;
    double sum = 0;
    if (!dead) {
      const f32x2 near = *reinterpret_cast<const f32x2*>(sums + 2 * (lane < g.runs ? lane : 0));
      m = near[0];
      for (int p = lane + kWave; p < g.runs; p += kWave) m = fmaxf(m, sums[2 * p]);
      m = max_of_wave(m);
      for (int p = lane; p < g.runs; p += kWave) {
        const f32x2 part = p == lane ? near : *reinterpret_cast<const f32x2*>(sums + 2 * p);
        sum += part[0] == m ? (double)part[1] : (double)part[1] * exp((double)part[0] - (double)m);
      }
      for (int o = 1; o < kWave && o < g.runs; o <<= 1) sum += __shfl_xor(sum, o, kWave);      // (lane 0's is of all; the lanes from there on have nothing)
      sum = (double)score - log(sum);
    }
    if (lane == 0) {
      top[i] = m;
      rest[i] = dead || !(sum > -INFINITY) ? -INFINITY : sum;
      done[i] = gone && score > -INFINITY ? score : -INFINITY;
    }
  }
  __syncthreads();
  auto total_of = [&](int list, float v) {
    const int i = quotient(list, g.of_beam);
    const double r = rest[i];
    return r > -INFINITY && v > -INFINITY ? v == top[i] ? r : (double)v - top[i] + r : -INFINITY;
  };
  const double mine = tid < g.beams ? done[tid] : -INFINITY;
  // f of all of the thread's own entries, below the levels down a list up to the first for which it is false
  auto each = [&](auto f) {
    if (mine > -INFINITY) f(mine, place_of(tid, INFINITY, g.end));
    for (int item = tid; item < lists * levels; item += kThreads) {
      int k;
      const int list = list_of(item, k), beam = quotient(list, g.of_beam), down = k == levels - 1 ? g.keep : k + 1;
      for (; k < down; ++k) {
        const float v = value[list * g.keep + k];
        const double total = total_of(list, v);
        if (!(total > -INFINITY) || !f(total, place_of(beam, v, index[list * g.keep + k]))) break;
      }
    }
  };
  for (;; levels = g.keep, by_list = true) {
    if (tid == 0) { count_at = 0; border_at = 0x7fffffff; }
    double largest_own = mine;
    for (int item = tid; item < lists * levels; item += kThreads) {
      int k;
      const int list = list_of(item, k);
      largest_own = fmax(largest_own, total_of(list, item == tid && !by_list ? ahead : value[list * g.keep + k]));
    }
    // the least of the groups' maxima with fewer than `keep` larger ones; as an integer in the order of the floats
    const float most = (float)largest_own;
    const int holders = lists * levels < kThreads ? lists * levels : kThreads, group = holders >= 32 * g.keep ? 4 : holders >= 16 * g.keep ? 2 : 1, groups = (holders + group - 1) / group;
    float most_of_group = most;
    if (group >= 2) most_of_group = fmaxf(most_of_group, __shfl_xor(most_of_group, 1, kWave));
    if (group >= 4) most_of_group = fmaxf(most_of_group, __shfl_xor(most_of_group, 2, kWave));
    largest[tid] = -INFINITY;
    __syncthreads();
    if (tid % group == 0) largest[tid / group] = most_of_group;
    __syncthreads();
    int larger = 0;
#pragma unroll 2
    for (int j = 0; j < groups; j += 4) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(&largest[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) larger += a[e] > most_of_group;
    }
    if (larger < g.keep) atomicMin(&border_at, in_order(most_of_group));
    __syncthreads();
    const float border = of_order(border_at);
    if (most >= border)
      each([&](double v, Key place) {
        if ((float)v < border) return false;
        const int at = atomicAdd(&count_at, 1);
        if (at < kMostCandidates) {
          value_of[at] = v;
          place_at[at] = place;
        }
        return true;
      });
    __syncthreads();
    if (count_at <= kMostCandidates || by_list) break;
    __syncthreads();
  }
  const int64_t out = (int64_t)blockIdx.x * g.keep;
  auto put = [&](int k, double total, Key place) {
    const int i = beam_of_place(place), t = token_of_place(place);
    g.scores_out[out + k] = (float)total;
    g.parent[out + k] = (int)(row0 + i);
    g.token[out + k] = t;
    if (g.ended_out) g.ended_out[out + k] = t == g.end || done[i] > -INFINITY;
  };
  const int count = count_at;
  int n = count < g.keep ? count : g.keep;
  if (count <= kMostCandidates) {
    for (int c = tid; c < count; c += kThreads) {
      const double v = value_of[c];
      const Key place = place_at[c];
      int k = 0;
      for (int j = 0; j < count; ++j) k += before(value_of[j], place_at[j], v, place);
      if (k < g.keep) put(k, v, place);
    }
  } else {
    // as many equal ones: the first of those that are left, again and again
    double last = INFINITY;
    Key last_place = 0;
    for (n = 0; n < g.keep; ++n) {
      double v = -INFINITY;
      Key place = ~0ull;
      each([&](double a, Key at) {
        if (before(last, last_place, a, at) && before(a, at, v, place)) { v = a; place = at; }
        return true;
      });
#pragma unroll
      for (int o = kWave / 2; o > 0; o >>= 1) {
        const double a = __shfl_xor(v, o, kWave);
        const Key at = __shfl_xor(place, o, kWave);
        if (before(a, at, v, place)) { v = a; place = at; }
      }
      if (lane == 0) { wave_value[tid / kWave] = v; wave_place[tid / kWave] = place; }
      __syncthreads();
      v = wave_value[0]; place = wave_place[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w)
        if (before(wave_value[w], wave_place[w], v, place)) { v = wave_value[w]; place = wave_place[w]; }
      __syncthreads();
      if (!(v > -INFINITY)) break;
      if (tid == 0) put(n, v, place);
      last = v;
      last_place = place;
    }
  }
  for (int k = n + tid; k < g.keep; k += kThreads) {
    g.scores_out[out + k] = -INFINITY;
    g.parent[out + k] = g.token[out + k] = -1;
    if (g.ended_out) g.ended_out[out + k] = 0;
  }
}

// Steps of U vectors of 16 bytes a lane, and runs of so many steps that there are enough of them to fill the chip: four waves a SIMD.  us of both kernels (before the last 6 us were gained): 512 rows of 131072 bf16
// in steps of 4 vectors and runs of 8 43.5, of 4 46, of 2 50, of 16 50; of 2 vectors in runs of 16 46; of one 52.  Four rows of 49999 fp32 in one step a run: 4 vectors 13.0, 2 13.1, one 15.3.
struct Shape { int vectors, steps, runs; };
Shape shape(int64_t rows, int64_t vocab, int dtype) {
  const int64_t vec = kWave * (dtype == AC_BF16 ? 8 : 4);
  Shape s{4, 1, 0};
  auto runs = [&]() { return (vocab + vec * s.vectors * s.steps - 1) / (vec * s.vectors * s.steps); };
  while (s.vectors > 1 && rows * runs() < 128) s.vectors /= 2;
  while (s.steps < 16 && rows * runs() >= 8192) s.steps *= 2;
  s.runs = (int)runs();
  return s;
}

}  // namespace

uint64_t beam_select_workspace_bytes(int64_t batch, int beams, int64_t vocab, int keep, int dtype) {
  return (uint64_t)(batch * beams) * shape(batch * beams, vocab, dtype).runs * (2 + 2 * keep) * 4;
}

hipError_t launch_beam_select(const BeamSelectArgs& b, hipStream_t s) {
  const Shape sh = shape(b.batch * b.beams, b.vocab, b.dtype);
  const int64_t parts = b.batch * b.beams * sh.runs;
  float* const w = (float*)b.workspace;
  BeamArgs g{b.logits, b.ld, b.scores, b.ended, b.scores_out, b.parent, b.token, b.ended_out, b.beams, (int)b.vocab, b.keep, b.end, sh.runs, sh.steps,
             divisor((uint32_t)sh.runs), divisor((uint32_t)(sh.runs * b.beams)), divisor((uint32_t)b.keep), w, w + 2 * parts, (int32_t*)(w + (2 + b.keep) * parts)};
  const dim3 grid((unsigned)((sh.runs + kWaves - 1) / kWaves), (unsigned)b.beams, (unsigned)b.batch);
  auto scan = [&](auto zero) {
    using T = decltype(zero);
    if (sh.vectors == 4) hipLaunchKernelGGL((beam_scan<T, 4>), grid, dim3(kThreads), 0, s, g);
    else if (sh.vectors == 2) hipLaunchKernelGGL((beam_scan<T, 2>), grid, dim3(kThreads), 0, s, g);
    else hipLaunchKernelGGL((beam_scan<T, 1>), grid, dim3(kThreads), 0, s, g);
  };
  if (b.dtype == AC_BF16) scan(bf16_t{});
  else scan(float{});
  hipLaunchKernelGGL(beam_rank, dim3((unsigned)b.batch), dim3(kThreads), 0, s, g);
  return hipGetLastError();
}

}  // namespace ac
