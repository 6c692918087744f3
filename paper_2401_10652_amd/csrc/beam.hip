// Beam search's selection.  A candidate is (beam i, token t) with total = score[i] + x[i, t] - log sum_t exp x[i, t]; within a beam totals are in the order of the logits, so a
// run of a row needs its `keep` largest logits and, for the sum, its maximum and the sum of exponentials behind it: one pass over the logits, which HBM bounds.  A second
// kernel puts a prompt's runs together and ranks their candidates by totals in 64 bits: of two beams' candidates the larger is wanted, however close they are.
#include "common.h"

namespace ac {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256, kWaves = kThreads / kWave, kMostCandidates = 512;

struct BeamArgs {
  const void* logits; int64_t ld;
  const float* scores; const int32_t* ended;
  float* scores_out; int32_t *parent, *token, *ended_out;
  int beams, vocab, keep, end, splits;
  int group;                          // lanes that share a maximum when the border is looked for
  float* sums;                        // [rows][splits][2]: maximum, sum of exponentials
  float* value; int32_t* index;       // [rows][splits][keep], largest first; -inf where there are no more
};

// (a, i) before (b, j): the larger, of equal ones the lower index
template <typename V> __device__ __forceinline__ bool before(V a, int i, V b, int j) { return a > b || (a == b && i < j); }

template <typename V> struct Found { V value[kMostCandidates]; int index[kMostCandidates]; V most[kThreads / 2]; V border; int count; V wave_value[kWaves]; int wave_index[kWaves]; };

// The `keep` first of the block's candidates: each(f) calls f(value, index) for all of a thread's own, `most` is the largest of them (-inf without any); put(rank, value, index)
// takes them.  The border: of the maxima over groups of lanes, twice as many as are kept, the keep-th largest; at least that many candidates reach it, and few
// more do, of which each counts those before it.  Where more do than there is room for (as many equal ones), the first are looked for one after another.  Returns how many there are.
template <typename V, typename Each, typename Put>
__device__ __forceinline__ int first_ones(Found<V>& s, int keep, int group, V most, Each each, Put put) {
  const V none = -(V)INFINITY;
  const int tid = threadIdx.x, groups = kThreads / group;
  V top = most;
  for (int o = 1; o < group; o <<= 1) top = fmax(top, __shfl_xor(top, o, kWave));
  if (tid % group == 0) s.most[tid / group] = top;
  if (tid == 0) s.count = 0;
  __syncthreads();
  if (tid < groups) {
    const V mine = s.most[tid];
    int rank = 0;
    for (int j = 0; j < groups; ++j) rank += before(s.most[j], j, mine, tid);
    if (rank == keep - 1) s.border = mine;
  }
  __syncthreads();
  const V border = s.border;
  if (most >= border)
    each([&](V v, int i) {
      if (v >= border && v > none) {
        const int at = atomicAdd(&s.count, 1);
        if (at < kMostCandidates) {
          s.value[at] = v;
          s.index[at] = i;
        }
      }
    });
  __syncthreads();
  const int count = s.count;
  if (count <= kMostCandidates) {
    for (int c = tid; c < count; c += kThreads) {
      const V v = s.value[c];
      const int i = s.index[c];
      int rank = 0;
      for (int j = 0; j < count; ++j) rank += before(s.value[j], s.index[j], v, i);
      if (rank < keep) put(rank, v, i);
    }
    __syncthreads();
    return count < keep ? count : keep;
  }
  V last = (V)INFINITY;
  int last_index = -1;
  for (int k = 0; k < keep; ++k) {
    V v = none;
    int i = 0x7fffffff;
    each([&](V a, int j) {
      if (before(last, last_index, a, j) && before(a, j, v, i)) { v = a; i = j; }
    });
    for (int o = kWave / 2; o > 0; o >>= 1) {
      const V a = __shfl_xor(v, o, kWave);
      const int j = __shfl_xor(i, o, kWave);
      if (before(a, j, v, i)) { v = a; i = j; }
    }
    if (tid % kWave == 0) { s.wave_value[tid / kWave] = v; s.wave_index[tid / kWave] = i; }
    __syncthreads();
    v = s.wave_value[0]; i = s.wave_index[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w)
      if (before(s.wave_value[w], s.wave_index[w], v, i)) { v = s.wave_value[w]; i = s.wave_index[w]; }
    __syncthreads();
    if (!(v > none)) return k;
    if (tid == 0) put(k, v, i);
    last = v;
    last_index = i;
  }
  return keep;
}

// 16 bytes that may begin at any element.
__device__ __forceinline__ void load_anywhere(const float* p, float (&v)[4]) {
  typedef f32x4 any_f32x4 __attribute__((aligned(4)));
  const f32x4 t = *reinterpret_cast<const any_f32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = t[i];
}
__device__ __forceinline__ void load_anywhere(const bf16_t* p, float (&v)[8]) {
  typedef bf16x8 any_bf16x8 __attribute__((aligned(2)));
  const bf16x8 t = *reinterpret_cast<const any_bf16x8*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = bf2f(t[i]);
}

// One block: 256 * NV vectors of 16 bytes of one row, in registers.  They are counted from the row's begin, wherever that lies, so that equal rows give equal sums.
template <typename T, int NV>
__global__ void __launch_bounds__(kThreads) beam_scan(BeamArgs g) {
  constexpr int VEC = Elem<T>::kVec;
  __shared__ Found<float> found;
  __shared__ float of_wave[kWaves][2];
  const int64_t row = (int64_t)blockIdx.z * g.beams + blockIdx.y, part = row * g.splits + blockIdx.x;
  if ((g.ended && g.ended[row] != 0) || !(g.scores[row] > -INFINITY)) return;       // (no candidate of its logits)
  const T* const from = (const T*)g.logits + row * g.ld;
  const int tid = threadIdx.x, first = (blockIdx.x * kThreads * NV + tid) * VEC;
  float x[NV][VEC], most = -INFINITY;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int at = first + v * kThreads * VEC;
    if (at <= g.vocab - VEC) {
      load_anywhere(from + at, x[v]);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[v][e] = at + e < g.vocab ? Elem<T>::ld(from + at + e) : -INFINITY;
    }
  }
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < VEC; ++e) most = fmaxf(most, x[v][e]);            // (NaN is no maximum; it is in the sum)
  float sum = 0.f;
  if (most < INFINITY) {
    const float ref = most > -INFINITY ? most : 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum += __builtin_amdgcn_exp2f((x[v][e] - ref) * kLog2e);
  } else {                                                                // infinities share the probability
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum += x[v][e] == INFINITY ? 1.f : x[v][e] != x[v][e] ? x[v][e] : 0.f;
  }
  float top = wave_max(most);
  auto scaled = [](float s, float m, float t) { return m == t ? s : s * __builtin_amdgcn_exp2f((m - t) * kLog2e); };
  sum = wave_sum(scaled(sum, most, top));
  if (tid % kWave == 0) { of_wave[tid / kWave][0] = top; of_wave[tid / kWave][1] = sum; }
  const int64_t list = part * g.keep;
  const int n = first_ones(found, g.keep, g.group, most, [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) f(x[v][e], first + v * kThreads * VEC + e);
  }, [&](int rank, float v, int i) {
    g.value[list + rank] = v;
    g.index[list + rank] = i;
  });
  for (int k = n + tid; k < g.keep; k += kThreads) g.value[list + k] = -INFINITY;
  if (tid == 0) {
    top = of_wave[0][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, of_wave[w][0]);
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += scaled(of_wave[w][1], of_wave[w][0], top);
    g.sums[part * 2] = top;
    g.sums[part * 2 + 1] = sum;
  }
}

// One block: a prompt.
__global__ void __launch_bounds__(kThreads) beam_rank(BeamArgs g) {
  __shared__ Found<double> found;
  __shared__ double top[64], rest[64];      // of each beam the maximum, and score minus the logarithm of the sum behind it
  const int tid = threadIdx.x, lane = tid % kWave, per = g.splits * g.keep, all = g.beams * per;
  const int64_t row0 = (int64_t)blockIdx.x * g.beams;
  for (int i = tid / kWave; i < g.beams; i += kWaves) {
    const float* sums = g.sums + (row0 + i) * g.splits * 2;
    const float score = g.scores[row0 + i];
    const bool dead = !(score > -INFINITY) || (g.ended && g.ended[row0 + i] != 0);
    float m = -INFINITY;
    double sum = 0;
    if (!dead) {
      for (int p = lane; p < g.splits; p += kWave) m = fmaxf(m, sums[2 * p]);
      m = wave_max(m);
      for (int p = lane; p < g.splits; p += kWave) sum += sums[2 * p] == m ? (double)sums[2 * p + 1] : (double)sums[2 * p + 1] * exp((double)sums[2 * p] - (double)m);
#pragma unroll
      for (int o = kWave / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    }
    if (lane == 0) {
      top[i] = m;
      rest[i] = dead ? -INFINITY : (double)score - log(sum);
    }
  }
  __syncthreads();
  // entry e of the prompt's lists
  auto entry = [&](int e, double& total, int& place) {
    const int i = e / per, in = e - i * per;
    total = -INFINITY;
    place = i * g.vocab;
    if (g.ended && g.ended[row0 + i] != 0) {
      if (in == 0) { total = g.scores[row0 + i]; place += g.end; }
    } else if (rest[i] > -INFINITY) {
      const float v = g.value[row0 * per + e];
      if (v > -INFINITY) {
        total = v == (float)top[i] ? rest[i] : (double)v - top[i] + rest[i];
        place += g.index[row0 * per + e];
      }
    }
  };
  double most = -INFINITY;
  for (int e = tid; e < all; e += kThreads) {
    double total;
    int place;
    entry(e, total, place);
    most = fmax(most, total);
  }
  const int64_t out = (int64_t)blockIdx.x * g.keep;
  const int n = first_ones(found, g.keep, g.group, most, [&](auto f) {
    for (int e = tid; e < all; e += kThreads) {
      double total;
      int place;
      entry(e, total, place);
      f(total, place);
    }
  }, [&](int rank, double total, int place) {
    const int i = place / g.vocab, t = place - i * g.vocab;
    g.scores_out[out + rank] = (float)total;
    g.parent[out + rank] = (int)(row0 + i);
    g.token[out + rank] = t;
    if (g.ended_out) g.ended_out[out + rank] = t == g.end || (g.ended && g.ended[row0 + i] != 0);
  });
  for (int k = n + tid; k < g.keep; k += kThreads) {
    g.scores_out[out + k] = -INFINITY;
    g.parent[out + k] = g.token[out + k] = -1;
    if (g.ended_out) g.ended_out[out + k] = 0;
  }
}

struct Shape { int vectors, splits; };
Shape shape(int64_t rows, int64_t vocab, int dtype) {
  const int vec = dtype == AC_BF16 ? 8 : 4;
  Shape s{4, 0};
  auto splits = [&](int v) { return (int)((vocab + kThreads * vec * v - 1) / (kThreads * vec * v)); };
  while (s.vectors > 1 && rows * splits(s.vectors) < 1024) s.vectors /= 2;
  s.splits = splits(s.vectors);
  return s;
}

}  // namespace

uint64_t beam_select_workspace_bytes(int64_t batch, int beams, int64_t vocab, int keep, int dtype) {
  return (uint64_t)(batch * beams) * shape(batch * beams, vocab, dtype).splits * (2 + 2 * keep) * 4;
}

hipError_t launch_beam_select(const BeamSelectArgs& b, hipStream_t s) {
  const Shape sh = shape(b.batch * b.beams, b.vocab, b.dtype);
  const int64_t parts = b.batch * b.beams * sh.splits;
  float* const w = (float*)b.workspace;
  BeamArgs g{b.logits, b.ld, b.scores, b.ended, b.scores_out, b.parent, b.token, b.ended_out, b.beams, (int)b.vocab, b.keep, b.end, sh.splits,
             b.keep <= 8 ? 16 : b.keep <= 16 ? 8 : b.keep <= 32 ? 4 : 2, w, w + 2 * parts, (int32_t*)(w + (2 + b.keep) * parts)};
  const dim3 grid((unsigned)sh.splits, (unsigned)b.beams, (unsigned)b.batch);
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
