// out = act(x W^T + bias) + residual with weights W[n][k] = (code - zero) * scale held in 4 bits, one scale (and zero) for each group
// of `group` columns of a row: the linear layers of a decoding step, whose few rows read every weight once.
//
// The codes go to the matrix cores as they are.  A bf16 with the code in the upper bits of its mantissa is 1 + code / 16 exactly
// (0x3f80 | code << 3), one shift and one and-or for two codes, so per group
//   sum_k x (code - zero) / 16 = sum_k x (1 + code / 16) - (1 + zero / 16) sum_k x,
// no larger than the sums of x themselves (with 16 + code, rows whose sums are a 32nd of fp32's range became infinities and their difference NaN),
// both sums by v_mfma_f32_16x16x32_bf16 in fp32 (the second with a matrix of ones, which leaves it in the layout of the first), and the
// scale multiplies a group's sum once, in fp32: no weight is ever rounded.  fp32 rows are three bf16 terms that sum to them exactly.
#include "common.h"

namespace ac {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 128;   // columns a wave takes at a time: 16 bytes of codes a lane

// Slots 0..7 of a fragment hold columns 0 4 1 5 2 6 3 7, the order in which a word of eight codes comes apart.
constexpr int kSlot[8] = {0, 4, 1, 5, 2, 6, 3, 7};

// Eight numbers of a row of x as NT bf16 terms in the order of the slots.  An fp32 number is three terms that sum to it.
template <typename T> struct Eight { T v[8]; };
__device__ __forceinline__ void to_terms(const Eight<bf16_t>& x, bf16x8 (&f)[1]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[0][i] = x.v[kSlot[i]];
}
__device__ __forceinline__ void to_terms(const Eight<float>& x, bf16x8 (&f)[3]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const Bf16Terms b = split_bf16(x.v[kSlot[i]]);
    f[0][i] = b.hi; f[1][i] = b.mid; f[2][i] = b.lo;
  }
}
// row[k .. k + 8): whole, or (MASKED) zeros from `cols` on.
template <bool MASKED, typename T>
__device__ __forceinline__ Eight<T> load_eight(const T* row, int k, int cols) {
  constexpr int V = Elem<T>::kVec;
  typedef T vec __attribute__((ext_vector_type(V)));
  Eight<T> r;
  if (MASKED) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = row[min(k + i, cols - 1)];
    int left = cols - k;
    asm volatile("" : "+v"(left));                       // (conditions of this piece alone: those of all, shared by the rows, were spilled)
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = i < left ? r.v[i] : (T)0.0f;
  } else {
#pragma unroll
    for (int j = 0; j < 8 / V; ++j) {
      const vec t = *reinterpret_cast<const vec*>(row + k + j * V);
#pragma unroll
      for (int i = 0; i < V; ++i) r.v[j * V + i] = t[i];
    }
  }
  return r;
}

// Word i of the lanes of quarter q of a wave becomes word q of quarter i.
__device__ __forceinline__ void transpose_quarters(u32x4& w) {
  auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  w = u32x4{(uint32_t)c[0], (uint32_t)c[1], (uint32_t)d[0], (uint32_t)d[1]};
}

__device__ __forceinline__ bf16x8 codes_over_16(uint32_t w) {
  u32x4 r;
  r[0] = (w << 3 & 0x00780078u) | 0x3f803f80u;
  r[1] = (w >> 1 & 0x00780078u) | 0x3f803f80u;
  r[2] = (w >> 5 & 0x00780078u) | 0x3f803f80u;
  r[3] = (w >> 9 & 0x00780078u) | 0x3f803f80u;
  return __builtin_bit_cast(bf16x8, r);
}

// NaN stays NaN in every activation here, ReLU's too: of an infinity in x the sums above make NaN, which must not come out as 0.
__device__ __forceinline__ float relu(float v) { return v < 0.f ? 0.f : v; }

// A block owns 16 * MB rows and 16 * CT columns; its waves take steps of 128 columns of k in turn, the next ones' codes and scales on their way while one
// is multiplied, and add their sums in LDS, in the order of the waves.  SUBS: runs of 32 columns that share a scale within a step (1, 2 or 4).
// One row 2048 x 2048 (2 MB of codes) 4.2 us and 16 rows 8192 x 2048 7.4, both mostly a launch and the latency of what no one has read yet; 16 rows 8192 x 8192 16.4
// (34 MB, 2.1 TB/s), 32768 x 8192 51 (2.7 TB/s).  Bound by the lines that loads touch: a load takes 64 bytes of each of 16 rows of codes or of x, and of rows a
// power of two apart few lines stay (8192 x 8032 14 us).  Loads that the compiler can count (none under a condition, x one or two steps ahead, again behind the end)
// took longer, and other orders of the steps made no difference.
constexpr int kMostWaves = 8;

template <typename T> struct Pair;                     // a group's scale and zero
template <> struct Pair<bf16_t> {
  uint32_t w;
  __device__ __forceinline__ static Pair of(bf16_t s, bf16_t z) { return Pair{__builtin_bit_cast(uint16_t, s) | (uint32_t)__builtin_bit_cast(uint16_t, z) << 16}; }
  __device__ __forceinline__ float scale() const { return __builtin_bit_cast(float, w << 16); }
  __device__ __forceinline__ float zero() const { return __builtin_bit_cast(float, w & 0xffff0000u); }
};
template <> struct Pair<float> {
  float s, z;
  __device__ __forceinline__ static Pair of(float s, float z) { return Pair{s, z}; }
  __device__ __forceinline__ float scale() const { return s; }
  __device__ __forceinline__ float zero() const { return z; }
};

// Scales and zeros lie in LDS, chunk_steps steps' at a time, a column's `pitch` apart: as a lane's own loads, two bytes of each of sixteen rows, they took as long as codes
// and x (16 rows 32768 x 8192 69 us, 8192 x 8192 21; one row 8192 x 2048 in groups of 32 12.2 and now 7.5).
template <typename T, int NT, int MB, int CT, int SUBS, bool VEC>
__global__ void __launch_bounds__(kMostWaves * 64) linear_w4(LinearW4Args g, int chunk_steps, int pitch) {
  extern __shared__ __attribute__((aligned(16))) float joined[];   // [waves][16 MB][16 CT], before that Pair<T> [16 CT][pitch]
  Pair<T>* const pairs = reinterpret_cast<Pair<T>*>(joined);
  constexpr int ROWS = 16 * MB, COLS = 16 * CT, GS = 4 / SUBS, AHEAD = 2;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const int c16 = lane % 16, quarter = lane / 16;
  const int64_t n0 = (int64_t)blockIdx.x * COLS, m0 = (int64_t)blockIdx.y * ROWS;
  const uint8_t* w[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int64_t n = n0 + 16 * c + c16 < g.n ? n0 + 16 * c + c16 : g.n - 1;
    w[c] = (const uint8_t*)g.w + n * g.ldw;
  }
  const T* x[MB];
#pragma unroll
  for (int r = 0; r < MB; ++r) {
    const int64_t m = m0 + 16 * r + c16 < g.m ? m0 + 16 * r + c16 : g.m - 1;     // (rows past the last are the last again, and are not stored)
    x[r] = (const T*)g.x + m * g.ldx + quarter * 8;
  }
  f32x4 total[MB][CT];
#pragma unroll
  for (int r = 0; r < MB; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c) total[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (bf16_t)1.0f;

  const int groups = quotient((int)g.k - 1, g.group) + 1;
  const uint32_t last_piece = ((int)g.k - 1) / 2 & ~15;
  struct Step { u32x4 codes[CT]; };
  auto load_x = [&](int r, int k0, Eight<T> (&to)[4]) __attribute__((always_inline)) {
    if (VEC && k0 + kStep <= (int)g.k) {
#pragma unroll
      for (int j = 0; j < 4; ++j) to[j] = load_eight<false>(x[r], k0 + j * 32, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) to[j] = load_eight<true>(x[r], k0 + j * 32, (int)g.k - quarter * 8);
    }
  };
  // (past the end of k, where x is zero, codes that are there)
  auto fetch = [&](int k0) __attribute__((always_inline)) {
    Step s;
    const uint32_t at = min((uint32_t)k0 / 2 + quarter * 16, last_piece);
#pragma unroll
    for (int c = 0; c < CT; ++c) s.codes[c] = *reinterpret_cast<const u32x4*>(w[c] + at);
    return s;
  };
  const int steps = ((int)g.k + kStep - 1) / kStep;
  Step ring[AHEAD];
#pragma unroll
  for (int d = 0; d < AHEAD; ++d)
    if (wave + d * waves < steps) ring[d] = fetch((wave + d * waves) * kStep);
  // four columns a wave and 16 groups of each at a time
  constexpr int PASSES = COLS / 16;                      // of four waves
  auto load_pairs = [&](int first, int count) __attribute__((always_inline)) {
    for (int j = lane % 16; j < count; j += 16) {
      T s[PASSES], z[PASSES];
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int64_t n = min(n0 + min((p * waves + wave) * 4 + lane / 16, COLS - 1), g.n - 1);
        s[p] = ((const T*)g.scale)[n * g.lds + first + j];
        z[p] = (T)8.0f;
        if (g.zero) z[p] = ((const T*)g.zero)[n * g.ldz + first + j];
      }
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int col = (p * waves + wave) * 4 + lane / 16;
        if (col < COLS) pairs[col * pitch + j] = Pair<T>::of(s[p], z[p]);
      }
    }
  };
  int i0 = wave;
  for (int c0 = 0; c0 < steps; c0 += chunk_steps) {
    const int c1 = min(c0 + chunk_steps, steps), g0 = quotient(c0 * kStep, g.group);
    if (c0 > 0) __syncthreads();
    load_pairs(g0, min(quotient(c1 * kStep - 1, g.group), groups - 1) + 1 - g0);
    __syncthreads();
    for (; i0 < c1; i0 += waves * AHEAD) {
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) {
        const int i = i0 + d * waves, k0 = i * kStep;
        if (i >= steps) break;
        Step& now = ring[d];
        bf16x8 xf[MB][4][NT];
#pragma unroll
        for (int r = 0; r < MB; ++r) {
          Eight<T> raw[4];
          load_x(r, k0, raw);
#pragma unroll
          for (int j = 0; j < 4; ++j) to_terms(raw[j], xf[r][j]);
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) transpose_quarters(now.codes[c]);
#pragma unroll
        for (int e = 0; e < GS; ++e) {
          f32x4 sum[MB], part[MB][CT];
#pragma unroll
          for (int r = 0; r < MB; ++r) {
            sum[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = e * SUBS; j < (e + 1) * SUBS; ++j)
#pragma unroll
              for (int t = NT - 1; t >= 0; --t) sum[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[r][j][t], ones, sum[r], 0, 0, 0);
          }
#pragma unroll
          for (int c = 0; c < CT; ++c) {
#pragma unroll
            for (int r = 0; r < MB; ++r) part[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = e * SUBS; j < (e + 1) * SUBS; ++j) {
              const bf16x8 wf = codes_over_16(now.codes[c][j]);
#pragma unroll
              for (int r = 0; r < MB; ++r)
#pragma unroll
                for (int t = NT - 1; t >= 0; --t) part[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[r][j][t], wf, part[r][c], 0, 0, 0);
            }
            const Pair<T> pair = pairs[(16 * c + c16) * pitch + min(quotient(k0 + e * SUBS * 32, g.group), groups - 1) - g0];
            const float s = pair.scale(), off = fmaf(pair.zero(), -0.0625f, -1.0f);
#pragma unroll
            for (int r = 0; r < MB; ++r)
#pragma unroll
              for (int i = 0; i < 4; ++i) total[r][c][i] = fmaf(s, fmaf(off, sum[r][i], part[r][c][i]), total[r][c][i]);
          }
        }
        if (i + AHEAD * waves < steps) now = fetch((i + AHEAD * waves) * kStep);
      }
    }
  }
  __syncthreads();

  // what the first element that this thread finishes is joined with, on its way before the waves meet
  const int e0 = threadIdx.x;
  const bool mine = e0 < ROWS * COLS && m0 + e0 / COLS < g.m && n0 + e0 % COLS < g.n;
  const float bias0 = mine && g.bias ? Elem<T>::ld((const T*)g.bias + n0 + e0 % COLS) : 0.f;
  const float resid0 = mine && g.resid ? Elem<T>::ld((const T*)g.resid + (m0 + e0 / COLS) * g.ldr + n0 + e0 % COLS) : 0.f;
#pragma unroll
  for (int r = 0; r < MB; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) joined[(wave * ROWS + 16 * r + 4 * quarter + i) * COLS + 16 * c + c16] = total[r][c][i];
  __syncthreads();
  for (int e = e0; e < ROWS * COLS; e += blockDim.x) {
    const int64_t m = m0 + e / COLS, n = n0 + e % COLS;
    if (m >= g.m || n >= g.n) continue;
    float v = 0.f;
    for (int u = 0; u < waves; ++u) v += joined[u * ROWS * COLS + e];
    v = fmaf(v, 16.0f, e == e0 ? bias0 : g.bias ? Elem<T>::ld((const T*)g.bias + n) : 0.f);
    v = g.act == AC_ACT_RELU ? relu(v) : apply_act_rt(v, g.act);
    v += e == e0 ? resid0 : g.resid ? Elem<T>::ld((const T*)g.resid + m * g.ldr + n) : 0.f;
    Elem<T>::st((T*)g.out + m * g.ldo + n, v);
  }
}

template <typename T, int NT, int MB, int CT, bool VEC>
hipError_t launch_subs(const LinearW4Args& g, hipStream_t s) {
  const int64_t steps = (g.k + kStep - 1) / kStep;
  int waves = 4;
  while (waves < kMostWaves && waves < steps) waves *= 2;
  const dim3 grid((unsigned)((g.n + 16 * CT - 1) / (16 * CT)), (unsigned)((g.m + 16 * MB - 1) / (16 * MB)));
  static_assert((size_t)kMostWaves * 16 * MB * 16 * CT * sizeof(float) <= 64 * 1024, "the waves' sums fit what a kernel has unasked");
  // chunks of whole rounds of the waves' steps
  const int64_t round = 2 * waves * kStep, a_round = round / g.group.d + 2, room = 32768 / (16 * CT * 2 * (int64_t)sizeof(T));
  const int64_t rounds = room > a_round ? room / a_round : 1, groups = (g.k + g.group.d - 1) / g.group.d, most = rounds * round / g.group.d + 2;
  const int pitch = (int)(groups < most ? groups : most) | 1;            // (odd: sixteen columns in sixteen banks)
  size_t lds = (size_t)waves * 16 * MB * 16 * CT * sizeof(float);
  if (lds < 16 * CT * 2 * sizeof(T) * pitch) lds = 16 * CT * 2 * sizeof(T) * pitch;
  if (lds > 64 * 1024) return hipErrorInvalidValue;
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(waves * kWave), lds, s, g, (int)(rounds * 2 * waves), pitch);
    return hipGetLastError();
  };
  if constexpr (CT * NT < 12) {
    if (g.group.d == 64) return run(linear_w4<T, NT, MB, CT, 2, VEC>);
    if constexpr (CT < 4) {
      if (g.group.d == 32) return run(linear_w4<T, NT, MB, CT, 1, VEC>);
    }
  }
  return run(linear_w4<T, NT, MB, CT, 4, VEC>);
}

template <typename T, int NT, int MB, int CT>
hipError_t launch_vec(const LinearW4Args& g, hipStream_t s) {
  constexpr int64_t V = Elem<T>::kVec;
  const bool vec = (uintptr_t)g.x % 16 == 0 && (g.m == 1 || g.ldx % V == 0);
  return vec ? launch_subs<T, NT, MB, CT, true>(g, s) : launch_subs<T, NT, MB, CT, false>(g, s);
}

// Column tiles of a wave share what it does for x: as many as leave a block for each of the 256 CUs (small groups at most two, for registers).  us, one tile and as
// many: 16 rows 8192 x 2048 8.7 and 7.5 (two tiles, 256 blocks), 16 rows 32768 x 8192 81 and 51 (four, 512); 64 rows 8192 x 2048 27 and 13 (four); fp32 512 rows 4096 x 1024 108 and 42 (four).
template <typename T, int NT, int MB>
hipError_t launch_columns(const LinearW4Args& g, hipStream_t s) {
  const int64_t rows = (g.m + 16 * MB - 1) / (16 * MB), columns = (g.n + 15) / 16;
  if (rows * ((columns + 3) / 4) >= 256 && g.group.d >= (NT == 3 ? 128 : 64)) return launch_vec<T, NT, MB, 4>(g, s);
  return rows * ((columns + 1) / 2) >= 256 ? launch_vec<T, NT, MB, 2>(g, s) : launch_vec<T, NT, MB, 1>(g, s);
}

// Rows a block: 32 share the weights' conversion, 16 fill the chip sooner and are taken below two blocks of 32 for each CU.  us, 32 and 16 rows: fp32 61 rows 1003 x 1096,
// groups of 32, 9.7 and 6.7 (126 blocks of 32); 64 rows 2048 x 2048 11.8 and 8.7 (256); 4096 x 2048 14.9 and 16.7 (512); bf16 64 rows 1024 x 8192 20 and 13 (128); 61 rows 2048 x
// 2048 7.6 and 6.7 (256); 300 rows 700 x 1000 10.0 and 6.6 (440); 64 rows 8192 x 2048 13 and 18 (1024).
template <typename T, int NT>
hipError_t launch_rows(const LinearW4Args& g, hipStream_t s) {
  const bool few = (g.m + 31) / 32 * ((g.n + 15) / 16) < 512;
  return g.m <= 16 || few ? launch_columns<T, NT, 1>(g, s) : launch_columns<T, NT, 2>(g, s);
}

// ---- many rows ---------------------------------------------------------------------------------------------------------
//
// Many rows are work for the matrix cores.  A block owns 128 rows and 128 columns; of its eight waves four own 32 columns each (whose codes are then converted
// once for all rows), and its two sets of four take a half of k each, so that two waves share a SIMD also where there are few blocks, and add up in LDS.  What no
// block has read yet takes two microseconds and more to come: x comes to LDS by direct loads, and the codes to the registers of the wave that multiplies
// with them, two steps of 64 columns of k at a time while the two before are multiplied, and blocks that read the same rows of x at a time begin at different
// steps, so that one has them brought to the cache for the others.  Codes become (code - zero) / 16 in bf16, exact for whole zeros; of
// another the whole part goes there and the rest, which bf16 holds as well, times x is a second product.  A group's sum is scaled in fp32.  Scales and zeros of eight groups at a time lie in LDS, each wave's its own.
//
// 512 rows 6144 x 2048, 192 blocks: 28.8 us, 450 TFLOP/s; 4096 rows 8192 x 2048 208 us, 660 (zeros that are no whole numbers: 39 and 304).  A step of the eight waves takes 1.4 us: 0.4 of matrix instructions on a
// SIMD, 0.5 to read x from LDS, and 0.7 to issue what converts codes and scales sums, which overlap in part.  With one step at a time and a barrier
// after each a twentieth more.
constexpr int kTileM = 128, kTileN = 128, kTileK = 64, kStages = 4;
constexpr int kXBytes = kTileM * kTileK * 2;
constexpr int kSetBytes = kStages * kXBytes + 4 * 2 * 1024;          // of a set of four waves: x, and two times eight groups' scales and zeros of each wave

// Sixteenths of codes 0 .. 7 of a word, less `zero`, as bf16 in their own order.  Read as e4m3, a byte of 0 .. 15 is that number times 2^-9 (0 .. 7 are its subnormal
// numbers, 8 .. 15 the ones with the least exponent): one conversion with the scale 2^5 makes fp32 of two.
__device__ __forceinline__ bf16x8 codes_less(uint32_t w, float zero) {
  const uint32_t even = w & 0x0f0f0f0fu, odd = w >> 4 & 0x0f0f0f0fu;
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(even, 32.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(odd, 32.f, false);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(even, 32.f, true), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(odd, 32.f, true);
  return bf16x8{f2bf(a[0] - zero), f2bf(b[0] - zero), f2bf(a[1] - zero), f2bf(b[1] - zero), f2bf(c[0] - zero), f2bf(d[0] - zero), f2bf(c[1] - zero), f2bf(d[1] - zero)};
}

// Of a zero's sixteenth the part that codes_less takes, whose differences fit bf16; what is left does as well.
__device__ __forceinline__ float whole_part(float zero) { return fabsf(zero) <= 240.f ? rintf(zero) * 0.0625f : 0.f; }

template <int ACT> __device__ __forceinline__ void activate8(float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = ACT == AC_ACT_RELU ? relu(v[e]) : apply_act_bf16<ACT>(v[e]);
}
__device__ __forceinline__ void activate(float (&v)[8], int act) {
  switch (act) {
    case AC_ACT_GELU_ERF: return activate8<AC_ACT_GELU_ERF>(v);
    case AC_ACT_GELU_TANH: return activate8<AC_ACT_GELU_TANH>(v);
    case AC_ACT_RELU: return activate8<AC_ACT_RELU>(v);
    case AC_ACT_SIGMOID: return activate8<AC_ACT_SIGMOID>(v);
    case AC_ACT_SILU: return activate8<AC_ACT_SILU>(v);
    default: return;
  }
}

// GS: groups of a step.
template <int GS>
__global__ void __launch_bounds__(512, 2) linear_w4_tiles(LinearW4Args g) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), l32 = lane % 32, half = lane / 32;
  const int set = wave / 4, w4 = wave % 4;
  const int64_t m0 = (int64_t)blockIdx.y * kTileM, n0 = (int64_t)blockIdx.x * kTileN;
  uint8_t* const ring = smem + set * kSetBytes;
  uint8_t* const scales = ring + kStages * kXBytes + w4 * 2048;          // [2][scale, zero][32][8]
  const int all = ((int)g.k + kTileK - 1) / kTileK, steps = (all + 1) / 2, first = set * steps;    // (the second set's last step may lie past k: zeros)
  const int groups = quotient((int)g.k - 1, g.group) + 1, col = w4 * 32 + l32;
  // consecutive blocks are on different XCDs; those of one that share rows of x begin at different steps
  const int turn = (blockIdx.x / 8 * 3) % steps;
  auto step_of = [&](int t) { return first + (t + turn >= steps ? t + turn - steps : t + turn); };

  // Direct loads by buffer addresses: base and step in scalar registers, 32 bits a lane; an offset past the buffer's range brings zeros.  (The compiler
  // waits for all loads in flight before it uses the result of any while a direct load of the other kind is among them.)
  constexpr uint32_t kPastRange = 0x80000000u;
  auto to_lds = [](const void* base, uint32_t lane_off, uint32_t off, uint8_t* to) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, 0x7fffffff, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)to, 16, lane_off, off, 0, 0);
  };
  // 1 KB a load: eight rows of x, the eight pieces of a row turned by the row.  Rows past the last are the last again.
  const int xpiece = (lane % 8 ^ lane / 8) * 8;
  const bf16_t* const x0 = (const bf16_t*)g.x + m0 * g.ldx;
  uint32_t xoff[kXBytes / 4096];
#pragma unroll
  for (int n = 0; n < kXBytes / 4096; ++n) xoff[n] = (uint32_t)(min((int64_t)(n * 32 + w4 * 8 + lane / 8), g.m - 1 - m0) * g.ldx + xpiece) * 2;
  auto load_x = [&](int t, int stage) __attribute__((always_inline)) {
    const int k0 = t < steps ? step_of(t) * kTileK : (int)g.k;
    const bool in = k0 + xpiece < (int)g.k;
#pragma unroll
    for (int n = 0; n < kXBytes / 4096; ++n) to_lds(x0, in ? xoff[n] : kPastRange, (uint32_t)k0 * 2, ring + stage * kXBytes + w4 * 1024 + n * 4096);
  };
  // a lane's codes of a step: of its column, columns 32 half .. 32 half + 31 of k (past the last, where x is zero, some that are there)
  const uint8_t* const w0 = (const uint8_t*)g.w + n0 * g.ldw;
  const uint32_t woff = (uint32_t)(min((int64_t)col, g.n - 1 - n0) * g.ldw), wlast = ((int)g.k - 1) / 2 & ~15;
  auto load_w = [&](int t) __attribute__((always_inline)) {
    return *reinterpret_cast<const u32x4*>(w0 + woff + min((uint32_t)step_of(t) * (kTileK / 2) + half * 16, wlast));
  };
  // Groups 8 c .. 8 c + 7 of the lane's column, the scales in the lower half of the wave and the zeros in the upper, to their place.
  const int sn = (int)min((int64_t)col, g.n - 1 - n0);
  const bf16_t *const s0 = (const bf16_t*)g.scale + n0 * g.lds, *const z0 = g.zero ? (const bf16_t*)g.zero + n0 * g.ldz : s0;
  const uint32_t soff = (uint32_t)(sn * (half && g.zero ? g.ldz : g.lds)) * 2;
  const bool wide = g.lds % 8 == 0 && (uintptr_t)g.scale % 16 == 0 && (!g.zero || (g.ldz % 8 == 0 && (uintptr_t)g.zero % 16 == 0));
  auto load_scales = [&](int c, int place) __attribute__((always_inline)) {
    if (wide && 8 * c + 8 <= groups) {
      if (half == 0) to_lds(s0, soff, 16 * c, scales + place * 1024);
      else to_lds(z0, soff, 16 * c, scales + place * 1024);
    } else {
      const bf16_t* const from = (half ? z0 : s0) + soff / 2;
      uint16_t v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __builtin_bit_cast(uint16_t, from[min(8 * c + e, groups - 1)]);
#pragma unroll
      for (int e = 0; e < 8; ++e) reinterpret_cast<uint16_t*>(scales + place * 1024 + lane * 16)[e] = v[e];
    }
  };
  auto chunk_of = [&](int step) { return min(quotient(step * kTileK, g.group), groups - 1) / 8; };
  const int chunk_first = chunk_of(first), chunk_last = chunk_of(first + steps - 1);
  auto chunk_after = [&](int c) { return c == chunk_last ? chunk_first : c + 1; };

  // this wave's loads have landed and its LDS reads are done; and every wave's
  auto landed = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(7 << 4);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto arrived = [&]() __attribute__((always_inline)) {
    landed();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  f32x16 total[4], zero16;
#pragma unroll
  for (int x = 0; x < 16; ++x) zero16[x] = 0.f;
#pragma unroll
  for (int r = 0; r < 4; ++r) total[r] = zero16;

  u32x4 codes[kStages];
  int chunk = chunk_of(step_of(0)), place = 0;
  bool asked = false;            // whether a chunk's scales have been asked for since the last barrier
  load_scales(chunk, 0);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    codes[t] = load_w(t);
    load_x(t, t);
  }
  load_scales(chunk_after(chunk), 1);
  arrived();
  for (int t0 = 0; t0 < steps; t0 += kStages) {
#pragma unroll
    for (int u = 0; u < kStages; ++u) {
      const int t = t0 + u;
      if (t >= steps) break;
      const int step = step_of(t), g0 = quotient(step * kTileK, g.group), c = min(g0, groups - 1) / 8;
      // A chunk's scales are on their way from the first step of the chunk before it, and every second step ends with all loads landed.  Where a set's part of k begins
      // or ends in the middle of a chunk, that chunk may be one step, an even one, and no barrier lies behind it: then the wave waits for its own loads.
      if (u % 2 == 0) asked = false;
      if (c != chunk) {
        if (asked) landed();
        asked = true;
        chunk = c;
        place ^= 1;
        load_scales(chunk_after(chunk), place ^ 1);      // (over those of the chunk before, which are not read any more)
      }
      if (u % 2 == 0) {
#pragma unroll
        for (int v = 2; v < 4; ++v) {
          codes[(u + v) % kStages] = load_w(t + v);
          load_x(t + v, (u + v) % kStages);
        }
      }
      const uint8_t* const xt = ring + u * kXBytes + l32 * (kTileK * 2);
      u32x4 cw = codes[u];
      // product q takes 16 columns of k: word q of the lane's codes, columns 32 half + 8 q; with groups of 32 words change halves first, so that both
      // halves of the wave are in one group
      if (GS == 2) {
        auto a = __builtin_amdgcn_permlane32_swap(cw[0], cw[1], false, false);
        auto b = __builtin_amdgcn_permlane32_swap(cw[2], cw[3], false, false);
        cw = u32x4{(uint32_t)a[0], (uint32_t)b[0], (uint32_t)a[1], (uint32_t)b[1]};
      }
      auto x_frag = [&](int q, int r) __attribute__((always_inline)) {
        const int piece = GS == 2 ? 2 * q + half : half * 4 + q;
        return *reinterpret_cast<const bf16x8*>(xt + r * 32 * (kTileK * 2) + (piece ^ (l32 & 7)) * 16);
      };
      float s[GS], z[GS], z_rest[GS];
#pragma unroll
      for (int e = 0; e < GS; ++e) {
        const uint8_t* const at = scales + place * 1024 + l32 * 16 + min(g0 + e, groups - 1) % 8 * 2;
        s[e] = bf2f(*reinterpret_cast<const bf16_t*>(at));
        const float zero = g.zero ? bf2f(*reinterpret_cast<const bf16_t*>(at + 512)) : 8.f;
        z[e] = whole_part(zero);
        z_rest[e] = fmaf(zero, 0.0625f, -z[e]);
      }
      const bool second = g.zero && __any(z_rest[0] != 0.f || z_rest[GS - 1] != 0.f);
      // a product's fragments are read and its codes converted under the one before
      bf16x8 a[4], b[2];
#pragma unroll
      for (int r = 0; r < 4; ++r) a[r] = x_frag(0, r);
      b[0] = codes_less(cw[0], z[0]);
      constexpr int EACH = 4 / GS;
#pragma unroll
      for (int e = 0; e < GS; ++e) {
        f32x16 part[4];
#pragma unroll
        for (int p = 0; p < EACH; ++p) {
          const int q = e * EACH + p;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            part[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[r], b[q & 1], p == 0 ? zero16 : part[r], 0, 0, 0);
            if (q < 3) a[r] = x_frag(q + 1, r);
          }
          if (q < 3) b[(q + 1) & 1] = codes_less(cw[q + 1], z[(q + 1) / EACH]);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int x = 0; x < 16; ++x) total[r][x] = fmaf(s[e], part[r][x], total[r][x]);
        asm volatile("" : "+v"(total[0]), "+v"(total[1]), "+v"(total[2]), "+v"(total[3]));    // (here and not later, or the groups' sums live side by side)
        __builtin_amdgcn_sched_barrier(0);
      }
      if (second) {              // (behind the step's other products: between two groups' its branch took 4 % with groups of 32 whether taken or not)
#pragma unroll
        for (int e = 0; e < GS; ++e) {
          bf16x8 rest;
#pragma unroll
          for (int x = 0; x < 8; ++x) rest[x] = f2bf(-z_rest[e]);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            f32x16 part = zero16;
#pragma unroll
            for (int p = 0; p < EACH; ++p) part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x_frag(e * EACH + p, r), rest, part, 0, 0, 0);
#pragma unroll
            for (int x = 0; x < 16; ++x) total[r][x] = fmaf(s[e], part[x], total[r][x]);
          }
        }
      }
      if (u % 2 == 1) arrived();
    }
  }

  // the sums meet in LDS (no load is on its way to it any more), and leave it row by row
  __builtin_amdgcn_s_waitcnt(7 << 4);
  __syncthreads();
  float* const joined = reinterpret_cast<float*>(smem);            // [128][128]
#pragma unroll
  for (int pass = 1; pass >= 0; --pass) {
    if (set == pass) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          float* const at = joined + (r * 32 + 8 * (x / 4) + 4 * half + x % 4) * kTileN + col;
          *at = pass == 1 ? total[r][x] : total[r][x] + *at;
        }
    }
    __syncthreads();
  }
  const bool wide_out = g.ldo % 8 == 0 && (uintptr_t)g.out % 16 == 0 && (!g.resid || (g.ldr % 8 == 0 && (uintptr_t)g.resid % 16 == 0));
  const int c8 = threadIdx.x % 16 * 8;
  const int64_t n = n0 + c8;
  if (n >= g.n) return;
  const int cols = (int)min(g.n - n, (int64_t)8);
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = g.bias && e < cols ? bf2f(((const bf16_t*)g.bias)[n + e]) : 0.f;
  for (int row = threadIdx.x / 16; row < kTileM && m0 + row < g.m; row += 32) {
    const f32x4 lo = *reinterpret_cast<const f32x4*>(joined + row * kTileN + c8), hi = *reinterpret_cast<const f32x4*>(joined + row * kTileN + c8 + 4);
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = fmaf(lo[e], 16.0f, bias[e]); v[4 + e] = fmaf(hi[e], 16.0f, bias[4 + e]); }
    activate(v, g.act);
    bf16_t* const out = (bf16_t*)g.out + (m0 + row) * g.ldo + n;
    const bf16_t* const resid = (const bf16_t*)g.resid + (m0 + row) * g.ldr + n;
    if (wide_out && cols == 8) {
      if (g.resid) {
        float r[8];
        load_vec(resid, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += r[e];
      }
      store_vec(out, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < cols) out[e] = f2bf(g.resid ? v[e] + bf2f(resid[e]) : v[e]);
    }
  }
}

// Rows of x that direct loads can take: 16-byte pieces that hold columns of k alone; and offsets within a tile of 32 bits.
// Products of up to 64 tiles are left to the kernel above, which has blocks for the whole chip then (us, tiles and rows: 256 rows 2048 x 2048, 32 tiles, 26
// and 13; 512 rows 2048 x 2048, 64 tiles, 26 and 23, 2048 x 8192 84 and 58; 128 rows 8192 x 2048, 64, 26 and 24; 200 rows 6000 x 1000, 73 tiles' area, 17 and 25; 384 rows 4096 x 1024, 96, 17 and
// 24; 512 rows 6144 x 2048, 192, 27 and 66).
bool tiles_take(const LinearW4Args& g) {
  return g.dtype == AC_BF16 && g.m >= 96 && g.m * g.n > 64 * kTileM * kTileN && (uintptr_t)g.x % 16 == 0 && g.ldx % 8 == 0 && g.k % 8 == 0 && g.k < 1 << 22 && g.ldx < 1 << 22 && g.ldw < 1 << 24 &&
         g.lds < 1 << 22 && g.ldz < 1 << 22;
}

template <int GS>
hipError_t launch_tiles(const LinearW4Args& g, hipStream_t s) {
  constexpr size_t lds = 2 * kSetBytes;
  static_assert(lds >= 4 * 64 * 64 * sizeof(float) && lds <= 160 * 1024, "one block a CU");
  static const hipError_t attr_status = hipFuncSetAttribute(reinterpret_cast<const void*>(linear_w4_tiles<GS>),
                                                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (attr_status != hipSuccess) return attr_status;
  const dim3 grid((unsigned)((g.n + kTileN - 1) / kTileN), (unsigned)((g.m + kTileM - 1) / kTileM));
  hipLaunchKernelGGL((linear_w4_tiles<GS>), grid, dim3(512), lds, s, g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_w4(const LinearW4Args& g, hipStream_t s) {
  if (g.m <= 0 || g.n <= 0) return hipSuccess;
  if (tiles_take(g)) return g.group.d == 32 ? launch_tiles<2>(g, s) : launch_tiles<1>(g, s);
  return g.dtype == AC_BF16 ? launch_rows<bf16_t, 1>(g, s) : launch_rows<float, 3>(g, s);
}

}  // namespace ac
