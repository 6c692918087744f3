// out = act(x W^T + bias) + residual with weights W[n][k] = (code - zero) * scale held in 4 bits, one scale (and zero) for each group
// of `group` columns of a row: the linear layers of a decoding step, whose few rows read every weight once.
//
// The codes go to the matrix cores as they are.  A bf16 with the code in the upper bits of its mantissa is 16 + code exactly
// (0x4180 | code << 3), one shift and one and-or for two codes, so per group
//   sum_k x (code - zero) = sum_k x (16 + code) - (16 + zero) sum_k x,
// both sums by v_mfma_f32_16x16x32_bf16 in fp32 (the second with a matrix of ones, which leaves it in the layout of the first), and the
// scale multiplies a group's sum once, in fp32: no weight is ever rounded.  fp32 rows are three bf16 terms that sum to them exactly.
#include "common.h"

namespace ac {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 128;   // columns a wave takes at a time: 16 bytes of codes a lane

// Slots 0..7 of a fragment hold columns 0 4 1 5 2 6 3 7, the order in which a word of eight codes comes apart.
constexpr int kSlot[8] = {0, 4, 1, 5, 2, 6, 3, 7};

// x[row][k .. k + 8) as NT bf16 terms, zeros past the row's end.
template <bool VEC>
__device__ __forceinline__ void load_x(const bf16_t* row, int64_t k, int64_t cols, bf16x8 (&f)[1]) {
  bf16x8 v;
  if (VEC && k + 8 <= cols) {
    v = *reinterpret_cast<const bf16x8*>(row + k);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < cols ? row[k + i] : (bf16_t)0.0f;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[0][i] = v[kSlot[i]];
}
template <bool VEC>
__device__ __forceinline__ void load_x(const float* row, int64_t k, int64_t cols, bf16x8 (&f)[3]) {
  float v[8];
  if (VEC && k + 8 <= cols) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(row + k), b = *reinterpret_cast<const f32x4*>(row + k + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < cols ? row[k + i] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const Bf16Terms b = split_bf16(v[kSlot[i]]);
    f[0][i] = b.hi; f[1][i] = b.mid; f[2][i] = b.lo;
  }
}

// Word i of the lanes of quarter q of a wave becomes word q of quarter i.
__device__ __forceinline__ void transpose_quarters(u32x4& w) {
  auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  w = u32x4{(uint32_t)c[0], (uint32_t)c[1], (uint32_t)d[0], (uint32_t)d[1]};
}

__device__ __forceinline__ bf16x8 codes_plus_16(uint32_t w) {
  u32x4 r;
  r[0] = (w << 3 & 0x00780078u) | 0x41804180u;
  r[1] = (w >> 1 & 0x00780078u) | 0x41804180u;
  r[2] = (w >> 5 & 0x00780078u) | 0x41804180u;
  r[3] = (w >> 9 & 0x00780078u) | 0x41804180u;
  return __builtin_bit_cast(bf16x8, r);
}

// A block owns 16 * MB rows and 16 * CT columns; its waves take steps of 128 columns of k in turn and add their sums in LDS, in the
// order of the waves.  SUBS: runs of 32 columns that share a scale within a step (1, 2 or 4).
template <typename T, int NT, int MB, int CT, int SUBS, bool VEC>
__global__ void __launch_bounds__(512) linear_w4(LinearW4Args g) {
  extern __shared__ float joined[];   // [waves][16 MB][16 CT]
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
  const int c16 = lane % 16, quarter = lane / 16;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * CT), m0 = (int64_t)blockIdx.y * (16 * MB);
  const uint8_t* w[CT];
  const T *scale[CT], *zero[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int64_t n = n0 + 16 * c + c16 < g.n ? n0 + 16 * c + c16 : g.n - 1;
    w[c] = (const uint8_t*)g.w + n * g.ldw;
    scale[c] = (const T*)g.scale + n * g.lds;
    zero[c] = g.zero ? (const T*)g.zero + n * g.ldz : nullptr;
  }
  const T* x[MB];
#pragma unroll
  for (int r = 0; r < MB; ++r) {
    const int64_t m = m0 + 16 * r + c16;
    x[r] = m < g.m ? (const T*)g.x + m * g.ldx : nullptr;
  }
  f32x4 total[MB][CT];
#pragma unroll
  for (int r = 0; r < MB; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c) total[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (bf16_t)1.0f;

  const int64_t groups = (g.k + g.group - 1) / g.group;
  for (int64_t k0 = (int64_t)wave * kStep; k0 < g.k; k0 += (int64_t)waves * kStep) {
    u32x4 codes[CT];
    const int64_t at = k0 / 2 + quarter * 16;
#pragma unroll
    for (int c = 0; c < CT; ++c) codes[c] = 2 * at < g.k ? *reinterpret_cast<const u32x4*>(w[c] + at) : u32x4{0, 0, 0, 0};
    bf16x8 xf[MB][4][NT];
#pragma unroll
    for (int r = 0; r < MB; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (x[r]) {
          load_x<VEC>(x[r], k0 + j * 32 + quarter * 8, g.k, xf[r][j]);
        } else {
#pragma unroll
          for (int t = 0; t < NT; ++t) xf[r][j][t] = bf16x8{};
        }
      }
#pragma unroll
    for (int c = 0; c < CT; ++c) transpose_quarters(codes[c]);
#pragma unroll
    for (int j0 = 0; j0 < 4; j0 += SUBS) {
      const int64_t gi = (k0 + j0 * 32) / g.group < groups ? (k0 + j0 * 32) / g.group : groups - 1;
      f32x4 sum[MB], part[MB][CT];
#pragma unroll
      for (int r = 0; r < MB; ++r) {
        sum[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = j0; j < j0 + SUBS; ++j)
#pragma unroll
          for (int t = NT - 1; t >= 0; --t) sum[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[r][j][t], ones, sum[r], 0, 0, 0);
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
#pragma unroll
        for (int r = 0; r < MB; ++r) part[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = j0; j < j0 + SUBS; ++j) {
          const bf16x8 wf = codes_plus_16(codes[c][j]);
#pragma unroll
          for (int r = 0; r < MB; ++r)
#pragma unroll
            for (int t = NT - 1; t >= 0; --t) part[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[r][j][t], wf, part[r][c], 0, 0, 0);
        }
        const float s = Elem<T>::ld(scale[c] + gi), off = -16.0f - (zero[c] ? Elem<T>::ld(zero[c] + gi) : 8.0f);
#pragma unroll
        for (int r = 0; r < MB; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i) total[r][c][i] = fmaf(s, fmaf(off, sum[r][i], part[r][c][i]), total[r][c][i]);
      }
    }
  }

  constexpr int ROWS = 16 * MB, COLS = 16 * CT;
#pragma unroll
  for (int r = 0; r < MB; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) joined[(wave * ROWS + 16 * r + 4 * quarter + i) * COLS + 16 * c + c16] = total[r][c][i];
  __syncthreads();
  for (int e = threadIdx.x; e < ROWS * COLS; e += blockDim.x) {
    const int64_t m = m0 + e / COLS, n = n0 + e % COLS;
    if (m >= g.m || n >= g.n) continue;
    float v = 0.f;
    for (int u = 0; u < waves; ++u) v += joined[u * ROWS * COLS + e];
    if (g.bias) v += Elem<T>::ld((const T*)g.bias + n);
    v = apply_act_rt(v, g.act);
    if (g.resid) v += Elem<T>::ld((const T*)g.resid + m * g.ldr + n);
    Elem<T>::st((T*)g.out + m * g.ldo + n, v);
  }
}

template <typename T, int NT, int MB, int CT, bool VEC>
hipError_t launch_subs(const LinearW4Args& g, hipStream_t s) {
  const int waves = 4;
  const dim3 grid((unsigned)((g.n + 16 * CT - 1) / (16 * CT)), (unsigned)((g.m + 16 * MB - 1) / (16 * MB)));
  const size_t lds = (size_t)waves * 16 * MB * 16 * CT * sizeof(float);
  if (g.group == 32)
    hipLaunchKernelGGL((linear_w4<T, NT, MB, CT, 1, VEC>), grid, dim3(waves * kWave), lds, s, g);
  else if (g.group == 64)
    hipLaunchKernelGGL((linear_w4<T, NT, MB, CT, 2, VEC>), grid, dim3(waves * kWave), lds, s, g);
  else
    hipLaunchKernelGGL((linear_w4<T, NT, MB, CT, 4, VEC>), grid, dim3(waves * kWave), lds, s, g);
  return hipGetLastError();
}

template <typename T, int NT>
hipError_t launch_rows(const LinearW4Args& g, hipStream_t s) {
  constexpr int64_t V = Elem<T>::kVec;
  const bool vec = (uintptr_t)g.x % 16 == 0 && (g.m == 1 || g.ldx % V == 0);
  return vec ? launch_subs<T, NT, 1, 1, true>(g, s) : launch_subs<T, NT, 1, 1, false>(g, s);
}

}  // namespace

hipError_t launch_linear_w4(const LinearW4Args& g, hipStream_t s) {
  if (g.m <= 0 || g.n <= 0) return hipSuccess;
  return g.dtype == AC_BF16 ? launch_rows<bf16_t, 1>(g, s) : launch_rows<float, 3>(g, s);
}

}  // namespace ac
