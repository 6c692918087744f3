// A paged cache of keys and values in 8 bits: the append, which rotates and stores the rows of a step, and the attention that reads
// it.  Codes are e4m3 with one power-of-two scale for a block of 16 tokens of a head.
//
// Why a power of two: a block fills token by token, and where a later token asks for a larger scale the older codes move by whole
// exponents, exactly but for subnormal ones; with any other scale each move would round once more.  Why 16 tokens: the quarters of a
// wave then hold one block each, see the attention.
#include "cache.h"

namespace ac {

namespace {

// ---- append ----------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return __builtin_amdgcn_readfirstlane(v);
}

// The least power of two s >= 2^-100 with v <= 448 s, for the bits of 0 <= v < inf: 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_of(uint32_t u) {
  int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  if (e < 27) e = 27;
  return __builtin_bit_cast(float, (uint32_t)e << 23);
}

// Four numbers as e4m3, to nearest, ties to even; what is not finite becomes NaN.
__device__ __forceinline__ uint32_t to_e4m3(const float (&v)[4], bool finite) {
  uint32_t r = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], r, true);
  if (finite) return r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (!(fabsf(v[i]) < INFINITY)) r |= 0x7fu << (8 * i);
  return r;
}
__device__ __forceinline__ void from_e4m3(uint32_t c, float (&v)[4]) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
}
__device__ __forceinline__ uint32_t move_codes(uint32_t c, float ratio) {
  float v[4];
  from_e4m3(c, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] *= ratio;
  return to_e4m3(v, false);
}

__device__ __forceinline__ void load4(const float* p, float (&v)[4]) { load_vec(p, v); }
__device__ __forceinline__ void load4(const bf16_t* p, float (&v)[4]) {
  const bf16x4 t = *reinterpret_cast<const bf16x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = bf2f(t[i]);
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { store_vec(p, v); }
__device__ __forceinline__ void store4(bf16_t* p, const float (&v)[4]) {
  bf16x4 t;
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = f2bf(v[i]);
  *reinterpret_cast<bf16x4*>(p) = t;
}

// The products and the sum of a turned pair are rounded one by one, as the formula is written, so that the scale, which jumps at a
// power of two, comes out the same wherever it is computed so in fp32.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
  const float ac = a * c, bs = b * s, as = a * s, bc = b * c;
  a = ac - bs;
  b = as + bc;
}

struct AppendArgs {
  const void *q, *k, *v;
  void* q_out;
  int64_t ldq, ldqo, ldk, ldv;
  int heads;
  ac_kv_cache cache;
  CacheRows rows;
  ac_rotary rot;
  Divisor blocks;                                      // blocks of 16 tokens a page
};

// A lane holds, of one of a block's 16 tokens (four lanes a token), HD / 32 chunks of four pairs: elements lo .. lo + 3 and hi .. hi + 3.
struct Chunk { int pair, lo, hi; };
__device__ __forceinline__ Chunk chunk(const ac_rotary& r, int i, int sub) {
  const int j = 4 * (sub + 4 * i);
  return r.interleaved || j >= r.pairs ? Chunk{j, 2 * j, 2 * j + 4} : Chunk{j, j, j + r.pairs};
}

// Cosines and sines of a lane's chunks, for row `row`, which stands at place `place` of its sequence.
template <int CH>
struct Angles { float c[CH][4], s[CH][4]; };
template <int CH>
__device__ __forceinline__ void load_angles(const ac_rotary& r, int sub, int64_t row, int64_t place, Angles<CH>& a) {
  if (r.pairs == 0) return;
  // bytes from the tables' begin, which 32 bits hold
  auto table_row = [&](int64_t p) { return (uint32_t)(p < 0 ? 0 : p < r.table_rows ? p : r.table_rows - 1) * (uint32_t)r.ld_table * 4u; };
  if (r.axes == 1 || !r.positions) {
    const uint32_t at = table_row(r.positions ? r.positions[row] : place);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const uint32_t in = at + (4 * (sub + 4 * i) < r.pairs ? 16 * (sub + 4 * i) : 0);
      load_vec((const float*)((const char*)r.cos + in), a.c[i]);
      load_vec((const float*)((const char*)r.sin + in), a.s[i]);
    }
  } else {
    uint32_t at[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) at[x] = table_row(x < r.axes ? r.positions[x * r.ld_positions + row] : 0);
    const int e0 = r.section[0], e1 = e0 + r.section[1], e2 = e1 + (r.axes > 2 ? r.section[2] : 0);
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pair = 4 * (sub + 4 * i) < r.pairs ? 4 * (sub + 4 * i) + e : 0;
        const uint32_t in = (pair < e0 ? at[0] : pair < e1 || r.axes == 2 ? at[1] : pair < e2 || r.axes == 3 ? at[2] : at[3]) + 4u * pair;
        a.c[i][e] = *(const float*)((const char*)r.cos + in);
        a.s[i][e] = *(const float*)((const char*)r.sin + in);
      }
  }
}
template <int CH>
__device__ __forceinline__ void turn_chunk(const ac_rotary& r, int i, int sub, const Angles<CH>& g, float (&a)[4], float (&b)[4]) {
  if (4 * (sub + 4 * i) >= r.pairs) return;
  const float(&cs)[4] = g.c[i], (&sn)[4] = g.s[i];
  if (r.interleaved) {
    turn(a[0], a[1], cs[0], sn[0]); turn(a[2], a[3], cs[1], sn[1]);
    turn(b[0], b[1], cs[2], sn[2]); turn(b[2], b[3], cs[3], sn[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) turn(a[e], b[e], cs[e], sn[e]);
  }
}

enum { KEYS, VALUES, QUERIES };
template <typename T, int HD, int kind>
__device__ __forceinline__ void append_head(const AppendArgs& g, int h, uint8_t* turned) {
  constexpr int CH = HD / 32, VL = (HD + kWave - 1) / kWave;
  const int lane = threadIdx.x % kWave, sub = lane % 4, t = lane / 4, blocks = g.blocks.d;
  const int64_t b = blockIdx.z;
  const Sequence sq = sequence(g.rows, b);
  const int64_t first = sq.length - sq.rows;                          // tokens before the rows; what would stand before token 0 is dropped
  const int64_t from = first > 0 ? first : 0;
  if (from >= sq.length) return;
  const T* src = (const T*)(kind == KEYS ? g.k : kind == VALUES ? g.v : g.q);
  const int64_t ld = kind == KEYS ? g.ldk : kind == VALUES ? g.ldv : g.ldq;
  uint8_t* const store = (uint8_t*)(kind == KEYS ? g.cache.k : g.cache.v);
  float* const scales = kind == KEYS ? g.cache.k_scale : g.cache.v_scale;
  auto piece = [&](int i) {
    const Chunk c = chunk(g.rot, i, sub);
    return kind == VALUES ? Chunk{c.pair, 2 * c.pair, 2 * c.pair + 4} : c;
  };
  for (int64_t blk = from / kBlock + blockIdx.x; blk * kBlock < sq.length; blk += gridDim.x) {
    const int64_t place = blk * kBlock + t, near = place < from ? from : place < sq.length ? place : sq.length - 1, row = sq.begin + near - first;
    const bool fresh = place == near;
    const int nth = quotient((int)blk, g.blocks), in_page = (int)blk - nth * blocks;
    const int64_t id = kind != QUERIES && nth < g.rows.ld_page_table ? g.rows.page_table[b * g.rows.ld_page_table + nth] : -1;
    float x[CH][4], y[CH][4];
    const T* from_row = src + row * ld + h * HD;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const Chunk c = piece(i);
      load4(from_row + c.lo, x[i]);
      load4(from_row + c.hi, y[i]);
    }
    if constexpr (kind != VALUES) {
      Angles<CH> ang;
      load_angles(g.rot, sub, row, near, ang);
#pragma unroll
      for (int i = 0; i < CH; ++i) turn_chunk(g.rot, i, sub, ang, x[i], y[i]);
    }
    if constexpr (kind == QUERIES) {
      if (!fresh) continue;
      T* dst = (T*)g.q_out + row * g.ldqo + h * HD;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const Chunk c = piece(i);
        store4(dst + c.lo, x[i]);
        store4(dst + c.hi, y[i]);
      }
      continue;
    }
    if (id < 0 || id >= g.cache.pages) continue;
    const int old = from > blk * kBlock ? (int)(from - blk * kBlock) : 0, end = sq.length - blk * kBlock < kBlock ? (int)(sq.length - blk * kBlock) : kBlock;
    // a block's codes, of keys and of values, are HD * 16 bytes side by side
    const int64_t in_cache = (int64_t)h * blocks + in_page;
    uint8_t* codes = store + id * g.cache.stride_page + in_cache * (HD * kBlock);
    float* scale = scales + id * g.cache.stride_scale + in_cache;
    float before = 0.f;
    if (old > 0) before = *scale;
    u32x4 held[VL];
    if (kind == VALUES && (old > 0 || end < kBlock)) {
#pragma unroll
      for (int i = 0; i < VL; ++i) held[i] = *reinterpret_cast<const u32x4*>(codes + (lane + i * kWave < HD ? lane + i * kWave : HD - 1) * kBlock);
    }
    uint32_t largest = 0;                                           // in the order of the magnitudes' bits: numbers, infinity, NaN
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) largest = max(largest, max(magnitude(x[i][e]), magnitude(y[i][e])));
    largest = wave_max_u32(fresh ? largest : 0);
    const bool finite = largest < 0x7f800000u;
    if (!finite) {
      largest = 0;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t u = magnitude(x[i][e]), w = magnitude(y[i][e]);
          if (u < 0x7f800000u) largest = max(largest, u);
          if (w < 0x7f800000u) largest = max(largest, w);
        }
      largest = wave_max_u32(fresh ? largest : 0);
    }
    float s = scale_of(largest), ratio = 1.f;
    if (old > 0) s = fmaxf(s, before);
    const float inv = __builtin_bit_cast(float, 0x7f000000u - __builtin_bit_cast(uint32_t, s));      // 1 / s of a power of two
    if (old > 0) ratio = before * inv;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[i][e] *= inv; y[i][e] *= inv; }
    if constexpr (kind == KEYS) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const Chunk c = piece(i);
        uint32_t* lo = (uint32_t*)(codes + t * HD + c.lo);
        uint32_t* hi = (uint32_t*)(codes + t * HD + c.hi);
        if (fresh) {
          *lo = to_e4m3(x[i], finite);
          *hi = to_e4m3(y[i], finite);
        } else if (t < old && ratio != 1.f) {
          *lo = move_codes(*lo, ratio);
          *hi = move_codes(*hi, ratio);
        }
      }
    } else {
      if (fresh) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const int d = 8 * (sub + 4 * i);
          const uint32_t lo = to_e4m3(x[i], finite), hi = to_e4m3(y[i], finite);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            turned[(d + e) * kBlock + t] = (uint8_t)(lo >> (8 * e));
            turned[(d + 4 + e) * kBlock + t] = (uint8_t)(hi >> (8 * e));
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        const int d = lane + j * kWave;
        if (d >= HD) break;
        u32x4 c = *reinterpret_cast<const u32x4*>(&turned[d * kBlock]);
        if (old > 0 || end < kBlock) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t moved = ratio != 1.f ? move_codes(held[j][i], ratio) : held[j][i];
            uint32_t r = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int at = 4 * i + e;
              r |= (at < old ? moved : at < end ? c[i] : held[j][i]) & (0xffu << (8 * e));
            }
            c[i] = r;
          }
        }
        *reinterpret_cast<u32x4*>(codes + d * kBlock) = c;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if (lane == 0) *scale = s;
  }
}

// One wave: one block of 16 tokens of one head's keys, values or queries, four lanes a token.  A block has one wave for its scale, so nothing is shared between
// waves, and where older tokens share it with the new rows the same wave moves them.  What bounds small calls is one load after another, and large ones half the
// instructions and half the bytes: what does not depend on the rows is asked for beside them, and keys, values and queries, which need different registers, have a
// path each (in one path 188 registers for heads of 128, 161 in three).  64 sequences, one row each, 32 and 8 heads of 128: 7.1 us; 8192 rows of 16 and 16 heads of 64, 86 MB, 23 us
// (3.7 TB/s); 65536 rows of 32 and 8 heads of 128, 1.5 GB, 375 us (3.9 TB/s).  Several heads a wave, which share their angles, were no faster.
template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_append(AppendArgs g) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[4][HD * kBlock];   // a block's values on the way to their order
  const int wave = threadIdx.x / kWave, kv = g.cache.heads, task = __builtin_amdgcn_readfirstlane(blockIdx.y * 4 + wave);
  if (task < kv)
    append_head<T, HD, KEYS>(g, task, nullptr);
  else if (task < 2 * kv)
    append_head<T, HD, VALUES>(g, task - kv, turned[wave]);
  else if (task - 2 * kv < g.heads)
    append_head<T, HD, QUERIES>(g, task - 2 * kv, nullptr);
}

// ---- attention ---------------------------------------------------------------------------------------------------------

// bf16 terms of a query's number and of a probability (times its value's scale).  bf16 rows are one term.  The probabilities keep 16 bits in two, or the output would be off by
// half as much again as its own rounding to bf16 has it (of 64 bits 0.0020 to 0.0024, and now 0.0017); HBM bounds this kernel, and the second term costs 1 to 4 % (64 sequences 128 and
// 131 us, one row over 64k tokens 57 and 57).  fp32: three terms, which sum to the number.
template <typename T> struct Terms;
template <> struct Terms<bf16_t> { static constexpr int kQuery = 1, kProb = 2; };
template <> struct Terms<float> { static constexpr int kQuery = 3, kProb = 3; };

__device__ __forceinline__ void to_terms(const float (&v)[8], bf16x8 (&f)[1]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[0][i] = f2bf(v[i]);
}
__device__ __forceinline__ void to_terms(const float (&v)[8], bf16x8 (&f)[2]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[0][i] = f2bf(v[i]);
    f[1][i] = f2bf(v[i] - bf2f(f[0][i]));
  }
}
__device__ __forceinline__ void to_terms(const float (&v)[8], bf16x8 (&f)[3]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const Bf16Terms b = split_bf16(v[i]);
    f[0][i] = b.hi; f[1][i] = b.mid; f[2][i] = b.lo;
  }
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) { load_vec(p, v); }
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}

// One block: 16 query rows over one run of keys, in steps of 64 that its four waves take in turn.  S^T = K Q^T and O^T = V^T P^T, both by
// v_mfma_f32_16x16x32_bf16 with a query row to a column, so a lane holds probabilities of one row and the running maximum and sum are
// per-lane scalars.  Row a of key tile j is token 16 (a / 4) + 4 j + a mod 4 of the step: quarter g of the wave then holds the scores of
// block g, with that block's two scales in one register each, and the probabilities of its 16 tokens in the order in which the cache
// holds their values.  No code passes through LDS.  What bounds it is HBM: a step's values are on their way while its scores are computed, the next step's
// keys while its values are multiplied, and page numbers are read two steps ahead.
// One row over 65536 tokens, 16 heads of 128, 268 MB: 49 us (5.5 TB/s) and 5 for the join; 64 rows over up to 8190 tokens each, 32 heads on 8 of 128: 121 us and 5.  Small calls
// are latency: lengths, page numbers, scales and keys come one after another, and the join is a launch more (33 tokens 5.5 us, eight times 5 rows over 2049 tokens 10.9).
template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_attention(CacheAttnArgs g) {
  constexpr int NT = Terms<T>::kQuery, NP = Terms<T>::kProb, W16 = HD / 64, REST = HD % 64 / 32, DT = HD / 16;
  constexpr int FR = HD / 32;                          // fragments of 32 of a row
  constexpr int LD = HD + 4;                           // floats a row of sums in LDS: rows begin four banks apart
  extern __shared__ float joined[];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c16 = lane % 16, quarter = lane / 16;
  const int kv = g.cache.heads, kvh = blockIdx.y % kv, tiles = gridDim.y / kv, group = g.group.d, blocks = g.blocks.d;
  const Sight sq(g, blockIdx.z);
  const int32_t* table = g.rows.page_table + blockIdx.z * g.rows.ld_page_table;
  const uint8_t* kbase = (const uint8_t*)g.cache.k + (int64_t)kvh * g.cache.page * HD + (c16 % 4) * HD + quarter * 16;
  const uint8_t* vbase = (const uint8_t*)g.cache.v + (int64_t)kvh * g.cache.page * HD + c16 * kBlock;

  for (int tile = blockIdx.y / kv; tile * 16 < sq.all; tile += tiles) {
    int seen = sq.held, fewest = sq.held;               // the most and the fewest of the tile's rows
    if (g.causal) {
      const int last = sq.first + quotient(tile * 16 + 15 < sq.all ? tile * 16 + 15 : sq.all - 1, g.group) + 1;
      if (last < sq.held) seen = last;
      fewest = sq.first + quotient(tile * 16, g.group) + 1;
    }
    if (seen < 0) seen = 0;
    const int len = run_length(seen, g.splits, g.least), k_lo = (int)blockIdx.x * len < seen ? blockIdx.x * len : seen;
    const int k_hi = seen - k_lo < len ? seen : k_lo + len;

    // page numbers of the step at key k0 (-1 behind the run's end), and where its codes lie
    auto number = [&](int k0, int block) {
      const int b = k0 / kBlock + block;
      return b * kBlock < k_hi ? table[quotient(b, g.blocks)] : -1;
    };
    auto offset = [&](int k0, int block, int page, int64_t stride, int in_block) {
      const int b = k0 / kBlock + block, in_page = b - quotient(b, g.blocks) * blocks;
      return page >= 0 && page < g.cache.pages ? page * stride + in_page * in_block : (int64_t)-1;
    };
    u32x4 kw[4][W16 + 1];
    u32x2 kr[4];
    auto load_keys = [&](int64_t at) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint8_t* kc = kbase + at + j * 4 * HD;
#pragma unroll
        for (int i = 0; i < W16; ++i) kw[j][i] = at >= 0 ? *reinterpret_cast<const u32x4*>(kc + i * 64) : u32x4{0, 0, 0, 0};
        kr[j] = REST && at >= 0 ? *reinterpret_cast<const u32x2*>(kc + W16 * 64 - quarter * 8) : u32x2{0, 0};
      }
    };

    int k0 = k_lo + wave * 64;
    int kp = number(k0, c16 / 4), vp = number(k0, quarter), kp2 = number(k0 + 256, c16 / 4), vp2 = number(k0 + 256, quarter);
    const int r = tile * 16 + c16, rr = r < sq.all ? r : sq.all - 1, rq = quotient(rr, g.group);
    const int sees = r >= sq.all ? 0 : g.causal ? sq.first + rq + 1 : sq.held;       // a row sees the keys before this one
    bf16x8 qf[FR][NT];
#pragma unroll
    for (int f = 0; f < FR; ++f) {
      const int d = f < 2 * W16 ? f / 2 * 64 + quarter * 16 + f % 2 * 8 : W16 * 64 + quarter * 8;
      float v[8];
      load8((const T*)g.q + (sq.begin + rq) * g.ldq + (int64_t)(kvh * group + rr - rq * group) * HD + d, v);
      to_terms(v, qf[f]);
    }
    load_keys(offset(k0, c16 / 4, kp, g.cache.stride_page, kBlock * HD));
    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    for (; k0 < k_hi; k0 += 256) {
      const int64_t va = offset(k0, quarter, vp, g.cache.stride_page, kBlock * HD);
      const int64_t sa = offset(k0, quarter, vp, g.cache.stride_scale, 1);
      u32x4 vw[DT];
#pragma unroll
      for (int d = 0; d < DT; ++d) vw[d] = va >= 0 ? *reinterpret_cast<const u32x4*>(vbase + va + d * 16 * kBlock) : u32x4{0, 0, 0, 0};
      const float ks = sa >= 0 ? g.cache.k_scale[sa + kvh * blocks] * g.scale : 0.f, vs = sa >= 0 ? g.cache.v_scale[sa + kvh * blocks] : 0.f;
      const int kp3 = number(k0 + 512, c16 / 4), vp3 = number(k0 + 512, quarter);

      f32x4 s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < FR; ++f) {
          const bf16x8 kf = f < 2 * W16 ? codes_bf16(kw[j][f / 2][f % 2 * 2], kw[j][f / 2][f % 2 * 2 + 1]) : codes_bf16(kr[j][0], kr[j][1]);
#pragma unroll
          for (int u = NT - 1; u >= 0; --u) s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[f][u], s[j], 0, 0, 0);
        }
      }
      load_keys(offset(k0 + 256, c16 / 4, kp2, g.cache.stride_page, kBlock * HD));
      kp = kp2; vp = vp2; kp2 = kp3; vp2 = vp3;

      const int vb = (k0 / kBlock + quarter) * kBlock;
      const int left = (va >= 0 ? sees : 0) - vb;        // of this lane's block, the tokens its row sees
      float big = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[j][i] = 4 * j + i < left ? s[j][i] * ks : -INFINITY;
          big = fmaxf(big, s[j][i]);
        }
      big = fmaxf(big, __shfl_xor(big, 16, 64));
      big = fmaxf(big, __shfl_xor(big, 32, 64));
      const float m_new = fmaxf(m, big), ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      m = m_new;
      float p[16], sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = __builtin_amdgcn_exp2f(s[e / 4][e % 4] - ref);
        sum += p[e];
      }
      l = fmaf(l, alpha, sum);
      bf16x8 pf[2][NP];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float pv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) pv[e] = p[8 * u + e] * vs;
        to_terms(pv, pf[u]);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= alpha;
      bool poisoned = false;                                         // whether a code that not every row sees is NaN
      if (k0 + 64 > fewest) {
        uint32_t any = 0;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) any |= (vw[d][i] & 0x7f7f7f7fu) + 0x01010101u;     // bit 7 of a byte: it is NaN
        poisoned = __any((any & 0x80808080u) != 0);
      }
      if (!poisoned) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const bf16x8 vf = codes_bf16(vw[d][2 * u], vw[d][2 * u + 1]);
#pragma unroll
            for (int x = NP - 1; x >= 0; --x) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u][x], o[d], 0, 0, 0);
          }
      } else {
        // A NaN times a probability of 0 is NaN, so NaN values are counted apart, among the tokens that a row sees.  (Tokens past the last may hold
        // anything.)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          f32x4 count = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t n0 = nan_bytes(vw[d][2 * u]), n1 = nan_bytes(vw[d][2 * u + 1]);
            const bf16x8 vf = codes_bf16(vw[d][2 * u] & ~n0, vw[d][2 * u + 1] & ~n1);
            const bf16x8 nf = codes_bf16(n0 & 0x38383838u, n1 & 0x38383838u);      // 0x38 is 1
            bf16x8 seen_f;
#pragma unroll
            for (int e = 0; e < 8; ++e) seen_f[e] = 8 * u + e < left ? (bf16_t)1.0f : (bf16_t)0.0f;
#pragma unroll
            for (int x = NP - 1; x >= 0; --x) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u][x], o[d], 0, 0, 0);
            count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(nf, seen_f, count, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (count[i] > 0.f) o[d][i] = __builtin_nanf("");
        }
      }
    }

    // join the four waves
    float* const ml = joined + 4 * 16 * LD;                 // [4][16][2], then each wave's factor of a row [16][4]
    float* const factor = ml + 4 * 16 * 2;
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(&joined[(wave * 16 + c16) * LD + d * 16 + quarter * 4]) = o[d];
    if (quarter == 0) { ml[(wave * 16 + c16) * 2] = m; ml[(wave * 16 + c16) * 2 + 1] = l; }
    __syncthreads();
    const int rows_left = sq.all - tile * 16;
    if (threadIdx.x < 16 && (int)threadIdx.x < rows_left) {
      const int rt = threadIdx.x;
      float top = ml[rt * 2];
#pragma unroll
      for (int u = 1; u < 4; ++u) top = fmaxf(top, ml[(u * 16 + rt) * 2]);
      const float ref = top == -INFINITY ? 0.f : top;
      float total = 0.f, f[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        f[u] = __builtin_amdgcn_exp2f(ml[(u * 16 + rt) * 2] - ref);
        total = fmaf(f[u], ml[(u * 16 + rt) * 2 + 1], total);
      }
      const float inv = g.splits > 1 ? 1.f : total == 0.f ? 0.f : 1.0f / total;
#pragma unroll
      for (int u = 0; u < 4; ++u) factor[rt * 4 + u] = f[u] * inv;
      if (g.splits > 1) {
        const int oq = quotient(tile * 16 + rt, g.group);
        const int64_t at = (blockIdx.x * g.rows.rows + sq.begin + oq) * g.heads + kvh * group + tile * 16 + rt - oq * group;
        g.part_ml[at * 2] = top;
        g.part_ml[at * 2 + 1] = total;
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 4 * HD; e += 256) {
      const int rt = e / (HD / 4), d = e % (HD / 4) * 4, ro = tile * 16 + rt;
      if (rt >= rows_left) break;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(&joined[(u * 16 + rt) * LD + d]);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf(factor[rt * 4 + u], x[i], v[i]);
      }
      const int oq = quotient(ro, g.group), ohead = kvh * group + ro - oq * group;
      if (g.splits == 1) {
        store4((T*)g.out + (sq.begin + oq) * g.ldo + (int64_t)ohead * HD + d, v);
      } else {
        store4(g.part_o + ((blockIdx.x * g.rows.rows + sq.begin + oq) * g.heads + ohead) * HD + d, v);
      }
    }
    __syncthreads();
  }
}

// Joins the runs' parts.  A team of HD / 4 lanes takes every g.teams-th part of one (row, head), each lane four elements; the teams of an item, side
// by side in a block, then add theirs up in LDS.  Rows that belong to no sequence have no parts and are left alone.
template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_attention_join(CacheAttnArgs g) {
  constexpr int LANES = HD / 4, TEAMS = 256 / LANES;
  __shared__ float sums[TEAMS][HD + 2];
  const int team = threadIdx.x / LANES, lane = threadIdx.x % LANES, each = TEAMS / g.teams, mine = team / g.teams, nth = team % g.teams;
  const int64_t items = g.rows.rows * g.heads, item = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * each + mine, row = item / g.heads;
  const bool live = mine < each && item < items && row >= g.rows.row_begin[0] && row < g.rows.row_begin[g.rows.batch];
  float top = -INFINITY, total = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
  if (live) {
#pragma unroll 4
    for (int i = nth; i < g.splits; i += g.teams) {
      const int64_t at = i * items + item;
      const float mi = g.part_ml[at * 2], li = g.part_ml[at * 2 + 1];
      const f32x4 o = *reinterpret_cast<const f32x4*>(g.part_o + at * HD + lane * 4);
      const float next = fmaxf(top, mi), ref = next == -INFINITY ? 0.f : next;
      const float a = __builtin_amdgcn_exp2f(top - ref), f = __builtin_amdgcn_exp2f(mi - ref);
      top = next;
      total = fmaf(total, a, f * li);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(v[e], a, f * o[e]);
    }
    float* to = sums[team];
#pragma unroll
    for (int e = 0; e < 4; ++e) to[lane * 4 + e] = v[e];
    if (lane == 0) { to[HD] = top; to[HD + 1] = total; }
  }
  __syncthreads();
  if (!live || nth != 0) return;
  float ref = top;
  for (int i = 1; i < g.teams; ++i) ref = fmaxf(ref, sums[team + i][HD]);
  if (ref == -INFINITY) ref = 0.f;
  float sum = 0.f, w[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < g.teams; ++i) {
    const float f = __builtin_amdgcn_exp2f(sums[team + i][HD] - ref);
    sum = fmaf(f, sums[team + i][HD + 1], sum);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = fmaf(f, sums[team + i][lane * 4 + e], w[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = sum == 0.f ? 0.f : w[e] / sum;
  store4((T*)g.out + row * g.ldo + (item - row * g.heads) * HD + lane * 4, w);
}

// How a call is computed: rows in tiles of 16, or of 128 by the kernel for prompts; and runs of keys.
struct Shape { bool prompt; int tiles, splits; };

// Tiles of 128 read the keys once where tiles of 16 read them eight times, but take longer for each step of keys: they are taken where the call is large, by heads x rows
// x tokens (us, 16 and 128 rows a tile).  Heads of 128: eight times 256 rows of 32 heads on 8 over 8192 tokens (5 * 10^8) 752 and 302; eight times 300 rows of 32 heads on 8 over 900
// (7 * 10^7) 127 and 73; four times 64 rows of 16 heads over 4096 (1.7 * 10^7) 37 and 34; 512 rows of 32 heads on 8 over 512 (8 * 10^6) 19 and 24; 128 rows of 16 heads over 2048 (4 * 10^6)
// 18 and 22.  Heads of 64: 64 rows of 16 heads over 65536 (7 * 10^7) 77 and 59; 700 rows of 16 heads over 700 (8 * 10^6) 12 and 18.  32 rows a key head and fewer leave three quarters
// of a large tile empty: eight times 8 rows of 32 heads on 8 over 8192 tokens 41 and 47.
constexpr int kPromptRows = 32, kPromptWork = 1 << 24;
// Runs of keys: as many as fill the chip's places, two blocks of 256 threads a CU (64k tokens, 16 heads of 128: 57 us, with twice as many 61) or one of 512, and, of
// several sequences, none longer than kLongRun, so that sequences of all lengths, of which the host knows only the longest, keep the chip filled to the end (64
// sequences of up to 8190 tokens, 8 key heads of 128: 131 us, with runs of 1024 135, of 4096 138).  Where a sequence has more than 32 rows of a key head, which are the many rows of
// fp32, blocks are many as it is and parts large: then only up to two blocks a place (fp32, us, without this and with: two times 2048 rows of 16 heads of 128 over 8192 tokens 1549, behind
// 136 MB of parts, and 1217 with none; eight times 64 rows of 16 heads on 4 over 8192 210 and 191; four times 40 rows of 16 heads of 64 over 16384 77 and 80).
// A run has 256 keys at least, a step of each wave: one row over 2400 tokens, 16 heads of 64, 8.5 us, with 512 9.9.  Up to 640 keys stay one run, as the second kernel costs
// more than it saves: 300 tokens 6.3 us and, in two runs, 7.9, 600 tokens 7.9 and 8.4; 1200 tokens 10.9 and 8.5.
constexpr int kMostSplits = 128, kLeastRun = 256, kWholeRun = 640, kLongRun = 2048, kPlaces = 512, kPromptPlaces = 256;
Shape shape(int heads, const ac_kv_cache& c, const CacheRows& r, int dtype) {
  const int64_t rows_of = r.max_rows < r.rows ? r.max_rows : r.rows, rows = rows_of * (heads / c.heads);
  const int64_t all = rows_of < r.rows / (r.batch > 0 ? r.batch : 1) ? rows_of * r.batch : r.rows;
  Shape s;
  s.prompt = dtype == AC_BF16 && c.pages > 0 && rows > kPromptRows && all * heads * (double)r.max_length >= kPromptWork;
  const int each = s.prompt ? 128 : 16;
  s.tiles = rows < 1 ? 1 : (int)((rows + each - 1) / each);
  const int64_t blocks = (int64_t)s.tiles * c.heads * r.batch;
  int64_t n = blocks > 0 ? (s.prompt ? kPromptPlaces : kPlaces) / blocks : 1;
  if (!s.prompt && r.batch > 1) {
    int64_t runs = r.max_length / kLongRun;
    if (r.rows * (heads / c.heads) > kPromptRows * r.batch && runs > 2 * kPlaces / blocks) runs = 2 * kPlaces / blocks;
    if (n < runs) n = runs;
  }
  const int64_t most = !s.prompt && r.max_length <= kWholeRun ? 1 : (r.max_length + kLeastRun - 1) / kLeastRun;
  if (n > most) n = most;
  if (n > kMostSplits) n = kMostSplits;
  s.splits = n < 1 ? 1 : (int)n;
  return s;
}

template <typename T, int HD>
hipError_t attention_rows_launch(const CacheAttnArgs& a, int tiles, hipStream_t s) {
  const int most = 65535 / a.cache.heads;
  if (tiles > most) tiles = most;
  const dim3 grid((unsigned)a.splits, (unsigned)(tiles * a.cache.heads), (unsigned)a.rows.batch);
  constexpr size_t lds = (size_t)(4 * 16 * (HD + 4) + 4 * 16 * 2 + 16 * 4) * sizeof(float);
  static const hipError_t attr_status = hipFuncSetAttribute(reinterpret_cast<const void*>(cache_attention<T, HD>),
                                                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (attr_status != hipSuccess) return attr_status;
  hipLaunchKernelGGL((cache_attention<T, HD>), grid, dim3(256), lds, s, a);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t attention_launch(CacheAttnArgs a, const Shape& shape, hipStream_t s) {
  const hipError_t e = shape.prompt ? launch_cache_prefill(a, shape.tiles, s) : attention_rows_launch<T, HD>(a, shape.tiles, s);
  if (e != hipSuccess || a.splits == 1) return e;
  constexpr int TEAMS = 256 / (HD / 4);
  a.teams = a.splits / 4 < 1 ? 1 : a.splits / 4 > TEAMS ? TEAMS : a.splits / 4;
  const int64_t items = a.rows.rows * a.heads, each = TEAMS / a.teams;
  const int64_t blocks = (items + each - 1) / each, in_row = blocks < 1 << 20 ? blocks : 1 << 20;      // (a launch has less than 2^32 threads in a row)
  hipLaunchKernelGGL((cache_attention_join<T, HD>), dim3((unsigned)in_row, (unsigned)((blocks + in_row - 1) / in_row)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t attention_width(const CacheAttnArgs& a, const Shape& shape, hipStream_t s) {
  switch (a.cache.head_dim) {
    case 32: return attention_launch<T, 32>(a, shape, s);
    case 64: return attention_launch<T, 64>(a, shape, s);
    case 96: return attention_launch<T, 96>(a, shape, s);
    case 128: return attention_launch<T, 128>(a, shape, s);
    case 192: return attention_launch<T, 192>(a, shape, s);
    case 256: return attention_launch<T, 256>(a, shape, s);
    default: return hipErrorNotSupported;
  }
}

template <typename T, int HD>
hipError_t append_launch(const AppendArgs& a, hipStream_t s) {
  int64_t n = a.rows.max_rows < a.rows.rows ? a.rows.max_rows : a.rows.rows;
  if (n < 1) n = 1;
  int64_t blocks = (n + 14) / kBlock + 1;              // n tokens touch that many at most
  if (blocks > 1 << 20) blocks = 1 << 20;              // (and more in turn: a launch has less than 2^32 threads in a row)
  const int tasks = 2 * a.cache.heads + a.heads;
  const dim3 grid((unsigned)blocks, (unsigned)((tasks + 3) / 4), (unsigned)a.rows.batch);
  hipLaunchKernelGGL((cache_append<T, HD>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t append_width(const AppendArgs& a, hipStream_t s) {
  switch (a.cache.head_dim) {
    case 32: return append_launch<T, 32>(a, s);
    case 64: return append_launch<T, 64>(a, s);
    case 96: return append_launch<T, 96>(a, s);
    case 128: return append_launch<T, 128>(a, s);
    case 192: return append_launch<T, 192>(a, s);
    case 256: return append_launch<T, 256>(a, s);
    default: return hipErrorNotSupported;
  }
}

}  // namespace

hipError_t launch_cache_append(const void* q, int64_t ldq, void* q_out, int64_t ldqo, int heads, const void* k, int64_t ldk, const void* v,
                               int64_t ldv, const ac_kv_cache& cache, const CacheRows& rows, const ac_rotary* rotary, int dtype,
                               hipStream_t s) {
  if (rows.batch <= 0 || rows.rows <= 0) return hipSuccess;
  AppendArgs a{q, k, v, q_out, ldq, ldqo, ldk, ldv, q ? heads : 0, cache, rows, rotary ? *rotary : ac_rotary{}, divisor(cache.page / kBlock)};
  return dtype == AC_BF16 ? append_width<bf16_t>(a, s) : append_width<float>(a, s);
}

uint64_t cache_attention_workspace_bytes(int heads, const ac_kv_cache& cache, const CacheRows& rows, int causal, int dtype) {
  const int n = shape(heads, cache, rows, dtype).splits;
  return n == 1 ? 0 : (uint64_t)n * rows.rows * heads * (cache.head_dim + 2) * sizeof(float);
}

hipError_t launch_cache_attention(const void* q, int64_t ldq, void* out, int64_t ldo, int heads, const ac_kv_cache& cache,
                                  const CacheRows& rows, int causal, float scale, void* workspace, int dtype, hipStream_t s) {
  if (rows.batch <= 0 || rows.rows <= 0) return hipSuccess;
  const Shape sh = shape(heads, cache, rows, dtype);
  const int n = sh.splits;
  float* parts = (float*)workspace;
  CacheAttnArgs a{q, out, ldq, ldo, heads, cache, rows, causal, scale * kLog2e, divisor(heads / cache.heads), divisor(cache.page / kBlock),
                  n, kLeastRun, parts, n > 1 ? parts + (uint64_t)n * rows.rows * heads * cache.head_dim : nullptr, 1};
  return dtype == AC_BF16 ? attention_width<bf16_t>(a, sh, s) : attention_width<float>(a, sh, s);
}

}  // namespace ac
