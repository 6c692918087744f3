// A paged cache of keys and values in 8 bits: the append, which rotates and stores the rows of a step, and the attention that reads
// it.  Codes are e4m3 with one power-of-two scale for a block of 16 tokens of a head.
//
// Why a power of two: a block fills token by token, and where a later token asks for a larger scale the older codes move by whole
// exponents, exactly but for subnormal ones; with any other scale each move would round once more.  Why 16 tokens: the quarters of a
// wave then hold one block each, see the attention.
#include "common.h"

namespace ac {

namespace {

constexpr int kBlock = 16;
constexpr float kLog2e = 1.4426950408889634f;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Sequence { int64_t begin, rows, length; };   // its first row, its rows, its tokens with them

__device__ __forceinline__ Sequence sequence(const ac_cache_rows& r, int64_t b) {
  const int64_t lo = r.row_begin[b], hi = r.row_begin[b + 1];
  const int64_t from = lo < 0 ? 0 : lo, to = hi < r.rows ? hi : r.rows;
  return Sequence{from, to > from ? to - from : 0, r.length[b]};
}

// ---- append ----------------------------------------------------------------------------------------------------------

// The least power of two s >= 2^-100 with v <= 448 s, for 0 <= v < inf: 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_of(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  if (e < 27) e = 27;
  return __builtin_bit_cast(float, (uint32_t)e << 23);
}

// Four numbers as e4m3, to nearest, ties to even; what is not finite becomes NaN.
__device__ __forceinline__ uint32_t to_e4m3(const float (&v)[4]) {
  uint32_t r = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], r, true);
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
  return to_e4m3(v);
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
  ac_cache_rows rows;
  ac_rotary rot;
};

// A lane holds, of one of a block's 16 tokens (four lanes a token), HD / 32 chunks of four pairs: elements lo .. lo + 3 and hi .. hi + 3.
struct Chunk { int pair, lo, hi; };
__device__ __forceinline__ Chunk chunk(const ac_rotary& r, int i, int sub) {
  const int j = 4 * (sub + 4 * i);
  return r.interleaved || j >= r.pairs ? Chunk{j, 2 * j, 2 * j + 4} : Chunk{j, j, j + r.pairs};
}

// Turns a chunk of row `row`, which stands at place `place` of its sequence.
__device__ __forceinline__ void turn_chunk(const ac_rotary& r, const Chunk& c, int64_t row, int64_t place, float (&a)[4], float (&b)[4]) {
  if (c.pair >= r.pairs) return;
  float cs[4], sn[4];
  if (r.axes == 1 || !r.positions) {
    int64_t p = r.positions ? r.positions[row] : place;
    p = p < 0 ? 0 : p < r.table_rows ? p : r.table_rows - 1;
    load_vec(r.cos + p * r.ld_table + c.pair, cs);
    load_vec(r.sin + p * r.ld_table + c.pair, sn);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int axis = 0, end = r.section[0];
      while (axis + 1 < r.axes && c.pair + i >= end) end += r.section[++axis];
      int64_t p = r.positions[axis * r.ld_positions + row];
      p = p < 0 ? 0 : p < r.table_rows ? p : r.table_rows - 1;
      cs[i] = r.cos[p * r.ld_table + c.pair + i];
      sn[i] = r.sin[p * r.ld_table + c.pair + i];
    }
  }
  if (r.interleaved) {
    turn(a[0], a[1], cs[0], sn[0]); turn(a[2], a[3], cs[1], sn[1]);
    turn(b[0], b[1], cs[2], sn[2]); turn(b[2], b[3], cs[3], sn[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) turn(a[i], b[i], cs[i], sn[i]);
  }
}

// One wave takes one block of 16 tokens of one head: of the keys, the values or the queries.
template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_append(AppendArgs g) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[4][HD * kBlock];   // a block's values on the way to their order
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, sub = lane % 4, t = lane / 4;
  const int task = blockIdx.y * 4 + wave, kv = g.cache.heads;
  if (task >= 2 * kv + g.heads) return;
  const int64_t page = g.cache.page, b = blockIdx.z;
  const Sequence sq = sequence(g.rows, b);
  const int64_t first = sq.length - sq.rows;                          // tokens before the rows; what would stand before token 0 is dropped
  const int64_t from = first > 0 ? first : 0;
  constexpr int CH = HD / 32;
  for (int64_t blk = from / kBlock + blockIdx.x; blk * kBlock < sq.length; blk += gridDim.x) {
    const int64_t place = blk * kBlock + t, row = sq.begin + place - first;
    const bool fresh = place >= from && place < sq.length;
    if (task >= 2 * kv) {
      const int h = task - 2 * kv;
      if (!fresh) continue;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const Chunk c = chunk(g.rot, i, sub);
        float x[4], y[4];
        const T* src = (const T*)g.q + row * g.ldq + (int64_t)h * HD;
        T* dst = (T*)g.q_out + row * g.ldqo + (int64_t)h * HD;
        load4(src + c.lo, x);
        load4(src + c.hi, y);
        turn_chunk(g.rot, c, row, place, x, y);
        store4(dst + c.lo, x);
        store4(dst + c.hi, y);
      }
      continue;
    }
    const int64_t nth = blk * kBlock / page;
    const int64_t id = nth < g.rows.ld_page_table ? g.rows.page_table[b * g.rows.ld_page_table + nth] : -1;
    if (id < 0 || id >= g.cache.pages) continue;
    const bool keys = task < kv;
    const int h = keys ? task : task - kv;
    const int64_t blocks = page / kBlock, in_page = blk % blocks;
    // a block's codes, of keys and of values, are HD * 16 bytes side by side
    uint8_t* codes = (uint8_t*)(keys ? g.cache.k : g.cache.v) + id * g.cache.stride_page + (h * blocks + in_page) * (HD * kBlock);
    float* scale = (keys ? g.cache.k_scale : g.cache.v_scale) + id * g.cache.stride_scale + h * blocks + in_page;
    float x[CH][4], y[CH][4], largest = 0.f;
    if (fresh) {
      const T* src = (keys ? (const T*)g.k + row * g.ldk : (const T*)g.v + row * g.ldv) + (int64_t)h * HD;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        Chunk c = chunk(g.rot, i, sub);
        if (!keys) c = Chunk{c.pair, 2 * c.pair, 2 * c.pair + 4};
        load4(src + c.lo, x[i]);
        load4(src + c.hi, y[i]);
        if (keys) turn_chunk(g.rot, c, row, place, x[i], y[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = fabsf(x[i][e]), w = fabsf(y[i][e]);
          if (u < INFINITY) largest = fmaxf(largest, u);
          if (w < INFINITY) largest = fmaxf(largest, w);
        }
      }
    }
    float s = scale_of(wave_max(largest)), ratio = 1.f;
    const int old = from > blk * kBlock ? (int)(from - blk * kBlock) : 0, end = sq.length - blk * kBlock < kBlock ? (int)(sq.length - blk * kBlock) : kBlock;
    if (old > 0) {
      const float before = *scale;
      s = fmaxf(s, before);
      ratio = before / s;
    }
    const float inv = 1.0f / s;
    if (fresh) {
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[i][e] *= inv; y[i][e] *= inv; }
    }
    if (keys) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const Chunk c = chunk(g.rot, i, sub);
        uint32_t* lo = (uint32_t*)(codes + t * HD + c.lo);
        uint32_t* hi = (uint32_t*)(codes + t * HD + c.hi);
        if (fresh) {
          *lo = to_e4m3(x[i]);
          *hi = to_e4m3(y[i]);
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
          const uint32_t lo = to_e4m3(x[i]), hi = to_e4m3(y[i]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            turned[wave][(d + e) * kBlock + t] = (uint8_t)(lo >> (8 * e));
            turned[wave][(d + 4 + e) * kBlock + t] = (uint8_t)(hi >> (8 * e));
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      for (int d = lane; d < HD; d += kWave) {
        u32x4 c = *reinterpret_cast<const u32x4*>(&turned[wave][d * kBlock]);
        u32x4* dst = reinterpret_cast<u32x4*>(codes + d * kBlock);
        if (old > 0 || end < kBlock) {
          const u32x4 held = *dst;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t moved = ratio != 1.f ? move_codes(held[i], ratio) : held[i];
            uint32_t r = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int at = 4 * i + e;
              r |= (at < old ? moved : at < end ? c[i] : held[i]) & (0xffu << (8 * e));
            }
            c[i] = r;
          }
        }
        *dst = c;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if (lane == 0) *scale = s;
  }
}

// ---- attention ---------------------------------------------------------------------------------------------------------

template <typename T> struct Terms;
template <> struct Terms<bf16_t> { static constexpr int kN = 1; };
template <> struct Terms<float> { static constexpr int kN = 3; };

__device__ __forceinline__ void to_terms(const float (&v)[8], bf16x8 (&f)[1]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[0][i] = f2bf(v[i]);
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

// Eight e4m3 codes as bf16, which holds each exactly.
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t lo, uint32_t hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The bytes of a word that are NaN, as 0xff each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t m = (w & 0x7f7f7f7fu) + 0x01010101u;      // bit 7 of a byte: its low seven bits were all ones
  return (m >> 7 & 0x01010101u) * 0xffu;
}

struct CacheAttnArgs {
  const void* q; void* out;
  int64_t ldq, ldo;
  int heads, group;                 // query heads, of a key head
  ac_kv_cache cache;
  ac_cache_rows rows;
  int causal;
  float scale;                      // times log2 e
  int splits; int64_t least;        // runs of keys, and the fewest keys of one (a multiple of 64)
  float* part_o; float* part_ml;    // [splits][rows][heads][head_dim], [splits][rows][heads][2]
};

// The keys that one of `splits` blocks takes of `seen` keys: runs of the same length, whole steps of 64.
__device__ __forceinline__ int64_t run_length(int64_t seen, int splits, int64_t least) {
  const int64_t even = (seen + splits - 1) / splits, n = (even + 63) / 64 * 64;
  return n > least ? n : least;
}

// One block: 16 query rows (the rows of a sequence with the query heads of one key head, head fastest) over one run of keys, in
// steps of 64 that its four waves take in turn.  S^T = K Q^T and O^T = V^T P^T, both by v_mfma_f32_16x16x32_bf16 with a query row
// to a column, so a lane holds probabilities of one row and the running maximum and sum are per-lane scalars.  Row a of key tile j is token
// 16 (a / 4) + 4 j + a mod 4 of the step: quarter g of the wave then holds the scores of block g, with that block's two scales in one
// register each, and the probabilities of its 16 tokens in the order in which the cache holds their values.  No code passes through LDS.
template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_attention(CacheAttnArgs g) {
  constexpr int NT = Terms<T>::kN, W16 = HD / 64, REST = HD % 64 / 32, DT = HD / 16;
  constexpr int FR = HD / 32;                          // fragments of 32 of a row
  extern __shared__ float joined[];                    // [4][16][HD] and [4][16][2]
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c16 = lane % 16, quarter = lane / 16;
  const int64_t page = g.cache.page, blocks = page / kBlock, b = blockIdx.z;
  const int kvh = blockIdx.y % g.cache.heads;
  const Sequence sq = sequence(g.rows, b);
  const int64_t all = sq.rows * g.group, first = sq.length - sq.rows;
  const int64_t held = sq.length < g.rows.ld_page_table * page ? sq.length : g.rows.ld_page_table * page;
  const int32_t* table = g.rows.page_table + b * g.rows.ld_page_table;
  const uint8_t* kbase = (const uint8_t*)g.cache.k + (int64_t)kvh * page * HD;
  const uint8_t* vbase = (const uint8_t*)g.cache.v + (int64_t)kvh * page * HD;

  for (int64_t tile = blockIdx.y / g.cache.heads; tile * 16 < all; tile += gridDim.y / g.cache.heads) {
    const int64_t r = tile * 16 + c16, rr = r < all ? r : all - 1;
    const int64_t row = sq.begin + rr / g.group;
    const int head = kvh * g.group + (int)(rr % g.group);
    const int64_t sees = r >= all ? 0 : g.causal ? first + rr / g.group + 1 : held;           // keys before this one
    int64_t seen = held, fewest = held;                                                        // the most and the fewest of the tile's rows
    if (g.causal) {
      const int64_t last = tile * 16 + 15 < all ? tile * 16 + 15 : all - 1;
      if (first + last / g.group + 1 < held) seen = first + last / g.group + 1;
      fewest = first + tile * 16 / g.group + 1;
    }
    if (seen < 0) seen = 0;
    const int64_t len = run_length(seen, g.splits, g.least), k_lo = blockIdx.x * len, k_hi = k_lo + len < seen ? k_lo + len : seen;

    bf16x8 qf[FR][NT];
#pragma unroll
    for (int f = 0; f < FR; ++f) {
      const int d = f < 2 * W16 ? f / 2 * 64 + quarter * 16 + f % 2 * 8 : W16 * 64 + quarter * 8;
      float v[8];
      load8((const T*)g.q + row * g.ldq + (int64_t)head * HD + d, v);
      to_terms(v, qf[f]);
    }
    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    for (int64_t k0 = k_lo + wave * 64; k0 < k_hi; k0 += 256) {
      // a lane reads keys of block c16 / 4 of the step and the values of block `quarter`
      const int64_t kb = k0 / kBlock + c16 / 4, vb = k0 / kBlock + quarter;
      int64_t kp = -1, vp = -1;
      if (kb * kBlock < k_hi) kp = table[kb / blocks];
      if (vb * kBlock < k_hi) vp = table[vb / blocks];
      const bool have_k = kp >= 0 && kp < g.cache.pages, have_v = vp >= 0 && vp < g.cache.pages;
      const uint8_t* kc = kbase + kp * g.cache.stride_page + (kb % blocks * kBlock + c16 % 4) * HD;
      const uint8_t* vc = vbase + vp * g.cache.stride_page + (vb % blocks * HD + c16) * kBlock;
      float ks = 0.f, vs = 0.f;
      if (have_v) {
        const int64_t at = vp * g.cache.stride_scale + kvh * blocks + vb % blocks;
        ks = g.cache.k_scale[at] * g.scale;
        vs = g.cache.v_scale[at];
      }
      f32x4 s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 kw[W16 + 1];
#pragma unroll
        for (int i = 0; i < W16; ++i) kw[i] = have_k ? *reinterpret_cast<const u32x4*>(kc + j * 4 * HD + i * 64 + quarter * 16) : u32x4{0, 0, 0, 0};
        u32x2 kr = {0, 0};
        if (REST && have_k) kr = *reinterpret_cast<const u32x2*>(kc + j * 4 * HD + W16 * 64 + quarter * 8);
#pragma unroll
        for (int f = 0; f < FR; ++f) {
          const bf16x8 kf = f < 2 * W16 ? codes_bf16(kw[f / 2][f % 2 * 2], kw[f / 2][f % 2 * 2 + 1]) : codes_bf16(kr[0], kr[1]);
#pragma unroll
          for (int u = NT - 1; u >= 0; --u) s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[f][u], s[j], 0, 0, 0);
        }
      }
      u32x4 vw[DT];
#pragma unroll
      for (int d = 0; d < DT; ++d) vw[d] = have_v ? *reinterpret_cast<const u32x4*>(vc + d * 16 * kBlock) : u32x4{0, 0, 0, 0};

      const int64_t left = (have_v ? sees : 0) - vb * kBlock;      // of this lane's block, the tokens its row sees
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
      bf16x8 pf[2][NT];
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
        for (int d = 0; d < DT; ++d) {
          // tokens past the last that the tile's rows see may hold anything
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t n = seen - vb * kBlock - 4 * i;
            vw[d][i] = n >= 4 ? vw[d][i] : n <= 0 ? 0u : vw[d][i] & (0xffffffffu >> (8 * (4 - (int)n)));
            any |= nan_bytes(vw[d][i]);
          }
        }
        poisoned = __any(any != 0);
      }
      if (!poisoned) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const bf16x8 vf = codes_bf16(vw[d][2 * u], vw[d][2 * u + 1]);
#pragma unroll
            for (int t = NT - 1; t >= 0; --t) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u][t], o[d], 0, 0, 0);
          }
      } else {
        // A NaN times a probability of 0 is NaN, so NaN values are counted apart, among the tokens that a row sees.
        bf16x8 seen_f[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) seen_f[e / 8][e % 8] = e < left ? (bf16_t)1.0f : (bf16_t)0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          f32x4 count = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t n0 = nan_bytes(vw[d][2 * u]), n1 = nan_bytes(vw[d][2 * u + 1]);
            const bf16x8 vf = codes_bf16(vw[d][2 * u] & ~n0, vw[d][2 * u + 1] & ~n1);
            const bf16x8 nf = codes_bf16(n0 & 0x38383838u, n1 & 0x38383838u);      // 0x38 is 1
#pragma unroll
            for (int t = NT - 1; t >= 0; --t) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u][t], o[d], 0, 0, 0);
            count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(nf, seen_f[u], count, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (count[i] > 0.f) o[d][i] = __builtin_nanf("");
        }
      }
    }

    // join the four waves
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    float* ml = joined + 4 * 16 * HD;
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(&joined[(wave * 16 + c16) * HD + d * 16 + quarter * 4]) = o[d];
    if (quarter == 0) { ml[(wave * 16 + c16) * 2] = m; ml[(wave * 16 + c16) * 2 + 1] = l; }
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * HD; e += 256) {
      const int rt = e / HD, d = e % HD;
      const int64_t rq = tile * 16 + rt;
      if (rq >= all) continue;
      float top = ml[rt * 2];
#pragma unroll
      for (int u = 1; u < 4; ++u) top = fmaxf(top, ml[(u * 16 + rt) * 2]);
      const float ref = top == -INFINITY ? 0.f : top;
      float total = 0.f, v = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float f = __builtin_amdgcn_exp2f(ml[(u * 16 + rt) * 2] - ref);
        total = fmaf(f, ml[(u * 16 + rt) * 2 + 1], total);
        v = fmaf(f, joined[(u * 16 + rt) * HD + d], v);
      }
      const int64_t orow = sq.begin + rq / g.group;
      const int ohead = kvh * g.group + (int)(rq % g.group);
      if (g.splits == 1) {
        Elem<T>::st((T*)g.out + orow * g.ldo + (int64_t)ohead * HD + d, total == 0.f ? 0.f : v / total);
      } else {
        const int64_t at = (blockIdx.x * g.rows.rows + orow) * g.heads + ohead;
        g.part_o[at * HD + d] = v;
        if (d == 0) { g.part_ml[at * 2] = top; g.part_ml[at * 2 + 1] = total; }
      }
    }
    __syncthreads();
  }
}

int64_t row_tiles(const ac_cache_rows& r, int group) {
  int64_t n = r.max_rows < r.rows ? r.max_rows : r.rows;
  if (n < 1) n = 1;
  return (n * group + 15) / 16;
}

template <typename T, int HD>
hipError_t attention_launch(const CacheAttnArgs& a, hipStream_t s) {
  int64_t tiles = row_tiles(a.rows, a.group);
  const int64_t most = 65535 / a.cache.heads;
  if (tiles > most) tiles = most;
  const dim3 grid((unsigned)a.splits, (unsigned)(tiles * a.cache.heads), (unsigned)a.rows.batch);
  constexpr size_t lds = (size_t)(4 * 16 * HD + 4 * 16 * 2) * sizeof(float);
  static const hipError_t attr_status = hipFuncSetAttribute(reinterpret_cast<const void*>(cache_attention<T, HD>),
                                                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (attr_status != hipSuccess) return attr_status;
  hipLaunchKernelGGL((cache_attention<T, HD>), grid, dim3(256), lds, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t attention_width(const CacheAttnArgs& a, hipStream_t s) {
  switch (a.cache.head_dim) {
    case 32: return attention_launch<T, 32>(a, s);
    case 64: return attention_launch<T, 64>(a, s);
    case 96: return attention_launch<T, 96>(a, s);
    case 128: return attention_launch<T, 128>(a, s);
    case 192: return attention_launch<T, 192>(a, s);
    case 256: return attention_launch<T, 256>(a, s);
    default: return hipErrorNotSupported;
  }
}

template <typename T, int HD>
hipError_t append_launch(const AppendArgs& a, hipStream_t s) {
  int64_t n = a.rows.max_rows < a.rows.rows ? a.rows.max_rows : a.rows.rows;
  if (n < 1) n = 1;
  const int64_t blocks = (n + 14) / kBlock + 1;        // n tokens touch that many at most
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
                               int64_t ldv, const ac_kv_cache& cache, const ac_cache_rows& rows, const ac_rotary* rotary, int dtype,
                               hipStream_t s) {
  if (rows.batch <= 0 || rows.rows <= 0) return hipSuccess;
  AppendArgs a{q, k, v, q_out, ldq, ldqo, ldk, ldv, q ? heads : 0, cache, rows, rotary ? *rotary : ac_rotary{}};
  return dtype == AC_BF16 ? append_width<bf16_t>(a, s) : append_width<float>(a, s);
}

uint64_t cache_attention_workspace_bytes(int heads, const ac_kv_cache& cache, const ac_cache_rows& rows, int causal, int dtype) { return 0; }

hipError_t launch_cache_attention(const void* q, int64_t ldq, void* out, int64_t ldo, int heads, const ac_kv_cache& cache,
                                  const ac_cache_rows& rows, int causal, float scale, void* workspace, int dtype, hipStream_t s) {
  if (rows.batch <= 0 || rows.rows <= 0) return hipSuccess;
  CacheAttnArgs a{q, out, ldq, ldo, heads, heads / cache.heads, cache, rows, causal, scale * kLog2e, 1, 64, nullptr, nullptr};
  return dtype == AC_BF16 ? attention_width<bf16_t>(a, s) : attention_width<float>(a, s);
}

}  // namespace ac
