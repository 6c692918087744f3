// The attention over an 8-bit cache for many rows: a stretch of a prompt behind what is cached already.  The matrix cores bound it, so what
// matters is that they never wait: codes come to LDS by direct loads a tile ahead, and a wave has the scores of the next tile of keys under
// way while it exponentiates those of the present one.
//
// A block owns 128 rows (the rows of a sequence with the query heads of one key head, head fastest); its eight waves are four groups of 32
// rows times two halves of the keys, whose tiles of 64 alternate, so that two waves share a SIMD and 256 blocks fill the chip (wide heads: four waves,
// one a SIMD).  S^T = K Q^T and
// O^T = V^T P^T by v_mfma_f32_32x32x16_bf16 with a row to a column.  Row x of a tile of 32 keys is token 4 (x / 8) + x mod 4 of block
// (x / 4) mod 2: lane half h then holds the scores of block h of the tile, in the order in which the cache holds the values of its 16 tokens, and the
// probabilities are the second product's operand as they stand.  Scales are powers of two: the conversion from e4m3 to bf16 multiplies by
// them, and nothing is rounded.  Probabilities are: to bf16, one term, with their sum taken before it, which puts outputs 0.0023 (in 2-norm) from 64 bits where their own rounding
// has them at 0.0017.  With a second term, as where rows are few, half as many matrix instructions again: 2048 rows behind 14336 tokens 425 us for 281, heads of 64 254 for 196.
//
// 2048 rows behind 14336 tokens, 16 heads of 128: 280 us, 0.92 PFLOP/s, of 1.27 that a large library product reaches.  What is left is issued beside the matrix
// instructions: 32 exponentials, their scaling and packing, and as many conversions of codes for every 32 of them.  The matrix cores are busy 37 % of the time, the vector units 58 %.  Heads of 128 spill 15
// registers, 64 bytes a lane (of 96 two): half of the 16 MB that this call writes, 8 being the output.
#include "cache.h"

namespace ac {

namespace {

constexpr int kTile = 64;      // keys
constexpr int kRowsOfBlock = 128;

// Where piece p (16 bytes) of a key's row lies in LDS: eight lanes that read the same piece of eight keys (0..3 of two blocks) fall into eight
// different pieces modulo 128 bytes.
template <int HD> __device__ __forceinline__ int swizzle(int token, int block) {
  constexpr int P = HD / 16;
  return P % 8 == 0 ? (token & 3) | (block & 1) << 2 : P % 4 == 0 ? (token >> 1 & 1) | (block & 1) << 1 : block & 1;
}

__device__ __forceinline__ bf16x8 scaled_bf16(uint32_t lo, uint32_t hi, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Two waves of 256 registers share a SIMD where that is enough for the sums of a row, else one has it alone.
template <int HD> constexpr int sides() { return HD <= 128 ? 2 : 1; }
template <int HD> constexpr size_t lds_bytes() {
  constexpr size_t ring = (size_t)sides<HD>() * (4 * kTile * HD + 64) + (HD + 1) * sizeof(int), join = sides<HD>() == 2 ? (size_t)kRowsOfBlock * (HD + 2) * sizeof(float) : 0;
  return ring > join ? ring : join;
}

template <int HD>
__global__ void __launch_bounds__(256 * sides<HD>(), sides<HD>()) cache_prefill(CacheAttnArgs g) {
  constexpr int TILE = kTile * HD, BLOCK = kBlock * HD, CHUNKS = TILE / 1024;   // bytes of a tile's keys or values and of a block; KB of the former
  constexpr int C = HD / 32, DT = HD / 32, SIDES = sides<HD>();
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), l32 = lane % 32, half = lane / 32;
  const int rowset = wave % 4, side = SIDES == 2 ? wave / 4 : 0;    // which 32 rows, which half of the tiles
  const int kv = g.cache.heads, kvh = blockIdx.x % kv, split = blockIdx.x / kv, group = g.group.d, blocks = g.blocks.d;
  const Sight sq(g, blockIdx.z);
  // most keys first
  const int tiles = (sq.all + kRowsOfBlock - 1) / kRowsOfBlock;
  const int32_t* table = g.rows.page_table + blockIdx.z * g.rows.ld_page_table;
  const uint32_t n_pages = (uint32_t)min(g.cache.pages, (int64_t)0x7fffffff);
  const uint8_t* kbase = (const uint8_t*)g.cache.k + (int64_t)kvh * g.cache.page * HD;
  const uint8_t* vbase = (const uint8_t*)g.cache.v + (int64_t)kvh * g.cache.page * HD;
  uint8_t* const ring = smem + side * 4 * TILE;        // two tiles of keys, two of values
  float* const scales = reinterpret_cast<float*>(smem + SIDES * 4 * TILE) + side * 16;
  int* const nan_at = reinterpret_cast<int*>(smem + SIDES * (4 * TILE + 64));    // of each element the first token with a NaN value; [HD]: of all
  const int k_block = lane >> 2 & 1, k_token = 4 * (l32 >> 3) + (lane & 3);      // what row l32 of a tile of 32 keys is

  for (int nth = blockIdx.y; nth < tiles; nth += gridDim.y) {
    const int tile = tiles - 1 - nth, row0 = tile * kRowsOfBlock + rowset * 32;
    // keys that the block's rows see at most; that this wave's see at most and at least
    auto sees_of = [&](int r) { return g.causal ? min(max(sq.first + quotient(min(r, sq.all - 1), g.group) + 1, 0), sq.held) : sq.held; };
    const int seen = sees_of(tile * kRowsOfBlock + kRowsOfBlock - 1);
    const bool active = row0 < sq.all;
    const int wave_seen = active ? sees_of(row0 + 31) : 0, fewest = sees_of(row0);
    const int len = run_length(seen, g.splits, g.least), k_lo = min(split * len, seen), k_hi = min(k_lo + len, seen);
    const int steps = ((k_hi - k_lo + kTile - 1) / kTile + SIDES - 1) / SIDES;      // of a side
    const int r = row0 + l32, rr = min(r, sq.all - 1), rq = quotient(rr, g.group), head = kvh * group + rr - rq * group;
    const int sees = r < sq.all ? sees_of(r) : 0;
    auto key_of = [&](int step) { return k_lo + (SIDES * step + side) * kTile; };
    const int limit = min(wave_seen, k_hi);
    const int mine = limit > key_of(0) ? ((limit - k_lo + kTile - 1) / kTile - side + SIDES - 1) / SIDES : 0;    // steps with keys that this wave's rows see

    // Lane x keeps the books of block x mod 4 of a tile: its page's number (-1 behind the run's end), and from it where its codes and scales lie.  A
    // block that is not there is read from the first page, and its scores are masked.
    auto number = [&](int step) __attribute__((always_inline)) {
      const int b = key_of(step) / kBlock + (lane & 3);
      return b * kBlock < k_hi ? table[quotient(b, g.blocks)] : -1;
    };
    struct Place { int64_t codes, scale; int there; };     // bytes and floats from the key head's first; there: bit i, block i (the same for all lanes)
    auto place_of = [&](int step, int page) __attribute__((always_inline)) {
      const int b = key_of(step) / kBlock + (lane & 3), in_page = b - quotient(b, g.blocks) * blocks;
      const bool have = (uint32_t)page < n_pages;
      const int64_t p = have ? page : 0, i = have ? in_page : 0;
      return Place{p * g.cache.stride_page + i * BLOCK, p * g.cache.stride_scale + i, (int)(__ballot(have) & 15)};
    };
    // 1 KB a load, the four waves of a side in turn
    auto load = [&](const uint8_t* from, bool values, uint8_t* to, const Place& p) __attribute__((always_inline)) {
      const int lo = (int)(uint32_t)p.codes, hi = (int)(p.codes >> 32);
#pragma unroll
      for (int n = 0; n < (CHUNKS + 3) / 4; ++n) {
        const int chunk = n * 4 + rowset, at = chunk * 1024 + lane * 16;
        if (CHUNKS % 4 != 0 && chunk >= CHUNKS) break;
        const int in = at % BLOCK, token = in / HD, piece = in % HD / 16;
        const uint32_t place = values ? in : token * HD + (piece ^ swizzle<HD>(token, at / BLOCK)) * 16;
        uint32_t olo, ohi;
        if (BLOCK % 1024 == 0) {
          olo = __builtin_amdgcn_readlane(lo, chunk * 1024 / BLOCK);
          ohi = __builtin_amdgcn_readlane(hi, chunk * 1024 / BLOCK);
        } else {               // (a KB of two blocks, with heads of 32 and 96)
          olo = __shfl(lo, at / BLOCK, 64);
          ohi = __shfl(hi, at / BLOCK, 64);
        }
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + (int64_t)((uint64_t)ohi << 32 | olo) + place),
                                         (__attribute__((address_space(3))) void*)(to + chunk * 1024), 16, 0, 0);
      }
    };
    // The keys of tile step + 2 with their scales, the values of tile step + 1 with theirs: the scales, eight floats, to the place that this
    // step's parity names (lanes 0 to 3 the keys', 4 to 7 the values').
    auto load_tiles = [&](int step, const Place& keys, const Place& values) __attribute__((always_inline)) {
      load(kbase, false, ring + (step & 1) * TILE, keys);
      load(vbase, true, ring + (2 + (step + 1 & 1)) * TILE, values);
      if (rowset == 0 && lane < 8) {
        const float* from = lane < 4 ? g.cache.k_scale + keys.scale : g.cache.v_scale + values.scale;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + kvh * blocks),
                                         (__attribute__((address_space(3))) void*)(scales + (step & 1) * 8), 4, 0, 0);
      }
    };
    // This wave's loads have landed and its LDS reads are done, then every wave's.  In between, of the values of tile `step` if not every row of
    // the block sees all its keys: a NaN value times a probability of 0 is NaN, so each wave takes NaN values among those that it loaded as zeros and notes
    // the first token of each element that has one, for the end.
    const int first_seen = sees_of(tile * kRowsOfBlock);
    auto landed = [&]() __attribute__((always_inline)) {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(7 << 4);
    };
    auto all_waves = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    auto arrived = [&](int step, int there) __attribute__((always_inline)) {
      landed();
      if (key_of(step) < k_hi && (key_of(step) + kTile > first_seen || there != 15)) {
        for (int n = 0; n < (CHUNKS + 3) / 4; ++n) {
          const int at = (n * 4 + rowset) * 1024 + lane * 16;
          if (CHUNKS % 4 != 0 && at >= TILE) break;
          u32x4* const mine = reinterpret_cast<u32x4*>(ring + (2 + (step & 1)) * TILE + at);
          const u32x4 w = *mine, x = {nan_bytes(w[0]), nan_bytes(w[1]), nan_bytes(w[2]), nan_bytes(w[3])};
          if ((x[0] | x[1] | x[2] | x[3]) != 0) {
            *mine = w & ~x;
            const int word = x[0] ? 0 : x[1] ? 1 : x[2] ? 2 : 3;
            const int token = key_of(step) + at / BLOCK * kBlock + 4 * word + __builtin_ctz(x[0] ? x[0] : x[1] ? x[1] : x[2] ? x[2] : x[3]) / 8;
            if (there >> (at / BLOCK) & 1) {
              atomicMin(&nan_at[at % BLOCK / kBlock], token);
              atomicMin(&nan_at[HD], token);
            }
          }
        }
        landed();
      }
      all_waves();
    };

    bf16x8 qf[2 * C];
#pragma unroll
    for (int f = 0; f < 2 * C; ++f)
      qf[f] = *reinterpret_cast<const bf16x8*>((const bf16_t*)g.q + (sq.begin + rq) * g.ldq + (int64_t)head * HD + f / 2 * 32 + half * 16 + f % 2 * 8);

    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    for (int e = threadIdx.x; e <= HD; e += blockDim.x) nan_at[e] = 0x7fffffff;

    auto key_frag = [&](int step, int t, int c) __attribute__((always_inline)) {
      const uint8_t* at = ring + step % 2 * TILE + (2 * t + k_block) * BLOCK + k_token * HD;
      return *reinterpret_cast<const u32x4*>(at + ((2 * c + half) ^ swizzle<HD>(k_token, k_block)) * 16);
    };
    auto value_frag = [&](int step, int t, int d) __attribute__((always_inline)) {
      return *reinterpret_cast<const u32x4*>(ring + (2 + step % 2) * TILE + (2 * t + half) * BLOCK + (d * 32 + l32) * kBlock);
    };
    auto zero = [](f32x16& x) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.f;
    };
    // of tile t of 32 keys, the scales of this lane's blocks: of the tile whose keys (values) came with step `step`
    auto key_scale = [&](int step, int t) { return scales[(step & 1) * 8 + 2 * t + k_block]; };
    auto value_scale = [&](int step, int t, int there) {
      const float s = scales[(step & 1) * 8 + 4 + 2 * t + half];
      return there >> (2 * t + half) & 1 ? s : 1.f;
    };
    auto bounded = [&](int step, int there) { return key_of(step) + kTile > fewest || there != 15; };   // not every row sees every key
    auto mask = [&](f32x16 (&s)[2], int step, int there) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int n = (there >> (2 * t + half) & 1 ? sees : 0) - key_of(step) - (2 * t + half) * kBlock;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i >= n) s[t][i] = -INFINITY;
      }
    };
    // The exponents' reference follows the maximum only where that is 2^8 above it: probabilities and their sum stay far inside fp32 and bf16, and
    // the sums are rarely rescaled.
    auto new_max = [&](float mx) __attribute__((always_inline)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * g.scale;
      if (__any(mx > m + 8.f)) {
        const float next = fmaxf(m, mx), ref = next == -INFINITY ? 0.f : next;
        const float a = __builtin_amdgcn_exp2f(m - ref);
        m = next;
        l *= a;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= a;
      }
    };
    auto scores = [&](f32x16 (&s)[2], int step) __attribute__((always_inline)) {
      zero(s[0]);
      zero(s[1]);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float ks = key_scale(step, t);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const u32x4 w = key_frag(step, t, c);
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(scaled_bf16(w[0], w[1], ks), qf[2 * c], s[t], 0, 0, 0);
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(scaled_bf16(w[2], w[3], ks), qf[2 * c + 1], s[t], 0, 0, 0);
        }
      }
    };
    auto take_max = [&](const f32x16 (&s)[2]) __attribute__((always_inline)) {
      float mx = s[0][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[t][i]);
      new_max(mx);
    };

    // Probabilities of `cur` (tile `step`, whose maximum m holds), their products with the tile's values, and meanwhile the scores of the tile
    // after it into `next` (of what LDS holds, behind the last tile): 16-byte fragments in turn, two matrix instructions each and each with its share
    // of the exponentials.
    auto work = [&](f32x16 (&cur)[2], f32x16 (&next)[2], int step, int there) __attribute__((always_inline)) {
      constexpr int NQK = 2 * C, N = NQK + 2 * DT, PD = 2, LAST = NQK + DT;   // LAST: fragments before the second half's products
      const float vs[2] = {value_scale(step - 1, 0, there), value_scale(step - 1, 1, there)}, ks[2] = {key_scale(step - 1, 0), key_scale(step - 1, 1)};
      zero(next[0]);
      zero(next[1]);
      auto frag = [&](int j) __attribute__((always_inline)) {
        if (j < NQK) return key_frag(step + 1, j / C, j % C);
        return value_frag(step, (j - NQK) / DT, (j - NQK) % DT);
      };
      u32x4 fr[PD];
#pragma unroll
      for (int j = 0; j < PD; ++j) fr[j] = frag(j);
      bf16x8 pf[2][2];
      float sum = 0.f;
      int done = 0;
      const float m_exp = m == -INFINITY ? 0.f : m;
      auto exponential = [&](int e) __attribute__((always_inline)) {
        const float p = __builtin_amdgcn_exp2f(fmaf(cur[e / 16][e % 16], g.scale, -m_exp));
        sum += p;
        pf[e / 16][e % 16 / 8][e % 8] = f2bf(p);
      };
      auto converted = [&](int h) __attribute__((always_inline)) {      // instruction h's codes, of fragment h / 2
        const int j = h / 2;
        const u32x4& w = fr[j % PD];
        return scaled_bf16(w[h % 2 * 2], w[h % 2 * 2 + 1], j < NQK ? ks[j / C] : vs[(j - NQK) / DT]);
      };
      bf16x8 a = converted(0);
#pragma unroll
      for (int h = 0; h < 2 * N; ++h) {
        const int j = h / 2, t = j < NQK ? j / C : (j - NQK) / DT, c = j < NQK ? j % C : (j - NQK) % DT;
        if (j < NQK) next[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[2 * c + h % 2], next[t], 0, 0, 0);
        else o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pf[t][h % 2], o[c], 0, 0, 0);
        if (h + 1 < 2 * N) a = converted(h + 1);
        if (h % 2 == 0 && j + PD < N) fr[j % PD] = frag(j + PD);
        // the first half's exponentials are done before the next tile's second half needs registers, the second's before its products
        const int due = h < 2 * C ? (h + 1) * 16 / (2 * C) : h < 2 * LAST ? 16 + (h + 1 - 2 * C) * 16 / (2 * (LAST - C)) : 32;
#pragma unroll
        for (int x = 0; x < (7 + C) / C; ++x)
          if (done < due) exponential(done++);
        __builtin_amdgcn_sched_barrier(0);
      }
      l += sum;
    };

    f32x16 s_a[2], s_b[2];
    // (the places of the first two tiles: as if the steps -2 and -1 had brought in the keys of tiles 0 and 1 and the values of tile 0)
    Place now = place_of(0, number(0)), next = place_of(1, number(1));
    int coming = number(2);
    load_tiles(-2, now, now);
    landed();
    all_waves();
    if (mine > 0) {
      scores(s_a, 0);
      if (bounded(0, now.there)) mask(s_a, 0, now.there);
      take_max(s_a);
    }
    load_tiles(-1, next, now);
    arrived(0, now.there);
    // Values of tile `step` and keys of step + 1 are in LDS, their other places free.
    auto iteration = [&](f32x16 (&cur)[2], f32x16 (&nxt)[2], int step) __attribute__((always_inline)) {
      const Place after = place_of(step + 2, coming);
      coming = number(step + 3);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      load_tiles(step, after, next);
      if (step < mine) {
        work(cur, nxt, step, now.there);
        if (step + 1 < mine) {
          if (bounded(step + 1, next.there)) mask(nxt, step + 1, next.there);
          take_max(nxt);
        }
      }
      arrived(step + 1, next.there);
      now.there = next.there;
      next = after;
    };
    for (int step = 0; step < steps; step += 2) {
      iteration(s_a, s_b, step);
      if (step + 1 < steps) iteration(s_b, s_a, step + 1);
    }

    // elements whose row sees a NaN value that was taken as zero
    if (nan_at[HD] != 0x7fffffff) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (nan_at[d * 32 + 8 * (i / 4) + 4 * half + i % 4] < sees) o[d][i] = __builtin_nanf("");
    }

    // the second half of the keys to LDS (pieces of four elements turned by the row, against bank conflicts), the first joins
    l += __shfl_xor(l, 32, 64);
    float* const joined = reinterpret_cast<float*>(smem);
    float* const ml = joined + kRowsOfBlock * HD;
    const int at = rowset * 32 + l32;
    auto place = [&](int d, int i) { return at * HD + d * 32 + ((8 * i + 4 * half + 4 * l32) & 31); };
    if (SIDES == 2) {
      __syncthreads();
      if (side == 1) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4*>(&joined[place(d, i)]) = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
        if (half == 0) { ml[2 * at] = m; ml[2 * at + 1] = l; }
      }
      __syncthreads();
    }
    if (side == 0 && r < sq.all) {
      const float m_other = SIDES == 2 ? ml[2 * at] : -INFINITY, l_other = SIDES == 2 ? ml[2 * at + 1] : 0.f;
      const float top = fmaxf(m, m_other), ref = top == -INFINITY ? 0.f : top;
      const float a = __builtin_amdgcn_exp2f(m - ref), b = __builtin_amdgcn_exp2f(m_other - ref);
      const float total = fmaf(a, l, b * l_other), inv = 1.0f / total;
      const int64_t part = ((int64_t)split * g.rows.rows + sq.begin + rq) * g.heads + head;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = d * 32 + 8 * i + 4 * half;
          f32x4 x = {0.f, 0.f, 0.f, 0.f}, y;
          if (SIDES == 2) x = *reinterpret_cast<const f32x4*>(&joined[place(d, i)]);
#pragma unroll
          for (int n = 0; n < 4; ++n) y[n] = fmaf(a, o[d][4 * i + n], b * x[n]);
          if (g.splits == 1) {
            bf16x4 w;
#pragma unroll
            for (int n = 0; n < 4; ++n) w[n] = f2bf(total == 0.f ? 0.f : y[n] * inv);
            *reinterpret_cast<bf16x4*>((bf16_t*)g.out + (sq.begin + rq) * g.ldo + (int64_t)head * HD + e) = w;
          } else {
            *reinterpret_cast<f32x4*>(g.part_o + part * HD + e) = y;
          }
        }
      if (g.splits > 1 && half == 0) { g.part_ml[part * 2] = top; g.part_ml[part * 2 + 1] = total; }
    }
    __syncthreads();
  }
}

template <int HD>
hipError_t prefill_launch(const CacheAttnArgs& a, int64_t tiles, hipStream_t s) {
  constexpr size_t lds = lds_bytes<HD>();
  static const hipError_t attr_status = hipFuncSetAttribute(reinterpret_cast<const void*>(cache_prefill<HD>),
                                                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (attr_status != hipSuccess) return attr_status;
  const dim3 grid((unsigned)(a.splits * a.cache.heads), (unsigned)(tiles < 65535 ? tiles : 65535), (unsigned)a.rows.batch);
  hipLaunchKernelGGL((cache_prefill<HD>), grid, dim3(256 * sides<HD>()), lds, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_prefill(const CacheAttnArgs& a, int64_t tiles, hipStream_t s) {
  switch (a.cache.head_dim) {
    case 32: return prefill_launch<32>(a, tiles, s);
    case 64: return prefill_launch<64>(a, tiles, s);
    case 96: return prefill_launch<96>(a, tiles, s);
    case 128: return prefill_launch<128>(a, tiles, s);
    case 192: return prefill_launch<192>(a, tiles, s);
    case 256: return prefill_launch<256>(a, tiles, s);
    default: return hipErrorNotSupported;
  }
}

}  // namespace ac
