// What the kernels of the 8-bit cache share.
#pragma once

#include "common.h"

namespace ac {

constexpr int kBlock = 16;
constexpr float kLog2e = 1.4426950408889634f;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Sequence { int64_t begin, rows, length; };   // its first row, its rows, its tokens with them

__device__ __forceinline__ Sequence sequence(const CacheRows& r, int64_t b) {
  const int64_t lo = r.row_begin[b], hi = r.row_begin[b + 1];
  const int64_t from = lo < 0 ? 0 : lo, to = hi < r.rows ? hi : r.rows, n = r.length[b];
  return Sequence{from, to > from ? to - from : 0, n > 0 ? n : 0};
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
  int heads;
  ac_kv_cache cache;
  CacheRows rows;
  int causal;
  int window, sinks;                // of a windowed call
  float scale;                      // times log2 e
  Divisor group, blocks;            // query heads of a key head, blocks of a page
  int splits, least;                // runs of keys, and the fewest keys of one (a multiple of 256)
  float* part_o; float* part_ml;    // [splits][rows][heads][head_dim], [splits][rows][heads][2]
  int teams;                        // that share the parts of one row and head
};

// The keys of one of `splits` runs over `seen` keys: runs of the same length, whole steps of a block's four waves.
__device__ __forceinline__ int run_length(int seen, int splits, int least) {
  const int even = (seen + splits - 1) / splits, n = (even + 255) / 256 * 256;
  return n > least ? n : least;
}

// What a sequence's rows see: the rows of a tile are (row of the sequence, query head of the key head), head fastest.
struct Sight {
  int begin, rows, first, held, all;     // first row, rows, token of row 0, tokens that have a place, rows times heads
  __device__ Sight(const CacheAttnArgs& g, int b) {
    const Sequence s = sequence(g.rows, b);
    const int64_t most = g.rows.ld_page_table * g.cache.page;
    // (the same for all lanes: scalar registers)
    begin = __builtin_amdgcn_readfirstlane((int)s.begin);
    rows = __builtin_amdgcn_readfirstlane((int)s.rows);
    first = __builtin_amdgcn_readfirstlane((int)(s.length - s.rows));
    held = __builtin_amdgcn_readfirstlane((int)(s.length < most ? s.length : most));
    all = rows * (int)g.group.d;
  }
};

// What the rows of a tile read of a windowed call: the sinks' blocks and those from the first row's window on, numbered one after another.  Runs and steps
// count these blocks (and 16 tokens for each); where windows reach the sinks nothing is left out, and they are the sequence's own.
struct Reach {
  int sinks, gap;                        // blocks with sinks, blocks left out behind them
  // seen: tokens up to the last row's place; first: the first row's place
  __device__ Reach(const CacheAttnArgs& g, int first, int seen) {
    const int low = min(first - g.window + 1, seen), begin = low > 0 ? low / kBlock : 0;
    sinks = (min(g.sinks, seen) + kBlock - 1) / kBlock;
    gap = begin > sinks ? begin - sinks : 0;
  }
  __device__ int block(int b) const { return b < sinks ? b : b + gap; }
};
// The first n of 16 tokens, as bits; and those of the block at token `at` that a row at `place` sees, of `seen` tokens that there are up to it.
__device__ __forceinline__ uint32_t first_of_16(int n) { return n <= 0 ? 0u : n >= 16 ? 0xffffu : (1u << n) - 1; }
__device__ __forceinline__ uint32_t seen_of_block(const CacheAttnArgs& g, int at, int place, int seen) {
  return first_of_16(seen - at) & (~first_of_16(place - g.window + 1 - at) | first_of_16(g.sinks - at));
}

// Rows in tiles of 128, for prompts: bf16, at least one page.
hipError_t launch_cache_prefill(const CacheAttnArgs& a, int64_t tiles, bool windowed, hipStream_t s);

}  // namespace ac
