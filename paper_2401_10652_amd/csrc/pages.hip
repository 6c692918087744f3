// The books of a paged cache: pages freed and taken, sequences that go on as others, pages moved to the front, and the copies that follow.
//
// Free pages are taken by number, the lowest first, and places that want one stand in the order of the table, so that what a call leaves does not depend on
// which thread came first: numbers of free pages and of wants are counted before them (prefix sums), and a want's rank finds the page of that rank.  uses is
// changed by integer atomics, whose order does not matter.  Pages are copied by one kernel, 16 bytes a lane.
//
// A call is bound by launches and by one memory latency after another, not by its bytes, so small books go through in one launch and middling updates in two.  us on the GPU, and in a row of calls from
// Python (which takes 3 to 4 us of the host a launch): an update of 16 sequences of 67 places 3.5 and 6.9 in one launch, 6.3 and 9.0 in two, 9.3 and 16 in four; 64 of 75 (4800 places, past
// what one block takes) 8.6 and 9.4 in two, 11.6 and 16.4 in four; 64 of 534 9.8 and 11.9; 1000 of 101 10.6 and 12.8; 250 of 2048 16.1 and 17.8; with 22706 pages two take 22 (whose second launch
// goes through uses alone) and four 16.3.  Forks of 128 sequences of 28 places 10.6 in two launches, 13.6 in five; compactions of 24 sequences 9.7 and 12.5.  One block for the ranks of wants
// and pages instead of two launches of many: 16.3 and 17.3 with 22706 pages, 11.9 and 13.6 with 1112.
#include "common.h"

namespace ac {

namespace {

constexpr int kChunk = 4096, kEach = kChunk / 256;      // pages that a block counts, and a thread of it
constexpr int kBlockTokens = 16;

struct PagesArgs {
  const int32_t* uses_from; const int32_t* table_from;
  int32_t* uses; int32_t* table;
  int pages, page, batch, chunks;
  int64_t places;
  const int32_t *drop_begin, *drop_end, *take_begin, *take_end;     // update
  const int32_t *parent, *length; int32_t* length_to;               // fork
  int32_t* count;                                                   // missing or used, or null
  int32_t *total, *need, *counts, *list, *source, *target, *tokens; // workspace: [0] pages of the list, [1] wants; need [batch]; counts [chunks]; the others [pages] or [batch]
  int32_t *drops, *dropped, *wanted;                                // workspace, of an update in two launches, else null: [batch] and, of each row, [places]: pages given up and places that want one
};

__device__ __forceinline__ bool names(const PagesArgs& g, int e) { return (uint32_t)e < (uint32_t)g.pages; }
__device__ __forceinline__ void add_use(const PagesArgs& g, int e, int n) {
  if (names(g, e)) __hip_atomic_fetch_add(g.uses + e, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Sum over the block's threads before this one; `sum`: over all of them.  n waves.
template <int WAVES>
__device__ __forceinline__ int sum_before(int v, int* of_wave, int& sum) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  if (lane == kWave - 1) of_wave[wave] = x;
  __syncthreads();
  int before = 0;
  sum = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    before += w < wave ? of_wave[w] : 0;
    sum += of_wave[w];
  }
  __syncthreads();
  return before + x - v;
}

// ---- rows of the table, a wave each ------------------------------------------------------------------------------------

constexpr int kAhead = 8;               // loads on their way (one by one 1024 rows of 1033 places take 7.2 us, so 6.1)
struct Range { int64_t from, to; };     // places
__device__ __forceinline__ Range places_in(const PagesArgs& g, const int32_t* begin, const int32_t* end, int b, bool whole) {
  if (!begin) return Range{0, 0};
  const uint32_t lo = (uint32_t)max(begin[b], 0), hi = (uint32_t)max(end[b], 0), page = (uint32_t)g.page;
  if (hi <= lo) return Range{0, 0};
  Range r = whole ? Range{(lo + page - 1) / page, hi / page} : Range{lo / page, (hi + page - 1) / page};
  if (r.to > g.places) r.to = g.places;
  return r;
}

// Frees what row b drops; the number of its places that want a page.  NOTED: uses stays as it is, and both are noted for the second launch.
template <bool NOTED>
__device__ __forceinline__ int update_row(const PagesArgs& g, int b, int lane) {
  const int32_t* from = g.table_from + b * g.places;
  int32_t* to = g.table + b * g.places;
  const Range drop = places_in(g, g.drop_begin, g.drop_end, b, true), take = places_in(g, g.take_begin, g.take_end, b, false);
  const bool apart = from != to;
  const int64_t end = apart ? g.places : drop.to;
  int wants = 0, drops = 0;
  const uint64_t lanes_before = (1ull << lane) - 1;
  for (int64_t i0 = apart ? 0 : drop.from; i0 < end; i0 += kAhead * kWave) {
    int was[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) was[a] = i0 + a * kWave + lane < end ? from[i0 + a * kWave + lane] : -1;
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int64_t i = i0 + a * kWave + lane;
      const int e = was[a];
      const bool gone = i < end && i >= drop.from && i < drop.to && names(g, e);
      if (NOTED) {
        const uint64_t which = __ballot(gone);
        if (gone) g.dropped[b * g.places + drops + __popcll(which & lanes_before)] = e;
        drops += __popcll(which);
      } else if (gone) {
        add_use(g, e, -1);
      }
      if (i < end && (apart || gone)) to[i] = gone ? -1 : e;
    }
  }
  // (in place a dropped entry may or may not be seen as it was: it wants a page either way)
  for (int64_t i0 = take.from; i0 < take.to; i0 += kWave) {
    const int64_t i = i0 + lane;
    const uint64_t which = __ballot(i < take.to && (!names(g, from[i]) || (i >= drop.from && i < drop.to)));
    if (NOTED && (which >> lane & 1)) g.wanted[b * g.places + wants + __popcll(which & lanes_before)] = (int)i;
    wants += __popcll(which);
  }
  if (NOTED && lane == 0) g.drops[b] = drops;
  return wants;
}

// Gives row b's places their pages, the first of them that of rank `rank`.
__device__ __forceinline__ void give_row(const PagesArgs& g, int b, int lane, int rank, int have) {
  const int32_t* from = g.table_from + b * g.places;
  int32_t* to = g.table + b * g.places;
  const Range drop = places_in(g, g.drop_begin, g.drop_end, b, true), take = places_in(g, g.take_begin, g.take_end, b, false);
  for (int64_t i0 = take.from; i0 < take.to; i0 += kWave) {
    const int64_t i = i0 + lane;
    const bool wants = i < take.to && (!names(g, from[i]) || (i >= drop.from && i < drop.to));
    const uint64_t all = __ballot(wants);
    const int mine = rank + __popcll(all & ((1ull << lane) - 1));
    if (wants) {
      const int e = mine < have ? g.list[mine] : -1;
      to[i] = e;
      if (e >= 0) g.uses[e] = 1;
    }
    rank += __popcll(all);
  }
}

// Row j goes on as its parent; whether it wants a page for a copy of the partly filled one.  (The first of a parent's rows is found among those before it, 64 at a time: 65535 rows take the last wave 1024
// loads, one after another.)
__device__ __forceinline__ int fork_row(const PagesArgs& g, int j, int lane) {
  const int p = g.parent[j];
  const bool none = (uint32_t)p >= (uint32_t)g.batch;
  bool first = true;
  if (!none) {
    for (int i = lane; __any(i < j) && first; i += kWave) first = !__any(i < j && g.parent[i] == p);
  }
  const int length = none ? 0 : max(g.length[p], 0), rest = length % g.page;
  const int64_t whole = length / g.page;
  const int32_t* old = g.table_from + j * g.places;
  const int32_t* from = g.table_from + (none ? 0 : p) * g.places;
  int32_t* to = g.table + j * g.places;
  for (int64_t i0 = 0; i0 < g.places; i0 += kAhead * kWave) {
    int was[kAhead], now[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int64_t i = i0 + a * kWave + lane;
      was[a] = i < g.places ? old[i] : -1;
      now[a] = i < g.places && !none && (i < whole || first) ? from[i] : -1;
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int64_t i = i0 + a * kWave + lane;
      if (now[a] != was[a]) {
        add_use(g, was[a], -1);
        add_use(g, now[a], 1);
      }
      if (i < g.places) to[i] = now[a];
    }
  }
  const int source = !none && !first && rest > 0 && whole < g.places ? from[whole] : -1;
  const bool wants = names(g, source);
  if (lane == 0) {
    g.length_to[j] = length;
    g.source[j] = source;
    g.tokens[j] = rest;
  }
  return wants;
}
__device__ __forceinline__ void give_copy(const PagesArgs& g, int j, int rank, int have) {
  const int source = g.source[j];
  int target = -1;
  if (names(g, source)) {
    if (rank < have) target = g.list[rank];
    const int32_t length = max(g.length[g.parent[j]], 0);
    g.table[j * g.places + length / g.page] = target;
    if (target >= 0) g.uses[target] = 1;
  }
  g.target[j] = target;
}

// ---- pages, a chunk a block ------------------------------------------------------------------------------------------------

// uses of the kEach pages from `first` on, as bits that are set for those in use; pages past the last are as in use in `there` alone.
struct Bits { uint32_t used, there; };
__device__ __forceinline__ Bits chunk_bits(const int32_t* uses, int pages, int first) {
  typedef int32_t any_i32x4 __attribute__((ext_vector_type(4), aligned(4)));
  Bits b{0, first >= pages ? 0u : pages - first >= kEach ? (1u << kEach) - 1 : (1u << (pages - first)) - 1};
  if (first + kEach <= pages) {
#pragma unroll
    for (int i = 0; i < kEach; i += 4) {
      const any_i32x4 u = *reinterpret_cast<const any_i32x4*>(uses + first + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) b.used |= u[e] > 0 ? 1u << (i + e) : 0u;
    }
  } else {
    for (int i = 0; first + i < pages; ++i) b.used |= uses[first + i] > 0 ? 1u << i : 0u;
  }
  return b;
}

__global__ void __launch_bounds__(256) pages_copy_uses(PagesArgs g) {
  for (int p = blockIdx.x * 256 + threadIdx.x; p < g.pages; p += gridDim.x * 256) g.uses[p] = g.uses_from[p];
}

template <bool FORK>
__global__ void __launch_bounds__(256) pages_rows(PagesArgs g) {
  const int lane = threadIdx.x % kWave, b = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
  if (!FORK && !g.take_begin && !g.dropped && b == 0 && lane == 0 && g.count) *g.count = 0;
  if (b >= g.batch) return;
  const int wants = FORK ? fork_row(g, b, lane) : g.dropped ? update_row<true>(g, b, lane) : update_row<false>(g, b, lane);
  if (lane == 0) g.need[b] = wants;
}

// Free pages of each chunk; the last block: the wants before each row.
__global__ void __launch_bounds__(256) pages_count(PagesArgs g) {
  __shared__ int of_wave[4];
  int sum;
  if ((int)blockIdx.x < g.chunks) {
    const Bits b = chunk_bits(g.uses, g.pages, blockIdx.x * kChunk + threadIdx.x * kEach);
    sum_before<4>(__popc(b.there & ~b.used), of_wave, sum);
    if (threadIdx.x == 0) g.counts[blockIdx.x] = sum;
    return;
  }
  int before = 0;
  for (int b0 = 0; b0 < g.batch; b0 += kChunk) {
    const int b = b0 + threadIdx.x * kEach;
    int v[kEach], mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine += v[i] = b + i < g.batch ? g.need[b + i] : 0;
    int at = before + sum_before<4>(mine, of_wave, sum);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (b + i < g.batch) g.need[b + i] = at;
      at += v[i];
    }
    before += sum;
  }
  if (threadIdx.x == 0) g.total[1] = before;
}

// Pages of the chunks before this block's, of `kind`; all: of all chunks.
__device__ __forceinline__ int chunks_before(const PagesArgs& g, int* of_wave, int& all) {
  int mine = 0, total = 0, sum;
  for (int c = threadIdx.x; c < g.chunks; c += 256) {
    const int n = g.counts[c];
    mine += c < (int)blockIdx.x ? n : 0;
    total += n;
  }
  sum_before<4>(total, of_wave, all);
  sum_before<4>(mine, of_wave, sum);
  return sum;
}

// The free pages' numbers, in order.
__global__ void __launch_bounds__(256) pages_list(PagesArgs g) {
  __shared__ int of_wave[4];
  int all, sum;
  const int before = chunks_before(g, of_wave, all), first = blockIdx.x * kChunk + threadIdx.x * kEach;
  const Bits b = chunk_bits(g.uses, g.pages, first);
  uint32_t free = b.there & ~b.used;
  int at = before + sum_before<4>(__popc(free), of_wave, sum);
  for (; free != 0; free &= free - 1) g.list[at++] = first + __builtin_ctz(free);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    g.total[0] = all;
    if (g.count) *g.count = g.total[1] > all ? g.total[1] - all : 0;
  }
}

// Both by one block, which stops looking for free pages when there are enough.  (Up to kRankPages: it goes through 16384 a microsecond and a half.)
constexpr int kRankThreads = 1024, kRankPages = 1 << 16;
__global__ void __launch_bounds__(kRankThreads) pages_rank(PagesArgs g) {
  __shared__ int of_wave[kRankThreads / kWave];
  const int tid = threadIdx.x;
  int sum, wants = 0, before = 0;
  Bits bits = chunk_bits(g.uses, g.pages, tid * kEach);            // (on their way while the wants are looked at)
  for (int b0 = 0; b0 < g.batch; b0 += kRankThreads) {
    const int b = b0 + tid, n = b < g.batch ? g.need[b] : 0, at = wants + sum_before<kRankThreads / kWave>(n, of_wave, sum);
    if (b < g.batch) g.need[b] = at;
    wants += sum;
  }
  for (int first = 0; first < g.pages && before < wants; first += kRankThreads * kEach) {
    if (first > 0) bits = chunk_bits(g.uses, g.pages, first + tid * kEach);
    uint32_t free = bits.there & ~bits.used;
    int at = before + sum_before<kRankThreads / kWave>(__popc(free), of_wave, sum);
    for (; free != 0; free &= free - 1) g.list[at++] = first + tid * kEach + __builtin_ctz(free);
    before += sum;
  }
  if (tid == 0) {
    g.total[0] = before;
    if (g.count) *g.count = wants > before ? wants - before : 0;
  }
}

template <bool FORK>
__global__ void __launch_bounds__(256) pages_give(PagesArgs g) {
  if (FORK) {
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j < g.batch) give_copy(g, j, g.need[j], *g.total);
  } else {
    const int b = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
    if (b < g.batch) give_row(g, b, threadIdx.x % kWave, g.need[b], *g.total);
  }
}

// ---- compaction ------------------------------------------------------------------------------------------------------------

// With n pages in use: a free page p < n is the target of rank p minus the pages in use before it, and a page p >= n in use the source whose rank is
// the number of pages in use behind it; both ranks run from 0 to the number of moves, which is the number of free pages among the first n.  list[p]: the rank of a source.
// at: pages in use before `first`.
__device__ __forceinline__ void moves_of(const Bits& bits, int first, int at, int n, const PagesArgs& g) {
  for (uint32_t there = bits.there; there != 0; there &= there - 1) {
    const int i = __builtin_ctz(there), p = first + i;
    const bool used = bits.used >> i & 1;
    if (!used && p < n) g.target[p - at] = p;
    if (used && p >= n) {
      g.source[n - 1 - at] = p;
      g.list[p] = n - 1 - at;
    }
    at += used;
    if (p == (n > 0 ? n - 1 : 0)) g.total[0] = n > 0 ? n - at : 0;
  }
}

// Pages in use of each chunk, and uses to where it goes.
__global__ void __launch_bounds__(256) compact_count(PagesArgs g) {
  __shared__ int of_wave[4];
  const int first = blockIdx.x * kChunk;
  int sum;
  sum_before<4>(__popc(chunk_bits(g.uses_from, g.pages, first + threadIdx.x * kEach).used), of_wave, sum);
  if (g.uses != g.uses_from)
    for (int p = first + threadIdx.x; p < g.pages && p < first + kChunk; p += 256) g.uses[p] = g.uses_from[p];
  if (threadIdx.x == 0 && (int)blockIdx.x < g.chunks) g.counts[blockIdx.x] = sum;      // (without pages there is one block, and no chunk)
}

__global__ void __launch_bounds__(256) compact_list(PagesArgs g) {
  __shared__ int of_wave[4];
  int n, sum;
  const int before = chunks_before(g, of_wave, n), first = blockIdx.x * kChunk + threadIdx.x * kEach;
  const Bits bits = chunk_bits(g.uses_from, g.pages, first);
  const int at = before + sum_before<4>(__popc(bits.used), of_wave, sum);
  moves_of(bits, first, at, n, g);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (g.pages == 0) g.total[0] = 0;
    g.total[1] = n;
    if (g.count) *g.count = n;
  }
}

// The table's entries and uses follow the pages.
__global__ void __launch_bounds__(256) compact_follow(PagesArgs g) {
  const int n = g.total[1], moves = g.total[0];
  const int64_t all = g.batch * g.places, first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  for (int64_t i = first; i < all; i += step) {
    const int was = g.table_from[i];
    int e = was;
    // (an entry that uses does not know of stays as it is: list has a rank for pages in use alone)
    if (names(g, e) && e >= n) {
      const int r = g.list[e];
      if ((uint32_t)r < (uint32_t)moves && g.source[r] == e) e = g.target[r];
    }
    if (g.table != g.table_from || e != was) g.table[i] = e;
  }
  for (int64_t i = first; i < moves; i += step) {
    const int from = g.source[i], to = g.target[i];
    g.uses[to] = g.uses_from[from];
    g.uses[from] = 0;
  }
}
// ---- an update in two launches ---------------------------------------------------------------------------------------------
//
// Behind the rows, which note what they drop and want: uses in LDS, from there the free pages, and each want finds its row among the wants before each row.
constexpr int kSecondThreads = 1024, kSecondWaves = kSecondThreads / kWave, kSecondPages = 8192, kSecondBatch = 1024, kSecondPlaces = 1 << 22;
__device__ __forceinline__ int row_of_rank(const int32_t* before, int batch, int r) {       // the last row with before[row] <= r
  int lo = 0;
  for (int step = kSecondBatch / 2; step > 0; step /= 2)
    if (lo + step < batch && before[lo + step] <= r) lo += step;
  return lo;
}
__global__ void __launch_bounds__(kSecondThreads) pages_second(PagesArgs g) {
  extern __shared__ __attribute__((aligned(16))) int32_t lds[];
  __shared__ int of_wave[kSecondWaves];
  const int tid = threadIdx.x, mine = tid < g.batch ? tid : -1;
  int32_t* const uses = lds;                                       // [pages], what it is at the end
  int32_t* const drops_before = uses + (g.pages + 3) / 4 * 4;      // [batch]
  int32_t* const wants_before = drops_before + g.batch;            // [batch]
  int32_t* const list = wants_before + g.batch;                    // [pages], free ones in order
  const int drops_mine = mine >= 0 ? g.drops[mine] : 0, wants_mine = mine >= 0 ? g.need[mine] : 0;
  for (int p = tid; p < g.pages; p += kSecondThreads) uses[p] = g.uses_from[p];
  int drops, wants, sum, before = 0;
  const int drops_at = sum_before<kSecondWaves>(drops_mine, of_wave, drops), wants_at = sum_before<kSecondWaves>(wants_mine, of_wave, wants);
  if (mine >= 0) { drops_before[mine] = drops_at; wants_before[mine] = wants_at; }
  __syncthreads();
  auto place_of = [&](int r) {
    const int b = row_of_rank(wants_before, g.batch, r);
    return b * g.places + g.wanted[b * g.places + r - wants_before[b]];
  };
  int64_t place = tid < wants ? place_of(tid) : 0;                 // (on its way while drops and free pages are looked at)
  for (int r = tid; r < drops; r += kSecondThreads) {
    const int b = row_of_rank(drops_before, g.batch, r);
    atomicAdd(&uses[g.dropped[b * g.places + r - drops_before[b]]], -1);
  }
  __syncthreads();
  for (int first = 0; first < g.pages && before < wants; first += kSecondThreads * kEach) {
    const Bits bits = chunk_bits(uses, g.pages, first + tid * kEach);
    uint32_t free = bits.there & ~bits.used;
    int at = before + sum_before<kSecondWaves>(__popc(free), of_wave, sum);
    for (; free != 0; free &= free - 1) list[at++] = first + tid * kEach + __builtin_ctz(free);
    before += sum;
  }
  if (tid == 0 && g.count) *g.count = wants > before ? wants - before : 0;
  __syncthreads();
  for (int r = tid; r < wants; r += kSecondThreads) {
    const int e = r < before ? list[r] : -1;
    g.table[place] = e;
    if (e >= 0) uses[e] = 1;
    if (r + kSecondThreads < wants) place = place_of(r + kSecondThreads);
  }
  __syncthreads();
  for (int p = tid; p < g.pages; p += kSecondThreads) g.uses[p] = uses[p];
}

// ---- all of it in one block -------------------------------------------------------------------------------------------------
//
// What the launches above do one after another, for tables of which each thread has a few entries: uses, lists and what is known of rows lie in LDS, and a barrier stands where a
// launch does.  What bounds it is one memory latency after another, and EACH, the entries of a thread: with one an update of 4 sequences of 67 places takes 2.8 us (3.9 with four), a fork of 4 of 28 with its
// copies 7.8 (9.0); with two 16 of 67 3.5 (4.4), 64 of 28 9.1 (10.0); with eight, for tables of 4800 places, updates take 9.8 and forks 15.0, in several launches 8.8 and 13.8.
constexpr int kOneThreads = 1024, kOneWaves = kOneThreads / kWave, kOnePages = 8192, kOneBatch = 1024, kOneEach = 4, kOnePlaces = kOneThreads * kOneEach;
enum { UPDATE, FORK_ROWS, COMPACT };

template <int KIND, int EACH>
__global__ void __launch_bounds__(kOneThreads) pages_at_once(PagesArgs g, Divisor of_row) {
  extern __shared__ __attribute__((aligned(16))) int32_t lds[];
  __shared__ int of_wave[kOneWaves];
  const int tid = threadIdx.x, places = (int)g.places, first_entry = tid * EACH, entries = (int)(g.batch * g.places);
  int32_t* const uses = lds;                                       // [pages], what it is at the end
  int32_t* const list = uses + (g.pages + 3) / 4 * 4;              // [pages]: free ones in order; of a compaction sources' ranks
  int32_t* const row = list + g.pages;                             // [4][batch]: of an update the ranges' ends, of a fork parent, whole pages and first; of a compaction targets [pages]
  const int mine = tid < g.batch ? tid : -1;
  int sum, wants = 0, before = 0, rank = 0;
  int32_t was[EACH], now[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) was[e] = now[e] = first_entry + e < entries ? g.table_from[first_entry + e] : -1;

  int source = -1, rest = 0, parent = -1, length = 0;              // of a fork, row `mine`
  if (KIND == UPDATE && mine >= 0) {
    const Range drop = places_in(g, g.drop_begin, g.drop_end, mine, true), take = places_in(g, g.take_begin, g.take_end, mine, false);
    row[mine] = (int)drop.from; row[g.batch + mine] = (int)drop.to; row[2 * g.batch + mine] = (int)take.from; row[3 * g.batch + mine] = (int)take.to;
  }
  if (KIND == FORK_ROWS && mine >= 0) {
    const int p = g.parent[mine];
    parent = (uint32_t)p < (uint32_t)g.batch ? p : -1;
    length = parent >= 0 ? max(g.length[parent], 0) : 0;
    rest = length % g.page;
    row[2 * g.batch + mine] = g.batch;
  }
  for (int p = tid; p < g.pages; p += kOneThreads) uses[p] = g.uses_from[p];
  __syncthreads();

  uint32_t wanting = 0;                                            // the thread's entries that want a page; of a fork whether its row does
  if (KIND == FORK_ROWS) {
    if (parent >= 0) atomicMin(&row[2 * g.batch + parent], mine);  // the first of a parent's
    __syncthreads();
    const bool first = parent >= 0 && row[2 * g.batch + parent] == mine;
    __syncthreads();
    if (mine >= 0) {
      const int whole = length / g.page;
      if (parent >= 0 && !first && rest > 0 && whole < places) source = g.table_from[parent * places + whole];
      if (!names(g, source)) source = -1;
      row[mine] = parent; row[g.batch + mine] = whole; row[2 * g.batch + mine] = first;
      g.length_to[mine] = length;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      now[e] = -1;
      if (first_entry + e >= entries) continue;
      const int b = quotient(first_entry + e, of_row), i = first_entry + e - b * places, p = row[b];
      if (p >= 0 && (i < row[g.batch + b] || row[2 * g.batch + b] != 0)) now[e] = g.table_from[p * places + i];
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (now[e] != was[e]) {
        if (names(g, was[e])) atomicAdd(&uses[was[e]], -1);
        if (names(g, now[e])) atomicAdd(&uses[now[e]], 1);
      }
    wanting = source >= 0;
  }
  if (KIND == UPDATE) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      if (first_entry + e >= entries) break;
      const int b = quotient(first_entry + e, of_row), i = first_entry + e - b * places;
      if (i >= row[b] && i < row[g.batch + b] && names(g, now[e])) {
        atomicAdd(&uses[now[e]], -1);
        now[e] = -1;
      }
      if (i >= row[2 * g.batch + b] && i < row[3 * g.batch + b] && !names(g, now[e])) wanting |= 1u << e;
    }
  }
  if (KIND != COMPACT) rank = sum_before<kOneWaves>(__popc(wanting), of_wave, wants);        // (which is a barrier, too)

  if (KIND == COMPACT) {
    int n = 0;
    for (int first = 0; first < g.pages; first += kOneThreads * kEach) {
      sum_before<kOneWaves>(__popc(chunk_bits(uses, g.pages, first + tid * kEach).used), of_wave, sum);
      n += sum;
    }
    PagesArgs in = g;
    in.list = list; in.target = row;
    for (int first = 0; first < g.pages; first += kOneThreads * kEach) {
      const Bits bits = chunk_bits(uses, g.pages, first + tid * kEach);
      moves_of(bits, first + tid * kEach, before + sum_before<kOneWaves>(__popc(bits.used), of_wave, sum), n, in);
      before += sum;
    }
    if (tid == 0 && g.count) *g.count = n;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (names(g, was[e]) && was[e] >= n && uses[was[e]] > 0) now[e] = row[list[was[e]]];
    __syncthreads();
    for (int p = tid; p < g.pages; p += kOneThreads)
      if (p >= n && uses[p] > 0) {
        const int to = row[list[p]];
        g.target[list[p]] = to;
        uses[to] = uses[p];
        uses[p] = 0;
      }
  } else if (KIND == FORK_ROWS || g.take_begin) {
    for (int first = 0; first < g.pages && before < wants; first += kOneThreads * kEach) {
      const Bits bits = chunk_bits(uses, g.pages, first + tid * kEach);
      uint32_t free = bits.there & ~bits.used;
      int at = before + sum_before<kOneWaves>(__popc(free), of_wave, sum);
      for (; free != 0; free &= free - 1) list[at++] = first + tid * kEach + __builtin_ctz(free);
      before += sum;
    }
    if (tid == 0 && g.count) *g.count = wants > before ? wants - before : 0;
    __syncthreads();
    auto give = [&]() {
      const int e = rank < before ? list[rank] : -1;
      ++rank;
      if (e >= 0) uses[e] = 1;
      return e;
    };
    if (KIND == FORK_ROWS) {
      int32_t* const target = row;                                 // (parents are not looked at any more)
      if (mine >= 0) {
        target[mine] = source >= 0 ? give() : -1;
        g.source[mine] = source;
        g.target[mine] = target[mine];
        g.tokens[mine] = rest;
        row[2 * g.batch + mine] = source >= 0;
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        if (first_entry + e >= entries) break;
        const int b = quotient(first_entry + e, of_row);
        if (row[2 * g.batch + b] != 0 && first_entry + e - b * places == row[g.batch + b]) now[e] = target[b];
      }
    } else {
#pragma unroll
      for (int e = 0; e < EACH; ++e)
        if (wanting >> e & 1) now[e] = give();
    }
  } else if (tid == 0 && g.count) {
    *g.count = 0;
  }
#pragma unroll
  for (int e = 0; e < EACH; ++e)
    if (first_entry + e < entries && (g.table != g.table_from || now[e] != was[e])) g.table[first_entry + e] = now[e];
  __syncthreads();
  for (int p = tid; p < g.pages; p += kOneThreads) g.uses[p] = uses[p];
}

// ---- copies -------------------------------------------------------------------------------------------------------------------

constexpr int kCaches = 16, kUnits = 1024;       // caches of a launch, 16-byte units of a block
struct CopyArgs {
  struct { uint8_t *k, *v; float *ks, *vs; int64_t stride_page, stride_scale; uint32_t half; int heads; Divisor head; } cache[kCaches];   // units of a page's keys and of one head's
  const int32_t *source, *target, *tokens;
  const int32_t* n_dev;                                  // null: n
  int n, pages, page;
};

// One block: 16 KB of a page's codes, keys before values.  A head's blocks lie one after another, so the first ones are its first units.  HBM bounds it: 504 pages of 128 KB in four layers, 265 MB
// read and written, 55 us (4.8 TB/s, of 5.05 that a large copy reaches); 96 pages, 101 MB, 22 us (4.6).
__global__ void __launch_bounds__(256) pages_copy(CopyArgs g) {
  const auto& c = g.cache[blockIdx.y];
  const int n = g.n_dev ? *g.n_dev : g.n;
  for (int pair = blockIdx.z; pair < n; pair += gridDim.z) {
    const int from = g.source[pair], to = g.target[pair];
    if ((uint32_t)from >= (uint32_t)g.pages || (uint32_t)to >= (uint32_t)g.pages || from == to) continue;
    const int tokens = g.tokens ? min(max(g.tokens[pair], 0), g.page) : g.page, blocks = (tokens + kBlockTokens - 1) / kBlockTokens, of_page = g.page / kBlockTokens;
    const uint32_t most = c.head.d / of_page * blocks;
    const int64_t src = from * c.stride_page, dst = to * c.stride_page;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    for (uint32_t u0 = blockIdx.x * kUnits; u0 < 2 * c.half; u0 += gridDim.x * kUnits) {
      u32x4 x[4];
      uint8_t* at[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t u = u0 + i * 256 + threadIdx.x;
        const bool values = u >= c.half;
        const uint32_t in = values ? u - c.half : u, in_head = in - quotient((int)in, c.head) * c.head.d;
        uint8_t* const base = values ? c.v : c.k;
        at[i] = u < 2 * c.half && in_head < most ? base + dst + (int64_t)in * 16 : nullptr;
        if (at[i]) x[i] = *reinterpret_cast<const u32x4*>(base + src + (int64_t)in * 16);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (at[i]) *reinterpret_cast<u32x4*>(at[i]) = x[i];
    }
    if (blockIdx.x == 0)
      for (int i = threadIdx.x; i < c.heads * of_page; i += 256)
        if (i % of_page < blocks) {
          c.ks[to * c.stride_scale + i] = c.ks[from * c.stride_scale + i];
          c.vs[to * c.stride_scale + i] = c.vs[from * c.stride_scale + i];
        }
  }
}

hipError_t copy_launch(const ac_kv_cache* caches, int n_caches, CopyArgs a, int64_t most, hipStream_t s) {
  if (most <= 0 || a.pages <= 0) return hipSuccess;
  for (int first = 0; first < n_caches; first += kCaches) {
    const int n = n_caches - first < kCaches ? n_caches - first : kCaches;
    int64_t units = 0;
    for (int i = 0; i < n; ++i) {
      const ac_kv_cache& c = caches[first + i];
      const uint32_t head = (uint32_t)((int64_t)c.page * c.head_dim / 16), half = head * c.heads;       // (below 2^30: a page has less than 2^34 codes)
      a.cache[i] = {(uint8_t*)c.k, (uint8_t*)c.v, c.k_scale, c.v_scale, c.stride_page, c.stride_scale, half, c.heads, divisor(head)};
      if (2 * (int64_t)half > units) units = 2 * (int64_t)half;
    }
    const int64_t pieces = (units + kUnits - 1) / kUnits;
    const dim3 grid((unsigned)(pieces < 4096 ? pieces : 4096), (unsigned)n, (unsigned)(most < 2048 ? most : 2048));
    hipLaunchKernelGGL(pages_copy, grid, dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

PagesArgs pages_args(const ac_page_books& from, const ac_page_books& to, void* workspace) {
  PagesArgs g{};
  g.uses_from = from.uses; g.table_from = from.page_table;
  g.uses = to.uses; g.table = to.page_table;
  g.pages = (int)from.pages; g.page = from.page; g.batch = (int)from.batch; g.places = from.ld_page_table;
  g.chunks = (g.pages + kChunk - 1) / kChunk;
  int32_t* w = (int32_t*)workspace;
  g.total = w; w += 64;
  g.counts = w; w += g.chunks;
  g.list = w; w += g.pages;
  const int most = g.pages > g.batch ? g.pages : g.batch;
  g.source = w; w += most;
  g.target = w; w += most;
  g.tokens = w; w += g.batch;
  g.need = w; w += g.batch;
  g.drops = w;
  return g;
}

// Whether one launch does it, and an update in two: see the head of this file.
bool at_once(const PagesArgs& g) { return g.pages <= kOnePages && g.batch <= kOneBatch && g.batch * g.places <= kOnePlaces; }
template <int KIND, int EACH>
hipError_t once_with(const PagesArgs& g, hipStream_t s) {
  constexpr int MOST = 2 * kOnePages + 4 + (kOnePages > 4 * kOneBatch ? kOnePages : 4 * kOneBatch);
  static const hipError_t attr_status = hipFuncSetAttribute(reinterpret_cast<const void*>(pages_at_once<KIND, EACH>), hipFuncAttributeMaxDynamicSharedMemorySize, MOST * (int)sizeof(int32_t));
  if (attr_status != hipSuccess) return attr_status;
  const int words = (g.pages + 3) / 4 * 4 + g.pages + (KIND == COMPACT ? g.pages : 4 * g.batch);
  hipLaunchKernelGGL((pages_at_once<KIND, EACH>), dim3(1), dim3(kOneThreads), (size_t)words * sizeof(int32_t), s, g, divisor((uint32_t)(g.places > 0 ? g.places : 1)));
  return hipGetLastError();
}
template <int KIND>
hipError_t once_launch(const PagesArgs& g, hipStream_t s) {
  const int64_t entries = g.batch * g.places;
  return entries <= kOneThreads ? once_with<KIND, 1>(g, s) : entries <= 2 * kOneThreads ? once_with<KIND, 2>(g, s) : once_with<KIND, kOneEach>(g, s);
}

bool in_two(int64_t pages, int64_t batch, int64_t places) { return pages <= kSecondPages && batch <= kSecondBatch && batch * places <= kSecondPlaces; }

template <bool FORK>
hipError_t rows_launch(const PagesArgs& g, hipStream_t s) {
  if (at_once(g)) return once_launch<FORK ? FORK_ROWS : UPDATE>(g, s);
  if (!FORK && in_two(g.pages, g.batch, g.places)) {
    static const hipError_t attr_status = hipFuncSetAttribute(reinterpret_cast<const void*>(pages_second), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                              (2 * kSecondPages + 2 * kSecondBatch + 4) * (int)sizeof(int32_t));
    if (attr_status != hipSuccess) return attr_status;
    PagesArgs n = g;
    n.dropped = g.drops + g.batch;
    n.wanted = n.dropped + g.batch * g.places;
    hipLaunchKernelGGL((pages_rows<FORK>), dim3((unsigned)(g.batch / 4 + 1)), dim3(256), 0, s, n);
    hipLaunchKernelGGL(pages_second, dim3(1), dim3(kSecondThreads), ((g.pages + 3) / 4 * 4 + g.pages + 2 * g.batch) * sizeof(int32_t), s, n);
    return hipGetLastError();
  }
  if (g.uses != g.uses_from && g.pages > 0)
    hipLaunchKernelGGL(pages_copy_uses, dim3((unsigned)(g.chunks < 1024 ? 4 * g.chunks : 4096)), dim3(256), 0, s, g);
  hipLaunchKernelGGL((pages_rows<FORK>), dim3((unsigned)(g.batch / 4 + 1)), dim3(256), 0, s, g);
  if (FORK || g.take_begin) {
    if (g.pages <= kRankPages) {
      hipLaunchKernelGGL(pages_rank, dim3(1), dim3(kRankThreads), 0, s, g);
    } else {
      hipLaunchKernelGGL(pages_count, dim3((unsigned)g.chunks + 1), dim3(256), 0, s, g);
      hipLaunchKernelGGL(pages_list, dim3((unsigned)g.chunks), dim3(256), 0, s, g);
    }
    hipLaunchKernelGGL((pages_give<FORK>), dim3((unsigned)(g.batch / (FORK ? 256 : 4) + 1)), dim3(256), 0, s, g);
  }
  return hipGetLastError();
}

}  // namespace

uint64_t pages_workspace_bytes(const ac_page_books& b) {
  const uint64_t most = b.pages > b.batch ? b.pages : b.batch;
  const uint64_t noted = in_two(b.pages, b.batch, b.ld_page_table) ? 2 * b.batch * b.ld_page_table : 0;
  return (64 + (b.pages + kChunk - 1) / kChunk + b.pages + 2 * most + 3 * b.batch + noted) * sizeof(int32_t);
}

hipError_t launch_pages_update(const ac_page_books& from, const ac_page_books& to, const int32_t* drop_begin, const int32_t* drop_end, const int32_t* take_begin,
                               const int32_t* take_end, int32_t* missing, void* workspace, hipStream_t s) {
  PagesArgs g = pages_args(from, to, workspace);
  g.drop_begin = drop_begin; g.drop_end = drop_end; g.take_begin = take_begin; g.take_end = take_end;
  g.count = missing;
  return rows_launch<false>(g, s);
}

hipError_t launch_cache_fork(const ac_kv_cache* caches, int n_caches, const ac_page_books& from, const ac_page_books& to, const int32_t* parent,
                             const int32_t* length, int32_t* length_to, int32_t* missing, void* workspace, hipStream_t s) {
  PagesArgs g = pages_args(from, to, workspace);
  g.parent = parent; g.length = length; g.length_to = length_to;
  g.count = missing;
  const hipError_t e = rows_launch<true>(g, s);
  if (e != hipSuccess) return e;
  CopyArgs c{};
  c.source = g.source; c.target = g.target; c.tokens = g.tokens; c.n = g.batch; c.pages = g.pages; c.page = g.page;
  return copy_launch(caches, n_caches, c, g.batch, s);
}

hipError_t launch_cache_compact(const ac_kv_cache* caches, int n_caches, const ac_page_books& from, const ac_page_books& to, int32_t* used, void* workspace,
                                hipStream_t s) {
  PagesArgs g = pages_args(from, to, workspace);
  g.count = used;
  hipError_t e;
  if (at_once(g)) {
    e = once_launch<COMPACT>(g, s);
  } else {
    const int blocks = g.chunks > 0 ? g.chunks : 1;
    hipLaunchKernelGGL(compact_count, dim3((unsigned)blocks), dim3(256), 0, s, g);
    hipLaunchKernelGGL(compact_list, dim3((unsigned)blocks), dim3(256), 0, s, g);
    const int64_t all = g.batch * g.places > g.pages ? g.batch * g.places : g.pages, each = (all + 1023) / 1024;
    hipLaunchKernelGGL(compact_follow, dim3((unsigned)(each < 1 ? 1 : each < 4096 ? each : 4096)), dim3(256), 0, s, g);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  CopyArgs c{};
  c.source = g.source; c.target = g.target; c.n_dev = g.total; c.pages = g.pages; c.page = g.page;
  return copy_launch(caches, n_caches, c, g.pages / 2, s);
}

hipError_t launch_cache_copy_pages(const ac_kv_cache* caches, int n_caches, const int32_t* source, const int32_t* target, const int32_t* tokens, int64_t n,
                                   hipStream_t s) {
  if (n <= 0 || n_caches <= 0 || caches[0].pages <= 0) return hipSuccess;
  CopyArgs c{};
  c.source = source; c.target = target; c.tokens = tokens; c.n = (int)n; c.pages = (int)caches[0].pages; c.page = caches[0].page;
  return copy_launch(caches, n_caches, c, n, s);
}

}  // namespace ac
