// Rows of a table by tokens, and the table's gradient (gfx950, 64-lane wavefronts).
//   y_i = scale W[t_i];   dW[v] = scale sum_{i: t_i = v} dy_i
// Tokens outside [0, V) are padding: zeros, and no gradient.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elements.h"

namespace ngsgd {

constexpr int kLookupThreads = 256;
constexpr int kLookupRows = 4;          // rows that a thread has in flight

struct EmbeddingForward {
  const void* tokens;
  int64_t N;
  const void* table;
  int64_t ldt;
  int64_t V;
  int D;
  float scale;
  void* y;
  int64_t ldy;
  int slabs;         // a row is cut into so many slabs,
  int slab;          // of so many pieces;
  int lanes;         // threads that share one, a power of two
};

// A token that is sorted: its row of the table (V: padding, which goes last) and its place among the tokens.
struct SortedToken {
  uint32_t key, place;
};

struct EmbeddingBackward {
  const void* dy;
  int64_t lddy;
  const void* tokens;
  int64_t N, V;
  int D;
  float scale;
  void* dtable;
  int64_t lddt;
  int accumulate;
  const SortedToken* sorted;
  float* parts;       // [chunks][2][pieces E]: sums that a chunk shares with the one before it, and the one behind it
  int chunk;          // sorted tokens that are added one after the other, a power of two
  int64_t chunks;
  int pieces, lanes, slabs;   // pieces of E columns of a row; threads that share a chunk, each with one of them; groups of so many pieces
  unsigned sum_groups;   // workgroups that add; those behind them write the rows that no token names,
  int clear_rows;        // so many rows (at most 64) to a wavefront
};

// ---- lookup -------------------------------------------------------------------------------------------------
// Bound by memory: y is written once, and of the table what the dies' caches do not hold is read.  A thread has pieces of E elements of kLookupRows rows in
// flight: their tokens first, then the table's rows (8 rows: 4 % slower; 8-byte stores for fp32 tables, so that loads are dense: the same).  The last piece
// of a row is moved back to end with it (its first elements are written twice, with the same values).  PAST: y is written past the caches.  (The compiler would
// make one ordinary store of the two kinds behind a condition.)  196613 x 4096 fp32 to bf16, a Zipf law over 50021 rows: 532 us, 1.61 GB written and
// 0.85 GB of the 3.0 GB read fetched, 4.6 TB/s, near what a copy reaches; 131072 x 4096 bf16 over 32000: 280 us, 4.8 TB/s.
template <typename W, typename T, typename I, int E, bool PAST>
__global__ __launch_bounds__(kLookupThreads) void embedding_forward_kernel(const EmbeddingForward a) {
  const int lane = threadIdx.x & (a.lanes - 1), per_round = kLookupThreads / a.lanes;
  const int64_t first = (int64_t)(blockIdx.x / a.slabs) * per_round * kLookupRows + threadIdx.x / a.lanes;
  I raw[kLookupRows];
#pragma unroll
  for (int k = 0; k < kLookupRows; ++k) raw[k] = static_cast<const I*>(a.tokens)[min(first + k * per_round, a.N - 1)];
  const int pieces = (a.D + E - 1) / E, from = (int)(blockIdx.x % a.slabs) * a.slab, to = min(from + a.slab, pieces);
  for (int p = from + lane; p < to; p += a.lanes) {
    const int at = min(p * E, a.D - E);
    Pack<W, E> w[kLookupRows];
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k) {
      const bool named = (uint64_t)(int64_t)raw[k] < (uint64_t)a.V;
      w[k] = *reinterpret_cast<const Pack<W, E>*>(static_cast<const W*>(a.table) + (named ? (int64_t)raw[k] : 0) * a.ldt + at);
    }
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k) {
      const bool named = (uint64_t)(int64_t)raw[k] < (uint64_t)a.V;
      if (first + k * per_round >= a.N) continue;
      Pack<T, E> y;
#pragma unroll
      for (int j = 0; j < E; ++j) y.v[j] = from_float<T>(named ? as_f32(a.scale * to_float(w[k].v[j])) : 0.f);
      T* const to = static_cast<T*>(a.y) + (first + k * per_round) * a.ldy + at;
      if constexpr (PAST) store_pack_past(to, y); else store_pack(to, y);
    }
  }
}

// ---- sorting ----------------------------------------------------------------------------------------------
template <typename I>
__device__ __forceinline__ uint32_t key_of(const I t, const int64_t V) { return (uint64_t)(int64_t)t < (uint64_t)V ? (uint32_t)t : (uint32_t)V; }

// Few tokens: each one's rank is counted, sum_j [key_j < key_i or (key_j = key_i and j < i)], among all (TILES = 0, up to kRankMost) or among the 1024 of its
// tile.  A workgroup's 16 wavefronts share 64 tokens and deal the others between them, 64 at a time.  Their keys come from LDS, four with one read that all lanes
// share: a wavefront's own copy, without a barrier.  Two instructions a pair: 4096 tokens 8.2 us, 1024 4.7 (8192 13.6, in tiles 4.7 and 4.6 to merge them; by
// v_readlane in 512 unrolled steps 22: the instructions came from memory).
constexpr int kRankThreads = 1024, kRankRounds = 4, kRankMost = kRankThreads * kRankRounds;   // tokens
template <typename I, bool TILES>
__global__ __launch_bounds__(kRankThreads) void embedding_rank_kernel(const I* tokens, const int N, const int64_t V, SortedToken* sorted) {
  constexpr int kRounds = TILES ? 1 : kRankRounds;
  __shared__ U32x4 keys[kRankThreads / 64][kRounds][16];
  __shared__ int counts[kRankThreads / 64][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = blockIdx.x * 64, i = first + lane;
  const int start = TILES ? first / kRankThreads * kRankThreads : 0, end = TILES ? min(start + kRankThreads, N) : N;   // of those that are compared
  I others[kRounds];
  const I own = tokens[min(i, N - 1)];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) others[r] = tokens[min(start + r * kRankThreads + (int)threadIdx.x, N - 1)];
  const uint32_t key = key_of(own, V);
#pragma unroll
  for (int r = 0; r < kRounds; ++r)
    reinterpret_cast<uint32_t*>(keys[wave][r])[lane] = start + r * kRankThreads + (int)threadIdx.x < end ? key_of(others[r], V) : 0xffffffffu;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  int count = 0;
  for (int r = 0, base = start + wave * 64; base < end; ++r, base += kRankThreads) {
    // those in front go first among equals
    const uint32_t limit = base < first ? key + 1 : key;
    if (base != first) {
#pragma unroll 4
      for (int k = 0; k < 16; ++k) {
        const U32x4 other = keys[wave][r][k];
        count += (other.x < limit) + (other.y < limit) + (other.z < limit) + (other.w < limit);
      }
    } else {
#pragma unroll 4
      for (int k = 0; k < 16; ++k) {
        const U32x4 other = keys[wave][r][k];
        count += (other.x < key + (4 * k < lane)) + (other.y < key + (4 * k + 1 < lane)) + (other.z < key + (4 * k + 2 < lane)) +
                 (other.w < key + (4 * k + 3 < lane));
      }
    }
  }
  counts[wave][lane] = count;
  __syncthreads();
  if (wave != 0 || i >= N) return;
  int rank = 0;
#pragma unroll
  for (int k = 0; k < kRankThreads / 64; ++k) rank += counts[k][lane];
  sorted[start + rank] = SortedToken{key, (uint32_t)i};
}

// Up to 32 sorted tiles into one list: a token goes behind those of the tiles in front whose keys are not above its own, and of the tiles behind whose keys are
// below.  A workgroup has 64 neighbours of a tile; a wavefront looks for them in every 16th tile, whose keys it copies to LDS while it looks in the one before
// (by reading the tiles from the cache in every step: 20011 tokens 8.6 us instead of 7.7).  The work grows with the square of the tiles: 32768 tokens 11.8, ranks in
// the tiles 5.6, where sorting by digits takes 25 in four launches; 65536 34, where it takes 25 too.
constexpr int kMergeTiles = 32, kMergeMost = kMergeTiles * kRankThreads, kMergeLoads = kRankThreads / 64;
__global__ __launch_bounds__(kRankThreads) void embedding_merge_kernel(const SortedToken* tiles, const int N, SortedToken* sorted) {
  constexpr int kWaves = kRankThreads / 64;
  __shared__ uint32_t keys[kWaves][kRankThreads];
  __shared__ int counts[kWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = blockIdx.x * 64 + lane;
  const int own = blockIdx.x * 64 / kRankThreads, n_tiles = (N + kRankThreads - 1) / kRankThreads;
  uint32_t next[kMergeLoads];
  const auto ask = [&](const int tile) {
#pragma unroll
    for (int r = 0; r < kMergeLoads; ++r) next[r] = tiles[min(tile * kRankThreads + r * 64 + lane, N - 1)].key;
  };
  if (wave < n_tiles) ask(wave);
  const SortedToken token = tiles[min(i, N - 1)];
  int count = 0;
  for (int tile = wave; tile < n_tiles; tile += kWaves) {
#pragma unroll
    for (int r = 0; r < kMergeLoads; ++r)
      keys[wave][r * 64 + lane] = tile * kRankThreads + r * 64 + lane < N ? next[r] : 0xffffffffu;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (tile + kWaves < n_tiles) ask(tile + kWaves);
    if (tile != own) {
      const uint32_t limit = tile < own ? token.key + 1 : token.key;
      int at = 0;
#pragma unroll
      for (int step = kRankThreads / 2; step > 0; step /= 2)
        if (keys[wave][at + step - 1] < limit) at += step;
      count += at + (keys[wave][at] < limit);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  counts[wave][lane] = count;
  __syncthreads();
  if (wave != 0 || i >= N) return;
  int rank = i - own * kRankThreads;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) rank += counts[k][lane];
  sorted[rank] = token;
}

// More: a radix sort from the lowest digit, each pass stable, as few passes as digits of 10 bits allow.  Latency bounds it (few workgroups, one step behind the
// other): a pass over 32769 tokens takes 12.4 us, over 262144 17.  A workgroup has a tile of kSortRounds tokens a thread; counts[tile][digit].
constexpr int kSortThreads = 1024, kSortBits = 10, kSortBins = 1 << kSortBits, kSortRounds = 4;
// Tiles up to which a workgroup adds up the counts in front of it itself.  A call of 8 columns with 64 tiles, and with 65 through a launch more: 45.0 and 43.6 us over
// 1000 rows (one pass), 77.7 and 79.2 over 131072 (two), 73.1 and 77.8 over 2^21 (three).
constexpr int kSortInline = 64;

struct EmbeddingSort {
  const void* tokens;          // of the first pass
  const SortedToken* in;       // of the others
  SortedToken* out;
  int64_t N, V;
  uint32_t* counts;            // [tiles][bins]
  uint32_t* totals;            // [bins], where there are more tiles than kSortInline
  int tiles;
  int shift, bins;             // of this pass's digit; a power of two, at least 4
};

template <typename I, bool FIRST>
__device__ __forceinline__ SortedToken sort_input(const EmbeddingSort& a, const int64_t i) {
  if (FIRST) return SortedToken{key_of(static_cast<const I*>(a.tokens)[i], a.V), (uint32_t)i};
  return a.in[i];
}

template <typename I, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(const EmbeddingSort a) {
  __shared__ uint32_t bins[kSortBins];
  const int64_t from = (int64_t)blockIdx.x * kSortThreads * kSortRounds + threadIdx.x;
  uint32_t key[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) key[r] = sort_input<I, FIRST>(a, min(from + r * kSortThreads, a.N - 1)).key;
  for (int d = threadIdx.x; d < a.bins; d += kSortThreads) bins[d] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r)
    if (from + r * kSortThreads < a.N) atomicAdd(&bins[key[r] >> a.shift & (a.bins - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < a.bins; d += kSortThreads) a.counts[(int64_t)blockIdx.x * a.bins + d] = bins[d];
}

// Many tiles: counts become those of the tiles in front.  A lane per digit; 16 wavefronts share the tiles.
__global__ __launch_bounds__(1024) void embedding_scan_kernel(const EmbeddingSort a) {
  __shared__ uint32_t sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * 64 + lane;
  const int share = (a.tiles + 15) / 16, from = min(wave * share, a.tiles), to = min(from + share, a.tiles);
  uint32_t sum = 0;
  if (d < a.bins) {
#pragma unroll 8
    for (int t = from; t < to; ++t) sum += a.counts[(int64_t)t * a.bins + d];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  uint32_t before = 0, total = 0;
  for (int k = 0; k < 16; ++k) {
    if (k < wave) before += sums[k][lane];
    total += sums[k][lane];
  }
  if (d >= a.bins) return;
#pragma unroll 8
  for (int t = from; t < to; ++t) {
    uint32_t* const at = a.counts + (int64_t)t * a.bins + d;
    const uint32_t here = *at;
    *at = before;
    before += here;
  }
  if (wave == 0) a.totals[d] = total;
}

// Places: digits in order, tiles in order within a digit, a tile's tokens in order within that.  A wavefront ranks 64 tokens at a time: lanes
// with the same digit find each other by one ballot a bit.  Then every thread has one of the digits.
template <typename I, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void embedding_scatter_kernel(const EmbeddingSort a) {
  static_assert(kSortBins == kSortThreads);
  constexpr int kWaves = kSortThreads / 64;
  __shared__ uint32_t bins[kWaves * kSortBins];   // of each wavefront: its count, then where its next token with that digit goes
  __shared__ uint32_t waves[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool owns = threadIdx.x < (unsigned)a.bins;
  uint32_t* const mine = bins + wave * a.bins;
  const int64_t from = ((int64_t)blockIdx.x * kSortThreads + wave * 64) * kSortRounds + lane;
  SortedToken token[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) token[r] = sort_input<I, FIRST>(a, min(from + r * 64, a.N - 1));
  // tokens with this thread's digit: in all tiles, and in those in front
  uint32_t total = 0, before = 0;
  if (owns) {
    const uint32_t* const counts = a.counts + threadIdx.x;
    if (a.totals != nullptr) {
      before = counts[(int64_t)blockIdx.x * a.bins];
      total = a.totals[threadIdx.x];
    } else {
      constexpr int kAhead = 16;
      for (int t = 0; t < a.tiles; t += kAhead) {
        uint32_t of[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) of[u] = counts[min(t + u, a.tiles - 1) * a.bins];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const uint32_t here = t + u < a.tiles ? of[u] : 0u;
          before += t + u < (int)blockIdx.x ? here : 0u;
          total += here;
        }
      }
    }
  }
  for (int d = threadIdx.x; d < kWaves * a.bins; d += kSortThreads) bins[d] = 0;
  __syncthreads();
  uint32_t rank[kSortRounds];                     // within the wavefront
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const bool here = from + r * 64 < a.N;
    const uint32_t digit = here ? token[r].key >> a.shift & (a.bins - 1) : 0;
    uint64_t same = __builtin_amdgcn_ballot_w64(here);
    for (int bit = 1; bit < a.bins; bit *= 2) {
      const bool set = (digit & bit) != 0;
      const uint64_t with = __builtin_amdgcn_ballot_w64(set);
      same &= set ? with : ~with;
    }
    const uint32_t in_front = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
    if (here) rank[r] = mine[digit] + in_front;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (here && in_front == 0) mine[digit] += (uint32_t)__builtin_popcountll(same);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  // tokens with lower digits than this thread's
  uint32_t below = total;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) {
    const uint32_t o = __shfl_up(below, k);
    if (lane >= k) below += o;
  }
  if (lane == 63) waves[wave] = below;
  __syncthreads();
  below -= total;
  for (int k = 0; k < wave; ++k) below += waves[k];
  if (owns) {
    uint32_t at = below + before, here[kWaves];
    uint32_t* const bin = bins + threadIdx.x;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) here[w] = bin[w * a.bins];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      bin[w * a.bins] = at;
      at += here[w];
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r)
    if (from + r * 64 < a.N) a.out[mine[token[r].key >> a.shift & (a.bins - 1)] + rank[r]] = token[r];
}

// ---- sums --------------------------------------------------------------------------------------------------
// A piece of a table's row: written, or added to what is there.  The last piece of a row is moved back to end with it.  The columns that the piece
// before has too are written twice, with the same values, but added once.
template <typename W, int E>
__device__ __forceinline__ void store_piece(const EmbeddingBackward& a, const uint32_t row, const int piece, const float (&sum)[E]) {
  const int at = min(piece * E, a.D - E);
  W* const out = static_cast<W*>(a.dtable) + row * a.lddt + at;
  if (!a.accumulate) {
    Pack<W, E> v;
#pragma unroll
    for (int j = 0; j < E; ++j) v.v[j] = from_float<W>(as_f32(a.scale * sum[j]));
    store_pack(out, v);
  } else {
    const int skip = piece * E - at;
    Pack<W, E> v = *reinterpret_cast<const Pack<W, E>*>(out);
#pragma unroll
    for (int j = 0; j < E; ++j) v.v[j] = from_float<W>(as_f32(to_float(v.v[j]) + a.scale * sum[j]));
    if (skip == 0) {
      store_pack(out, v);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (j >= skip) out[j] = v.v[j];
    }
  }
}

constexpr int kSumThreads = 256, kSumAhead = 8;   // rows that a thread has in flight

// The sums of a chunk of sorted tokens, of the columns of this thread's piece.  A token whose rows are all in the chunk is done; the first one's and the last
// one's sums are parts if the chunks beside this one have rows of theirs.  Bound by memory: 262144 x 2048 bf16 over 131072 rows in fp32 (1.04 GB read, 1.07
// GB written with the rows that are cleared) 450 us, 4.7 TB/s, what a copy reaches; 8192 wavefronts instead of 4096 480, 2048 585.
template <typename T, typename W, int E>
__device__ __forceinline__ void embedding_sum_chunk(const EmbeddingBackward& a, const int64_t chunk, const int piece) {
  const int64_t from = chunk * a.chunk, to = min(from + a.chunk, a.N);
  const int at = min(piece * E, a.D - E);
  float sum[E];
#pragma unroll
  for (int j = 0; j < E; ++j) sum[j] = 0.f;
  uint32_t key = a.sorted[from].key;
  bool before = from > 0 && a.sorted[from - 1].key == key;   // the chunk in front has rows of this token
  const auto finish = [&](const bool behind) {
    if (piece >= a.pieces) return;
    if (!before && !behind) {
      store_piece<W, E>(a, key, piece, sum);
    } else {
      float* const part = a.parts + ((chunk * 2 + (before ? 0 : 1)) * a.pieces + piece) * E;
#pragma unroll
      for (int j = 0; j < E; ++j) part[j] = sum[j];
    }
  };
  for (int64_t p = from; p < to; p += kSumAhead) {
    SortedToken token[kSumAhead];
    Pack<T, E> row[kSumAhead];
#pragma unroll
    for (int k = 0; k < kSumAhead; ++k) token[k] = a.sorted[min(p + k, to - 1)];
#pragma unroll
    for (int k = 0; k < kSumAhead; ++k)
      if (token[k].key < (uint32_t)a.V && piece < a.pieces)
        row[k] = *reinterpret_cast<const Pack<T, E>*>(static_cast<const T*>(a.dy) + token[k].place * a.lddy + at);
#pragma unroll
    for (int k = 0; k < kSumAhead; ++k) {
      if (p + k >= to || token[k].key >= (uint32_t)a.V) continue;
      if (token[k].key != key) {
        finish(false);
        key = token[k].key;
        before = false;
#pragma unroll
        for (int j = 0; j < E; ++j) sum[j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < E; ++j) sum[j] += to_float(row[k].v[j]);
    }
  }
  if (key < (uint32_t)a.V) finish(to < a.N && a.sorted[to].key == key);
}

// Very few tokens: no sorting.  A wavefront has all of them in its lanes, walks over rows of the table (and slabs of 64 pieces) and finds those that name
// one by a ballot for each 64: one launch instead of three.  50000 x 1024 bf16 with 64 tokens 16 us (6.4 TB/s of zeros; sorted 25), two rows
// with 128 tokens 17 (sorted 16 in three launches).
constexpr int kFewRounds = 2, kFewTokens = kFewRounds * 64;
template <typename T, typename W, typename I, int E>
__global__ __launch_bounds__(kSumThreads) void embedding_few_kernel(const EmbeddingBackward a) {
  const int lane = threadIdx.x & 63, N = (int)a.N;
  I raw[kFewRounds];
#pragma unroll
  for (int r = 0; r < kFewRounds; ++r) raw[r] = static_cast<const I*>(a.tokens)[min(r * 64 + lane, N - 1)];
  uint32_t key[kFewRounds];
#pragma unroll
  for (int r = 0; r < kFewRounds; ++r) key[r] = r * 64 + lane < N ? key_of(raw[r], a.V) : (uint32_t)a.V;
  const int64_t units = a.V * a.slabs, step = (int64_t)gridDim.x * (kSumThreads / 64);
  for (int64_t u = (int64_t)blockIdx.x * (kSumThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); u < units; u += step) {
    const uint32_t v = (uint32_t)(u / a.slabs);
    const int piece = (int)(u % a.slabs) * 64 + lane, at = min(piece * E, a.D - E);
    float sum[E];
#pragma unroll
    for (int j = 0; j < E; ++j) sum[j] = 0.f;
    bool named = false;
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r) {
      uint64_t mask = __builtin_amdgcn_ballot_w64(key[r] == v);
      named |= mask != 0;
      while (mask != 0) {
        const int here = __builtin_popcountll(mask);
        Pack<T, E> row[kSumAhead];
#pragma unroll
        for (int k = 0; k < kSumAhead; ++k) {
          if (k >= here) break;
          const int64_t i = r * 64 + __builtin_ctzll(mask);
          mask &= mask - 1;
          if (piece < a.pieces) row[k] = *reinterpret_cast<const Pack<T, E>*>(static_cast<const T*>(a.dy) + i * a.lddy + at);
        }
#pragma unroll
        for (int k = 0; k < kSumAhead; ++k) {
          if (k >= here) break;
#pragma unroll
          for (int j = 0; j < E; ++j) sum[j] += to_float(row[k].v[j]);
        }
      }
    }
    if (piece < a.pieces && (named || !a.accumulate)) store_piece<W, E>(a, v, piece, sum);
  }
}

// First place in [low, high) of the sorted tokens whose key is not below this one (high, if there is none): a lane for each of 64 places at a time.
__device__ __forceinline__ int64_t wave_lower_bound(const SortedToken* sorted, int64_t low, int64_t high, const uint32_t key) {
  const int lane = threadIdx.x & 63;
  while (low < high) {
    const int64_t step = (high - low + 63) / 64, at = low + (lane + 1) * step - 1;   // the last place of the lane's share
    const int below = __builtin_popcountll(__builtin_amdgcn_ballot_w64(at < high && sorted[at].key < key));
    low += below * step;
    high = min(high, low + step - 1);                                                // (that share's last place is not below)
  }
  return low;
}

// Zeros in those of a.clear_rows rows that no token names.
template <typename W>
__device__ __forceinline__ void embedding_clear_rows(const EmbeddingBackward& a, const int64_t first) {
  constexpr int E = 16 / sizeof(W);
  const int lane = threadIdx.x & 63;
  // the tokens that name these rows: looked for among few, or each row's for itself among many
  const int64_t from = wave_lower_bound(a.sorted, 0, a.N, (uint32_t)first), to = wave_lower_bound(a.sorted, from, a.N, (uint32_t)(first + a.clear_rows));
  const int64_t v = first + lane;
  bool named = false;
  if (to - from <= 64) {
    const uint32_t at = from + lane < to ? a.sorted[from + lane].key - (uint32_t)first : 64u;
    uint32_t low = at < 32 ? 1u << at : 0u, high = at >= 32 && at < 64 ? 1u << (at - 32) : 0u;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
      low |= __shfl_xor(low, k);
      high |= __shfl_xor(high, k);
    }
    named = ((lane < 32 ? low : high) >> (lane & 31) & 1u) != 0;
  } else {
    int64_t low = from, high = to;
    while (low < high) {
      const int64_t mid = (low + high) / 2;
      if (a.sorted[mid].key < (uint32_t)v) low = mid + 1; else high = mid;
    }
    named = low < to && a.sorted[low].key == (uint32_t)v;
  }
  for (uint64_t rows = __builtin_amdgcn_ballot_w64(lane < a.clear_rows && v < a.V && !named); rows != 0; rows &= rows - 1) {
    W* const row = static_cast<W*>(a.dtable) + (first + __builtin_ctzll(rows)) * a.lddt;
    Pack<W, E> zeros;
#pragma unroll
    for (int j = 0; j < E; ++j) zeros.v[j] = from_float<W>(0.f);
    const int full = a.D / E;
    for (int p = lane; p < full; p += 64) store_pack(row + p * E, zeros);
    if (full * E + lane < a.D) row[full * E + lane] = from_float<W>(0.f);
  }
}

template <typename T, typename W, int E, bool WAVE>
__global__ __launch_bounds__(kSumThreads) void embedding_sum_kernel(const EmbeddingBackward a) {
  if (blockIdx.x >= a.sum_groups) {
    const int64_t wave = (int64_t)(blockIdx.x - a.sum_groups) * (kSumThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (wave * a.clear_rows < a.V) embedding_clear_rows<W>(a, wave * a.clear_rows);
    return;
  }
  if (WAVE) {   // (uniform)
    const int64_t unit = (int64_t)blockIdx.x * (kSumThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t chunk = unit / a.slabs;
    if (chunk < a.chunks) embedding_sum_chunk<T, W, E>(a, chunk, (int)(unit % a.slabs) * 64 + (threadIdx.x & 63));
  } else {
    const int64_t chunk = ((int64_t)blockIdx.x * kSumThreads + threadIdx.x) / a.lanes;
    if (chunk < a.chunks) embedding_sum_chunk<T, W, E>(a, chunk, threadIdx.x & (a.lanes - 1));
  }
}

// A workgroup per chunk in which a token begins that goes on behind it, and slab of pieces: the parts of all chunks that have rows of it, dealt to groups of
// a.lanes threads, whose sums are added two by two.  The longest run bounds it: 34000 of 262144 tokens, 133 parts of 2048 columns, 14 us.
constexpr int kJoinThreads = 512, kJoinAhead = 4;
template <typename W, int E>
__global__ __launch_bounds__(kJoinThreads) void embedding_join_kernel(const EmbeddingBackward a) {
  __shared__ float parts[E][kJoinThreads];
  const int64_t chunk = blockIdx.x / a.slabs, from = chunk * a.chunk, to = from + a.chunk;
  if (to >= a.N) return;
  const uint32_t key = a.sorted[to - 1].key, behind = a.sorted[to].key, in_front = from > 0 ? a.sorted[from - 1].key : ~key;
  if (key >= (uint32_t)a.V || behind != key || in_front == key) return;
  int64_t last = chunk + 1;              // the chunk with its last row: a lane looks where each of the next ones ends
  for (;;) {
    const int64_t end = (last + (threadIdx.x & 63) + 1) * a.chunk;
    const uint64_t goes_on = __builtin_amdgcn_ballot_w64(end < a.N && a.sorted[end].key == key);
    if (~goes_on != 0) {
      last += __builtin_ctzll(~goes_on);
      break;
    }
    last += 64;
  }
  const int lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes, groups = kJoinThreads / a.lanes;
  const int piece = (int)(blockIdx.x % a.slabs) * 64 + lane;
  float sum[E];
#pragma unroll
  for (int j = 0; j < E; ++j) sum[j] = 0.f;
  if (piece < a.pieces) {
    for (int64_t c = chunk + group; c <= last; c += groups * kJoinAhead) {
      Pack<float, E> part[kJoinAhead];
#pragma unroll
      for (int k = 0; k < kJoinAhead; ++k) {
        const int64_t of = min(c + k * groups, last);
        part[k] = *reinterpret_cast<const Pack<float, E>*>(a.parts + ((of * 2 + (of == chunk ? 1 : 0)) * a.pieces + piece) * E);
      }
#pragma unroll
      for (int k = 0; k < kJoinAhead; ++k) {
        const bool here = c + k * groups <= last;   // (behind a condition, the compiler would load one after the other)
#pragma unroll
        for (int j = 0; j < E; ++j) sum[j] += here ? part[k].v[j] : 0.f;
      }
    }
  }
  int half = groups;
  while (half / 2 > last - chunk) half /= 2;   // (the groups behind these have nothing)
  if (group < half) {
#pragma unroll
    for (int j = 0; j < E; ++j) parts[j][threadIdx.x] = sum[j];
  }
  while (half > 1) {
    half /= 2;
    __syncthreads();
    if (group < half) {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        sum[j] += parts[j][threadIdx.x + half * a.lanes];
        parts[j][threadIdx.x] = sum[j];
      }
    }
  }
  if (group == 0 && piece < a.pieces) store_piece<W, E>(a, key, piece, sum);
}

}  // namespace ngsgd
