// C ABI of the embedding: argument checks, launches.  Declarations and contracts are in include/ngsgd.h.
#include "embedding.h"

#include <algorithm>
#include <cmath>

#include "host.h"

using namespace ngsgd;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;
constexpr int32_t kMostColumns = 1 << 25;

int check_types(const int index_type, const int table_type, const int type, const int64_t N, const int64_t V, const int32_t D) {
  if (!known_index(index_type) || !known_type(type) || !known_type(table_type) || (table_type != type && table_type != NGSGD_FLOAT32)) return NGSGD_EINVAL;
  return N < 0 || N > kMostRows || V < 1 || V > kMostRows || D < 1 || D > kMostColumns ? NGSGD_EINVAL : NGSGD_OK;
}

// f(element, table's element, token) for the types of a call
template <typename F>
int with_types(const int type, const int table_type, const int index_type, F f) {
  const auto g = [&](auto t, auto w) { return index_type == NGSGD_INT32 ? f(t, w, int32_t()) : f(t, w, int64_t()); };
  if (type == NGSGD_FLOAT32) return g(float(), float());
  if (type == NGSGD_BFLOAT16) return table_type == NGSGD_FLOAT32 ? g(bf16(), float()) : g(bf16(), bf16());
  return table_type == NGSGD_FLOAT32 ? g(fp16(), float()) : g(fp16(), fp16());
}

// Rows of the table from here on are cut into eight slabs, one for each die (workgroups go to them in turn), whose cache then holds eight times as many rows'
// parts (196613 x 4096 fp32 to bf16: 1.37 -> 0.85 GB fetched).  What a call takes without and with them, us, 131072 tokens (from 23 KB of y on so many that y has 3 GB) of
// a Zipf law over 50021 rows: fp32 4096 columns 631, 598; 4104 592, 595; 5120 795, 765; 6152 868, 801; 8192 863, 745; 16384 841, 776; fp32 to bf16 4096 361, 357; 4104
// 369, 408; 5120 461, 497; 6152 577, 578; 8192 719, 680; bf16 8192 623, 607; 8200 595, 616; 10240 783, 805; 12296 881, 825; 16384 849, 766.  Between 16 and 24 KB it
// depends on how a slab's pieces fill a power of two of threads: up to 5 % are won, and up to 10 % lost.  Narrower rows lose (131072 x 4096 bf16 281 -> 300), and so
// do two or more slabs of a die one after the other (530 -> 550 and more: pieces of y that are written together get short).
constexpr size_t kSlabBytes = 16384;
constexpr int kDies = 8;
// What is larger than all dies' caches is written past them, which leaves them to the table (65536 x 1024 bf16 29 -> 26 us, 131072 x 4096 309 -> 281).
constexpr size_t kPastBytes = (size_t)32 << 20;

template <typename W, typename T, typename I, int E>
int launch_forward(EmbeddingForward a, hipStream_t s) {
  const int pieces = (a.D + E - 1) / E;
  a.slabs = a.D * sizeof(W) >= kSlabBytes ? kDies : 1;
  a.slab = (pieces + a.slabs - 1) / a.slabs;
  for (a.lanes = 1; a.lanes < a.slab && a.lanes < kLookupThreads; a.lanes *= 2) {
  }
  const int64_t rows = (int64_t)kLookupThreads / a.lanes * kLookupRows;
  const int64_t most = ((int64_t)1 << 23) / a.slabs * rows, N = a.N;   // (a launch has less than 2^32 threads)
  for (int64_t first = 0; first < N; first += most) {
    a.N = std::min(most, N - first);
    const dim3 grid((unsigned)((a.N + rows - 1) / rows * a.slabs));
    if (E > 1 && (size_t)N * a.D * sizeof(T) > kPastBytes)
      hipLaunchKernelGGL((embedding_forward_kernel<W, T, I, E, (E > 1)>), grid, dim3(kLookupThreads), 0, s, a);
    else
      hipLaunchKernelGGL((embedding_forward_kernel<W, T, I, E, false>), grid, dim3(kLookupThreads), 0, s, a);
    LAUNCH_CHECK();
    a.tokens = static_cast<const I*>(a.tokens) + most;
    a.y = static_cast<T*>(a.y) + most * a.ldy;
  }
  return NGSGD_OK;
}

// How a gradient is computed: all by sizes, so that a workspace for more tokens serves fewer.
constexpr int64_t kSortTile = kSortThreads * kSortRounds;
constexpr int64_t kSumWaves = 4096;        // wavefronts that the sums are cut into, if there are as many
constexpr int64_t kFewGroups = 4096;       // workgroups that walk over a table
constexpr int kLeastChunk = 16, kMostChunk = 512;

struct BackwardPlan {
  int e, pieces, lanes, slabs, chunk;
  int64_t chunks, most_chunks;             // most_chunks: of N tokens or fewer
};
BackwardPlan backward_plan(const int64_t N, const int D, const int element_bytes) {
  BackwardPlan p;
  p.e = D >= 16 / element_bytes ? 16 / element_bytes : 1;
  p.pieces = (D + p.e - 1) / p.e;
  for (p.lanes = 1; p.lanes < p.pieces && p.lanes < 64; p.lanes *= 2) {
  }
  p.slabs = (p.pieces + 63) / 64;
  const int64_t units = std::max<int64_t>(1, kSumWaves * (64 / p.lanes) / p.slabs);   // chunks that fill the chip
  for (p.chunk = kLeastChunk; p.chunk < kMostChunk && (N + p.chunk - 1) / p.chunk > units; p.chunk *= 2) {
  }
  p.chunks = (N + p.chunk - 1) / p.chunk;
  p.most_chunks = std::max(std::min((N + kLeastChunk - 1) / kLeastChunk, units), (N + kMostChunk - 1) / kMostChunk);
  return p;
}

struct Workspace {
  SortedToken *sorted, *other;
  uint32_t *counts, *totals;
  float* parts;
};
Workspace layout(Carver& c, const int64_t N, const int D) {
  Workspace w{};
  size_t floats = 0;                       // of any type
  for (const int bytes : {2, 4}) {
    const BackwardPlan p = backward_plan(N, D, bytes);
    floats = std::max(floats, (size_t)p.most_chunks * 2 * p.pieces * p.e);
  }
  w.sorted = c.take<SortedToken>(N);
  w.parts = c.take<float>(floats);
  if (N > kRankMost) w.other = c.take<SortedToken>(N);
  if (N > kMergeMost) {
    w.counts = c.take<uint32_t>((N + kSortTile - 1) / kSortTile * kSortBins);
    w.totals = c.take<uint32_t>(kSortBins);
  }
  return w;
}

template <typename I, bool FIRST>
int sort_pass(const EmbeddingSort& a, hipStream_t s) {
  hipLaunchKernelGGL((embedding_count_kernel<I, FIRST>), dim3((unsigned)a.tiles), dim3(kSortThreads), 0, s, a);
  LAUNCH_CHECK();
  if (a.totals != nullptr) {
    hipLaunchKernelGGL(embedding_scan_kernel, dim3((unsigned)((a.bins + 63) / 64)), dim3(1024), 0, s, a);
    LAUNCH_CHECK();
  }
  hipLaunchKernelGGL((embedding_scatter_kernel<I, FIRST>), dim3((unsigned)a.tiles), dim3(kSortThreads), 0, s, a);
  LAUNCH_CHECK();
  return NGSGD_OK;
}

template <typename I>
int sort_tokens(const void* tokens, const int64_t N, const int64_t V, const Workspace& w, hipStream_t s) {
  if (N <= kMergeMost) {
    const dim3 grid((unsigned)((N + 63) / 64)), threads(kRankThreads);
    if (N <= kRankMost) {
      hipLaunchKernelGGL((embedding_rank_kernel<I, false>), grid, threads, 0, s, static_cast<const I*>(tokens), (int)N, V, w.sorted);
      LAUNCH_CHECK();
      return NGSGD_OK;
    }
    hipLaunchKernelGGL((embedding_rank_kernel<I, true>), grid, threads, 0, s, static_cast<const I*>(tokens), (int)N, V, w.other);
    LAUNCH_CHECK();
    hipLaunchKernelGGL(embedding_merge_kernel, grid, threads, 0, s, w.other, (int)N, w.sorted);
    LAUNCH_CHECK();
    return NGSGD_OK;
  }
  int bits = 1;                            // of the keys 0 .. V
  while ((int64_t)1 << bits <= V) ++bits;
  const int passes = (bits + kSortBits - 1) / kSortBits, digit = std::max(2, (bits + passes - 1) / passes);
  EmbeddingSort a{tokens, nullptr, nullptr, N, V, w.counts, nullptr, (int)((N + kSortTile - 1) / kSortTile), 0, 1 << digit};
  if (a.tiles > kSortInline) a.totals = w.totals;
  for (int pass = 0; pass < passes; ++pass, a.shift += digit) {
    a.out = (passes - pass) % 2 == 1 ? w.sorted : w.other;   // the last one's
    if (pass == 0)
      NG_TRY((sort_pass<I, true>(a, s)));
    else
      NG_TRY((sort_pass<I, false>(a, s)));
    a.in = a.out;
  }
  return NGSGD_OK;
}

template <typename T, typename W, int E>
int launch_sums(const EmbeddingBackward& a, const unsigned grid, hipStream_t s) {
  if (grid == 0) return NGSGD_OK;
  if (a.lanes == 64)
    hipLaunchKernelGGL((embedding_sum_kernel<T, W, E, true>), dim3(grid), dim3(kSumThreads), 0, s, a);
  else
    hipLaunchKernelGGL((embedding_sum_kernel<T, W, E, false>), dim3(grid), dim3(kSumThreads), 0, s, a);
  LAUNCH_CHECK();
  if (a.chunks > 1) {
    hipLaunchKernelGGL((embedding_join_kernel<W, E>), dim3((unsigned)(a.chunks * a.slabs)), dim3(kJoinThreads), 0, s, a);
    LAUNCH_CHECK();
  }
  return NGSGD_OK;
}

template <typename T, typename W, typename I, int E>
int launch_few(const EmbeddingBackward& a, hipStream_t s) {
  const int64_t groups = std::min<int64_t>((a.V * a.slabs + kSumThreads / 64 - 1) / (kSumThreads / 64), kFewGroups);
  hipLaunchKernelGGL((embedding_few_kernel<T, W, I, E>), dim3((unsigned)groups), dim3(kSumThreads), 0, s, a);
  LAUNCH_CHECK();
  return NGSGD_OK;
}

}  // namespace

extern "C" int ngsgd_embedding_forward(const void* dev_tokens, int32_t index_type, int64_t N, const void* dev_table, int64_t ldt, int32_t table_type,
                                       int64_t V, int32_t D, float scale, void* dev_y, int64_t ldy, int32_t type, void* hip_stream) {
  NG_TRY(check_types(index_type, table_type, type, N, V, D));
  if (!std::isfinite(scale)) return NGSGD_EINVAL;
  if (N == 0) return NGSGD_OK;
  if (dev_tokens == nullptr || !on_index(dev_tokens, index_type)) return NGSGD_EINVAL;
  if (!good_matrix(dev_table, ldt, table_type, V, D) || !good_matrix(dev_y, ldy, type, N, D)) return NGSGD_EINVAL;
  const EmbeddingForward a{dev_tokens, N, dev_table, ldt, V, D, scale, dev_y, ldy, 1, 0, 1};
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  return with_types(type, table_type, index_type, [&](auto t, auto w, auto i) {
    using T = decltype(t);
    constexpr int E = 16 / sizeof(T);
    return a.D >= E ? launch_forward<decltype(w), T, decltype(i), E>(a, s) : launch_forward<decltype(w), T, decltype(i), 1>(a, s);
  });
}

extern "C" int ngsgd_embedding_workspace_bytes(int64_t max_tokens, int64_t V, int32_t D, size_t* out_bytes) {
  if (out_bytes == nullptr || max_tokens < 0 || max_tokens > kMostRows || V < 1 || V > kMostRows || D < 1 || D > kMostColumns) return NGSGD_EINVAL;
  Carver c(nullptr);
  (void)layout(c, max_tokens, D);
  *out_bytes = align_up(std::max<size_t>(c.off, 1), 256);
  return NGSGD_OK;
}

extern "C" int ngsgd_embedding_backward(const void* dev_dy, int64_t lddy, int32_t type, const void* dev_tokens, int32_t index_type, int64_t N,
                                        int64_t V, int32_t D, float scale, void* dev_dtable, int64_t lddt, int32_t table_type, int32_t accumulate,
                                        void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
  NG_TRY(check_types(index_type, table_type, type, N, V, D));
  if (!std::isfinite(scale) || (accumulate != 0 && accumulate != 1)) return NGSGD_EINVAL;
  if (N > 0 && (dev_tokens == nullptr || !on_index(dev_tokens, index_type))) return NGSGD_EINVAL;
  if (!good_matrix(dev_dy, lddy, type, N, D) || !good_matrix(dev_dtable, lddt, table_type, V, D)) return NGSGD_EINVAL;
  size_t need = 0;
  NG_TRY(ngsgd_embedding_workspace_bytes(N, V, D, &need));
  NG_TRY(check_workspace(dev_workspace, workspace_bytes, need));
  const BackwardPlan p = backward_plan(N, D, type_bytes(type));
  if (p.chunks * p.slabs >= (int64_t)1 << 23) return NGSGD_EINVAL;   // a launch has less than 2^32 threads (no memory holds such rows)
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  EmbeddingBackward a{dev_dy, lddy, dev_tokens, N, V, D, scale, dev_dtable, lddt, accumulate, nullptr, nullptr, p.chunk, p.chunks, p.pieces, p.lanes, p.slabs, 0, 1};
  if (N > 0 && N <= kFewTokens)
    return with_types(type, table_type, index_type, [&](auto t, auto wt, auto i) {
      using T = decltype(t);
      using W = decltype(wt);
      using I = decltype(i);
      return p.e == 1 ? launch_few<T, W, I, 1>(a, s) : launch_few<T, W, I, 16 / sizeof(T)>(a, s);
    });
  Carver c(dev_workspace);
  const Workspace w = layout(c, N, D);
  if (N > 0) NG_TRY(index_type == NGSGD_INT32 ? sort_tokens<int32_t>(dev_tokens, N, V, w, s) : sort_tokens<int64_t>(dev_tokens, N, V, w, s));
  a.sorted = w.sorted;
  a.parts = w.parts;
  a.sum_groups = (unsigned)((p.chunks * p.slabs * p.lanes + kSumThreads - 1) / kSumThreads);
  while (a.clear_rows < 64 && a.clear_rows * 8192ll < V) a.clear_rows *= 2;
  const int64_t clear_waves = accumulate ? 0 : (V + a.clear_rows - 1) / a.clear_rows;
  const unsigned grid = a.sum_groups + (unsigned)((clear_waves + kSumThreads / 64 - 1) / (kSumThreads / 64));
  return with_types(type, table_type, NGSGD_INT32, [&](auto t, auto wt, auto) {
    using T = decltype(t);
    using W = decltype(wt);
    return p.e == 1 ? launch_sums<T, W, 1>(a, grid, s) : launch_sums<T, W, 16 / sizeof(T)>(a, grid, s);
  });
}
