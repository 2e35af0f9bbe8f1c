// Paged cache: launch parameter blocks and what its kernels share (no entry points here).
#pragma once
#include "common.h"

namespace spiffy {

constexpr int kLayersPerLaunch = 64;      // layer pointers travel as kernel arguments (4 KB at most)

struct PagedView {
  int n_pages, page_size, n_seqs, max_pages;
  int32_t *refs, *table, *len;
};

struct PageLayers {
  int n;
  void *k[kLayersPerLaunch], *v[kLayersPerLaunch], *summary[kLayersPerLaunch];
};
struct RowLayers {
  const void *k[kLayersPerLaunch], *v[kLayersPerLaunch];
};

struct Heads {
  int Hq, Hkv, hd, f32;
};

// New rows of all sequences, and the masks that say what they attend to
struct NewRows {
  const int32_t* start;     // [n_seqs + 1]
  int T;
  const uint64_t* mask;     // [T][words], NULL = all
  int words;
};

// Scratch of the page operations: page ids, a page -> page map, and per sequence or pair what the first kernel decided
struct PagesWs {
  int32_t *ids, *ids2, *map, *item_a, *item_b, *count;
};

struct PagesArgs {
  PagedView c;
  Heads h;
  PagesWs ws;
  PageLayers layers;
  // append
  NewRows rows;
  RowLayers row_layers;
  long long row_stride;
  const int32_t* node;
  int node_stride;
  // fork, free
  const int32_t *src, *dst;
  int n;
  int32_t* status;      // or n_used of a compaction
};
size_t pages_workspace_bytes(const PagedView& c);
PagesWs carve_pages(const PagedView& c, void* base);
hipError_t launch_append_plan(const PagesArgs& a, hipStream_t st);
hipError_t launch_append_rows(const PagesArgs& a, hipStream_t st);
hipError_t launch_fork_plan(const PagesArgs& a, hipStream_t st);
hipError_t launch_fork_rows(const PagesArgs& a, bool first, hipStream_t st);
hipError_t launch_free(const PagesArgs& a, hipStream_t st);
hipError_t launch_compact_plan(const PagesArgs& a, hipStream_t st);
hipError_t launch_compact_rows(const PagesArgs& a, bool first, hipStream_t st);

struct SummaryArgs {
  PagedView c;
  Heads h;
  PageLayers layers;
  const int32_t* start;     // [n_seqs] or NULL
};
hipError_t launch_page_summary(const SummaryArgs& a, hipStream_t st);

struct SelectArgs {
  PagedView c;
  Heads h;
  const void *summary, *q;
  long long q_stride;
  NewRows rows;
  int max_rows, n_sel, keep_first, keep_last;
  int32_t* selected;
  double* scores;           // [n_seqs][Hkv][max_pages], and more behind
};
size_t page_select_workspace_bytes(const PagedView& c, const Heads& h);
hipError_t launch_page_select(const SelectArgs& a, hipStream_t st);

struct TreeAttnArgs {
  PagedView c;
  Heads h;
  const void *pk, *pv;      // pool of the layer
  const void *q, *k, *v;
  long long q_stride, kv_stride, out_stride;
  NewRows rows;
  int max_rows;
  const int32_t* selected;  // [n_seqs][Hkv][n_sel] or NULL
  int n_sel;
  float scale;
  void *out, *workspace;
};
bool tree_attn_fits(const PagedView& c, const Heads& h, int max_rows);      // its workgroups
size_t tree_attn_workspace_bytes(const PagedView& c, const Heads& h, int max_rows);
hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t st);

// ---- device -----------------------------------------------------------------------------------------------------------------

// Row of the pool of row `off` of a (page, kv head), these numbered page by page.  Pages may have 2^31 - 1 rows: 64 bits, like what a row
// is multiplied by.
__host__ __device__ __forceinline__ long long pool_row(unsigned head_of_page, int page_size, int off) {
  return (long long)((unsigned long long)head_of_page * (unsigned)page_size + (unsigned)off);
}
// Pieces at, at + step, .. of the first n of each kv head's `stride` pieces of a page, counted head by head: a page can hold 2^31 pieces and
// more, and no piece costs a division.  0 <= at < step <= 1024, n >= 1.
struct HeadPieces {
  long long n, stride;
  long long place, in_head;             // place of the present piece in the page, and in its head
  int heads, rest;                      // what a step is: whole heads, and pieces
  __host__ __device__ __forceinline__ HeadPieces(long long n, long long stride, int at, int step) : n(n), stride(stride) {
    const int m = n > 1024 ? 1025 : (int)n;
    heads = step / m;
    rest = step - heads * m;
    in_head = at - at / m * m;
    place = at / m * stride + in_head;
  }
  __host__ __device__ __forceinline__ void next() {
    in_head += rest;
    place += heads * stride + rest;
    if (in_head >= n) in_head -= n, place += stride - n;
  }
};
__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
__device__ __forceinline__ int seq_len(const PagedView& c, int s) {
  return clamp_int(c.len[s], 0, c.max_pages * c.page_size);      // below 2^31: checked on the host
}
__device__ __forceinline__ int pages_of(int rows, int page_size) { return (int)(((unsigned)rows + page_size - 1) / page_size); }

struct RowRange {
  int first, n;
};
__device__ __forceinline__ RowRange rows_of(const NewRows& r, int s) {
  const int a = clamp_int(r.start[s], 0, r.T), b = clamp_int(r.start[s + 1], a, r.T);
  return RowRange{a, b - a};
}
// Sequence of new row t: the first that ends behind it (n_seqs: none).  All lanes of the wavefront call it with the same t.
__device__ __forceinline__ int seq_of_row(const NewRows& r, int n_seqs, int t) {
  for (int b = 0; b < n_seqs; b += kWave) {
    const int i = b + (int)(threadIdx.x & 63);
    const unsigned long long behind = __ballot(i < n_seqs && r.start[i + 1] > t);
    if (behind) return b + __ffsll(behind) - 1;
  }
  return n_seqs;
}

// Exclusive sum over the workgroup's threads, in thread order; `total` for all.  `tmp` holds blockDim / 64 ints in LDS; every thread
// calls it, and it may be called again at once.
__device__ __forceinline__ int block_scan(int x, int* tmp, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = (blockDim.x + 63) >> 6;
  int v = x;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int u = __shfl_up(v, o, kWave);
    if (lane >= o) v += u;
  }
  if (lane == kWave - 1) tmp[wave] = v;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < n_waves; ++w) {
    const int t = tmp[w];
    if (w < wave) before += t;
    all += t;
  }
  __syncthreads();
  total = all;
  return before + v - x;
}

}  // namespace spiffy
