// Which pages a query reads: summaries of the pages' keys, bounds on the scores they can give, and the pages of the highest bounds.
//
// For channel bounds lo <= k <= hi of a page, q . k <= sum_c max(q_c lo_c, q_c hi_c) for each of its keys, and max(q lo, q hi) is q hi
// where q > 0 and q lo elsewhere.
#include "paged.h"

namespace spiffy {

namespace {

template <typename T> struct Piece;       // 16 bytes of a row
template <> struct Piece<float> { typedef f32x4 type; static constexpr int n = 4; };
template <> struct Piece<bf16_t> { typedef bf16x8 type; static constexpr int n = 8; };

constexpr int kSeqChunk = SPIFFY_MAX_SEQS / 256;

// A wavefront a (page, kv head, layer): 64 / (16-byte pieces of a row) rows at a time, the row groups joined at the end.
template <typename T>
__global__ __launch_bounds__(256) void page_summary_kernel(const SummaryArgs a) {
  __shared__ int first[SPIFFY_MAX_SEQS + 1];       // pages to do in front of each sequence
  __shared__ int tmp[4];
  typedef typename Piece<T>::type piece_t;
  constexpr int N = Piece<T>::n;
  const PagedView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, ps = c.page_size;
  int run = 0;
  for (int b = 0; b < c.n_seqs; b += 256) {
    const int s = b + tid;
    int n = 0;
    if (s < c.n_seqs) {
      const int len = seq_len(c, s), start = a.start ? clamp_int(a.start[s], 0, len) : 0;
      n = start < len ? pages_of(len, ps) - start / ps : 0;
    }
    int sum;
    const int at = run + block_scan(n, tmp, sum);
    if (s < c.n_seqs) first[s] = at;
    run += sum;
  }
  if (tid == 0) first[c.n_seqs] = run;
  __syncthreads();
  const int pieces = a.h.hd / N, groups = kWave / pieces, grp = lane / pieces, pc = lane - grp * pieces;
  const long long jobs = (long long)run * a.h.Hkv * a.layers.n, step = (long long)gridDim.x * 4;
  for (long long j = (long long)blockIdx.x * 4 + (tid >> 6); j < jobs; j += step) {
    const int h = (int)(j % a.h.Hkv);
    const int i = (int)(j / a.h.Hkv % run), layer = (int)(j / a.h.Hkv / run);
    int lo = 0, hi = c.n_seqs;                     // the last sequence whose pages start at or before i
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= i) lo = mid; else hi = mid;
    }
    const int s = lo, len = seq_len(c, s);
    const int slot = pages_of(len, ps) - (first[s + 1] - i);
    const int page = c.table[(long long)s * c.max_pages + slot];
    if (page < 0 || page >= c.n_pages) continue;
    const int rows = min(ps, len - slot * ps);
    const T* k = reinterpret_cast<const T*>(a.layers.k[layer]) + ((long long)page * a.h.Hkv + h) * ps * a.h.hd;
    float least[N], most[N];
#pragma unroll
    for (int e = 0; e < N; ++e) least[e] = INFINITY, most[e] = -INFINITY;
    if (grp < groups) {
#pragma unroll 8
      for (int r = grp; r < rows; r += groups) {
        const piece_t x = *reinterpret_cast<const piece_t*>(k + (long long)r * a.h.hd + pc * N);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          least[e] = fminf(least[e], (float)x[e]);
          most[e] = fmaxf(most[e], (float)x[e]);
        }
      }
    }
    for (int g = 1; g < groups; ++g) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        least[e] = fminf(least[e], __shfl(least[e], (pc + g * pieces) & 63, kWave));
        most[e] = fmaxf(most[e], __shfl(most[e], (pc + g * pieces) & 63, kWave));
      }
    }
    if (grp == 0) {
      T* out = reinterpret_cast<T*>(a.layers.summary[layer]) + ((long long)page * a.h.Hkv + h) * 2 * a.h.hd + pc * N;
      piece_t x, y;
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = (T)least[e], y[e] = (T)most[e];
      *reinterpret_cast<piece_t*>(out) = x;
      *reinterpret_cast<piece_t*>(out + a.h.hd) = y;
    }
  }
}

// Scores of 64 pages (a lane each) of one (sequence, kv head); the four wavefronts share the rows.  Sums are fp64.
template <typename T>
__global__ __launch_bounds__(256) void page_score_kernel(const SelectArgs a) {
  __shared__ double best[4][kWave];
  const PagedView& c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = a.h.Hq / a.h.Hkv, hd = a.h.hd;
  const int kvh = blockIdx.y, s = blockIdx.z, slot = blockIdx.x * kWave + lane;
  const int used = pages_of(seq_len(c, s), c.page_size);
  if ((int)blockIdx.x * kWave >= used) return;
  const RowRange r = rows_of(a.rows, s);
  const int n = (r.n < a.max_rows ? r.n : a.max_rows) * g;
  const int page = slot < used ? c.table[(long long)s * c.max_pages + slot] : -1;
  const bool there = page >= 0 && page < c.n_pages;
  const T* sum = reinterpret_cast<const T*>(a.summary) + ((long long)(there ? page : 0) * a.h.Hkv + kvh) * 2 * hd;
  double top = -INFINITY;
  for (int i = wave; i < n; i += 4) {
    const T* q = reinterpret_cast<const T*>(a.q) + (r.first + i / g) * a.q_stride + (kvh * g + i % g) * hd;
    double x = 0;
    for (int ch = 0; ch < hd; ++ch) {
      const float v = to_f32(q[ch]);
      x += (double)v * (double)to_f32(sum[(v > 0.f ? hd : 0) + ch]);
    }
    top = x > top ? x : top;
  }
  best[wave][lane] = top;
  __syncthreads();
  if (wave == 0 && slot < used) {
#pragma unroll
    for (int w = 1; w < 4; ++w) top = best[w][lane] > top ? best[w][lane] : top;
    if (!there) top = -INFINITY;
    if (slot < a.keep_first || slot >= used - a.keep_last) top = INFINITY;
    a.scores[((long long)s * a.h.Hkv + kvh) * c.max_pages + slot] = top;
  }
}

// Order of doubles as order of unsigned integers
__device__ __forceinline__ unsigned long long order_of(double x) {
  const unsigned long long b = __double_as_longlong(x + 0.0);       // -0 counts as 0
  return b >> 63 ? ~b : b | 1ull << 63;
}

// One workgroup a (sequence, kv head): the n_sel-th highest score digit by digit (8 bits a pass), then the pages above it and the first
// ones equal to it in ascending order.
constexpr int kPickThreads = 512;
__global__ __launch_bounds__(kPickThreads) void page_pick_kernel(const SelectArgs a) {
  __shared__ int hist[256], tmp[kPickThreads / 64];
  __shared__ int s_digit, s_left;
  const PagedView& c = a.c;
  const int tid = threadIdx.x, kvh = blockIdx.x, s = blockIdx.y;
  const int used = pages_of(seq_len(c, s), c.page_size);
  const long long list = (long long)s * a.h.Hkv + kvh;
  const double* score = a.scores + list * c.max_pages;
  int32_t* out = a.selected + list * a.n_sel;
  const int n = a.n_sel < used ? a.n_sel : used;
  unsigned long long prefix = 0, known = 0;        // the digits found so far, and which bits they are
  int left = n;                                    // pages still to find among those with these digits
  if (n < used) {
    for (int shift = 56; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int j = tid; j < used; j += kPickThreads) {
        const unsigned long long o = order_of(score[j]);
        if ((o & known) == prefix) atomicAdd(&hist[o >> shift & 255], 1);
      }
      __syncthreads();
      int total;
      const int mine = tid < 256 ? hist[255 - tid] : 0;             // the highest digit first
      const int before = block_scan(mine, tmp, total);
      if (tid < 256 && before < left && left <= before + mine) s_digit = 255 - tid, s_left = left - before;
      __syncthreads();
      prefix |= (unsigned long long)s_digit << shift;
      known |= 255ull << shift;
      left = s_left;
    }
  }
  int done = 0, ties = 0;
  for (int b = 0; b < used && n; b += kPickThreads) {
    const int j = b + tid;
    const unsigned long long o = j < used ? order_of(score[j]) : 0;
    const bool more = j < used && (n == used || o > prefix), tie = j < used && n < used && o == prefix;
    int t_all, all;
    const int t = ties + block_scan(tie, tmp, t_all);
    const bool take = more || (tie && t < left);
    const int at = done + block_scan(take, tmp, all);
    if (take && at < n) out[at] = j;
    ties += t_all;
    done += all;
  }
  for (int j = n + tid; j < a.n_sel; j += kPickThreads) out[j] = -1;
}

}  // namespace

hipError_t launch_page_summary(const SummaryArgs& a, hipStream_t st) {
  const int grid = 2048;
  if (a.h.f32) page_summary_kernel<float><<<grid, 256, 0, st>>>(a);
  else page_summary_kernel<bf16_t><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

size_t page_select_workspace_bytes(const PagedView& c, const Heads& h) {
  return sizeof(double) * (size_t)c.n_seqs * h.Hkv * c.max_pages;
}
hipError_t launch_page_select(const SelectArgs& a, hipStream_t st) {
  const dim3 grid(cdiv(a.c.max_pages, kWave), a.h.Hkv, a.c.n_seqs);
  if (a.h.f32) page_score_kernel<float><<<grid, 256, 0, st>>>(a);
  else page_score_kernel<bf16_t><<<grid, 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  page_pick_kernel<<<dim3(a.h.Hkv, a.c.n_seqs), kPickThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace spiffy
