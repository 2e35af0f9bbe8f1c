// Which pages a query reads: summaries of the pages' keys, bounds on the scores they can give, and the pages of the highest bounds.
//
// For channel bounds lo <= k <= hi of a page, q . k <= sum_c max(q_c lo_c, q_c hi_c) for each of its keys, and max(q lo, q hi) is q hi
// where q > 0 and q lo elsewhere.
#include <cfloat>

#include "paged.h"

namespace spiffy {

namespace {

template <typename T> struct Piece;       // 16 bytes of a row
template <> struct Piece<float> { typedef f32x4 type; static constexpr int n = 4; };
template <> struct Piece<bf16_t> { typedef bf16x8 type; static constexpr int n = 8; };

// A wavefront a (page, kv head, layer): 64 / (16-byte pieces of a row) rows at a time, the row groups joined at the end.  Bound by memory: 106696
// rows of 8 kv heads of 128 in two layers, 451 MB, 89 us (5.1 TB/s).
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

typedef double f64x4 __attribute__((ext_vector_type(4)));

// Scores of 16 pages of one (sequence, kv head) a wavefront or `share` of them (1, 2 or 4, which divide the row tiles of 16 among
// themselves), on fp64 matrix instructions: with q+ = max(q, 0) and q- = min(q, 0) a bound is q+ . hi + q- . lo.  Operand A is 16 rows
// by 4 channels, B 4 channels by 16 pages; group grp of 16 lanes takes the 16-byte pieces 4 i + grp of a row, element e of all
// four at once, so no operand needs another lane's data.  Which accumulator is which row does not matter: only the maximum over
// the rows is wanted, and rows beyond the last repeat it.  0 * inf is not what the bound means, and shows as NaN: then the 16
// pages are scored element by element instead.
// Trees of 6 to 16 tokens, 32 heads over 8, 4693 pages: 837 us in fp64 vector code, 55 with four row tiles a wavefront one after the other, 41
// with a wavefront a row tile and the next pieces in flight; the matrix instructions alone are 16 us.
template <typename T>
__global__ __launch_bounds__(256) void page_score_kernel(const SelectArgs a, int share) {
  typedef typename Piece<T>::type piece_t;
  constexpr int N = Piece<T>::n;
  __shared__ double s_top[4][16];
  const PagedView& c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, grp = lane >> 4, g = a.h.Hq / a.h.Hkv, hd = a.h.hd;
  const int kvh = blockIdx.y, s = blockIdx.z, part = wave % share, slot = (blockIdx.x * (4 / share) + wave / share) * 16 + l16;
  const int used = pages_of(seq_len(c, s), c.page_size);
  if ((int)(blockIdx.x * (4 / share)) * 16 >= used) return;      // the whole workgroup
  const RowRange r = rows_of(a.rows, s);
  const int R = (r.n < a.max_rows ? r.n : a.max_rows) * g;
  const int page = slot < used ? c.table[(long long)s * c.max_pages + slot] : -1;
  const bool there = page >= 0 && page < c.n_pages;
  const T* lo = reinterpret_cast<const T*>(a.summary) + ((long long)(there ? page : 0) * a.h.Hkv + kvh) * 2 * hd;
  auto row = [&](int i) {
    return reinterpret_cast<const T*>(a.q) + (long long)(r.first + i / g) * a.q_stride + (kvh * g + i % g) * hd;
  };
  double top = -INFINITY;
  bool odd = false;
  for (int r0 = 16 * part; r0 < R && !odd; r0 += 16 * share) {
    f64x4 x = {0., 0., 0., 0.}, y = {0., 0., 0., 0.};      // two sums: an instruction need not wait for the one before it
    const T* q = row(min(r0 + l16, R - 1));
    struct Pieces {
      piece_t least, most, row;
    };
    auto load = [&](int i) {
      const int ch = (4 * i + grp) * N;
      return ch < hd ? Pieces{*reinterpret_cast<const piece_t*>(lo + ch), *reinterpret_cast<const piece_t*>(lo + hd + ch), *reinterpret_cast<const piece_t*>(q + ch)}
                     : Pieces{};
    };
    Pieces next = load(0);
    for (int i = 0; 4 * N * i < hd; ++i) {
      const Pieces p = next;
      next = load(i + 1);                                  // behind the last channel: zeros
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float l = to_f32((T)p.least[e]), m = to_f32((T)p.most[e]), v = to_f32((T)p.row[e]);
        const bool up = v > 0.f;                           // NaN goes with the negative ones and makes the row's score NaN
        x = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(up ? v : 0.f), (double)m, x, 0, 0, 0);
        y = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(up ? 0.f : v), (double)l, y, 0, 0, 0);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= there && (x[e] != x[e] || y[e] != y[e]);
    odd = __any(odd);
#pragma unroll
    for (int e = 0; e < 4; ++e) top = x[e] + y[e] > top ? x[e] + y[e] : top;
  }
  if (odd) {                                               // the same rows, shared by the four groups
    top = -INFINITY;
    for (int i = 16 * part + grp; i < R; i += (i & 15) < 12 ? 4 : 16 * share - 12) {
      const T* q = row(i);
      double x = 0;
      for (int ch = 0; ch < hd; ++ch) {
        const float v = to_f32(q[ch]);
        x += (double)v * (double)to_f32(lo[(v > 0.f ? hd : 0) + ch]);
      }
      top = x > top ? x : top;
    }
  }
#pragma unroll
  for (int o = 16; o < kWave; o <<= 1) {
    const double y = __shfl_xor(top, o, kWave);
    top = y > top ? y : top;
  }
  if (share > 1) {
    if (grp == 0) s_top[wave][l16] = top;
    __syncthreads();
    if (part) return;
    for (int w = 1; w < share; ++w) top = s_top[wave + w][l16] > top ? s_top[wave + w][l16] : top;
  }
  top = there ? fmin(top, DBL_MAX) : -INFINITY;           // an infinite bound stays below the pages that are always taken
  if (slot < a.keep_first || slot >= used - a.keep_last) top = INFINITY;
  if (grp == 0 && slot < used) a.scores[((long long)s * a.h.Hkv + kvh) * c.max_pages + slot] = top;
}

// Order of doubles as order of unsigned integers
__device__ __forceinline__ unsigned long long order_of(double x) {
  const unsigned long long b = __double_as_longlong(x + 0.0);       // -0 counts as 0
  return b >> 63 ? ~b : b | 1ull << 63;
}

// One workgroup a (sequence, kv head): the n_sel-th highest score is found digit by digit, 12 bits a pass, until a digit's pages are all
// taken; the first digit is sign and exponent, the second already tells a few hundred pages apart, so it takes two or three
// passes (9 us at 521 pages; 8-bit digits, all eight of them, 12, counting every page against all others in LDS 25).  Then the
// pages above and the first ones equal to it are written in ascending order.  Up to kKeep pages a thread the scores stay in registers.
constexpr int kPickThreads = 512, kDigit = 12, kBins = 1 << kDigit, kKeep = 8;
__global__ __launch_bounds__(kPickThreads) void page_pick_kernel(const SelectArgs a) {
  __shared__ __align__(16) int hist[kBins];
  __shared__ int tmp[kPickThreads / 64];
  __shared__ int s_digit, s_left, s_here;
  const PagedView& c = a.c;
  const int tid = threadIdx.x, kvh = blockIdx.x, s = blockIdx.y;
  const int used = pages_of(seq_len(c, s), c.page_size);
  const long long list = (long long)s * a.h.Hkv + kvh;
  const double* score = a.scores + list * c.max_pages;
  int32_t* out = a.selected + list * a.n_sel;
  const int n = a.n_sel < used ? a.n_sel : used;
  for (int j = n + tid; j < a.n_sel; j += kPickThreads) out[j] = -1;
  if (n == used) {
    for (int j = tid; j < used; j += kPickThreads) out[j] = j;
    return;
  }
  unsigned long long kept[kKeep];
#pragma unroll
  for (int i = 0; i < kKeep; ++i) kept[i] = tid + i * kPickThreads < used ? order_of(score[tid + i * kPickThreads]) : 0;
  const int rounds = (used + kPickThreads - 1) / kPickThreads;
  unsigned long long prefix = 0, known = 0;        // the digits found so far, and which bits they are
  int left = n;                                    // pages still to find among those with these digits
  for (int shift = 64 - kDigit; ; shift = shift > kDigit ? shift - kDigit : 0) {
    const unsigned long long digit = (kBins - 1ull) & ~(known >> shift);      // the last one is shorter
#pragma unroll
    for (int i = 0; i < kBins / kPickThreads; ++i) hist[tid + i * kPickThreads] = 0;
    __syncthreads();
    auto count = [&](int j, unsigned long long o) {
      if (j < used && (o & known) == prefix) atomicAdd(&hist[o >> shift & digit], 1);
    };
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (i < rounds) count(tid + i * kPickThreads, kept[i]);
    for (int i = kKeep; i < rounds; ++i) {
      const int j = tid + i * kPickThreads;
      count(j, j < used ? order_of(score[j]) : 0);
    }
    __syncthreads();
    int bins[kBins / kPickThreads], mine = 0, total;               // this thread's bins, the highest first
#pragma unroll
    for (int i = 0; i < kBins / kPickThreads; ++i) mine += bins[i] = hist[kBins - 1 - (tid * (kBins / kPickThreads) + i)];
    int before = block_scan(mine, tmp, total);
#pragma unroll
    for (int i = 0; i < kBins / kPickThreads; ++i) {
      if (before < left && left <= before + bins[i])
        s_digit = kBins - 1 - (tid * (kBins / kPickThreads) + i), s_left = left - before, s_here = bins[i];
      before += bins[i];
    }
    __syncthreads();
    prefix |= (unsigned long long)s_digit << shift;
    known |= digit << shift;
    left = s_left;
    if (left == s_here || shift == 0) break;       // all that have these digits, or as many of equal ones
  }
  int done = 0, ties = 0;
  for (int i = 0; i < rounds; ++i) {
    const int j = i * kPickThreads + tid;
    unsigned long long o = j < used ? order_of(score[j]) & known : 0;
    const bool tie = j < used && o == prefix;
    int t_all, all;
    const int t = ties + block_scan(tie, tmp, t_all);
    const bool take = j < used && (o > prefix || (tie && t < left));
    const int at = done + block_scan(take, tmp, all);
    if (take && at < n) out[at] = j;
    ties += t_all;
    done += all;
  }
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
  const int tiles = cdiv(a.max_rows * (a.h.Hq / a.h.Hkv), 16), share = tiles >= 4 ? 4 : (tiles >= 2 ? 2 : 1);
  const dim3 grid(cdiv(a.c.max_pages, 16 * (4 / share)), a.h.Hkv, a.c.n_seqs);
  if (a.h.f32) page_score_kernel<float><<<grid, 256, 0, st>>>(a, share);
  else page_score_kernel<bf16_t><<<grid, 256, 0, st>>>(a, share);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  page_pick_kernel<<<dim3(a.h.Hkv, a.c.n_seqs), kPickThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace spiffy
