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
// with a wavefront a row tile and the next pieces in flight; two or four row tiles a wavefront at once, whose page bounds are converted
// once, 41 and 46: the matrix instructions are the bound.
//
// score_pages: the highest score over the row tiles part, part + share, .. of the page in table entry `slot`, a lane's (lane % 16 after
// lane % 16); all lanes of the wavefront call it.
template <typename T>
__device__ __forceinline__ double score_pages(const SelectArgs& a, int s, int kvh, int slot, int used, const RowRange& r, int part, int share) {
  typedef typename Piece<T>::type piece_t;
  constexpr int N = Piece<T>::n;
  const PagedView& c = a.c;
  const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4, g = a.h.Hq / a.h.Hkv, hd = a.h.hd;
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
  return there ? fmin(top, DBL_MAX) : -INFINITY;           // an infinite bound stays below the pages that are always taken
}
__device__ __forceinline__ bool always_taken(const SelectArgs& a, int slot, int used) { return slot < a.keep_first || slot >= used - a.keep_last; }

template <typename T>
__global__ __launch_bounds__(256) void page_score_kernel(const SelectArgs a, int share) {
  __shared__ double s_top[4][16];
  const PagedView& c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, grp = lane >> 4;
  const int kvh = blockIdx.y, s = blockIdx.z, part = wave % share, slot = (blockIdx.x * (4 / share) + wave / share) * 16 + l16;
  const int used = pages_of(seq_len(c, s), c.page_size);
  if ((int)(blockIdx.x * (4 / share)) * 16 >= used) return;      // the whole workgroup
  double top = score_pages<T>(a, s, kvh, slot, used, rows_of(a.rows, s), part, share);
  if (share > 1) {
    if (grp == 0) s_top[wave][l16] = top;
    __syncthreads();
    if (part) return;
    for (int w = 1; w < share; ++w) top = s_top[wave + w][l16] > top ? s_top[wave + w][l16] : top;
  }
  if (always_taken(a, slot, used)) top = INFINITY;
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
struct PickShared {
  alignas(16) int hist[kBins];
  int tmp[kPickThreads / 64];
  int digit, left, here;
};
// The n-th highest of keys key(0) .. key(used - 1), 0 < n < used: those whose `known` bits are above `prefix` are among the n highest, of
// those that have just these bits `left` are, the first ones; `all` of them if there are no more.
struct Cut {
  unsigned long long prefix, known;
  int left;
  bool all;
};
template <typename Key>
__device__ __forceinline__ Cut cut_at(PickShared& sh, int used, int n, Key key) {
  const int tid = threadIdx.x;
  unsigned long long kept[kKeep];
#pragma unroll
  for (int i = 0; i < kKeep; ++i) kept[i] = tid + i * kPickThreads < used ? key(tid + i * kPickThreads) : 0;
  const int rounds = (used + kPickThreads - 1) / kPickThreads;
  Cut c{0, 0, n, false};                           // the digits found so far, which bits they are, pages still to find among those with them
  for (int shift = 64 - kDigit; ; shift = shift > kDigit ? shift - kDigit : 0) {
    const unsigned long long digit = (kBins - 1ull) & ~(c.known >> shift);      // the last one is shorter
#pragma unroll
    for (int i = 0; i < kBins / kPickThreads; ++i) sh.hist[tid + i * kPickThreads] = 0;
    __syncthreads();
    auto count = [&](int j, unsigned long long o) {
      if (j < used && (o & c.known) == c.prefix) atomicAdd(&sh.hist[o >> shift & digit], 1);
    };
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (i < rounds) count(tid + i * kPickThreads, kept[i]);
    for (int i = kKeep; i < rounds; ++i) {
      const int j = tid + i * kPickThreads;
      count(j, j < used ? key(j) : 0);
    }
    __syncthreads();
    int bins[kBins / kPickThreads], mine = 0, total;               // this thread's bins, the highest first
#pragma unroll
    for (int i = 0; i < kBins / kPickThreads; ++i) mine += bins[i] = sh.hist[kBins - 1 - (tid * (kBins / kPickThreads) + i)];
    int before = block_scan(mine, sh.tmp, total);
#pragma unroll
    for (int i = 0; i < kBins / kPickThreads; ++i) {
      if (before < c.left && c.left <= before + bins[i])
        sh.digit = kBins - 1 - (tid * (kBins / kPickThreads) + i), sh.left = c.left - before, sh.here = bins[i];
      before += bins[i];
    }
    __syncthreads();
    c.prefix |= (unsigned long long)sh.digit << shift;
    c.known |= digit << shift;
    c.left = sh.left;
    c.all = c.left == sh.here;
    if (c.all || shift == 0) return c;             // all that have these digits, or as many of equal ones
  }
}
// Calls taken(j, at) for the pages of a cut, in ascending order; at counts them.  Every thread calls it, each for its own pages.
template <typename Key, typename Taken>
__device__ __forceinline__ void take_cut(PickShared& sh, const Cut& c, int used, Key key, Taken taken) {
  const int tid = threadIdx.x;
  int done = 0, ties = 0;
  for (int i = 0; i * kPickThreads < used; ++i) {
    const int j = i * kPickThreads + tid;
    const unsigned long long o = j < used ? key(j) & c.known : 0;
    const bool tie = j < used && o == c.prefix;
    int t_all, all;
    const int t = ties + block_scan(tie, sh.tmp, t_all);
    const bool take = j < used && (o > c.prefix || (tie && t < c.left));
    const int at = done + block_scan(take, sh.tmp, all);
    if (j < used) taken(j, at, take);
    ties += t_all;
    done += all;
  }
}
// The -1 behind the last page, and everything if all pages are taken
__device__ __forceinline__ bool all_taken(int32_t* out, int n, int n_sel, int used) {
  for (int j = n + (int)threadIdx.x; j < n_sel; j += kPickThreads) out[j] = -1;
  if (n < used) return false;
  for (int j = threadIdx.x; j < used; j += kPickThreads) out[j] = j;
  return true;
}

__global__ __launch_bounds__(kPickThreads) void page_pick_kernel(const SelectArgs a) {
  __shared__ PickShared sh;
  const PagedView& c = a.c;
  const int kvh = blockIdx.x, s = blockIdx.y;
  const int used = pages_of(seq_len(c, s), c.page_size);
  const long long list = (long long)s * a.h.Hkv + kvh;
  const double* score = a.scores + list * c.max_pages;
  int32_t* out = a.selected + list * a.n_sel;
  const int n = a.n_sel < used ? a.n_sel : used;
  if (all_taken(out, n, a.n_sel, used)) return;
  auto key = [&](int j) { return order_of(score[j]); };
  const Cut cut = cut_at(sh, used, n, key);
  take_cut(sh, cut, used, key, [&](int j, int at, bool take) {
    if (take && at < n) out[at] = j;
  });
}

// ---- many rows and pages in bf16: the fp64 products are the bound (16 trees of 16 tokens over 64000 rows, 32 heads over 8: 100 us at 42
// Tflop/s), and almost all pages are far from the last that is taken.  So every page first gets an interval that its score lies in, from
// bf16 matrix instructions, and only pages whose intervals leave open whether they are taken, some two or three, get exact scores.
// Trees of 6 to 16 tokens, 64 of 4693 pages: 14 us and 18 for the choice, instead of 42 and 10.
//
// A row's score and, beside it, S = q+ . |hi| + |q-| . |lo| are sums of exact products in fp32, one of a channel's two being zero.  Each of up to
// hd additions is off by at most 2^-23 of S, truncated or rounded in any order, so a sum by hd 2^-23 S at most; twice that is taken.
// With values below 2^60 what is lost where the instruction takes a subnormal number for zero is at most 2 hd 2^-126 2^60 < 2^-56.
// Pages or rows with larger values, infinities or NaN get the interval of all numbers.
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
constexpr unsigned kLarge = 127 + 60;                      // exponent field from which on a value is not summed in fp32

// A wavefront 16 pages and all row tiles; NK: steps of 32 channels.  A page's bounds stay in registers; they and the first rows are on their way
// together, other rows one tile ahead (loaded where they are used: 24 us instead of 14).
template <int NK>
__global__ __launch_bounds__(256) void page_range_kernel(const SelectArgs a) {
  const PagedView& c = a.c;
  const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4, g = a.h.Hq / a.h.Hkv, hd = a.h.hd;
  const int kvh = blockIdx.y, s = blockIdx.z, first = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 16, slot = first + l16;
  const int used = pages_of(seq_len(c, s), c.page_size);
  if (first >= used) return;                               // the wavefront
  const RowRange r = rows_of(a.rows, s);
  const int R = (r.n < a.max_rows ? r.n : a.max_rows) * g;
  const u32x4 plain = {0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
  auto abs_of = [&](u32x4 x) { return __builtin_bit_cast(bf16x8, x & plain); };
  auto large = [&](u32x4 x) {
    const i16x8 y = __builtin_bit_cast(i16x8, x & plain);
    short z = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) z = max(z, y[e]);
    return (unsigned)z >= kLarge << 7;
  };
  u32x4 row[NK], l[NK], h[NK];
  auto load_row = [&](int r0) {
    const int i = min(r0 + l16, R - 1);
    const bf16_t* q = reinterpret_cast<const bf16_t*>(a.q) + (long long)(r.first + i / g) * a.q_stride + (kvh * g + i % g) * hd;
#pragma unroll
    for (int k = 0; k < NK; ++k) row[k] = 32 * k + grp * 8 < hd ? *reinterpret_cast<const u32x4*>(q + 32 * k + grp * 8) : u32x4{};
  };
  if (R > 0) load_row(0);
  const int page = slot < used ? c.table[(long long)s * c.max_pages + slot] : -1;
  const bool there = page >= 0 && page < c.n_pages;
  const bf16_t* lo = reinterpret_cast<const bf16_t*>(a.summary) + ((long long)(there ? page : 0) * a.h.Hkv + kvh) * 2 * hd;
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    const bool in = 32 * k + grp * 8 < hd;
    l[k] = in ? *reinterpret_cast<const u32x4*>(lo + 32 * k + grp * 8) : u32x4{};
    h[k] = in ? *reinterpret_cast<const u32x4*>(lo + hd + 32 * k + grp * 8) : u32x4{};
  }
  float least = -INFINITY, most = -INFINITY;
  bool odd_page = false, odd_row = false;
#pragma unroll
  for (int k = 0; k < NK; ++k) odd_page |= large(l[k]) || large(h[k]);
  for (int r0 = 0; r0 < R; r0 += 16) {
    u32x4 q[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) q[k] = row[k];
    if (r0 + 16 < R) load_row(r0 + 16);
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      odd_row |= large(q[k]);
      // negative numbers are negative as integers too
      const u32x4 up = __builtin_bit_cast(u32x4, __builtin_elementwise_max(__builtin_bit_cast(i16x8, q[k]), i16x8{}));
      const u32x4 down = __builtin_bit_cast(u32x4, __builtin_elementwise_min(__builtin_bit_cast(i16x8, q[k]), i16x8{}));
      x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, up), __builtin_bit_cast(bf16x8, h[k]), x, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, up), abs_of(h[k]), y, 0, 0, 0);
      x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, down), __builtin_bit_cast(bf16x8, l[k]), x, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(abs_of(down), abs_of(l[k]), y, 0, 0, 0);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float off = y[e] * (hd * 0x1p-22f) + 0x1p-50f;
      least = fmaxf(least, x[e] - off);
      most = fmaxf(most, x[e] + off);
    }
  }
  // of the lanes of a page, and of all rows
#pragma unroll
  for (int o = 16; o < kWave; o <<= 1) {
    least = fmaxf(least, __shfl_xor(least, o, kWave));
    most = fmaxf(most, __shfl_xor(most, o, kWave));
    odd_page |= __shfl_xor((int)odd_page, o, kWave) != 0;
  }
  const bool odd = odd_page || __any(odd_row);
  if (odd) least = -INFINITY, most = INFINITY;
  if (!there) least = most = -INFINITY;
  if (always_taken(a, slot, used)) least = most = INFINITY;
  if (grp == 0 && slot < used) reinterpret_cast<float2*>(a.scores)[((long long)s * a.h.Hkv + kvh) * c.max_pages + slot] = make_float2(least, most);
}

// One workgroup a (sequence, kv head).  With the cut through the lower ends, H = the pages above it (and at it, if all of these are taken): at
// most n.  V = the highest upper end outside H.  A page of H whose lower end is above V is taken, for only others of H can be
// higher; one whose upper end is below the n-th highest lower end is not; the rest is decided by exact scores.  Up to kPairs
// (open page, row) go without matrix instructions (the choice takes 18 us instead of 27), up to kFew open pages are counted against one another:
// near scores share most of their digits.
constexpr int kFew = 256, kPairs = 512;
__global__ __launch_bounds__(kPickThreads) void page_choose_kernel(const SelectArgs a) {
  __shared__ PickShared sh;
  __shared__ double s_top[kPickThreads / kWave][16];
  __shared__ unsigned long long s_few[kFew];
  __shared__ int s_ids[kFew];
  __shared__ float2 s_end[kPickThreads / kWave];
  const PagedView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kvh = blockIdx.x, s = blockIdx.y;
  const int used = pages_of(seq_len(c, s), c.page_size);
  const long long list = (long long)s * a.h.Hkv + kvh, lists = (long long)c.n_seqs * a.h.Hkv;
  float2* range = reinterpret_cast<float2*>(a.scores) + list * c.max_pages;
  unsigned long long* exact = reinterpret_cast<unsigned long long*>(a.scores) + (lists + list) * c.max_pages;      // in the order of scores
  int32_t* ids = reinterpret_cast<int32_t*>(a.scores + 2 * lists * c.max_pages) + list * c.max_pages;
  int32_t* out = a.selected + list * a.n_sel;
  const int n = a.n_sel < used ? a.n_sel : used;
  if (all_taken(out, n, a.n_sel, used)) return;
  const RowRange r = rows_of(a.rows, s);
  const Cut cut = cut_at(sh, used, n, [&](int j) { return order_of(range[j].x); });
  auto high = [&](float x) {
    const unsigned long long o = order_of(x) & cut.known;
    return o > cut.prefix || (cut.all && o == cut.prefix);
  };
  float v = -INFINITY, t = INFINITY;                       // t: the n-th highest lower end
  for (int j = tid; j < used; j += kPickThreads) {
    const float2 y = range[j];
    const bool in = high(y.x);
    v = in ? v : fmaxf(v, y.y);
    t = in || order_of(y.x) == cut.prefix ? fminf(t, y.x) : t;
  }
  v = wave_max(v);
  t = -wave_max(-t);
  if (lane == 0) s_end[wave] = make_float2(v, t);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPickThreads / kWave; ++w) v = fmaxf(v, s_end[w].x), t = fminf(t, s_end[w].y);
  int sure = 0, open = 0;
  for (int b = 0; b < used; b += kPickThreads) {
    const int j = b + tid;
    const float2 y = j < used ? range[j] : make_float2(-INFINITY, -INFINITY);
    const bool is_sure = j < used && y.x > v;
    const bool is_open = j < used && !is_sure && y.y >= t;
    int both, all = is_sure + (is_open << 16);             // 512 of each at most
    const int at = block_scan(all, sh.tmp, both) >> 16;
    if (is_open) (open + at < kFew ? s_ids[open + at] : ids[open + at]) = j;
    sure += both & 0xffff;
    open += both >> 16;
  }
  __syncthreads();                                         // the list is read by others than its writers
  const int want = n - sure;
  // What was open is settled in the intervals: above all others or below.
  auto id = [&](int i) { return i < kFew ? s_ids[i] : ids[i]; };
  auto settle = [&](int i, bool take) { range[id(i)].x = take ? INFINITY : -INFINITY; };
  if (want <= 0 || want >= open || r.n == 0) {             // without new rows all scores are the same
    for (int i = tid; i < open; i += kPickThreads) settle(i, i < want);
  } else {
    const int g = a.h.Hq / a.h.Hkv, R = min(r.n, a.max_rows) * g;
    if (open <= kFew && (long long)open * R <= kPairs) {   // 16 lanes a page and row
      for (int i = tid; i < open; i += kPickThreads) s_few[i] = order_of(-INFINITY);
      __syncthreads();
      for (int i = tid >> 4; i < open * R; i += kPickThreads / 16) {
        const int at = i / R, slot = s_ids[at], page = c.table[(long long)s * c.max_pages + slot];
        const bool there = page >= 0 && page < c.n_pages;
        const bf16_t* lo = reinterpret_cast<const bf16_t*>(a.summary) + ((long long)(there ? page : 0) * a.h.Hkv + kvh) * 2 * a.h.hd;
        const int row = i - at * R;
        const bf16_t* q = reinterpret_cast<const bf16_t*>(a.q) + (long long)(r.first + row / g) * a.q_stride + (kvh * g + row % g) * a.h.hd;
        double x = 0.;
        for (int ch = (lane & 15) * 8; ch < a.h.hd; ch += 128) {
          const bf16x8 l = *reinterpret_cast<const bf16x8*>(lo + ch), h = *reinterpret_cast<const bf16x8*>(lo + a.h.hd + ch);
          const bf16x8 y = *reinterpret_cast<const bf16x8*>(q + ch);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float z = to_f32((bf16_t)y[e]);
            x += (double)z * (double)to_f32(z > 0.f ? (bf16_t)h[e] : (bf16_t)l[e]);
          }
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) x += __shfl_xor(x, o, kWave);
        x = there && x == x ? fmin(x, DBL_MAX) : -INFINITY;
        if ((lane & 15) == 0) atomicMax(&s_few[at], order_of(always_taken(a, slot, used) ? INFINITY : x));
      }
      __syncthreads();
    } else {
      const int tiles = (R + 15) / 16, share = tiles >= 8 ? 8 : (tiles >= 4 ? 4 : (tiles >= 2 ? 2 : 1));
      const int groups = kPickThreads / kWave / share, part = wave % share;
      for (int b = 0; b < open; b += 16 * groups) {
        const int i = b + wave / share * 16 + (lane & 15), slot = i < open ? id(i) : used;
        const double x = score_pages<bf16_t>(a, s, kvh, slot, used, r, part, share);
        if (lane < 16) s_top[wave][lane] = x;
        __syncthreads();
        if (part == 0 && lane < 16 && i < open) {
          double top = x;
          for (int w = 1; w < share; ++w) top = s_top[wave + w][lane] > top ? s_top[wave + w][lane] : top;
          const unsigned long long o = order_of(always_taken(a, slot, used) ? INFINITY : top);
          if (open <= kFew) s_few[i] = o;
          else exact[i] = o;
        }
        __syncthreads();
      }
    }
    if (open <= kFew) {
      for (int i = tid; i < open; i += kPickThreads) {
        int higher = 0;
        for (int k = 0; k < open; ++k) higher += s_few[k] > s_few[i] || (s_few[k] == s_few[i] && k < i);
        settle(i, higher < want);
      }
    } else {
      auto key = [&](int i) { return exact[i]; };
      const Cut last = cut_at(sh, open, want, key);
      take_cut(sh, last, open, key, [&](int i, int, bool take) { settle(i, take); });
    }
  }
  __syncthreads();
  int done = 0;
  for (int b = 0; b < used; b += kPickThreads) {
    const int j = b + tid;
    const float x = j < used ? range[j].x : -INFINITY;
    const bool take = x > v || x == INFINITY;
    int all;
    const int at = done + block_scan(take, sh.tmp, all);
    if (take && at < n) out[at] = j;
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

namespace {
// Tiles of 16 rows by 16 pages from which on bf16 pages get intervals first (choosing 8 of them, scores / intervals): 1056 tiles of one sequence 19
// / 17 us, 1024 of sixteen 19 / 20, 4096 of sixteen 27 / 21, 32768 of sixteen 70 / 39, 65536 118 / 49; 264 tiles, 32 of 521 pages, 17.5 / 18.2.
// Where pages are all alike every score has to be exact, by one workgroup a list (32 heads over 8, 16 trees, 4693 equal pages 61 / 272).
constexpr int kManyTiles = 2048;
bool by_range(const SelectArgs& a, int tiles) {
  return !a.h.f32 && (long long)a.c.n_seqs * a.h.Hkv * cdiv(a.c.max_pages, 16) * tiles >= kManyTiles;
}
}  // namespace

// scores or intervals, and for the latter exact scores of some and which pages these are
size_t page_select_workspace_bytes(const PagedView& c, const Heads& h) {
  return (size_t)c.n_seqs * h.Hkv * c.max_pages * (h.f32 ? sizeof(double) : 2 * sizeof(double) + sizeof(int32_t));
}
hipError_t launch_page_select(const SelectArgs& a, hipStream_t st) {
  const int tiles = cdiv(a.max_rows * (a.h.Hq / a.h.Hkv), 16), share = tiles >= 4 ? 4 : (tiles >= 2 ? 2 : 1);
  const dim3 lists(a.h.Hkv, a.c.n_seqs);
  hipError_t e;
  if (by_range(a, tiles)) {
    const dim3 grid(cdiv(a.c.max_pages, 64), a.h.Hkv, a.c.n_seqs);
    if (a.h.hd <= 64) page_range_kernel<2><<<grid, 256, 0, st>>>(a);
    else if (a.h.hd <= 128) page_range_kernel<4><<<grid, 256, 0, st>>>(a);
    else page_range_kernel<8><<<grid, 256, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    page_choose_kernel<<<lists, kPickThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  const dim3 grid(cdiv(a.c.max_pages, 16 * (4 / share)), a.h.Hkv, a.c.n_seqs);
  if (a.h.f32) page_score_kernel<float><<<grid, 256, 0, st>>>(a, share);
  else page_score_kernel<bf16_t><<<grid, 256, 0, st>>>(a, share);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  page_pick_kernel<<<lists, kPickThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace spiffy
