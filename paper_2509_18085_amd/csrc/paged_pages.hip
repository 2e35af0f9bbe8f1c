// Upkeep of a paged cache: append accepted rows, fork, free, compact.
//
// The reference counts are the whole state of the allocator: a page is free while its count is 0, and calls take the lowest free
// ones, so what a call does depends on the cache alone, not on the order in which anything ran.  Every call but free has two
// kernels: a plan by one workgroup (who gets which page: sums over sequences and a scan of the counts, 4 to 10 microseconds of
// latency) and the copies, which read the plan from the workspace and are bound by memory.
#include "paged.h"

namespace spiffy {

namespace {

constexpr int kPlanThreads = 512, kPlanWaves = kPlanThreads / 64;
constexpr int kScanPages = 16;                           // pages that a thread has in flight
constexpr int kSkip = -2;                                // item_b: nothing to do for this sequence or pair

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Ids p in [lo, hi) for which pred(p) holds, ascending, the first `want` of them into out (out == NULL: only counted, all).
// Returns how many; all threads of a workgroup of kPlanThreads call it.  tmp: kScanPages * kPlanWaves + kPlanWaves ints of LDS.
template <typename Pred>
__device__ int list_pages(int lo, int hi, int want, int32_t* out, int* tmp, Pred pred) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int* counts = tmp + kPlanWaves;
  int found = 0;
  for (long long base = lo; base < hi && found < want; base += kScanPages * kPlanThreads) {
    bool is[kScanPages];
#pragma unroll
    for (int u = 0; u < kScanPages; ++u) {
      const long long p = base + u * kPlanThreads + tid;
      is[u] = p < hi && pred((int)p);
    }
    unsigned long long b[kScanPages];
#pragma unroll
    for (int u = 0; u < kScanPages; ++u) {
      b[u] = __ballot(is[u]);
      if (lane == 0) counts[u * kPlanWaves + wave] = __popcll(b[u]);
    }
    __syncthreads();
    int total;
    const int mine = tid < kScanPages * kPlanWaves ? counts[tid] : 0;
    const int before = block_scan(mine, tmp, total);
    if (tid < kScanPages * kPlanWaves) counts[tid] = before;
    __syncthreads();
    if (out) {
#pragma unroll
      for (int u = 0; u < kScanPages; ++u) {
        const int at = found + counts[u * kPlanWaves + wave] + __popcll(b[u] & ((1ull << lane) - 1));
        if (is[u] && at < want) out[at] = (int)(base + u * kPlanThreads + tid);
      }
    }
    found += total;
    __syncthreads();
  }
  return found < want ? found : want;
}

// ---- append -----------------------------------------------------------------------------------------------------------------

// Whether new row i of a sequence is appended, given its node's mask row (NULL = every row)
__device__ __forceinline__ bool row_kept(const uint64_t* bits, int words, int i) {
  return !bits || (i < 64 * words && (bits[i >> 6] >> (i & 63) & 1));
}

__global__ __launch_bounds__(kPlanThreads) void append_plan_kernel(const PagesArgs a) {
  __shared__ int tmp[(kScanPages + 1) * kPlanWaves];
  __shared__ int need[SPIFFY_MAX_SEQS + 1];      // pages each sequence asks for, then where its pages start in the list
  __shared__ int s_total;
  const PagedView& c = a.c;
  const int tid = threadIdx.x, ps = c.page_size;
  long long asked = 0;
  for (int s = tid; s < c.n_seqs; s += kPlanThreads) {
    const RowRange r = rows_of(a.rows, s);
    const int len = seq_len(c, s), had = pages_of(len, ps);
    int n = r.n, status = SPIFFY_PAGES_DONE;
    if (a.node) {
      const int node = a.node[(long long)s * a.node_stride];
      n = 0;
      if (node >= r.n) status = SPIFFY_PAGES_BAD;
      else if (node >= 0) {
        const uint64_t* bits = a.rows.mask + (long long)(r.first + node) * a.rows.words;
        const int lim = r.n < 64 * a.rows.words ? r.n : 64 * a.rows.words;
        for (int w = 0; 64 * w < lim; ++w) n += __popcll(lim - 64 * w < 64 ? bits[w] & ((1ull << (lim - 64 * w)) - 1) : bits[w]);
      }
    }
    int more = 0;
    if (n > 0) {
      const int rest = len % ps;
      if (rest) {                                // the last page is written: it has to be this sequence's alone
        const int p = c.table[(long long)s * c.max_pages + had - 1];
        if (p < 0 || p >= c.n_pages || c.refs[p] != 1) status = SPIFFY_PAGES_BAD;
      }
      const long long pages = ((long long)len + n + ps - 1) / ps;
      if (status == SPIFFY_PAGES_DONE && pages > c.max_pages) status = SPIFFY_PAGES_NO_ENTRY;
      more = (int)(pages - had);
    }
    if (status != SPIFFY_PAGES_DONE) n = more = 0;
    need[s] = more;
    asked += more;
    a.ws.item_a[s] = len;
    a.ws.item_b[s] = n;
    if (a.status) a.status[s] = status;
  }
  if (tid == 0) s_total = 0;
  __syncthreads();
  // pages asked for, counted no further than n_pages + 1 (the sum of 4096 large requests passes 31 bits)
  int mine = asked > c.n_pages ? c.n_pages + 1 : (int)asked;
  for (int o = 32; o; o >>= 1) {
    const long long t = (long long)mine + __shfl_xor(mine, o, kWave);
    mine = t > c.n_pages ? c.n_pages + 1 : (int)t;
  }
  if ((tid & 63) == 0 && mine) {
    int old = s_total, seen;
    do {
      seen = old;
      const long long t = (long long)seen + mine;
      old = atomicCAS(&s_total, seen, t > c.n_pages ? c.n_pages + 1 : (int)t);
    } while (old != seen);
  }
  __syncthreads();
  const int total = s_total;
  const int have = total ? list_pages(0, c.n_pages, total < c.n_pages ? total : c.n_pages, a.ws.ids, tmp, [&](int p) { return c.refs[p] == 0; }) : 0;
  // where each sequence's pages start; with too few of them, one sequence after the other
  if (total <= have) {
    int run = 0;
    for (int b = 0; b < c.n_seqs; b += kPlanThreads) {
      const int s = b + tid;
      int sum;
      const int at = run + block_scan(s < c.n_seqs ? need[s] : 0, tmp, sum);
      if (s < c.n_seqs) need[s] = at;
      run += sum;
    }
    if (tid == 0) need[c.n_seqs] = run;
  } else if (tid == 0) {
    int run = 0;
    for (int s = 0; s < c.n_seqs; ++s) {
      const int n = need[s];
      need[s] = run;
      if (n <= have - run) run += n;
      else {
        a.ws.item_b[s] = 0;
        if (a.status) a.status[s] = SPIFFY_PAGES_NO_PAGE;
      }
    }
    need[c.n_seqs] = run;
  }
  __syncthreads();                               // also orders the workgroup's global writes of item_b and ids
  for (int i = tid; i < need[c.n_seqs]; i += kPlanThreads) {
    int lo = 0, hi = c.n_seqs;                   // the last sequence whose pages start at or before i
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (need[mid] <= i) lo = mid; else hi = mid;
    }
    const int p = a.ws.ids[i];
    c.table[(long long)lo * c.max_pages + pages_of(a.ws.item_a[lo], ps) + (i - need[lo])] = p;
    c.refs[p] = 1;
  }
  for (int s = tid; s < c.n_seqs; s += kPlanThreads) {
    const int n = a.ws.item_b[s];
    if (n > 0) c.len[s] = a.ws.item_a[s] + n;
  }
}

// A wavefront a row and `layers` layers: 16 bytes a lane, head by head into the page.  Paths of 48 trees of 12 to 40 tokens in 28 layers 11.9 us
// (15.9 with a wavefront a row and layer).
__global__ __launch_bounds__(256) void append_rows_kernel(const PagesArgs a, int layers) {
  const PagedView& c = a.c;
  const int lane = threadIdx.x & 63, ps = c.page_size;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.rows.T) return;
  const int s = seq_of_row(a.rows, c.n_seqs, t);
  if (s >= c.n_seqs) return;
  const RowRange r = rows_of(a.rows, s);
  const int i = t - r.first;
  if (i < 0 || i >= r.n || a.ws.item_b[s] <= 0) return;
  int rank = i;
  if (a.node) {
    const int node = clamp_int(a.node[(long long)s * a.node_stride], 0, r.n - 1);
    const uint64_t* bits = a.rows.mask + (long long)(r.first + node) * a.rows.words;
    if (!row_kept(bits, a.rows.words, i)) return;
    rank = 0;
    for (int w = 0; w < i >> 6; ++w) rank += __popcll(bits[w]);
    rank += __popcll(bits[i >> 6] & ((1ull << (i & 63)) - 1));
  }
  const int pos = a.ws.item_a[s] + rank, slot = pos / ps, off = pos - slot * ps;
  const int page = slot < c.max_pages ? c.table[(long long)s * c.max_pages + slot] : -1;
  if (page < 0 || page >= c.n_pages) return;
  const int es = a.h.f32 ? 4 : 2, seg = a.h.hd * es / 16;       // 16-byte pieces of a head's row
  const long long from = (long long)t * a.row_stride * es;
  const int last = min((int)(blockIdx.y + 1) * layers, a.layers.n);
  for (int x = lane; x < a.h.Hkv * seg; x += kWave) {
    const int h = x / seg;
    const long long to = (((long long)page * a.h.Hkv + h) * ps + off) * seg + (x - h * seg);
#pragma unroll 4
    for (int l = blockIdx.y * layers; l < last; ++l) {
      const u32x4 k = reinterpret_cast<const u32x4*>((const char*)a.row_layers.k[l] + from)[x];
      const u32x4 v = reinterpret_cast<const u32x4*>((const char*)a.row_layers.v[l] + from)[x];
      reinterpret_cast<u32x4*>(a.layers.k[l])[to] = k;
      reinterpret_cast<u32x4*>(a.layers.v[l])[to] = v;
    }
  }
}

// ---- fork -------------------------------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(const PagesArgs a) {
  __shared__ int tmp[(kScanPages + 1) * kPlanWaves];
  __shared__ int claim[SPIFFY_MAX_SEQS];         // the first pair that names a destination
  const PagedView& c = a.c;
  const int tid = threadIdx.x, ps = c.page_size;
  for (int s = tid; s < c.n_seqs; s += kPlanThreads) claim[s] = 0x7fffffff;
  __syncthreads();
  for (int i = tid; i < a.n; i += kPlanThreads) {
    const int d = a.dst[i];
    if (d >= 0 && d < c.n_seqs) atomicMin(&claim[d], i);
  }
  __syncthreads();
  // item_a: length of the source; item_b: the page its last rows go to, counted first and named below
  int want = 0;
  for (int b = 0; b < a.n; b += kPlanThreads) {
    const int i = b + tid;
    int needs = 0;
    if (i < a.n) {
      const int s = a.src[i], d = a.dst[i];
      bool ok = s >= 0 && s < c.n_seqs && d >= 0 && d < c.n_seqs && claim[d] == i && seq_len(c, d) == 0;
      int len = 0;
      if (ok) {
        len = seq_len(c, s);
        if (len % ps) {
          const int p = c.table[(long long)s * c.max_pages + len / ps];
          ok = p >= 0 && p < c.n_pages;
          needs = ok;
        }
      }
      a.ws.item_a[i] = ok ? len : kSkip;
      if (a.status) a.status[i] = ok ? SPIFFY_PAGES_DONE : SPIFFY_PAGES_BAD;
    }
    int sum;
    const int at = want + block_scan(needs, tmp, sum);
    if (i < a.n) a.ws.item_b[i] = needs ? at : -1;
    want += sum;
  }
  const int have = want ? list_pages(0, c.n_pages, want < c.n_pages ? want : c.n_pages, a.ws.ids, tmp, [&](int p) { return c.refs[p] == 0; }) : 0;
  __syncthreads();                               // lengths are read above and written below
  for (int i = tid; i < a.n; i += kPlanThreads) {
    const int len = a.ws.item_a[i], at = a.ws.item_b[i];
    if (len < 0) continue;
    if (at >= have) {
      a.ws.item_a[i] = kSkip;
      if (a.status) a.status[i] = SPIFFY_PAGES_NO_PAGE;
      continue;
    }
    if (at >= 0) {
      const int p = a.ws.ids[at];
      a.ws.item_b[i] = p;
      c.refs[p] = 1;
    }
    c.len[a.dst[i]] = len;
  }
}

// One workgroup a (pair, layer, k or v): the rows of the last page; the first layer's also the table row and the references.  48 forks in
// 28 layers 41 us (176 MB read and written, 4.3 TB/s).
__global__ __launch_bounds__(256) void fork_rows_kernel(const PagesArgs a, int first) {
  const PagedView& c = a.c;
  const int i = blockIdx.x, layer = blockIdx.y, part = blockIdx.z, tid = threadIdx.x, ps = c.page_size;
  const int len = a.ws.item_a[i];
  if (len < 0) return;
  const int full = len / ps, rest = len - full * ps, page = a.ws.item_b[i];
  const int32_t* from = c.table + (long long)a.src[i] * c.max_pages;
  if (first && layer == 0 && part == 0) {
    int32_t* to = c.table + (long long)a.dst[i] * c.max_pages;
    for (int j = tid; j < full; j += 256) {
      const int p = from[j];
      to[j] = p;
      if (p >= 0 && p < c.n_pages) atomicAdd(&c.refs[p], 1);
    }
    if (tid == 0 && rest) to[full] = page;
  }
  if (!rest) return;
  const int old = from[full];
  const int es = a.h.f32 ? 4 : 2, seg = a.h.hd * es / 16;
  u32x4* pool = reinterpret_cast<u32x4*>(part ? a.layers.v[layer] : a.layers.k[layer]);
  const long long page_pieces = (long long)a.h.Hkv * ps * seg;
  const u32x4* x = pool + old * page_pieces;
  u32x4* y = pool + page * page_pieces;
  for (HeadPieces w((long long)rest * seg, (long long)ps * seg, tid, 256); w.place < page_pieces; w.next()) y[w.place] = x[w.place];
  if (part == 0 && a.layers.summary[layer]) {
    u32x4* sum = reinterpret_cast<u32x4*>(a.layers.summary[layer]);
    const int m = a.h.Hkv * 2 * seg;
    for (int u = tid; u < m; u += 256) sum[(long long)page * m + u] = sum[(long long)old * m + u];
  }
}

// ---- free -------------------------------------------------------------------------------------------------------------------

__global__ __launch_bounds__(256) void free_kernel(const PagesArgs a) {
  __shared__ int s_len;
  const PagedView& c = a.c;
  const int s = a.src[blockIdx.x];
  if (s < 0 || s >= c.n_seqs) return;
  if (threadIdx.x == 0) s_len = atomicExch(&c.len[s], 0);       // of several workgroups with one sequence the first frees it
  __syncthreads();
  const int pages = pages_of(clamp_int(s_len, 0, c.max_pages * c.page_size), c.page_size);
  int32_t* row = c.table + (long long)s * c.max_pages;
  for (int j = threadIdx.x; j < pages; j += 256) {
    const int p = row[j];
    row[j] = -1;
    if (p >= 0 && p < c.n_pages && atomicSub(&c.refs[p], 1) <= 0) atomicAdd(&c.refs[p], 1);
  }
}

// ---- compact ----------------------------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(const PagesArgs a) {
  __shared__ int tmp[(kScanPages + 1) * kPlanWaves];
  const PagedView& c = a.c;
  const int tid = threadIdx.x;
  const int used = list_pages(0, c.n_pages, c.n_pages, nullptr, tmp, [&](int p) { return c.refs[p] > 0; });
  const int to = list_pages(0, used, c.n_pages, a.ws.ids, tmp, [&](int p) { return c.refs[p] <= 0; });
  const int from = list_pages(used, c.n_pages, c.n_pages, a.ws.ids2, tmp, [&](int p) { return c.refs[p] > 0; });
  const int moves = to < from ? to : from;       // equal
  for (int p = used + tid; p < c.n_pages; p += kPlanThreads) a.ws.map[p] = p;
  __syncthreads();
  for (int i = tid; i < moves; i += kPlanThreads) {
    const int x = a.ws.ids2[i], y = a.ws.ids[i];
    a.ws.map[x] = y;
    c.refs[y] = c.refs[x];
    c.refs[x] = 0;
  }
  if (tid == 0) {
    a.ws.count[0] = moves;
    a.ws.count[1] = used;
    if (a.status) a.status[0] = used;
  }
}

// 2048 workgroups take (page, layer, k or v) after another.  835 MB read and written in 174 us: the rate of a copy.
__global__ __launch_bounds__(256) void compact_rows_kernel(const PagesArgs a, int first) {
  const PagedView& c = a.c;
  const int tid = threadIdx.x, moves = a.ws.count[0], used = a.ws.count[1];
  if (moves <= 0) return;
  if (first) {
    const long long n = (long long)c.n_seqs * c.max_pages;
    for (long long j = (long long)blockIdx.x * 256 + tid; j < n; j += (long long)gridDim.x * 256) {
      const int p = c.table[j];
      if (p >= used && p < c.n_pages) c.table[j] = a.ws.map[p];
    }
  }
  const int es = a.h.f32 ? 4 : 2;
  const long long page_pieces = (long long)a.h.Hkv * c.page_size * (a.h.hd * es / 16);
  const int sum_pieces = a.h.Hkv * 2 * (a.h.hd * es / 16);
  const long long jobs = 2ll * moves * a.layers.n;
  for (long long j = blockIdx.x; j < jobs; j += gridDim.x) {
    const int part = (int)(j & 1), i = (int)((j >> 1) % moves), layer = (int)((j >> 1) / moves);
    const long long x = a.ws.ids2[i], y = a.ws.ids[i];
    u32x4* pool = reinterpret_cast<u32x4*>(part ? a.layers.v[layer] : a.layers.k[layer]);
    for (long long u = tid; u < page_pieces; u += 256) pool[y * page_pieces + u] = pool[x * page_pieces + u];
    if (part == 0 && a.layers.summary[layer]) {
      u32x4* sum = reinterpret_cast<u32x4*>(a.layers.summary[layer]);
      for (int u = tid; u < sum_pieces; u += 256) sum[y * sum_pieces + u] = sum[x * sum_pieces + u];
    }
  }
}

}  // namespace

PagesWs carve_pages(const PagedView& c, void* base) {
  PagesWs w;
  int32_t* p = reinterpret_cast<int32_t*>(base);
  auto take = [&](size_t n) {
    int32_t* r = p;
    p += align_up(n, 64);
    return r;
  };
  w.ids = take(c.n_pages);
  w.ids2 = take(c.n_pages);
  w.map = take(c.n_pages);
  w.item_a = take(SPIFFY_MAX_SEQS);
  w.item_b = take(SPIFFY_MAX_SEQS);
  w.count = take(2);
  return w;
}
size_t pages_workspace_bytes(const PagedView& c) {
  return sizeof(int32_t) * (3 * align_up((size_t)c.n_pages, 64) + 2 * align_up((size_t)SPIFFY_MAX_SEQS, 64) + 64);
}

hipError_t launch_append_plan(const PagesArgs& a, hipStream_t st) {
  append_plan_kernel<<<1, kPlanThreads, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_append_rows(const PagesArgs& a, hipStream_t st) {
  // layers of a wavefront: as many as leave 8192 of them, since most rows of a tree are not on its path and a wavefront only finds that out
  const long long jobs = (long long)a.rows.T * a.layers.n;
  const int layers = jobs <= 8192 ? 1 : (jobs / 8192 < a.layers.n ? (int)(jobs / 8192) : a.layers.n);
  append_rows_kernel<<<dim3(cdiv(a.rows.T, 4), cdiv(a.layers.n, layers)), 256, 0, st>>>(a, layers);
  return hipGetLastError();
}
hipError_t launch_fork_plan(const PagesArgs& a, hipStream_t st) {
  fork_plan_kernel<<<1, kPlanThreads, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_fork_rows(const PagesArgs& a, bool first, hipStream_t st) {
  fork_rows_kernel<<<dim3(a.n, a.layers.n, 2), 256, 0, st>>>(a, first);
  return hipGetLastError();
}
hipError_t launch_free(const PagesArgs& a, hipStream_t st) {
  free_kernel<<<a.n, 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_compact_plan(const PagesArgs& a, hipStream_t st) {
  compact_plan_kernel<<<1, kPlanThreads, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_compact_rows(const PagesArgs& a, bool first, hipStream_t st) {
  compact_rows_kernel<<<2048, 256, 0, st>>>(a, first);
  return hipGetLastError();
}

}  // namespace spiffy
