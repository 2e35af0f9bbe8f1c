// Attention of drafted token trees over a paged cache.
//
// One workgroup a (new row, query head): the four wavefronts take keys in turn, the lanes share the channels, each wavefront with a
// running maximum and sum of its own; they are joined through LDS.
#include "paged.h"

namespace spiffy {

namespace {

constexpr int kMaxCh = 4;       // channels of a lane: head_dim <= 256

template <typename T>
__global__ __launch_bounds__(256) void tree_attn_kernel(const TreeAttnArgs a) {
  __shared__ float s_m[4], s_l[4], s_o[4][256];
  const PagedView& c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hd = a.h.hd, ps = c.page_size;
  const int t = blockIdx.x, h = blockIdx.y, kvh = h / (a.h.Hq / a.h.Hkv);
  const int s = seq_of_row(a.rows, c.n_seqs, t);
  if (s >= c.n_seqs) return;
  const RowRange r = rows_of(a.rows, s);
  const int row = t - r.first;
  if (row < 0 || row >= r.n || row >= a.max_rows) return;
  const T* q = reinterpret_cast<const T*>(a.q) + t * a.q_stride + h * hd;
  float qv[kMaxCh], o[kMaxCh];
#pragma unroll
  for (int i = 0; i < kMaxCh; ++i) {
    qv[i] = lane + 64 * i < hd ? to_f32(q[lane + 64 * i]) * a.scale : 0.f;
    o[i] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  auto key = [&](const T* k, const T* v) {
    float x = 0.f, w[kMaxCh];
#pragma unroll
    for (int i = 0; i < kMaxCh; ++i) {
      const bool in = lane + 64 * i < hd;
      x += qv[i] * (in ? to_f32(k[lane + 64 * i]) : 0.f);
      w[i] = in ? to_f32(v[lane + 64 * i]) : 0.f;
    }
    x = wave_sum(x);
    const float m2 = fmaxf(m, x), keep = m == -INFINITY ? 0.f : __expf(m - m2), p = x == -INFINITY ? 0.f : __expf(x - m2);
    m = m2;
    l = l * keep + p;
#pragma unroll
    for (int i = 0; i < kMaxCh; ++i) o[i] = o[i] * keep + p * w[i];
  };
  const int len = seq_len(c, s), used = pages_of(len, ps);
  const int32_t* sel = a.selected ? a.selected + ((long long)s * a.h.Hkv + kvh) * a.n_sel : nullptr;
  for (int u = 0; u < (sel ? a.n_sel : used); ++u) {
    const int slot = sel ? sel[u] : u;
    if (slot < 0 || slot >= used) continue;
    const int page = c.table[(long long)s * c.max_pages + slot];
    if (page < 0 || page >= c.n_pages) continue;
    const long long base = ((long long)page * a.h.Hkv + kvh) * ps;
    for (int j = wave; j < ps && slot * ps + j < len; j += 4)
      key(reinterpret_cast<const T*>(a.pk) + (base + j) * hd, reinterpret_cast<const T*>(a.pv) + (base + j) * hd);
  }
  const uint64_t* bits = a.rows.mask ? a.rows.mask + (long long)t * a.rows.words : nullptr;
  for (int j = wave; j < r.n && j < a.max_rows; j += 4) {
    if (bits && (j >= 64 * a.rows.words || !(bits[j >> 6] >> (j & 63) & 1))) continue;
    const long long at = (r.first + j) * a.kv_stride + kvh * hd;
    key(reinterpret_cast<const T*>(a.k) + at, reinterpret_cast<const T*>(a.v) + at);
  }
  if (lane == 0) s_m[wave] = m, s_l[wave] = l;
#pragma unroll
  for (int i = 0; i < kMaxCh; ++i) s_o[wave][lane + 64 * i] = o[i];
  __syncthreads();
  float top = -INFINITY;
  for (int w = 0; w < 4; ++w) top = fmaxf(top, s_m[w]);
  const int ch = threadIdx.x;
  if (ch >= hd) return;
  float sum = 0.f, x = 0.f;
  for (int w = 0; w < 4; ++w) {
    if (s_m[w] == -INFINITY && !(s_l[w] != s_l[w])) continue;
    const float f = __expf(s_m[w] - top);
    sum += s_l[w] * f;
    x += s_o[w][ch] * f;
  }
  reinterpret_cast<T*>(a.out)[t * a.out_stride + h * hd + ch] = from_f32<T>(sum == 0.f ? 0.f : x / sum);
}

}  // namespace

size_t tree_attn_workspace_bytes(const PagedView&, const Heads&, int, int) { return 256; }

hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t st) {
  const dim3 grid(a.rows.T, a.h.Hq);
  if (a.h.f32) tree_attn_kernel<float><<<grid, 256, 0, st>>>(a);
  else tree_attn_kernel<bf16_t><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace spiffy
