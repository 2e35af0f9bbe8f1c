// Attention of drafted token trees over a paged cache, many rows a kv head (bf16, head_dim up to 128).
//
// With more than 64 rows the matrix instructions are the bound, and a key has to serve them all: eight wavefronts share tiles of 64
// keys through LDS for 128 rows.  Wavefronts w and w + 4 have the same 32 rows and one half of every tile each; two wavefronts a
// SIMD, so that one's exponentials run under the other's matrix instructions; they are joined through LDS at the end.
//
// S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 instructions.  Accumulator element x of lane (column l32 = lane % 32, half = lane / 32) is
// key 8 (x / 4) + 4 half + x % 4, so elements 8 i .. 8 i + 7 are the second product's operand of its i-th step as they stand, with V's
// rows taken in that order by the transposing LDS read (four rows a lane).  Rows lie in LDS as in memory, their 16-byte
// pieces permuted so that neither kind of read meets a bank twice.
//
// Step t runs tile t + 1's first product between tile t's exponentials, then tile t's second product.  Keys are one tile ahead of values in
// LDS and both one more in registers, so a load has a whole step to arrive; one barrier a step.  A row's place in the pool is
// looked up a step before that, from a list of the unit's pages in LDS: pages of any size.
//
// Measured: 128 rows over 131001 rows of 8 kv heads 118 us (537 MB at 4.6 TB/s, memory again), 252 rows 186 to 230 (135 Gflop at 0.6 to
// 0.7 PFLOP/s: a SIMD's matrix pipe works 36% of the time, its vector pipe as much; the clock is 1.9 GHz), 1024 rows of 32 kv heads, 32 states of 32 tokens
// behind 1024 rows, 38 to 41; a prompt of 1024 tokens, 32 heads over 8, behind one row 43.  Tiles of new rows are not pipelined: load, LDS,
// scores, product, one after the other.  Tried: 256 rows a workgroup, a wavefront 64 keys of each tile (no registers left for reads ahead, 440 us at 252
// rows); values and keys to LDS in front of a step (222), their loads at its start (231: the eight wavefronts wait for one another's);
// more or fewer workgroups than CUs (+13 to +30%).
#include <type_traits>

#include "paged_attn.h"

namespace spiffy {

namespace {

constexpr int kThreads = 512, kTile = 64;
constexpr int kWideEntries = 4098;                        // pages that are looked up at a time ...
constexpr int kWideKeys = 65536;                          // ... for so many keys at most

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) bf16x4* lds_bf16x4_ptr_t;
typedef const __attribute__((address_space(3))) bf16x8* lds_bf16x8_ptr_t;

// QUAD: head_dim == HDP, pages of a multiple of the four (64 channels: eight) rows of a wavefront's load lie in one page, their place is the same for all
// lanes but for a constant.
template <int HDP, bool QUAD>
__global__ __launch_bounds__(kThreads, 2) void tree_wide_kernel(const TreeAttnArgs a, const AttnWs ws, int want, int row_tiles, unsigned magic) {
  constexpr int ROWS = kWideRows;
  constexpr int NK = HDP / 16, NN = HDP / 32;             // steps of the first product, 32-channel tiles of the second
  constexpr int PIECES = HDP / 8, RPT = kTile * PIECES / kThreads;      // 16-byte pieces of a row; rows of a thread
  constexpr int RSTEP = kThreads / PIECES, WROWS = kWave / PIECES;      // rows of all threads, of a wavefront
  constexpr int ROWB = HDP * 2, TILEB = kTile * ROWB;
  __shared__ __align__(256) unsigned char s_kv[4 * TILEB];              // K tiles 0, 1, V tiles 0, 1
  __shared__ __align__(16) int2 s_page[kWideEntries];     // page, rows in it
  __shared__ uint64_t bits[(SPIFFY_MAX_TREE / 64) * ROWS];              // [words][ROWS]: what the rows attend to
  __shared__ unsigned long long s_any[SPIFFY_MAX_TREE / 64];
  __shared__ int s_bad;                                   // the first key of a batch that has no row
  __shared__ unsigned s_odd[kTile / 32];                  // new rows of a tile whose values are not all finite
  const PagedView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, half = lane >> 5;
  const int hd = QUAD ? HDP : a.h.hd, ps = c.page_size, g = a.h.Hq / a.h.Hkv;

  int kvh, tile;
  const Unit u = find_unit<true>(a, want, row_tiles, kvh, tile);
  if (u.s < 0) return;
  if (u.index == 0 && kvh == 0 && tile == 0 && tid == 0) ws.plan[u.s] = make_int2(u.units, u.slot);
  const int R = u.rows.n * g, r0 = tile * ROWS;
  if (r0 >= R) return;
  const int lo = u.lo(), hi = u.hi();
  const int group = wave & 3, part = wave >> 2;          // which 32 rows, which half of a tile
  const int row = r0 + group * 32 + l32;                  // this lane's column
  const bool busy = r0 + group * 32 < R;                  // the same for the wavefront: it has rows

  const float sign = a.scale > 0.f ? 1.f : (a.scale < 0.f ? -1.f : 0.f);
  const float scale = sign == 0.f ? 1.f : fabsf(a.scale) * 1.4426950408889634f;
  bf16x8 q[NK];
  {
    const int r = min(row, R - 1);
    const bf16_t* p = reinterpret_cast<const bf16_t*>(a.q) + (u.rows.first + r / g) * a.q_stride + (kvh * g + r % g) * hd;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int ch = 16 * i + 8 * half;
      q[i] = ch < hd ? *reinterpret_cast<const bf16x8*>(p + ch) : bf16x8{};
      if (sign != 1.f)
#pragma unroll
        for (int e = 0; e < 8; ++e) q[i][e] = (bf16_t)((float)q[i][e] * sign);
    }
  }
  float m = -INFINITY, l = 0.f;
  f32x16 o[NN];
#pragma unroll
  for (int n = 0; n < NN; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[n][e] = 0.f;

  // ---- LDS: where pieces lie, what a lane reads
  auto k_at = [](int r, int piece) { return r * ROWB + 16 * (piece ^ (r & (PIECES - 1))); };
  auto v_at = [](int r, int piece) { return r * ROWB + 16 * (piece ^ ((HDP == 128 ? r & 3 : r >> 1 & 1) << 2)); };
  // addresses of a lane's fragments in tile 0; another tile or step is a constant away
  unsigned ka[NK], va[NN];
  const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)s_kv;
#pragma unroll
  for (int i = 0; i < NK; ++i) ka[i] = lds + k_at(32 * part + l32, 2 * i + half);
#pragma unroll
  for (int n = 0; n < NN; ++n) {                          // lane i of 16 names row i / 4, channels 4 (i % 4) ..; it gets channel i of four rows
    const int r = 32 * part + 4 * half + ((lane & 15) >> 2), ch = 32 * n + 16 * (l32 >> 4) + 4 * (lane & 3);
    va[n] = lds + 2 * TILEB + v_at(r, ch >> 3) + (ch & 7) * 2;
  }
  // the last of eight by the fourth's address, whose piece is 8 away (tiles begin at multiples of 256): one register less, and no scratch memory
  auto k_frag = [&](int buf, int i) { return *(lds_bf16x8_ptr_t)(size_t)((i == 7 ? ka[3] ^ 128 : ka[i]) + buf * TILEB); };
  auto v_half = [&](int buf, int i, int n, int e) {       // keys 16 i + 8 e + 4 half .. + 3 of this half tile, channel 32 n + l32
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr_t)(size_t)(va[n] + buf * TILEB + (16 * i + 8 * e) * ROWB));
  };
  auto joined = [](bf16x4 x, bf16x4 y) { return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7); };
  auto scores = [&](int buf, f32x16& s) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < NK; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(buf, i), q[i], s, 0, 0, 0);
  };
  // keys that this column does not attend to (a bit a key of the tile)
  auto hide = [&](f32x16& s, unsigned long long seen) {
    const unsigned bits = (unsigned)(seen >> (32 * part)) >> (4 * half);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (!(bits >> (8 * (e >> 2) + (e & 3)) & 1)) s[e] = -INFINITY;
  };
  // as in the kernel for few rows: a column is rescaled when a score passes the maximum in use by 2^8.  Returns the maximum in use.
  auto follow = [&](f32x16& s) {
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
    top = reduce_32(top, [](float p, float r) { return fmaxf(p, r); }) * scale;
    float base = m;
    if (__any(top > m + 8.f || fabsf(m) >= kFarScore)) {
      const float m2 = top > m + 8.f ? top : m, f = weight(m, m2);
      m = m2;
      l *= f;
#pragma unroll
      for (int n = 0; n < NN; ++n) o[n] *= f;
      base = m == -INFINITY ? 0.f : m;
      const bool far = fabsf(base) >= kFarScore;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = far ? far_score(s[e], scale, base) : s[e];
      base = far ? 0.f : base;
    }
    return base;
  };
  // Probabilities 2 i and 2 i + 1, rounded to bf16 (by up to 2^-8 of themselves, as the stored values are), and the sum of what they are then
  const bf16x2 ones = {(bf16_t)1.f, (bf16_t)1.f};
  auto soften = [&](const f32x16& s, int i, float base, bf16x8 (&x)[2]) {
    f32x2 p;
    p[0] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * i], scale, -base));
    p[1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * i + 1], scale, -base));
    const bf16x2 r = __builtin_convertvector(p, bf16x2);
    l = __builtin_amdgcn_fdot2_f32_bf16(r, ones, l, false);
    x[i >> 2][2 * (i & 3)] = r[0];
    x[i >> 2][2 * (i & 3) + 1] = r[1];
  };
  // Second product of one half tile whose scores are s; seen: as for hide
  auto finish = [&](int buf, f32x16& s, bf16x8 (&x)[2]) {
    const float base = follow(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) soften(s, i, base, x);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int n = 0; n < NN; ++n)
        o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(joined(v_half(buf, i, n, 0), v_half(buf, i, n, 1)), x[i], o[n], 0, 0, 0);
  };
  // Step t of the pipeline, BUF = t % 2: scores `next` of tile t + 1 between the exponentials of s.  fetch(i), i = 0 .. 7: loads that start
  // on the way; all of them at once would hold every wavefront up until the CU's 64 bytes a clock have let them through
  auto step = [&](auto BUF, f32x16& s, f32x16& next, auto fetch) {
    constexpr int buf = decltype(BUF)::value;
    bf16x8 k[NK], x[2];
    bf16x4 v[2][NN][2];
#pragma unroll
    for (int i = 0; i < NK; ++i) k[i] = k_frag(1 - buf, i);
    const float base = follow(s);
#pragma unroll
    for (int e = 0; e < 16; ++e) next[e] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < NK) next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[i < NK ? i : 0], q[i < NK ? i : 0], next, 0, 0, 0);
      soften(s, i, base, x);
      if (i < 2 * NN) {
        v[i / NN][i % NN][0] = v_half(buf, i / NN, i % NN, 0);
        v[i / NN][i % NN][1] = v_half(buf, i / NN, i % NN, 1);
      }
      fetch(i);
    }
    // issue order: a matrix instruction, two exponentials with what is around them, two reads of values
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < NK) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
      if (i < 2 * NN) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      if (QUAD && i % 2 == 1 && i / 2 < 2 * RPT) {
        __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int n = 0; n < NN; ++n) o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(joined(v[i][n][0], v[i][n][1]), x[i], o[n], 0, 0, 0);
  };

  auto fill_bits = [&]() {
    if (hi <= u.tree0) return;
    const int words = (u.rows.n + 63) >> 6;
    for (int i = tid; i < words * ROWS; i += kThreads) {
      const int r = i % ROWS, w = i / ROWS, left = u.rows.n - 64 * w;
      uint64_t b = r0 + r < R ? (left < 64 ? (1ull << left) - 1 : ~0ull) : 0;
      if (a.rows.mask && b) b &= w < a.rows.words ? a.rows.mask[(long long)(u.rows.first + (r0 + r) / g) * a.rows.words + w] : 0;
      bits[i] = b;
      if (b) atomicOr(&s_any[w], (unsigned long long)b);
    }
  };

  const int my_row = tid / PIECES, my_piece = tid % PIECES;
  const bf16_t* pk = reinterpret_cast<const bf16_t*>(a.pk);
  const bf16_t* pv = reinterpret_cast<const bf16_t*>(a.pv);
  const long long row_of_page = (long long)a.h.Hkv * ps;
  const int cache_hi = min(hi, u.eff);
  const int batch_keys = (int)min((long long)(kWideEntries - 2) * ps, (long long)kWideKeys);
  auto entry = [&](int key) {                             // key / ps: the product is at most one too low
    const int e = (int)__umulhi((unsigned)key, magic);
    return key - e * ps >= ps ? e + 1 : e;
  };
  auto fill_pages = [&](int batch) {                      // s_bad holds the batch's end
    const int end = min(cache_hi, batch + batch_keys), e0 = entry(batch), e1 = entry(end - 1), len = seq_len(c, u.s);
    for (int e = e0 + tid; e <= e1; e += kThreads) {
      const int slot = a.selected ? a.selected[((long long)u.s * a.h.Hkv + kvh) * a.n_sel + e] : e;
      int id = -1, rows = 0;
      if (slot >= 0 && slot < c.max_pages) {
        id = c.table[(long long)u.s * c.max_pages + slot];
        rows = id >= 0 && id < c.n_pages ? clamp_int(len - slot * ps, 0, ps) : 0;
      }
      // page and kv head (QUAD: their number, which fits 32 bits, since 2^32 times four rows of 128 bytes are more than there is memory)
      s_page[e - e0] = make_int2(QUAD ? (rows ? id * a.h.Hkv : 0) + kvh : id, rows);
      if (rows < ps) atomicMin(&s_bad, e * ps + rows);
    }
  };

  // ---- the new rows
  // They come first, for their loads need no page: they, the masks and the first list of pages wait together.
  const long long first = u.rows.first;
  bf16x8 nk[RPT], nv[RPT];
  auto load_new = [&](int at) {
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int r = my_row + i * RSTEP;
      nk[i] = nv[i] = bf16x8{};
      if (at + r < u.rows.n && my_piece * 8 < hd) {
        const long long from = (first + at + r) * a.kv_stride + kvh * hd + my_piece * 8;
        nk[i] = *reinterpret_cast<const bf16x8*>(reinterpret_cast<const bf16_t*>(a.k) + from);
        nv[i] = *reinterpret_cast<const bf16x8*>(reinterpret_cast<const bf16_t*>(a.v) + from);
      }
    }
  };
  const int new_at = max(lo - u.tree0, 0);                // whole words: units begin at multiples of 128
  if (new_at < hi - u.tree0) load_new(new_at);
  if (tid < SPIFFY_MAX_TREE / 64) s_any[tid] = 0;
  if (tid < kTile / 32) s_odd[tid] = 0;
  if (tid == 0) s_bad = min(cache_hi, lo + batch_keys);
  __syncthreads();
  if (lo < cache_hi) fill_pages(lo);
  fill_bits();
  __syncthreads();
  for (int at = new_at; at < hi - u.tree0; at += kTile) {
    if (!s_any[at >> 6]) continue;
    if (at > new_at) {
      load_new(at);
      __syncthreads();                                    // the tile before is done with
      if (tid < kTile / 32) s_odd[tid] = 0;
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int r = my_row + i * RSTEP;
      bf16x8 y = nv[i];
      bool odd = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool ok = finite_bits((bf16_t)y[e]);
        odd |= !ok;
        y[e] = ok ? (bf16_t)y[e] : (bf16_t)0.f;
      }
      if (odd) atomicOr(&s_odd[r >> 5], 1u << (r & 31));
      *reinterpret_cast<bf16x8*>(s_kv + k_at(r, my_piece)) = nk[i];
      *reinterpret_cast<bf16x8*>(s_kv + 2 * TILEB + v_at(r, my_piece)) = y;
    }
    __syncthreads();
    const uint64_t seen = bits[(at >> 6) * ROWS + group * 32 + l32];
    if (__any(seen != 0)) {
      f32x16 s;
      bf16x8 x[2];
      scores(0, s);
      hide(s, seen);
      finish(0, s, x);
      // values that are not finite, key by key, only in the columns that attend to the key
      for (unsigned odd = s_odd[part]; odd; odd &= odd - 1) {
        const int y = __ffs(odd) - 1, key = at + 32 * part + y;      // held by half y / 4 % 2, step y / 16, element 4 (y / 8 % 2) + y % 4
        const bool mine = seen >> (key & 63) & 1;
        const bf16_t* from = reinterpret_cast<const bf16_t*>(a.v) + (first + key) * a.kv_stride + kvh * hd;
        const int slot = 4 * (y >> 3 & 1) + (y & 3);
#pragma unroll
        for (int n = 0; n < NN; ++n) {
          const bf16_t z = 32 * n + l32 < hd && half == (y >> 2 & 1) ? from[32 * n + l32] : (bf16_t)0.f;
          bf16x8 w, p;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            w[j] = j == slot && !finite_bits(z) ? z : (bf16_t)0.f;
            p[j] = y >> 4 ? x[1][j] : x[0][j];
          }
          f32x16 more;
#pragma unroll
          for (int e = 0; e < 16; ++e) more[e] = 0.f;
          more = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, p, more, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 16; ++e) o[n][e] = mine ? o[n][e] + more[e] : o[n][e];
        }
      }
    }
  }

  // ---- the cache
  for (int batch = lo; batch < cache_hi; batch += batch_keys) {
    const int end = min(cache_hi, batch + batch_keys), e0 = entry(batch);
    __syncthreads();                                      // the new rows' tiles or the last batch's are done with
    if (batch > lo) {
      if (tid == 0) s_bad = end;
      __syncthreads();
      fill_pages(batch);
      __syncthreads();
    }
    const int tiles = (end - batch + kTile - 1) / kTile, bad = s_bad;      // below `bad` every key has a row
    // row of the pool that holds a key, -1: none
    auto find = [&](int key) {
      const int e = entry(min(key, end - 1)), off = min(key, end - 1) - e * ps;
      const int2 p = s_page[e - e0];
      return key < end && off < p.y ? p.x * row_of_page + (long long)kvh * ps + off : -1ll;      // QUAD: only whether there is one
    };
    // Where this thread's rows of tile t lie.  QUAD: rows of one wavefront, the first of them; otherwise each lane's piece, -1: none.
    long long at[RPT];
    u32x4 kx[RPT], vx[RPT];
    const int lane_at = (my_row & (WROWS - 1)) * HDP + my_piece * 8;
    // QUAD: the list's entry is read a step before it is used
    int page[RPT], off[RPT];
    auto quad_key = [&](int t, int i) {                   // batches begin at multiples of WROWS
      return min(batch + t * kTile + __builtin_amdgcn_readfirstlane(my_row) + i * RSTEP, end - 1) & -WROWS;
    };
    auto look_ahead = [&](int t) {
      if constexpr (QUAD)
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
          const int key = quad_key(t, i), e = entry(key);
          page[i] = s_page[e - e0].x;
          off[i] = key - e * ps;
        }
    };
    auto look_up = [&](int t) {
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        if constexpr (QUAD) {
          at[i] = pool_row(__builtin_amdgcn_readfirstlane(page[i]), ps, off[i]) * HDP;
        } else {
          const long long r = find(batch + t * kTile + my_row + i * RSTEP);
          at[i] = r >= 0 && my_piece * 8 < hd ? r * hd + my_piece * 8 : -1;
        }
      }
    };
    auto piece_of = [&](const bf16_t* pool, long long row) { return *reinterpret_cast<const u32x4*>(pool + row + lane_at); };
    auto load = [&](const bf16_t* pool, u32x4 (&x)[RPT]) {
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        if constexpr (QUAD) x[i] = piece_of(pool, at[i]);
        else x[i] = at[i] >= 0 ? *reinterpret_cast<const u32x4*>(pool + at[i]) : u32x4{};
      }
    };
    // rows that are none, or that hold what is none of the sequence's: zeros
    auto clear = [&](int t, u32x4 (&x)[RPT]) {
      if (!QUAD || batch + (t + 1) * kTile <= bad) return;
#pragma unroll
      for (int i = 0; i < RPT; ++i)
        if (find(batch + t * kTile + my_row + i * RSTEP) < 0) x[i] = u32x4{};
    };
    auto put_keys = [&](int buf, const u32x4 (&x)[RPT]) {
#pragma unroll
      for (int i = 0; i < RPT; ++i) *reinterpret_cast<u32x4*>(s_kv + buf * TILEB + k_at(my_row + i * RSTEP, my_piece)) = x[i];
    };
    auto put_values = [&](int buf, const u32x4 (&x)[RPT]) {
#pragma unroll
      for (int i = 0; i < RPT; ++i) *reinterpret_cast<u32x4*>(s_kv + (2 + buf) * TILEB + v_at(my_row + i * RSTEP, my_piece)) = x[i];
    };
    // tile 0 and the keys of tile 1 into LDS, the keys of tile 2 and the values of tile 1 on their way: all of them start together (behind
    // the last tile its rows come again)
    {
      u32x4 k0[RPT], v0[RPT], k1[RPT];
      look_ahead(0);
      look_up(0);
      load(pk, k0);
      load(pv, v0);
      look_ahead(1);
      look_up(1);
      load(pk, k1);
      load(pv, vx);
      look_ahead(2);
      look_up(2);
      load(pk, kx);
      look_ahead(3);
      clear(0, k0);
      clear(0, v0);
      clear(1, k1);
      put_keys(0, k0);
      put_values(0, v0);
      put_keys(1, k1);
    }
    __syncthreads();
    f32x16 sa, sb;
    if (busy) scores(0, sa);
    // Step t starts when every wavefront is done with step t - 1: tile t's keys and tile t - 1's values give way to the keys of tile t + 2
    // and the values of tile t + 1, which the next step's barrier makes visible; those behind them start.
    auto turn = [&](int t, auto BUF, f32x16& s, f32x16& next) {
      constexpr int buf = decltype(BUF)::value;
      __syncthreads();
      if constexpr (QUAD) {
        // A thread's values of tile t + 1 and keys of tile t + 2, loaded during the last step, go to LDS during this one, each just before the
        // load that takes its registers.  Behind the last tile its rows come again, and nobody reads them.
        long long at_v[RPT];
#pragma unroll
        for (int i = 0; i < RPT; ++i) at_v[i] = at[i];
        look_up(t + 3);
        look_ahead(t + 4);
        clear(t + 2, kx);
        clear(t + 1, vx);
        auto fetch = [&](int i) {
          if (i < RPT) {
            *reinterpret_cast<u32x4*>(s_kv + (3 - buf) * TILEB + v_at(my_row + i * RSTEP, my_piece)) = vx[i];
            vx[i] = piece_of(pv, at_v[i]);
          } else if (i < 2 * RPT) {
            *reinterpret_cast<u32x4*>(s_kv + buf * TILEB + k_at(my_row + (i - RPT) * RSTEP, my_piece)) = kx[i - RPT];
            kx[i - RPT] = piece_of(pk, at[i - RPT]);
          }
        };
        if (!busy) {
#pragma unroll
          for (int i = 0; i < 2 * RPT; ++i) fetch(i);
          return;
        }
        if (batch + (t + 1) * kTile > bad) hide(s, __ballot(find(batch + t * kTile + lane) >= 0));
        step(BUF, s, next, [&](int i) {                   // `next` behind the last tile: scores of what LDS holds, and nothing reads them
          if (i % 2 == 1) fetch(i / 2);
        });
      } else {
        if (t + 2 < tiles) put_keys(buf, kx);
        if (t + 1 < tiles) put_values(1 - buf, vx);
        if (t + 2 < tiles) load(pv, vx);
        if (t + 3 < tiles) {
          look_up(t + 3);
          load(pk, kx);
        }
        if (!busy) return;
        if (batch + (t + 1) * kTile > bad) hide(s, __ballot(find(batch + t * kTile + lane) >= 0));
        step(BUF, s, next, [](int) {});
      }
    };
    for (int t = 0; t < tiles; t += 2) {
      turn(t, std::integral_constant<int, 0>{}, sa, sb);
      if (t + 1 < tiles) turn(t + 1, std::integral_constant<int, 1>{}, sb, sa);
    }
  }

  // ---- results: rows of a lane's column, four channels at a time
  // Places are worked out again: kept through the loop they are the registers that it lacks.
  int thread = tid, rows_of_head = g;
  asm volatile("" : "+v"(thread), "+s"(rows_of_head));
  const int at_row = (thread >> 6 & 3) * 32 + (thread & 31), out_row = r0 + at_row;
  float sum = reduce_32(l, [](float p, float r) { return p + r; });
  {
    // The upper halves' results go through LDS, 32 channels at a time.
    constexpr int LD = 36;
    static_assert(4 * 32 * LD * sizeof(float) <= sizeof(s_kv) && 4 * 32 * sizeof(float2) <= sizeof(s_page), "join buffers");
    float* join = reinterpret_cast<float*>(s_kv) + at_row * LD + 4 * half;
    float2* stat = reinterpret_cast<float2*>(s_page);
    __syncthreads();                                      // tiles and bits are done with
    if (part == 1 && half == 0) stat[at_row] = make_float2(m, sum);
    __syncthreads();
    const float2 other = stat[at_row];
    const float top = fmaxf(m, other.x), f = weight(m, top), fo = weight(other.x, top);
#pragma unroll
    for (int n = 0; n < NN; ++n) {
      if (part == 1)
#pragma unroll
        for (int e = 0; e < 16; e += 4) *reinterpret_cast<f32x4*>(join + 2 * e) = f32x4{o[n][e], o[n][e + 1], o[n][e + 2], o[n][e + 3]};
      __syncthreads();
      if (part == 0)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const f32x4 z = *reinterpret_cast<const f32x4*>(join + 2 * e);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][e + i] = o[n][e + i] * f + z[i] * fo;
        }
      __syncthreads();
    }
    if (part == 1) return;
    sum = sum * f + other.y * fo;
    m = top;
  }
  if (out_row >= R) return;
  const long long at = ((long long)(u.slot + u.index) * a.h.Hkv + kvh) * ws.rows + out_row;
  bf16_t* out = reinterpret_cast<bf16_t*>(a.out) + (u.rows.first + out_row / rows_of_head) * a.out_stride + (kvh * g + out_row % rows_of_head) * hd;
  if (u.units > 1 && half == 0) ws.ml[at] = make_float2(m, sum);
#pragma unroll
  for (int n = 0; n < NN; ++n)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int ch = 32 * n + 2 * e + 4 * half;
      if (ch >= hd) continue;
      const f32x4 z = {o[n][e], o[n][e + 1], o[n][e + 2], o[n][e + 3]};
      if (u.units > 1) *reinterpret_cast<f32x4*>(ws.o + at * hd + ch) = z;
      else store_row(out + ch, z, sum);
    }
}

}  // namespace

hipError_t launch_tree_wide(const TreeAttnArgs& a, const AttnWs& ws, int want, int row_tiles, hipStream_t st) {
  const int ps = a.c.page_size;
  const unsigned magic = 0xffffffffu / (unsigned)ps;
  const unsigned grid = (unsigned)grid_of((long long)want + a.c.n_seqs, a.h.Hkv, row_tiles);
  const bool quad = ps % (a.h.hd == 64 ? 8 : 4) == 0;
  if (a.h.hd == 128 && quad) tree_wide_kernel<128, true><<<grid, kThreads, 0, st>>>(a, ws, want, row_tiles, magic);
  else if (a.h.hd == 64 && quad) tree_wide_kernel<64, true><<<grid, kThreads, 0, st>>>(a, ws, want, row_tiles, magic);
  else if (a.h.hd > 64) tree_wide_kernel<128, false><<<grid, kThreads, 0, st>>>(a, ws, want, row_tiles, magic);
  else tree_wide_kernel<64, false><<<grid, kThreads, 0, st>>>(a, ws, want, row_tiles, magic);
  return hipGetLastError();
}

}  // namespace spiffy
