// Attention of drafted token trees over a paged cache.
//
// The new rows of a sequence that share a kv head (all its rows times the query heads of the group) are the columns of S^T = K Q^T and of
// O^T = V^T P^T, sixteen to a matrix instruction, RT such tiles to a workgroup; keys are read once for all of them.  An accumulator
// element i of lane (column l16 = lane % 16, group grp = lane / 16) of S^T is the score of key 4 grp + i: with keys numbered that
// way inside a step the probabilities are the second product's operand as they stand, no lane needs another's.  Its other operand
// needs one channel of several keys a lane: a lane loads VW neighbouring channels of its keys (whole rows by 16 lanes, 16 bytes each)
// and the m-th instruction takes the m-th of them, so the channel order of the accumulators is (piece, row of the fragment,
// m) and nothing is transposed across lanes.  Keys and values go from memory to registers without LDS: no two wavefronts of a
// workgroup use the same ones.
//
// Work is cut along the keys.  A sequence's keys are numbered through its cache (pages in table order, or the selected pages), then, from
// a multiple of 128 on, its new rows, and divided evenly into as many units as its share of the call's keys, so a long sequence
// beside short ones is spread over all of the GPU.  The four wavefronts of a unit take steps of 32 (fp32: 16) keys in turn, each with
// its own running maximum and sum; they are joined in LDS, and units of one sequence by a second kernel, always in the same order.
//
// Up to 64 rows a kv head memory is the bound: one token over 131001 rows of 8 kv heads takes 103 us (537 MB, 5.2 TB/s; a large copy reaches 4.9),
// 8 tokens (two row tiles) 103, 16 (four) 109; 64 sequences of 64 to 16384 rows, a token each, 181 (923 MB).  Short calls are latency: one
// token over 500 rows 10.8 us in one piece (five steps one after the other), over 32 pages of 64 rows 7.8 and 4 of the join.  A workgroup a row and head, reading keys a wavefront at a time,
// took 7235 us at the 64 sequences.
#include "paged_attn.h"

namespace spiffy {

namespace {

// Workgroups that the units of a call are to make.  Four row tiles take a CU for one workgroup, two leave no room for a third, and more than one round of them only
// adds starts and joins (one tree of 16 tokens over 131001 rows, 256 / 512 / 1024: 105 / 116 / 142 us; two row tiles, one of 3000 rows, 256 / 512:
// 16.9 / 19.4); one row tile leaves room for two or three and wants a second round where lengths differ.
constexpr int target_groups(int rt) { return rt > 1 ? 256 : 1024; }
constexpr int kWideGroups = 256;        // the wide kernel: one workgroup a CU
// Calls whose tables (or selections) have room for up to 576 keys a sequence (fp32: 288) are not cut; the host, which chooses, does not know the
// lengths.  One token of one sequence, cut and joined / in one piece, bf16 over 200 rows 11.4 / 8.5 us, 450 11.4 / 10.7, 700 11.4 / 12.8;
// fp32 over 200 13.4 / 12.3, 450 13.6 / 17.8.  So one token over 500 rows takes 10.8 us under a table of 544 rows, 11.3 under one of 131072; over
// 200 rows 8.4 and 11.3.
constexpr int kUncutBytes = 1152;       // keys times the element size
constexpr int kEntries = 1026;          // pages that are looked up at a time
constexpr int kBatch = 1024;            // ... by keys: pages of one row, and
constexpr int kBatchFast = 16384;       // pages of 16 rows, from an entry's middle to another's
constexpr int kMaxWords = SPIFFY_MAX_TREE / 64;

template <typename T> struct Vec;
template <> struct Vec<float> { typedef f32x4 k, v8, v4; };
template <> struct Vec<bf16_t> { typedef bf16x8 k; typedef bf16x8 v8; typedef bf16x4 v4; };
template <typename T, int N> struct ValueVec { typedef typename Vec<T>::v8 type; };
template <> struct ValueVec<bf16_t, 4> { typedef bf16x4 type; };

// Wavefronts a SIMD that the registers are to leave room for: accumulators, and keys and values in flight, beside some 60 others
constexpr int waves_of(int hdp, int rt) {
  const int regs = rt * hdp / 4 + hdp / 2;                // two row tiles of 256 channels: all there are; the steps over new rows spill, those over the cache do not
  return regs <= 64 ? 3 : (regs <= 128 ? 2 : 1);
}

// FAST: head_dim == HDP, pages of a power of two rows, 16 at least: a 16-key tile lies in one page.  Otherwise every lane looks its
// rows up, and channels from head_dim on count as zero.
template <typename T, int HDP, int RT, bool FAST>
__global__ __launch_bounds__(256, waves_of(HDP, RT)) void tree_attn_kernel(const TreeAttnArgs a, const AttnWs ws, int want,
                                                                                      int row_tiles, int log_ps) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NT = BF ? 2 : 1;                          // 16-key tiles of a step
  constexpr int KW = 16 / sizeof(T), NC = HDP / (4 * KW); // channels of a lane's piece of a key, pieces
  constexpr int VW = HDP / 16 < KW ? HDP / 16 : KW, NP = HDP / (16 * VW);
  constexpr int STEP = 16 * NT;
  constexpr int LD = HDP + 4;                             // row stride of the join buffer: 16 rows in 16 different bank groups
  constexpr bool QLDS = RT > 1;                           // queries stay in LDS: registers for a second wavefront a SIMD
  typedef typename Vec<T>::k kvec_t;
  typedef typename ValueVec<T, VW>::type vvec_t;
  // probabilities as the second product takes them: bf16 of eight keys, fp32 of four
  typedef typename Vec<T>::k pvec_t;
  __shared__ __align__(16) float join[4][16][LD];
  __shared__ __align__(16) kvec_t s_q[QLDS ? RT * NC * kWave : 1];
  __shared__ uint64_t bits[kMaxWords * RT * 16];          // [words][RT * 16]
  __shared__ int page_id[kEntries], page_rows[kEntries];
  __shared__ float s_m[4][RT * 16], s_l[4][RT * 16];
  const PagedView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, grp = lane >> 4;
  const int hd = FAST ? HDP : a.h.hd, ps = c.page_size, g = a.h.Hq / a.h.Hkv;

  int kvh, tile;
  const Unit u = find_unit<(RT > 1)>(a, want, row_tiles, kvh, tile);
  if (u.s < 0) return;
  if (u.index == 0 && kvh == 0 && tile == 0 && tid == 0) ws.plan[u.s] = make_int2(u.units, u.slot);
  const int R = u.rows.n * g, r0 = tile * RT * 16;
  if (r0 >= R) return;
  const int lo = u.lo(), hi = u.hi();

  // The scale is taken as positive; its sign goes to the queries, and a scale of zero makes them zero.
  const float sign = a.scale > 0.f ? 1.f : (a.scale < 0.f ? -1.f : 0.f);
  const float scale = sign == 0.f ? 1.f : fabsf(a.scale) * 1.4426950408889634f;
  auto load_query = [&](int t, int i) {
    const int r = min(r0 + t * 16 + l16, R - 1), ch = i * 4 * KW + grp * KW;
    const T* p = reinterpret_cast<const T*>(a.q) + (u.rows.first + r / g) * a.q_stride + (kvh * g + r % g) * hd;
    kvec_t x = FAST || ch < hd ? *reinterpret_cast<const kvec_t*>(p + ch) : kvec_t{};
    if (sign != 1.f)
#pragma unroll
      for (int e = 0; e < KW; ++e) x[e] = (T)((float)x[e] * sign);
    return x;
  };
  kvec_t q[QLDS ? 1 : NC];
  if constexpr (QLDS) {
    for (int i = wave; i < RT * NC; i += 4) s_q[i * kWave + lane] = load_query(i / NC, i % NC);
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i) q[i] = load_query(0, i);
  }

  // the tree's bits of this workgroup's rows
  auto fill_bits = [&]() {
    if (hi <= u.tree0) return;
    const int words = (u.rows.n + 63) >> 6;
    for (int i = tid; i < words * RT * 16; i += 256) {
      const int r = i % (RT * 16), w = i / (RT * 16);
      const int row = r0 + r < R ? (r0 + r) / g : 0, left = u.rows.n - 64 * w;
      uint64_t b = left < 64 ? (1ull << left) - 1 : ~0ull;
      if (a.rows.mask) b &= w < a.rows.words ? a.rows.mask[(long long)(u.rows.first + row) * a.rows.words + w] : 0;
      bits[i] = b;
    }
  };

  float m[RT], l[RT];
  f32x4 o[RT][NP][VW];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int e = 0; e < VW; ++e) o[t][p][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  kvec_t k[NT][NC];
  vvec_t v[4 * NT][NP];
  auto load_key = [&](const T* row, int n) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int ch = i * 4 * KW + grp * KW;
      k[n][i] = FAST || ch < hd ? *reinterpret_cast<const kvec_t*>(row + ch) : kvec_t{};
    }
  };
  auto load_value = [&](const T* row, int j) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int ch = p * 16 * VW + l16 * VW;
      v[j][p] = FAST || ch < hd ? *reinterpret_cast<const vvec_t*>(row + ch) : vvec_t{};
    }
  };
  // Row tile t against the step's keys, not yet scaled
  auto scores = [&](int t, f32x4* s) {
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const kvec_t x = QLDS ? s_q[(t * NC + i) * kWave + lane] : q[QLDS ? 0 : i];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if constexpr (BF) {
          s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[n][i], x, s[n], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[n][i][e], x[e], s[n], 0, 0, 0);
        }
      }
    }
  };
  // Running maximum and sum; returns the probabilities.  A column is rescaled only when a score passes its maximum in use by 2^8: with a
  // maximum that is too low by less all is as exact, probabilities are just up to 256 instead of 1.  No column's arithmetic depends
  // on another's.  In bf16 a probability is rounded by up to 2^-8 of itself, as the stored values are, since the second product
  // takes both operands in one type and fp32 has a sixteenth of the rate; their sum is not.  Against 64 bits an output is off by 0.0023 of its
  // root mean square, by 0.0017 with probabilities in fp32.
  auto soften = [&](int t, f32x4* s) {
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[n][i]);
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    top = reduce_16(reduce_32(top, larger), larger) * scale;
    if (__any(top > m[t] + 8.f)) {
      const float m2 = top > m[t] + 8.f ? top : m[t], f = weight(m[t], m2);
      m[t] = m2;
      l[t] *= f;
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int e = 0; e < VW; ++e) o[t][p][e] *= f;
    }
    float base = m[t] == -INFINITY ? 0.f : m[t];          // no score so far: every difference is minus infinity
    if (__any(fabsf(base) >= kFarScore)) {
      const bool far = fabsf(base) >= kFarScore;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = far ? far_score(s[n][i], scale, base) : s[n][i];
      base = far ? 0.f : base;
    }
    pvec_t x;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][i], scale, -base));
        l[t] += p;
        x[4 * n + i] = (T)p;
      }
    return x;
  };
  auto multiply = [&](pvec_t w, pvec_t x, f32x4 acc) {    // w: one channel of this lane's keys
    if constexpr (BF) {
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, acc, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w[j], x[j], acc, 0, 0, 0);
      return acc;
    }
  };
  auto add_values = [&](const pvec_t* x) {                // all row tiles: a channel's operand is put together once
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        pvec_t w;
#pragma unroll
        for (int j = 0; j < 4 * NT; ++j) w[j] = (T)v[j][p][e];
#pragma unroll
        for (int t = 0; t < RT; ++t) o[t][p][e] = multiply(w, x[t], o[t][p][e]);
      }
  };

  const T* pk = reinterpret_cast<const T*>(a.pk);
  const T* pv = reinterpret_cast<const T*>(a.pv);
  const long long row_of_page = (long long)a.h.Hkv * ps;  // rows of k or v from one page to the next
  const int cache_hi = min(hi, u.eff);
  constexpr int BATCH = FAST ? kBatchFast : kBatch;
  auto entry = [&](int key) { return FAST ? key >> log_ps : key / ps; };
  auto fill_pages = [&](int batch) {
    const int end = min(cache_hi, batch + BATCH), e0 = entry(batch), e1 = entry(end - 1), len = seq_len(c, u.s);
    for (int e = e0 + tid; e <= e1; e += 256) {
      const int slot = a.selected ? a.selected[((long long)u.s * a.h.Hkv + kvh) * a.n_sel + e] : e;
      int id = -1, rows = 0;
      if (slot >= 0 && slot < c.max_pages) {
        id = c.table[(long long)u.s * c.max_pages + slot];
        rows = id >= 0 && id < c.n_pages ? clamp_int(len - slot * ps, 0, ps) : 0;
      }
      page_id[e - e0] = rows ? id : 0;
      page_rows[e - e0] = rows;
    }
  };

  // ---- the new rows
  // They come first, for their loads need no page: they, the masks and the first list of pages wait together.
  const long long first = u.rows.first;
  auto load_new = [&](int at) {                           // rows beyond the last repeat it
#pragma unroll
    for (int n = 0; n < NT; ++n)
      load_key(reinterpret_cast<const T*>(a.k) + (first + min(at + 16 * n + l16, u.rows.n - 1)) * a.kv_stride + kvh * hd, n);
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j)
      load_value(reinterpret_cast<const T*>(a.v) + (first + min(at + 16 * (j >> 2) + 4 * grp + (j & 3), u.rows.n - 1)) * a.kv_stride + kvh * hd, j);
  };
  int new_at = max(lo - u.tree0, 0) + wave * STEP;
  if (new_at < hi - u.tree0) load_new(new_at);
  if (lo < cache_hi) fill_pages(lo);
  fill_bits();
  __syncthreads();
  for (int at = new_at; at < hi - u.tree0; at += 4 * STEP) {
    unsigned seen[RT], any = 0;                           // bit x: the row of this lane's column attends to new row at + x
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      seen[t] = (unsigned)(bits[(at >> 6) * (RT * 16) + t * 16 + l16] >> (at & 63)) & (unsigned)((1ull << STEP) - 1);
      any |= seen[t];
    }
    if (!__any(any != 0)) continue;
    if (at > new_at) load_new(at);
    unsigned odd = 0;                                     // bit j: this lane's j-th key has values that are not finite, taken for 0 here
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j) {
      const int key = at + 16 * (j >> 2) + 4 * grp + (j & 3);
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        if (key >= u.rows.n) v[j][p] = vvec_t{};
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          const bool ok = finite_bits((T)v[j][p][e]);
          odd |= ok ? 0u : 1u << j;
          v[j][p][e] = ok ? (T)v[j][p][e] : (T)0.f;
        }
      }
    }
    pvec_t x[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      f32x4 s[NT];
      scores(t, s);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(seen[t] >> (16 * n + 4 * grp + i) & 1)) s[n][i] = -INFINITY;
      x[t] = soften(t, s);
    }
    add_values(x);
    // Zero times NaN is NaN: a value that is not finite is added key by key, only in the columns that attend to the key.
    if (__any(odd != 0)) {
#pragma unroll 1
      for (int y = 0; y < STEP; ++y) {
        const int owner = y >> 2 & 3, slot = (y >> 4) * 4 + (y & 3);
        if (!__any(grp == owner && (odd >> slot & 1))) continue;
        const T* row = reinterpret_cast<const T*>(a.v) + (first + min(at + y, u.rows.n - 1)) * a.kv_stride + kvh * hd;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const int ch = p * 16 * VW + l16 * VW;
          const vvec_t z = grp == owner && (FAST || ch < hd) ? *reinterpret_cast<const vvec_t*>(row + ch) : vvec_t{};
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            pvec_t w;
#pragma unroll
            for (int j = 0; j < 4 * NT; ++j) w[j] = j != slot || finite_bits((T)z[e]) ? (T)0.f : (T)z[e];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              const f32x4 more = multiply(w, x[t], f32x4{0.f, 0.f, 0.f, 0.f});
              const bool mine = seen[t] >> y & 1;
#pragma unroll
              for (int i = 0; i < 4; ++i) o[t][p][e][i] = mine ? o[t][p][e][i] + more[i] : o[t][p][e][i];
            }
          }
        }
      }
    }
  }

  // ---- the cache
  for (int batch = lo; batch < cache_hi; batch += BATCH) {
    const int end = min(cache_hi, batch + BATCH), e0 = entry(batch);
    if (batch > lo) {
      __syncthreads();
      fill_pages(batch);
      __syncthreads();
    }
    if constexpr (FAST) {
      int have[NT];                                       // rows of the tiles; they and where the tiles lie are the same in all lanes
      long long where[NT];
      auto find = [&](int& at) {                          // the first step from `at` on that has rows
        for (; at < end; at += 4 * STEP) {
          bool some = false;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const int key = at + 16 * n, e = (min(key, end - 1) >> log_ps) - e0, off = key & (ps - 1);
            const int page = __builtin_amdgcn_readfirstlane(page_id[e]), rows = __builtin_amdgcn_readfirstlane(page_rows[e]);
            have[n] = key < end ? min(rows - off, 16) : 0;
            where[n] = (page * row_of_page + (long long)kvh * ps + (have[n] > 0 ? off : 0)) * HDP;
            some |= have[n] > 0;
          }
          if (some) break;
        }
      };
      int at = batch + __builtin_amdgcn_readfirstlane(wave) * STEP;
      find(at);
      if (at < end)
#pragma unroll
        for (int n = 0; n < NT; ++n) load_key(pk + where[n] + l16 * HDP, n);
      while (at < end) {
        // values are in flight during the scores, the next step's keys during the second product
#pragma unroll
        for (int j = 0; j < 4 * NT; ++j) load_value(pv + where[j >> 2] + (4 * grp + (j & 3)) * HDP, j);
        int had[NT];
        bool whole = true;
#pragma unroll
        for (int n = 0; n < NT; ++n) had[n] = have[n], whole &= have[n] == 16;
        pvec_t x[RT];
        auto weigh = [&](int t) {
          f32x4 s[NT];
          scores(t, s);
          if (!whole) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (4 * grp + i >= had[n]) s[n][i] = -INFINITY;
          }
          x[t] = soften(t, s);
        };
#pragma unroll
        for (int t = 0; t < RT; ++t) weigh(t);
        at += 4 * STEP;
        find(at);
        if (at < end)
#pragma unroll
          for (int n = 0; n < NT; ++n) load_key(pk + where[n] + l16 * HDP, n);
        if (!whole) {                                     // rows behind the last one may hold anything
#pragma unroll
          for (int j = 0; j < 4 * NT; ++j)
            if (4 * grp + (j & 3) >= had[j >> 2])
#pragma unroll
              for (int p = 0; p < NP; ++p) v[j][p] = vvec_t{};
        }
        add_values(x);
      }
    } else {
      for (int at = batch + wave * STEP; at < end; at += 4 * STEP) {
        auto row_of = [&](int key, bool& there) {         // row of the pool; row 0 where there is none
          const int kk = min(key, end - 1), e = kk / ps, off = kk - e * ps;
          there = key < end && off < page_rows[e - e0];
          return there ? page_id[e - e0] * row_of_page + (long long)kvh * ps + off : 0ll;
        };
        bool there[NT][4], dummy;
#pragma unroll
        for (int n = 0; n < NT; ++n) load_key(pk + row_of(at + 16 * n + l16, dummy) * hd, n);
#pragma unroll
        for (int j = 0; j < 4 * NT; ++j) {
          load_value(pv + row_of(at + 16 * (j >> 2) + 4 * grp + (j & 3), there[j >> 2][j & 3]) * hd, j);
          if (!there[j >> 2][j & 3])
#pragma unroll
            for (int p = 0; p < NP; ++p) v[j][p] = vvec_t{};
        }
        pvec_t x[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          f32x4 s[NT];
          scores(t, s);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!there[n][i]) s[n][i] = -INFINITY;
          x[t] = soften(t, s);
        }
        add_values(x);
      }
    }
  }

  // ---- the four wavefronts' results, joined in their order, a row tile at a time
  auto plus = [](float x, float y) { return x + y; };
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float sum = reduce_16(reduce_32(l[t], plus), plus);
    if (grp == 0) s_m[wave][t * 16 + l16] = m[t], s_l[wave][t * 16 + l16] = sum;
  }
  __syncthreads();
  const long long part = ((long long)(u.slot + u.index) * a.h.Hkv + kvh) * ws.rows + r0;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (r0 + t * 16 >= R) break;
    {
      const int r = t * 16 + l16;
      const float top = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r])), f = weight(m[t], top);
      float* to = join[wave][l16];
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < VW; e += 4)
            *reinterpret_cast<f32x4*>(to + p * 16 * VW + (4 * grp + i) * VW + e) =
                f32x4{o[t][p][e][i], o[t][p][e + 1][i], o[t][p][e + 2][i], o[t][p][e + 3][i]} * f;
    }
    __syncthreads();
    for (int y = tid; y < 16 * (HDP / 4); y += 256) {
      const int rr = y / (HDP / 4), r = t * 16 + rr, ch = y % (HDP / 4) * 4;
      if (r0 + r >= R || ch >= hd) continue;
      const float top = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
      float sum = 0.f;
      f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        sum += s_l[w][r] * weight(s_m[w][r], top);
        z += *reinterpret_cast<const f32x4*>(join[w][rr] + ch);
      }
      if (u.units > 1) {
        *reinterpret_cast<f32x4*>(ws.o + (part + r) * hd + ch) = z;
        if (ch == 0) ws.ml[part + r] = make_float2(top, sum);
      } else {
        T* out = reinterpret_cast<T*>(a.out) + (u.rows.first + (r0 + r) / g) * a.out_stride + (kvh * g + (r0 + r) % g) * hd + ch;
        store_row(out, z, sum);
      }
    }
    if (t + 1 < RT) __syncthreads();
  }
}

// One workgroup (of one wavefront or four) a (new row, query head): the partial results of its sequence's units, in order.
template <typename T>
__global__ __launch_bounds__(256) void tree_join_kernel(const TreeAttnArgs a, const AttnWs ws) {
  __shared__ float s_top[4];
  __shared__ __align__(16) f32x4 s_o[256];
  __shared__ float s_l[256];
  const int tid = threadIdx.x, n = blockDim.x, t = blockIdx.x, h = blockIdx.y, g = a.h.Hq / a.h.Hkv, kvh = h / g, hd = a.h.hd;
  const int s = seq_of_row(a.rows, a.c.n_seqs, t);
  if (s >= a.c.n_seqs) return;
  const RowRange r = rows_of(a.rows, s);
  const int row = t - r.first;
  if (row < 0 || row >= r.n || row >= a.max_rows) return;
  const int2 plan = ws.plan[s];
  if (plan.x <= 1) return;
  const long long step = (long long)a.h.Hkv * ws.rows, first = plan.y * step + (long long)kvh * ws.rows + row * g + (h - kvh * g);
  float top = -INFINITY;
  for (int i = tid; i < plan.x; i += n) top = fmaxf(top, ws.ml[first + i * step].x);
  top = wave_max(top);
  if (n > kWave) {
    if ((tid & 63) == 0) s_top[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
  }
  const int pieces = hd / 4, groups = n / pieces, grp = tid / pieces, pc = tid - grp * pieces;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  if (grp < groups) {
#pragma unroll 4
    for (int i = grp; i < plan.x; i += groups) {
      const float2 ml = ws.ml[first + i * step];
      const float f = weight(ml.x, top);
      o += *reinterpret_cast<const f32x4*>(ws.o + (first + i * step) * hd + pc * 4) * f;
      l += ml.y * f;
    }
  }
  s_o[tid] = o;
  s_l[tid] = l;
  __syncthreads();
  if (tid >= pieces) return;
  for (int i = 1; i < groups; ++i) {
    o += s_o[i * pieces + pc];
    l += s_l[i * pieces + pc];
  }
  store_row(reinterpret_cast<T*>(a.out) + t * a.out_stride + h * hd + pc * 4, o, l);
}

// Row tiles of a workgroup: enough for all rows of a (sequence, kv head), but
// - two at most (fp32 with more than 128 channels: one; registers), since four leave a CU one workgroup, whose four wavefronts wait for their loads
//   at the same time: trees of 16 tokens, 32 heads over 8, four / two, one sequence of 3000 rows 22.6 / 16.8 us, 16 of 700 29.8 / 22.3,
//   100 of 3000 325 / 297; 24 rows in heads of 256 over 60000 rows, two / one, 48 / 68;
// - four where the keys and values that the call's tables (or selections) have room for pass 256 MB, which a second reading does not find in a
//   cache, and these workgroups fit in one round: one sequence of 131001 rows 109 / 122, 16 of 10000 134 / 145, of 4096 58 / 57.  The lengths
//   are the device's: under a table of 131072 rows that is little used four are taken too (3000 rows 23.3 us, 17.0 under a table that fits; 16
//   sequences of 700 30.3 and 22.4);
// - one in calls of one piece while that is no more than kOneTile workgroups: trees of 16 tokens over 200 rows, two / one, 14 sequences 11.9 /
//   11.6, 8 11.7 / 9.5, 20 14.0 / 18.5.
constexpr int kOneTile = 512;
constexpr long long kFarBytes = 1ll << 28;
int row_tiles_of(const Heads& h, int max_rows, long long lists, long long cache_keys, bool whole) {
  const int rows = max_rows * (h.Hq / h.Hkv);
  const bool far = cache_keys >= kFarBytes / (4ll * h.hd) / lists;
  const int most = h.f32 ? (h.hd > 128 ? 1 : 2) : (h.hd <= 128 && lists <= target_groups(4) && far ? 4 : 2);
  const int need = rows <= 16 || (whole && lists * cdiv(rows, 16) <= kOneTile) ? 1 : (rows <= 32 ? 2 : 4);
  return need < most ? need : most;
}
struct Shape {
  bool wide;                // csrc/paged_attn_wide.hip
  int rt, tiles, want, rows;
  long long slots;
};
// cache_keys: as many as a sequence's cache can hold, or as are selected
Shape shape_of(const Heads& h, int n_seqs, int max_rows, long long cache_keys) {
  Shape s;
  s.rows = max_rows * (h.Hq / h.Hkv);
  s.wide = !h.f32 && h.hd <= 128 && s.rows > 64;
  const bool whole = !s.wide && (cache_keys + max_rows) * (h.f32 ? 4 : 2) <= kUncutBytes;
  s.rt = row_tiles_of(h, max_rows, (long long)n_seqs * h.Hkv, cache_keys, whole);
  s.tiles = cdiv(s.rows, s.wide ? kWideRows : 16 * s.rt);
  s.want = (s.wide ? kWideGroups : target_groups(s.rt)) / (h.Hkv * s.tiles);
  if (s.want < 1 || whole) s.want = 1;
  // a sequence of two units or more has more than one full one, so its units are less than twice its blocks over a unit's, and all
  // blocks over a unit's are `want` at most; with one unit wanted no sequence is cut
  s.slots = s.want == 1 ? 0 : 2ll * s.want + 2;
  return s;
}
size_t plan_bytes(const PagedView& c) { return align_up(sizeof(int2) * (size_t)c.n_seqs, 256); }
size_t ml_bytes(const Heads& h, const Shape& s) { return align_up(sizeof(float2) * (size_t)s.slots * h.Hkv * s.rows, 256); }

template <typename T, int HDP, int RT, bool FAST>
hipError_t launch_one(const TreeAttnArgs& a, const AttnWs& ws, const Shape& s, int log_ps, hipStream_t st) {
  const long long grid = grid_of((long long)s.want + a.c.n_seqs, a.h.Hkv, s.tiles);
  tree_attn_kernel<T, HDP, RT, FAST><<<(unsigned)grid, 256, 0, st>>>(a, ws, s.want, s.tiles, log_ps);
  return hipGetLastError();
}
template <typename T, int HDP, int RT>
hipError_t launch_mode(const TreeAttnArgs& a, const AttnWs& ws, const Shape& s, hipStream_t st) {
  const int ps = a.c.page_size;
  if (a.h.hd == HDP && ps >= 16 && (ps & (ps - 1)) == 0) return launch_one<T, HDP, RT, true>(a, ws, s, __builtin_ctz(ps), st);
  return launch_one<T, HDP, RT, false>(a, ws, s, 0, st);
}
template <typename T, int HDP>
hipError_t launch_rows(const TreeAttnArgs& a, const AttnWs& ws, const Shape& s, hipStream_t st) {
  constexpr int most = sizeof(T) == 4 ? (HDP > 128 ? 1 : 2) : (HDP > 128 ? 2 : 4);
  if constexpr (most >= 4)
    if (s.rt == 4) return launch_mode<T, HDP, 4>(a, ws, s, st);
  if constexpr (most >= 2)
    if (s.rt == 2) return launch_mode<T, HDP, 2>(a, ws, s, st);
  return launch_mode<T, HDP, 1>(a, ws, s, st);
}

}  // namespace

bool tree_attn_fits(const PagedView& c, const Heads& h, int max_rows) {
  const Shape s = shape_of(h, c.n_seqs, max_rows, 1ll << 31);
  return grid_of((long long)s.want + c.n_seqs, h.Hkv, s.rt == 4 ? 2 * s.tiles : s.tiles) < 1 << 23;      // two row tiles a workgroup where there are fewer keys
}
size_t tree_attn_workspace_bytes(const PagedView& c, const Heads& h, int max_rows) {
  const Shape s = shape_of(h, c.n_seqs, max_rows, 1ll << 31);      // whether pages are selected is the call's matter: the larger of both
  return plan_bytes(c) + ml_bytes(h, s) + sizeof(float) * (size_t)s.slots * h.Hkv * s.rows * h.hd;
}

hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t st) {
  const long long cache = (long long)(a.selected ? a.n_sel : a.c.max_pages) * a.c.page_size;
  const Shape s = shape_of(a.h, a.c.n_seqs, a.max_rows, cache);
  AttnWs ws;
  unsigned char* p = reinterpret_cast<unsigned char*>(a.workspace);
  ws.plan = reinterpret_cast<int2*>(p);
  ws.ml = reinterpret_cast<float2*>(p + plan_bytes(a.c));
  ws.o = reinterpret_cast<float*>(p + plan_bytes(a.c) + ml_bytes(a.h, s));
  ws.rows = s.rows;
  hipError_t e;
  if (s.wide) e = launch_tree_wide(a, ws, s.want, s.tiles, st);
  else if (a.h.f32) e = a.h.hd <= 64 ? launch_rows<float, 64>(a, ws, s, st) : a.h.hd <= 128 ? launch_rows<float, 128>(a, ws, s, st) : launch_rows<float, 256>(a, ws, s, st);
  else e = a.h.hd <= 64 ? launch_rows<bf16_t, 64>(a, ws, s, st) : a.h.hd <= 128 ? launch_rows<bf16_t, 128>(a, ws, s, st) : launch_rows<bf16_t, 256>(a, ws, s, st);
  if (e != hipSuccess) return e;
  // no sequence can have more than one unit: nothing to join
  if (s.want == 1 || (cache + kAlign - 1) / kAlign + a.max_rows / kAlign <= kMinBlocks) return hipSuccess;
  // few rows have many partial results each and wait for them: four wavefronts a row; many rows: one
  const dim3 grid(a.rows.T, a.h.Hq);
  const int threads = (long long)a.rows.T * a.h.Hq <= 2048 ? 256 : 64;
  if (a.h.f32) tree_join_kernel<float><<<grid, threads, 0, st>>>(a, ws);
  else tree_join_kernel<bf16_t><<<grid, threads, 0, st>>>(a, ws);
  return hipGetLastError();
}

}  // namespace spiffy
