// What the kernels of the tree attention share: how a call's keys are cut into units, and partial results.
#pragma once
#include "paged.h"

namespace spiffy {

constexpr int kAlign = 128;             // keys of a block: units are whole blocks, four wavefronts' steps
constexpr int kMinBlocks = 1;           // blocks of a unit at least (two: one token over 500 rows 13.0 us instead of 11.9, fp32 chains 17.3 instead of 14.1)

__device__ __forceinline__ bool finite_bits(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ bool finite_bits(bf16_t x) { return (__builtin_bit_cast(unsigned short, x) & 0x7f80u) != 0x7f80u; }

// A probability is exp2 of s * scale - m in one rounding, m the rounded s * scale of a column's highest score: what m was rounded by is the same
// for all keys of a column and cancels, while it is below 32.  From 2^30 on it could be 64 and more, an infinity or nothing for every key.
// There fp32 products that are not equal are 64 apart or more, so a key has the highest score or no weight: far_score makes it 0 or minus
// infinity, for a maximum of 0 (what is not finite comes out as NaN, as it does nearer by).
constexpr float kFarScore = 0x1p30f;
__device__ __forceinline__ float far_score(float s, float scale, float m) { return s * scale < m ? -INFINITY : s - s; }

// Weight of a partial result whose maximum is m in one whose maximum is top (logarithms to base 2)
__device__ __forceinline__ float weight(float m, float top) { return m == top ? 1.f : __builtin_amdgcn_exp2f(m - top); }

// A sequence's keys are numbered through its cache, then, from a block's border on, through its new rows.  `blocks` is what they
// cost: a last block of new rows that is not full counts nothing (one token must not make a block of its own) and goes with the last unit.
struct Keys {
  RowRange rows;
  int eff, tree0, total;                // keys of the cache, number of the first new row, end of the numbering
  int blocks;
};
// One unit: blocks first .. of them are divided evenly
struct Unit : Keys {
  int s, index, units, slot;            // slot of the sequence's first partial result
  __device__ __forceinline__ int border(int i) const { return (int)((long long)i * blocks / units) * kAlign; }
  __device__ __forceinline__ int lo() const { return border(index); }
  __device__ __forceinline__ int hi() const { return index == units - 1 ? total : border(index + 1); }
};

__device__ __forceinline__ Keys keys_of(const TreeAttnArgs& a, int s) {
  Keys k;
  k.rows = rows_of(a.rows, s);
  if (k.rows.n > a.max_rows) k.rows.n = a.max_rows;
  // below 2^31 - 2^16 (checked on the host), so that numbers of new rows and of batches fit behind it
  k.eff = a.selected ? a.n_sel * a.c.page_size : seq_len(a.c, s);
  const int cache = (k.eff + kAlign - 1) / kAlign, blocks = cache + k.rows.n / kAlign;
  k.tree0 = cache * kAlign;
  k.total = k.tree0 + k.rows.n;
  k.blocks = k.rows.n > 0 ? (blocks > 0 ? blocks : 1) : 0;
  return k;
}
// Units of at most `most` blocks
__device__ __forceinline__ int units_of(int blocks, int most) { return (int)(((unsigned)blocks + most - 1) / most); }
__device__ __forceinline__ int most_of(long long blocks, int want) {
  const long long most = (blocks + want - 1) / want;      // 4096 sequences of 2^24 blocks: 36 bits, an int's only with `want` of 32 and more
  return most < kMinBlocks ? kMinBlocks : (most > (1 << 25) ? 1 << 25 : (int)most);
}

// Sum over the lanes up to and with this one, on vector instructions (rows of 16 lanes, then the last lane of one or two rows to the next)
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ int wave_scan(int x) {
  x = dpp_add<0x111, 0xF>(x);      // row_shr:1, 2, 4, 8
  x = dpp_add<0x112, 0xF>(x);
  x = dpp_add<0x114, 0xF>(x);
  x = dpp_add<0x118, 0xF>(x);
  x = dpp_add<0x142, 0xA>(x);      // row_bcast:15 to rows 1 and 3
  return dpp_add<0x143, 0xC>(x);   // row_bcast:31 to rows 2 and 3
}

// A workgroup's part of a call.  (unit, kv head) after (unit, kv head) goes to the next XCD (workgroup ids go round the eight of them), with all
// its row tiles, which read the same keys: units differ in size, and a range of them to each XCD would not end together (64 sequences of
// 64 to 16384 rows: 185 us so, 179 this way; calls of equal units are 2% slower).
struct Place {
  int unit, kvh, tile;                  // unit -1: none
};
__device__ __forceinline__ Place place_of(int units, int kv_heads, int tiles) {
  const int xcd = blockIdx.x & 7, j = blockIdx.x >> 3, group = j / tiles * 8 + xcd;
  return group < units * kv_heads ? Place{group / kv_heads, group % kv_heads, j % tiles} : Place{-1, 0, 0};
}
// workgroups of a launch for up to so many units
inline long long grid_of(long long units, int kv_heads, int tiles) { return (units * kv_heads + 7) / 8 * 8 * tiles; }

// This workgroup's unit, found by every thread; s < 0: there is none.  Up to 64 sequences a wavefront finds it by itself, a sequence a
// lane.  There can be up to one unit a sequence more than `want`.  ONE_ROUND: `want` fills the GPU once, so the units of up to `want`
// sequences grow until there are no more (16 trees over 3000 to 4100 rows, 32 units wanted: 81 us with the 48 that there were, 55
// with 32).
template <bool ONE_ROUND>
__device__ __forceinline__ Unit find_unit(const TreeAttnArgs& a, int want, int tiles, int& kvh, int& tile) {
  __shared__ long long sums[8];
  __shared__ int tmp[8], found[3];
  const int tid = threadIdx.x, lane = tid & 63, threads = blockDim.x, n_seqs = a.c.n_seqs;
  Unit u;
  if (n_seqs <= kWave) {
    Keys k = keys_of(a, lane < n_seqs ? lane : 0);
    const int blocks = lane < n_seqs ? k.blocks : 0;      // 64 times 2^24 of them fit
    int most = most_of(__builtin_amdgcn_readlane(wave_scan(blocks), kWave - 1), want);
    int n = units_of(blocks, most), at = wave_scan(n);
    for (int i = 0; ONE_ROUND && i < 8 && n_seqs <= want && __builtin_amdgcn_readlane(at, kWave - 1) > want; ++i) {
      most += most / 8 + 1;
      n = units_of(blocks, most);
      at = wave_scan(n);
    }
    const int slot = wave_scan(n > 1 ? n : 0);            // like `at`: up to and with this sequence
    const Place p = place_of(__builtin_amdgcn_readlane(at, kWave - 1), a.h.Hkv, tiles);
    kvh = p.kvh;
    tile = p.tile;
    const unsigned long long ends = p.unit < 0 ? 0 : __ballot(at > p.unit);
    const int s = ends ? __ffsll(ends) - 1 : 0;
    u.s = ends ? s : -1;
    u.units = __builtin_amdgcn_readlane(n, s);
    u.index = p.unit - (__builtin_amdgcn_readlane(at, s) - u.units);
    u.slot = __builtin_amdgcn_readlane(slot, s) - (u.units > 1 ? u.units : 0);
    u.rows.first = __builtin_amdgcn_readlane(k.rows.first, s);
    u.rows.n = __builtin_amdgcn_readlane(k.rows.n, s);
    u.eff = __builtin_amdgcn_readlane(k.eff, s);
    u.tree0 = __builtin_amdgcn_readlane(k.tree0, s);
    u.total = __builtin_amdgcn_readlane(k.total, s);
    u.blocks = __builtin_amdgcn_readlane(k.blocks, s);
    return u;
  }
  long long blocks = 0;
  for (int s = tid; s < n_seqs; s += threads) blocks += keys_of(a, s).blocks;
#pragma unroll
  for (int o = 32; o; o >>= 1) blocks += __shfl_xor(blocks, o, kWave);
  if (lane == 0) sums[tid >> 6] = blocks;
  if (tid == 0) found[0] = -1;
  __syncthreads();
  blocks = 0;
  for (int w = 0; w < threads >> 6; ++w) blocks += sums[w];
  const int most = most_of(blocks, want);
  int n_units = 0;
  for (int b = 0; b < n_seqs; b += threads) {
    const int s = b + tid;
    int all;
    block_scan(s < n_seqs ? units_of(keys_of(a, s).blocks, most) : 0, tmp, all);
    n_units += all;
  }
  const Place p = place_of(__builtin_amdgcn_readfirstlane(n_units), a.h.Hkv, tiles);
  kvh = p.kvh;
  tile = p.tile;
  int before = 0, slots = 0;
  for (int b = 0; p.unit >= 0 && b < n_seqs; b += threads) {
    const int s = b + tid, n = s < n_seqs ? units_of(keys_of(a, s).blocks, most) : 0;
    int all, all_slots;
    const int at = before + block_scan(n, tmp, all), slot = slots + block_scan(n > 1 ? n : 0, tmp, all_slots);
    if (p.unit >= at && p.unit < at + n) found[0] = s, found[1] = at, found[2] = slot;
    before += all;
    slots += all_slots;
  }
  __syncthreads();
  u.s = __builtin_amdgcn_readfirstlane(found[0]);
  if (u.s < 0) return u;
  static_cast<Keys&>(u) = keys_of(a, u.s);
  u.units = units_of(u.blocks, most);
  u.index = p.unit - __builtin_amdgcn_readfirstlane(found[1]);
  u.slot = __builtin_amdgcn_readfirstlane(found[2]);
  return u;
}

// four channels of a finished row; a sum of zero means that there was nothing to attend to
template <typename T>
__device__ __forceinline__ void store_row(T* to, f32x4 o, float sum) {
  typedef T out4 __attribute__((ext_vector_type(4)));
  const float f = 1.f / sum;
  *reinterpret_cast<out4*>(to) = sum == 0.f ? out4{} : out4{from_f32<T>(o[0] * f), from_f32<T>(o[1] * f), from_f32<T>(o[2] * f), from_f32<T>(o[3] * f)};
}

struct AttnWs {
  int2* plan;       // [n_seqs]: units of a sequence, slot of its first partial result
  float2* ml;       // [slots][Hkv][rows]: maximum (base 2) and sum
  float* o;         // [slots][Hkv][rows][hd]
  int rows;         // rows of a (slot, kv head)
};

// Keys and rows of a wide call (more than 64 rows a kv head, bf16, head_dim <= 128), csrc/paged_attn_wide.hip
constexpr int kWideRows = 128;          // rows of a workgroup
hipError_t launch_tree_wide(const TreeAttnArgs& a, const AttnWs& ws, int want, int row_tiles, hipStream_t st);

}  // namespace spiffy
