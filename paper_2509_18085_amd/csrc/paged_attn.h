// What the kernels of the tree attention share: how a call's keys are cut into units, and partial results.
#pragma once
#include "paged.h"

namespace spiffy {

constexpr int kAlign = 128;             // keys: unit borders, four wavefronts' steps
constexpr int kMinChunk = 256;          // keys of a unit at least

__device__ __forceinline__ bool finite_bits(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ bool finite_bits(bf16_t x) { return (__builtin_bit_cast(unsigned short, x) & 0x7f80u) != 0x7f80u; }

// Weight of a partial result whose maximum is m in one whose maximum is top (logarithms to base 2)
__device__ __forceinline__ float weight(float m, float top) { return m == top ? 1.f : __builtin_amdgcn_exp2f(m - top); }

struct Unit {
  int s, index, units, slot;            // slot of the sequence's first partial result
  long long chunk;
  RowRange rows;
  int eff, tree0, total;                // keys of the cache, number of the first new row, end of the numbering
};

__device__ __forceinline__ void measure(const TreeAttnArgs& a, int s, Unit& u) {
  u.rows = rows_of(a.rows, s);
  if (u.rows.n > a.max_rows) u.rows.n = a.max_rows;
  // below 2^31 - 2^16 (checked on the host), so that numbers of new rows and of batches fit behind it
  u.eff = a.selected ? a.n_sel * a.c.page_size : seq_len(a.c, s);
  u.tree0 = (u.eff + kAlign - 1) / kAlign * kAlign;
  u.total = u.tree0 + u.rows.n;
}
__device__ __forceinline__ int units_of(int total, long long chunk) {
  const int n = (int)((total + chunk / 2) / chunk);
  return n < 1 ? 1 : n;
}

__device__ __forceinline__ long long chunk_of(long long keys, int want) {
  const long long chunk = ((keys + want - 1) / want + kAlign - 1) / kAlign * kAlign;
  return chunk < kMinChunk ? kMinChunk : chunk;
}

// A workgroup's part of a call: `per` workgroups (kv heads times row tiles) a unit, those of one unit next to each other on one XCD.  Only
// the workgroups of units that there are take part in the spread over the XCDs: a launch is sized for the most units that the
// sequences can make.
struct Place {
  int unit, part;                       // unit -1: none
};
__device__ __forceinline__ Place place_of(int units, int per) {
  const int active = units * per;
  if ((int)blockIdx.x >= active) return Place{-1, 0};
  const int logical = xcd_contiguous(blockIdx.x, active);
  return Place{logical / per, logical % per};
}

// This workgroup's unit, found by every thread; s < 0: there is none.  Up to 64 sequences a wavefront finds it by itself, a sequence a
// lane.  part: which of the unit's workgroups.
__device__ __forceinline__ Unit find_unit(const TreeAttnArgs& a, int want, int per, int& part) {
  __shared__ long long sums[8];
  __shared__ int tmp[8], found[3];
  const int tid = threadIdx.x, lane = tid & 63, threads = blockDim.x, n_seqs = a.c.n_seqs;
  Unit u;
  if (n_seqs <= kWave) {
    u.rows.n = u.total = 0;
    if (lane < n_seqs) measure(a, lane, u);
    long long keys = u.rows.n > 0 ? u.total : 0;
#pragma unroll
    for (int o = 32; o; o >>= 1) keys += __shfl_xor(keys, o, kWave);
    u.chunk = chunk_of(keys, want);
    const int n = u.rows.n > 0 ? units_of(u.total, u.chunk) : 0;
    int at = n, slot = n > 1 ? n : 0;                      // sums up to and with this sequence
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int x = __shfl_up(at, o, kWave), y = __shfl_up(slot, o, kWave);
      if (lane >= o) at += x, slot += y;
    }
    const Place p = place_of(__shfl(at, kWave - 1, kWave), per);
    const int id = p.unit;
    part = p.part;
    const unsigned long long ends = id < 0 ? 0 : __ballot(at > id);
    const int s = ends ? __ffsll(ends) - 1 : 0;
    u.s = ends ? s : -1;
    u.units = __shfl(n, s, kWave);
    u.index = id - (__shfl(at, s, kWave) - u.units);
    u.slot = __shfl(slot, s, kWave) - (u.units > 1 ? u.units : 0);
    u.rows.first = __shfl(u.rows.first, s, kWave);
    u.rows.n = __shfl(u.rows.n, s, kWave);
    u.eff = __shfl(u.eff, s, kWave);
    u.tree0 = __shfl(u.tree0, s, kWave);
    u.total = __shfl(u.total, s, kWave);
    return u;
  }
  long long keys = 0;
  for (int s = tid; s < n_seqs; s += threads) {
    measure(a, s, u);
    if (u.rows.n > 0) keys += u.total;
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) keys += __shfl_xor(keys, o, kWave);
  if (lane == 0) sums[tid >> 6] = keys;
  if (tid == 0) found[0] = -1;
  __syncthreads();
  keys = 0;
  for (int w = 0; w < threads >> 6; ++w) keys += sums[w];
  const long long chunk = chunk_of(keys, want);
  int n_units = 0;
  for (int b = 0; b < n_seqs; b += threads) {
    const int s = b + tid;
    int all;
    if (s < n_seqs) measure(a, s, u);
    block_scan(s < n_seqs && u.rows.n > 0 ? units_of(u.total, chunk) : 0, tmp, all);
    n_units += all;
  }
  const Place p = place_of(n_units, per);
  const int id = p.unit;
  part = p.part;
  int before = 0, slots = 0;
  for (int b = 0; id >= 0 && b < n_seqs; b += threads) {
    const int s = b + tid;
    int n = 0;
    if (s < n_seqs) {
      measure(a, s, u);
      n = u.rows.n > 0 ? units_of(u.total, chunk) : 0;
    }
    int all, all_slots;
    const int at = before + block_scan(n, tmp, all), slot = slots + block_scan(n > 1 ? n : 0, tmp, all_slots);
    if (id >= at && id < at + n) found[0] = s, found[1] = at, found[2] = slot;
    before += all;
    slots += all_slots;
  }
  __syncthreads();
  u.s = found[0];
  if (u.s < 0) return u;
  measure(a, u.s, u);
  u.chunk = chunk;
  u.units = units_of(u.total, chunk);
  u.index = id - found[1];
  u.slot = found[2];
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
