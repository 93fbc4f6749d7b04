// Work split of the decode attention over the block-scaled cache, shared by its kernels and the merge.
//
// The streams of a step, one per (group of rows, KV head), are laid end to end, group after group and head after head, in
// tiles of eight entries (128 tokens); share c of N takes tiles [c * T / N, (c + 1) * T / N).  A share therefore holds any
// number of whole streams and at most two cut ones, at its two ends: the results of whole streams go straight to the
// output, a cut one leaves a partial result in a slot of its own (slot 2 c: the stream started in an earlier share; slot
// 2 c + 1: it starts here and ends in a later one).  The merge finds a cut stream's shares by the same arithmetic.
// Everything is computed on the device from the step's tables, so neither the grid nor the workspace depends on the step.
#pragma once
#include "common.cuh"

namespace mv {
namespace blk {

constexpr int PS = 16;          // tokens per page
constexpr int TILE_ENTRIES = 8;
constexpr int MAXQV = 64;       // q-vectors (rows of a group x query heads of a KV head)
constexpr int SHARES = 296;     // two per SM of a 148-SM part

struct Tables {
  const int32_t *row_off, *ent_off, *tile_off;
  const int4* entries;
  int32_t* counts;
  int max_rows, max_groups, max_entries;
};

struct Args {
  const __nv_bfloat16* q;
  const unsigned char *k8, *v8;
  const float* scale;  // [pages][Hkv][2]
  __nv_bfloat16* out;
  float* part_o;       // [2 * SHARES][MAXQV][D]
  float2* part_ml;     // [2 * SHARES][MAXQV]: reference exponent, sum
  Tables t;
  int64_t num_pages;
  int Hq, Hkv, G;
  float scale_log2;    // softmax scale * log2 e
};

__host__ __device__ inline size_t part_o_bytes(int d) { return size_t(2) * SHARES * MAXQV * d * sizeof(float); }
inline size_t workspace_bytes(int d) { return part_o_bytes(d) + size_t(2) * SHARES * MAXQV * sizeof(float2); }

// Sizes of the step, bounded by the capacities whatever the arrays hold.
struct Step {
  int n_groups;
  int64_t n_tiles;  // of all streams
};
__device__ __forceinline__ Step step_of(const Args& a) {
  Step s;
  s.n_groups = max(0, min(a.t.counts[1], a.t.max_groups));
  s.n_tiles = s.n_groups > 0 ? int64_t(max(0, a.t.tile_off[s.n_groups])) * a.Hkv : 0;
  return s;
}
__device__ __forceinline__ int64_t share_begin(int64_t tiles, int c) { return tiles * c / SHARES; }
// the share that holds tile x
__device__ __forceinline__ int share_of(int64_t tiles, int64_t x) { return int(((x + 1) * SHARES - 1) / tiles); }

// The group whose streams hold tile x: the last one with tile_off[g] <= x / Hkv.  Called by a whole warp.
__device__ __forceinline__ int find_group(const int32_t* tile_off, int n_groups, int key) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n_groups;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int p = lo + (lane + 1) * step;
    const unsigned m = __ballot_sync(0xffffffffu, p < hi && tile_off[p] <= key);
    lo += __popc(m) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// A run of tiles of one stream inside a share.
struct Segment {
  int group, head, tile, n_tiles;  // first tile inside the stream, tiles here
  int row0, n_qv;
  int ent0, n_ent;                 // entries of the segment
  int slot;                        // partial slot, or -1: the whole stream is here
  bool ok;                         // false: the tables name rows or entries out of range (the segment is skipped)
};
// The segment at tile x of a share that ends at x_end; g is its group (advanced past empty groups by the caller's next call).
__device__ __forceinline__ Segment segment_at(const Args& a, const Step& st, int c, int64_t x, int64_t x_end, int g) {
  Segment s;
  const int t0 = a.t.tile_off[g], tiles = a.t.tile_off[g + 1] - t0;
  const int64_t in_group = x - int64_t(t0) * a.Hkv;
  s.group = g;
  s.head = int(in_group / tiles);
  s.tile = int(in_group - int64_t(s.head) * tiles);
  s.n_tiles = int(min(int64_t(tiles - s.tile), x_end - x));
  const int r0 = a.t.row_off[g], r1 = a.t.row_off[g + 1], e0 = a.t.ent_off[g], e1 = a.t.ent_off[g + 1];
  s.row0 = r0;
  s.n_qv = (r1 - r0) * a.G;
  s.ent0 = e0 + s.tile * TILE_ENTRIES;
  s.n_ent = min(e1 - s.ent0, s.n_tiles * TILE_ENTRIES);
  s.slot = s.n_tiles == tiles ? -1 : 2 * c + (s.tile > 0 ? 0 : 1);
  s.ok = in_group >= 0 && s.head < a.Hkv && r0 >= 0 && r1 >= r0 && r1 <= a.t.max_rows && (r1 - r0) <= MAXQV / a.G && e0 >= 0 && e1 <= a.t.max_entries && s.n_ent > 0 &&
         s.n_ent > (s.n_tiles - 1) * TILE_ENTRIES;
  return s;
}

__device__ __forceinline__ int scale_exponent(float s) { return int((__float_as_uint(s) >> 23) & 0xffu) - 127; }  // 128: NaN
__device__ __forceinline__ float exp2_int(int e) { return __int_as_float((127 + max(-127, min(e, 127))) << 23); }

}  // namespace blk
}  // namespace mv
