// Work split of the decode attention over the block-scaled cache, shared by its kernels and the merge.
//
// The streams of a step, one per (group of rows, KV head), are laid end to end, group after group and head after head, on a
// line of cost: a stream takes `stream_cost` and then `tile_cost` for each of its tiles of eight entries (128 tokens).  Share c
// of N takes the tiles whose points lie in [c * T / N, (c + 1) * T / N).  A share therefore holds any number of whole
// streams and at most two cut ones, at its two ends: the results of whole streams go straight to the output, a cut one
// leaves a partial result in a slot of its own (slot 2 c: the stream started in an earlier share; slot 2 c + 1: it starts
// here and ends in a later one), and the share records which streams it cut, for the merge.
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

struct Cut {       // a cut stream at one end of a share
  int stream;      // group * Hkv + head; -1: none
  int row0, n_qv;
  int ends;        // the stream ends in this share
};

struct Args {
  const __nv_bfloat16* q;
  const unsigned char *k8, *v8;
  const float* scale;  // [pages][Hkv][2]
  __nv_bfloat16* out;
  float* part_o;       // [2 * SHARES][MAXQV][D]
  float2* part_ml;     // [2 * SHARES][MAXQV]: reference exponent, sum
  Cut* cuts;           // [2 * SHARES]
  Tables t;
  int64_t num_pages;
  int Hq, Hkv, G;
  int group_rows;      // MAXQV / G: the most rows of a group
  float scale_log2;    // softmax scale * log2 e
  int cost_shift;      // see tile_cost
};

inline size_t part_o_bytes(int d) { return size_t(2) * SHARES * MAXQV * d * sizeof(float); }
inline size_t part_ml_bytes() { return size_t(2) * SHARES * MAXQV * sizeof(float2); }
inline size_t workspace_bytes(int d) { return part_o_bytes(d) + part_ml_bytes() + ((2 * SHARES * sizeof(Cut) + 255) & ~size_t(255)); }

// Costs in units of about 0.3 us of a share, fitted to clock readings of the tensor kernel: a tile takes 1.2 us with 16
// q-vectors (as long as its bytes take to arrive) and 0.5 to 0.6 more for every further 16; a stream's set-up, first
// references and epilogue, and what else delays a share that holds two, another 6 us.  In a step of more than some hundred
// million tiles the unit grows by 2^shift, so that 32 bits hold the sum: 64-bit arithmetic would lengthen the start of every
// launch, which is instruction fetches for the most part.
constexpr int COST_PER_TILE = 10, COST_PER_STREAM = 26;  // the largest
__device__ __forceinline__ uint32_t tile_cost(int blocks, int shift) { return max(1, (2 + 2 * blocks) >> shift); }
__device__ __forceinline__ uint32_t stream_cost(int blocks, int shift) { return (18 + 2 * blocks) >> shift; }

// A run of tiles of one stream inside a share.
struct Segment {
  int group, head, tile, n_tiles;  // first tile inside the stream, tiles here
  int row0, n_qv;
  int ent0, n_ent;                 // entries of the segment
  int slot;                        // partial slot, or -1: the whole stream is here
  bool ends;                       // the stream ends here
};

// The segments of one share, in order.  Every warp that needs them walks by itself; begin() is called by a whole warp.
struct Walk {
  int n_groups, share, g, head, tile;
  int r0, n_qv, e0, e1, tiles;            // of group g
  uint32_t per, per_tile, per_stream;     // costs of one of its streams (per: all of it), of a tile, of the set-up
  uint32_t base, x_end;                   // cost position of group g's first stream; end of the share

  // Group with these offsets.  False where they are not a group's: rows or entries outside the arrays, more q-vectors than a stream
  // holds, or a number of tiles that does not follow from the entries.  Such a group counts as empty: everything behind this
  // check stays inside the arrays whatever the tables hold.
  __device__ __forceinline__ bool take_group(const Args& a, int row0, int row1, int ent0, int ent1, int n_tiles) {
    const bool ents = ent0 >= 0 && ent1 >= ent0 && ent1 <= a.t.max_entries && n_tiles == int((uint32_t(ent1 - ent0) + TILE_ENTRIES - 1) / TILE_ENTRIES);
    const bool rows = row0 >= 0 && row1 > row0 && row1 <= a.t.max_rows && row1 - row0 <= a.group_rows;
    const bool sound = ents && (rows || n_tiles == 0);
    r0 = row0;
    n_qv = sound ? (row1 - row0) * a.G : 0;
    e0 = ent0;
    e1 = ent1;
    tiles = sound ? n_tiles : 0;
    const int blocks = max(1, min(MAXQV / 16, (n_qv + 15) / 16));
    per_tile = tile_cost(blocks, a.cost_shift);
    per_stream = stream_cost(blocks, a.cost_shift);
    per = tiles > 0 ? per_stream + per_tile * uint32_t(tiles) : 0;
    return sound;
  }
  // Two passes over the groups, 32 at a time: the total cost, then the group that holds the share's first tile.  The loads of
  // a pass do not wait for anything (the arrays are as long as the capacities say), so a step of up to 32 groups costs one
  // round trip to memory.
  __device__ __forceinline__ void begin(const Args& a, int c) {
    const int lane = threadIdx.x & 31;
    share = c;
    const int counted = __ldcg(a.t.counts + 1);
    int row[2], ent[2], til[2];
    bool sound = true;
    auto load = [&](int i) {
      const bool there = i < a.t.max_groups;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        row[k] = there ? __ldcg(a.t.row_off + i + k) : 0;
        ent[k] = there ? __ldcg(a.t.ent_off + i + k) : 0;
        til[k] = there ? __ldcg(a.t.tile_off + i + k) : 0;
      }
    };
    auto cost_of = [&](int i) {
      const bool fine = take_group(a, row[0], row[1], ent[0], ent[1], int(uint32_t(til[1]) - uint32_t(til[0])));
      sound = sound && (fine || i >= n_groups);
      return i < n_groups ? uint32_t(a.Hkv) * per : 0u;
    };
    load(lane);
    n_groups = max(0, min(counted, a.t.max_groups));
    uint32_t sum = 0;
#pragma unroll 1
    for (int i = lane;;) {
      sum += cost_of(i);
      i += 32;
      if (i - lane >= n_groups) break;
      load(i);
    }
    if (c == 0 && !sound) atomicExch(a.t.counts + 4, int(MV_ERR_INVALID_ARG));  // (its groups are skipped)
    const uint32_t total = __reduce_add_sync(0xffffffffu, sum);
    const uint32_t each = total / SHARES, more = total % SHARES;  // the first `more` shares hold one unit more
    const uint32_t x = each * c + min(uint32_t(c), more);
    x_end = x + each + (uint32_t(c) < more ? 1 : 0);
    g = n_groups;
    if (x >= x_end) {
      g = n_groups = 0;
      return;
    }
    base = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < n_groups; i0 += 32) {
      if (n_groups > 32) load(i0 + lane);
      const uint32_t own = cost_of(i0 + lane);
      uint32_t upto = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      const unsigned past = __ballot_sync(0xffffffffu, base + upto > x);
      if (past) {
        const int l = __ffs(past) - 1;
        g = i0 + l;
        base += __shfl_sync(0xffffffffu, upto - own, l);
        // the lane's members hold its own group
        r0 = __shfl_sync(0xffffffffu, r0, l);
        n_qv = __shfl_sync(0xffffffffu, n_qv, l);
        e0 = __shfl_sync(0xffffffffu, e0, l);
        e1 = __shfl_sync(0xffffffffu, e1, l);
        tiles = __shfl_sync(0xffffffffu, tiles, l);
        per = __shfl_sync(0xffffffffu, per, l);
        per_tile = __shfl_sync(0xffffffffu, per_tile, l);
        per_stream = __shfl_sync(0xffffffffu, per_stream, l);
        break;
      }
      base += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (g >= n_groups) return;
    head = int((x - base) / per);
    base += uint32_t(head) * per;                 // from here on: of the stream
    const uint32_t at = x - base;                 // the share starts at the first tile whose point is not before x
    tile = at > per_stream ? int((at - per_stream + per_tile - 1) / per_tile) : 0;
  }
  // The next segment; false at the end of the share.
  __device__ __forceinline__ bool next(const Args& a, Segment& s) {
    while (g < n_groups) {
      if (tile >= tiles) {
        tile = 0;
        base += per;
        if (++head >= a.Hkv || tiles <= 0) {
          head = 0;
          if (++g < n_groups)
            (void)take_group(a, __ldcg(a.t.row_off + g), __ldcg(a.t.row_off + g + 1), __ldcg(a.t.ent_off + g), __ldcg(a.t.ent_off + g + 1),
                             int(uint32_t(__ldcg(a.t.tile_off + g + 1)) - uint32_t(__ldcg(a.t.tile_off + g))));
        }
        continue;
      }
      const uint32_t first = base + per_stream;  // point of the stream's first tile; the share holds the tiles whose points lie before its end
      const int end = x_end > first ? min(tiles, int((x_end - first + per_tile - 1) / per_tile)) : 0;
      if (end <= tile) return false;
      s.group = g;
      s.head = head;
      s.tile = tile;
      s.n_tiles = end - tile;
      s.row0 = r0;
      s.n_qv = n_qv;
      s.ent0 = e0 + tile * TILE_ENTRIES;
      s.n_ent = min(e1 - s.ent0, s.n_tiles * TILE_ENTRIES);
      s.ends = end == tiles;
      s.slot = tile == 0 && s.ends ? -1 : 2 * share + (tile > 0 ? 0 : 1);
      tile = end;
      return true;
    }
    return false;
  }
};

// What a share leaves for the merge: the streams it cut (one thread).
struct CutLog {
  Cut first{-1, 0, 0, 0}, last{-1, 0, 0, 0};
  __device__ __forceinline__ void add(const Args& a, const Segment& s) {
    if (s.slot < 0) return;
    (s.tile > 0 ? first : last) = Cut{s.group * a.Hkv + s.head, s.row0, s.n_qv, s.ends ? 1 : 0};
  }
  __device__ __forceinline__ void store(const Args& a, int share) const {
    reinterpret_cast<int4*>(a.cuts)[2 * share] = make_int4(first.stream, first.row0, first.n_qv, first.ends);
    reinterpret_cast<int4*>(a.cuts)[2 * share + 1] = make_int4(last.stream, last.row0, last.n_qv, last.ends);
  }
};

__device__ __forceinline__ int scale_exponent(float s) { return int((__float_as_uint(s) >> 23) & 0xffu) - 127; }  // 128: NaN
__device__ __forceinline__ float exp2_int(int e) { return __int_as_float((127 + max(-127, min(e, 127))) << 23); }

}  // namespace blk
}  // namespace mv
