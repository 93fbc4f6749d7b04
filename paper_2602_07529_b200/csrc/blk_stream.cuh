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
  float scale_log2;    // softmax scale * log2 e
};

inline size_t part_o_bytes(int d) { return size_t(2) * SHARES * MAXQV * d * sizeof(float); }
inline size_t part_ml_bytes() { return size_t(2) * SHARES * MAXQV * sizeof(float2); }
inline size_t workspace_bytes(int d) { return part_o_bytes(d) + part_ml_bytes() + ((2 * SHARES * sizeof(Cut) + 255) & ~size_t(255)); }

// Costs in units of about 0.3 us of a share, fitted to clock readings of the tensor kernel: a tile takes 1.2 us with 16
// q-vectors (as long as its bytes take to arrive) and 0.5 to 0.6 more for every further 16, a stream's set-up, first references and
// epilogue another 4 us.
__device__ __forceinline__ int tile_cost(int n_qv) { return 2 + 2 * ((n_qv + 15) / 16); }
__device__ __forceinline__ int stream_cost(int n_qv) { return 10 + 2 * ((n_qv + 15) / 16); }
// quotient of non-negative numbers, in 32 bits where they fit
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  return ((x | y) >> 32) == 0 ? int64_t(uint32_t(x) / uint32_t(y)) : x / y;
}

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
  int r0, n_qv, e0, e1, tiles;       // of group g
  int per, per_tile, per_stream;     // costs of one of its streams (per: all of it), of a tile, of the set-up
  int64_t base, x_end;               // cost position of group g's first stream; end of the share

  __device__ __forceinline__ void take_group(int row0, int row1, int ent0, int ent1, int n_tiles, int G) {
    r0 = row0;
    n_qv = (row1 - row0) * G;
    e0 = ent0;
    e1 = ent1;
    tiles = n_tiles;
    const int qv = max(1, min(MAXQV, n_qv));
    per_tile = tile_cost(qv);
    per_stream = stream_cost(qv);
    per = tiles > 0 ? per_stream + int(min(int64_t(per_tile) * tiles, int64_t(1) << 30)) : 0;
  }
  // Two passes over the groups, 32 at a time: the total cost, then the group that holds the share's first tile.  The loads of
  // a pass do not wait for anything (the arrays are as long as the capacities say), so a step of up to 32 groups costs one
  // round trip to memory.
  __device__ __forceinline__ void begin(const Args& a, int c) {
    const int lane = threadIdx.x & 31;
    share = c;
    const int counted = __ldcg(a.t.counts + 1);
    int64_t total = 0;
    int row[2], ent[2], til[2];
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
      if (i >= n_groups) return int64_t(0);
      take_group(row[0], row[1], ent[0], ent[1], til[1] - til[0], a.G);
      return int64_t(a.Hkv) * per;
    };
    load(lane);
    n_groups = max(0, min(counted, a.t.max_groups));
    for (int i = lane;;) {
      total += cost_of(i);
      i += 32;
      if (i - lane >= n_groups) break;
      load(i);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    const int64_t x = total * c / SHARES;
    x_end = total * (c + 1) / SHARES;
    g = n_groups;
    base = 0;
    if (x >= x_end) {
      g = n_groups = 0;
      return;
    }
    for (int i0 = 0; i0 < n_groups; i0 += 32) {
      if (n_groups > 32) load(i0 + lane);
      const int64_t own = cost_of(i0 + lane);
      int64_t upto = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      const unsigned past = __ballot_sync(0xffffffffu, base + upto > x);
      if (past) {
        const int l = __ffs(past) - 1;
        g = i0 + l;
        base += __shfl_sync(0xffffffffu, upto - own, l);
        const int q0 = __shfl_sync(0xffffffffu, row[0], l), q1 = __shfl_sync(0xffffffffu, row[1], l);
        const int f0 = __shfl_sync(0xffffffffu, ent[0], l), f1 = __shfl_sync(0xffffffffu, ent[1], l);
        take_group(q0, q1, f0, f1, __shfl_sync(0xffffffffu, til[1] - til[0], l), a.G);
        break;
      }
      base += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (g >= n_groups) return;
    const int64_t in_group = x - base;
    head = int(quotient(in_group, per));
    const int64_t behind = in_group - int64_t(head) * per - per_stream;  // the share starts at the first tile whose point is not before x
    tile = behind > 0 ? int(quotient(behind + per_tile - 1, per_tile)) : 0;
  }
  // The next sound segment; false at the end of the share.
  __device__ __forceinline__ bool next(const Args& a, Segment& s, bool report) {
    while (g < n_groups) {
      if (tile >= tiles) {
        tile = 0;
        if (++head >= a.Hkv || tiles <= 0) {
          head = 0;
          base += int64_t(a.Hkv) * per;
          if (++g < n_groups)
            take_group(__ldcg(a.t.row_off + g), __ldcg(a.t.row_off + g + 1), __ldcg(a.t.ent_off + g), __ldcg(a.t.ent_off + g + 1),
                       __ldcg(a.t.tile_off + g + 1) - __ldcg(a.t.tile_off + g), a.G);
        }
        continue;
      }
      const int64_t left = x_end - (base + int64_t(head) * per + per_stream);  // tiles whose points lie before the share's end
      const int end = left > 0 ? int(min(int64_t(tiles), quotient(left + per_tile - 1, per_tile))) : 0;
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
      if (r0 >= 0 && n_qv > 0 && n_qv <= MAXQV && r0 + n_qv / a.G <= a.t.max_rows && e0 >= 0 && e1 <= a.t.max_entries &&
          s.n_ent > (s.n_tiles - 1) * TILE_ENTRIES)
        return true;
      if (report) atomicExch(a.t.counts + 4, int(MV_ERR_INVALID_ARG));  // rows or entries out of range: the segment is skipped
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
