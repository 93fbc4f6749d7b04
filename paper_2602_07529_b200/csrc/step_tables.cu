// Tables of a decode step built on the device: frontier layers (Eq. 1), positions (Sec. 4.2), slots, and the block table
// of every group of rows (Eq. 3 / Sec. 4.3 visibility at page granularity), from a batch description in device memory.
//
// Integers only.  One CTA per request, two launches of the same kernel: the first leaves every request's counts (rows,
// groups, entries, tiles, error), the second sums the counts of the requests before its own and writes; a batch of one request takes
// one launch that does both.  Analysing twice costs a few microseconds of mostly idle SMs and saves storing the per-node results.
// What bounds it is latency: launches, a few dependent loads, shared-memory sweeps over the request's nodes, and the arrival
// of the instructions (one piece of code for both launches, loops not unrolled), not the bytes written.
// Measured: one request 10.2 us (8.2 in a graph), 128 requests of 512 to 16K tokens and 2 to 8 branches 18.4 us, 512 layered ones 26 us (4.8 MB of
// tables, 0.7 us at the memory's rate); with a kernel of its own for each launch 14, 20 and 30 us.
//
// The DAG mask needs no closure matrix.  For one group of at most 64 rows, a node's mask is the set of the group's rows
// that see it: a sweep over the nodes from last to first hands every node's mask on to its parents (parents have smaller
// indices), one 64-bit OR per edge.
#include "common.cuh"
#include "trace.h"

namespace {

constexpr int NT = 256;
constexpr int PS = 16;                 // tokens per page
constexpr int kMaxNew = mv::kMaxAppendTokens;
constexpr int64_t kMaxTokens = int64_t(1) << 30;  // of one node, and bound on a position: everything below fits int32

struct ReqCounts {  // what the first launch leaves per request
  int32_t rows, groups, entries, tiles;
};

enum Mode { COUNT = 1, WRITE = 2 };  // what a launch does (or both)

struct BuildArgs {
  mv_dag_batch b;  // device pointers
  mv_step_shape s;
  mv_step_tables t;
  ReqCounts* req;   // [n_req]
  int32_t* err;     // [n_req]
  int blocks;       // block tables wanted
  int mode;
};

// The request's arrays in shared memory, n nodes.
struct Nodes {
  unsigned long long *mask, *suffix;  // suffix [n + 1]: rows whose layer is at least the index (layerwise visibility)
  int *len, *add, *page0, *layer, *start, *row0, *ent0;  // row0, ent0: [n + 1]
  int *parents;                     // the request's parent lists, or null (too many: read from global memory)
};

constexpr int kParentsPerNode = 4;  // staged parent indices per node of capacity
constexpr size_t smem_bytes(int n) {
  return size_t(n + 1) * (2 * 8 + 7 * 4) + size_t(n) * kParentsPerNode * 4 + 64;
}

__device__ __forceinline__ Nodes carve(unsigned char* p, int n) {
  Nodes x;
  x.mask = reinterpret_cast<unsigned long long*>(p);
  x.suffix = x.mask + n + 1;
  x.len = reinterpret_cast<int*>(x.suffix + n + 1);
  x.add = x.len + n + 1;
  x.page0 = x.add + n + 1;
  x.layer = x.page0 + n + 1;
  x.start = x.layer + n + 1;
  x.row0 = x.start + n + 1;
  x.ent0 = x.row0 + n + 1;
  x.parents = x.ent0 + n + 1;
  return x;
}

// dst[0 .. n] = exclusive running sum of f(0 .. n - 1); warp 0 only
template <typename F>
__device__ __forceinline__ void warp_scan(int* dst, int n, F f) {
  const int lane = threadIdx.x & 31;
  int base = 0;
#pragma unroll 1
  for (int v0 = 0; v0 < n; v0 += 32) {
    const int v = v0 + lane;
    const int own = v < n ? f(v) : 0;
    int x = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (v < n) dst[v] = base + x - own;
    base += __shfl_sync(0xffffffffu, x, 31);
  }
  if (lane == 0) dst[n] = base;
}

// What one node contributes to the block table of one group: rows [j0, j1) of the group are new tokens of the node itself.
struct NodeView {
  int len, tot, j0, j1, pages, same;  // same: leading pages of which every row sees all there is
  unsigned long long mask, own;       // rows that see the node; those of them that are its own new tokens
};
__device__ __forceinline__ unsigned long long bits_below(int n) { return n >= 64 ? ~0ull : (1ull << n) - 1; }

__device__ __forceinline__ NodeView view_of(const Nodes& x, int v, int g0, int g1) {
  NodeView w;
  w.len = x.len[v];
  w.tot = w.len + x.add[v];
  w.mask = x.mask[v];
  const int r0 = x.row0[v], r1 = x.row0[v + 1];
  const int a = max(r0, g0), b = min(r1, g1);
  w.j0 = a - r0;
  w.j1 = max(a, b) - r0;
  w.own = b > a ? bits_below(b - g0) & ~bits_below(a - g0) : 0;
  w.pages = w.mask ? (w.tot + PS - 1) / PS : 0;
  // new token j sees len + j + 1 tokens of its node, every other row sees all of them
  w.same = (w.own == 0 || w.len + w.j0 + 1 >= w.tot) ? w.pages : (w.len + w.j0 + 1) / PS;
  return w;
}
// Entries of page p >= same: one per count of visible tokens.  Own rows j in [jl, jh) see fewer than `full` tokens (a
// different count each); the rest of those that reach the page see `full`.
struct PageView {
  int full, jl, jh;
  unsigned long long rest;  // rows that see `full` tokens
};
__device__ __forceinline__ PageView page_of(const NodeView& w, int p, int g0, int row0) {
  PageView q;
  q.full = min(PS, w.tot - PS * p);
  q.jl = max(w.j0, PS * p - w.len);
  q.jh = max(q.jl, min(w.j1, PS * p + q.full - w.len - 1));
  const int jf = min(w.j1, max(w.j0, PS * p + q.full - w.len - 1));  // first own row that sees `full`
  q.rest = (w.mask & ~w.own) | (jf < w.j1 ? bits_below(row0 + w.j1 - g0) & ~bits_below(row0 + jf - g0) : 0);
  return q;
}
__device__ __forceinline__ int entries_of(const Nodes& x, int v, int g0, int g1) {
  const NodeView w = view_of(x, v, g0, g1);
  int n = w.same;
#pragma unroll 1
  for (int p = w.same; p < w.pages; ++p) {
    const PageView q = page_of(w, p, g0, x.row0[v]);
    n += q.jh - q.jl + (q.rest != 0);
    if (PS * p > w.len + w.j1 && q.rest == 0) break;  // tokens of later groups: nobody here sees them
  }
  return n;
}

__global__ void __launch_bounds__(NT) step_tables_kernel(const __grid_constant__ BuildArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int s_err;
  __shared__ unsigned long long s_sum[8];  // rows, groups, entries, tiles before this request; the same in all
  __shared__ int s_run[2], s_status;       // entries and tiles of the request's groups so far; largest error of all requests
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x;
  const mv_step_tables& t = a.t;
  if (tid == 0) s_err = s_status = 0;
  if (tid < 8) s_sum[tid] = 0;
  if (tid < 2) s_run[tid] = 0;
  __syncthreads();
  auto fail = [&](mv_status e) { atomicMax(&s_err, int(e)); };
  mv::grid_dependency_launch_dependents();

  // ---- the request's nodes, checked by both launches (the second runs ahead of the first one's end)
  const int cap = a.s.max_req_nodes;
  Nodes x = carve(smem, cap);
  int lo = 0, n = 0;
  const int32_t* plist = nullptr;
  if (r < a.b.n_req) {
    lo = a.b.node_off[r];
    const int hi = a.b.node_off[r + 1];
    n = hi - lo;
    mv_status range = MV_OK;
    if (lo < 0 || hi < lo || hi > a.s.n_nodes || (r == 0 && lo != 0)) range = MV_ERR_INVALID_ARG;
    else if (n > cap) range = MV_ERR_UNSUPPORTED;
    if (range != MV_OK) {
      n = 0;
      if (tid == 0) fail(range);
    }
    const int e_lo = n > 0 ? a.b.parent_off[lo] : 0, e_hi = n > 0 ? a.b.parent_off[hi] : 0;
    const bool lists_ok = e_lo >= 0 && e_hi >= e_lo && e_hi <= a.s.n_parents;
    const bool staged = lists_ok && e_hi - e_lo <= kParentsPerNode * cap;
    if (staged)
      for (int e = e_lo + tid; e < e_hi; e += NT) x.parents[e - e_lo] = a.b.parent_idx[e];
    plist = staged ? x.parents - e_lo : a.b.parent_idx;
#pragma unroll 1
    for (int v = tid; v < n; v += NT) {
      const int g = lo + v;
      const int len = a.b.node_len[g], add = a.b.node_new[g];
      const int p0 = a.b.page_off[g], p1 = a.b.page_off[g + 1], e0 = a.b.parent_off[g], e1 = a.b.parent_off[g + 1];
      x.len[v] = len;
      x.add[v] = add;
      x.page0[v] = p0;
      if (len < 0 || add < 0 || p0 < 0 || p1 < p0 || p1 > a.s.n_pages || e0 < e_lo || e1 < e0 || e1 > e_hi || !lists_ok) {
        fail(MV_ERR_INVALID_ARG);
      } else {
        if (int64_t(len) + add > int64_t(p1 - p0) * PS) fail(MV_ERR_PAGE_CAPACITY);
        if (int64_t(len) + add > kMaxTokens || (a.blocks && add > kMaxNew)) fail(MV_ERR_UNSUPPORTED);
      }
    }
    if (tid == 0) x.row0[0] = 0;
    __syncthreads();
    if (s_err == 0) {  // the offsets are sound: parent lists and page ids
#pragma unroll 1
      for (int v = tid; v < n; v += NT)
#pragma unroll 1
        for (int e = a.b.parent_off[lo + v]; e < a.b.parent_off[lo + v + 1]; ++e)
          if (plist[e] < 0 || plist[e] >= v) fail(MV_ERR_NOT_TOPOLOGICAL);
      // (page ids are only passed on here: one launch is enough to check them)
      const int q0 = n > 0 ? x.page0[0] : 0, q1 = n > 0 && (a.mode & COUNT) ? a.b.page_off[hi] : 0;
      for (int q = q0 + tid; q < q1; q += NT) {
        const int page = a.b.page_idx[q];
        if (page < 0 || page >= a.s.num_pages) fail(MV_ERR_INVALID_ARG);
      }
    }
  }
  __syncthreads();
  const bool sound = s_err == 0;
  __syncthreads();  // s_err may change again below
  if (!sound) n = 0;

  // ---- layers and positions, node after node (parents come first): warp 0, a lane per parent
  if (warp == 0) {
    const bool aligned = a.b.pos_mode == MV_POS_FRONTIER_ALIGNED;
#pragma unroll 1
    for (int v = 0; v < n; ++v) {
      int L = 0, st = 0;
#pragma unroll 1
      for (int e = a.b.parent_off[lo + v] + lane; e < a.b.parent_off[lo + v + 1]; e += 32) {
        const int p = plist[e];
        L = max(L, x.layer[p] + 1);
        if (!aligned) st = max(st, int(min(int64_t(x.start[p]) + x.len[p] + x.add[p], kMaxTokens)));
      }
      L = __reduce_max_sync(0xffffffffu, L);
      st = __reduce_max_sync(0xffffffffu, st);
      if (lane == 0) {
        x.layer[v] = L;
        x.start[v] = st;
      }
      __syncwarp();
    }
    if (aligned && n > 0) {
      // one start per layer: a layer ends at its start plus its longest node (ent0 holds the longest node, then the start)
      for (int k = lane; k <= n; k += 32) x.ent0[k] = 0;
      __syncwarp();
      for (int v = lane; v < n; v += 32) atomicMax(&x.ent0[x.layer[v]], x.len[v] + x.add[v]);
      __syncwarp();
      if (lane == 0) {
        int64_t at = 0;
        for (int k = 0; k < n; ++k) {
          const int64_t longest = x.ent0[k];
          x.ent0[k] = int(at);
          at = min(at + longest, kMaxTokens);
        }
      }
      __syncwarp();
      for (int v = lane; v < n; v += 32) x.start[v] = x.ent0[x.layer[v]];
    }
    int64_t sum = 0;
    for (int v = lane; v < n; v += 32) {
      sum += x.add[v];
      if (int64_t(x.start[v]) + x.len[v] + x.add[v] > kMaxTokens) fail(MV_ERR_UNSUPPORTED);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (sum > t.max_rows) fail(MV_ERR_WORKSPACE);
    warp_scan(x.row0, n, [&](int v) { return x.add[v]; });
  }
  __syncthreads();
  const int bad = s_err;
  const int rows = bad == 0 && r < a.b.n_req ? x.row0[n] : 0;
  if (a.mode == COUNT && bad != 0) {
    if (tid == 0) {
      a.req[r] = ReqCounts{0, 0, 0, 0};
      a.err[r] = bad;
    }
    return;
  }

  const int per = t.rows_per_group;
  const int groups = a.blocks ? (rows + per - 1) / per : 0;
  long long row_base = 0, group_base = 0, ent_base = 0, tile_base = 0;
#pragma unroll 1
  for (int phase = (a.mode & COUNT) ? COUNT : WRITE; phase <= ((a.mode & WRITE) ? WRITE : COUNT); phase += WRITE - COUNT) {
    const bool write = phase == WRITE;
    if (write) {
      // ---- where this request's part begins, and the sums over all requests
      if (a.mode == WRITE) {
        mv::grid_dependency_wait();  // the first launch has completed
        unsigned long long c[8] = {};
        int worst = 0;
#pragma unroll 1
        for (int i = tid; i < a.b.n_req; i += NT) {
          const int4 q = __ldcg(reinterpret_cast<const int4*>(a.req) + i);
          if (i < r) { c[0] += q.x; c[1] += q.y; c[2] += q.z; c[3] += q.w; }
          c[4] += q.x; c[5] += q.y; c[6] += q.z; c[7] += q.w;
          worst = max(worst, __ldcg(a.err + i));
        }
        worst = __reduce_max_sync(0xffffffffu, worst);
        if (lane == 0 && worst) atomicMax(&s_status, worst);
#pragma unroll
        for (int k = 0; k < 8; ++k) {  // a warp's sum in two halves (each thread's sum is below 2^47)
          const unsigned low = __reduce_add_sync(0xffffffffu, unsigned(c[k] & 0xffffffu)), high = __reduce_add_sync(0xffffffffu, unsigned(c[k] >> 24));
          if (lane == 0) atomicAdd(&s_sum[k], (static_cast<unsigned long long>(high) << 24) + low);
        }
      } else if (tid == 0 && r < a.b.n_req) {  // the only request
        s_sum[4] = rows;
        s_sum[5] = groups;
        s_sum[6] = s_run[0];
        s_sum[7] = s_run[1];
        s_status = max(bad, s_err);
        s_run[0] = s_run[1] = 0;
      }
      __syncthreads();
      int status = s_status;
      if (status == 0 && (s_sum[4] > t.max_rows || (a.blocks && (s_sum[5] > t.max_groups || s_sum[6] > t.max_entries)))) status = MV_ERR_WORKSPACE;
      long long rows_all = 0, groups_all = 0, ents_all = 0, tiles_all = 0;
      if (status == 0) {
        row_base = s_sum[0]; group_base = s_sum[1]; ent_base = s_sum[2]; tile_base = s_sum[3];
        rows_all = s_sum[4]; groups_all = s_sum[5]; ents_all = s_sum[6]; tiles_all = s_sum[7];
      }
      // what lies behind the step: unused rows, empty groups (shared out over the CTAs)
      const int64_t me = int64_t(r) * NT + tid, all = int64_t(gridDim.x) * NT;
#pragma unroll 1
      for (int64_t i = rows_all + me; i < t.max_rows; i += all) {
        t.pos_id[i] = 0;
        t.slot[i] = -1;
      }
      if (a.blocks)
#pragma unroll 1
        for (int64_t i = groups_all + me; i <= t.max_groups; i += all) {
          t.group_row_off[i] = int(rows_all);
          t.group_ent_off[i] = int(ents_all);
          t.group_tile_off[i] = int(tiles_all);
        }
      if (r == 0 && tid < 8) t.counts[tid] = tid == 0 ? int(rows_all) : tid == 1 ? int(groups_all) : tid == 2 ? int(ents_all) : tid == 3 ? int(tiles_all) : tid == 4 ? status : 0;
      if (status != 0 || r >= a.b.n_req) return;  // (an empty batch has a grid of one CTA)
#pragma unroll 1
      for (int i = tid; i < rows; i += NT) {
        int v = 0;
#pragma unroll 1
        for (int step = 1 << (31 - __clz(max(n, 1))); step > 0; step >>= 1)  // last node whose first row is at most i (nodes without rows are passed over)
          if (v + step < n && x.row0[v + step] <= i) v += step;
        const int tok = x.len[v] + (i - x.row0[v]);
        t.pos_id[row_base + i] = x.start[v] + tok;
        t.slot[row_base + i] = int64_t(a.b.page_idx[x.page0[v] + tok / PS]) * PS + tok % PS;
      }
    }

    // ---- groups of rows
#pragma unroll 1
    for (int k = 0; k < (bad == 0 ? groups : 0); ++k) {
      const int g0 = k * per, g1 = min(rows, g0 + per);
      if (warp == 0 && !(write && groups == 1 && (a.mode & COUNT))) {  // (one group: the count has left its masks)
#pragma unroll 1
        for (int v = lane; v < n; v += 32) {
          const int b0 = max(x.row0[v], g0), b1 = min(x.row0[v + 1], g1);
          x.mask[v] = b1 > b0 ? bits_below(b1 - g0) & ~bits_below(b0 - g0) : 0;
        }
        if (a.b.vis_mode == MV_VIS_ANCESTORS) {
          __syncwarp();
#pragma unroll 1
          for (int v = n - 1; v > 0; --v) {
            const unsigned long long m = x.mask[v];
            if (m == 0) continue;
#pragma unroll 1
            for (int e = a.b.parent_off[lo + v] + lane; e < a.b.parent_off[lo + v + 1]; e += 32) atomicOr(&x.mask[plist[e]], m);
            __syncwarp();
          }
        } else {
          for (int v = lane; v <= n; v += 32) x.suffix[v] = 0;
          __syncwarp();
          for (int v = lane; v < n; v += 32) atomicOr(&x.suffix[x.layer[v]], x.mask[v]);
          __syncwarp();
          if (lane == 0)
#pragma unroll 1
            for (int L = n - 1; L >= 0; --L) x.suffix[L] |= x.suffix[L + 1];
          __syncwarp();
          for (int v = lane; v < n; v += 32) x.mask[v] |= x.suffix[x.layer[v] + 1];
        }
      }
      __syncthreads();
#pragma unroll 1
      for (int v = tid; v < n; v += NT) x.ent0[v] = entries_of(x, v, g0, g1);
      __syncthreads();
      if (warp == 0) warp_scan(x.ent0, n, [&](int v) { return x.ent0[v]; });
      __syncthreads();
      const int found = x.ent0[n];
      if (write) {
        if (tid == 0) {
          t.group_row_off[group_base + k] = int(row_base) + g0;
          t.group_ent_off[group_base + k] = int(ent_base) + s_run[0];
          t.group_tile_off[group_base + k] = int(tile_base) + s_run[1];
        }
        int4* const dst = reinterpret_cast<int4*>(t.entries) + ent_base + s_run[0];
#pragma unroll 1
        for (int i = tid; i < found; i += NT) {
          int v = 0;
#pragma unroll 1
          for (int step = 1 << (31 - __clz(max(n, 1))); step > 0; step >>= 1)  // last node whose first entry is at most i
            if (v + step < n && x.ent0[v + step] <= i) v += step;
          const NodeView w = view_of(x, v, g0, g1);
          int at = i - x.ent0[v], p = at, tokens;
          unsigned long long m = w.mask;
          if (at < w.same) {
            tokens = min(PS, w.tot - PS * p);
          } else {
            at -= w.same;
            p = w.same;
            PageView q = page_of(w, p, g0, x.row0[v]);
            while (p + 1 < w.pages) {
              const int here = q.jh - q.jl + (q.rest != 0);
              if (at < here) break;
              at -= here;
              q = page_of(w, ++p, g0, x.row0[v]);
            }
            if (at < q.jh - q.jl) {
              tokens = w.len + q.jl + at + 1 - PS * p;
              m = 1ull << (x.row0[v] + q.jl + at - g0);
            } else {
              tokens = q.full;
              m = q.rest;
            }
          }
          dst[i] = make_int4(a.b.page_idx[x.page0[v] + p], tokens, int(uint32_t(m)), int(uint32_t(m >> 32)));
        }
      }
      __syncthreads();
      if (tid == 0) {
        s_run[0] += found;
        s_run[1] += (found + 7) / 8;
        if (s_run[0] > t.max_entries) fail(MV_ERR_WORKSPACE);  // counting: stop before the running sums could overflow
      }
      __syncthreads();
      if (!write && s_err != 0) break;
    }
  }
  if (a.mode == COUNT && tid == 0) {
    a.req[r] = s_err == 0 ? ReqCounts{rows, groups, s_run[0], s_run[1]} : ReqCounts{0, 0, 0, 0};
    a.err[r] = s_err;
  }
}

}  // namespace

extern "C" size_t mv_step_tables_workspace_bytes(int32_t n_req) {
  const size_t n = size_t(n_req > 0 ? n_req : 0);
  return ((n * (sizeof(ReqCounts) + sizeof(int32_t)) + 255) & ~size_t(255)) + 256;
}

extern "C" mv_status mv_step_tables_build(const mv_dag_batch* b, const mv_step_shape* s, const mv_step_tables* t, void* workspace,
                                          size_t workspace_bytes, void* cuda_stream) {
  mv::NvtxRange nvtx_range("mv_step_tables_build");
  if (!b || !s || !t) return MV_ERR_INVALID_ARG;
  if (b->n_req < 0 || s->n_nodes < 0 || s->n_parents < 0 || s->n_pages < 0 || s->num_pages < 0) return MV_ERR_INVALID_ARG;
  if (b->page_size != PS) return MV_ERR_INVALID_ARG;
  if (b->vis_mode != MV_VIS_ANCESTORS && b->vis_mode != MV_VIS_LAYERWISE) return MV_ERR_INVALID_ARG;
  if (b->pos_mode != MV_POS_MAX_PARENT_END && b->pos_mode != MV_POS_FRONTIER_ALIGNED) return MV_ERR_INVALID_ARG;
  if (b->n_req > 0 && !b->node_off) return MV_ERR_INVALID_ARG;
  if (s->n_nodes > 0 && (!b->node_len || !b->node_new || !b->parent_off || !b->page_off)) return MV_ERR_INVALID_ARG;
  if ((s->n_parents > 0 && !b->parent_idx) || (s->n_pages > 0 && !b->page_idx)) return MV_ERR_INVALID_ARG;
  if (s->max_req_nodes < 1 || s->max_req_nodes > MV_STEP_MAX_REQ_NODES) return MV_ERR_UNSUPPORTED;
  if (t->max_rows < 0 || t->max_groups < 0 || t->max_entries < 0 || !t->counts) return MV_ERR_INVALID_ARG;
  if (t->max_rows > 0 && (!t->pos_id || !t->slot)) return MV_ERR_INVALID_ARG;
  const bool blocks = t->max_groups > 0;
  if (blocks) {
    if (t->rows_per_group < 1 || t->rows_per_group > 64) return MV_ERR_UNSUPPORTED;
    if (!t->group_row_off || !t->group_ent_off || !t->group_tile_off) return MV_ERR_INVALID_ARG;
    if (t->max_entries > 0 && (!t->entries || (reinterpret_cast<uintptr_t>(t->entries) & 15) != 0)) return MV_ERR_INVALID_ARG;
  }
  if (!workspace || workspace_bytes < mv_step_tables_workspace_bytes(b->n_req) || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
    return MV_ERR_WORKSPACE;
  BuildArgs a;
  a.b = *b;
  a.s = *s;
  a.t = *t;
  a.req = static_cast<ReqCounts*>(workspace);
  a.err = reinterpret_cast<int32_t*>(a.req + b->n_req);
  a.blocks = blocks ? 1 : 0;
  static std::atomic<uint64_t> opted{0};  // per device
  const size_t smem = smem_bytes(s->max_req_nodes);
  constexpr size_t kStatic = 1024;  // the kernel's static arrays (under a hundred bytes) count in the 48 KB too
  if (smem + kStatic > 48 * 1024 && !mv::opt_in_smem(step_tables_kernel, int(smem_bytes(MV_STEP_MAX_REQ_NODES)), opted)) return MV_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(b->n_req > 0 ? b->n_req : 1), 1, 1);
  cfg.blockDim = dim3(NT, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  const bool two = b->n_req > 1;
  if (two) {
    a.mode = COUNT;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, step_tables_kernel, a);
    mv::g_launches++;
    if (e != cudaSuccess) {
      (void)cudaGetLastError();
      return MV_ERR_CUDA;
    }
  }
  // the second launch may become resident while the first runs: its analysis reads only the caller's arrays
  a.mode = two ? WRITE : COUNT | WRITE;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = two ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, step_tables_kernel, a);
  mv::g_launches++;
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return MV_ERR_CUDA;
  }
  return MV_OK;
}

extern "C" mv_status mv_step_tables_read_status(const mv_step_tables* t, void* cuda_stream, int32_t* status) {
  if (!t || !t->counts || !status) return MV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (cudaMemcpyAsync(status, t->counts + 4, sizeof(int32_t), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaStreamSynchronize(st) != cudaSuccess) {
    (void)cudaGetLastError();
    return MV_ERR_CUDA;
  }
  return MV_OK;
}
