// Tables of a step with any number of new tokens per node, built on the device: per receiving node the list of pages its tokens
// see (Eq. 3 / Sec. 4.3 visibility; its own pages last), and query tiles of at most rows_per_tile consecutive new tokens.
//
// Integers only.  One CTA per request, two launches of the same kernel: the first leaves every request's counts (rows, tiles, entries,
// key tiles, error), the second sums the counts of the requests before its own and writes; a batch of one request takes one launch that
// does both.  The receiving nodes are taken 64 at a time: a sweep over the nodes from last to first hands the set of receiving
// nodes that see a node on to its parents (parents have smaller indices), one 64-bit OR per edge; then a team of warps per
// receiving node walks the nodes that it sees and copies their page ids.
// Bound by latency: launches, dependent loads, sweeps over the request's nodes.  One request, 600 new tokens behind 24, 7.8 us
// in a graph, 8.2 us called; 128 requests of 512 to 16384 tokens, two to eight branches each and new tokens on all of them, 17.6 and
// 19.4 us (what they read and write takes 0.3 us at the measured copy rate).
#include "common.cuh"
#include "trace.h"

namespace {

constexpr int NT = 256, WARPS = NT / 32;
constexpr int PS = 16;
constexpr int KEYS = 8;  // pages of a key tile
constexpr int64_t kMaxTokens = int64_t(1) << 30;  // of one node
constexpr int BATCH = 64;                         // receiving nodes at a time
constexpr int kParentsPerNode = 4;

enum Mode { COUNT = 1, WRITE = 2 };

struct BuildArgs {
  mv_dag_batch b;  // device pointers
  mv_step_shape s;
  mv_chunk_tables t;
  int4* req;       // [n_req] rows, tiles, entries, key tiles
  int32_t* err;    // [n_req]
  int mode;
};

struct Nodes {
  unsigned long long* mask;  // receiving nodes of the batch that see the node
  int *len, *add, *page0, *layer, *row0, *recv;  // row0 [n + 1]; recv: the receiving nodes in order
  int* parents;
};
constexpr size_t smem_bytes(int n) { return size_t(n + 1) * (8 + 6 * 4) + size_t(n) * kParentsPerNode * 4 + 64; }
__device__ __forceinline__ Nodes carve(unsigned char* p, int n) {
  Nodes x;
  x.mask = reinterpret_cast<unsigned long long*>(p);
  x.len = reinterpret_cast<int*>(x.mask + n + 1);
  x.add = x.len + n + 1;
  x.page0 = x.add + n + 1;
  x.layer = x.page0 + n + 1;
  x.row0 = x.layer + n + 1;
  x.recv = x.row0 + n + 1;
  x.parents = x.recv + n + 1;
  return x;
}
__device__ __forceinline__ int pages_of(const Nodes& x, int v) { return (x.len[v] + x.add[v] + PS - 1) / PS; }
__device__ __forceinline__ int scan_up(int x) {  // inclusive, over a warp
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// key tiles that tile j of a node walks
__device__ __forceinline__ int units_of(int64_t before, int len, int add, int per, int j) {
  const int64_t own = (int64_t(len) + min(int64_t(add), int64_t(j + 1) * per) + PS - 1) / PS;
  return int((before + own + KEYS - 1) / KEYS);
}

__global__ void __launch_bounds__(NT) chunk_tables_kernel(const __grid_constant__ BuildArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int s_err, s_status, s_recv;
  __shared__ unsigned long long s_sum[8];   // rows, tiles, entries, key tiles before this request; the same in all
  __shared__ long long s_run[3];            // tiles, entries, key tiles of the request's receiving nodes so far
  __shared__ long long s_ent[BATCH], s_unit[BATCH];
  __shared__ int s_before[BATCH], s_tile[BATCH];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x;
  const mv_chunk_tables& t = a.t;
  if (tid == 0) s_err = s_status = s_recv = 0;
  if (tid < 8) s_sum[tid] = 0;
  if (tid < 3) s_run[tid] = 0;
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
        if (int64_t(len) + add > kMaxTokens) fail(MV_ERR_UNSUPPORTED);
      }
    }
    __syncthreads();
    if (s_err == 0) {  // the offsets are sound: parent lists and page ids
#pragma unroll 1
      for (int v = tid; v < n; v += NT) {
#pragma unroll 1
        for (int e = a.b.parent_off[lo + v]; e < a.b.parent_off[lo + v + 1]; ++e)
          if (plist[e] < 0 || plist[e] >= v) fail(MV_ERR_NOT_TOPOLOGICAL);
      }
      // (page ids are only passed on here: one launch is enough to check them)
      const int q0 = n > 0 ? x.page0[0] : 0, q1 = n > 0 && (a.mode & COUNT) ? a.b.page_off[hi] : 0;
#pragma unroll 4
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

  // ---- rows, receiving nodes, layers: warp 0
  if (warp == 0) {
    int rows = 0, recv = 0;
    int64_t all = 0;
#pragma unroll 1
    for (int v0 = 0; v0 < n; v0 += 32) {
      const int v = v0 + lane, add = v < n ? x.add[v] : 0;
      const int upto = scan_up(add);  // (up to 32 * 2^30: what passes 32 bits is refused below)
      if (v < n) x.row0[v] = rows + upto - add;
      const unsigned m = __ballot_sync(0xffffffffu, add > 0);
      if (add > 0) x.recv[recv + __popc(m & ((1u << lane) - 1))] = v;
      recv += __popc(m);
      rows += __shfl_sync(0xffffffffu, upto, 31);
      all += add;
    }
    if (lane == 0) {
      x.row0[n] = rows;
      s_recv = recv;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    if (lane == 0 && all > t.max_rows) fail(MV_ERR_WORKSPACE);
    if (a.b.vis_mode == MV_VIS_LAYERWISE)
#pragma unroll 1
      for (int v = 0; v < n; ++v) {
        int L = 0;
#pragma unroll 1
        for (int e = a.b.parent_off[lo + v] + lane; e < a.b.parent_off[lo + v + 1]; e += 32) L = max(L, x.layer[plist[e]] + 1);
        L = __reduce_max_sync(0xffffffffu, L);
        if (lane == 0) x.layer[v] = L;
        __syncwarp();
      }
  }
  __syncthreads();
  int bad = s_err;
  __syncthreads();
  const int rows = bad == 0 ? x.row0[n] : 0, recv = bad == 0 ? s_recv : 0;
  const int per = t.rows_per_tile;
  long long row_base = 0, tile_base = 0, ent_base = 0, unit_base = 0;
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
          const int4 q = __ldcg(a.req + i);
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
        for (int k = 0; k < 3; ++k) s_sum[5 + k] = s_run[k];
        s_status = s_err;
      }
      __syncthreads();
      if (tid < 3) s_run[tid] = 0;
      int status = s_status;
      if (status == 0 && (s_sum[4] > t.max_rows || s_sum[5] > t.max_tiles || s_sum[6] > t.max_entries)) status = MV_ERR_WORKSPACE;
      if (status == 0 && s_sum[7] > INT32_MAX) status = MV_ERR_UNSUPPORTED;
      if (r == 0 && tid < 8) t.counts[tid] = tid < 4 ? (status == 0 ? int(s_sum[4 + tid]) : 0) : tid == 4 ? status : 0;
      if (status != 0 || r >= a.b.n_req) return;  // (an empty batch has a grid of one CTA)
      row_base = s_sum[0]; tile_base = s_sum[1]; ent_base = s_sum[2]; unit_base = s_sum[3];
      __syncthreads();
    }

    // ---- receiving nodes, BATCH at a time
#pragma unroll 1
    for (int k0 = 0; k0 < recv; k0 += BATCH) {
      const int k1 = min(recv, k0 + BATCH), here = k1 - k0;
      if (!(write && recv <= BATCH && (a.mode & COUNT))) {  // (one batch: the count has left its masks)
        if (warp == 0) {
          for (int v = lane; v < n; v += 32) x.mask[v] = 0;
          __syncwarp();
          for (int k = k0 + lane; k < k1; k += 32) x.mask[x.recv[k]] = 1ull << (k - k0);
          __syncwarp();
          if (a.b.vis_mode == MV_VIS_ANCESTORS) {
#pragma unroll 1
            for (int v = n - 1; v > 0; --v) {
              const unsigned long long m = x.mask[v];
              if (m == 0) continue;
#pragma unroll 1
              for (int e = a.b.parent_off[lo + v] + lane; e < a.b.parent_off[lo + v + 1]; e += 32) atomicOr(&x.mask[plist[e]], m);
              __syncwarp();
            }
          } else {
#pragma unroll 1
            for (int v = lane; v < n; v += 32) {
              unsigned long long m = 0;
#pragma unroll 1
              for (int k = 0; k < here; ++k)
                if (x.layer[x.recv[k0 + k]] > x.layer[v] || x.recv[k0 + k] == v) m |= 1ull << k;
              x.mask[v] = m;
            }
          }
        }
        __syncthreads();
      }
      // counts: a warp per receiving node
#pragma unroll 1
      for (int k = warp; k < here; k += WARPS) {
        const int own = x.recv[k0 + k], len = x.len[own], add = x.add[own];
        long long before = 0;
#pragma unroll 1
        for (int u = lane; u < n; u += 32)
          if (((x.mask[u] >> k) & 1) && u != own) before += pages_of(x, u);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
        const int tiles = int((int64_t(add) + per - 1) / per);
        long long units = 0;
#pragma unroll 1
        for (int j = lane; j < tiles; j += 32) units += units_of(before, len, add, per, j);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) units += __shfl_xor_sync(0xffffffffu, units, o);
        if (lane == 0) {
          s_before[k] = int(min(before, (long long)INT32_MAX));
          s_ent[k] = before + pages_of(x, own);
          s_tile[k] = tiles;
          s_unit[k] = units;
        }
      }
      __syncthreads();
      const long long tiles0 = s_run[0], ents0 = s_run[1], units0 = s_run[2];
      if (write) {
        int team = 1;  // warps per receiving node
        while (team < WARPS && 2 * team * here <= WARPS) team *= 2;
        const int member = warp % team;
#pragma unroll 1
        for (int k = warp / team; k < here; k += WARPS / team) {
          long long e = ent_base + ents0, tile = tile_base + tiles0, unit = unit_base + units0;
          for (int i = 0; i < k; ++i) {
            e += s_ent[i];
            tile += s_tile[i];
            unit += s_unit[i];
          }
          const int own = x.recv[k0 + k], len = x.len[own], add = x.add[own], before = s_before[k];
          // tiles
          if (member == 0) {
            int4* const dst = reinterpret_cast<int4*>(t.tiles) + tile * 2;
            long long at = unit;
#pragma unroll 1
            for (int j0 = 0; j0 < s_tile[k]; j0 += 32) {
              const int j = j0 + lane;
              const bool there = j < s_tile[k];
              const int units = there ? units_of(before, len, add, per, j) : 0;
              // 32 tiles may walk more than 2^31 key tiles only in steps that were refused above
              const int upto = scan_up(units);
              if (there) {
                dst[2 * j] = make_int4(int(row_base) + x.row0[own] + j * per, min(per, add - j * per), int(e), before);
                dst[2 * j + 1] = make_int4(len + j * per, int(at + upto - units), units, 0);
              }
              at += __shfl_sync(0xffffffffu, upto, 31);
            }
          }
          // pages: the nodes it sees in order, its own at the end
          int2* out = reinterpret_cast<int2*>(t.entries) + e;
          auto copy = [&](int u) {
            const int tot = x.len[u] + x.add[u], pages = (tot + PS - 1) / PS;
            const int32_t* const ids = a.b.page_idx + x.page0[u];
#pragma unroll 4
            for (int p = member * 32 + lane; p < pages; p += team * 32) out[p] = make_int2(__ldg(ids + p), min(PS, tot - PS * p));
            out += pages;
          };
#pragma unroll 1
          for (int u0 = 0; u0 < n; u0 += 32) {
            const int u = u0 + lane;
            unsigned m = __ballot_sync(0xffffffffu, u < n && u != own && ((x.mask[u] >> k) & 1));
#pragma unroll 1
            for (; m; m &= m - 1) copy(u0 + __ffs(m) - 1);
          }
          copy(own);
        }
      }
      __syncthreads();
      if (tid == 0) {
        for (int i = 0; i < here; ++i) {
          s_run[0] += s_tile[i];
          s_run[1] += s_ent[i];
          s_run[2] += s_unit[i];
        }
        if (s_run[0] > t.max_tiles || s_run[1] > t.max_entries) fail(MV_ERR_WORKSPACE);
        if (s_run[2] > INT32_MAX) fail(MV_ERR_UNSUPPORTED);
      }
      __syncthreads();
      if (!write && s_err != 0) break;
    }
  }
  if (a.mode == COUNT && tid == 0) {
    a.req[r] = s_err == 0 ? make_int4(rows, int(s_run[0]), int(s_run[1]), int(s_run[2])) : make_int4(0, 0, 0, 0);
    a.err[r] = s_err;
  }
}

}  // namespace

extern "C" size_t mv_chunk_tables_workspace_bytes(int32_t n_req) {
  const size_t n = size_t(n_req > 0 ? n_req : 0);
  return ((n * (sizeof(int4) + sizeof(int32_t)) + 255) & ~size_t(255)) + 256;
}

extern "C" mv_status mv_chunk_tables_build(const mv_dag_batch* b, const mv_step_shape* s, const mv_chunk_tables* t, void* workspace,
                                           size_t workspace_bytes, void* cuda_stream) {
  mv::NvtxRange nvtx_range("mv_chunk_tables_build");
  if (!b || !s || !t) return MV_ERR_INVALID_ARG;
  if (b->n_req < 0 || s->n_nodes < 0 || s->n_parents < 0 || s->n_pages < 0 || s->num_pages < 0) return MV_ERR_INVALID_ARG;
  if (b->page_size != PS) return MV_ERR_INVALID_ARG;
  if (b->vis_mode != MV_VIS_ANCESTORS && b->vis_mode != MV_VIS_LAYERWISE) return MV_ERR_INVALID_ARG;
  if (b->n_req > 0 && !b->node_off) return MV_ERR_INVALID_ARG;
  if (s->n_nodes > 0 && (!b->node_len || !b->node_new || !b->parent_off || !b->page_off)) return MV_ERR_INVALID_ARG;
  if ((s->n_parents > 0 && !b->parent_idx) || (s->n_pages > 0 && !b->page_idx)) return MV_ERR_INVALID_ARG;
  if (s->max_req_nodes < 1 || s->max_req_nodes > MV_STEP_MAX_REQ_NODES) return MV_ERR_UNSUPPORTED;
  if (t->max_rows < 0 || t->max_tiles < 0 || t->max_entries < 0 || !t->counts) return MV_ERR_INVALID_ARG;
  if (t->rows_per_tile < 1 || t->rows_per_tile > 256) return MV_ERR_UNSUPPORTED;
  if ((t->max_tiles > 0 && !t->tiles) || (t->max_entries > 0 && !t->entries)) return MV_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(t->tiles) & 15) || (reinterpret_cast<uintptr_t>(t->entries) & 15) || (reinterpret_cast<uintptr_t>(t->counts) & 3))
    return MV_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < mv_chunk_tables_workspace_bytes(b->n_req) || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
    return MV_ERR_WORKSPACE;
  BuildArgs a;
  a.b = *b;
  a.s = *s;
  a.t = *t;
  a.req = static_cast<int4*>(workspace);
  a.err = reinterpret_cast<int32_t*>(a.req + b->n_req);
  static std::atomic<uint64_t> opted{0};  // per device
  const size_t smem = smem_bytes(s->max_req_nodes);
  constexpr size_t kStatic = 4096;  // the kernel's static arrays count in the 48 KB too
  if (smem + kStatic > 48 * 1024 && !mv::opt_in_smem(chunk_tables_kernel, int(smem_bytes(MV_STEP_MAX_REQ_NODES)), opted)) return MV_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(b->n_req > 0 ? b->n_req : 1), 1, 1);
  cfg.blockDim = dim3(NT, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  const bool two = b->n_req > 1;
  if (two) {
    a.mode = COUNT;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, chunk_tables_kernel, a);
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, chunk_tables_kernel, a);
  mv::g_launches++;
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return MV_ERR_CUDA;
  }
  return MV_OK;
}

extern "C" mv_status mv_chunk_tables_read_status(const mv_chunk_tables* t, void* cuda_stream, int32_t* status) {
  if (!t || !t->counts || !status) return MV_ERR_INVALID_ARG;
  if (cudaMemcpyAsync(status, t->counts + 4, sizeof(int32_t), cudaMemcpyDeviceToHost, static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess ||
      cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess) {
    (void)cudaGetLastError();
    return MV_ERR_CUDA;
  }
  return MV_OK;
}
