// Decode attention over the block-scaled 8-bit cache: the merge of cut streams and the entry point (the attention kernel and the
// mathematics: decode_attn_fp8_blk_tc.cu).
#include "blk_stream.cuh"
#include "trace.h"

namespace mv {
mv_status decode_blk_tc(const blk::Args& a, int head_dim, cudaStream_t st);
}

namespace {

using bf16 = __nv_bfloat16;
using mv::blk::Args;
using mv::blk::MAXQV;
using mv::blk::PS;
using mv::blk::SHARES;

// Merge of the cut streams:
//   out = sum_i w_i O_i / sum_i w_i l_i,  w_i = 2^(m_i - max m) over the stream's parts i.
// A job is a q-vector of a cut stream.  Every CTA reads the shares' records (one round trip to memory, all loads at once),
// counts the jobs and takes its own.  Where there are fewer jobs than warps, several warps deal out the parts of one among
// themselves; where there are more, a warp takes two at a time.
// Bound by latency: the records, the references and parts, and the instructions' own arrival; the CTAs start as those of the
// attention kernel leave their registers, so there are no more of them than fit at once.  Against CTAs that belong to
// a share each, calls of one request of 8K tokens and 4 KV heads 34 -> 18 us, of 64K tokens and 2 KV heads 39 -> 22.5; against one
// job at a time, 128 mixed requests 439 -> 432.  With 148 CTAs a short request 15.0 instead of 15.2 us, mixed ones 113 to 116.
constexpr int MERGE_WARPS = 8, ACCS = 4, ACC_LOADS = 2, PAIR = 2, MERGE_CTAS = SHARES;
static_assert(SHARES % 2 == 0 && SHARES <= MERGE_WARPS * 64, "a thread takes two shares");
template <int D>
__global__ void __launch_bounds__(MERGE_WARPS * 32) decode_blk_merge_kernel(const Args a) {
  constexpr int VEC = D / 32;  // elements of the head vector per lane
  __shared__ float so[MERGE_WARPS][D], ssum[MERGE_WARPS], stop[MERGE_WARPS];
  __shared__ int4 started[SHARES];   // the stream that starts in a share and ends in a later one
  __shared__ int continued[SHARES];  // the stream that started in an earlier share
  __shared__ int before[SHARES];     // jobs of the shares before
  __shared__ int of_warp[MERGE_WARPS], cut_in_warp[MERGE_WARPS];
  mv::grid_dependency_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int counted = __ldcg(a.t.counts + 1);
  int jobs_here = 0, n0 = 0;
  bool c0 = false, c1 = false;
  if (tid < SHARES / 2) {
    const int4* const cuts = reinterpret_cast<const int4*>(a.cuts) + 4 * tid;
    const int4 f0 = __ldcg(cuts), l0 = __ldcg(cuts + 1), f1 = __ldcg(cuts + 2), l1 = __ldcg(cuts + 3);
    continued[2 * tid] = f0.x;
    continued[2 * tid + 1] = f1.x;
    started[2 * tid] = l0;
    started[2 * tid + 1] = l1;
    c0 = l0.x >= 0;
    c1 = l1.x >= 0;
    n0 = c0 ? (l0.z + PAIR - 1) / PAIR * PAIR : 0;
    jobs_here = n0 + (c1 ? (l1.z + PAIR - 1) / PAIR * PAIR : 0);
  }
  int upto = jobs_here;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  const int cut_here = __popc(__ballot_sync(0xffffffffu, c0)) + __popc(__ballot_sync(0xffffffffu, c1));
  if (lane == 31) {
    of_warp[warp] = upto;
    cut_in_warp[warp] = cut_here;
  }
  __syncthreads();
  int jobs = 0, n_cut = 0, at = upto - jobs_here;
#pragma unroll
  for (int w = 0; w < MERGE_WARPS; ++w) {
    if (w < warp) at += of_warp[w];
    jobs += of_warp[w];
    n_cut += cut_in_warp[w];
  }
  if (tid < SHARES / 2) {
    before[2 * tid] = at;
    before[2 * tid + 1] = at + n0;
  }
  __syncthreads();
  {
    const int warps = int(gridDim.x) * MERGE_WARPS;
    const int nq = jobs <= warps ? 1 : PAIR;  // jobs of a warp at a time
    int per = 1;  // warps of one job: while there are enough, and each gets two parts or more on average
    while (per < MERGE_WARPS && 2 * per * jobs <= warps && 4 * per * n_cut <= SHARES + n_cut) per *= 2;
    const int sub = warp % per, slots = MERGE_WARPS / per * nq;
    for (int j0 = blockIdx.x * slots; j0 < jobs; j0 += gridDim.x * slots) {
      const int j = j0 + warp / per * nq;
      const bool mine = j < jobs;
      // the share c where the job's stream starts: the last one that has no more than j jobs before it and one of its own
      int c = 0;
      if (mine) {
        for (int i0 = 0; i0 < SHARES; i0 += 32) {
          const int i = i0 + lane;
          const unsigned here = __ballot_sync(0xffffffffu, i < SHARES && started[min(i, SHARES - 1)].x >= 0 && before[min(i, SHARES - 1)] <= j);
          if (here) c = i0 + 31 - __clz(here);
        }
      }
      const int4 own = started[c];
      const int v = mine ? j - before[c] : 0, n_qv = mine ? own.z : 0, head = own.x % a.Hkv;
      // the last share that holds something of the stream; between two tiles lie fewer shares than a tile costs units, which may hold nothing
      static_assert(mv::blk::COST_PER_TILE < 32, "the next tile is among the next 32 shares");
      int c1 = c;
      for (int i0 = c + 1; i0 < SHARES; i0 += 32) {
        const unsigned here = __ballot_sync(0xffffffffu, i0 + lane < SHARES && continued[min(i0 + lane, SHARES - 1)] == own.x);
        if (!here) break;
        c1 = i0 + 31 - __clz(here);
      }
      auto holds = [&](int i) { return i == c || continued[i] == own.x; };
      // parts sub, sub + per, ... of the stream (slot 2 c + 1, then slots 2 i of the shares behind).  Accumulator m is for q-vector
      // v + m / of_one, with a reference of its own; of_one accumulators share the parts of one q-vector
      const int of_one = ACCS / nq;
      float top[ACCS], sum[ACCS] = {}, acc[ACCS][VEC] = {};
#pragma unroll
      for (int m = 0; m < ACCS; ++m) top[m] = -INFINITY;
      for (int i0 = c + sub; i0 <= c1 && v < n_qv; i0 += per * of_one * ACC_LOADS) {
        float2 ml[ACCS][ACC_LOADS];
        float y[ACCS][ACC_LOADS][VEC];
#pragma unroll
        for (int m = 0; m < ACCS; ++m)
#pragma unroll
          for (int k = 0; k < ACC_LOADS; ++k) {
            const int i = i0 + (m % of_one * ACC_LOADS + k) * per, x = v + m / of_one;
            ml[m][k] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[m][k][e] = 0.f;
            if (i <= c1 && x < n_qv && holds(i)) {
              const int at = (2 * i + (i == c)) * MAXQV + x;
              ml[m][k] = __ldcg(&a.part_ml[at]);
              const float* src = a.part_o + int64_t(at) * D + lane * VEC;
              if (VEC == 4) {
                const float4 z = __ldcg(reinterpret_cast<const float4*>(src));
                y[m][k][0] = z.x; y[m][k][1] = z.y; y[m][k][VEC - 2] = z.z; y[m][k][VEC - 1] = z.w;
              } else {
                const float2 z = __ldcg(reinterpret_cast<const float2*>(src));
                y[m][k][0] = z.x; y[m][k][1] = z.y;
              }
            }
          }
#pragma unroll
        for (int m = 0; m < ACCS; ++m) {
          const float now = mv::max3(top[m], ml[m][0].x, ml[m][1].x);
          const float f = top[m] == -INFINITY ? 1.f : mv::fast_exp2(top[m] - now);  // nothing seen so far: zeros (or NaN)
          sum[m] *= f;
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[m][e] *= f;
#pragma unroll
          for (int k = 0; k < ACC_LOADS; ++k) {
            const float w = ml[m][k].x == -INFINITY ? 1.f : mv::fast_exp2(ml[m][k].x - now);
            sum[m] = fmaf(w, ml[m][k].y, sum[m]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[m][e] = fmaf(w, y[m][k][e], acc[m][e]);
          }
          top[m] = now;
        }
      }
      auto join = [&](int m, int n) {  // accumulator n into m
        const float now = fmaxf(top[m], top[n]);
        const float f = top[m] == -INFINITY ? 1.f : mv::fast_exp2(top[m] - now), w = top[n] == -INFINITY ? 1.f : mv::fast_exp2(top[n] - now);
        sum[m] = fmaf(w, sum[n], sum[m] * f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[m][e] = fmaf(w, acc[n][e], acc[m][e] * f);
        top[m] = now;
      };
      join(0, 1);
      join(2, 3);
      if (nq == 1) join(0, 2);
      if (per > 1) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) so[warp][lane * VEC + e] = acc[0][e];
        if (lane == 0) {
          ssum[warp] = sum[0];
          stop[warp] = top[0];
        }
        __syncthreads();
        float all = -INFINITY;
        for (int k = 0; k < per; ++k) all = fmaxf(all, stop[warp - sub + k]);
        sum[0] = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[0][e] = 0.f;
        for (int k = 0; k < per; ++k) {
          const int o = warp - sub + k;
          const float w = stop[o] == -INFINITY ? 1.f : mv::fast_exp2(stop[o] - all);
          sum[0] = fmaf(w, ssum[o], sum[0]);
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[0][e] = fmaf(w, so[o][lane * VEC + e], acc[0][e]);
        }
        __syncthreads();
      }
#pragma unroll
      for (int m = 0; m < ACCS; m += 2) {
        const int x = v + m / of_one;
        if (sub == 0 && m % of_one == 0 && x < n_qv) {
          const float inv = sum[m] == 0.f ? 0.f : 1.f / sum[m];
          uint32_t* const out = reinterpret_cast<uint32_t*>(a.out + (int64_t(own.y + x / a.G) * a.Hq + head * a.G + x % a.G) * D + lane * VEC);
          if (VEC == 4) *reinterpret_cast<uint2*>(out) = make_uint2(mv::pack_bf16(acc[m][0] * inv, acc[m][1] * inv), mv::pack_bf16(acc[m][VEC - 2] * inv, acc[m][VEC - 1] * inv));
          else *out = mv::pack_bf16(acc[m][0] * inv, acc[m][1] * inv);
        }
      }
    }
  }
  // groups that have rows but no entries see nothing: zeros
  const int n_groups = max(0, min(counted, a.t.max_groups));
  for (int g = blockIdx.x; g < n_groups; g += gridDim.x)
    if (a.t.tile_off[g + 1] == a.t.tile_off[g] && a.t.ent_off[g + 1] == a.t.ent_off[g]) {
      const int r0 = max(0, a.t.row_off[g]), r1 = min(a.t.max_rows, a.t.row_off[g + 1]);
      for (int64_t i = int64_t(r0) * a.Hq * D / 8 + tid; i < int64_t(r1) * a.Hq * D / 8; i += blockDim.x) reinterpret_cast<uint4*>(a.out)[i] = make_uint4(0, 0, 0, 0);
    }
}

template <int D>
mv_status merge(const Args& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(MERGE_CTAS, 1, 1);
  cfg.blockDim = dim3(MERGE_WARPS * 32, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, decode_blk_merge_kernel<D>, a);
  mv::g_launches++;
  if (e != cudaSuccess) (void)cudaGetLastError();
  return e == cudaSuccess ? MV_OK : MV_ERR_CUDA;
}

}  // namespace

extern "C" size_t mv_decode_fp8_blk_workspace_bytes(const mv_attn_geom* g) {
  if (mv::check_geom(g) != MV_OK) return 0;
  return mv::blk::workspace_bytes(g->head_dim);
}

extern "C" mv_status mv_dag_decode_attn_fp8_blk(const mv_step_tables* t, const mv_attn_geom* g, const void* q_rot, const void* k_pages8,
                                                const void* v_pages8, const float* kv_scale, void* out, void* workspace,
                                                size_t workspace_bytes, void* cuda_stream) {
  mv::NvtxRange nvtx_range("mv_dag_decode_attn_fp8_blk");
  if (!t || t->max_rows < 0 || t->max_groups < 0 || t->max_entries < 0 || !t->counts) return MV_ERR_INVALID_ARG;
  const mv_status st = mv::check_geom(g);
  if (st != MV_OK) return st;
  if (g->dtype != MV_BF16) return MV_ERR_UNSUPPORTED;
  const int G = g->n_q_heads / g->n_kv_heads;
  if (G > MAXQV || t->rows_per_group < 1 || t->rows_per_group > MAXQV / G) return MV_ERR_UNSUPPORTED;
  if (g->num_pages > INT32_MAX / PS / g->n_kv_heads) return MV_ERR_UNSUPPORTED;  // the rows of a pool are TMA coordinates
  if (t->max_rows == 0) return MV_OK;
  // Tables of positions and slots only: no row has a group, so nothing could be written for those that there may be.
  if (t->max_groups == 0) return q_rot || out ? MV_ERR_INVALID_ARG : MV_OK;
  if (!t->group_row_off || !t->group_ent_off || !t->group_tile_off || (t->max_entries > 0 && !t->entries)) return MV_ERR_INVALID_ARG;
  if (!q_rot || !k_pages8 || !v_pages8 || !kv_scale || !out) return MV_ERR_INVALID_ARG;
  for (const void* p : {q_rot, k_pages8, v_pages8, static_cast<const void*>(kv_scale), static_cast<const void*>(out),
                        static_cast<const void*>(t->entries)})
    if ((reinterpret_cast<uintptr_t>(p) & 15) != 0) return MV_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < mv::blk::workspace_bytes(g->head_dim) || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
    return MV_ERR_WORKSPACE;
  Args a;
  a.q = static_cast<const bf16*>(q_rot);
  a.k8 = static_cast<const unsigned char*>(k_pages8);
  a.v8 = static_cast<const unsigned char*>(v_pages8);
  a.scale = kv_scale;
  a.out = static_cast<bf16*>(out);
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + mv::blk::part_o_bytes(g->head_dim));
  a.cuts = reinterpret_cast<mv::blk::Cut*>(static_cast<char*>(workspace) + mv::blk::part_o_bytes(g->head_dim) + mv::blk::part_ml_bytes());
  a.t = mv::blk::Tables{t->group_row_off, t->group_ent_off, t->group_tile_off, reinterpret_cast<const int4*>(t->entries), t->counts,
                        t->max_rows, t->max_groups, t->max_entries};
  a.num_pages = g->num_pages;
  a.Hq = g->n_q_heads;
  a.Hkv = g->n_kv_heads;
  a.G = G;
  a.group_rows = MAXQV / G;
  a.scale_log2 = mv::softmax_scale(g) * 1.4426950408889634f;
  a.cost_shift = 0;
  const int64_t tiles = (int64_t(t->max_entries) / mv::blk::TILE_ENTRIES + t->max_groups) * g->n_kv_heads;  // the most there may be
  while (((tiles * mv::blk::COST_PER_TILE + int64_t(t->max_groups) * g->n_kv_heads * mv::blk::COST_PER_STREAM) >> a.cost_shift) >= (int64_t(1) << 31))
    ++a.cost_shift;
  if (a.cost_shift > 3) return MV_ERR_UNSUPPORTED;  // a tile costs at least 1
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const mv_status e = mv::decode_blk_tc(a, g->head_dim, s);
  if (e != MV_OK) return e;
  return g->head_dim == 128 ? merge<128>(a, s) : merge<64>(a, s);
}
