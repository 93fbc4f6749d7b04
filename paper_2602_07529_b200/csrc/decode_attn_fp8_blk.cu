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
using mv::blk::SHARES;

// Merge of the cut streams: CTA (c, y) takes the stream that starts in share c and ends in a later one, if there is one, and of
// its q-vectors y, y + MERGE_Y, ...
//   out = sum_i w_i O_i / sum_i w_i l_i,  w_i = 2^(m_i - max m) over the stream's parts i.
// Bound by latency: two dependent round trips (the shares' records; references and parts) and the instructions' own arrival, which is why the
// CTAs are few.  Where there are fewer q-vectors than warps, several warps
// deal out the parts of one among themselves.
constexpr int MERGE_WARPS = 8, MERGE_Y = 2, MERGE_LOADS = 8;
template <int D>
__global__ void __launch_bounds__(MERGE_WARPS * 32) decode_blk_merge_kernel(const Args a) {
  constexpr int VEC = D / 32;  // elements of the head vector per lane
  __shared__ float so[MERGE_WARPS][D], ssum[MERGE_WARPS], stop[MERGE_WARPS];
  mv::grid_dependency_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = blockIdx.x;
  const int4* const cuts = reinterpret_cast<const int4*>(a.cuts);
  auto first_of = [&](int i) { return i < SHARES ? __ldcg(cuts + 2 * i) : make_int4(-1, 0, 0, 0); };
  int4 r = first_of(c + 1 + lane);
  const int4 own = __ldcg(cuts + 2 * c + 1);
  const int counted = __ldcg(a.t.counts + 1);
  if (own.x >= 0) {
    // the shares behind that hold something of the stream (shares that hold nothing at all may lie between)
    unsigned parts = 0;  // of the 32 shares behind c
    int c1 = c;
    for (int i0 = c + 1; i0 < SHARES; i0 += 32) {
      if (i0 > c + 1) r = first_of(i0 + lane);
      const unsigned all = __ballot_sync(0xffffffffu, r.x == own.x), last = __ballot_sync(0xffffffffu, r.x == own.x && r.w != 0);
      if (i0 == c + 1) parts = all;
      if (all) c1 = i0 + 31 - __clz(all);
      if (last) break;
    }
    auto holds = [&](int i) {  // share i >= c
      return i == c || (i - c <= 32 ? ((parts >> (i - c - 1)) & 1) != 0 : __ldcg(&a.cuts[2 * i].stream) == own.x);
    };
    const int n_qv = own.z, head = own.x % a.Hkv;
    const int mine = (n_qv - int(blockIdx.y) + MERGE_Y - 1) / MERGE_Y;  // q-vectors of this CTA
    int per = 1;  // warps of one q-vector
    while (per < MERGE_WARPS && 2 * per * mine <= MERGE_WARPS && 4 * per <= c1 - c + 1) per *= 2;
    const int sub = warp % per;
    for (int v0 = 0; v0 < mine; v0 += MERGE_WARPS / per) {
      const int v = blockIdx.y + (v0 + warp / per) * MERGE_Y;
      // parts sub, sub + per, ... of the stream (part i: slot 2 c + 1, then slots 2 i of the shares behind), against the warp's own reference
      float top = -INFINITY, sum = 0.f, acc[VEC] = {};
      for (int i0 = c + sub; i0 <= c1 && v < n_qv; i0 += per * MERGE_LOADS) {
        float2 ml[MERGE_LOADS];
        float y[MERGE_LOADS][VEC];
        bool there[MERGE_LOADS];
#pragma unroll
        for (int k = 0; k < MERGE_LOADS; ++k) {
          const int i = i0 + k * per;
          there[k] = i <= c1 && holds(i);
          ml[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
          for (int e = 0; e < VEC; ++e) y[k][e] = 0.f;
          if (there[k]) {
            const int at = (2 * i + (i == c)) * MAXQV + v;
            ml[k] = __ldcg(&a.part_ml[at]);
            const float* src = a.part_o + int64_t(at) * D + lane * VEC;
            if (VEC == 4) {
              const float4 z = __ldcg(reinterpret_cast<const float4*>(src));
              y[k][0] = z.x; y[k][1] = z.y; y[k][VEC - 2] = z.z; y[k][VEC - 1] = z.w;
            } else {
              const float2 z = __ldcg(reinterpret_cast<const float2*>(src));
              y[k][0] = z.x; y[k][1] = z.y;
            }
          }
        }
        float now = top;
#pragma unroll
        for (int k = 0; k < MERGE_LOADS; ++k) now = fmaxf(now, ml[k].x);
        const float f = top == -INFINITY ? 1.f : mv::fast_exp2(top - now);  // nothing seen so far: zeros (or NaN)
        sum *= f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] *= f;
#pragma unroll
        for (int k = 0; k < MERGE_LOADS; ++k) {
          const float w = ml[k].x == -INFINITY ? 1.f : mv::fast_exp2(ml[k].x - now);
          sum = fmaf(w, ml[k].y, sum);
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] = fmaf(w, y[k][e], acc[e]);
        }
        top = now;
      }
      if (per > 1) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) so[warp][lane * VEC + e] = acc[e];
        if (lane == 0) {
          ssum[warp] = sum;
          stop[warp] = top;
        }
        __syncthreads();
        float all = -INFINITY;
        for (int k = 0; k < per; ++k) all = fmaxf(all, stop[warp - sub + k]);
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
        for (int k = 0; k < per; ++k) {
          const int o = warp - sub + k;
          const float w = stop[o] == -INFINITY ? 1.f : mv::fast_exp2(stop[o] - all);
          sum = fmaf(w, ssum[o], sum);
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] = fmaf(w, so[o][lane * VEC + e], acc[e]);
        }
        __syncthreads();
      }
      if (sub == 0 && v < n_qv) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        uint32_t* const out = reinterpret_cast<uint32_t*>(a.out + (int64_t(own.y + v / a.G) * a.Hq + head * a.G + v % a.G) * D + lane * VEC);
        if (VEC == 4) *reinterpret_cast<uint2*>(out) = make_uint2(mv::pack_bf16(acc[0] * inv, acc[1] * inv), mv::pack_bf16(acc[VEC - 2] * inv, acc[VEC - 1] * inv));
        else *out = mv::pack_bf16(acc[0] * inv, acc[1] * inv);
      }
    }
  }
  // groups that have rows but no entries see nothing: zeros
  const int n_groups = max(0, min(counted, a.t.max_groups));
  for (int g = c; g < n_groups; g += gridDim.x)
    if (a.t.tile_off[g + 1] <= a.t.tile_off[g]) {
      const int r0 = max(0, a.t.row_off[g]), r1 = min(a.t.max_rows, a.t.row_off[g + 1]);
      for (int64_t i = int64_t(r0) * a.Hq * D / 8 + blockIdx.y * blockDim.x + tid; i < int64_t(r1) * a.Hq * D / 8; i += int64_t(gridDim.y) * blockDim.x) reinterpret_cast<uint4*>(a.out)[i] = make_uint4(0, 0, 0, 0);
    }
}

template <int D>
mv_status merge(const Args& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(SHARES, MERGE_Y, 1);
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
  if (t->max_rows == 0 || t->max_groups == 0) return MV_OK;
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
