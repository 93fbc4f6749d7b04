// RoPE fused into the write of a block-scaled 8-bit KV cache: one power-of-two scale per (page of 16 tokens, KV head), K and
// V apart, that follows the data.
//
//   scale of a block = 2^e, e = ceil(log2(max |k| / 316)) over its new tokens before the rotation (a rotated element is at
//   most sqrt 2 times the largest raw one, 316 * sqrt 2 < 448, the format's largest value), resp.
//   ceil(log2(max |v| / 448)), held in [-60, 40]; a block that holds tokens already keeps the larger of its scale and that one.
// Powers of two, because a block that grows then moves its stored tokens without a second rounding (only what falls among
// the format's subnormals is rounded again).  The bound on K uses the raw elements because those are exact: the
// scale, unlike a maximum taken after the rotation, does not depend on how cosine, sine and products were rounded.
// Non-finite input: the block's scale becomes NaN, its bytes stay finite, so that whoever does not see the block can still
// multiply them by a weight of zero.
//
// The rows of a page form a run of consecutive rows; the CTA whose chunk holds the run's first row writes the whole block,
// a warp per (run, KV head, K or V), so no two warps touch a block and no atomics are needed.
//
// Bound by memory for a prompt: 17K tokens, 32 query and 8 KV heads of 128, 420 MB in 77 us (5.5 TB/s, 83 % of the measured copy
// rate).  Measured there: 4, 8, 16 rows per CTA 82.6, 78.0, 82.7 us; with 8 rows, registers for 3, 4, 5 CTAs per SM 78.0, 76.1, 93.2;
// two pairs of q per thread at a time instead of four 77.9.  Bound by the launch for a decode step: 9.5 us a call from a host program,
// 4 to 5 us in a graph.
#include "common.cuh"
#include "rope.cuh"
#include "trace.h"

namespace {

using bf16 = __nv_bfloat16;
constexpr int PS = 16;
constexpr int NT = 256;
constexpr int E_MIN = -60, E_MAX = 40;

struct Args {
  const bf16 *q, *k, *v;  // q_rot may be q and k_rot may be k, so those carry no __restrict__
  bf16 *q_rot, *k_rot;
  unsigned char *k8, *v8;
  float* scale;
  const int32_t* pos_id;
  const int64_t* slot;
  int32_t* status;
  int64_t num_pages;
  int max_rows, Hq, Hkv;
};

__device__ __forceinline__ float2 bf2(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float pow2f(int e) {  // 2^e, zero below the normal range
  return e < -126 ? 0.f : __int_as_float((127 + min(e, 127)) << 23);
}
// four floats times inv -> four bytes
__device__ __forceinline__ uint32_t quantise4(float a, float b, float c, float d, float inv) {
  return mv::pack_e4m3x2(a * inv, b * inv) | (mv::pack_e4m3x2(c * inv, d * inv) << 16);
}
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  const float2 a = mv::unpack_e4m3x2(w & 0xffffu), b = mv::unpack_e4m3x2(w >> 16);
  return quantise4(a.x, a.y, b.x, b.y, f);
}

// The block of one (run, KV head) in one pool: L tokens of rows row0 .. row0 + L - 1 go to slots off .. off + L - 1 of the page.
template <int D, bool IS_K>
__device__ __forceinline__ void write_block(const Args& a, int row0, int L, int64_t page, int off, int h, const float (*cs)[D / 2],
                                            const float (*sn)[D / 2]) {
  constexpr int HALF = D / 2;
  constexpr int LPT = HALF / 4;      // lanes per token: a lane holds elements c .. c + 3 of both halves
  constexpr int TPP = 32 / LPT;      // tokens per pass
  constexpr int PASSES = PS / TPP;
  const int lane = threadIdx.x & 31, tk = lane / LPT, c = (lane % LPT) * 4;
  const int64_t block = page * a.Hkv + h;
  float* const scale_at = a.scale + block * 2 + (IS_K ? 0 : 1);
  unsigned char* const dst = (IS_K ? a.k8 : a.v8) + block * (PS * D);
  const bf16* const src = (IS_K ? a.k : a.v) + (int64_t(row0) * a.Hkv + h) * D;
  uint2 lo[PASSES], hi[PASSES];
  uint32_t most = 0;  // largest magnitude as a bf16 bit pattern, in each half-word (NaN and infinity are the largest)
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int j = i * TPP + tk;
    lo[i] = hi[i] = make_uint2(0, 0);
    if (i * TPP < L && j < L) {
      const bf16* s = src + int64_t(j) * a.Hkv * D + c;
      lo[i] = *reinterpret_cast<const uint2*>(s);
      hi[i] = *reinterpret_cast<const uint2*>(s + HALF);
    }
  }
  int e_old = -128;
  if (off > 0) e_old = int((__float_as_uint(*scale_at) >> 23) & 0xffu) - 127;  // 128: the scale is NaN
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    most = __vmaxu2(most, __vmaxu2(lo[i].x & 0x7fff7fffu, lo[i].y & 0x7fff7fffu));
    most = __vmaxu2(most, __vmaxu2(hi[i].x & 0x7fff7fffu, hi[i].y & 0x7fff7fffu));
  }
  const uint32_t amax = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
  // amax = m * 2^x with 1 <= m < 2; 316 = (1 + 30/128) * 2^8, 448 = (1 + 96/128) * 2^8
  constexpr uint32_t BOUND = IS_K ? 30u : 96u;
  int e = int(amax >> 7) - 127 - 8 + ((amax & 127u) > BOUND ? 1 : 0);
  // At the bound itself the quotient is the power of two 2^e, and CUDA's log2 does not return e for every one of them: the
  // rule is taken as it reads, in double precision, so that a program that states it with that function gets the same scale.
  if ((amax & 127u) == BOUND && e >= E_MIN && e <= E_MAX) e = int(ceil(log2(double(pow2f(e)))));
  e = max(max(min(e, E_MAX), E_MIN), e_old);
  const bool finite = amax < 0x7f80u && e_old < 128;
  if (!finite) {
    // the block is lost to whoever sees it; its bytes only have to stay finite
    for (int x = lane; x < L * D / 16; x += 32) *reinterpret_cast<uint4*>(dst + off * D + x * 16) = make_uint4(0, 0, 0, 0);
    if (lane == 0) *scale_at = __uint_as_float(0x7fc00000u);
  } else {
    if (off > 0 && e > e_old) {
      const float f = pow2f(e_old - e);
      for (int x = lane; x < off * D / 16; x += 32) {
        uint4 w = *reinterpret_cast<const uint4*>(dst + x * 16);
        w = make_uint4(rescale4(w.x, f), rescale4(w.y, f), rescale4(w.z, f), rescale4(w.w, f));
        *reinterpret_cast<uint4*>(dst + x * 16) = w;
      }
    }
    if (lane == 0 && e != e_old) *scale_at = pow2f(e);
  }
  if (!IS_K && !finite) return;
  const float inv = pow2f(-e);
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int j = i * TPP + tk;
    if (i * TPP >= L || j >= L) continue;
    float x0[4], x1[4];
    const float2 a0 = bf2(lo[i].x), a1 = bf2(lo[i].y), b0 = bf2(hi[i].x), b1 = bf2(hi[i].y);
    x0[0] = a0.x; x0[1] = a0.y; x0[2] = a1.x; x0[3] = a1.y;
    x1[0] = b0.x; x1[1] = b0.y; x1[2] = b1.x; x1[3] = b1.y;
    if (IS_K) {
      const float4 cc = *reinterpret_cast<const float4*>(&cs[j][c]), ss = *reinterpret_cast<const float4*>(&sn[j][c]);
      const float cv[4] = {cc.x, cc.y, cc.z, cc.w}, sv[4] = {ss.x, ss.y, ss.z, ss.w};
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float l = x0[n], r = x1[n];
        x0[n] = l * cv[n] - r * sv[n];
        x1[n] = r * cv[n] + l * sv[n];
      }
      if (a.k_rot) {
        bf16* o = a.k_rot + (int64_t(row0 + j) * a.Hkv + h) * D + c;
        *reinterpret_cast<uint2*>(o) = make_uint2(mv::pack_bf16(x0[0], x0[1]), mv::pack_bf16(x0[2], x0[3]));
        *reinterpret_cast<uint2*>(o + HALF) = make_uint2(mv::pack_bf16(x1[0], x1[1]), mv::pack_bf16(x1[2], x1[3]));
      }
      if (!finite) continue;
    }
    unsigned char* o = dst + (off + j) * D + c;
    *reinterpret_cast<uint32_t*>(o) = quantise4(x0[0], x0[1], x0[2], x0[3], inv);
    *reinterpret_cast<uint32_t*>(o + HALF) = quantise4(x1[0], x1[1], x1[2], x1[3], inv);
  }
}

template <int D, int TPC>
__global__ void __launch_bounds__(NT, 4) rope_write_kv_blk_kernel(const Args a, const __grid_constant__ mv::ThetaTable tt) {
  constexpr int HALF = D / 2, CH = HALF / 8;
  constexpr int ROWS = TPC + PS - 1;  // the chunk and what the last run may hold beyond it
  __shared__ __align__(16) float cs[ROWS][HALF], sn[ROWS][HALF];
  __shared__ int64_t s_slot[ROWS + 1];  // slots of rows t0 - 1 .. ; -1: no row, or none to write
  __shared__ int s_run[TPC][2], s_runs, s_end;  // runs that start in the chunk: first row, rows; rows whose angles are needed
  const int t0 = blockIdx.x * TPC, tid = threadIdx.x;
  mv::grid_dependency_launch_dependents();
  for (int i = tid; i <= ROWS; i += NT) {
    const int t = t0 - 1 + i;
    int64_t sl = t >= 0 && t < a.max_rows ? a.slot[t] : -1;
    if (sl >= 0 && (sl >> 4) >= a.num_pages) {
      atomicExch(a.status, int(MV_ERR_INVALID_ARG));
      sl = -1;
    }
    s_slot[i] = sl < 0 ? -1 : sl;
  }
  __syncthreads();
  if (tid < 32) {
    // lane i: does a run start at row t0 + i?  A run goes on while the slot counts up inside the page.
    int runs = 0, end = 0;
    for (int i0 = 0; i0 < TPC; i0 += 32) {
      const int i = i0 + tid;
      const int64_t sl = i < TPC ? s_slot[i + 1] : -1;
      const bool first = sl >= 0 && ((sl & 15) == 0 || s_slot[i] != sl - 1);
      int len = 0;
      if (first) {
        len = 1;
        while (len < PS && i + len < ROWS && s_slot[i + len + 1] == sl + len && ((sl + len) & 15) != 0) ++len;
      }
      const unsigned m = __ballot_sync(0xffffffffu, first);
      if (first) {
        const int at = runs + __popc(m & ((1u << tid) - 1));
        s_run[at][0] = i;
        s_run[at][1] = len;
      }
      runs += __popc(m);
      end = max(end, int(__reduce_max_sync(0xffffffffu, sl >= 0 ? unsigned(max(i + 1, i + len)) : 0u)));
    }
    if (tid == 0) {
      s_runs = runs;
      s_end = end;
    }
  }
  __syncthreads();
  const int end = s_end;
  for (int x = tid; x < end * HALF; x += NT) {
    const int tl = x / HALF, i = x % HALF;
    if (s_slot[tl + 1] < 0) continue;
    float c, s;
    mv::rope_cos_sin(__ldg(a.pos_id + t0 + tl), tt.theta[i], c, s);
    cs[tl][i] = c;
    sn[tl][i] = s;
  }
  __syncthreads();
  // K and V: a warp per (run, KV head, pool)
  const int runs = s_runs, warp = tid >> 5;
  for (int x = warp; x < runs * a.Hkv * 2; x += NT / 32) {
    const int run = x / (a.Hkv * 2), h = (x >> 1) % a.Hkv;
    const int i = s_run[run][0], len = s_run[run][1];
    const int64_t sl = s_slot[i + 1];
    if (x & 1) write_block<D, false>(a, t0 + i, len, sl >> 4, int(sl & 15), h, cs + i, sn + i);
    else write_block<D, true>(a, t0 + i, len, sl >> 4, int(sl & 15), h, cs + i, sn + i);
  }
  // q: 16-byte pieces of both halves, UNITS of them per thread at a time so that their loads are in flight together
  if (a.q) {
    constexpr int UNITS = TPC == 1 ? 1 : 4;
    const int here = min(TPC, a.max_rows - t0), units = here * a.Hq * CH;
#pragma unroll 1
    for (int x0 = tid; x0 < units; x0 += NT * UNITS) {
      uint4 lo[UNITS], hi[UNITS];
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int x = x0 + i * NT;
        if (x < units) {
          const int64_t at = int64_t(t0) * a.Hq * D + int64_t(x / CH) * D + (x % CH) * 8;
          lo[i] = *reinterpret_cast<const uint4*>(a.q + at);
          hi[i] = *reinterpret_cast<const uint4*>(a.q + at + HALF);
        }
      }
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int x = x0 + i * NT;
        if (x >= units) break;
        const int tl = x / (a.Hq * CH), c = (x % CH) * 8;
        if (s_slot[tl + 1] < 0) continue;
        const int64_t at = int64_t(t0) * a.Hq * D + int64_t(x / CH) * D + c;
        const uint32_t lw[4] = {lo[i].x, lo[i].y, lo[i].z, lo[i].w}, hw[4] = {hi[i].x, hi[i].y, hi[i].z, hi[i].w};
        uint32_t ol[4], oh[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const float2 l = bf2(lw[n]), r = bf2(hw[n]);
          const float2 cc = *reinterpret_cast<const float2*>(&cs[tl][c + 2 * n]), ss = *reinterpret_cast<const float2*>(&sn[tl][c + 2 * n]);
          ol[n] = mv::pack_bf16(l.x * cc.x - r.x * ss.x, l.y * cc.y - r.y * ss.y);
          oh[n] = mv::pack_bf16(r.x * cc.x + l.x * ss.x, r.y * cc.y + l.y * ss.y);
        }
        *reinterpret_cast<uint4*>(a.q_rot + at) = make_uint4(ol[0], ol[1], ol[2], ol[3]);
        *reinterpret_cast<uint4*>(a.q_rot + at + HALF) = make_uint4(oh[0], oh[1], oh[2], oh[3]);
      }
    }
  }
}

constexpr int MANY = 8;  // rows per CTA of a prompt
template <int D>
void launch(const Args& a, double rope_base, cudaStream_t st) {
  const mv::ThetaTable tt = mv::theta_table(rope_base, D);
  // Few rows (a decode step): one per CTA spreads them over the SMs; many (a prompt): MANY per CTA share the angles' staging.  The host knows the
  // tables' capacity, not the step's rows.  One / MANY rows per CTA, us in a graph, 32 query and 8 KV heads of 128: runs of 16 rows (a prompt)
  // 1024 rows 14.3 / 13.5, 2047 19.6 / 16.1, 4096 31.6 / 24.6, 8192 56 / 39; single rows (a decode step) 256 rows 5.8 / 21.9, 2047 26.4 / 34.4,
  // 4096 49.7 / 51.3; 64 rows in tables of 2048 5.7 / 27.1, of 8192 15.5 / 31.3.  8 and 2 heads of 64, single rows: 1024 6.4 / 6.1, 2047 11.1 / 7.2.
  // So a decode step should not come in tables made for 2048 rows and more.
  if (a.max_rows < 2048) rope_write_kv_blk_kernel<D, 1><<<a.max_rows, NT, 0, st>>>(a, tt);
  else rope_write_kv_blk_kernel<D, MANY><<<(a.max_rows + MANY - 1) / MANY, NT, 0, st>>>(a, tt);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

extern "C" mv_status mv_rope_write_kv_fp8_blk(const mv_step_tables* t, const mv_attn_geom* g, const void* q, const void* k, const void* v,
                                              void* q_rot, void* k_rot, void* k_pages8, void* v_pages8, float* kv_scale, void* cuda_stream) {
  mv::NvtxRange nvtx_range("mv_rope_write_kv_fp8_blk");
  if (!t || t->max_rows < 0 || !t->counts || (t->max_rows > 0 && (!t->pos_id || !t->slot))) return MV_ERR_INVALID_ARG;
  const mv_status st = mv::check_geom(g);
  if (st != MV_OK) return st;
  if (g->dtype != MV_BF16) return MV_ERR_UNSUPPORTED;
  if (g->rope_base <= 0.0) return MV_ERR_INVALID_ARG;
  if (t->max_rows == 0) return MV_OK;
  if (!k || !v || !k_pages8 || !v_pages8 || !kv_scale) return MV_ERR_INVALID_ARG;
  if ((q == nullptr) != (q_rot == nullptr)) return MV_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, static_cast<const void*>(q_rot), static_cast<const void*>(k_rot), static_cast<const void*>(k_pages8),
                        static_cast<const void*>(v_pages8), static_cast<const void*>(kv_scale)})
    if (!aligned16(p)) return MV_ERR_INVALID_ARG;
  Args a;
  a.q = static_cast<const bf16*>(q);
  a.k = static_cast<const bf16*>(k);
  a.v = static_cast<const bf16*>(v);
  a.q_rot = static_cast<bf16*>(q_rot);
  a.k_rot = static_cast<bf16*>(k_rot);
  a.k8 = static_cast<unsigned char*>(k_pages8);
  a.v8 = static_cast<unsigned char*>(v_pages8);
  a.scale = kv_scale;
  a.pos_id = t->pos_id;
  a.slot = t->slot;
  a.status = t->counts + 4;
  a.num_pages = g->num_pages;
  a.max_rows = t->max_rows;
  a.Hq = g->n_q_heads;
  a.Hkv = g->n_kv_heads;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (g->head_dim == 128) launch<128>(a, g->rope_base, s);
  else launch<64>(a, g->rope_base, s);
  mv::g_launches++;
  return cudaGetLastError() == cudaSuccess ? MV_OK : MV_ERR_CUDA;
}
