// Decode attention over the block-scaled 8-bit cache: the register kernel, the merge of cut streams and the entry point.
//
// For the q-vectors x of a stream (rows of a group x query heads of one KV head) and the tokens j its entries name,
//   s_xj = <q_x, K_j> * sK[page] * c_x,  c_x = softmax scale * log2 e        (log2 units)
//   out_x = sum_j 2^(s_xj) sV[page] V_j / sum_j 2^(s_xj)
// The scale of V is a power of two, 2^e, so it goes into the exponent: weights p_xj = 2^(s_xj + e_j - m_x) multiply the
// stored bytes, and the denominator takes p_xj 2^(-e_j).  The running reference m_x follows the largest s + e, which
// keeps the weights of whatever dominates the NUMERATOR near one however much the pages' scales differ; with
// exponents in [-60, 40] a token that matters to the denominator alone still gets a weight above 2^-126.
// Block scale NaN: the scores of the rows that see the page become NaN; a row that does not see it multiplies
// finite bytes by zero.
//
// Register kernel (head_dim 64, and the shapes the tensor-memory kernel does not take): a warp takes a page at a time, K
// and V straight from global memory into registers (no shared memory, no barriers in the loop), converted to half precision
// there, which holds every 8-bit float exactly, and multiplied by mma.sync.  The contraction order is free, so every lane
// owns contiguous bytes: lane (r, c) of the 8 x 4 fragment grid loads bytes [c * D/4, (c + 1) * D/4) of tokens r and r + 8
// of K, and bytes [r * D/8, (r + 1) * D/8) of tokens 2c, 2c + 1, 2c + 8, 2c + 9 of V.  The score fragments of the first
// product are then the weight fragments of the second.
#include "blk_stream.cuh"
#include "trace.h"

namespace mv {
mv_status decode_blk_tc(const blk::Args& a, cudaStream_t st);
}

namespace {

using bf16 = __nv_bfloat16;
using mv::blk::Args;
using mv::blk::MAXQV;
using mv::blk::PS;
using mv::blk::SHARES;

constexpr int NT = 256, NW = NT / 32;

__device__ __forceinline__ uint32_t half2_of_e4m3x2(uint32_t v) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"(uint16_t(v)));
  return h;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int D>
struct PageRegs {  // one page of one KV head as a warp holds it: raw bytes, token count, mask, scales
  uint4 k[2][D / 64];
  uint32_t v[4][D / 32];
  int tokens;
  uint64_t mask;
  float ks;  // NaN if either scale is
  int ev;
};

template <int D>
constexpr int smem_bytes() { return MAXQV * (D + 8) * 2 + MAXQV * 4 + NW * 16 * (D + 4) * 4 + NW * MAXQV * 8 + MAXQV * 8; }

// MT blocks of 16 q-vectors at a time; a stream with more is walked again for the rest.
template <int D, int MT>
__global__ void __launch_bounds__(NT, 2) decode_blk_kernel(const Args a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int QS = D + 8;  // halves per q-vector in shared memory
  constexpr int OS = D + 4;
  __half* const sq = reinterpret_cast<__half*>(smem);                                  // [64][QS]
  float* const sc = reinterpret_cast<float*>(smem + MAXQV * QS * 2);                   // [64] factor of a score
  float* const so = sc + MAXQV;                                                       // [NW][16][OS]
  float2* const sml = reinterpret_cast<float2*>(so + NW * 16 * OS);                    // [NW][64]
  float2* const sall = sml + NW * MAXQV;                                               // [64] reference, sum over the warps
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int fr = lane >> 2, fc = lane & 3;  // fragment row / column of the lane
  mv::grid_dependency_wait();
  mv::grid_dependency_launch_dependents();
  mv::blk::Walk walk;
  walk.begin(a, blockIdx.x);
  mv::blk::Segment s;
  mv::blk::CutLog cuts;
  while (walk.next(a, s, tid == 0)) {
    cuts.add(a, s);
    // ---- q-vectors as half precision, scaled by a power of two to magnitudes below 2 (exact for what is within 2^-14 of the
    // largest element): a warp per q-vector
    __syncthreads();
    for (int v = warp; v < MAXQV; v += NW) {
      __half* const dst = sq + v * QS;
      if (v >= s.n_qv) {
        for (int i = lane; i < D / 2; i += 32) reinterpret_cast<uint32_t*>(dst)[i] = 0;
        if (lane == 0) sc[v] = 0.f;
        continue;
      }
      const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + (int64_t(s.row0 + v / a.G) * a.Hq + s.head * a.G + v % a.G) * D);
      uint32_t w[D / 64];
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        w[i] = __ldcg(src + i * 32 + lane);
        most = __vmaxu2(most, w[i] & 0x7fff7fffu);
      }
      const uint32_t amax = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
      const int e = min(max(int(amax >> 7), 1) - 127, 126);
      const float inv = amax < 0x7f80u ? mv::blk::exp2_int(-e) : __uint_as_float(0x7fc00000u);  // not finite: the products become NaN
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
        reinterpret_cast<uint32_t*>(dst)[i * 32 + lane] = pack_half(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xffff0000u) * inv);
      if (lane == 0) sc[v] = mv::blk::exp2_int(e) * a.scale_log2;
    }
    __syncthreads();
    for (int v0 = 0; v0 < s.n_qv; v0 += MT * 16) {
      float o[MT][D / 8][4], m[MT][2], l[MT][2], cf[MT][2];
      int row[MT][2];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int v = v0 + t * 16 + i * 8 + fr;
          m[t][i] = -INFINITY;
          l[t][i] = 0.f;
          cf[t][i] = v < MAXQV ? sc[v] : 0.f;
          row[t][i] = v < s.n_qv ? v / a.G : -1;
        }
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][j][i] = 0.f;

      // entry e of the segment, for this warp: window of 32 entries per lane, 4 apart
      int4 we = make_int4(0, 0, 0, 0);
      float2 ws = make_float2(0.f, 0.f);
      auto window = [&](int i0) {  // lane's entry: warp + NW * (i0 + lane)
        const int e = warp + NW * (i0 + lane);
        we = make_int4(-1, 0, 0, 0);
        if (e < s.n_ent) {
          we = __ldcg(a.t.entries + s.ent0 + e);
          if (we.x < 0 || we.x >= a.num_pages || we.y < 1 || we.y > PS) {
            atomicExch(a.t.counts + 4, int(MV_ERR_INVALID_ARG));
            we = make_int4(-1, 0, 0, 0);
          } else {
            ws = __ldcg(reinterpret_cast<const float2*>(a.scale) + int64_t(we.x) * a.Hkv + s.head);
          }
        }
      };
      auto fetch = [&](int i, PageRegs<D>& p) {
        const int src = i & 31;
        const int page = __shfl_sync(0xffffffffu, we.x, src);
        p.tokens = __shfl_sync(0xffffffffu, we.y, src);
        p.mask = (uint64_t(uint32_t(__shfl_sync(0xffffffffu, we.w, src))) << 32) | uint32_t(__shfl_sync(0xffffffffu, we.z, src));
        const int ek = mv::blk::scale_exponent(__shfl_sync(0xffffffffu, ws.x, src));
        p.ev = mv::blk::scale_exponent(__shfl_sync(0xffffffffu, ws.y, src));
        p.ks = ek == 128 || p.ev == 128 ? __uint_as_float(0x7fc00000u) : mv::blk::exp2_int(ek);
        if (p.ev == 128) p.ev = 0;
        if (page < 0) {
          p.tokens = 0;
          return;
        }
        const int64_t base = (int64_t(page) * a.Hkv + s.head) * (PS * D);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i2 = 0; i2 < D / 64; ++i2)
            p.k[t][i2] = __ldcg(reinterpret_cast<const uint4*>(a.k8 + base + (t * 8 + fr) * D + fc * (D / 4)) + i2);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const unsigned char* vp = a.v8 + base + ((t >> 1) * 8 + fc * 2 + (t & 1)) * D + fr * (D / 8);
          if (D == 64) {
            const uint2 w = __ldcg(reinterpret_cast<const uint2*>(vp));
            p.v[t][0] = w.x; p.v[t][1] = w.y;
          } else {
            const uint4 w = __ldcg(reinterpret_cast<const uint4*>(vp));
            p.v[t][0] = w.x; p.v[t][1] = w.y; p.v[t][D / 32 - 2] = w.z; p.v[t][D / 32 - 1] = w.w;
          }
        }
      };
      const int n_mine = s.n_ent > warp ? (s.n_ent - warp + NW - 1) / NW : 0;
      PageRegs<D> cur, nxt;
      cur.tokens = nxt.tokens = 0;
      if (n_mine > 0) {
        window(0);
        fetch(0, cur);
      }
      for (int i = 0; i < n_mine; ++i) {
        if (i + 1 < n_mine) {
          if (((i + 1) & 31) == 0) window(i + 1);
          fetch(i + 1, nxt);
        }
        if (cur.tokens > 0) {
          uint32_t kf[2][D / 16][2];  // [token half][k-step][fragment register]
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i2 = 0; i2 < D / 64; ++i2) {
              const uint32_t w[4] = {cur.k[t][i2].x, cur.k[t][i2].y, cur.k[t][i2].z, cur.k[t][i2].w};
#pragma unroll
              for (int n = 0; n < 4; ++n) {
                kf[t][i2 * 4 + n][0] = half2_of_e4m3x2(w[n] & 0xffffu);
                kf[t][i2 * 4 + n][1] = half2_of_e4m3x2(w[n] >> 16);
              }
            }
          if (cur.tokens < PS) {
            // what lies behind the page's last token may be anything; it meets weights of zero, so it must be finite
#pragma unroll
            for (int t = 0; t < 4; ++t)
              if ((t >> 1) * 8 + fc * 2 + (t & 1) >= cur.tokens)
#pragma unroll
                for (int j = 0; j < D / 32; ++j) cur.v[t][j] = 0;
          }
          uint32_t pf[MT][4];
          const float vinv = mv::blk::exp2_int(-cur.ev);
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            if (v0 + t * 16 >= s.n_qv) continue;
            float sv[2][4] = {};
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const __half* q0 = sq + (v0 + t * 16 + fr) * QS + fc * (D / 4) + k * 4;
              const uint2 r0 = *reinterpret_cast<const uint2*>(q0), r1 = *reinterpret_cast<const uint2*>(q0 + 8 * QS);
              const uint32_t af[4] = {r0.x, r1.x, r0.y, r1.y};
              mma_f16(sv[0], af, kf[0][k][0], kf[0][k][1]);
              mma_f16(sv[1], af, kf[1][k][0], kf[1][k][1]);
            }
            float mx[2], f[2], sum[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const bool sees = row[t][r] >= 0 && ((cur.mask >> (row[t][r] & 63)) & 1);
              const float c = cf[t][r] * cur.ks;
              mx[r] = -INFINITY;
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  float& w = sv[h][r * 2 + j];
                  w = sees && h * 8 + fc * 2 + j < cur.tokens ? fmaf(w, c, float(cur.ev)) : -INFINITY;
                  mx[r] = fmaxf(mx[r], w);
                }
              mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
              mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2));
              const float now = fmaxf(m[t][r], mx[r]);
              f[r] = m[t][r] == -INFINITY ? 1.f : mv::fast_exp2(m[t][r] - now);
              m[t][r] = now;
              const float ref = now == -INFINITY ? 0.f : now;
              sum[r] = 0.f;
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  float& w = sv[h][r * 2 + j];
                  w = mv::fast_exp2(w - ref);
                  sum[r] += w;
                }
              l[t][r] = l[t][r] * f[r] + sum[r] * vinv;
            }
            if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
              for (int j = 0; j < D / 8; ++j) {
                o[t][j][0] *= f[0];
                o[t][j][1] *= f[0];
                o[t][j][2] *= f[1];
                o[t][j][3] *= f[1];
              }
            }
            pf[t][0] = pack_half(sv[0][0], sv[0][1]);
            pf[t][1] = pack_half(sv[0][2], sv[0][3]);
            pf[t][2] = pack_half(sv[1][0], sv[1][1]);
            pf[t][3] = pack_half(sv[1][2], sv[1][3]);
          }
#pragma unroll
          for (int j = 0; j < D / 8; ++j) {  // column block j: byte j of the lane's D / 8 bytes
            const uint32_t sel = uint32_t(j & 3) | (uint32_t((j & 3) + 4) << 4);
            const uint32_t b0 = half2_of_e4m3x2(__byte_perm(cur.v[0][j / 4], cur.v[1][j / 4], sel));
            const uint32_t b1 = half2_of_e4m3x2(__byte_perm(cur.v[2][j / 4], cur.v[3][j / 4], sel));
#pragma unroll
            for (int t = 0; t < MT; ++t)
              if (v0 + t * 16 < s.n_qv) mma_f16(o[t][j], pf[t], b0, b1);
          }
        }
        cur = nxt;
      }
      // ---- the warps' results into one: (reference, sum) of every q-vector, then the head vectors, 16 at a time
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float y = l[t][r];
          y += __shfl_xor_sync(0xffffffffu, y, 1);
          y += __shfl_xor_sync(0xffffffffu, y, 2);
          if (fc == 0) sml[warp * MAXQV + t * 16 + r * 8 + fr] = make_float2(m[t][r], y);
        }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if (v0 + t * 16 >= s.n_qv) break;
        float w[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int v = t * 16 + r * 8 + fr;
          float all = -INFINITY, sum = 0.f;
#pragma unroll
          for (int k = 0; k < NW; ++k) all = fmaxf(all, sml[k * MAXQV + v].x);
#pragma unroll
          for (int k = 0; k < NW; ++k) {
            const float2 y = sml[k * MAXQV + v];
            sum += y.x == -INFINITY ? y.y : y.y * mv::fast_exp2(y.x - all);  // nothing seen: the sum is 0 (or NaN)
          }
          w[r] = m[t][r] == -INFINITY ? 1.f : mv::fast_exp2(m[t][r] - all);  // (its head vector is 0 or NaN)
          if (warp == 0 && fc == 0) sall[v] = make_float2(all, sum);
        }
        float* const mine = so + warp * 16 * OS;
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) mine[(fr + (i >> 1) * 8) * OS + (fc * 2 + (i & 1)) * (D / 8) + j] = o[t][j][i] * w[i >> 1];
        __syncthreads();
        for (int i = tid; i < 16 * D / 4; i += NT) {
          const int v = i / (D / 4), c = (i % (D / 4)) * 4, qv = v0 + t * 16 + v;
          if (qv >= s.n_qv) break;
          float4 y = *reinterpret_cast<const float4*>(so + v * OS + c);
#pragma unroll
          for (int k = 1; k < NW; ++k) {
            const float4 z = *reinterpret_cast<const float4*>(so + (k * 16 + v) * OS + c);
            y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
          }
          const float2 ml = sall[t * 16 + v];
          if (s.slot < 0) {
            const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
            uint2 pk = make_uint2(mv::pack_bf16(y.x * inv, y.y * inv), mv::pack_bf16(y.z * inv, y.w * inv));
            *reinterpret_cast<uint2*>(a.out + (int64_t(s.row0 + qv / a.G) * a.Hq + s.head * a.G + qv % a.G) * D + c) = pk;
          } else {
            *reinterpret_cast<float4*>(a.part_o + (int64_t(s.slot) * MAXQV + qv) * D + c) = y;
            if (c == 0) a.part_ml[s.slot * MAXQV + qv] = ml;
          }
        }
        __syncthreads();
      }
    }
  }
  if (tid == 0) cuts.store(a, blockIdx.x);
}

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

bool launch_pdl(void (*kernel)(const Args), dim3 grid, int threads, int smem, const Args& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(unsigned(threads), 1, 1);
  cfg.dynamicSmemBytes = size_t(smem);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
  mv::g_launches++;
  if (e != cudaSuccess) (void)cudaGetLastError();
  return e == cudaSuccess;
}

template <int D, int MT>
bool launch(const Args& a, cudaStream_t st) {
  static std::atomic<uint64_t> opted{0};  // per device
  constexpr int smem = smem_bytes<D>();
  if (smem > 48 * 1024 && !mv::opt_in_smem(decode_blk_kernel<D, MT>, smem, opted)) return false;
  if (!launch_pdl(decode_blk_kernel<D, MT>, dim3(SHARES), NT, smem, a, st)) return false;
  return launch_pdl(decode_blk_merge_kernel<D>, dim3(SHARES, MERGE_Y), MERGE_WARPS * 32, 0, a, st);
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
  if (g->head_dim == 128) {
    const mv_status e = mv::decode_blk_tc(a, s);
    if (e != MV_OK) return e;
    return launch_pdl(decode_blk_merge_kernel<128>, dim3(SHARES, MERGE_Y), MERGE_WARPS * 32, 0, a, s) ? MV_OK : MV_ERR_CUDA;
  }
  return launch<64, 1>(a, s) ? MV_OK : MV_ERR_CUDA;
}
