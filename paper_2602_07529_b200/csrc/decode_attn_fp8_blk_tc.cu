// Decode attention over the block-scaled 8-bit cache on the tensor cores with accumulators in tensor memory (head_dim 128).
// The mathematics is that of the register kernel (decode_attn_fp8_blk.cu): weights 2^(s + e - m) with the exponent e of V's
// block scale folded in, denominators corrected by 2^(-e).
//
// Both products run with the CACHE as the 128-row operand, straight on the pool's bytes: S^T = K Q^T puts a tile's 128 tokens
// on the 128 lanes of tensor memory and the q-vectors on its columns, O^T = V^T P^T the 128 elements of the head vector on the
// lanes.  A softmax thread therefore owns a token and works on exactly the q-vectors there are (16, 32, 48 or 64 columns),
// all 128 lanes always busy, instead of owning one of at most 64 q-vectors; per tile it reads one mask, one token count
// and one pair of scales.
//   - Q is two K-major tiles of 8-bit floats, the rounded element and its rounded remainder at one power-of-two scale per
//     q-vector: a bf16 element has eight significant bits, value plus remainder hold nine, so the split is exact
//     for elements within 2^-9 of the largest (and off by at most 2^-17 of the largest below).
//   - The weights are two tiles as well, value and 16 times the remainder, accumulated in columns of their own
//     and joined at the end (O = O_hi + O_lo / 16): at least eight significant bits where a weight is within 2^-6 of the
//     largest, down to a quantum of 2^-18 of the largest.  The factor 16 keeps long tails of small weights.
//   - The reference exponent of a q-vector moves only when a weight would pass the format's largest value (448): every
//     thread looks at its own weights and one barrier votes, so the maximum over the tokens (a reduction across lanes) is taken only
//     on a stream's first tile and in the rare tile that lifts it.
// The softmax warps keep the sums of a token (one per q-vector) in tensor memory as well, and walk the columns sixteen at a time
// in a loop that is not unrolled: four warps on four quarters of the SM share no instruction fetches, and with the columns unrolled
// (per-thread arrays, a code path per number of columns) misses of the SM's instruction cache cost three cycles per instruction.
// A CTA is four softmax warps, a producer warp (TMA) and an issuer warp (products); two CTAs per SM hide each other's
// hand-overs.  K and V tiles (16 KB each) share a ring of five slots; the scores of tile t + 1 are computed into the other
// of two score buffers while the weights of tile t are.
// Every wait is bounded; the softmax warps vote once per tile, and the vote carries a failed wait, so that they leave together.
#include "blk_stream.cuh"
#include "tmap_cache.h"
#include "umma.cuh"

namespace {

using bf16 = __nv_bfloat16;
using mv::blk::Args;
using mv::blk::MAXQV;
using mv::blk::PS;
using mv::blk::SHARES;
using mv::blk::TILE_ENTRIES;

constexpr int D = 128;
constexpr int TILE = 128;                 // tokens per tile
constexpr int PIECE = TILE * D;           // 16 KB: K or V of a tile
constexpr int RING = 5;
constexpr int METAS = 3;                  // tiles whose descriptions are live: K of tile j waits for the second product of tile j - 3
constexpr int OFF_P = RING * PIECE;       // weights: [128 tokens][128 bytes], 128-byte swizzle
constexpr int OFF_Q = OFF_P + PIECE;      // Q values [64][128], then Q remainders
constexpr int Q_BYTES = MAXQV * D;
constexpr int OFF_META = OFF_Q + 2 * Q_BYTES;
constexpr int NT = 192;
constexpr float TOP = 448.f;              // largest 8-bit float
constexpr float HEADROOM = 5.f;           // a reference that moves puts the largest weight at 2^5
constexpr float LO_SCALE = 16.f;

struct Entry {       // one page of a tile, as the softmax threads need it
  uint32_t see_lo, see_hi;  // q-vectors that see it
  uint32_t rest;            // tokens | (exponent of V's scale + 127) << 8 | (exponent of K's scale + 127) << 16; K's is 255 (NaN) if either scale is NaN
};
struct Meta {
  float factor[MAXQV];      // of a score
  float minus_ref[MAXQV];   // minus the reference (+infinity: none yet; -infinity: no such q-vector)
  Entry entry[METAS][TILE_ENTRIES];
  uint64_t full[RING], empty[RING], described[METAS], s_full[2], q_full, p_full, pv_done, drained;
  int abort;
  uint32_t tmem;
};
static_assert(sizeof(Meta) <= 1024, "meta area");
constexpr int SMEM = OFF_META + 1024;
static_assert(2 * (SMEM + 1024) <= 228 * 1024, "two CTAs per SM");

__device__ __forceinline__ uint32_t bar(const void* p) { return mv::smem_u32(p); }

struct Cta {
  const Args* a;
  unsigned char* smem;
  uint32_t base;
  Meta* meta;
  int32_t* status;
};

// Bounded wait.  False once a wait of this CTA has run out (this one or an earlier one, of any role).  Out of line: the kernel's
// loops have to stay small (see above).
__device__ __noinline__ bool wait_slow(uint32_t b, uint32_t parity, volatile int* abort, int32_t* status) {
  if (*abort) return false;
  if (!mv::mbar_wait_bounded(b, parity, 2000000000ull, abort)) {
    if (!*abort) atomicExch(status, int(MV_ERR_TIMEOUT));
    *abort = 1;
    return false;
  }
  return true;
}
__device__ __forceinline__ bool wait_or_flag(const Cta& c, uint32_t b, uint32_t parity) {
  return mv::mbar_try_wait(b, parity) || wait_slow(b, parity, &c.meta->abort, c.status);
}
__device__ __forceinline__ bool warp_wait(const Cta& c, uint32_t b, uint32_t parity) {
  return __all_sync(0xffffffffu, wait_or_flag(c, b, parity));
}
// Barriers of the four softmax warps that carry a predicate.
__device__ __forceinline__ bool vote_any(bool p) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(uint32_t(p)) : "memory");
  return r != 0;
}
__device__ __forceinline__ bool vote_all(bool p) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(uint32_t(p)) : "memory");
  return r != 0;
}

// two floats -> two 8-bit floats each: value, and 16 times the remainder (bytes 0 and 1 of the results)
__device__ __forceinline__ void split_e4m3x2(float x, float y, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(x, y);
  const uint32_t hb = *reinterpret_cast<const uint32_t*>(&h);
  uint16_t w, v;
  uint32_t back;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;\n" : "=h"(w) : "r"(hb));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(back) : "h"(w));
  const __half2 r = __hmul2(__hsub2(h, *reinterpret_cast<const __half2*>(&back)), __float2half2_rn(LO_SCALE));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;\n" : "=h"(v) : "r"(*reinterpret_cast<const uint32_t*>(&r)));
  hi = w;
  lo = v;
}

// The share's segments, walked in the same way by both roles.
struct Walk {
  mv::blk::Step st;
  int64_t x, x_end;
  int share, g;
  __device__ __forceinline__ void begin(const Args& a, int c) {
    st = mv::blk::step_of(a);
    share = c;
    x = st.n_tiles > 0 ? mv::blk::share_begin(st.n_tiles, c) : 0;
    x_end = st.n_tiles > 0 ? mv::blk::share_begin(st.n_tiles, c + 1) : 0;
    g = x < x_end ? mv::blk::find_group(a.t.tile_off, st.n_groups, int(x / a.Hkv)) : 0;
  }
  // the next sound segment; false at the end of the share
  __device__ __forceinline__ bool next(const Args& a, mv::blk::Segment& s, bool report) {
    while (x < x_end) {
      while (g + 1 < st.n_groups && int64_t(a.t.tile_off[g + 1]) * a.Hkv <= x) ++g;
      if (a.t.tile_off[g + 1] <= a.t.tile_off[g]) return false;  // offsets that do not count up
      s = mv::blk::segment_at(a, st, share, x, x_end, g);
      x += s.n_tiles;
      if (s.ok) return true;
      if (report) atomicExch(a.t.counts + 4, int(MV_ERR_INVALID_ARG));
    }
    return false;
  }
};

// ---- producer warp ---------------------------------------------------------------------------------------
__device__ __forceinline__ void producer(const Cta& c, const CUtensorMap* tm_k, const CUtensorMap* tm_v) {
  const Args& a = *c.a;
  Meta* const meta = c.meta;
  const int lane = threadIdx.x & 31;
  const uint64_t policy = mv::l2_policy_evict_first();  // the cache is read once per call
  Walk w;
  w.begin(a, blockIdx.x);
  mv::blk::Segment s;
  int piece = 0, tile = 0;
  bool ok = true;
  while (ok && w.next(a, s, lane == 0)) {
    const uint64_t live = s.n_qv >= 64 ? ~0ull : (1ull << s.n_qv) - 1;
    const uint64_t one_row = a.G >= 64 ? ~0ull : (1ull << a.G) - 1;
    const int rows = s.n_qv / a.G;
    // a window of 32 entries, one per lane: entries a window ahead of their scales, scales a window ahead of their use
    auto entry_at = [&](int i0) {
      int4 e = make_int4(-1, 0, 0, 0);
      if (i0 + lane < s.n_ent) {
        e = __ldcg(a.t.entries + s.ent0 + i0 + lane);
        if (e.x < 0 || e.x >= a.num_pages || e.y < 1 || e.y > PS) {
          atomicExch(a.t.counts + 4, int(MV_ERR_INVALID_ARG));
          e = make_int4(-1, 0, 0, 0);
        }
      }
      return e;
    };
    auto scale_at = [&](const int4& e) {
      return e.x >= 0 ? __ldcg(reinterpret_cast<const float2*>(a.scale) + int64_t(e.x) * a.Hkv + s.head) : make_float2(0.f, 1.f);
    };
    int4 e0 = entry_at(0), e1 = entry_at(32);
    float2 s0 = scale_at(e0), s1 = make_float2(0.f, 1.f);
    for (int t = 0; t < s.n_tiles && ok; ++t, ++tile) {
      const int at = (t * TILE_ENTRIES) & 31;
      if (at == 0 && t > 0) {
        e0 = e1;
        s0 = s1;
        e1 = entry_at(t * TILE_ENTRIES + 32);
      }
      if (at == 16) s1 = scale_at(e1);
      const int page = __shfl_sync(0xffffffffu, e0.x, at + (lane & 7));
      const unsigned present = __ballot_sync(0xffffffffu, lane < 8 && page >= 0);
      const uint32_t bytes = uint32_t(__popc(present)) * (PS * D);
      const int row = (page * a.Hkv + s.head) * PS;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv, ++piece) {
        const int slot = piece % RING;
        int go = 1;
        if (lane == 0) go = wait_or_flag(c, bar(&meta->empty[slot]), ((piece / RING) & 1) ^ 1) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, go, 0) != 0;
        if (!ok) break;
        if (kv == 0) {
          if (lane >= at && lane < at + TILE_ENTRIES) {
            Entry d;
            d.see_lo = d.see_hi = 0;
            d.rest = 127 << 8 | 127 << 16;
            if (e0.x >= 0) {
              const uint64_t mask = (uint64_t(uint32_t(e0.w)) << 32) | uint32_t(e0.z);
              uint64_t see = 0;
              if ((mask & ((rows >= 64 ? 0ull : (1ull << rows)) - 1)) == (rows >= 64 ? ~0ull : (1ull << rows) - 1)) see = live;
              else
                for (int r = 0; r < rows; ++r)
                  if ((mask >> r) & 1) see |= one_row << (r * a.G);
              uint32_t ek = uint32_t(mv::blk::scale_exponent(s0.x) + 127), ev = uint32_t(mv::blk::scale_exponent(s0.y) + 127);
              if (ev == 255) {
                ek = 255;
                ev = 127;
              }
              d.see_lo = uint32_t(see);
              d.see_hi = uint32_t(see >> 32);
              d.rest = uint32_t(e0.y) | ev << 8 | ek << 16;
            }
            meta->entry[tile % METAS][lane - at] = d;
          }
          __syncwarp();
          if (lane == 0) mv::mbar_arrive(bar(&meta->described[tile % METAS]));
        }
        const uint32_t fb = bar(&meta->full[slot]);
        if (lane == 0) mv::mbar_arrive_expect_tx(fb, bytes);
        __syncwarp();
        if (lane < 8 && page >= 0)
          mv::tma_load_2d_hint(c.base + slot * PIECE + lane * (PS * D), kv ? tm_v : tm_k, 0, row, fb, policy);
      }
    }
  }
  if (!ok) {
    // what is in flight must land before the CTA may leave
    if (lane == 0)
      for (int k = 1; k <= min(piece, RING); ++k)
        (void)mv::mbar_wait_bounded(bar(&meta->full[(piece - k) % RING]), ((piece - k) / RING) & 1, 20000000ull);
    __syncwarp();
  }
}

// ---- softmax warps ---------------------------------------------------------------------------------------
// q-vectors of the segment to the two K-major tiles (128-byte rows, 16-byte pieces XOR-swizzled with row % 8), eight threads per
// q-vector; factors and references of the segment
__device__ __forceinline__ void stage_q(const Cta& c, const mv::blk::Segment& s, int cols) {
  const Args& a = *c.a;
  const int tid = threadIdx.x, x0 = tid >> 3, ch = tid & 7;
  uint4 raw[4][2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = i * 16 + x0;
    raw[i][0] = raw[i][1] = make_uint4(0, 0, 0, 0);
    if (x < s.n_qv) {
      const uint4* src = reinterpret_cast<const uint4*>(a.q + (int64_t(s.row0 + x / a.G) * a.Hq + s.head * a.G + x % a.G) * D + ch * 16);
      raw[i][0] = __ldcg(src);
      raw[i][1] = __ldcg(src + 1);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = i * 16 + x0;
    if (i * 16 >= cols) break;
    const uint32_t w[8] = {raw[i][0].x, raw[i][0].y, raw[i][0].z, raw[i][0].w, raw[i][1].x, raw[i][1].y, raw[i][1].z, raw[i][1].w};
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = __vmaxu2(most, w[k] & 0x7fff7fffu);
    uint32_t amax = max(most & 0xffffu, most >> 16);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    // largest element into [128, 256)
    const int e = max(int(amax >> 7), 1) - 127 - 7;
    const float inv = amax < 0x7f80u ? mv::blk::exp2_int(-e) : __uint_as_float(0x7fc00000u);  // not finite: NaN
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t h2[2], l2[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t v = w[2 * k + j];
        const float p = __uint_as_float(v << 16) * inv, q = __uint_as_float(v & 0xffff0000u) * inv;
        h2[j] = mv::pack_e4m3x2(p, q);
        const float2 back = mv::unpack_e4m3x2(h2[j]);
        l2[j] = mv::pack_e4m3x2(p - back.x, q - back.y);
      }
      hi[k] = h2[0] | (h2[1] << 16);
      lo[k] = l2[0] | (l2[1] << 16);
    }
    unsigned char* dst = c.smem + OFF_Q + x * 128 + ((ch ^ (x & 7)) << 4);
    *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(dst + Q_BYTES) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    if (ch == 0) {
      c.meta->factor[x] = x < s.n_qv ? mv::blk::exp2_int(max(-126, min(e, 126))) * a.scale_log2 : 0.f;
      c.meta->minus_ref[x] = x < s.n_qv ? INFINITY : -INFINITY;
    }
  }
}

// Tensor-memory columns of a segment with `cols` columns of q-vectors: score buffers, O (values, then remainders), sums.  With 64
// columns there is room for one score buffer only.
struct Columns {
  int s1, o, sums;
  __device__ __forceinline__ explicit Columns(int cols) : s1(cols < 64 ? cols : 0), o(s1 + cols), sums(s1 + 3 * cols) {}
};

// The tiles of one segment and its result.  False: a wait ran out.
__device__ __forceinline__ bool run_segment(const Cta& c, const mv::blk::Segment& s, int& tile) {
  const Args& a = *c.a;
  Meta* const meta = c.meta;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int nb = (s.n_qv + 15) / 16, cols = nb * 16;
  const Columns at(cols);
  const uint32_t lanes = meta->tmem + (uint32_t(warp * 32) << 16);  // this warp's lanes
  float* const xch = reinterpret_cast<float*>(c.smem + OFF_P);       // exchange area: the weight tile while no product reads it
  const uint64_t live = s.n_qv >= 64 ? ~0ull : (1ull << s.n_qv) - 1;
  unsigned char* const p_row = c.smem + OFF_P + tid * 128;
  const int sw = tid & 7;
  bool ok = true;
#pragma unroll 1
  for (int t = 0; t < s.n_tiles; ++t, ++tile) {
    ok = ok && warp_wait(c, bar(&meta->described[tile % METAS]), (tile / METAS) & 1);
    const Entry en = meta->entry[tile % METAS][tid >> 4];
    const int tokens = en.rest & 0xff, ev = int((en.rest >> 8) & 0xff) - 127;
    const float ks = (en.rest >> 16) == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((en.rest >> 16) << 23);
    const bool valid = (tid & 15) < tokens;
    const uint64_t see = valid ? (uint64_t(en.see_hi) << 32) | en.see_lo : 0;
    const float evf = float(ev);
    const uint64_t ks2 = mv::pack_f32x2(ks, ks), ev2 = mv::pack_f32x2(evf, evf);
    const bool plain = __all_sync(0xffffffffu, see == live);
    const uint32_t s_t = lanes + ((tile & 1) ? at.s1 : 0);
    ok = ok && warp_wait(c, bar(&meta->s_full[tile & 1]), (tile >> 1) & 1);
    if (tile > 0) ok = ok && warp_wait(c, bar(&meta->pv_done), (tile - 1) & 1);  // the weight tile is free
    mv::um::fence_after();
    // Weights of the thread's token against the references as they stand, into the weight tile (row = token; values, then
    // remainders) and, times `sign` 2^(-e), into the token's sums.  Returns the largest weight.
    auto pass = [&](float sign, bool first) {
      float top = 0.f;
      const float vinv = sign * mv::blk::exp2_int(-ev);
      const uint64_t vinv2 = mv::pack_f32x2(vinv, vinv);
#pragma unroll 1
      for (int b = 0; b < nb; ++b) {
        uint32_t sc[16], l[16];
        mv::um::ld16(s_t + b * 16, sc);
        mv::um::ld16(lanes + at.sums + b * 16, l);
        mv::um::wait_ld();
        float p[16];
        const float4* const fa = reinterpret_cast<const float4*>(meta->factor + b * 16);
        const float4* const mr = reinterpret_cast<const float4*>(meta->minus_ref + b * 16);
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const float4 f = fa[j / 4], m = mr[j / 4];
          mv::unpack_f32x2(mv::fma_f32x2(mv::pack_u32x2(sc[j], sc[j + 1]), mv::mul_f32x2(mv::pack_f32x2(f.x, f.y), ks2), mv::add_f32x2(mv::pack_f32x2(m.x, m.y), ev2)), p[j], p[j + 1]);
          mv::unpack_f32x2(mv::fma_f32x2(mv::pack_u32x2(sc[j + 2], sc[j + 3]), mv::mul_f32x2(mv::pack_f32x2(f.z, f.w), ks2), mv::add_f32x2(mv::pack_f32x2(m.z, m.w), ev2)), p[j + 2], p[j + 3]);
#pragma unroll
          for (int i = 0; i < 4; ++i) p[j + i] = mv::fast_exp2(p[j + i]);
        }
        if (!plain) {
          const uint32_t mine = uint32_t(see >> (b * 16));
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (!((mine >> j) & 1)) p[j] = 0.f;
        }
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 16; j += 2) most = mv::max3(most, p[j], p[j + 1]);
        top = fmaxf(top, most);
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t h0, l0, h1, l1;
          split_e4m3x2(p[k * 4], p[k * 4 + 1], h0, l0);
          split_e4m3x2(p[k * 4 + 2], p[k * 4 + 3], h1, l1);
          hi[k] = h0 | (h1 << 16);
          lo[k] = l0 | (l1 << 16);
        }
        *reinterpret_cast<uint4*>(p_row + ((b ^ sw) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(p_row + (((b + nb) ^ sw) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        // A weight past the format's range only says that the references have to move; what it adds here is taken back then, so it must
        // not overflow (capped, it still exceeds what the move leaves of it, and the sum loses nothing but a rounding).
        if (most > 0x1p60f)
#pragma unroll
          for (int j = 0; j < 16; ++j) p[j] = p[j] > 0x1p60f ? 0x1p60f : p[j];
        if (first)
#pragma unroll
          for (int j = 0; j < 16; ++j) l[j] = 0;
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          float x, y;
          mv::unpack_f32x2(mv::fma_f32x2(mv::pack_f32x2(p[j], p[j + 1]), vinv2, mv::pack_u32x2(l[j], l[j + 1])), x, y);
          l[j] = __float_as_uint(x);
          l[j + 1] = __float_as_uint(y);
        }
        mv::um::st16(lanes + at.sums + b * 16, l);
      }
      mv::um::wait_st();
      return top;
    };
    float sign = 1.f;
    bool lift = t == 0;  // no references yet
    for (;;) {
      if (lift) {
        // ---- references move: the largest exponent of every q-vector over the tile's tokens
        if (!vote_all(ok)) return false;
#pragma unroll 1
        for (int b = 0; b < nb; ++b) {
          uint32_t sc[16];
          mv::um::ld16(s_t + b * 16, sc);
          mv::um::wait_ld();
          int best = 0;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int q = b * 16 + j;
            float y = fmaf(__uint_as_float(sc[j]), meta->factor[q] * ks, evf);
            if (!((see >> q) & 1) || y != y) y = -INFINITY;
            const int k = __float_as_int(y);
            const int m = __reduce_max_sync(0xffffffffu, k < 0 ? k ^ 0x7fffffff : k);  // ordered as the floats are
            if (lane == j) best = m;
          }
          if (lane < 16) xch[warp * MAXQV + b * 16 + lane] = __int_as_float(best < 0 ? best ^ 0x7fffffff : best);
        }
        (void)vote_all(true);
        if (tid < cols) {
          const float m = fmaxf(fmaxf(xch[tid], xch[MAXQV + tid]), fmaxf(xch[2 * MAXQV + tid], xch[3 * MAXQV + tid]));
          const float now = meta->minus_ref[tid], want = HEADROOM - m;
          float f = 1.f;
          if (tid < s.n_qv && m > -INFINITY && want < now) {
            f = mv::fast_exp2(want - now);  // 0 where there was none
            meta->minus_ref[tid] = want;
          }
          xch[4 * MAXQV + tid] = f;
        }
        (void)vote_all(true);
        if (t > 0) {
#pragma unroll 1
          for (int b = 0; b < 3 * nb; ++b) {  // O and the sums, which lie side by side
            uint32_t o[16];
            mv::um::ld16(lanes + at.o + b * 16, o);
            mv::um::wait_ld();
            const float* f = xch + 4 * MAXQV + (b % nb) * 16;
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f[j]);
            mv::um::st16(lanes + at.o + b * 16, o);
          }
          mv::um::wait_st();
        }
        (void)vote_all(true);  // every thread has read the exchange area
      }
      const float top = ok ? pass(sign, t == 0) : 0.f;
      if (lift) break;
      if (sign < 0.f) {  // the weights taken back
        sign = 1.f;
        lift = true;
        continue;
      }
      if (!vote_any(top > TOP || !ok)) break;
      sign = -1.f;
    }
    if (!__all_sync(0xffffffffu, valid)) {
      // no token here: whatever the slot holds meets a weight of zero, so it must be finite
      const int vp = 2 * tile + 1, vslot = vp % RING;
      ok = ok && warp_wait(c, bar(&meta->full[vslot]), (vp / RING) & 1);
      if (!valid) {
        uint4* const row = reinterpret_cast<uint4*>(c.smem + vslot * PIECE + tid * 128);
#pragma unroll
        for (int k = 0; k < 8; ++k) row[k] = make_uint4(0, 0, 0, 0);
      }
    }
    mv::fence_proxy_async();
    mv::um::fence_before();
    __syncwarp();
    if (lane == 0 && ok) mv::mbar_arrive(bar(&meta->p_full));
  }
  // ---- the segment's result: sums over the tokens, then the head vectors (thread = element)
  ok = ok && warp_wait(c, bar(&meta->pv_done), (tile - 1) & 1);
  if (!vote_all(ok)) return false;
  mv::um::fence_after();
#pragma unroll 1
  for (int b = 0; b < nb; ++b) {
    // sixteen columns over 32 lanes by halving: after four steps a lane holds one column's sum over half the lanes
    uint32_t l[16];
    mv::um::ld16(lanes + at.sums + b * 16, l);
    mv::um::wait_ld();
    float y[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) y[j] = __uint_as_float(l[j]);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
      const bool up = (lane & o) != 0;
#pragma unroll
      for (int j = 0; j < o; ++j) {
        const float keep = up ? y[j + o] : y[j], give = up ? y[j] : y[j + o];
        y[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    }
    y[0] += __shfl_xor_sync(0xffffffffu, y[0], 16);
    if (lane < 16) xch[warp * MAXQV + b * 16 + lane] = y[0];
  }
  (void)vote_all(true);
  if (tid < s.n_qv) {
    const float sum = (xch[tid] + xch[MAXQV + tid]) + (xch[2 * MAXQV + tid] + xch[3 * MAXQV + tid]);
    xch[4 * MAXQV + tid] = sum == 0.f ? 0.f : 1.f / sum;
    if (s.slot >= 0) a.part_ml[s.slot * MAXQV + tid] = make_float2(-meta->minus_ref[tid], sum);  // no token seen: reference -infinity, sum 0
  }
  (void)vote_all(true);
  int r = 0, h = 0;  // row and head of q-vector q
#pragma unroll 1
  for (int b = 0; b < nb; ++b) {
    uint32_t o0[16], o1[16];
    mv::um::ld16(lanes + at.o + b * 16, o0);
    mv::um::ld16(lanes + at.o + (nb + b) * 16, o1);
    mv::um::wait_ld();
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int q = b * 16 + j;
      if (q < s.n_qv) {
        const float y = fmaf(__uint_as_float(o1[j]), 1.f / LO_SCALE, __uint_as_float(o0[j]));
        if (s.slot >= 0) a.part_o[(int64_t(s.slot) * MAXQV + q) * D + tid] = y;
        else a.out[(int64_t(s.row0 + r) * a.Hq + s.head * a.G + h) * D + tid] = __float2bfloat16_rn(y * xch[4 * MAXQV + q]);
        if (++h == a.G) {
          h = 0;
          ++r;
        }
      }
    }
  }
  mv::um::fence_before();
  (void)vote_all(true);  // O and the exchange area have been read
  return true;
}

__device__ __forceinline__ void softmax_warps(const Cta& c) {
  Walk w;
  w.begin(*c.a, blockIdx.x);
  mv::blk::Segment s;
  int tile = 0;  // tiles of the share so far: ring position, score buffer and phases follow from it
  bool ok = true;
  while (ok && w.next(*c.a, s, false)) {
    stage_q(c, s, (s.n_qv + 15) / 16 * 16);
    mv::fence_proxy_async();
    (void)vote_all(true);  // the factors are there for all
    if ((threadIdx.x & 31) == 0) mv::mbar_arrive(bar(&c.meta->q_full));
    ok = run_segment(c, s, tile);
  }
}

// ---- issuer warp: the whole warp walks and waits, one elected lane issues ----------------------------------
__device__ __forceinline__ void issuer(const Cta& c) {
  Meta* const meta = c.meta;
  const bool lead = mv::um::elect_one();
  const uint32_t tmem = meta->tmem;
  const uint64_t q_desc = mv::um::smem_desc(c.base + OFF_Q, 16, 1024);
  const uint64_t p_desc = mv::um::smem_desc(c.base + OFF_P, PIECE, 1024);
  Walk w;
  w.begin(*c.a, blockIdx.x);
  mv::blk::Segment s;
  int tile = 0, segment = 0;
  bool ok = true;
  while (ok && w.next(*c.a, s, false)) {
    const int cols = (s.n_qv + 15) / 16 * 16;
    const Columns at(cols);
    const uint32_t o_t = tmem + at.o;
    const uint32_t idesc_s = mv::um::idesc_e4m3(128, cols, 0, 0), idesc_o = mv::um::idesc_e4m3(128, 2 * cols, 1, 1);
    ok = warp_wait(c, bar(&meta->q_full), segment & 1);
    ++segment;
    // S^T = K Q^T of tile t of the share into score buffer t & 1: K is the 128-row operand, values of Q then remainders
    auto scores = [&](int t) {
      const int slot = (2 * t) % RING;
      ok = ok && warp_wait(c, bar(&meta->full[slot]), ((2 * t) / RING) & 1);
      if (!ok) return;
      mv::um::fence_after();
      if (lead) {
        const uint64_t k_desc = mv::um::smem_desc(c.base + slot * PIECE, 16, 1024);
        const uint32_t s_t = tmem + ((t & 1) ? at.s1 : 0);
        mv::um::mma8_ss<false>(s_t, k_desc, q_desc, idesc_s);
#pragma unroll
        for (int k = 1; k < D / 32; ++k) mv::um::mma8_ss<true>(s_t, k_desc + uint32_t((k * 32) >> 4), q_desc + uint32_t((k * 32) >> 4), idesc_s);
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
          mv::um::mma8_ss<true>(s_t, k_desc + uint32_t((k * 32) >> 4), q_desc + uint32_t((Q_BYTES + k * 32) >> 4), idesc_s);
        mv::um::commit(bar(&meta->s_full[t & 1]));
        mv::um::commit(bar(&meta->empty[slot]));
      }
      __syncwarp();
    };
    scores(tile);
#pragma unroll 1
    for (int t = 0; t < s.n_tiles && ok; ++t, ++tile) {
      // the other score buffer was read before the weights of tile t - 1 were handed over; a single one before those of tile t are
      if (t + 1 < s.n_tiles && cols < 64) scores(tile + 1);
      const int vp = 2 * tile + 1, vslot = vp % RING;
      ok = ok && warp_wait(c, bar(&meta->p_full), tile & 1);
      if (t + 1 < s.n_tiles && cols == 64) scores(tile + 1);
      ok = ok && warp_wait(c, bar(&meta->full[vslot]), (vp / RING) & 1);
      if (!ok) break;
      mv::um::fence_after();
      if (lead) {
        // O^T += V^T P^T: V is the 128-row operand, read across its rows (32 tokens per instruction)
        const uint64_t v_desc = mv::um::smem_desc(c.base + vslot * PIECE, PIECE, 1024);
        if (t == 0) mv::um::mma8_ss<false>(o_t, v_desc, p_desc, idesc_o);
        else mv::um::mma8_ss<true>(o_t, v_desc, p_desc, idesc_o);
#pragma unroll
        for (int k = 1; k < TILE / 32; ++k) mv::um::mma8_ss<true>(o_t, v_desc + uint32_t((k * 4096) >> 4), p_desc + uint32_t((k * 4096) >> 4), idesc_o);
        mv::um::commit(bar(&meta->pv_done));
        mv::um::commit(bar(&meta->empty[vslot]));
      }
      __syncwarp();
    }
  }
  if (!ok) {
    // products may still be in flight: they must have completed before the CTA frees its tensor memory
    if (lead) mv::um::commit(bar(&meta->drained));
    (void)mv::mbar_wait_bounded(bar(&meta->drained), 0, 20000000ull);
    __syncwarp();
  }
}

__global__ void __launch_bounds__(NT, 2) decode_blk_tc_kernel(const Args a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Meta* const meta = reinterpret_cast<Meta*>(smem + OFF_META);
  const int tid = threadIdx.x, warp = tid >> 5;
  const uint32_t base = mv::smem_u32(smem);
  if ((base & 1023u) != 0) {  // the swizzle pattern is anchored at 1024-byte boundaries
    if (tid == 0) atomicExch(a.t.counts + 4, int(MV_ERR_UNSUPPORTED));
    return;
  }
  if (tid == 0) {
    meta->abort = 0;
    for (int i = 0; i < RING; ++i) {
      mv::mbar_init(bar(&meta->full[i]), 1);   // the producer's arrive (+ the bytes TMA reports)
      mv::mbar_init(bar(&meta->empty[i]), 1);  // one tcgen05.commit after the product that read the piece
    }
    for (int i = 0; i < METAS; ++i) mv::mbar_init(bar(&meta->described[i]), 1);
    for (int i = 0; i < 2; ++i) mv::mbar_init(bar(&meta->s_full[i]), 1);
    mv::mbar_init(bar(&meta->q_full), 4);   // the softmax warps
    mv::mbar_init(bar(&meta->p_full), 4);
    mv::mbar_init(bar(&meta->pv_done), 1);
    mv::mbar_init(bar(&meta->drained), 1);
    mv::mbar_fence_init();
    mv::fence_proxy_async();
  }
  if (warp == 0) {
    mv::um::tmem_alloc(mv::smem_u32(&meta->tmem), 256);
    mv::um::tmem_relinquish();
  }
  mv::um::fence_before();
  __syncthreads();
  mv::um::fence_after();
  // launched with programmatic stream serialisation: what is above may overlap the end of the kernel before
  mv::grid_dependency_wait();
  mv::grid_dependency_launch_dependents();
  Cta c{&a, smem, base, meta, a.t.counts + 4};
  if (warp == 4) producer(c, &tm_k, &tm_v);
  else if (warp == 5) issuer(c);
  else softmax_warps(c);
  mv::um::fence_before();
  __syncthreads();
  if (warp == 0) mv::um::tmem_dealloc(meta->tmem, 256);
}

struct Maps {
  CUtensorMap k, v;
};

}  // namespace

namespace mv {
// Attention kernel of mv_dag_decode_attn_fp8_blk at head_dim 128 (the caller validated the arguments and launches the merge).
mv_status decode_blk_tc(const blk::Args& a, cudaStream_t st) {
  static std::atomic<uint64_t> opted{0};  // per device
  if (!opt_in_smem(decode_blk_tc_kernel, SMEM, opted)) return MV_ERR_CUDA;
  static thread_local KeyedCache<Maps, 4> cache;
  const int64_t rows = a.num_pages * a.Hkv * PS;  // 128-byte rows of a pool
  const TmapKey key{current_device(), a.k8, a.v8, nullptr, rows, 9};
  Maps* hit = cache.find(key);
  if (!hit) {
    hit = cache.claim(key);
    if (!make_tmap_u8_2d(&hit->k, a.k8, uint64_t(rows), PS) || !make_tmap_u8_2d(&hit->v, a.v8, uint64_t(rows), PS)) {
      cache.drop();
      return MV_ERR_CUDA;
    }
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(SHARES, 1, 1);
  cfg.blockDim = dim3(NT, 1, 1);
  cfg.dynamicSmemBytes = SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, decode_blk_tc_kernel, a, hit->k, hit->v);
  g_launches++;
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return MV_ERR_CUDA;
  }
  return MV_OK;
}
}  // namespace mv
