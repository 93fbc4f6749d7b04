// Decode attention over the block-scaled 8-bit cache on the tensor cores, accumulators in tensor memory.
// For the q-vectors x of a stream (rows of a group x query heads of one KV head) and the tokens j its entries name,
//   s_xj = <q_x, K_j> * sK[page] * c,  c = softmax scale * log2 e        (log2 units)
//   out_x = sum_j 2^(s_xj) sV[page] V_j / sum_j 2^(s_xj)
// The scale of V is a power of two, 2^e, so it goes into the exponent: weights p_xj = 2^(s_xj + e_j - m_x) multiply the
// stored bytes, and the denominator takes p_xj 2^(-e_j).  The reference m_x follows the largest s + e, which
// keeps the weights of whatever dominates the NUMERATOR near one however much the pages' scales differ; with
// exponents in [-80, 40] a token that matters to the denominator alone still gets a weight above 2^-126.
// Block scale NaN: the scores of the rows that see the page become NaN; a row that does not see it multiplies
// finite bytes by zero.
//
// Both products run with the CACHE as the 128-row operand, straight on the pool's bytes: S^T = K Q^T puts a tile's 128 tokens
// on the 128 lanes of tensor memory and the q-vectors on its columns, O^T = V^T P^T the 128 elements of the head vector on the
// lanes.  A softmax thread therefore owns a token and works on exactly the q-vectors there are (16, 32, 48 or 64 columns),
// all 128 lanes always busy, instead of owning one of at most 64 q-vectors; per tile it reads one mask, one token count
// and one pair of scales.
//   - Q is two K-major tiles of 8-bit floats, the rounded element and its rounded remainder at one power-of-two scale per
//     q-vector: a bf16 element has eight significant bits, value plus remainder hold nine, so the split is exact
//     for elements within 2^-9 of the vector's largest (and off by at most 2^-17 of the largest below).  A power of its own for every
//     vector costs a multiplication per pair of scores (128 mixed requests 441 -> 460 us); with one for the whole stream a head 2^12 below
//     another lost 2 % of its result, one 2^16 below 28 %.
//   - The weights are three tiles of 8-bit floats with five exponent bits (the upper byte of a half-precision number): the weight in
//     half precision cut to its upper byte, what is left of it rounded to one, and what is left then.  All have the same scale.  A
//     weight is off by at most 1.5 * 2^-10 of itself (2^-11 in half precision, 2^-10 behind the third byte) or 2^-17, where the largest
//     one stands at 2^12 or more: 2^-29 of it.  That far down because history is long: a sink that takes 97 % of a row leaves each of
//     64K other tokens 2^-21 of its weight, and together they may be all of the result.
//     Three and not two: a value with three mantissa bits and 16 times its remainder end at 2^-19 of the largest weight.
//   - The reference exponent of a q-vector moves only when a weight would pass the format's largest value (57344): every
//     thread looks at its own weights and one barrier votes, so the maximum over the tokens (a reduction across lanes) is taken only
//     on a stream's first tile and in the rare tile that lifts it.
// The softmax warps keep the sums of a token (one per q-vector) in tensor memory as well, and walk the columns sixteen at a time (the
// references and the results eight at a time) in a loop that is not unrolled: with the columns unrolled (per-thread arrays, a code path per number of columns) misses of
// the SM's instruction cache cost three cycles per instruction.
// A CTA is four softmax warps (a thread per token), a producer warp each for K and V and an issuer warp for either product; two
// CTAs per SM hide each other's hand-overs.  K and V tiles have two slots apiece (V one where the weights need the other), scores and
// weights two buffers, so that the products of one tile overlap the weights of the next.
// With head_dim 64 a cache row is 64 bytes: everything is the same but for the swizzle, and the second product takes V's 64 elements
// twice to fill the 128 lanes.
// Measured (cache not in the L2, a call with its merge): 128 requests of mixed length, 64 query over 8 KV heads, 2.1 GB of cache, 511 us
// (4.1 TB/s; one set of inputs again and again 459); 32 layered requests, 446 MB, 101 us (4.4 TB/s); 16 requests, 107 MB, 36 us; 64K
// tokens alone, 136 MB, 34 us; a short request 15.7 us; 37 requests of 64-element heads 29 us.
// What bounds it: with 16 q-vectors the bytes (5.6 TB/s of DRAM reads inside the kernel); with 64 the loop over the weights (2.2 TB/s, the tensor
// pipe 17 % busy, 47 % of the issue slots; more warps do not fit the registers); in small calls the chain of launch, tables, first
// bytes, epilogue and merge, about 13 us.
// Slower: eight softmax warps per CTA (register limit of 80), the column loop unrolled by two (instruction fetches), scores or sums
// loaded ahead of their use (registers), the second product held back until the next scores are out.
// Every wait is bounded; the softmax warps vote once per tile, and the vote carries a failed wait, so that they leave together.
#include <algorithm>

#include "blk_stream.cuh"
#include "umma.cuh"

namespace {

using bf16 = __nv_bfloat16;
using mv::blk::Args;
using mv::blk::MAXQV;
using mv::blk::PS;
using mv::blk::SHARES;
using mv::blk::TILE_ENTRIES;

constexpr int TILE = 128;                 // tokens per tile
constexpr int RING = 4;                   // K in slots 0 and 2, V in slots 1 and 3 (see Slots)
constexpr int METAS = 4;                  // descriptions that may be live: K of tile j waits for the scores of tile j - 2, which wait for the weights of tile j - 4
// Weights of a tile.  Up to 32 columns: [128 tokens][128 bytes], the three bytes of a weight `cols` apart, 128-byte swizzle, and one
// product over 3 * cols columns whose thirds are joined at the end.  From 48 columns on: three tiles [128 tokens][64 bytes], 64-byte
// swizzle, and three products that add up in the same columns.  Two tiles of weights either way; at head_dim 128 the wide ones take
// V's second slot as well (with one tile of weights 64 columns wait for the product before: 128 mixed requests 483 instead of 440 us).
// Narrow or wide: an instruction of the second product costs some 47 cycles however few its columns, so three times as many do not pay
// up to 32 columns: 48 requests of 8 q-vectors 104 us against 144, 32 layered ones of up to 24 92 against 96, 128 mixed ones 440 against 468.
constexpr int P_NARROW = TILE * 128, P_THIRD = TILE * 64, P_WIDE = 3 * P_THIRD;
constexpr int SOFTMAX = 128;
constexpr int NT = SOFTMAX + 128;         // and four warps: K, V, first products, second products
constexpr float TOP = 57344.f;            // largest 8-bit float with five exponent bits
constexpr float HEADROOM = 12.f;          // a reference that moves puts the largest weight at 2^12
constexpr float CAP = 0x1p20f;            // what a weight past TOP counts as until the references have moved
// Least exponent of a scale of V, below what the cache write gives (2^-60): a scale of zero (a block nobody has quantised, or zeros) counts
// as 2^-80.  Sums hold weight * 2^80 at most, below 2^124 for 2^23 tokens, and weights go down to 2^-126, which leaves 2^46 for the other end.
constexpr int V_MIN = -80;

// One page of a tile, as the softmax threads need it: K's exponent (biased) in bits 23 to 30, V's in bits 15 to 22, the tokens in the low
// byte, and two marks.
constexpr uint32_t ALL_SEE = 256, LOST = 512;  // sixteen tokens that every q-vector sees; either scale is NaN
struct Meta {
  alignas(16) float minus_ref[MAXQV];    // minus the reference of a q-vector (+infinity: none yet; -infinity: no such q-vector); read four at a time
  alignas(16) uint16_t unit[MAXQV];      // power of two of a q-vector's 8-bit floats, upper half of the float; read eight at a time
  uint2 see[METAS][TILE_ENTRIES];        // q-vectors that see a page
  uint32_t page[METAS][TILE_ENTRIES];
  uint2 seen[METAS];                     // q-vectors that see some page of the tile
  uint64_t full[RING], empty[RING], described[METAS], s_full[2], q_full, p_full[2], pv_done[2], drained[2];
  int abort;
  uint32_t tmem;
};
static_assert(sizeof(Meta) <= 1024, "meta area");
static_assert(offsetof(Meta, minus_ref) % 16 == 0 && offsetof(Meta, unit) % 16 == 0, "vector loads");

// Shared memory.  A row of the cache is a token's D bytes, and so is a row of the tiles: 128 bytes with the 128-byte swizzle, or 64
// bytes with the 64-byte swizzle.
template <int D>
struct Lay {
  static constexpr int PIECE = TILE * D;           // K or V of a tile
  static constexpr int P = RING * PIECE;           // weights
  static constexpr bool BORROWS = D == 128;        // V's second slot holds weights in segments of 48 and 64 columns
  static constexpr int PW = BORROWS ? P - PIECE : P;
  static constexpr int Q = PW + 2 * P_WIDE;        // Q values [64][D], then Q remainders
  static constexpr int Q_BYTES = MAXQV * D;
  static_assert(P + 2 * P_NARROW <= Q && Q % 1024 == 0, "room for both kinds");
  static constexpr int META = Q + 2 * Q_BYTES;
  static constexpr int SMEM = META + 1024;
  static_assert(2 * (SMEM + 1024) <= 228 * 1024, "two CTAs per SM");
  // operand of the cache or of Q: groups of eight rows follow one another; where a row is 64 bytes, the first operand of the second product, which
  // is 128 elements high, takes the 64 elements twice (distance 0 between its blocks)
  static __device__ __forceinline__ uint64_t desc(uint32_t addr) {
    return D == 128 ? mv::um::smem_desc(addr, 16, 1024) : mv::um::smem_desc_64b(addr, 0, 512);
  }
};

__device__ __forceinline__ uint32_t bar(const void* p) { return mv::smem_u32(p); }
__device__ __forceinline__ int columns_of(int n_qv) { return (n_qv + 15) / 16 * 16; }
__device__ __forceinline__ bool in_thirds(int cols) { return cols <= 32; }

// Slots of K (0 and 2) or V (1 and 3) in the order in which tiles take them: in turn, or the first one alone while the second holds
// weights.  The tile after such a segment takes the first slot again, and with it waits for the segment's last product: the second is free then.
struct Slots {
  int first;
  uint32_t second = 0, phase = 0;  // phase: bit per slot, parity of its next fill
  __device__ __forceinline__ void begin(bool both) { second = both ? second : 0; }
  __device__ __forceinline__ int slot() const { return first + 2 * int(second); }
  __device__ __forceinline__ uint32_t parity() const { return (phase >> second) & 1; }
  __device__ __forceinline__ void advance(bool both) {
    phase ^= 1u << second;
    second = both ? second ^ 1 : 0;
  }
};
template <int D>
__device__ __forceinline__ bool both_slots_of_v(int cols) { return in_thirds(cols) || !Lay<D>::BORROWS; }

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
// Barriers of the softmax warps that carry a predicate.
__device__ __forceinline__ bool vote_any(bool p) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(uint32_t(p)), "n"(SOFTMAX) : "memory");
  return r != 0;
}
__device__ __forceinline__ bool vote_all(bool p) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 2, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(uint32_t(p)), "n"(SOFTMAX) : "memory");
  return r != 0;
}

// Four weights (not negative) -> the three bytes of each: upper byte of the half-precision number, the remainder rounded to its upper
// byte, the second remainder likewise (half a step is added to the magnitude, whose bits count up across exponents).  The differences are
// exact.  A NaN stays one in the first byte.
__device__ __forceinline__ void split_weights(float x0, float x1, float x2, float x3, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  constexpr uint32_t UPPER = 0xff00ff00u, HALF_STEP = 0x00800080u;
  uint32_t h[2], m[2], l[2];
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(h[0]) : "f"(x1), "f"(x0));
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(h[1]) : "f"(x3), "f"(x2));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(h[i]), "r"(h[i] & UPPER));
    m[i] = r + HALF_STEP;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(l[i]) : "r"(r), "r"(m[i] & UPPER));
    l[i] += HALF_STEP;
  }
  hi = __byte_perm(h[0], h[1], 0x7531);
  mid = __byte_perm(m[0], m[1], 0x7531);
  lo = __byte_perm(l[0], l[1], 0x7531);
}

// ---- producer warps: one for K and the tiles' descriptions, one for V ---------------------------------------
// Eight boxes, a page each, make a piece; one lane sends them all, with the rows in uniform registers.  Sending a box occupies its
// warp for about 75 cycles: a warp that sent K and V of a tile could not keep up with the stream.
template <int D, bool IS_K>
__device__ __forceinline__ void producer(const Cta& c, mv::blk::Walk& w, mv::blk::Segment& s, bool more, const CUtensorMap* map) {
  const Args& a = *c.a;
  Meta* const meta = c.meta;
  const int lane = threadIdx.x & 31;
  const bool lead = mv::um::elect_one();
  const uint64_t policy = mv::l2_policy_evict_first();  // the cache is read once per call
  int tile = 0;
  Slots ring{IS_K ? 0 : 1};
  bool ok = true;
  // a window of 32 entries, one per lane
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
  for (; ok && more; more = ok && w.next(a, s)) {
    // what the softmax threads need of an entry
    auto describe = [&](const int4& e, const float2& sc, uint64_t& see) {
      uint32_t page = 127u << 23 | 127u << 15;
      see = 0;
      if (e.x >= 0) {
        const int rows = s.n_qv / a.G;
        const uint64_t all_rows = rows >= 64 ? ~0ull : (1ull << rows) - 1;
        const uint64_t mask = ((uint64_t(uint32_t(e.w)) << 32) | uint32_t(e.z)) & all_rows;
        if (mask == all_rows) {
          see = s.n_qv >= 64 ? ~0ull : (1ull << s.n_qv) - 1;
        } else {
          const uint64_t one_row = a.G >= 64 ? ~0ull : (1ull << a.G) - 1;
#pragma unroll 1
          for (int r = 0; r < rows; ++r)
            if ((mask >> r) & 1) see |= one_row << (r * a.G);
        }
        const uint32_t ek = uint32_t(mv::blk::scale_exponent(sc.x) + 127), ev = uint32_t(mv::blk::scale_exponent(sc.y) + 127);
        page = ek << 23 | (ev == 255 ? 127u : max(ev, uint32_t(127 + V_MIN))) << 15 | (ek == 255 || ev == 255 ? LOST : 0u) | (mask == all_rows && e.y == PS ? ALL_SEE : 0u) | uint32_t(e.y);
      }
      return page;
    };
    const bool both = IS_K || both_slots_of_v<D>(columns_of(s.n_qv));
    ring.begin(both);
    int4 e0 = entry_at(0), e1 = entry_at(32);
    float2 s0 = make_float2(0.f, 1.f);
    if (IS_K) s0 = scale_at(e0);
    uint32_t page0 = 0;
    uint64_t see0 = 0;
#pragma unroll 1
    for (int t = 0; t < s.n_tiles; ++t, ++tile) {
      const int at = (t * TILE_ENTRIES) & 31;
      if (at == 0 && t > 0) {
        e0 = e1;
        e1 = entry_at(t * TILE_ENTRIES + 32);
      }
      const unsigned present = (__ballot_sync(0xffffffffu, e0.x >= 0) >> at) & 0xffu;
      const int my_row = (e0.x * a.Hkv + s.head) * PS;
      const int slot = ring.slot();
      ok = warp_wait(c, bar(&meta->empty[slot]), ring.parity() ^ 1);
      if (!ok) break;
      ring.advance(both);
      const uint32_t fb = bar(&meta->full[slot]), dst = c.base + slot * Lay<D>::PIECE;
      if (lead) mv::mbar_arrive_expect_tx(fb, uint32_t(__popc(present)) * (PS * D));
#pragma unroll
      for (int j = 0; j < TILE_ENTRIES; ++j) {
        const int row = __shfl_sync(0xffffffffu, my_row, at + j);
        if (lead && ((present >> j) & 1)) mv::tma_load_2d_hint(dst + j * (PS * D), map, 0, row, fb, policy);
      }
      __syncwarp();
      if (IS_K) {
        if (at == 0) page0 = describe(e0, s0, see0);
        const bool mine = lane >= at && lane < at + TILE_ENTRIES;
        const uint32_t any_lo = __reduce_or_sync(0xffffffffu, mine ? uint32_t(see0) : 0), any_hi = __reduce_or_sync(0xffffffffu, mine ? uint32_t(see0 >> 32) : 0);
        if (mine) {
          meta->see[tile % METAS][lane - at] = make_uint2(uint32_t(see0), uint32_t(see0 >> 32));
          meta->page[tile % METAS][lane - at] = page0;
        }
        if (lane == 0) meta->seen[tile % METAS] = make_uint2(any_lo, any_hi);
        __syncwarp();
        if (lane == 0) mv::mbar_arrive(bar(&meta->described[tile % METAS]));
        if (at == 16) s0 = scale_at(e1);  // of the next window
      }
    }
  }
  if (!ok) {
    // what is in flight must land before the CTA may leave: the last fills of this warp's slots
    if (lane == 0)
      for (int k = 0; k < 2; ++k) (void)mv::mbar_wait_bounded(bar(&meta->full[ring.first + 2 * k]), ((ring.phase >> k) & 1) ^ 1, 20000000ull);
    __syncwarp();
  }
}

// ---- softmax warps ---------------------------------------------------------------------------------------
// q-vectors of the segment to the two K-major tiles (16-byte pieces XOR-swizzled as TMA does it for the cache), eight threads per
// q-vector, each vector at its own power of two: what a row gets does not depend on the rows and heads that share its stream.
template <int D>
__device__ __forceinline__ void stage_q(const Cta& c, const mv::blk::Segment& s, int cols) {
  const Args& a = *c.a;
  constexpr int ROWS = SOFTMAX / 8, STEPS = MAXQV / ROWS;  // q-vectors at a time
  constexpr int LOADS = D / 64;                            // 16-byte loads of a thread
  const int tid = threadIdx.x, x0 = tid >> 3, ch = tid & 7;
  uint4* const raw = reinterpret_cast<uint4*>(c.smem + Lay<D>::P);  // the q-vectors as they are, in the weight tiles
  uint4 in[STEPS][LOADS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int x = i * ROWS + x0;
#pragma unroll
    for (int k = 0; k < LOADS; ++k) in[i][k] = make_uint4(0, 0, 0, 0);
    if (x < s.n_qv) {
      const uint4* src = reinterpret_cast<const uint4*>(a.q + (int64_t(s.row0 + x / a.G) * a.Hq + s.head * a.G + x % a.G) * D + ch * (D / 8));
#pragma unroll
      for (int k = 0; k < LOADS; ++k) in[i][k] = __ldcg(src + k);
    }
  }
  if (tid < cols) c.meta->minus_ref[tid] = tid < s.n_qv ? INFINITY : -INFINITY;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int x = i * ROWS + x0;
    if (x < cols) {
#pragma unroll
      for (int k = 0; k < LOADS; ++k) raw[(x * 8 + ch) * LOADS + k] = in[i][k];  // (each thread reads back its own)
    }
  }
#pragma unroll 1
  for (int x = x0; x < cols; x += ROWS) {
    uint32_t w[4 * LOADS], hi[2 * LOADS], lo[2 * LOADS], m = 0;
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const uint4 u = raw[(x * 8 + ch) * LOADS + k];
      w[4 * k] = u.x; w[4 * k + 1] = u.y; w[4 * k + 2] = u.z; w[4 * k + 3] = u.w;
      m = __vmaxu2(m, __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu)));
    }
    // largest element into [128, 256) (a vector that is not finite gives NaN at any power)
    m = max(m & 0xffffu, m >> 16);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    const int e = max(-120, max(min(int(m >> 7), 254), 1) - 127 - 7);
    const float inv = mv::blk::exp2_int(-e);
    if (ch == 0) c.meta->unit[x] = uint16_t(__float_as_uint(mv::blk::exp2_int(e)) >> 16);
#pragma unroll
    for (int k = 0; k < 2 * LOADS; ++k) {
      uint32_t h2[2], l2[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float p = __uint_as_float(w[2 * k + j] << 16) * inv, q = __uint_as_float(w[2 * k + j] & 0xffff0000u) * inv;
        // infinities become NaN: inf * 0
        h2[j] = mv::pack_e4m3x2(fmaf(p, 0.f, p), fmaf(q, 0.f, q));
        const float2 back = mv::unpack_e4m3x2(h2[j]);
        l2[j] = mv::pack_e4m3x2(p - back.x, q - back.y);
      }
      hi[k] = h2[0] | (h2[1] << 16);
      lo[k] = l2[0] | (l2[1] << 16);
    }
    unsigned char* const row = c.smem + Lay<D>::Q + x * D;
    if constexpr (D == 128) {
      unsigned char* const dst = row + ((ch ^ (x & 7)) << 4);
      *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(dst + Lay<D>::Q_BYTES) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    } else {
      unsigned char* const dst = row + ((((ch >> 1) ^ ((x >> 1) & 3)) << 4) | ((ch & 1) << 3));
      *reinterpret_cast<uint2*>(dst) = make_uint2(hi[0], hi[1]);
      *reinterpret_cast<uint2*>(dst + Lay<D>::Q_BYTES) = make_uint2(lo[0], lo[1]);
    }
  }
}

// Tensor-memory columns of a segment with `cols` columns of q-vectors: two score buffers, O (in three parts up to 32 columns), sums.
struct Columns {
  int parts, s1, o, sums;
  __device__ __forceinline__ explicit Columns(int cols) : parts(in_thirds(cols) ? 3 : 1), s1(cols), o(2 * cols), sums((2 + parts) * cols) {}
};

// The tiles of one segment and its result.  False: a wait ran out.
template <int D>
__device__ __forceinline__ bool run_segment(const Cta& c, const mv::blk::Segment& s, int& tile, Slots& v_ring) {
  const Args& a = *c.a;
  Meta* const meta = c.meta;
  const int tid = threadIdx.x, token = tid, quarter = tid >> 5, lane = tid & 31;
  const int nb = (s.n_qv + 15) / 16, cols = nb * 16, n8 = cols / 8;
  auto each_eight = [&](auto f) {  // f for every eight columns
#pragma unroll 1
    for (int b = 0; b < n8; ++b) f(b);
  };
  const Columns at(cols);
  const uint32_t lanes = meta->tmem + (uint32_t(quarter * 32) << 16);  // this warp's lanes
  const bool thirds = in_thirds(cols);
  const int sw = thirds ? token & 7 : (token >> 1) & 3;                           // swizzle of the token's row of weights
  const int p_next = thirds ? nb : 0, p_plane = thirds ? 0 : P_THIRD;             // from one byte of a weight to the next: pieces of the row, or bytes
  bool ok = true;
  v_ring.begin(both_slots_of_v<D>(cols));
  const float scale = a.scale_log2;
  uint64_t referenced = 0;  // q-vectors that have a reference (or saw scores that were not numbers)
#pragma unroll 1
  for (int t = 0; t < s.n_tiles; ++t, ++tile) {
    // the tile's description and scores, and a weight tile that no product reads any more
    const bool arrived = ok && wait_or_flag(c, bar(&meta->described[tile % METAS]), (tile / METAS) & 1) &&
                         wait_or_flag(c, bar(&meta->s_full[tile & 1]), (tile >> 1) & 1) &&
                         (tile < 2 || wait_or_flag(c, bar(&meta->pv_done[tile & 1]), ((tile - 2) >> 1) & 1));
    ok = __all_sync(0xffffffffu, arrived);
    mv::um::fence_after();
    const uint32_t page = meta->page[tile % METAS][token >> 4];
    const uint2 by = meta->see[tile % METAS][token >> 4];
    const bool plain = __all_sync(0xffffffffu, page & ALL_SEE);
    const uint32_t vs_bits = (page << 8) & 0x7f800000u;
    const float evf = float(int(vs_bits >> 23) - 127), vinv = __uint_as_float((254u << 23) - vs_bits);  // exponent; 2^-exponent
    const float fk = (page & LOST ? __uint_as_float(0x7fc00000u) : __uint_as_float(page & 0x7f800000u)) * scale;
    const uint64_t fk2 = mv::pack_f32x2(fk, fk), ev2 = mv::pack_f32x2(evf, evf);
    const uint32_t s_t = lanes + ((tile & 1) ? at.s1 : 0);
    unsigned char* const p_tile = c.smem + (thirds ? Lay<D>::P + (tile & 1) * P_NARROW : Lay<D>::PW + (tile & 1) * P_WIDE);
    unsigned char* const p_row = p_tile + token * (thirds ? 128 : 64);
    float* const xch = reinterpret_cast<float*>(p_tile);  // exchange area until the weights stand
    bool valid = true;
    uint64_t see = ~0ull;
    if (!plain) {
      valid = (token & 15) < int(page & 255u);
      see = valid ? (uint64_t(by.y) << 32) | by.x : 0;
    }
    // Weights of the thread's token against the references as they stand, into the weight tile (row = token) and, times
    // `sign` 2^(-e), into the token's sums.  Returns the largest weight.
    auto pass = [&](float sign, bool first) {
      float top = 0.f;
      const uint64_t vinv2 = mv::pack_f32x2(sign * vinv, sign * vinv);
      mv::um::wait_st();  // the sums as the last pass left them
#pragma unroll 1
      for (int u = 0; u < nb; ++u) {
        constexpr int W = 16;
        const int col = u * W;
        uint32_t sc[W];
        mv::um::ld16(s_t + col, sc);
        const float4* const mr = reinterpret_cast<const float4*>(meta->minus_ref + col);
        const uint4* const un = reinterpret_cast<const uint4*>(meta->unit + col);
        float p[W];
        mv::um::wait_ld();
#pragma unroll
        for (int j = 0; j < W; j += 4) {
          const float4 y = mr[j / 4];
          const uint32_t u0 = j % 8 ? un[j / 8].z : un[j / 8].x, u1 = j % 8 ? un[j / 8].w : un[j / 8].y;
          const uint64_t f01 = mv::mul_f32x2(mv::pack_u32x2(u0 << 16, u0 & 0xffff0000u), fk2), f23 = mv::mul_f32x2(mv::pack_u32x2(u1 << 16, u1 & 0xffff0000u), fk2);
          mv::unpack_f32x2(mv::fma_f32x2(mv::pack_u32x2(sc[j], sc[j + 1]), f01, mv::add_f32x2(mv::pack_f32x2(y.x, y.y), ev2)), p[j], p[j + 1]);
          mv::unpack_f32x2(mv::fma_f32x2(mv::pack_u32x2(sc[j + 2], sc[j + 3]), f23, mv::add_f32x2(mv::pack_f32x2(y.z, y.w), ev2)), p[j + 2], p[j + 3]);
#pragma unroll
          for (int i = 0; i < 4; ++i) p[j + i] = mv::fast_exp2(p[j + i]);
        }
        if (!plain) {
          const uint32_t mine = uint32_t(see >> col);
#pragma unroll
          for (int j = 0; j < W; ++j)
            if (!((mine >> j) & 1)) p[j] = 0.f;
        }
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < W; j += 2) most = mv::max3(most, p[j], p[j + 1]);
        top = fmaxf(top, most);
        uint32_t hi[W / 4], mid[W / 4], lo[W / 4];
#pragma unroll
        for (int k = 0; k < W / 4; ++k) split_weights(p[k * 4], p[k * 4 + 1], p[k * 4 + 2], p[k * 4 + 3], hi[k], mid[k], lo[k]);
        *reinterpret_cast<uint4*>(p_row + ((u ^ sw) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(p_row + p_plane + (((u + p_next) ^ sw) << 4)) = make_uint4(mid[0], mid[1], mid[2], mid[3]);
        *reinterpret_cast<uint4*>(p_row + 2 * p_plane + (((u + 2 * p_next) ^ sw) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        // A weight past the format's range only says that the references have to move; what it adds here is taken back then, so it must
        // not overflow (capped, it still exceeds what the move leaves of it, and the sum loses nothing but a rounding).
        if (most > CAP)
#pragma unroll
          for (int j = 0; j < W; ++j) p[j] = p[j] > CAP ? CAP : p[j];
        uint32_t l[W];
        mv::um::ld16(lanes + at.sums + col, l);
        mv::um::wait_ld();
#pragma unroll
        for (int j = 0; j < W; j += 2) {
          float x, y;
          mv::unpack_f32x2(mv::fma_f32x2(mv::pack_f32x2(p[j], p[j + 1]), vinv2, first ? 0ull : mv::pack_u32x2(l[j], l[j + 1])), x, y);
          l[j] = __float_as_uint(x);
          l[j + 1] = __float_as_uint(y);
        }
        mv::um::st16(lanes + at.sums + col, l);
      }
      return top;
    };
    // q-vectors that see their first tokens need a reference; once one has it, it moves (all of them do) only where a weight passes
    // the format's range
    const uint2 seen2 = meta->seen[tile % METAS];
    const uint64_t seen = (uint64_t(seen2.y) << 32) | seen2.x;
    uint64_t todo = seen & ~referenced;
    referenced |= seen;
    float sign = 1.f;
    bool fresh = t == 0, moving = false;
    for (;;) {
      if (todo) {
        // ---- references: the largest exponent of these q-vectors over the tile's tokens
        if (moving) (void)vote_all(true);  // the exchange area is the weight tile
        each_eight([&](int b) {
          if (((todo >> (b * 8)) & 0xff) == 0) return;
          uint32_t sc[8];
          mv::um::ld8(s_t + b * 8, sc);
          mv::um::wait_ld();
          int best = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int q = b * 8 + j;
            float y = fmaf(__uint_as_float(sc[j]), __uint_as_float(uint32_t(meta->unit[q]) << 16) * fk, evf);
            if (!((see >> q) & 1) || y != y) y = -INFINITY;
            const int k = __float_as_int(y);
            const int m = __reduce_max_sync(0xffffffffu, k < 0 ? k ^ 0x7fffffff : k);  // ordered as the floats are
            if (lane == j) best = m;
          }
          if (lane < 8) xch[quarter * MAXQV + b * 8 + lane] = __int_as_float(best < 0 ? best ^ 0x7fffffff : best);
        });
        if (!vote_all(ok)) return false;
        // what O and the sums take: 0 is a factor like any other (a reference that moves by more than 126), and where there was no
        // reference nothing has to move, they are zero (or NaN) there
        float f = 1.f;
        if (tid < s.n_qv && ((todo >> tid) & 1)) {
          const float m = fmaxf(fmaxf(xch[tid], xch[MAXQV + tid]), fmaxf(xch[2 * MAXQV + tid], xch[3 * MAXQV + tid]));
          const float now = meta->minus_ref[tid], want = HEADROOM - m;  // minus the references, old and new
          if (m > -INFINITY && want < now) {
            if (now < INFINITY) f = mv::fast_exp2(want - now);
            meta->minus_ref[tid] = want;
          }
        }
        if (tid < cols) xch[4 * MAXQV + tid] = f;
        if (vote_any(f != 1.f)) {
          ok = ok && warp_wait(c, bar(&meta->pv_done[(tile - 1) & 1]), ((tile - 1) >> 1) & 1);  // (some reference is older: t > 0)
          mv::um::fence_after();
          mv::um::wait_st();
          each_eight([&](int b) {
            const float* const f = xch + 4 * MAXQV + b * 8;
#pragma unroll 1
            for (int k = 0; k <= at.parts; ++k) {  // O and the sums, which lie side by side
              uint32_t o[8];
              mv::um::ld8(lanes + at.o + k * cols + b * 8, o);
              mv::um::wait_ld();
#pragma unroll
              for (int j = 0; j < 8; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f[j]);
              mv::um::st8(lanes + at.o + k * cols + b * 8, o);
            }
          });
          mv::um::wait_st();
          if (!vote_all(ok)) return false;  // every thread has read the exchange area
        }
      }
      const float top = ok ? pass(sign, fresh) : 0.f;
      fresh = false;
      if (moving) break;
      if (sign < 0.f) {  // the weights taken back
        sign = 1.f;
        todo = ~0ull;
        moving = true;
        continue;
      }
      mv::um::fence_before();
      if (!vote_any(top > TOP || !ok)) break;
      if (!vote_all(ok)) return false;
      todo = 0;
      sign = -1.f;
    }
    if (!plain && !__all_sync(0xffffffffu, valid)) {
      // no token here: whatever the slot holds meets a weight of zero, so it must be finite
      const int vslot = v_ring.slot();
      ok = ok && warp_wait(c, bar(&meta->full[vslot]), v_ring.parity());
      if (!valid) {
        uint4* const row = reinterpret_cast<uint4*>(c.smem + vslot * Lay<D>::PIECE + token * D);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) row[k] = make_uint4(0, 0, 0, 0);
      }
    }
    mv::fence_proxy_async();
    mv::um::fence_before();
    __syncwarp();
    if (lane == 0 && ok) mv::mbar_arrive(bar(&meta->p_full[tile & 1]));
    v_ring.advance(both_slots_of_v<D>(cols));
  }
  // ---- the segment's result: sums over the tokens, then the head vectors (thread = element; at 64 elements the upper half of the lanes holds them once more)
  ok = ok && warp_wait(c, bar(&meta->pv_done[(tile - 1) & 1]), ((tile - 1) >> 1) & 1);  // (products complete in order)
  if (!vote_all(ok)) return false;
  mv::um::fence_after();
  mv::um::wait_st();
  float* const xch = reinterpret_cast<float*>(c.smem + Lay<D>::P);
  each_eight([&](int b) {
    // eight columns over 32 lanes by halving: after three steps a lane holds one column's sum over eight lanes
    uint32_t l[8];
    mv::um::ld8(lanes + at.sums + b * 8, l);
    mv::um::wait_ld();
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = __uint_as_float(l[j]);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      const bool up = (lane & o) != 0;
#pragma unroll
      for (int j = 0; j < o; ++j) {
        const float keep = up ? y[j + o] : y[j], give = up ? y[j] : y[j + o];
        y[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    }
    y[0] += __shfl_xor_sync(0xffffffffu, y[0], 8);
    y[0] += __shfl_xor_sync(0xffffffffu, y[0], 16);
    if (lane < 8) xch[quarter * MAXQV + b * 8 + lane] = y[0];
  });
  (void)vote_all(true);
  if (tid < s.n_qv) {
    const float sum = (xch[tid] + xch[MAXQV + tid]) + (xch[2 * MAXQV + tid] + xch[3 * MAXQV + tid]);
    xch[4 * MAXQV + tid] = sum == 0.f ? 0.f : 1.f / sum;
    if (s.slot >= 0) a.part_ml[s.slot * MAXQV + tid] = make_float2(-meta->minus_ref[tid], sum);  // no token seen: reference -infinity, sum 0
  }
  (void)vote_all(true);
  each_eight([&](int b) {
    uint32_t o0[8], o1[8] = {}, o2[8] = {};
    mv::um::ld8(lanes + at.o + b * 8, o0);
    if (thirds) {
      mv::um::ld8(lanes + at.o + cols + b * 8, o1);
      mv::um::ld8(lanes + at.o + 2 * cols + b * 8, o2);
    }
    const int left = s.n_qv - b * 8;
    int h = (b * 8) % a.G;  // head of the q-vector inside the group
    bf16* out = a.out + (int64_t(s.row0 + b * 8 / a.G) * a.Hq + s.head * a.G + h) * D + token;
    float* part = a.part_o + (int64_t(s.slot) * MAXQV + b * 8) * D + token;
    const int next_row = (a.Hq - a.G) * D;
    mv::um::wait_ld();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float y = __uint_as_float(o0[j]) + (__uint_as_float(o1[j]) + __uint_as_float(o2[j]));
      if (j < left && (D == 128 || token < D)) {
        if (s.slot >= 0) part[j * D] = y;
        else *out = __float2bfloat16_rn(y * xch[4 * MAXQV + b * 8 + j]);
      }
      out += D;
      if (++h == a.G) {
        h = 0;
        out += next_row;
      }
    }
  });
  mv::um::fence_before();
  (void)vote_all(true);  // O and the exchange area have been read
  return true;
}

template <int D>
__device__ __forceinline__ void softmax_warps(const Cta& c, mv::blk::Walk& w, mv::blk::Segment& s, bool more) {
  mv::blk::CutLog cuts;
  int tile = 0;  // tiles of the share so far: score and weight buffers and their phases follow from it
  Slots v_ring{1};
  bool ok = true;
  while (more) {
    cuts.add(*c.a, s);
    stage_q<D>(c, s, columns_of(s.n_qv));
    mv::fence_proxy_async();
    (void)vote_all(true);  // references and units are there for all
    if ((threadIdx.x & 31) == 0) mv::mbar_arrive(bar(&c.meta->q_full));
    ok = run_segment<D>(c, s, tile, v_ring);
    more = ok && w.next(*c.a, s);
  }
  if (threadIdx.x == 0) cuts.store(*c.a, blockIdx.x);
}

// ---- issuer warps: the whole warp walks and waits, one elected lane issues ----------------------------------
// After a wait has run out, products may still be in flight: they must have completed before the CTA frees its tensor memory.
__device__ __forceinline__ void drain(const Cta& c, int which, bool lead) {
  if (lead) mv::um::commit(bar(&c.meta->drained[which]));
  (void)mv::mbar_wait_bounded(bar(&c.meta->drained[which]), 0, 20000000ull);
  __syncwarp();
}

// S^T = K Q^T of every tile into score buffer tile & 1: K is the 128-row operand, values of Q then remainders
template <int D>
__device__ __forceinline__ void score_issuer(const Cta& c, mv::blk::Walk& w, mv::blk::Segment& s, bool more) {
  Meta* const meta = c.meta;
  const bool lead = mv::um::elect_one();
  const uint64_t q_desc = Lay<D>::desc(c.base + Lay<D>::Q);
  int tile = 0, segment = 0;
  bool ok = true;
  for (; more; more = ok && w.next(*c.a, s)) {
    const int cols = columns_of(s.n_qv);
    const Columns at(cols);
    const uint32_t idesc = mv::um::idesc_e4m3(128, cols, 0, 0);
    ok = warp_wait(c, bar(&meta->q_full), segment & 1);
    ++segment;
#pragma unroll 1
    for (int t = 0; t < s.n_tiles && ok; ++t, ++tile) {
      // the buffer was read before the weights of the tile that last used it, two tiles ago, were handed over
      const int last = tile - 2, slot = (2 * tile) % RING;
      if (t > 0 && last >= 0) ok = warp_wait(c, bar(&meta->p_full[last & 1]), (last >> 1) & 1);
      ok = ok && warp_wait(c, bar(&meta->full[slot]), ((2 * tile) / RING) & 1);
      if (!ok) break;
      mv::um::fence_after();
      if (lead) {
        const uint64_t k_desc = Lay<D>::desc(c.base + slot * Lay<D>::PIECE);
        const uint32_t s_t = meta->tmem + ((tile & 1) ? at.s1 : 0);
        mv::um::mma8_ss<false>(s_t, k_desc, q_desc, idesc);
#pragma unroll
        for (int k = 1; k < D / 32; ++k) mv::um::mma8_ss<true>(s_t, k_desc + uint32_t((k * 32) >> 4), q_desc + uint32_t((k * 32) >> 4), idesc);
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
          mv::um::mma8_ss<true>(s_t, k_desc + uint32_t((k * 32) >> 4), q_desc + uint32_t((Lay<D>::Q_BYTES + k * 32) >> 4), idesc);
        mv::um::commit(bar(&meta->s_full[tile & 1]));
        mv::um::commit(bar(&meta->empty[slot]));
      }
      __syncwarp();
    }
  }
  if (!ok) drain(c, 0, lead);
}

// O^T += V^T P^T of every tile: V is the 128-row operand, read across its rows (32 tokens per instruction)
template <int D>
__device__ __forceinline__ void output_issuer(const Cta& c, mv::blk::Walk& w, mv::blk::Segment& s, bool more) {
  Meta* const meta = c.meta;
  const bool lead = mv::um::elect_one();
  int tile = 0;
  Slots v_ring{1};
  bool ok = true;
  for (; more; more = ok && w.next(*c.a, s)) {
    const int cols = columns_of(s.n_qv);
    const bool both = both_slots_of_v<D>(cols);
    v_ring.begin(both);
    const uint32_t o_t = meta->tmem + Columns(cols).o;
    const bool thirds = in_thirds(cols);
    const uint32_t idesc = mv::um::idesc_e4m3_e5m2(128, thirds ? 3 * cols : cols, 1, 1);
#pragma unroll 1
    for (int t = 0; t < s.n_tiles; ++t, ++tile) {
      const int vslot = v_ring.slot();
      ok = warp_wait(c, bar(&meta->full[vslot]), v_ring.parity()) && warp_wait(c, bar(&meta->p_full[tile & 1]), (tile >> 1) & 1);
      if (!ok) break;
      mv::um::fence_after();
      if (lead) {
        const uint64_t v_desc = Lay<D>::desc(c.base + vslot * Lay<D>::PIECE);
        if (thirds) {
          const uint64_t p_desc = mv::um::smem_desc(c.base + Lay<D>::P + (tile & 1) * P_NARROW, 16, 1024);
          if (t == 0) mv::um::mma8_ss<false>(o_t, v_desc, p_desc, idesc);
          else mv::um::mma8_ss<true>(o_t, v_desc, p_desc, idesc);
#pragma unroll
          for (int k = 1; k < TILE / 32; ++k) mv::um::mma8_ss<true>(o_t, v_desc + uint32_t((k * 32 * D) >> 4), p_desc + uint32_t((k * 32 * 128) >> 4), idesc);
        } else {
#pragma unroll 1
          for (int third = 0; third < 3; ++third) {
            const uint64_t p_desc = mv::um::smem_desc_64b(c.base + Lay<D>::PW + (tile & 1) * P_WIDE + third * P_THIRD, 16, 512);
            if (t == 0 && third == 0) mv::um::mma8_ss<false>(o_t, v_desc, p_desc, idesc);
            else mv::um::mma8_ss<true>(o_t, v_desc, p_desc, idesc);
#pragma unroll
            for (int k = 1; k < TILE / 32; ++k) mv::um::mma8_ss<true>(o_t, v_desc + uint32_t((k * 32 * D) >> 4), p_desc + uint32_t((k * 32 * 64) >> 4), idesc);
          }
        }
        mv::um::commit(bar(&meta->pv_done[tile & 1]));
        mv::um::commit(bar(&meta->empty[vslot]));
      }
      v_ring.advance(both);
      __syncwarp();
    }
  }
  if (!ok) drain(c, 1, lead);
}

template <int D>
__global__ void __launch_bounds__(NT, 2) decode_blk_tc_kernel(const Args a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Meta* const meta = reinterpret_cast<Meta*>(smem + Lay<D>::META);
  const int tid = threadIdx.x, warp = tid >> 5;
  const uint32_t base = mv::smem_u32(smem);
  if ((base & 1023u) != 0) {  // the swizzle pattern is anchored at 1024-byte boundaries
    mv::grid_dependency_wait();
    if (tid == 0) {
      atomicExch(a.t.counts + 4, int(MV_ERR_UNSUPPORTED));
      mv::blk::CutLog().store(a, blockIdx.x);
    }
    return;
  }
  if (tid == 0) {
    meta->abort = 0;
    for (int i = 0; i < RING; ++i) {
      mv::mbar_init(bar(&meta->full[i]), 1);   // the producer's arrive (+ the bytes TMA reports)
      mv::mbar_init(bar(&meta->empty[i]), 1);  // one tcgen05.commit after the product that read the piece
    }
    for (int i = 0; i < METAS; ++i) mv::mbar_init(bar(&meta->described[i]), 1);
    for (int i = 0; i < 2; ++i) {
      mv::mbar_init(bar(&meta->s_full[i]), 1);
      mv::mbar_init(bar(&meta->p_full[i]), SOFTMAX / 32);
      mv::mbar_init(bar(&meta->pv_done[i]), 1);
      mv::mbar_init(bar(&meta->drained[i]), 1);
    }
    mv::mbar_init(bar(&meta->q_full), SOFTMAX / 32);
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
  // every role walks the share's segments by itself; the beginning, common to all, is one piece of code that the warps fetch together
  mv::blk::Walk w;
  mv::blk::Segment s;
  w.begin(a, blockIdx.x);
  const bool more = w.next(a, s);
  if (warp < SOFTMAX / 32) softmax_warps<D>(c, w, s, more);
  else if (warp == SOFTMAX / 32) producer<D, true>(c, w, s, more, &tm_k);
  else if (warp == SOFTMAX / 32 + 1) producer<D, false>(c, w, s, more, &tm_v);
  else if (warp == SOFTMAX / 32 + 2) score_issuer<D>(c, w, s, more);
  else output_issuer<D>(c, w, s, more);
  mv::um::fence_before();
  __syncthreads();
  if (warp == 0) mv::um::tmem_dealloc(meta->tmem, 256);
}

template <int D>
mv_status launch(const Args& a, cudaStream_t st) {
  static std::atomic<uint64_t> opted{0};  // per device
  if (!mv::opt_in_smem(decode_blk_tc_kernel<D>, Lay<D>::SMEM, opted)) return MV_ERR_CUDA;
  // a pool's map: a row is a token of a KV head (no pages: no entry is accepted, nothing is read).  Made anew for every call, which does not show in its time.
  const int64_t rows = std::max<int64_t>(1, a.num_pages * a.Hkv * PS);
  CUtensorMap tm_k, tm_v;
  if (!mv::make_tmap_u8_2d(&tm_k, a.k8, uint64_t(rows), PS, D) || !mv::make_tmap_u8_2d(&tm_v, a.v8, uint64_t(rows), PS, D)) return MV_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(SHARES, 1, 1);
  cfg.blockDim = dim3(NT, 1, 1);
  cfg.dynamicSmemBytes = Lay<D>::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, decode_blk_tc_kernel<D>, a, tm_k, tm_v);
  mv::g_launches++;
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return MV_ERR_CUDA;
  }
  return MV_OK;
}

}  // namespace

namespace mv {
// Attention kernel of mv_dag_decode_attn_fp8_blk (the caller validated the arguments and launches the merge).
mv_status decode_blk_tc(const blk::Args& a, int head_dim, cudaStream_t st) { return head_dim == 128 ? launch<128>(a, st) : launch<64>(a, st); }
}  // namespace mv
