// Attention of chunks of new tokens over the block-scaled 8-bit cache, on the 5th-generation tensor cores.
// For query head h of KV head g and new token i of a node,
//   out_i = sum_j 2^(c (<q_i, K_j> - r_i)) V_j / sum_j 2^(c (<q_i, K_j> - r_i)),   c = softmax scale * log2 e,
// over the tokens j of the pages on the node's list; of its own pages, which stand last, only those up to i itself.
//
// A query tile is 2 R consecutive new tokens of a node, R = 128 / G for a group of G query heads: two operands of 128 rows, row
// token * G + head, so that any number of tokens and any group fill the tensor cores' rows and every tile of 128 keys that comes in
// serves 256 q-vectors.  The second half is left out where the tile has no more than R tokens.
//
// The cache holds bytes with four exponent and three mantissa bits at a power-of-two scale per (page, KV head).  Each is a bf16 number
// exactly (three mantissa bits of seven, exponents within range), so a warpgroup turns the bytes of a tile into bf16 operands between
// TMA and the products, and everything behind it is plain bf16 arithmetic with 32-bit accumulators: the byte's exponent
// and mantissa are moved to the low end of a bf16 pattern, which is the value times 2^-120 (the format's subnormals are bf16 subnormals
// there), and one multiplication by 2^(120 + e) brings the page's scale in.  Softmax weights are rounded to bf16 (off by at most 2^-8 of each, as
// in the other prefill kernels); their sum is of the unrounded ones, in 32 bits.
// A page whose scale is NaN: its keys become NaN, so the scores of whoever sees it; its values stay finite, so whoever does not
// see it multiplies them by zero.
//
// Warps (512 threads): 0 TMA for K and V, 1 issues the products, 2 takes and frees the tensor memory, 3 the walk over the work and TMA for
// q; 4-7 bytes to bf16; 8-11 and 12-15 softmax of the two halves, a thread per q-vector (weights written over the scores as packed bf16, O in
// tensor memory rescaled only when the row's reference moved by more than 2^8).  A tile that moves no reference has a way of its own, with the
// scores in registers.
// One CTA per SM walks its share of the work: (query tile, KV head) after (query tile, KV head) lie on a line of cost, a constant
// and then one unit per key tile, which the shares cut evenly (few query tiles are dealt out differently: deal).  What a cut leaves in two or
// more shares is joined by a second kernel.
// Every wait is bounded.
//
// Bound by the tensor cores for a long list: 2048 new tokens behind 64K, 32 query and 8 KV heads of 128, 2.2 * 10^12 operations, take
// 1.99 ms at 1965 MHz, 67 % of the rate measured of a library product in a burst; in a loop of seconds the power limit takes the clock to 1670 MHz:
// 2.31 ms, 68 % of the rate of such products under that limit (2.25 to 2.37 from one GPU to the next).  A prompt with its DAG, 17 thousand tokens,
// 64 and 8 heads: 3.04 to 3.1 ms, 62 %, and 3.4 (3.33 to 3.45), 67 %, at 1785 MHz.
// A key tile takes 3800 cycles, 2048 of them products of the two halves; the rest is the chain scores ->
// weights -> products of a half that the other half does not cover, and shared memory (320 KB to and fro a tile, 2500 cycles at 128 bytes a
// cycle).  A (tile, head) item costs 14500 cycles besides (first tile, epilogue 5000).  Small steps are bound by latency:
// 9.8 us for 40 new tokens alone (12 with a joining launch, where the tables have room for longer lists); 40 behind 960 18.4, behind 4000 25.8 (see deal).
// Built and measured slower: weights from threads in pairs, or through the 16-lane shapes of tensor memory (row maxima then cross
// threads); a part of the exponentials by a polynomial (2 % slower: the multiply-add pipe feeds the conversion of the bytes as well); eight
// warps for the bytes instead of four (registers); two issuing warps; halves kept in turns by a token.  What decided most is the size of the
// code that all roles run at once: see Cta::wait.
#include <algorithm>
#include <cmath>

#include "blk_stream.cuh"
#include "trace.h"
#include "umma.cuh"

namespace {

using bf16 = __nv_bfloat16;
constexpr int PS = 16, KEYS = 8;        // tokens of a page; pages of a key tile
constexpr int BQ = 128, BK = 128;       // q-vectors of a half; keys of a tile
constexpr int SHARES = 148;             // CTAs
// cost of a (query tile, head) besides its key tiles.  The cycles above would make it 3.8, but part of them passes beside the neighbours' key tiles:
// 1, 2, 3, 4 give 39.5, 38.5, 40.7, 43.0 us for chunks on branches (heads of 64), 89.8, 92.4, 93.9, 93.3 for 16 prompts of 500 tokens, 61.5, 58.4, 53.9, 55.5 for
// 64 times 40 tokens behind 300 (32 and 8 heads of 128); over 31 steps of both head sizes 1.006, 1, 1.002, 1.004 times as long.
constexpr int SETUP = 2;
constexpr int FEW = 32;                 // query tiles up to which a step may be dealt out in pieces (Walk::pieces)
constexpr int WHOLE = 4, MANY = 16;     // key tiles of a list that stays whole where nothing is joined; of one whose pieces have two of them at least
constexpr int FEW_OVER = 3, CUT_OVER = 1, CUT_SHORT = 6;  // key tiles: see deal
constexpr int NT = 512;
// Registers of the warpgroups: launched with 128 per thread, 56 + 72 + 2 * 192 = 4 * 128
constexpr int REGS_TMA = 56, REGS_BYTES = 72, REGS_SOFTMAX = 192;
static_assert(REGS_TMA + REGS_BYTES + 2 * REGS_SOFTMAX <= 4 * (65536 / NT), "registers of an SM");
constexpr int RAW = 4;                  // pieces of bytes in flight: half a tile of K, the other half, then of V
constexpr int RING = 4;                 // bf16 tiles (K0 V0 K1 V1 ...)
constexpr int METAS = 4;                // descriptions of key tiles: K of tile t waits for K of t - 1 converted, so for the scores of t - 3, so for the weights of t - 4
constexpr int SOFTMAX_WARPS = 4;        // of a half
constexpr int SEGS = 4;                 // segments handed over
constexpr int MAXQV = 2 * BQ;
constexpr float RESCALE_THRESHOLD = 8.f;  // log2 units: weights stay below 2^8
// A reference is kept as the raw score it was.  Weights are 2^(c s - c r) by one fused multiply-add per pair of scores, where c r is a rounded
// product: off by 2^-24 of it, the same for all of a row.  Up to FAR that is below 2^-12 of a weight; beyond, the scores are first
// brought near zero by subtracting r, which is exact for those that matter (scales of a cache go up to 2^40).
constexpr float FAR = 4096.f;
constexpr int kMaxList = 1 << 26;       // pages of a list: its slots are counted in 32 bits
constexpr int V_MIN = -80;              // a scale of zero (a block nobody has quantised) counts as 2^-80

struct alignas(16) Cut {  // the cut (tile, head)s at the ends of a share
  int begun, item, row0, rows;  // item (tile * Hkv + head, -1: none) begun in an earlier share; one that goes on in a later share, its rows
};

struct Args {
  const int4* tiles;
  const int2* entries;
  int32_t* counts;
  const float2* scale;  // [pages][Hkv]: K, V
  bf16* out;
  float* part_o;        // [2 SHARES][MAXQV][D]
  float2* part_ml;      // [2 SHARES][MAXQV]: reference (a score), sum
  Cut* cuts;            // [SHARES]
  int64_t num_pages;
  int max_rows, max_tiles, max_entries;
  int Hq, Hkv, G, R;
  int join;             // a joining launch follows
  int out_32;           // out is aligned to 32 bytes
  float scale_log2;
};

constexpr size_t part_o_bytes(int d) { return size_t(2) * SHARES * MAXQV * d * sizeof(float); }
constexpr size_t part_ml_bytes() { return size_t(2) * SHARES * MAXQV * sizeof(float2); }
constexpr size_t workspace_need(int d) { return part_o_bytes(d) + part_ml_bytes() + ((SHARES * sizeof(Cut) + 255) & ~size_t(255)); }

// A run of key tiles of one (query tile, KV head) inside a share.
struct Segment {
  int row0, rows, key0;    // tokens of the query tile; index of the first one inside its node
  int ent0, before, n_ent; // its list: first entry, entries of other nodes, entries up to its last token
  int head, item;
  int k0, k1;              // key tiles
  int slot;                // partial result, or -1: all key tiles are here
};

// Few query tiles: every share is one piece of one (tile, head).  Lists are cut into equal pieces of at most `len` key tiles, the least with
// which there are shares enough.  A list that stays whole costs nothing besides; a piece has to be written and joined, which takes as long as
// two to three key tiles, and more where the pieces are many (hence MANY).  So a list stays whole
//   where no joining launch follows (the tables have no room for longer ones): always, it has at most WHOLE key tiles;
//   else: of two key tiles, or where a cut would shorten it by no more than one.
// Left to the line of cost: lists so unlike that the longest one left whole has more than FEW_OVER key tiles above an even share, and, since
// equal pieces have no other advantage, cuts whose pieces have more than CUT_OVER above it (unless they are short: CUT_SHORT).
// mine: key tiles of tile `lane`; even: a share of the line of cost; whole: key tiles of a list that is not cut.
// Gives the share's tile (-1: none; -2: the line is better), the pieces of its list, and which one of the heads' pieces it is.  (Not inlined: it
// runs once, and what lies between the roles moves them against the lines of the instruction cache.  Inlined, long steps took 2 % longer.)
// Measured against the line (second figures), us in a graph, behind 0, 130, 300, 472, 960, 4000 tokens:
//   40 new tokens, 32 and 8 heads of 128: 9.8 11.8 14.1 17.2 18.4 25.8 / 12.1 15.0 16.4 16.5 17.8 30.6; 8 and 2 heads of 64: 8.7 10.6 12.4 15.0 15.2 19.7 /
//   11.1 13.2 13.5 14.4 14.7 22.0; 16 requests, 32 and 8 heads of 128: 13.9 15.8 18.1 22.7 29.1 82.5 / 13.9 17.6 22.5 30.9 37.7 87.5; 500 new tokens, 8 and 2
//   heads of 64: 16.0 17.1 17.2 17.4 19.1 24.2 / 15.2 16.8 16.6 16.8 19.7 23.9.  Of 260 steps (1 to 16 requests, 40 or 500 new tokens, seven kinds of
// heads of 64 and 128, behind 0 to 16000) the line takes more than 3 % longer at 131, up to 36 %, and less at 31, up to 6 % (mostly lists of 4 to 8 key tiles cut
// into single ones).
__device__ __noinline__ int3 deal(int mine, int hkv, int c, int64_t even, int whole) {
  const int lane = threadIdx.x & 31;
  const int64_t all = int64_t(__reduce_add_sync(0xffffffffu, unsigned(mine))) * hkv;
  int len = max(1, int((all + SHARES - 1) / SHARES)), n;
  for (;; len += (len + 7) / 8) {
    const int at_most = mine > MANY ? max(2, len) : len;
    n = mine <= max(whole, len + 1) ? int(mine > 0) : (mine + at_most - 1) / at_most;
    if (int64_t(__reduce_add_sync(0xffffffffu, unsigned(n))) * hkv <= SHARES) break;  // (at the latest with a piece for each)
  }
  const bool cut = __any_sync(0xffffffffu, n > 1);
  if (len > (cut ? max(int64_t(CUT_SHORT), even + CUT_OVER) : max(int64_t(WHOLE), even + FEW_OVER))) return make_int3(-2, 0, 0);
  int upto = n * hkv;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  const unsigned m = __ballot_sync(0xffffffffu, upto > c);
  if (m == 0) return make_int3(-1, 0, 0);
  const int from = __ffs(m) - 1;
  return make_int3(from, __shfl_sync(0xffffffffu, n, from), c - __shfl_sync(0xffffffffu, upto - n * hkv, from));
}

// The segments of a share, in order: one warp walks and hands them to the others through shared memory (their code and registers
// would not bear it: 660 bytes of spills a thread where every warp walked by itself).
struct Walk {
  int n_tiles, share, t, head, k, units;
  int64_t base, x_end;     // cost position of tile t; end of the share
  Segment s;

  __device__ __forceinline__ int64_t point(const Args& a, int unit0, int tile) const { return (int64_t(unit0) + int64_t(SETUP) * tile) * a.Hkv; }
  // Tile t's record.  One that is not a tile's (rows or entries outside the arrays, key tiles that do not follow) counts as
  // having no key tiles: what lies behind this check stays inside the arrays whatever the tables hold.
  __device__ __forceinline__ void take(const Args& a) { take(a, __ldcg(a.tiles + 2 * t), __ldcg(a.tiles + 2 * t + 1)); }
  __device__ __forceinline__ void take(const Args& a, const int4& p, const int4& q) {
    s.row0 = p.x;
    s.rows = p.y;
    s.ent0 = p.z;
    s.before = p.w;
    s.key0 = q.x;
    base = point(a, q.y, t);
    bool sound = p.x >= 0 && p.y >= 1 && p.y <= 2 * a.R && p.x <= a.max_rows - p.y && p.z >= 0 && p.w >= 0 && q.x >= 0 && q.x < (1 << 30) && q.y >= 0;
    const int64_t n = sound ? int64_t(p.w) + (q.x + p.y + PS - 1) / PS : 0;
    sound = sound && n <= int64_t(a.max_entries) - p.z && n <= kMaxList && (n + KEYS - 1) / KEYS == q.z;
    if (!sound && (threadIdx.x & 31) == 0) atomicExch(a.counts + 4, int(MV_ERR_INVALID_ARG));
    s.n_ent = sound ? int(n) : 0;
    units = sound ? q.z : 0;
  }
  __device__ __forceinline__ void begin(const Args& a, int c) {
    const int lane = threadIdx.x & 31;
    int units_at = 0;
    if (lane < min(FEW, a.max_tiles)) units_at = __ldcg(reinterpret_cast<const int32_t*>(a.tiles) + 8 * lane + 6);  // asked for with the counts
    share = c;
    n_tiles = max(0, min(__ldcg(a.counts + 1), a.max_tiles));
    const int total_units = max(0, __ldcg(a.counts + 3));
    const int64_t total = n_tiles > 0 ? point(a, total_units, n_tiles) : 0;
    if (n_tiles <= FEW && n_tiles * a.Hkv <= SHARES) {
      int mine = lane < n_tiles ? units_at : 0;
      if (lane < n_tiles && (mine < 1 || mine > min((a.max_entries - 1) / KEYS + 1, kMaxList / KEYS))) {  // no sound record
        atomicExch(a.counts + 4, int(MV_ERR_INVALID_ARG));
        mine = 0;
      }
      const int3 part = deal(mine, a.Hkv, c, total / SHARES, a.join ? 2 : WHOLE);
      if (part.x >= -1) {
        t = n_tiles;
        if (part.x < 0) return;
        t = part.x;
        n_tiles = t + 1;  // and no other
        take(a);
        head = part.z / part.y;
        const int i = part.z - part.y * head;
        k = int(int64_t(units) * i / part.y);
        x_end = base + int64_t(head) * (SETUP + units) + SETUP + int64_t(units) * (i + 1) / part.y;
        return;
      }
    }
    const int64_t each = total / SHARES, more = total % SHARES;
    const int64_t x = each * c + min(int64_t(c), more);
    x_end = x + each + (c < more ? 1 : 0);
    t = n_tiles;
    if (x >= x_end) return;
    // the last tile whose position is not behind x: 32 probes at a time
    int lo = 0, hi = n_tiles;  // tile lo is not behind x (or lo = 0), tile hi is
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, at = min(lo + lane * step, hi - 1);
      const bool before = lane == 0 || point(a, __ldcg(reinterpret_cast<const int32_t*>(a.tiles) + 8 * int64_t(at) + 5), at) <= x;
      const unsigned m = __ballot_sync(0xffffffffu, before);
      const int top = 31 - __clz(m);  // the highest lane whose tile is not behind x
      const int new_lo = min(lo + top * step, hi - 1);
      if (top < 31) hi = min(hi, max(new_lo + 1, min(lo + (top + 1) * step, hi)));
      lo = new_lo;
    }
    t = lo;
    take(a);
    const int64_t per = SETUP + units, at = max(int64_t(0), x - base);
    head = int(min(int64_t(a.Hkv), at / per));
    const int64_t in = at - head * per;
    k = in > SETUP ? int(min(in - SETUP, int64_t(units))) : 0;
  }
  // The next segment in s; false at the end of the share.
  __device__ __forceinline__ bool next(const Args& a) {
    while (t < n_tiles) {
      if (head >= a.Hkv || units == 0) {
        head = k = 0;
        if (++t < n_tiles) take(a);
        continue;
      }
      if (k >= units) {
        k = 0;
        ++head;
        continue;
      }
      const int64_t first = base + int64_t(head) * (SETUP + units) + SETUP;  // point of its first key tile
      const int end = int(max(int64_t(0), min(int64_t(units), x_end - first)));
      if (end <= k) return false;
      s.head = head;
      s.item = t * a.Hkv + head;
      s.k0 = k;
      s.k1 = end;
      s.slot = k == 0 && end == units ? -1 : 2 * share + (k > 0 ? 0 : 1);
      k = end;
      return true;
    }
    return false;
  }
};

// What the converters and the softmax threads need of a key tile.
struct alignas(16) Meta {
  uint32_t factor[2][KEYS];  // of a page of K, of V, as two bf16 numbers: the byte's pattern times the lower times the upper one
  uint32_t valid[BK / 32];   // keys that hold a token
  uint32_t twice;            // some upper factor is not one
};
struct Shared {
  Meta meta[METAS];
  Segment seg[SEGS];
  uint64_t seg_full[SEGS], seg_empty[SEGS], q_full, q_empty, raw_full[RAW], raw_empty[RAW], described[METAS], kv_full[RING], kv_empty[RING], s_full[2], p_full[2][2], o_done[2], drained;
  int abort;
  uint32_t tmem;
};

template <int D>
struct Lay {
  static constexpr int TILE = BK * D * 2;   // a bf16 tile: [D / 64 column blocks][128 rows][128 bytes]
  static constexpr int BLOCK = BK * 128;    // a column block
  static constexpr int BYTES = BK / 2 * D;  // half a tile of the cache
  static constexpr int Q = 0;               // both halves
  static constexpr int KV = 2 * TILE;
  static constexpr int RAWS = KV + RING * TILE;
  static constexpr int SHARED = RAWS + RAW * BYTES;
  static constexpr int SMEM = SHARED + ((int(sizeof(Shared)) + 127) & ~127);
  static_assert(SMEM <= 227 * 1024, "shared memory of an SM");
};

__device__ __forceinline__ uint32_t bar(const void* p) { return mv::smem_u32(p); }

// Bounded waits.  False once a wait of this CTA has run out (this one or an earlier one, of any role): the caller then issues
// nothing further, leaves its loops, and whoever has copies or products in flight waits for them (again bounded) before the CTA ends.
struct Cta {
  const Args* a;
  unsigned char* smem;
  uint32_t base;
  Shared* sh;
  // (Small: all roles run at once, and what they execute has to stay in the SM's instruction cache.  With the polling loops of
  // mbar_wait_bounded in each of these places the kernel took 1.6 times as long as soon as one more loop was added to it.)
  __device__ __forceinline__ bool wait(const uint64_t& b, uint32_t parity) const {
    uint64_t since = 0;
    for (uint32_t n = 1; !mv::mbar_try_wait(bar(&b), parity); ++n) {
      if (n % 256 != 0) continue;
      const uint64_t now = mv::global_timer_ns();
      if (since == 0) since = now;
      volatile int* const abort = &sh->abort;
      if (*abort == 0 && now - since <= 2000000000ull) continue;
      if (*abort == 0) atomicExch(a->counts + 4, int(MV_ERR_TIMEOUT));
      *abort = 1;
      return false;
    }
    return true;
  }
  __device__ __forceinline__ bool warp_wait(const uint64_t& b, uint32_t parity) const { return __all_sync(0xffffffffu, wait(b, parity)); }
};

// The segments as the other warps get them.  next() is null at the end of the share and after a wait has run out (then ok is false).
struct Reader {
  int n = 0;
  __device__ __forceinline__ const Segment* next(const Cta& c, bool& ok) {
    if (!ok) return nullptr;
    ok = c.warp_wait(c.sh->seg_full[n % SEGS], (n / SEGS) & 1);
    const Segment* s = &c.sh->seg[n % SEGS];
    return ok && s->item >= 0 ? s : nullptr;
  }
  __device__ __forceinline__ void done(const Cta& c) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mv::mbar_arrive(bar(&c.sh->seg_empty[n % SEGS]));
    ++n;
  }
};
constexpr int READERS = 2 + 4 + 2 * SOFTMAX_WARPS;  // warps

// ---- bytes of K and V: four boxes, a page each, make a piece; and the tiles' descriptions
__device__ __forceinline__ uint32_t bf16_power(int exponent) { return uint32_t(127 + exponent) << 7; }

template <int D>
__device__ __forceinline__ void byte_loader(const Cta& c, const CUtensorMap* map_k, const CUtensorMap* map_v) {
  const Args& a = *c.a;
  Shared* const sh = c.sh;
  const int lane = threadIdx.x & 31;
  const bool lead = mv::um::elect_one();
  int tile = 0;  // key tiles of the share so far
  int pieces = 0;
  bool ok = true;
  Reader rd;
  for (const Segment* at_seg; (at_seg = rd.next(c, ok)); rd.done(c)) {
    const int first = at_seg->k0 * KEYS, n_tiles = at_seg->k1 - at_seg->k0, last = min(at_seg->n_ent, at_seg->k1 * KEYS), head = at_seg->head;
    const int2* const list = a.entries + at_seg->ent0;
    // a window of 32 entries, one per lane
    auto entry_at = [&](int i0) {
      int2 e = make_int2(-1, 0);
      if (i0 + lane < last) {
        e = __ldcg(list + i0 + lane);
        if (e.x < 0 || e.x >= a.num_pages || e.y < 1 || e.y > PS) {
          atomicExch(a.counts + 4, int(MV_ERR_INVALID_ARG));
          e = make_int2(-1, 0);
        }
      }
      return e;
    };
    auto scale_at = [&](const int2& e) { return e.x >= 0 ? __ldcg(a.scale + int64_t(e.x) * a.Hkv + head) : make_float2(1.f, 1.f); };
    int2 e0 = entry_at(first), e1 = entry_at(first + 32);
    float2 s0 = scale_at(e0), s1 = make_float2(1.f, 1.f);
#pragma unroll 1
    for (int t = 0; t < n_tiles; ++t, ++tile) {
      const int at = (t * KEYS) & 31;
      if (at == 0 && t > 0) {
        e0 = e1;
        s0 = s1;
        e1 = entry_at(first + t * KEYS + 32);
      }
      const unsigned present = (__ballot_sync(0xffffffffu, e0.x >= 0) >> at) & 0xffu;
      const int my_row = (e0.x * a.Hkv + head) * PS;
#pragma unroll 1
      for (int p = 0; p < 4 && ok; ++p) {  // K, K, V, V
        const int half = (p & 1) * 4;
        ok = c.warp_wait(sh->raw_empty[p], (tile & 1) ^ 1);
        if (!ok) break;
        const uint32_t fb = bar(&sh->raw_full[p]), dst = c.base + Lay<D>::RAWS + p * Lay<D>::BYTES;
        if (lead) mv::mbar_arrive_expect_tx(fb, uint32_t(__popc((present >> half) & 0xfu)) * (PS * D));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int row = __shfl_sync(0xffffffffu, my_row, at + half + j);
          if (lead && ((present >> (half + j)) & 1)) mv::tma_load_2d(dst + j * (PS * D), p < 2 ? map_k : map_v, 0, row, fb);
        }
        ++pieces;
        __syncwarp();
        if (p == 0) {
          // its description: the slot's last readers were through before the wait above ended (see METAS)
          Meta& m = sh->meta[tile % METAS];
          const bool mine = lane >= at && lane < at + KEYS;
          uint32_t fk = 0x3f800000u, fv = 0x3f800000u;  // a page that is not there: zeros
          if (e0.x >= 0) {
            const int ek = mv::blk::scale_exponent(s0.x);
            int ev = mv::blk::scale_exponent(s0.y);
            if (ek == 128 || ev == 128) {
              fk |= 0x7fc0u;
              ev = 0;
            } else {
              fk = bf16_power(min(120 + max(ek, V_MIN), 127)) | bf16_power(max(ek - 7, 0)) << 16;
            }
            fv = bf16_power(min(120 + max(ev, V_MIN), 127)) | bf16_power(max(ev - 7, 0)) << 16;
          }
          // keys that hold a token: sixteen bits per page
          const uint32_t bits = e0.x >= 0 ? (1u << e0.y) - 1 : 0;
          const uint32_t pair = bits | (__shfl_down_sync(0xffffffffu, bits, 1) << 16);
          const bool twice = __any_sync(0xffffffffu, mine && ((fk >> 16) != 0x3f80u || (fv >> 16) != 0x3f80u));
          if (mine) {
            m.factor[0][lane - at] = fk;
            m.factor[1][lane - at] = fv;
            if (((lane - at) & 1) == 0) m.valid[(lane - at) / 2] = pair;
          }
          if (lane == 0) m.twice = twice ? 1 : 0;
          __syncwarp();
          if (lane == 0) mv::mbar_arrive(bar(&sh->described[tile % METAS]));
        }
      }
      if (!ok) break;
      if (at == 16) s1 = scale_at(e1);
    }
  }
  if (!ok) {
    // what is in flight must land before the CTA may leave: the last fill of every piece's slot
    if (lane == 0)
      for (int k = 1; k <= min(pieces, RAW); ++k)
        (void)mv::mbar_wait_bounded(bar(&sh->raw_full[(pieces - k) % RAW]), ((pieces - k) / RAW) & 1, 20000000ull);
    __syncwarp();
  }
}

// ---- the walk, and q: both halves of the segment's query tile
template <int D>
__device__ __forceinline__ void q_loader(const Cta& c, const CUtensorMap* map) {
  const Args& a = *c.a;
  Shared* const sh = c.sh;
  const bool lead = mv::um::elect_one();
  Walk w;
  w.begin(a, blockIdx.x);
  Cut cut{-1, -1, 0, 0};
  int n = 0, loads = 0;
  bool ok = true;
  for (bool more = true; ok && more; ++n) {
    more = w.next(a);
    ok = c.warp_wait(sh->seg_empty[n % SEGS], ((n / SEGS) & 1) ^ 1);
    if (!ok) break;
    const Segment& s = w.s;
    if (lead) {
      sh->seg[n % SEGS] = s;
      if (!more) sh->seg[n % SEGS].item = -1;
      mv::mbar_arrive(bar(&sh->seg_full[n % SEGS]));
    }
    __syncwarp();
    if (!more) break;
    if (s.slot >= 0) {
      if (s.k0 > 0) cut.begun = s.item;
      else cut = Cut{cut.begun, s.item, s.row0, s.rows};
    }
    ok = c.warp_wait(sh->q_empty, (n & 1) ^ 1);
    if (!ok) break;
    const int halves = s.rows > a.R ? 2 : 1;
    if (lead) {
      mv::mbar_arrive_expect_tx(bar(&sh->q_full), uint32_t(halves * (D / 64) * a.G * a.R * 128));
      for (int i = 0; i < halves; ++i)
        for (int b = 0; b < D / 64; ++b)
          mv::tma_load_3d(c.base + Lay<D>::Q + i * Lay<D>::TILE + b * Lay<D>::BLOCK, map, b * 64, s.head * a.G, s.row0 + i * a.R, bar(&sh->q_full));
    }
    ++loads;
    __syncwarp();
  }
  if (lead) a.cuts[blockIdx.x] = cut;  // for the merge
  if (!ok && loads > 0 && lead) (void)mv::mbar_wait_bounded(bar(&sh->q_full), (loads - 1) & 1, 20000000ull);  // in flight
  __syncwarp();
}

// ---- bytes to bf16
// Four bytes to two pairs of bf16: value * 2^-120 in each half, then the factor.
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t x, uint32_t y) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}
// Two bytes, each to the low end of a half-word (the selector), exponent and mantissa four bits up to where bf16 has them, the sign with them
// to bit 11 and from there to bit 15.  Shifts as multiplications: those have a pipe of their own and twice the rate.
__device__ __forceinline__ uint32_t widen(uint32_t w, uint32_t selector) {
  const uint32_t p = __byte_perm(w, 0, selector);
  uint32_t r;
  asm("mad.lo.u32 %0, %1, 16, 0;" : "=r"(r) : "r"(p));
  asm("mad.lo.u32 %0, %1, 240, %0;" : "+r"(r) : "r"(p & 0x00800080u));
  return r;
}
// Half a tile: 64 keys from row0 on.  A thread has two rows and D / 64 pieces of 16 bytes of each.
template <int D>
__device__ __forceinline__ void convert_half(const unsigned char* raw, unsigned char* dst, int row0, const uint32_t* factor, bool twice) {
  const int tid = threadIdx.x & 127, q8 = tid >> 3, j = tid & 7;
  // Eight threads read 16 bytes each and write 32.  The rows of a pair are chosen so that both meet all banks once: of
  // 128-byte rows, r and r xor 5 (bit 2 sets the read pieces apart, bit 0 the written ones); of 64-byte rows, r and r + 1.
  auto row_of = [&](int i) {  // inside the half
    if (D == 64) return 32 * i + q8 * 2 + (j >> 2);
    const int p = q8 & 3;
    return 32 * i + (q8 >> 2) * 8 + ((j >> 2) ? (p ^ 5) : p);
  };
  constexpr int PIECES = D / 64;
  uint4 in[2][PIECES];
  uint32_t both[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {  // all loads before the first store (the compiler cannot tell the areas apart)
    const int row = row_of(i);
    both[i] = factor[(row0 + row) >> 4];
#pragma unroll
    for (int h = 0; h < PIECES; ++h) {
      const int ch = h * 4 + (j & 3);  // 16-byte piece of the row
      in[i][h] = *reinterpret_cast<const uint4*>(raw + row * D + ((D == 128 ? ch ^ (row & 7) : ch ^ ((row >> 1) & 3)) << 4));
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = row_of(i);
    const uint32_t f = __byte_perm(both[i], 0, 0x1010);
    const int k0 = (2 * (j & 3)) ^ (row & 7), k1 = (2 * (j & 3) + 1) ^ (row & 7);
#pragma unroll
    for (int h = 0; h < PIECES; ++h) {
      const uint32_t w[4] = {in[i][h].x, in[i][h].y, in[i][h].z, in[i][h].w};
      uint32_t o[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        o[2 * k] = mul_bf16x2(widen(w[k], 0x4140), f);
        o[2 * k + 1] = mul_bf16x2(widen(w[k], 0x4342), f);
      }
      unsigned char* const at = dst + h * Lay<D>::BLOCK + (row0 + row) * 128;
      *reinterpret_cast<uint4*>(at + (k0 << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<uint4*>(at + (k1 << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
    }
  }
  if (twice) {  // (scales above 2^7) the upper factors, over what this thread has just stored
#pragma unroll 1
    for (int n = 0; n < 4 * PIECES; ++n) {
      const int i = n & 1, h = (n >> 1) & (PIECES - 1), row = row_of(i), k = (2 * (j & 3) + n / (2 * PIECES)) ^ (row & 7);
      const uint32_t g = __byte_perm(both[i], 0, 0x3232);
      uint4* const at = reinterpret_cast<uint4*>(dst + h * Lay<D>::BLOCK + (row0 + row) * 128 + (k << 4));
      const uint4 y = *at;
      *at = make_uint4(mul_bf16x2(y.x, g), mul_bf16x2(y.y, g), mul_bf16x2(y.z, g), mul_bf16x2(y.w, g));
    }
  }
}
template <int D>
__device__ __forceinline__ void converters(const Cta& c) {
  const int lane = threadIdx.x & 31;
  Shared* const sh = c.sh;
  int tile = 0;
  bool ok = true;
  Reader rd;
  for (const Segment* s; (s = rd.next(c, ok)); rd.done(c)) {
#pragma unroll 1
    for (int left = s->k1 - s->k0; left > 0 && ok; --left, ++tile) {
      const Meta& m = sh->meta[tile % METAS];
      ok = c.warp_wait(sh->described[tile % METAS], (tile / METAS) & 1);
#pragma unroll 1
      for (int p = 0; p < 4 && ok; ++p) {
        const int e = 2 * tile + (p >> 1);
        ok = ((p & 1) || c.warp_wait(sh->kv_empty[e % RING], ((e / RING) & 1) ^ 1)) && c.warp_wait(sh->raw_full[p], tile & 1);
        if (!ok) break;
        convert_half<D>(c.smem + Lay<D>::RAWS + p * Lay<D>::BYTES, c.smem + Lay<D>::KV + (e % RING) * Lay<D>::TILE, (p & 1) * 64, m.factor[p >> 1], m.twice != 0);
        if (p & 1) mv::fence_proxy_async();  // ordinary stores, read next by the tensor core
        __syncwarp();
        if (lane == 0) {
          if (p & 1) mv::mbar_arrive(bar(&sh->kv_full[e % RING]));
          mv::mbar_arrive(bar(&sh->raw_empty[p]));
        }
      }
    }
  }
}

// ---- products: the whole warp walks and waits, one elected lane issues
// S_i = Q_i K^T over the first n_cols keys (a multiple of 16): both operands K-major
template <int D>
__device__ __forceinline__ void issue_qk(uint32_t s_tmem, uint64_t q_desc, uint64_t k_desc, int n_cols) {
  const uint32_t idesc = mv::um::idesc_bf16(BQ, n_cols, 0, 0);
  mv::um::mma_ss<false>(s_tmem, q_desc, k_desc, idesc);
#pragma unroll
  for (int k = 1; k < D / 16; ++k) {
    const uint32_t off = ((k >> 2) * Lay<D>::BLOCK + (k & 3) * 32) >> 4;
    mv::um::mma_ss<true>(s_tmem, q_desc + off, k_desc + off, idesc);
  }
}
// O_i (+)= P_i V over keys 64 part .. of the first k_steps * 16: P from tensor memory (two bf16 per column), V MN-major
template <int D>
__device__ __forceinline__ void issue_pv(uint32_t o_tmem, uint32_t p_tmem, uint64_t v_desc, bool accumulate, int part, int k_steps) {
  constexpr uint32_t idesc = mv::um::idesc_bf16(BQ, D, 0, 1);
#pragma unroll
  for (int k = 0; k < BK / 32; ++k) {
    const int step = part * (BK / 32) + k;
    if (step >= k_steps) break;
    if (k > 0 || accumulate) mv::um::mma_ts<true>(o_tmem, p_tmem + step * 8, v_desc + uint32_t((step * 2048) >> 4), idesc);
    else mv::um::mma_ts<false>(o_tmem, p_tmem + step * 8, v_desc + uint32_t((step * 2048) >> 4), idesc);
  }
}

// The two halves in turn: P V of one tile and the scores of the next for the first half, then for the second.  (With a warp for each half
// their products alternate in the pipe, both are done late, and the halves fall into step: either all compute weights or all wait.)
template <int D>
__device__ __forceinline__ void issuer(const Cta& c) {
  const Args& a = *c.a;
  Shared* const sh = c.sh;
  const bool lead = mv::um::elect_one();
  const uint32_t tmem = sh->tmem;
  const uint64_t q0 = mv::um::smem_desc(c.base + Lay<D>::Q, 16, 1024);
  auto k_desc = [&](int e) { return mv::um::smem_desc(c.base + Lay<D>::KV + (e % RING) * Lay<D>::TILE, 16, 1024); };
  auto v_desc = [&](int e) { return mv::um::smem_desc(c.base + Lay<D>::KV + (e % RING) * Lay<D>::TILE, Lay<D>::BLOCK, 1024); };
  bool ok = true;
  auto full = [&](int e) { ok = ok && c.warp_wait(sh->kv_full[e % RING], (e / RING) & 1); };
  int tile = 0, n_second = 0;  // key tiles; those of the second half
  Reader rd;
  for (const Segment* s; (s = rd.next(c, ok)); rd.done(c)) {
    const int n_tiles = s->k1 - s->k0, halves = s->rows > a.R ? 2 : 1;
    int pages = s->n_ent - s->k0 * KEYS;  // left
    ok = c.warp_wait(sh->q_full, rd.n & 1);
    full(2 * tile);
    if (!ok) break;
    mv::um::fence_after();
    auto scores = [&](int i, int e, int left) {
      issue_qk<D>(tmem + 128 * i, q0 + uint32_t((i * Lay<D>::TILE) >> 4), k_desc(e), min(left, KEYS) * 16);
      mv::um::commit(bar(&sh->s_full[i]));
      mv::mbar_arrive(bar(&sh->s_full[i]));  // and hands on the tile's description, which came here through the converters' barriers
    };
    auto scores_done = [&](int e, bool last) {  // of both halves
      mv::um::commit(bar(&sh->kv_empty[e % RING]));
      if (last) mv::um::commit(bar(&sh->q_empty));
    };
    if (lead) {
      scores(0, 2 * tile, pages);
      if (halves == 2) scores(1, 2 * tile, pages);
      scores_done(2 * tile, n_tiles == 1);
    }
    __syncwarp();
#pragma unroll 1
    for (int t = 0; t < n_tiles; ++t, ++tile, pages -= KEYS) {
      const int e = 2 * tile + 1;
      const bool go_on = t + 1 < n_tiles;
      full(e);
      bool next_there = go_on && __all_sync(0xffffffffu, mv::mbar_try_wait(bar(&sh->kv_full[(e + 1) % RING]), ((e + 1) / RING) & 1));  // asked while there is time
#pragma unroll 1
      for (int i = 0; i < halves; ++i) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {  // the first 64 keys while the weights of the others are being computed
          ok = ok && c.warp_wait(sh->p_full[i][part], (i ? n_second : tile) & 1);
          if (!ok) break;
          mv::um::fence_after();
          if (lead) issue_pv<D>(tmem + 256 + 128 * i, tmem + 128 * i, v_desc(e), t > 0 || part > 0, part, min(pages, KEYS));
          __syncwarp();
        }
        n_second += i;
        if (!ok) break;
        if (go_on && !next_there) {
          full(e + 1);
          if (!ok) break;
          next_there = true;
        }
        if (go_on) mv::um::fence_after();
        if (lead) {
          if (go_on) scores(i, e + 1, pages - KEYS);
          else mv::um::commit(bar(&sh->o_done[i]));
        }
        __syncwarp();
      }
      if (!ok) break;
      if (lead) {
        mv::um::commit(bar(&sh->kv_empty[e % RING]));
        if (go_on) scores_done(e + 1, t + 2 == n_tiles);
      }
      __syncwarp();
    }
    if (!ok) break;
  }
  if (!ok) {  // products may still be in flight: they must have completed before the tensor memory is freed
    __syncwarp();
    if (lead) mv::um::commit(bar(&sh->drained));
    (void)mv::mbar_wait_bounded(bar(&sh->drained), 0, 20000000ull);
    __syncwarp();
  }
}

// ---- softmax of half i: thread = q-vector = tensor-memory lane
__device__ __forceinline__ void store_32_bytes(void* p, const uint32_t (&x)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"l"(p), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
}
template <int D>
__device__ __forceinline__ void softmax_warp(const Cta& c, int i) {
  const Args& a = *c.a;
  Shared* const sh = c.sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int v = (warp & 3) * 32 + lane;                       // q-vector of the half
  const int token = v / a.G;                                  // its token, inside the half
  const uint32_t lanes = sh->tmem + (uint32_t((warp & 3) * 32) << 16);
  const uint32_t s_t = lanes + i * 128, o_t = lanes + 256 + i * 128;
  int tile = 0, j = 0, done = 0;                              // key tiles of the share, of this half; its segments
  bool ok = true;
  Reader rd;
  for (const Segment* s; (s = rd.next(c, ok)); rd.done(c)) {
    const int first = i * a.R, rows = min(a.R, s->rows - first);  // tokens of the half
    const int k0 = s->k0, k1 = s->k1;
    if (rows <= 0) {
      tile += k1 - k0;
      continue;
    }
    const int own = s->before * PS + s->key0 + first;            // slot of the half's first token in the node's list
    // reference (a score); a row that is no token's has one that nothing passes, so that its weights are zero
    float r = token < rows ? -INFINITY : INFINITY;
    uint64_t l[2] = {0, 0};                                      // sums: two chains of even and odd columns
    bool far = false;                                            // some row's reference is beyond FAR
    const uint64_t scale2 = mv::pack_f32x2(a.scale_log2, a.scale_log2);
    auto weights = [&](int k, const uint32_t* x, uint64_t nref) {  // of 32 columns, two to a column
      uint32_t p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x0, x1;
        mv::unpack_f32x2(mv::fma_f32x2(mv::pack_u32x2(x[2 * e], x[2 * e + 1]), scale2, nref), x0, x1);
        const float p0 = mv::fast_exp2(x0), p1 = mv::fast_exp2(x1);
        l[e & 1] = mv::add_f32x2(l[e & 1], mv::pack_f32x2(p0, p1));
        p[e] = mv::pack_bf16(p0, p1);
      }
      mv::um::st16(s_t + 16 * k, p);
    };
    auto hand_over = [&](int half) {  // the weights of 64 keys (and a rescaled O) are in place
      mv::um::wait_st();
      mv::um::fence_before();
      __syncwarp();
      if (lane == 0) mv::mbar_arrive(bar(&sh->p_full[i][half]));
    };
#pragma unroll 1
    for (int t = k0; t < k1; ++t, ++tile, ++j) {
      ok = c.warp_wait(sh->s_full[i], j & 1);
      if (!ok) break;
      mv::um::fence_after();
      const uint4 held = *reinterpret_cast<const uint4*>(sh->meta[tile % METAS].valid);
      if (!far) {
        // The way of nearly all tiles: no reference moves but a row's first one, none is far.  The scores stay in registers.
        uint32_t x[4][32];
#pragma unroll
        for (int k = 0; k < 4; ++k) mv::um::ld32(s_t + 32 * k, x[k]);
        mv::um::wait_ld();
        if (own + 1 - t * BK < BK || (held.x & held.y & held.z & held.w) != ~0u) {  // some key is not seen
          const int seen = own + 1 - t * BK + token;  // slots of the tile that the row sees
          const uint32_t words[4] = {held.x, held.y, held.z, held.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int n = seen - 32 * k;
            const uint32_t see = n >= 32 ? words[k] : n <= 0 ? 0u : words[k] & ((1u << n) - 1);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!((see >> e) & 1)) x[k][e] = __float_as_uint(-INFINITY);
          }
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int e = 0; e < 32; e += 2) mx[(e >> 1) & 3] = mv::max3(mx[(e >> 1) & 3], __uint_as_float(x[k][e]), __uint_as_float(x[k][e + 1]));
        // a reference moves only when a weight would otherwise pass 2^8
        const float most = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        const float ref = r == -INFINITY ? most : r, n = ref == -INFINITY ? 0.f : -(ref * a.scale_log2);  // (-inf: nothing seen so far)
        const bool fine = ref == INFINITY ? r == INFINITY : !((most - ref) * a.scale_log2 > RESCALE_THRESHOLD) && fabsf(n) <= FAR;
        if (__all_sync(0xffffffffu, fine)) {
          r = ref;
          const uint64_t nref = mv::pack_f32x2(n, n);
          weights(0, x[0], nref);
          weights(1, x[1], nref);
          hand_over(0);
          weights(2, x[2], nref);
          weights(3, x[3], nref);
          hand_over(1);
          continue;
        }
      }
      // The other tiles: such that move a reference, and those with one that is far.  The scores are read again, 32 columns at a time.
      const uint32_t* const valid = sh->meta[tile % METAS].valid;
      const int seen = own + 1 - t * BK + token;
      auto read = [&](int k, uint32_t (&x)[32]) {
        // (on a ragged tile only the leading columns were computed, the rest holds something older and is masked)
        mv::um::ld32(s_t + 32 * k, x);
        mv::um::wait_ld();
        const int n = seen - 32 * k;
        const uint32_t held = valid[k], see = n >= 32 ? held : n <= 0 ? 0u : held & ((1u << n) - 1);
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if (!((see >> e) & 1)) x[e] = __float_as_uint(-INFINITY);
      };
      float mx = -INFINITY;
#pragma unroll 1
      for (int k = 0; k < 4; ++k) {
        uint32_t x[32];
        read(k, x);
        float m2[2] = {mx, -INFINITY};
#pragma unroll
        for (int e = 0; e < 32; e += 2) m2[(e >> 1) & 1] = mv::max3(m2[(e >> 1) & 1], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
        mx = fmaxf(m2[0], m2[1]);
      }
      const bool move = r == -INFINITY ? mx > -INFINITY : (mx - r) * a.scale_log2 > RESCALE_THRESHOLD;
      const float f = (move && r != -INFINITY) ? mv::fast_exp2((r - mx) * a.scale_log2) : 1.f;
      if (move) r = mx;
      if (t > k0 && __any_sync(0xffffffffu, f != 1.f)) {
        // (the tile's scores were issued behind the product before, so O holds the tiles before and no product is writing it)
#pragma unroll
        for (int h = 0; h < 2; ++h) l[h] = mv::mul_f32x2(l[h], mv::pack_f32x2(f, f));
#pragma unroll 1
        for (int k = 0; k < D; k += 32) {
          uint32_t o[32];
          mv::um::ld32(o_t + k, o);
          mv::um::wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
          mv::um::st32(o_t + k, o);
        }
      }
      const float ref = r == -INFINITY ? 0.f : r * a.scale_log2;
      const bool beyond = fabsf(ref) > FAR && r != INFINITY;  // (a row's own matter: its neighbours subtract zero)
      const uint64_t nref = beyond ? 0 : mv::pack_f32x2(-ref, -ref), minus = beyond ? mv::pack_f32x2(-r, -r) : 0;
      far = __any_sync(0xffffffffu, beyond);
#pragma unroll 1
      for (int k = 0; k < 4; ++k) {
        uint32_t x[32];
        read(k, x);
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          float x0, x1;
          mv::unpack_f32x2(mv::add_f32x2(mv::pack_u32x2(x[e], x[e + 1]), minus), x0, x1);
          x[e] = __float_as_uint(x0);
          x[e + 1] = __float_as_uint(x1);
        }
        weights(k, x, nref);
        if (k & 1) hand_over(k >> 1);
      }
    }
    if (!ok) break;
    // ---- the segment's result
    ok = c.warp_wait(sh->o_done[i], done & 1);
    ++done;
    if (!ok) break;
    mv::um::fence_after();
    float sum, odd;
    mv::unpack_f32x2(mv::add_f32x2(l[0], l[1]), sum, odd);
    sum += odd;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int slot = s->slot;
    const bool live = token < rows;
    bf16* pair_dst[2];  // of this thread's row and its neighbour's, the even one first
    bool pair_live[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int w = (v & ~1) + n, t = w / a.G;
      pair_dst[n] = a.out + ((int64_t(s->row0) + first + t) * a.Hq + s->head * a.G + (w - t * a.G)) * D;
      pair_live[n] = t < rows;
    }
    const int64_t at = int64_t(slot) * MAXQV + i * BQ + v;
    if (slot >= 0 && live) a.part_ml[at] = make_float2(r, sum);
#pragma unroll 1
    for (int k = 0; k < D; k += 32) {
      uint32_t o[32];
      mv::um::ld32(o_t + k, o);
      mv::um::wait_ld();
      if (slot < 0) {
        // 64 bytes of a row.  Two neighbouring rows are exchanged in halves, so that a pair of threads writes 64 bytes side by side: what
        // costs is the number of places a store goes to.
        const bool odd_row = lane & 1;
        uint32_t p[2][8];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          const uint32_t lo = mv::pack_bf16(__uint_as_float(o[2 * n]) * inv, __uint_as_float(o[2 * n + 1]) * inv);
          const uint32_t hi = mv::pack_bf16(__uint_as_float(o[2 * n + 16]) * inv, __uint_as_float(o[2 * n + 17]) * inv);
          const uint32_t got = __shfl_xor_sync(0xffffffffu, odd_row ? lo : hi, 1);
          p[0][n] = odd_row ? got : lo;  // of the even row
          p[1][n] = odd_row ? hi : got;  // of the odd one
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
          if (pair_live[n]) {
            bf16* const to = pair_dst[n] + k + (odd_row ? 16 : 0);
            if (a.out_32) {
              store_32_bytes(to, p[n]);
            } else {
              reinterpret_cast<uint4*>(to)[0] = make_uint4(p[n][0], p[n][1], p[n][2], p[n][3]);
              reinterpret_cast<uint4*>(to)[1] = make_uint4(p[n][4], p[n][5], p[n][6], p[n][7]);
            }
          }
      } else if (live) {
#pragma unroll
        for (int n = 0; n < 4; ++n) store_32_bytes(a.part_o + at * D + k + n * 8, *reinterpret_cast<uint32_t(*)[8]>(&o[8 * n]));
      }
      __syncwarp();
    }
    mv::um::fence_before();
  }
}

template <int D>
__global__ void __launch_bounds__(NT, 1) chunk_attn_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap tm_q,
                                                           const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Shared* const sh = reinterpret_cast<Shared*>(smem + Lay<D>::SHARED);
  const int tid = threadIdx.x, warp = tid >> 5;
  const uint32_t base = mv::smem_u32(smem);
  if ((base & 1023u) != 0) {  // the swizzle pattern is anchored at 1024-byte boundaries
    mv::grid_dependency_wait();
    if (tid == 0) atomicExch(a.counts + 4, int(MV_ERR_UNSUPPORTED));
    if (tid == 0) a.cuts[blockIdx.x] = Cut{-1, -1, 0, 0};
    return;
  }
  if (tid == 0) {
    sh->abort = 0;
    for (int i = 0; i < SEGS; ++i) {
      mv::mbar_init(bar(&sh->seg_full[i]), 1);
      mv::mbar_init(bar(&sh->seg_empty[i]), READERS);
    }
    mv::mbar_init(bar(&sh->q_full), 1);
    mv::mbar_init(bar(&sh->q_empty), 1);
    for (int i = 0; i < RAW; ++i) {
      mv::mbar_init(bar(&sh->raw_full[i]), 1);
      mv::mbar_init(bar(&sh->raw_empty[i]), 4);  // the converters' warps
    }
    for (int i = 0; i < METAS; ++i) mv::mbar_init(bar(&sh->described[i]), 1);
    for (int i = 0; i < RING; ++i) {
      mv::mbar_init(bar(&sh->kv_full[i]), 4);
      mv::mbar_init(bar(&sh->kv_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mv::mbar_init(bar(&sh->s_full[i]), 2);  // the products, and the issuer's word
      for (int k = 0; k < 2; ++k) mv::mbar_init(bar(&sh->p_full[i][k]), SOFTMAX_WARPS);
      mv::mbar_init(bar(&sh->o_done[i]), 1);
    }
    mv::mbar_init(bar(&sh->drained), 1);
    mv::mbar_fence_init();
    mv::fence_proxy_async();
  }
  if (warp == 2) {  // the whole tensor memory of the SM: S0 S1 O0 O1, 128 columns each
    mv::um::tmem_alloc(mv::smem_u32(&sh->tmem), 512);
    mv::um::tmem_relinquish();
  }
  mv::um::fence_before();
  __syncthreads();
  mv::um::fence_after();
  // launched with programmatic stream serialisation: what is above may overlap the end of the kernel before
  mv::grid_dependency_wait();
  mv::grid_dependency_launch_dependents();
  const Cta c{&a, smem, base, sh};
  if (warp < 4) {
    mv::um::reg_dec<REGS_TMA>();
    if (warp == 0) byte_loader<D>(c, &tm_k, &tm_v);
    else if (warp == 1) issuer<D>(c);
    else if (warp == 3) q_loader<D>(c, &tm_q);
  } else if (warp < 8) {
    mv::um::reg_dec<REGS_BYTES>();
    converters<D>(c);
  } else {
    mv::um::reg_inc<REGS_SOFTMAX>();
    softmax_warp<D>(c, (warp - 8) >> 2);
  }
  mv::um::fence_before();
  __syncthreads();
  if (warp == 2) mv::um::tmem_dealloc(sh->tmem, 512);
}

// Joins the cut items: out = sum_i w_i O_i / sum_i w_i l_i, w_i = 2^(c (r_i - max r)) over the item's parts i.  The items that start in a
// share and end in a later one are listed; their q-vectors are dealt to the warps of all CTAs, FLY parts of each in flight.
constexpr int MERGE_WARPS = 16, MERGE_CTAS = 4 * SHARES;
template <int D>
__global__ void __launch_bounds__(MERGE_WARPS * 32, 3) chunk_merge_kernel(const Args a) {
  constexpr int VEC = D / 32, FLY = 8 / VEC;
  __shared__ int s_own[SHARES], s_more[SHARES + 1], s_row0[SHARES], s_rows[SHARES], s_list[SHARES], s_n[MERGE_WARPS];
  // item that goes on behind a share; begun before it; the former's rows; shares that have one
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mv::grid_dependency_wait();
  static_assert(SHARES <= MERGE_WARPS * 32, "a thread per share");
  if (threadIdx.x < SHARES) {
    const int4 cut = __ldcg(reinterpret_cast<const int4*>(a.cuts) + threadIdx.x);
    s_more[threadIdx.x] = cut.x;
    s_own[threadIdx.x] = cut.y;
    s_row0[threadIdx.x] = cut.z;
    s_rows[threadIdx.x] = cut.w;
  }
  if (threadIdx.x == 0) s_more[SHARES] = -1;
  const bool here = threadIdx.x < SHARES && s_own[threadIdx.x] >= 0;  // (its own word)
  const unsigned m = __ballot_sync(0xffffffffu, here);
  if (lane == 0) s_n[warp] = __popc(m);
  __syncthreads();
  int n_items = 0, at = __popc(m & ((1u << lane) - 1));
#pragma unroll
  for (int w = 0; w < MERGE_WARPS; ++w) {
    if (w < warp) at += s_n[w];
    n_items += s_n[w];
  }
  if (n_items == 0) return;  // (all of the CTA)
  if (here) s_list[at] = threadIdx.x;
  __syncthreads();
  for (int x = blockIdx.x * MERGE_WARPS + warp; x < n_items * MAXQV; x += MERGE_CTAS * MERGE_WARPS) {
    const int c = s_list[x / MAXQV], q = x % MAXQV, item = s_own[c], head = item % a.Hkv;
    const int2 rows = make_int2(s_row0[c], s_rows[c]);
    const int half = q / BQ, v = q % BQ, token = v / a.G;
    if (token >= min(a.R, rows.y - half * a.R)) continue;
    // the parts: slot 2 c + 1, then slots 2 i of the shares behind, without gaps
    int parts = 1;
    while (s_more[c + parts] == item) ++parts;
    float top = -INFINITY, sum = 0.f, acc[VEC] = {};
    for (int p0 = 0; p0 < parts; p0 += FLY) {
      float2 ml[FLY];
      float y[FLY][VEC];
#pragma unroll
      for (int k = 0; k < FLY; ++k) {
        const int p = p0 + k;
        ml[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) y[k][e] = 0.f;
        if (p < parts) {
          const int64_t at = int64_t(p == 0 ? 2 * c + 1 : 2 * (c + p)) * MAXQV + q;
          ml[k] = __ldcg(a.part_ml + at);
          const float* src = a.part_o + at * D + lane * VEC;
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
      for (int k = 0; k < FLY; ++k) now = fmaxf(now, ml[k].x);
      const float f = top == -INFINITY ? 1.f : mv::fast_exp2((top - now) * a.scale_log2);  // nothing seen so far: zeros (or NaN)
      sum *= f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] *= f;
#pragma unroll
      for (int k = 0; k < FLY; ++k) {
        const float wt = ml[k].x == -INFINITY ? 1.f : mv::fast_exp2((ml[k].x - now) * a.scale_log2);
        sum = fmaf(wt, ml[k].y, sum);
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = fmaf(wt, y[k][e], acc[e]);
      }
      top = now;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int64_t row = int64_t(rows.x) + half * a.R + token;
    uint32_t* const out = reinterpret_cast<uint32_t*>(a.out + (row * a.Hq + head * a.G + (v - token * a.G)) * D + lane * VEC);
    if (VEC == 4) *reinterpret_cast<uint2*>(out) = make_uint2(mv::pack_bf16(acc[0] * inv, acc[1] * inv), mv::pack_bf16(acc[VEC - 2] * inv, acc[VEC - 1] * inv));
    else *out = mv::pack_bf16(acc[0] * inv, acc[1] * inv);
  }
}

template <typename K, typename... T>
mv_status launch_after(K kernel, dim3 grid, int threads, int smem, cudaStream_t st, const T&... args) {
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  mv::g_launches++;
  if (e != cudaSuccess) (void)cudaGetLastError();
  return e == cudaSuccess ? MV_OK : MV_ERR_CUDA;
}

// The warpgroups' shares of the registers are taken from what the block is launched with: with fewer than the shares add up to, the
// request for more would never be met.
template <typename K>
mv_status registers_suffice(K kernel, std::atomic<int>& regs) {
  if (regs == 0) {  // (a property of the build, asked for once)
    cudaFuncAttributes f{};
    if (cudaFuncGetAttributes(&f, kernel) != cudaSuccess) {
      (void)cudaGetLastError();
      return MV_ERR_CUDA;
    }
    regs = f.numRegs;
  }
  return regs >= (REGS_TMA + REGS_BYTES + 2 * REGS_SOFTMAX) / 4 ? MV_OK : MV_ERR_UNSUPPORTED;
}

template <int D>
mv_status launch(const Args& a, const void* q, const void* k8, const void* v8, cudaStream_t st) {
  static std::atomic<uint64_t> opted{0};  // per device
  if (!mv::opt_in_smem(chunk_attn_kernel<D>, Lay<D>::SMEM, opted)) return MV_ERR_CUDA;
  static std::atomic<int> regs{0};
  const mv_status fits = registers_suffice(chunk_attn_kernel<D>, regs);
  if (fits != MV_OK) return fits;
  // a pool's row is a token of a KV head (no pages: no entry is accepted, nothing is read)
  const int64_t rows = std::max<int64_t>(1, a.num_pages * a.Hkv * PS);
  CUtensorMap tm_q, tm_k, tm_v;
  if (!mv::make_tmap_bf16_heads(&tm_q, q, uint64_t(a.max_rows), uint64_t(a.Hq), D, uint32_t(a.G), uint32_t(a.R)) ||
      !mv::make_tmap_u8_2d(&tm_k, k8, uint64_t(rows), PS, D) || !mv::make_tmap_u8_2d(&tm_v, v8, uint64_t(rows), PS, D))
    return MV_ERR_CUDA;
  const mv_status e = launch_after(chunk_attn_kernel<D>, dim3(SHARES), NT, Lay<D>::SMEM, st, a, tm_q, tm_k, tm_v);
  if (e != MV_OK) return e;
  if (!a.join) return MV_OK;
  return launch_after(chunk_merge_kernel<D>, dim3(MERGE_CTAS), MERGE_WARPS * 32, 0, st, a);
}

}  // namespace

extern "C" size_t mv_chunk_attn_workspace_bytes(const mv_attn_geom* g) {
  if (mv::check_geom(g) != MV_OK) return 0;
  return workspace_need(g->head_dim);
}

extern "C" mv_status mv_dag_chunk_attn_fp8_blk(const mv_chunk_tables* t, const mv_attn_geom* g, const void* q_rot, const void* k_pages8,
                                               const void* v_pages8, const float* kv_scale, void* out, void* workspace,
                                               size_t workspace_bytes, void* cuda_stream) {
  mv::NvtxRange nvtx_range("mv_dag_chunk_attn_fp8_blk");
  if (!t || t->max_rows < 0 || t->max_tiles < 0 || t->max_entries < 0 || !t->counts) return MV_ERR_INVALID_ARG;
  const mv_status st = mv::check_geom(g);
  if (st != MV_OK) return st;
  if (g->dtype != MV_BF16) return MV_ERR_UNSUPPORTED;
  if (!(g->sm_scale >= 0.f) || !std::isfinite(g->sm_scale)) return MV_ERR_INVALID_ARG;  // (the largest score is found before it is scaled)
  const int G = g->n_q_heads / g->n_kv_heads;
  if (G > BQ || t->rows_per_tile < 1 || t->rows_per_tile > 2 * (BQ / G)) return MV_ERR_UNSUPPORTED;
  if (g->num_pages > INT32_MAX / PS / g->n_kv_heads) return MV_ERR_UNSUPPORTED;  // the rows of a pool are TMA coordinates
  if (t->max_tiles > INT32_MAX / g->n_kv_heads) return MV_ERR_UNSUPPORTED;       // (tile, head) is counted in an int
  if (t->max_rows == 0 || t->max_tiles == 0) return t->max_rows > 0 && (q_rot || out) ? MV_ERR_INVALID_ARG : MV_OK;
  if (!t->tiles || (t->max_entries > 0 && !t->entries)) return MV_ERR_INVALID_ARG;
  if (!q_rot || !k_pages8 || !v_pages8 || !kv_scale || !out || q_rot == out) return MV_ERR_INVALID_ARG;
  for (const void* p : {q_rot, k_pages8, v_pages8, static_cast<const void*>(kv_scale), static_cast<const void*>(out),
                        static_cast<const void*>(t->tiles), static_cast<const void*>(t->entries)})
    if ((reinterpret_cast<uintptr_t>(p) & 15) != 0) return MV_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(t->counts) & 3) return MV_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < workspace_need(g->head_dim) || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MV_ERR_WORKSPACE;
  const uintptr_t at_q = reinterpret_cast<uintptr_t>(q_rot), at_out = reinterpret_cast<uintptr_t>(out);
  const uintptr_t bytes = uintptr_t(t->max_rows) * uintptr_t(g->n_q_heads) * uintptr_t(g->head_dim) * sizeof(bf16);
  if (at_q < at_out + bytes && at_out < at_q + bytes) return MV_ERR_INVALID_ARG;  // rows are read after others have been written
  Args a;
  a.tiles = reinterpret_cast<const int4*>(t->tiles);
  a.entries = reinterpret_cast<const int2*>(t->entries);
  a.counts = t->counts;
  a.scale = reinterpret_cast<const float2*>(kv_scale);
  a.out = static_cast<bf16*>(out);
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + part_o_bytes(g->head_dim));
  a.cuts = reinterpret_cast<Cut*>(static_cast<char*>(workspace) + part_o_bytes(g->head_dim) + part_ml_bytes());
  a.num_pages = g->num_pages;
  a.max_rows = t->max_rows;
  a.max_tiles = t->max_tiles;
  a.max_entries = t->max_entries;
  a.Hq = g->n_q_heads;
  a.Hkv = g->n_kv_heads;
  a.G = G;
  a.R = BQ / G;
  // where no list can be long enough to be cut there is nothing to join.  (The host knows the tables' capacities, not the step: tables made for
  // steps that grow have the second launch, 2 us, in the short ones too.)
  a.join = !(t->max_tiles <= FEW && t->max_tiles * g->n_kv_heads <= SHARES && t->max_entries <= WHOLE * KEYS);
  a.out_32 = (reinterpret_cast<uintptr_t>(out) & 31) == 0;
  a.scale_log2 = mv::softmax_scale(g) * 1.4426950408889634f;
  if (!std::isfinite(a.scale_log2)) return MV_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return g->head_dim == 128 ? launch<128>(a, q_rot, k_pages8, v_pages8, s) : launch<64>(a, q_rot, k_pages8, v_pages8, s);
}
