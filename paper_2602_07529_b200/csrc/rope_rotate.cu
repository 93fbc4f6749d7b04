// Rotary embedding by itself, in the forms of mv_rope_form, forward and backward, and the making of a form.
//
//   a' = A (a cos x - b sin x),  b' = A (b cos x + a sin x),  x = pos * theta_i
// over the pairs (a, b) of q's and k's heads; the backward pass is the transposed map: the same with -sin.  Elements outside the
// rotated part are copied (left alone where the call works in place).
//
// Bound by memory: every element is read and written once.  A CTA takes TPC tokens: their cosines and sines once into shared
// memory (double-precision angles, rope.cuh), then all heads of q and k in 16-byte vectors, UNITS pieces in flight per thread.  As halves
// a piece is two vectors, half the rotated part apart; as pairs it is one vector, which holds whole pairs, so neighbouring threads read neighbouring bytes.
// Measured: 17K tokens, 32 query and 8 KV heads of 128, 349 MB, 60.5 to 64 us from one GPU to the next (83 to 88 % of the measured
// copy rate); on one GPU 4, 8, 16 tokens per CTA
// 65.0, 61.0, 66.6 us, four pieces in flight instead of two 62.5, vectors that do not pass L2 by 63.5.  64 tokens: 3.1 us in a graph, the rest
// of a call is the host's.
#include <algorithm>
#include <cmath>
#include <limits>

#include "common.cuh"
#include "rope.cuh"
#include "trace.h"

namespace {

constexpr int NT = 256;

struct Args {
  const void *q, *k;
  void *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;  // elements between tokens
  const int32_t* pos_id;
  int64_t n;
  int Hq, Hkv;       // zero where the tensor is absent
  float sign;        // -1: backward
  int q_in_place, k_in_place;
};

template <typename T>
struct Vec;  // 16 bytes
template <>
struct Vec<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  __device__ static __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ static __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(mv::pack_bf16(x[0], x[1]), mv::pack_bf16(x[2], x[3]), mv::pack_bf16(x[4], x[5]), mv::pack_bf16(x[6], x[7]));
  }
};

template <bool STREAMS>
__device__ __forceinline__ uint4 load(const void* p) { return STREAMS ? __ldcs(static_cast<const uint4*>(p)) : *static_cast<const uint4*>(p); }
template <bool STREAMS>
__device__ __forceinline__ void store(void* p, const uint4& v) {
  if (STREAMS) __stcs(static_cast<uint4*>(p), v);
  else *static_cast<uint4*>(p) = v;
}

template <typename T, int D, int TPC, bool PAIRS>
__global__ void __launch_bounds__(NT) rope_rotate_kernel(const Args a, const __grid_constant__ mv::FormTable f) {
  constexpr int N = Vec<T>::N, HALF = D / 2;
  constexpr int PER_HEAD = PAIRS ? D / N : HALF / N;  // pieces
  constexpr int VECS = PAIRS ? 1 : 2;                 // vectors of a piece
  constexpr int UNITS = TPC == 1 ? 1 : PAIRS ? 4 : 2;
  constexpr bool STREAMS = TPC > 1;                   // what a prompt reads and writes here does not stay in L2
  __shared__ __align__(16) float cs[TPC][HALF], sn[TPC][HALF];
  const int64_t t0 = int64_t(blockIdx.x) * TPC;
  const int tid = threadIdx.x, here = int(min(int64_t(TPC), a.n - t0));
  mv::grid_dependency_launch_dependents();
  for (int x = tid; x < here * HALF; x += NT) {
    const int tl = x / HALF, i = x % HALF;
    if (i >= f.half) continue;
    float c, s;
    mv::rope_cos_sin(__ldg(a.pos_id + t0 + tl), f.t.theta[i], c, s);
    cs[tl][i] = c * f.amplitude;
    sn[tl][i] = s * f.amplitude * a.sign;
  }
  __syncthreads();
  const int heads = a.Hq + a.Hkv, units = here * heads * PER_HEAD;
  struct At {
    int tl, lo, hi, c;   // token, elements of the vectors inside the head, first pair (-1: not turned)
    const T* src;
    T* dst;
    bool skip;
  };
  auto place = [&](int x) {
    At p;
    const int y = x / PER_HEAD, u = x % PER_HEAD;
    p.tl = y / heads;
    const int h = y - p.tl * heads;
    const int64_t t = t0 + p.tl;
    bool in_place;
    if (h < a.Hq) {
      p.src = static_cast<const T*>(a.q) + t * a.q_stride + int64_t(h) * D;
      p.dst = static_cast<T*>(a.q_out) + t * a.q_out_stride + int64_t(h) * D;
      in_place = a.q_in_place;
    } else {
      p.src = static_cast<const T*>(a.k) + t * a.k_stride + int64_t(h - a.Hq) * D;
      p.dst = static_cast<T*>(a.k_out) + t * a.k_out_stride + int64_t(h - a.Hq) * D;
      in_place = a.k_in_place;
    }
    if (PAIRS) {
      p.lo = u * N;
      p.hi = 0;
      p.c = p.lo >= f.first && p.lo < f.first + 2 * f.half ? (p.lo - f.first) / 2 : -1;
    } else {
      const mv::Piece q = mv::piece_at<N>(f, u * N);
      p.lo = q.lo;
      p.hi = q.hi;
      p.c = q.turns ? u * N : -1;
    }
    p.skip = in_place && p.c < 0;
    return p;
  };
#pragma unroll 1
  for (int x0 = tid; x0 < units; x0 += NT * UNITS) {
    uint4 in[UNITS][VECS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int x = x0 + i * NT;
      if (x < units) {
        const At p = place(x);
        if (p.skip) continue;
        in[i][0] = load<STREAMS>(p.src + p.lo);
        if (!PAIRS) in[i][VECS - 1] = load<STREAMS>(p.src + p.hi);
      }
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int x = x0 + i * NT;
      if (x >= units) break;
      const At p = place(x);
      if (p.skip) continue;
      uint4 lo = in[i][0], hi = in[i][VECS - 1];
      if (p.c >= 0) {
        const float *c = &cs[p.tl][p.c], *s = &sn[p.tl][p.c];
        float l[N], r[N];
        Vec<T>::unpack(lo, l);
        if (PAIRS) {
#pragma unroll
          for (int n = 0; n < N; n += 2) mv::turn_pair(l[n], l[n + 1], c[n / 2], s[n / 2]);
        } else {
          Vec<T>::unpack(hi, r);
          mv::turn_piece<N>(false, l, r, c, s);
          hi = Vec<T>::pack(r);
        }
        lo = Vec<T>::pack(l);
      }
      store<STREAMS>(p.dst + p.lo, lo);
      if (!PAIRS) store<STREAMS>(p.dst + p.hi, hi);
    }
  }
}

template <typename T, int D, bool PAIRS>
void launch(const Args& a, const mv::FormTable& f, cudaStream_t st) {
  // few tokens: one per CTA spreads them over the SMs; many: eight share the staging of the angles
  constexpr int MANY = 8;
  if (a.n < 2048) rope_rotate_kernel<T, D, 1, PAIRS><<<unsigned(a.n), NT, 0, st>>>(a, f);
  else rope_rotate_kernel<T, D, MANY, PAIRS><<<unsigned((a.n + MANY - 1) / MANY), NT, 0, st>>>(a, f);
}
template <typename T>
void launch_d(const Args& a, const mv::FormTable& f, int d, cudaStream_t st) {
  if (d == 128) f.pairs ? launch<T, 128, true>(a, f, st) : launch<T, 128, false>(a, f, st);
  else f.pairs ? launch<T, 64, true>(a, f, st) : launch<T, 64, false>(a, f, st);
}

// a tensor's pointers and strides; `size`: bytes of an element
bool sound(const void* in, int64_t in_stride, const void* out, int64_t out_stride, int64_t least, int64_t size, int64_t n) {
  if ((reinterpret_cast<uintptr_t>(in) | reinterpret_cast<uintptr_t>(out)) & 15) return false;
  if (in_stride < least || out_stride < least || (in_stride * size) % 16 || (out_stride * size) % 16) return false;
  const int64_t most = std::numeric_limits<int64_t>::max() / size / (n > 0 ? n : 1);  // no offset overflows
  return in_stride <= most && out_stride <= most && (in != out || in_stride == out_stride);
}

// n rows of `length` bytes, `stride` apart (a sound tensor's: n * stride fits an int64_t, length is at most stride)
struct Rows {
  const void* base;
  int64_t stride, length;
};
// floor(a / b), b > 0
int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0 ? 1 : 0); }
// Do some row of a and some row of b share a byte?  Rows of one stride (tensors side by side in the rows of one projection) by arithmetic;
// others, where the areas meet at all, row after row.
bool overlap(const Rows& a, const Rows& b, int64_t n) {
  if (!a.base || !b.base) return false;
  const int64_t d = int64_t(reinterpret_cast<uintptr_t>(b.base) - reinterpret_cast<uintptr_t>(a.base));
  const int64_t end_a = (n - 1) * a.stride + a.length, end_b = (n - 1) * b.stride + b.length;
  if (d >= end_a || -d >= end_b) return false;
  // rows i of a and j of b meet where -b.length < d + j * b.stride - i * a.stride < a.length
  if (a.stride == b.stride) {  // so where j - i is in lo .. hi
    const int64_t lo = floor_div(-b.length - d, a.stride) + 1, hi = -floor_div(d - a.length, a.stride) - 1;
    return std::max(lo, 1 - n) <= std::min(hi, n - 1);
  }
  for (int64_t i = 0; i < n; ++i) {
    const int64_t at = i * a.stride - d;  // row i, as b counts
    const int64_t lo = floor_div(at - b.length, b.stride) + 1, hi = -floor_div(-at - a.length, b.stride) - 1;
    if (std::max<int64_t>(lo, 0) <= std::min(hi, n - 1)) return true;
  }
  return false;
}

}  // namespace

extern "C" mv_status mv_rope_form_init(mv_rope_form* form, int32_t layout, int32_t first, int32_t rotary_dim, double base, int32_t scaling,
                                       double factor, double length, double slow, double fast, float amplitude) {
  if (!form || (layout != MV_ROPE_HALVES && layout != MV_ROPE_PAIRS)) return MV_ERR_INVALID_ARG;
  if (scaling < MV_ROPE_PLAIN || scaling > MV_ROPE_RAMP) return MV_ERR_INVALID_ARG;
  if (!(base >= 1.0) || !std::isfinite(base) || !(amplitude > 0.f) || !(amplitude <= 1024.f)) return MV_ERR_INVALID_ARG;
  if (scaling != MV_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return MV_ERR_INVALID_ARG;
  if (scaling == MV_ROPE_RAMP && (!(length > 0.0) || !std::isfinite(length) || !(slow >= 0.0) || !(fast > slow) || !std::isfinite(fast))) return MV_ERR_INVALID_ARG;
  if (first < 0 || first > 112 || (first & 15) || rotary_dim < 16 || rotary_dim > 128 || (rotary_dim & 15)) return MV_ERR_UNSUPPORTED;
  if (scaling == MV_ROPE_BASE) {
    const double r = double(rotary_dim);
    base *= std::pow(factor, r / (r - 2.0));
    if (!std::isfinite(base)) return MV_ERR_INVALID_ARG;
  }
  *form = mv_rope_form{};
  form->layout = layout;
  form->first = first;
  form->rotary_dim = rotary_dim;
  form->amplitude = amplitude;
  const mv::ThetaTable plain = mv::theta_table(base, rotary_dim);  // the very angles of the calls without a form
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double t = plain.theta[i];
    if (scaling == MV_ROPE_LINEAR) t /= factor;
    if (scaling == MV_ROPE_RAMP) {
      const double turns = length * t / 6.283185307179586476925;
      const double w = std::fmin(1.0, std::fmax(0.0, (turns - slow) / (fast - slow)));
      t = w * t + (1.0 - w) * t / factor;
    }
    form->theta[i] = t;
  }
  return MV_OK;
}

extern "C" mv_status mv_rope_rotate(const mv_rope_form* form, const mv_attn_geom* g, const int32_t* pos_id, int64_t n_tokens, int32_t backward,
                                    const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out, int64_t q_out_stride,
                                    void* k_out, int64_t k_out_stride, void* cuda_stream) {
  mv::NvtxRange nvtx_range("mv_rope_rotate");
  const mv_status st = mv::check_geom(g);
  if (st != MV_OK) return st;
  if (!mv::form_ok(form, g->head_dim) || n_tokens < 0 || (backward != 0 && backward != 1)) return MV_ERR_INVALID_ARG;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr)) return MV_ERR_INVALID_ARG;
  const int64_t size = g->dtype == MV_BF16 ? 2 : 4;
  if (q && !sound(q, q_stride, q_out, q_out_stride, int64_t(g->n_q_heads) * g->head_dim, size, n_tokens)) return MV_ERR_INVALID_ARG;
  if (k && !sound(k, k_stride, k_out, k_out_stride, int64_t(g->n_kv_heads) * g->head_dim, size, n_tokens)) return MV_ERR_INVALID_ARG;
  if (n_tokens == 0 || (!q && !k)) return MV_OK;
  if (!pos_id || (reinterpret_cast<uintptr_t>(pos_id) & 3)) return MV_ERR_INVALID_ARG;
  if (n_tokens > int64_t(INT32_MAX)) return MV_ERR_UNSUPPORTED;
  const int64_t token_q = int64_t(g->n_q_heads) * g->head_dim * size, token_k = int64_t(g->n_kv_heads) * g->head_dim * size;
  const Rows in_q{q, q_stride * size, token_q}, in_k{k, k_stride * size, token_k}, in_pos{pos_id, 4, 4};
  const Rows to_q{q_out, q_out_stride * size, token_q}, to_k{k_out, k_out_stride * size, token_k};
  if ((q != q_out && overlap(to_q, in_q, n_tokens)) || (k != k_out && overlap(to_k, in_k, n_tokens)) || overlap(to_q, in_k, n_tokens) ||
      overlap(to_k, in_q, n_tokens) || overlap(to_q, to_k, n_tokens) || overlap(to_q, in_pos, n_tokens) || overlap(to_k, in_pos, n_tokens))
    return MV_ERR_INVALID_ARG;
  if (g->n_q_heads > 4096) return MV_ERR_UNSUPPORTED;
  Args a;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.pos_id = pos_id;
  a.n = n_tokens;
  a.Hq = q ? g->n_q_heads : 0;
  a.Hkv = k ? g->n_kv_heads : 0;
  a.sign = backward ? -1.f : 1.f;
  a.q_in_place = q == q_out;
  a.k_in_place = k == k_out;
  const mv::FormTable f = mv::form_table(*form);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (g->dtype == MV_BF16) launch_d<__nv_bfloat16>(a, f, g->head_dim, s);
  else launch_d<float>(a, f, g->head_dim, s);
  mv::g_launches++;
  if (cudaGetLastError() != cudaSuccess) return MV_ERR_CUDA;
  return MV_OK;
}
