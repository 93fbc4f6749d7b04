// Pages of any number of pools copied in one launch: page dst[i] of every pool becomes page src[i] (forks, compaction).
//
// Bound by memory: every page is read and written once.  A pool's share of the work is the line of its n * V vectors (V vectors
// to a page), cut into blocks of BLOCK; a CTA takes one block of one pool, four vectors in flight per thread, so small pages (the
// scales of a block-scaled cache) lie many to a CTA and large ones over several.  With a count on the device the grid covers
// the most pairs there may be, and CTAs behind the count leave at once.
#include "common.cuh"
#include "trace.h"

namespace {

constexpr int NT = 256, ILP = 4, BLOCK = NT * ILP;
constexpr int MAX_POOLS = MV_PAGES_MAX_POOLS;

struct Pool {
  char* base;
  int64_t page_bytes;
};
struct Args {
  const int32_t *src, *dst, *count;
  int32_t* status;
  int64_t num_pages;
  int n, n_pools;
  Pool pool[MAX_POOLS];
  uint32_t first[MAX_POOLS + 1];  // CTAs of the pools before
};

template <typename V>
__device__ __forceinline__ void copy_block(const Args& a, const Pool& p, int64_t block, int n) {
  const int64_t per = p.page_bytes / int64_t(sizeof(V));  // vectors of a page
  const int64_t at = block * BLOCK;
  const int64_t pair0 = at / per, off0 = at - pair0 * per;
  V x[ILP];
  V* to[ILP];
#pragma unroll
  for (int i = 0; i < ILP; ++i) {
    int64_t off = off0 + i * NT + int(threadIdx.x), pair = pair0;
    if (off >= per) {  // (pages larger than a block: at most one further)
      if (per >= BLOCK) {
        off -= per;
        ++pair;
      } else {
        const uint32_t more = uint32_t(off) / uint32_t(per);
        off -= int64_t(more) * per;
        pair += more;
      }
    }
    to[i] = nullptr;
    if (pair >= n) continue;
    const int32_t from = __ldg(a.src + pair), into = __ldg(a.dst + pair);
    if (from < 0 || into < 0 || from >= a.num_pages || into >= a.num_pages) {
      if (a.status && off == 0) atomicExch(a.status, int(MV_ERR_INVALID_ARG));
      continue;
    }
    if (from == into) continue;
    to[i] = reinterpret_cast<V*>(p.base + into * p.page_bytes) + off;
    x[i] = __ldcs(reinterpret_cast<const V*>(p.base + from * p.page_bytes) + off);
  }
#pragma unroll
  for (int i = 0; i < ILP; ++i)
    if (to[i]) __stcs(to[i], x[i]);
}

__global__ void __launch_bounds__(NT) pages_copy_kernel(const __grid_constant__ Args a) {
  mv::grid_dependency_launch_dependents();
  int lo = 0, hi = a.n_pools;  // the pool of this CTA: the last one whose first CTA is not behind it
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.first[mid] <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const int n = a.count ? max(0, min(a.n, __ldcg(a.count))) : a.n;
  const Pool& p = a.pool[lo];
  const int64_t block = blockIdx.x - a.first[lo];
  if (((reinterpret_cast<uintptr_t>(p.base) | uintptr_t(p.page_bytes)) & 15) == 0) copy_block<uint4>(a, p, block, n);
  else copy_block<uint32_t>(a, p, block, n);
}

}  // namespace

extern "C" mv_status mv_pages_copy(const mv_page_pool* pools, int32_t n_pools, int64_t num_pages, const int32_t* src, const int32_t* dst,
                                   int32_t n, const int32_t* count, int32_t* status, void* cuda_stream) {
  mv::NvtxRange nvtx_range("mv_pages_copy");
  if (!pools || n_pools < 1 || num_pages < 0 || n < 0) return MV_ERR_INVALID_ARG;
  if (n_pools > MAX_POOLS || num_pages > INT32_MAX) return MV_ERR_UNSUPPORTED;
  for (const void* p : {static_cast<const void*>(src), static_cast<const void*>(dst), static_cast<const void*>(count), static_cast<const void*>(status)})
    if (reinterpret_cast<uintptr_t>(p) & 3) return MV_ERR_INVALID_ARG;
  Args a;
  int64_t ctas = 0;
  for (int i = 0; i < n_pools; ++i) {
    const int64_t bytes = pools[i].page_bytes;
    if (!pools[i].base || bytes <= 0 || (bytes & 3) || (reinterpret_cast<uintptr_t>(pools[i].base) & 3)) return MV_ERR_INVALID_ARG;
    if (bytes > (int64_t(1) << 31)) return MV_ERR_UNSUPPORTED;
    a.pool[i] = Pool{static_cast<char*>(pools[i].base), bytes};
    a.first[i] = uint32_t(ctas);
    const int64_t per = ((reinterpret_cast<uintptr_t>(pools[i].base) | uintptr_t(bytes)) & 15) == 0 ? bytes / 16 : bytes / 4;
    if (n > 0 && per > (int64_t(1) << 62) / n) return MV_ERR_UNSUPPORTED;
    ctas += (int64_t(n) * per + BLOCK - 1) / BLOCK;
    if (ctas > INT32_MAX) return MV_ERR_UNSUPPORTED;
  }
  a.first[n_pools] = uint32_t(ctas);
  if (n == 0 || num_pages == 0) return MV_OK;
  if (!src || !dst) return MV_ERR_INVALID_ARG;
  a.src = src;
  a.dst = dst;
  a.count = count;
  a.status = status;
  a.num_pages = num_pages;
  a.n = n;
  a.n_pools = n_pools;
  pages_copy_kernel<<<unsigned(ctas), NT, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
  mv::g_launches++;
  return cudaGetLastError() == cudaSuccess ? MV_OK : MV_ERR_CUDA;
}
