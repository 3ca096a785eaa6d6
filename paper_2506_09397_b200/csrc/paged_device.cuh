// Device helpers of the operators over a paged cache.
#pragma once
#include "../../include/sled.h"
#include "common.cuh"
#include "paged.h"

namespace sled {

__device__ __forceinline__ void set_status(int32_t* status, int32_t code) {
  if (status) atomicCAS(status, 0, code);
}

// A request's rows and keys, or ok = false where they do not fit the arrays of the call.
struct ReqView {
  int row0, m, n;
  bool ok;
};
__device__ __forceinline__ ReqView req_view(const PagedCache& c, const PagedRows& r, int i) {
  ReqView v;
  v.row0 = r.cu_q[i];
  const int row1 = r.cu_q[i + 1];
  v.m = row1 - v.row0;
  v.n = c.n_kv[i];
  const int before = i > 0 ? r.cu_q[i - 1] : 0;   // rows that run backwards would be another request's as well
  v.ok = v.row0 >= 0 && v.row0 >= before && row1 >= v.row0 && row1 <= r.T && v.n >= v.m &&
         v.n <= static_cast<int64_t>(c.table_cols) * c.ps && (!r.parents || v.m <= kMaxTreeNodes);
  return v;
}
// why a request is left out
__device__ __forceinline__ int32_t req_fault(const PagedRows& r, const ReqView& v) {
  return r.parents && v.m > kMaxTreeNodes && v.row0 >= 0 && v.row0 + static_cast<int64_t>(v.m) <= r.T ? SLED_ERR_K_RANGE : SLED_ERR_ARG;
}

__device__ __forceinline__ bool page_exists(const PagedCache& c, int page) {
  return static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages);
}
// page of a table entry that is about to be read; entries outside the pool are reported and read as page 0
__device__ __forceinline__ int checked_page(const PagedCache& c, int page) {
  if (page_exists(c, page)) return page;
  set_status(c.status, SLED_ERR_ARG);
  return 0;
}

// What node j of a request sees among the request's own nodes, as a bit set of kMaxTreeNodes bits: itself and its
// ancestors.  Nothing for an unused node (parent -2) or one that hangs on an unused node; a parent that is not an
// earlier node is reported and makes the node unused.  parents: the request's own entries.
__device__ __forceinline__ void ancestors_of(const int32_t* parents, int j, uint32_t bits[kMaxTreeNodes / 32], int32_t* status) {
#pragma unroll
  for (int w = 0; w < kMaxTreeNodes / 32; ++w) bits[w] = 0;
  int a = j;
  while (true) {   // strictly downwards: ends after at most j + 1 steps
#pragma unroll
    for (int w = 0; w < kMaxTreeNodes / 32; ++w)
      if (w == (a >> 5)) bits[w] |= 1u << (a & 31);
    const int p = parents[a];
    if (p == -1) return;
    if (p < -2 || p >= a) set_status(status, SLED_ERR_ARG);
    if (p < 0 || p >= a) break;
    a = p;
  }
#pragma unroll
  for (int w = 0; w < kMaxTreeNodes / 32; ++w) bits[w] = 0;
}

// request that owns row t: the last i with cu_q[i] <= t (cu_q need not be sorted where it is wrong: the result is
// checked by the caller)
__device__ __forceinline__ int req_of_row(const int32_t* cu_q, int n_reqs, int t) {
  int lo = 0, hi = n_reqs;   // cu_q[lo] <= t < cu_q[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu_q[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// order-preserving map of a float to an unsigned integer; -0 counts as 0, a NaN as larger than everything
__device__ __forceinline__ uint32_t rank_bits(float f) {
  if (f != f) return 0xffffffffu;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// Exclusive prefix sum over the block (blockDim.x a multiple of 32, at most 1024); *total receives the block's sum.
// scratch: 33 words of shared memory.  All threads call it.
__device__ __forceinline__ int block_scan(int v, int* scratch, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) scratch[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int s = lane < nw ? scratch[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    if (lane < nw) scratch[lane] = s;
    if (lane == 31) scratch[32] = s;
  }
  __syncthreads();
  *total = scratch[32];
  const int before = warp ? scratch[warp - 1] : 0;
  return before + x - v;
}

// The want-th largest of n keys (1 <= want <= n), found digit by digit from the top: key(i) -> uint32_t.  *greater
// receives how many keys are larger than the result.  hist: 256 words of shared memory, scratch: 2 words.  All threads
// of the block call it.
template <typename KeyFn>
__device__ __forceinline__ uint32_t select_largest(KeyFn key, int n, int want, int* hist, int* scratch, int* greater) {
  uint32_t prefix = 0, mask = 0;
  int above = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int b = threadIdx.x; b < 256; b += blockDim.x) hist[b] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const uint32_t x = key(i);
      if ((x & mask) == prefix) atomicAdd(&hist[(x >> shift) & 255], 1);
    }
    __syncthreads();
    if (threadIdx.x < 32) {   // lane b owns digits 8b .. 8b+7, counted from the top
      const int lane = threadIdx.x, top = 255 - 8 * lane;
      int own = 0;
#pragma unroll
      for (int d = 0; d < 8; ++d) own += hist[top - d];
      int incl = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      int run = above + incl - own;
      if (run < want && run + own >= want) {
        for (int d = 0; d < 8; ++d) {
          const int c = hist[top - d];
          if (run + c >= want) { scratch[0] = top - d; scratch[1] = run; break; }
          run += c;
        }
      }
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(scratch[0]) << shift;
    mask |= 255u << shift;
    above = scratch[1];
    __syncthreads();
  }
  *greater = above;
  return prefix;
}

}  // namespace sled
