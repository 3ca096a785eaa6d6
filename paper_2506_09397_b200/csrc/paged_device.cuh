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
// entry of a list of chosen blocks, a column of the page table; where rows of two requests overlap, one of them may find
// entries that nobody wrote
__device__ __forceinline__ int checked_block(const PagedCache& c, int block) {
  if (static_cast<unsigned>(block) < static_cast<unsigned>(c.table_cols)) return block;
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

// An edge for the `want` largest of n keys (1 <= want <= n): they are the keys above it and, of those equal to it, as many
// as are missing (want - *greater).  Found digit by digit from the top (11, 11 and 10 bits); it ends early where a digit
// divides the keys as wanted.  key(i) -> uint32_t.  hist: 2048 words of shared memory, scratch: 36.  All threads of the
// block (a power of two of them, 32 .. 1024) call it.
template <typename KeyFn>
__device__ __forceinline__ uint32_t select_largest(KeyFn key, int n, int want, int* hist, int* scratch, int* greater) {
  uint32_t prefix = 0, mask = 0;
  int above = 0;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048, per = bins / static_cast<int>(blockDim.x);
    for (int b = threadIdx.x; b < bins; b += blockDim.x) hist[b] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const uint32_t x = key(i);
      if ((x & mask) == prefix) atomicAdd(&hist[(x >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    const int top = bins - 1 - static_cast<int>(threadIdx.x) * per;   // this thread's digits, counted from the top
    int own = 0, total;
    for (int d = 0; d < per; ++d) own += hist[top - d];
    int run = above + block_scan(own, scratch, &total);
    if (run < want && run + own >= want) {
      for (int d = 0; d < per; ++d) {
        const int c = hist[top - d];
        if (run + c >= want) { scratch[33] = top - d; scratch[34] = run; scratch[35] = c; break; }
        run += c;
      }
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(scratch[33]) << shift;
    mask |= static_cast<uint32_t>(bins - 1) << shift;
    above = scratch[34];
    if (above + scratch[35] == want && prefix != 0) {   // everything that begins like this is wanted
      *greater = want;
      return prefix - 1;
    }
    __syncthreads();
  }
  *greater = above;
  return prefix;
}

}  // namespace sled
