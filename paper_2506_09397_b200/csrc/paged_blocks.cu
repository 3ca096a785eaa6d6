// Bounds of the keys of every block (page) of a cache, and the choice of the blocks that a query attends to.
//
// bounds[page][kv head][0/1][d] = smallest / largest k_d over the block's keys.  For a query q every key of the block has
// q.k <= sum_d max(q_d low_d, q_d high_d) = sum_d max(q_d, 0) high_d + min(q_d, 0) low_d: the block's score for that
// query, the largest over the heads that share the KV head.  A query reads the n_local blocks that end with its own and,
// of the earlier ones, those of largest score, the lower block first among equals.
#include <algorithm>

#include "paged_device.cuh"

namespace sled {

namespace {

// One warp per (page of a request, KV head): the lanes share the head dimension, every key row is read once.
template <typename T, int H>
__global__ void __launch_bounds__(256) block_bounds_kernel(PagedCache c, const int32_t* first, T* bounds) {
  constexpr int D = H / 32;
  const int i = blockIdx.y;
  const int lane = threadIdx.x & 31;
  const int n = c.n_kv[i];
  if (n < 0 || n > static_cast<int64_t>(c.table_cols) * c.ps) {
    if (threadIdx.x == 0 && blockIdx.x == 0) set_status(c.status, SLED_ERR_ARG);
    return;
  }
  const int from = first ? max(0, first[i]) : 0;
  const int b0 = from / c.ps, nb = (n + c.ps - 1) / c.ps;
  const int work = max(0, nb - b0) * c.Hkv;
  for (int w = blockIdx.x * 8 + (threadIdx.x >> 5); w < work; w += gridDim.x * 8) {
    const int b = b0 + w / c.Hkv, g = w % c.Hkv;
    const int page = c.table[static_cast<int64_t>(i) * c.table_stride + b];
    if (!page_exists(c, page)) {
      if (lane == 0) set_status(c.status, SLED_ERR_ARG);
      continue;
    }
    const int64_t at = (static_cast<int64_t>(page) * c.Hkv + g) * c.ps * H;
    const T* k = reinterpret_cast<const T*>(c.k) + at + lane * D;
    const int count = min(c.ps, n - b * c.ps);
    float lo[D], hi[D];
#pragma unroll
    for (int d = 0; d < D; ++d) { lo[d] = INFINITY; hi[d] = -INFINITY; }
    bool nan[D] = {};
    for (int e = 0; e < count; ++e)
#pragma unroll
      for (int d = 0; d < D; ++d) {
        const float x = to_f32(k[static_cast<int64_t>(e) * H + d]);
        nan[d] |= x != x;
        lo[d] = fminf(lo[d], x);
        hi[d] = fmaxf(hi[d], x);
      }
    T* out = bounds + (static_cast<int64_t>(page) * c.Hkv + g) * 2 * H + lane * D;
#pragma unroll
    for (int d = 0; d < D; ++d) {
      out[d] = from_f32<T>(nan[d] ? NAN : lo[d]);
      out[H + d] = from_f32<T>(nan[d] ? NAN : hi[d]);
    }
  }
}

// One block per (token, KV head): scores of the earlier blocks into `scores`, then the choice, ascending, into `list`.
template <typename T, int H>
__global__ void __launch_bounds__(256) block_choice_kernel(PagedCache c, PagedRows r, const T* bounds, int n_blocks, int n_local,
                                                           float* scores, int32_t* list) {
  constexpr int D = H / 32;
  __shared__ int hist[256], scratch[33], pick[2];
  const int t = blockIdx.x, g = blockIdx.y, group = r.Hq / c.Hkv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = req_of_row(r.cu_q, c.n_reqs, t);
  const ReqView v = req_view(c, r, i);
  const int j = t - v.row0;
  if (!v.ok || j < 0 || j >= v.m) return;
  const int own = (v.n - v.m + j) / c.ps;
  int32_t* mine = list + (static_cast<int64_t>(t) * c.Hkv + g) * n_blocks;
  if (own + 1 <= n_blocks) {   // everything is read
    for (int b = threadIdx.x; b <= own; b += blockDim.x) mine[b] = b;
    return;
  }
  const int early = own + 1 - n_local, want = n_blocks - n_local;   // early > want
  float* sc = scores + (static_cast<int64_t>(t) * c.Hkv + g) * c.table_cols;
  for (int b = warp; b < early; b += 8) {
    const int page = checked_page(c, c.table[static_cast<int64_t>(i) * c.table_stride + b]);
    const T* lo = bounds + (static_cast<int64_t>(page) * c.Hkv + g) * 2 * H + lane * D;
    float best = -INFINITY;
    for (int hh = 0; hh < group; ++hh) {
      const T* q = reinterpret_cast<const T*>(r.q) + t * r.q_stride + static_cast<int64_t>(g * group + hh) * H + lane * D;
      float s = 0.f;
#pragma unroll
      for (int d = 0; d < D; ++d) {
        const float x = to_f32(q[d]);
        s = fmaf(fmaxf(x, 0.f), to_f32(lo[H + d]), s);
        s = fmaf(fminf(x, 0.f), to_f32(lo[d]), s);
      }
      s = warp_sum(s);
      best = s != s || best != best ? NAN : fmaxf(best, s);
    }
    if (lane == 0) sc[b] = best;
  }
  __syncthreads();
  int greater = 0;
  uint32_t edge = 0xffffffffu;
  if (want > 0) edge = select_largest([&](int b) { return rank_bits(sc[b]); }, early, want, hist, pick, &greater);
  int taken = 0, ties = 0;
  const int tie_want = want - greater;
  for (int b0 = 0; b0 < early && want > 0; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    const uint32_t x = b < early ? rank_bits(sc[b]) : 0;
    const bool tie = b < early && x == edge;
    int n_tie, n_take;
    const int tie_rank = ties + block_scan(tie, scratch, &n_tie);
    const bool take = b < early && (x > edge || (tie && tie_rank < tie_want));
    const int at = taken + block_scan(take, scratch, &n_take);
    if (take) mine[at] = b;
    taken += n_take;
    ties += n_tie;
  }
  for (int b = threadIdx.x; b < n_local; b += blockDim.x) mine[want + b] = early + b;
}

template <typename T, int H>
int bounds_typed(const PagedCache& c, const int32_t* first, void* bounds, cudaStream_t s) {
  block_bounds_kernel<T, H><<<dim3(std::min(64, (c.table_cols * c.Hkv + 7) / 8), c.n_reqs), 256, 0, s>>>(c, first, static_cast<T*>(bounds));
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}
template <typename T, int H>
int choice_typed(const PagedCache& c, const PagedRows& r, const void* bounds, int n_blocks, int n_local, float* scores, int32_t* list, cudaStream_t s) {
  block_choice_kernel<T, H><<<dim3(r.T, c.Hkv), 256, 0, s>>>(c, r, static_cast<const T*>(bounds), n_blocks, n_local, scores, list);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace

int launch_block_bounds(const PagedCache& c, const int32_t* first, void* bounds, cudaStream_t s) {
  if (c.dtype == 1) {
    if (c.h == 32) return bounds_typed<__nv_bfloat16, 32>(c, first, bounds, s);
    if (c.h == 64) return bounds_typed<__nv_bfloat16, 64>(c, first, bounds, s);
    if (c.h == 128) return bounds_typed<__nv_bfloat16, 128>(c, first, bounds, s);
  } else {
    if (c.h == 32) return bounds_typed<float, 32>(c, first, bounds, s);
    if (c.h == 64) return bounds_typed<float, 64>(c, first, bounds, s);
    if (c.h == 128) return bounds_typed<float, 128>(c, first, bounds, s);
  }
  return -1;
}

int launch_block_choice(const PagedCache& c, const PagedRows& r, const void* bounds, int n_blocks, int n_local, float* scores,
                        int32_t* list, cudaStream_t s) {
  if (c.dtype == 1) {
    if (c.h == 32) return choice_typed<__nv_bfloat16, 32>(c, r, bounds, n_blocks, n_local, scores, list, s);
    if (c.h == 64) return choice_typed<__nv_bfloat16, 64>(c, r, bounds, n_blocks, n_local, scores, list, s);
    if (c.h == 128) return choice_typed<__nv_bfloat16, 128>(c, r, bounds, n_blocks, n_local, scores, list, s);
  } else {
    if (c.h == 32) return choice_typed<float, 32>(c, r, bounds, n_blocks, n_local, scores, list, s);
    if (c.h == 64) return choice_typed<float, 64>(c, r, bounds, n_blocks, n_local, scores, list, s);
    if (c.h == 128) return choice_typed<float, 128>(c, r, bounds, n_blocks, n_local, scores, list, s);
  }
  return -1;
}

}  // namespace sled
