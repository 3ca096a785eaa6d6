// Eviction from a paged cache by accumulated attention weight.
//
// Per (layer, request, KV head) with n keys in slots 0 .. n-1 and a budget of m < n: the first n_sink slots and the last
// n_recent stay, and of the candidates between them the m - n_sink - n_recent of largest weight (the lower slot first
// among equals).  The order of keys inside a cache does not matter to attention - a key carries its position - but the
// newest ones have to stay last, in order, for the next eviction to know them.  So only what has to move moves: kept
// candidates below m - n_recent stay where they are, the holes between them take the kept candidates from behind, both
// ascending, and then the newest keys close up behind them.
#include "paged_device.cuh"

namespace sled {

namespace {

// One block per (KV head, request, layer).
__global__ void __launch_bounds__(512) evict_kernel(PagedCache c, float* weights, float* weights_out, int64_t weight_layer, int budget,
                                                    int n_sink, int n_recent, int32_t* pairs, int row_words) {
  __shared__ int hist[256], scratch[33], pick[2];
  const int g = blockIdx.x, i = blockIdx.y, layer = blockIdx.z;
  const int n = c.n_kv[i];
  if (n < 0 || n > static_cast<int64_t>(c.table_cols) * c.ps) {
    if (threadIdx.x == 0) set_status(c.status, SLED_ERR_ARG);
    return;
  }
  const int32_t* table = c.table + static_cast<int64_t>(i) * c.table_stride;
  bool missing = false;   // nothing of a request with a page outside the pool is touched
  for (int b = threadIdx.x; b < (n + c.ps - 1) / c.ps; b += blockDim.x) missing |= !page_exists(c, table[b]);
  if (__syncthreads_or(missing)) {
    if (threadIdx.x == 0) set_status(c.status, SLED_ERR_ARG);
    return;
  }
  const float* w = weights + weight_layer * layer;
  float* w_out = weights_out + weight_layer * layer;
  const bool in_place = weights == weights_out;
  auto row = [&](int x) { return (static_cast<int64_t>(table[x / c.ps]) * c.Hkv + g) * c.ps + x % c.ps; };
  const int last = min(n, budget);
  if (!in_place && n <= budget)
    for (int x = threadIdx.x; x < last; x += blockDim.x) { const int64_t at = row(x); w_out[at] = w[at]; }
  if (n <= budget) return;
  const int m = budget, tail = m - n_recent, cand_end = n - n_recent;   // slots below `tail` end up holding candidates and sinks
  const int n_cand = cand_end - n_sink, want = tail - n_sink;
  int32_t* holes = pairs + ((static_cast<int64_t>(layer) * c.n_reqs + i) * c.Hkv + g) * static_cast<int64_t>(c.table_cols) * c.ps;
  int32_t* movers = holes + (static_cast<int64_t>(c.table_cols) * c.ps) / 2;
  uint32_t edge = 0xffffffffu;
  int greater = 0;
  if (want > 0) edge = select_largest([&](int a) { return rank_bits(w[row(n_sink + a)]); }, n_cand, want, hist, pick, &greater);
  const int tie_want = want - greater;
  int ties = 0, n_holes = 0, n_movers = 0;
  for (int x0 = n_sink; x0 < cand_end; x0 += blockDim.x) {
    const int x = x0 + threadIdx.x;
    const uint32_t b = x < cand_end ? rank_bits(w[row(x)]) : 0;
    const bool tie = want > 0 && x < cand_end && b == edge;
    int total;
    const int tie_rank = ties + block_scan(tie, scratch, &total);
    ties += total;
    const bool keep = want > 0 && x < cand_end && (b > edge || (tie && tie_rank < tie_want));
    const bool hole = x < tail && !keep, mover = x >= tail && x < cand_end && keep;
    const int at_h = n_holes + block_scan(hole, scratch, &total);
    n_holes += total;
    const int at_m = n_movers + block_scan(mover, scratch, &total);
    n_movers += total;
    if (hole) holes[at_h] = x;
    if (mover) movers[at_m] = x;
  }
  __syncthreads();
  char* kl = const_cast<char*>(c.k) + c.layer_bytes * layer;
  char* vl = const_cast<char*>(c.v) + c.layer_bytes * layer;
  // the kept candidates from behind into the holes: sources lie at or above `tail`, destinations below
  for (int e = threadIdx.x; e < n_holes * row_words; e += blockDim.x) {
    const int p = e / row_words, o = e % row_words;
    const int64_t to = row(holes[p]) * row_words + o, from = row(movers[p]) * row_words + o;
    reinterpret_cast<uint4*>(kl)[to] = reinterpret_cast<const uint4*>(kl)[from];
    reinterpret_cast<uint4*>(vl)[to] = reinterpret_cast<const uint4*>(vl)[from];
  }
  if (in_place) {
    for (int p = threadIdx.x; p < n_holes; p += blockDim.x) w_out[row(holes[p])] = w[row(movers[p])];
  } else {
    for (int x = threadIdx.x; x < tail; x += blockDim.x) { const int64_t at = row(x); w_out[at] = w[at]; }
    __syncthreads();
    for (int p = threadIdx.x; p < n_holes; p += blockDim.x) w_out[row(holes[p])] = w[row(movers[p])];
  }
  __syncthreads();
  // the newest keys, in order, from n - n_recent + a to m - n_recent + a: reads run ahead of the writes that reach them
  const int per = blockDim.x / row_words;
  for (int a0 = 0; a0 < n_recent; a0 += per) {
    const int a = a0 + threadIdx.x / row_words, o = threadIdx.x % row_words;
    const bool mine = threadIdx.x / row_words < per && a < n_recent;
    uint4 kx, vx;
    float wx = 0.f;
    if (mine) {
      const int64_t from = row(cand_end + a);
      kx = reinterpret_cast<const uint4*>(kl)[from * row_words + o];
      vx = reinterpret_cast<const uint4*>(vl)[from * row_words + o];
      wx = w[from];
    }
    __syncthreads();
    if (mine) {
      const int64_t to = row(tail + a);
      reinterpret_cast<uint4*>(kl)[to * row_words + o] = kx;
      reinterpret_cast<uint4*>(vl)[to * row_words + o] = vx;
      if (o == 0) w_out[to] = wx;
    }
    __syncthreads();
  }
}

}  // namespace

int launch_evict(const PagedCache& c, float* weights, float* weights_out, int64_t weight_layer, int budget, int n_sink, int n_recent,
                 int32_t* pairs, cudaStream_t s) {
  const int row_words = c.h * (c.dtype == 1 ? 2 : 4) / 16;
  evict_kernel<<<dim3(c.Hkv, c.n_reqs, c.n_layers), 512, 0, s>>>(c, weights, weights_out, weight_layer, budget, n_sink, n_recent, pairs, row_words);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace sled
