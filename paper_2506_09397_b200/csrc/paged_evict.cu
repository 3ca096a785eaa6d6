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

constexpr int kThreads = 512;
constexpr int kMostCached = 8192;    // keys whose ranks stay in shared memory

// One block per (KV head, request, layer).  The weights are read once (their order-preserving bits stay in shared memory),
// the edge of the choice is found digit by digit, every thread then goes through a stretch of slots and writes down the
// holes and the keys that fill them; the rest is copying, 16 bytes a thread, four rows under way.  Bound by the rows that move: 32 layers of 8
// contexts of 1500 .. 6000 keys down to 2048, 8 KV heads of 128, 306 us, 4.7 TB/s read and written (256 threads 349 us, 1024
// 311); one layer's worth of 16 KB in 11 us is launch, selection and latency.
__global__ void __launch_bounds__(kThreads) evict_kernel(PagedCache c, const float* weights, float* weights_out, int64_t weight_layer, int budget,
                                                         int n_sink, int n_recent, int32_t* pairs, int row_words) {
  __shared__ int hist[2048], scratch[36];
  __shared__ uint32_t cached[kMostCached];
  pdl_launch_dependents();
  pdl_wait();
  const int g = blockIdx.x, i = blockIdx.y, layer = blockIdx.z;
  const int n = c.n_kv[i];
  if (n < 0 || n > static_cast<int64_t>(c.table_cols) * c.ps) {
    if (threadIdx.x == 0) set_status(c.status, SLED_ERR_ARG);
    return;
  }
  const int32_t* table = c.table + static_cast<int64_t>(i) * c.table_stride;
  bool missing_page = false;   // nothing of a request with a page outside the pool is touched
  for (int b = threadIdx.x; b < (n + c.ps - 1) / c.ps; b += kThreads) missing_page |= !page_exists(c, table[b]);
  if (__syncthreads_or(missing_page)) {
    if (threadIdx.x == 0) set_status(c.status, SLED_ERR_ARG);
    return;
  }
  const float* w = weights + weight_layer * layer;
  float* w_out = weights_out + weight_layer * layer;
  const bool in_place = weights == weights_out;
  // row of a slot in the pool: fits 31 bits
  const int shift = (c.ps & (c.ps - 1)) == 0 ? __ffs(c.ps) - 1 : -1;   // a division costs more than the rest of it
  auto row = [&](int x) {
    const int page = shift >= 0 ? x >> shift : x / c.ps;
    return (table[page] * c.Hkv + g) * c.ps + (x - page * c.ps);
  };
  if (n <= budget) {
    if (!in_place)
      for (int x = threadIdx.x; x < n; x += kThreads) { const int at = row(x); w_out[at] = w[at]; }
    return;
  }
  const int tail = budget - n_recent, cand_end = n - n_recent;   // slots below `tail` end up holding sinks and candidates
  const int n_cand = cand_end - n_sink, want = tail - n_sink;
  int32_t* to_rows = pairs + ((static_cast<int64_t>(layer) * c.n_reqs + i) * c.Hkv + g) * static_cast<int64_t>(c.table_cols) * c.ps;
  int32_t* from_rows = to_rows + static_cast<int64_t>(c.table_cols) * c.ps / 2;
  for (int a = threadIdx.x; a < min(n_cand, kMostCached); a += kThreads) cached[a] = rank_bits(w[row(n_sink + a)]);
  __syncthreads();
  auto rank = [&](int a) { return a < kMostCached ? cached[a] : rank_bits(w[row(n_sink + a)]); };
  uint32_t edge = 0xffffffffu;
  int greater = want, total;
  if (want > 0) edge = select_largest(rank, n_cand, want, hist, scratch, &greater);
  const int missing = want - greater;
  // a thread goes through a stretch of candidates, in order
  const int per = (n_cand + kThreads - 1) / kThreads, a0 = min(static_cast<int>(threadIdx.x) * per, n_cand), a1 = min(a0 + per, n_cand);
  int ties = 0;
  for (int a = a0; a < a1; ++a) ties += rank(a) == edge;
  ties = block_scan(ties, scratch, &total);
  auto kept = [&](uint32_t x) { return want > 0 && (x > edge || (x == edge && ties < missing)); };
  const int ties0 = ties;
  int holes = 0, movers = 0;
  for (int a = a0; a < a1; ++a) {
    const uint32_t x = rank(a);
    const bool k = kept(x);
    holes += n_sink + a < tail && !k;
    movers += n_sink + a >= tail && k;
    ties += x == edge;
  }
  int n_moves;
  holes = block_scan(holes, scratch, &n_moves);
  movers = block_scan(movers, scratch, &total);
  ties = ties0;
  for (int a = a0; a < a1; ++a) {
    const uint32_t x = rank(a);
    const bool k = kept(x);
    if (n_sink + a < tail && !k) to_rows[holes++] = row(n_sink + a);
    if (n_sink + a >= tail && k) from_rows[movers++] = row(n_sink + a);
    ties += x == edge;
  }
  if (!in_place)
    for (int x = threadIdx.x; x < tail; x += kThreads) { const int at = row(x); w_out[at] = w[at]; }
  __syncthreads();
  uint4* kl = reinterpret_cast<uint4*>(const_cast<char*>(c.k) + c.layer_bytes * layer);
  uint4* vl = reinterpret_cast<uint4*>(const_cast<char*>(c.v) + c.layer_bytes * layer);
  // the kept candidates from behind into the holes: sources lie at or above `tail`, destinations below
  const int rows_at_once = kThreads / row_words, word = threadIdx.x % row_words, mine = threadIdx.x / row_words;
  if (mine < rows_at_once)
    for (int p0 = mine; p0 < n_moves; p0 += 4 * rows_at_once) {
      uint4 kx[4], vx[4];
      int to[4];
      float wx[4];
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const int p = p0 + z * rows_at_once;
        if (p < n_moves) {
          const int64_t from = from_rows[p];
          to[z] = to_rows[p];
          kx[z] = kl[from * row_words + word];
          vx[z] = vl[from * row_words + word];
          wx[z] = w[from];
        }
      }
#pragma unroll
      for (int z = 0; z < 4; ++z)
        if (p0 + z * rows_at_once < n_moves) {
          kl[static_cast<int64_t>(to[z]) * row_words + word] = kx[z];
          vl[static_cast<int64_t>(to[z]) * row_words + word] = vx[z];
          if (word == 0) w_out[to[z]] = wx[z];
        }
    }
  __syncthreads();
  // the newest keys, in order, from cand_end + a to tail + a: every round reads its rows before it writes them, and rows
  // that a round writes have been read in it or before
  for (int r0 = 0; r0 < n_recent; r0 += 4 * rows_at_once) {
    uint4 kx[4], vx[4];
    float wx[4];
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const int a = r0 + z * rows_at_once + mine;
      if (mine < rows_at_once && a < n_recent) {
        const int64_t from = row(cand_end + a);
        kx[z] = kl[from * row_words + word];
        vx[z] = vl[from * row_words + word];
        wx[z] = w[from];
      }
    }
    __syncthreads();
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const int a = r0 + z * rows_at_once + mine;
      if (mine < rows_at_once && a < n_recent) {
        const int64_t to = row(tail + a);
        kl[to * row_words + word] = kx[z];
        vl[to * row_words + word] = vx[z];
        if (word == 0) w_out[to] = wx[z];
      }
    }
    __syncthreads();
  }
}

}  // namespace

int launch_evict(const PagedCache& c, float* weights, float* weights_out, int64_t weight_layer, int budget, int n_sink, int n_recent,
                 int32_t* pairs, cudaStream_t s) {
  const int row_words = c.h * (c.dtype == 1 ? 2 : 4) / 16;
  SLED_LAUNCH_PDL(evict_kernel, dim3(c.Hkv, c.n_reqs, c.n_layers), dim3(kThreads), 0, s, c, static_cast<const float*>(weights), weights_out,
                  weight_layer, budget, n_sink, n_recent, pairs, row_words);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace sled
