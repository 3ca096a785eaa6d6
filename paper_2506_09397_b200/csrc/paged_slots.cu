// Places of a step's tokens: which pages requests give back and get, and where every new token goes.
//
// With h_i = ceil(n_kv_i / ps) pages in the table row of request i and w_i = ceil((n_keep_i + n_new_i) / ps) wanted, it gives
// back max(0, h_i - w_i) and takes max(0, w_i - h_i); returned page number k (all requests in order) goes to place n_free + k
// of the stack, taken page number k comes from place n_free + returned - 1 - k.  Token j of request i has the position
// n_keep_i + j and the slot page(position / ps) ps + position % ps.
//
// One launch: every block adds up the lengths of all requests by itself (a few KB, from L2) and keeps the running sums in
// shared memory, so that its threads find the request of a row, or of a page, by bisection; nothing is passed between
// blocks.  A taken page that has just been returned is looked up where the returning request had it, not on the stack.
//
// Latency only: 64 requests with a few tokens each 4.2 us (lengths, sums, table, one behind the other), 300 prompts with 440,000
// tokens 8.8 us (their 5 MB of results would take 0.8; two blocks an SM - with four, six 11.4, 9.9 -, five rows a thread).
#include "kernels.h"
#include "paged_device.cuh"

namespace sled {

namespace {

constexpr int kThreads = 256;
constexpr int kMostSums = 8192;     // running sums in shared memory: of every request, or of every few

struct SlotsSums {
  int rows, take, back;             // of the requests before
};

// One request, or nothing where its numbers do not hold together.
struct SlotsReq {
  int keep, have, want, rows;
  __device__ __forceinline__ int take() const { return max(0, want - have); }
  __device__ __forceinline__ int back() const { return max(0, have - want); }
};
// pages of n keys; the sum is below 2^32 for every length and page size that the call accepts
__device__ __forceinline__ int pages_of(int n, int page_size) { return static_cast<int>((static_cast<unsigned>(n) + page_size - 1) / page_size); }
__device__ __forceinline__ bool slots_req(const SlotsCall& a, int i, SlotsReq& r) {
  const int n = a.n_kv[i], keep = a.n_keep ? a.n_keep[i] : n, fresh = a.n_new[i];
  const long long most = static_cast<long long>(a.table_cols) * a.page_size;       // below 2^31
  if (n < 0 || keep < 0 || keep > n || fresh < 0 || n > most || keep + static_cast<long long>(fresh) > most) return false;
  r.keep = keep;
  r.have = pages_of(n, a.page_size);
  r.want = pages_of(keep + fresh, a.page_size);
  r.rows = fresh;
  return true;
}

template <typename T>
__device__ __forceinline__ T warp_scan(T x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// group: requests to a running sum
__global__ void __launch_bounds__(kThreads) page_slots_kernel(const SlotsCall a, int group, int n_sums) {
  extern __shared__ SlotsSums sums[];      // [n_sums + 1]
  __shared__ long long parts[3][kThreads / 32];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (n_sums + kThreads - 1) / kThreads, g0 = min(static_cast<int>(threadIdx.x) * per, n_sums), g1 = min(g0 + per, n_sums);
  const int n_free = *a.n_free;
  long long own[3] = {0, 0, 0};
  bool ok = true;
  for (int i = g0 * group; i < min(g1 * group, a.n_reqs); ++i) {
    SlotsReq r;
    if (!slots_req(a, i, r)) { ok = false; break; }
    own[0] += r.rows;
    own[1] += r.take();
    own[2] += r.back();
  }
  long long total[3], before[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const long long x = warp_scan(own[k], lane);
    if (lane == 31) parts[k][warp] = x;
    before[k] = x - own[k];
  }
  ok = __syncthreads_and(ok);
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    total[k] = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) before[k] += parts[k][w];
      total[k] += parts[k][w];
    }
  }
  ok = ok && total[0] <= a.n_rows && n_free >= 0 && n_free + total[2] <= a.free_cap;
  const bool enough = n_free + total[2] >= total[1];
  const int64_t first_row = blockIdx.x * blockDim.x + threadIdx.x, step = gridDim.x * blockDim.x;
  if (!ok || !enough) {      // nothing happens
    if (blockIdx.x == 0) {
      if (threadIdx.x == 0) {
        set_status(a.status, ok ? SLED_ERR_NO_PAGES : SLED_ERR_ARG);
        *a.n_free_out = n_free;
        a.cu_q[a.n_reqs] = 0;
      }
      for (int i = threadIdx.x; i < a.n_reqs; i += blockDim.x) {
        a.n_kv_out[i] = a.n_kv[i];
        a.cu_q[i] = 0;
      }
    }
    for (int64_t t = first_row; t < a.n_rows; t += step) {
      if (a.positions) a.positions[t] = 0;
      if (a.slots) a.slots[t] = -1;
    }
    return;
  }
  // running sums; the first block also writes what there is per request
  SlotsSums s{static_cast<int>(before[0]), static_cast<int>(before[1]), static_cast<int>(before[2])};
  for (int g = g0; g < g1; ++g) {
    sums[g] = s;
    for (int i = g * group; i < min((g + 1) * group, a.n_reqs); ++i) {
      SlotsReq r;
      slots_req(a, i, r);
      if (blockIdx.x == 0) {
        a.n_kv_out[i] = r.keep + r.rows;
        a.cu_q[i] = s.rows;
      }
      s.rows += r.rows;
      s.take += r.take();
      s.back += r.back();
    }
  }
  const int n_rows = static_cast<int>(total[0]), n_back = static_cast<int>(total[2]), top = n_free + n_back;
  if (threadIdx.x == 0) {
    sums[n_sums] = SlotsSums{n_rows, static_cast<int>(total[1]), n_back};
    if (blockIdx.x == 0) {
      a.cu_q[a.n_reqs] = n_rows;
      *a.n_free_out = top - static_cast<int>(total[1]);
    }
  }
  __syncthreads();

  // returned page number k, where the request that returns it has it
  auto returned = [&](int k) {
    int lo = 0, hi = n_sums;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (sums[mid].back <= k) lo = mid; else hi = mid;
    }
    int at = sums[lo].back;
    SlotsReq r;
    for (int i = lo * group; i < a.n_reqs; ++i) {
      slots_req(a, i, r);
      if (k < at + r.back()) return a.table[static_cast<int64_t>(i) * a.table_stride + r.want + (k - at)];
      at += r.back();
    }
    return -1;      // not reached: k is less than their number
  };
  for (int64_t k = first_row; k < n_back; k += step) a.free_pages[n_free + k] = returned(static_cast<int>(k));

  // a block's rows are neighbours: a thread's next row is mostly of the same request
  int begin = 0, end = 0, req = 0, taken = 0;      // the request of the last row, and its rows
  SlotsReq r{};
  const int64_t each = (a.n_rows + static_cast<int64_t>(gridDim.x) * kThreads - 1) / (static_cast<int64_t>(gridDim.x) * kThreads) * kThreads;
  const int64_t last = min((blockIdx.x + 1) * each, static_cast<int64_t>(a.n_rows));
  for (int64_t row = blockIdx.x * each + threadIdx.x; row < last; row += kThreads) {
    const int t = static_cast<int>(row);
    if (t >= n_rows) {
      if (a.positions) a.positions[t] = 0;
      if (a.slots) a.slots[t] = -1;
      continue;
    }
    if (t >= end) {
      int lo = 0, hi = n_sums;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid].rows <= t) lo = mid; else hi = mid;
      }
      begin = sums[lo].rows;
      taken = sums[lo].take;
      for (req = lo * group;; ++req) {             // ends: the group has the row
        slots_req(a, req, r);
        end = begin + r.rows;
        if (t < end) break;
        begin = end;
        taken += r.take();
      }
    }
    const int x = r.keep + (t - begin), p = x / a.page_size, off = x - p * a.page_size;
    int32_t* entry = a.table + static_cast<int64_t>(req) * a.table_stride + p;
    int page;
    if (p < r.have) {
      page = *entry;
    } else {
      const int k = top - 1 - (taken + p - r.have);
      page = k < n_free ? a.free_pages[k] : returned(k - n_free);
      if (off == 0) *entry = page;                 // its first slot is a new token's
    }
    if (a.positions) a.positions[t] = x;
    if (a.slots) a.slots[t] = static_cast<int64_t>(page) * a.page_size + off;
  }
}

}  // namespace

int launch_page_slots(const SlotsCall& a, cudaStream_t s) {
  static std::atomic<bool> configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!allow_shared(page_slots_kernel, (kMostSums + 1) * static_cast<int>(sizeof(SlotsSums)), dev, configured)) return -1;
  const int group = (a.n_reqs + kMostSums - 1) / kMostSums > 1 ? (a.n_reqs + kMostSums - 1) / kMostSums : 1;
  const int n_sums = (a.n_reqs + group - 1) / group;
  // a thread has a few rows where there are many: every block goes through the lengths once
  const int blocks = max(1, min(2 * sms, static_cast<int>((static_cast<int64_t>(a.n_rows) + kThreads - 1) / kThreads)));
  SLED_LAUNCH_PDL(page_slots_kernel, dim3(blocks), dim3(kThreads), (n_sums + 1) * sizeof(SlotsSums), s, a, group, n_sums);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace sled
