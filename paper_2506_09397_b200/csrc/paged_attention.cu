// Attention of a batch's newest tokens over a paged cache: a tree (or chain) of tokens per request, optionally with the
// attention weight of every cached key added up, or over the blocks of the cache that were chosen per query.
//
// For a query row r (token, head) and the keys x it sees: s_x = scale q.k_x, p_x = exp(s_x - lse), lse = ln sum exp s_x,
// o = sum p_x v_x.  One pass over the keys with the running maximum and sum; a row that sees nothing gets o = 0 and
// lse = -inf.
#include "paged_schedule.cuh"

namespace sled {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Adds every key's attention weight: one block per (page of a request, KV head), a warp takes every fourth key of the
// page and goes through the rows in order.
template <typename T, int H>
__global__ void __launch_bounds__(128) key_weight_kernel(PagedCache c, PagedRows r, float* key_weights) {
  constexpr int D = H / 32;
  const int i = blockIdx.z, g = blockIdx.y, group = r.group;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const ReqView v = req_view(c, r, i);
  const int x0 = blockIdx.x * c.ps;
  if (!v.ok || v.m == 0 || x0 >= v.n) return;
  const int prefix = v.n - v.m;
  const int page = c.table[static_cast<int64_t>(i) * c.table_stride + blockIdx.x];
  if (!page_exists(c, page)) return;   // reported by the attention kernel
  for (int e = warp; e < c.ps && x0 + e < v.n; e += 4) {
    const int x = x0 + e;
    const int64_t at = (static_cast<int64_t>(page) * c.Hkv + g) * c.ps + e;
    const T* k = reinterpret_cast<const T*>(c.k) + at * H + lane * D;
    float sum = 0.f;
    for (int j = 0; j < v.m; ++j) {
      if (!r.parents && x > prefix + j) continue;
      if (r.parents && x >= prefix) {
        uint32_t bits[kMaxTreeNodes / 32];
        ancestors_of(r.parents + v.row0, j, bits, nullptr);
        if (!((bits[(x - prefix) >> 5] >> ((x - prefix) & 31)) & 1u)) continue;
      }
      for (int hh = 0; hh < group; ++hh) {
        const int head = g * group + hh, t = v.row0 + j;
        const float lse = r.lse[static_cast<int64_t>(t) * r.Hq + head];
        const T* q = reinterpret_cast<const T*>(r.q) + t * r.q_stride + static_cast<int64_t>(head) * H + lane * D;
        float s = 0.f;
#pragma unroll
        for (int d = 0; d < D; ++d) s = fmaf(to_f32(q[d]), to_f32(k[d]), s);
        s = warp_sum(s) * r.scale;
        if (lse != -INFINITY) sum += exp2f((s - lse) * kLog2e);
      }
    }
    if (lane == 0) key_weights[at] += sum;
  }
}

// The same from the scores that the attention kernel left: every key's sum over the rows of exp2(score - lse).  A thread
// has four keys and every fourth row, the rows' sums meet in shared memory; one addition per key, no atomics.
__global__ void __launch_bounds__(256) key_weight_sum_kernel(PagedCache c, PagedRows r, const float* scores, int64_t keys, float* key_weights) {
  constexpr int kRowsAtOnce = 512;
  __shared__ float lse[kRowsAtOnce];
  __shared__ float4 sums[4][64];
  pdl_wait();
  const AttentionLine line{c, r, kWholeRows};
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (share.from >= share.to) return;
  const int quad = threadIdx.x & 63, part = threadIdx.x >> 6, group = r.group;
  for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
    const int rows = w.v.m * group, end = min(sg.t1 * kTile, w.v.n);
    const float* mine = scores + (static_cast<int64_t>(w.v.row0) * r.Hq + sg.g * group) * keys;
    auto row_of = [&](int i) { return i / group * static_cast<int64_t>(r.Hq) + i % group; };
    auto bring_lse = [&](int first, int here) {
      __syncthreads();
      for (int i = threadIdx.x; i < here; i += 256) {
        const float l = r.lse[static_cast<int64_t>(w.v.row0) * r.Hq + sg.g * group + row_of(first + i)];
        lse[i] = l * kLog2e;
      }
      __syncthreads();
    };
    if (rows <= kRowsAtOnce) bring_lse(0, rows);
    for (int x0 = sg.t0 * kTile; x0 < end; x0 += 256) {
      const int x = x0 + quad * 4, own = x0 + threadIdx.x;
      float* to = nullptr;   // of this thread's key, under way while the scores are
      float old = 0.f;
      if (own < end) {
        const int page = c.table[static_cast<int64_t>(sg.req) * c.table_stride + quotient(own, c.ps)];
        if (page_exists(c, page)) {
          to = key_weights + (static_cast<int64_t>(page) * c.Hkv + sg.g) * c.ps + own % c.ps;
          old = *to;
        }
      }
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int first = 0; first < rows; first += kRowsAtOnce) {
        const int here = min(kRowsAtOnce, rows - first);
        if (rows > kRowsAtOnce) bring_lse(first, here);
        if (x < end) {
#pragma unroll 4
          for (int i = part; i < here; i += 4) {
            const float4 s = *reinterpret_cast<const float4*>(mine + row_of(first + i) * keys + x);
            const float l = lse[i];
            // A row that saw nothing adds nothing, whatever its query holds; nor does a row to a key that it does not see
            // (a score of -infinity), also where the row is no number.
            const bool some = l != -INFINITY;
            sum.x += some && s.x != -INFINITY ? exp2f(s.x - l) : 0.f;
            sum.y += some && s.y != -INFINITY ? exp2f(s.y - l) : 0.f;
            sum.z += some && s.z != -INFINITY ? exp2f(s.z - l) : 0.f;
            sum.w += some && s.w != -INFINITY ? exp2f(s.w - l) : 0.f;
          }
        }
      }
      sums[part][quad] = sum;
      __syncthreads();
      const float* s = reinterpret_cast<const float*>(sums) + threadIdx.x;   // and now a key per thread
      if (to) *to = old + ((s[0] + s[256]) + (s[512] + s[768]));
      __syncthreads();
    }
  });
}

// Rows per request and KV head (on average) above which the tcgen05 kernels are used.  Warp-level tensor cores and tcgen05,
// us, 8 KV heads of 128, in brackets with weights:
//   rows                       24                     28                     32                     36
//   8 contexts of 8192 keys    59 67 (104 109)        61 68 (110 109)        60 69 (118 109)        82 70 (168 116)
//   one of 1000                15.1 15.5 (25 28)      15.5 15.6 (25 28)      15.9 15.7 (26 27)      19.4 15.9 (31 31)
//   32 of 128 .. 16384         113 117 (214 236)      114 117 (230 236)      116 118 (239 236)      185 122 (2600 298: scores not kept)
// So up to 32 rows calls without weights over long contexts give away up to 9 us, and those with weights gain as much.
constexpr int kTcRows = 24;
int64_t parts_bytes(int dtype, int h) {
  const int64_t a = dtype == 1 ? paged_mma_workspace(h) : paged_f32_workspace(h), b = dtype == 1 && h >= 64 ? paged_tc_workspace(h) : 0;
  return ((a > b ? a : b) + 255) / 256 * 256;
}

// With few rows the scores are kept for the weights, 4 bytes per row and key, where they take no more than this; otherwise
// the weights are computed from the keys again, which takes a small part of the memory and many times as long (8 contexts
// of 8192 keys, one token: 65 us and 215; four tokens: 78 and 585).  The host knows the width of the page table, not the
// keys: 33 contexts of 2000 keys, one token, take 67 us with a table of 125 columns and 1170 with one of 8192.
constexpr int64_t kMostScoreBytes = 512LL << 20;
bool keeps_scores(int64_t rows_heads, int64_t keys) { return keys == 0 || rows_heads <= kMostScoreBytes / 4 / keys; }

template <typename T, int H>
int launch_rows(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* key_weights, char* ws, cudaStream_t s) {
  int n = 1;
  if constexpr (sizeof(T) == 2 && H >= 64) {
    // many rows per request: the tcgen05 kernels
    if (!list && paged_tc_serves(c, r) && static_cast<int64_t>(r.T) * (r.group) > static_cast<int64_t>(kTcRows) * c.n_reqs) {
      n = launch_paged_tc(c, r, ws, s);
      if (n < 0 || !key_weights) return n;
      const int w = launch_paged_weigh(c, r, key_weights, s);
      return w < 0 ? w : n + w;
    }
  }
  const int64_t keys = static_cast<int64_t>(c.table_cols) * c.ps;
  const bool keep = key_weights && keeps_scores(static_cast<int64_t>(r.T) * r.Hq, keys);
  float* scores = keep ? reinterpret_cast<float*>(ws + parts_bytes(c.dtype, H)) : nullptr;
  n = sizeof(T) == 4 ? launch_paged_f32(c, r, list, list_len, scores, ws, s) : launch_paged_mma(c, r, list, list_len, scores, ws, s);
  if (n < 0) return n;
  if (keep) {
    int sms = 0;
    if (paged_device(&sms) < 0) return -1;
    SLED_LAUNCH_PDL(key_weight_sum_kernel, dim3(4 * sms), dim3(256), 0, s, c, r, scores, keys, key_weights);
    return cudaGetLastError() == cudaSuccess ? n + 1 : -1;
  }
  if (key_weights) {
    key_weight_kernel<T, H><<<dim3(c.table_cols, c.Hkv, c.n_reqs), 128, 0, s>>>(c, r, key_weights);
    ++n;
  }
  return cudaGetLastError() == cudaSuccess ? n : -1;
}

}  // namespace

int64_t paged_attention_workspace(int dtype, int h, int64_t rows_heads, int64_t keys, bool weigh) {
  return parts_bytes(dtype, h) + (weigh && keeps_scores(rows_heads, keys) ? rows_heads * keys * 4 : 0);
}

int launch_paged_attention(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* key_weights, char* ws,
                           cudaStream_t s) {
  if (c.dtype == 1) {
    if (c.h == 32) return launch_rows<__nv_bfloat16, 32>(c, r, list, list_len, key_weights, ws, s);
    if (c.h == 64) return launch_rows<__nv_bfloat16, 64>(c, r, list, list_len, key_weights, ws, s);
    if (c.h == 128) return launch_rows<__nv_bfloat16, 128>(c, r, list, list_len, key_weights, ws, s);
  } else {
    if (c.h == 32) return launch_rows<float, 32>(c, r, list, list_len, key_weights, ws, s);
    if (c.h == 64) return launch_rows<float, 64>(c, r, list, list_len, key_weights, ws, s);
    if (c.h == 128) return launch_rows<float, 128>(c, r, list, list_len, key_weights, ws, s);
  }
  return -1;
}

}  // namespace sled
