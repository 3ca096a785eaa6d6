// Attention over a paged cache of e4m3 codes with a scale for every block of 16 slots and KV head.
//
// For a query row r (token, head) and the keys x it sees, of block b: s_x = scale ks_b (q . c_x), o = sum p_x vs_b d_x over the
// codes c of K and d of V, p the softmax of s.  One pass over the keys with the running maximum and sum; a row that sees
// nothing gets o = 0 and lse = -infinity.  A warp per row, key by key, in fp32.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "kernels.h"
#include "paged_device.cuh"

namespace sled {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float decode(uint8_t c) { return __half2float(__half(__nv_cvt_fp8_to_halfraw(c, __NV_E4M3))); }

template <int H>
__global__ void __launch_bounds__(128) scaled_rows_kernel(const PagedCache c, const CacheScales sc, const PagedRows r) {
  constexpr int D = H / 32;
  pdl_enter();
  const int lane = threadIdx.x & 31;
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < c.n_reqs; i += blockDim.x) {
      const ReqView v = req_view(c, r, i);
      if (!v.ok) set_status(c.status, req_fault(r, v));
    }
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (at >= static_cast<int64_t>(r.T) * r.Hq) return;
  const int t = static_cast<int>(at / r.Hq), head = static_cast<int>(at % r.Hq), g = head / r.group;
  const int i = req_of_row(r.cu_q, c.n_reqs, t);
  const ReqView v = req_view(c, r, i);
  if (!v.ok || t < v.row0 || t >= v.row0 + v.m) return;
  const int j = t - v.row0, prefix = v.n - v.m;
  uint32_t bits[kMaxTreeNodes / 32] = {};
  bool dead = false;
  if (r.parents) {
    ancestors_of(r.parents + v.row0, j, bits, c.status);
    uint32_t any = 0;
    for (uint32_t b : bits) any |= b;
    dead = any == 0;
  }
  const float scale = r.scale * kLog2e;
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(r.q) + t * r.q_stride + static_cast<int64_t>(head) * H + lane * D;
  float qf[D], o[D], m = -INFINITY, l = 0.f;
  for (int d = 0; d < D; ++d) { qf[d] = to_f32(q[d]); o[d] = 0.f; }
  const int end = dead ? 0 : r.parents ? v.n : prefix + j + 1;
  for (int x = 0; x < end; ++x) {
    if (r.parents && x >= prefix && !((bits[(x - prefix) >> 5] >> ((x - prefix) & 31)) & 1u)) continue;
    const int page = checked_page(c, c.table[static_cast<int64_t>(i) * c.table_stride + x / c.ps]);
    const int64_t row = (static_cast<int64_t>(page) * c.Hkv + g) * c.ps + x % c.ps;
    float s = 0.f;
    for (int d = 0; d < D; ++d) s = fmaf(qf[d], decode(reinterpret_cast<const uint8_t*>(c.k)[row * H + lane * D + d]), s);
    s = warp_sum(s) * sc.k[row / kScaleBlock] * scale;
    const float top = fmaxf(m, s), f = top == -INFINITY ? 1.f : exp2f(m - top), p = exp2f(s - (top == -INFINITY ? 0.f : top));
    m = top;
    l = l * f + p;
    const float pv = p * sc.v[row / kScaleBlock];
    for (int d = 0; d < D; ++d) o[d] = fmaf(pv, decode(reinterpret_cast<const uint8_t*>(c.v)[row * H + lane * D + d]), o[d] * f);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(r.out) + t * r.out_stride + static_cast<int64_t>(head) * H + lane * D;
  for (int d = 0; d < D; ++d) out[d] = __float2bfloat16_rn(o[d] * inv);
  if (r.lse && lane == 0) r.lse[static_cast<int64_t>(t) * r.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

int64_t paged_scaled_workspace(int) { return 0; }

int launch_paged_scaled(const PagedCache& c, const CacheScales& sc, const PagedRows& r, char*, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(r.T) * r.Hq + 3) / 4));
  if (c.h == 128) SLED_LAUNCH_PDL(scaled_rows_kernel<128>, grid, dim3(128), 0, s, c, sc, r);
  else if (c.h == 64) SLED_LAUNCH_PDL(scaled_rows_kernel<64>, grid, dim3(128), 0, s, c, sc, r);
  else SLED_LAUNCH_PDL(scaled_rows_kernel<32>, grid, dim3(128), 0, s, c, sc, r);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace sled
