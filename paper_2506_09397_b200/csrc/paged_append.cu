// New keys and values into a paged cache: as they are, or as e4m3 codes with a scale for every block of 16 slots and KV head.
//
// A block that receives keys: let m be the largest finite |x| of its new rows and 2^e, e >= -126, the smallest power of two with
// m <= 448 2^e.  Its scale becomes s' = max(2^e, s) where it has older keys (s their scale), else 2^e; code = e4m3(x / s').
// With powers of two nothing is lost by the quotient, and older codes that move from s to s' only lose what falls below the
// smallest code.
//
// A warp does one (block, KV head) of K or of V: it holds all of the block's new rows in registers, so that they are read
// once, and a lane writes the 8 codes of the 8 elements that it read.  Bound by its bytes for prompts, by latency (row offsets,
// lengths, table, then rows and scale together) for decoding steps.
#include <cuda_fp8.h>

#include <cuda_fp16.h>

#include "kernels.h"
#include "paged_device.cuh"

namespace sled {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMany = 16;            // rows of a block's span for long calls

// eight elements, as they lie in memory
template <typename T>
struct Eight {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p, bool whole) {
    if (whole) {
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    } else {
      T x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = p[i];
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const uint4*>(x)[i];
    }
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ float at(int i) const {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
    if constexpr (sizeof(T) == 4) return __uint_as_float(u[i]);
    return __uint_as_float(i & 1 ? u[i >> 1] & 0xffff0000u : u[i >> 1] << 16);
  }
};

// the smallest power of two, at least 2^-126, of which 448 = 1.75 2^8 times is no less than m (finite, not negative)
__device__ __forceinline__ float least_scale(float m) {
  const uint32_t u = __float_as_uint(m);
  const int e = static_cast<int>(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);      // biased
  return __uint_as_float(static_cast<uint32_t>(max(e, 1)) << 23);
}

__device__ __forceinline__ uint32_t code(float x) {
  if (!(fabsf(x) < INFINITY)) return 0x7fu | (__float_as_uint(x) >> 24 & 0x80u);
  return __nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3);
}
// codes of x0 (low byte) and x1; ok: both are finite
__device__ __forceinline__ uint32_t code_pair(float x0, float x1) {
  return __nv_cvt_float2_to_fp8x2(make_float2(x0, x1), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float decode(uint32_t c) { return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(c), __NV_E4M3))); }

// T: the rows' type; kCodes: the cache holds codes, otherwise T.  kSpan rows of the call per block.
template <typename T, int H, bool kCodes, int kSpan>
__global__ void __launch_bounds__(kThreads) append_kernel(const PagedCache c, const NewRows a, bool whole) {
  constexpr int kLanes = H / 8, kAtOnce = 32 / kLanes, kPasses = kScaleBlock / kAtOnce;      // lanes of a row, rows at a time
  __shared__ int2 found[kSpan];                // of every row that begins a block: request and key; -1
  pdl_enter();
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kSpan;
  PagedRows r{};
  r.cu_q = a.cu_q;
  r.T = a.T;
  if (threadIdx.x < kSpan) {
    int2 mine = make_int2(-1, 0);
    const int64_t t = t0 + threadIdx.x;
    if (t < a.T) {
      const int i = req_of_row(a.cu_q, c.n_reqs, static_cast<int>(t));
      const ReqView v = req_view(c, r, i);
      if (v.ok && t >= v.row0 && t < v.row0 + v.m) {
        const int x = v.n - v.m + static_cast<int>(t - v.row0);
        if (t == v.row0 || x % kScaleBlock == 0) mine = make_int2(i, x);
      }
    }
    found[threadIdx.x] = mine;
  }
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < c.n_reqs; i += kThreads)
      if (!req_view(c, r, i).ok) set_status(c.status, SLED_ERR_ARG);
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 2 * c.Hkv, sub_row = lane / kLanes, col = lane % kLanes * 8;
#pragma unroll 1
  for (int s = 0; s < kSpan; ++s) {
    const int req = found[s].x, x = found[s].y;
    if (req < 0) continue;
    const int n = c.n_kv[req], off = x % kScaleBlock, count = min(kScaleBlock - off, n - x);
    const int page = c.table[static_cast<int64_t>(req) * c.table_stride + x / c.ps];
    if (!page_exists(c, page)) {
      if (threadIdx.x == 0) set_status(c.status, SLED_ERR_ARG);
      continue;
    }
    const int slot0 = x % c.ps - off;           // the block's first slot
#pragma unroll 1
    for (int task = warp; task < per; task += kWarps) {
      const int g = task >> 1;
      const bool is_v = task & 1;
      const T* src = reinterpret_cast<const T*>(is_v ? a.v : a.k) + (t0 + s) * (is_v ? a.v_stride : a.k_stride) + static_cast<int64_t>(g) * H + col;
      const int64_t stride = is_v ? a.v_stride : a.k_stride;
      const int64_t head = static_cast<int64_t>(page) * c.Hkv + g;
      const int64_t first = (head * c.ps + slot0) * H + col;       // element of the cache: the block's first slot, this lane's columns
      Eight<T> y[kPasses];
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int e = p * kAtOnce + sub_row - off;                 // of the new rows
        if (e >= 0 && e < count) y[p].load(src + e * stride, whole);
        else y[p].zero();
      }
      if constexpr (!kCodes) {
        T* to = reinterpret_cast<T*>(const_cast<char*>(is_v ? c.v : c.k)) + first;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const int e = p * kAtOnce + sub_row - off;
          if (e >= 0 && e < count) y[p].store(to + static_cast<int64_t>(p * kAtOnce + sub_row) * H);
        }
      } else {
        uint8_t* to = reinterpret_cast<uint8_t*>(const_cast<char*>(is_v ? c.v : c.k)) + first;
        float* scale = (is_v ? a.v_scale : a.k_scale) + head * (c.ps / kScaleBlock) + slot0 / kScaleBlock;
        const float before = off > 0 ? *scale : 0.f;
        float most = 0.f;
        bool odd = false;
#pragma unroll
        for (int p = 0; p < kPasses; ++p)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float z = fabsf(y[p].at(i));
            const bool fine = z < INFINITY;
            odd |= !fine;
            most = fmaxf(most, fine ? z : 0.f);
          }
        const float now = fmaxf(least_scale(warp_max(most)), before), inv = 1.f / now;
        odd |= (__float_as_uint(now) & 0x7fffffu) != 0;      // a scale of the caller's own that is no power of two: true quotients
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const int e = p * kAtOnce + sub_row - off;
          if (e < 0 || e >= count) continue;
          uint2 w = make_uint2(0, 0);
          if (!odd) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              const uint32_t two = code_pair(y[p].at(i) * inv, y[p].at(i + 1) * inv) << (i & 2) * 8;
              if (i < 4) w.x |= two; else w.y |= two;
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t one = code(__fdiv_rn(y[p].at(i), now)) << (i & 3) * 8;
              if (i < 4) w.x |= one; else w.y |= one;
            }
          }
          *reinterpret_cast<uint2*>(to + static_cast<int64_t>(p * kAtOnce + sub_row) * H) = w;
        }
        if (off > 0 && now != before) {         // older keys of the block follow its scale
#pragma unroll 1
          for (int e = sub_row; e < off; e += kAtOnce) {
            uint2* at = reinterpret_cast<uint2*>(to + static_cast<int64_t>(e) * H);
            const uint2 old = *at;
            uint2 w = make_uint2(0, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t one = code(__fdiv_rn(decode((i < 4 ? old.x : old.y) >> (i & 3) * 8 & 0xffu) * before, now)) << (i & 3) * 8;
              if (i < 4) w.x |= one; else w.y |= one;
            }
            *at = w;
          }
        }
        if (lane == 0) *scale = now;
      }
    }
  }
}

template <typename T, int H, bool kCodes>
int launch(const PagedCache& c, const NewRows& a, cudaStream_t s) {
  constexpr uintptr_t kRow = 16 / sizeof(T);
  const bool whole = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 15) == 0 && a.k_stride % kRow == 0 && a.v_stride % kRow == 0;
  int sms = 0;
  if (paged_device(&sms) < 0) return -1;
  // A block per row (most of them then find that another row begins their cache block) while that fills the GPU a few times;
  // a block per 16 rows beyond.
  if (a.T <= 16 * sms)
    SLED_LAUNCH_PDL((append_kernel<T, H, kCodes, 1>), dim3(a.T), dim3(kThreads), 0, s, c, a, whole);
  else
    SLED_LAUNCH_PDL((append_kernel<T, H, kCodes, kMany>), dim3((a.T + kMany - 1LL) / kMany), dim3(kThreads), 0, s, c, a, whole);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T, int H>
int launch_h(const PagedCache& c, const NewRows& a, cudaStream_t s) {
  return c.dtype == E4M3 ? launch<T, H, true>(c, a, s) : launch<T, H, false>(c, a, s);
}

template <typename T>
int launch_type(const PagedCache& c, const NewRows& a, cudaStream_t s) {
  if (c.h == 128) return launch_h<T, 128>(c, a, s);
  return c.h == 64 ? launch_h<T, 64>(c, a, s) : launch_h<T, 32>(c, a, s);
}

}  // namespace

int launch_append(const PagedCache& c, const NewRows& a, cudaStream_t s) {
  return a.dtype == BF16 ? launch_type<__nv_bfloat16>(c, a, s) : launch_type<float>(c, a, s);
}

}  // namespace sled
