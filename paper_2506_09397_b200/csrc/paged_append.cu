// New keys and values into a paged cache: as they are, or as e4m3 codes with a scale for every block of 16 slots and KV head.
//
// A block that receives keys: let m be the largest finite |x| of its new rows and 2^e, e >= -126, the smallest power of two with
// m <= 448 2^e.  Its scale becomes s' = max(2^e, |s|) where it has older keys (s their scale), else 2^e; code = e4m3(x / s').
// With powers of two nothing is lost by the quotient, and older codes that move from s to s' only lose what falls below the
// smallest code.
//
// A warp does one (block, KV head) of K or of V: it holds all of the block's new rows in registers, so that they are read
// once, and a lane writes the 8 codes of the 8 elements that it read.  Bound by its bytes for prompts, by latency (row offsets,
// lengths, table, then rows and scale together) for decoding steps: 12 prompts of 2000 .. 16384 tokens, 8 KV heads of 128, in 8 bits 110 us (87 %
// of the copy rate), 48 requests with 1 .. 9 tokens 5.9 us, 20 chunks of 200 .. 2000 tokens as they are, heads of 64, 12 us.
#include <cuda_fp8.h>

#include <cuda_fp16.h>

#include "kernels.h"
#include "paged_device.cuh"

namespace sled {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSome = 8, kMany = 32;            // rows of a block's span for longer calls

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
  // the largest of `top` and the bits of all |x|, of bf16 in pairs; largest_of(top): the bits as those of a float.  Infinities and
  // NaN count as what their bits say, no less than 0x7f800000
  static __device__ __forceinline__ uint32_t largest_of(uint32_t top) { return sizeof(T) == 4 ? top : max(top << 16, top & 0xffff0000u); }
  __device__ __forceinline__ uint32_t largest(uint32_t top) const {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, u[i] & 0x7fffffffu);
      return top;
    } else {
      uint32_t two = __vimax3_u16x2(u[0] & 0x7fff7fffu, u[1] & 0x7fff7fffu, top);      // (of 16 bits `top` is a pair)
      return __vimax3_u16x2(u[2] & 0x7fff7fffu, u[3] & 0x7fff7fffu, two);
    }
  }
  __device__ __forceinline__ float at(int i) const {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
    if constexpr (sizeof(T) == 4) return __uint_as_float(u[i]);
    return __uint_as_float(i & 1 ? u[i >> 1] & 0xffff0000u : u[i >> 1] << 16);
  }
};

// the smallest power of two, at least 2^-126, of which 448 = 1.75 2^8 times is no less than the number with the bits u
// (finite, not negative)
__device__ __forceinline__ float least_scale(uint32_t u) {
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

// req_of_row by a warp, in rounds of 32 samples: a dependent load for a factor of 32 instead of one for a factor of 2
__device__ __forceinline__ int req_of_row_by_warp(const int32_t* cu_q, int n_reqs, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n_reqs;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const bool before = lane == 0 || (at < hi && cu_q[at] <= t);
    lo += (__popc(__ballot_sync(0xffffffffu, before)) - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// A cache block that receives keys: the row of the call that holds the first of them, the block's page and first slot there, how
// many older keys it has and how many new ones it gets.
struct Target {
  int row, page, slot0, off, count;
};

// T: the rows' type; kCodes: the cache holds codes, otherwise T.  kSpan rows of the call per block.
template <typename T, int H, bool kCodes, int kSpan>
__global__ void __launch_bounds__(kThreads) append_kernel(const PagedCache c, const NewRows a, bool whole) {
  constexpr int kLanes = H / 8, kAtOnce = 32 / kLanes, kPasses = kScaleBlock / kAtOnce;      // lanes of a row, rows at a time
  __shared__ Target targets[kSpan];
  __shared__ int n_targets;
  pdl_launch_dependents();
  if (threadIdx.x == 0) n_targets = 0;
  __syncthreads();
  pdl_wait();
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kSpan;
  PagedRows r{};
  r.cu_q = a.cu_q;
  r.T = a.T;
  int alone = 0;
  if (kSpan == 1 && threadIdx.x < 32) alone = req_of_row_by_warp(a.cu_q, c.n_reqs, static_cast<int>(t0));
  if (threadIdx.x < kSpan) {
    const int64_t t = t0 + threadIdx.x;
    if (t < a.T) {
      const int i = kSpan == 1 ? alone : req_of_row(a.cu_q, c.n_reqs, static_cast<int>(t));
      const ReqView v = req_view(c, r, i);
      if (v.ok && t >= v.row0 && t < v.row0 + v.m) {
        const int x = v.n - v.m + static_cast<int>(t - v.row0), off = x % kScaleBlock;
        if (t == v.row0 || off == 0) {
          const int p = x / c.ps, page = c.table[static_cast<int64_t>(i) * c.table_stride + p];
          if (page_exists(c, page)) targets[atomicAdd(&n_targets, 1)] = Target{static_cast<int>(t), page, x - p * c.ps - off, off, min(kScaleBlock - off, v.n - x)};
          else set_status(c.status, SLED_ERR_ARG);
        }
      }
    }
  }
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < c.n_reqs; i += kThreads)
      if (!req_view(c, r, i).ok) set_status(c.status, SLED_ERR_ARG);
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 2 * c.Hkv, sub_row = lane / kLanes, col = lane % kLanes * 8;
  const int n_tasks = n_targets * per;
  // where a task is: K or V of a head of a target
  struct Task {
    Target to;
    int g;
    bool is_v;
  };
  auto task_at = [&](int task) {
    const int k = task / per, rest = task - k * per;
    return Task{targets[k], rest >> 1, (rest & 1) != 0};
  };
  auto bring = [&](const Task& k, Eight<T>* y) {
    const int64_t stride = k.is_v ? a.v_stride : a.k_stride, step = kAtOnce * stride;
    const int e0 = sub_row - k.to.off;                 // of the new rows
    const T* src = reinterpret_cast<const T*>(k.is_v ? a.v : a.k) + k.to.row * stride + static_cast<int64_t>(k.g) * H + col + e0 * stride;
    if (whole && k.to.count == kScaleBlock) {          // a whole block, of aligned rows
#pragma unroll
      for (int p = 0; p < kPasses; ++p) y[p].load(src + p * step, true);
    } else {
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int e = p * kAtOnce + e0;
        if (e >= 0 && e < k.to.count) y[p].load(src + p * step, whole);
        else y[p].zero();
      }
    }
  };
  auto put = [&](const Task& k, const Eight<T>* y) {
    const int off = k.to.off, count = k.to.count;
    const int64_t head = static_cast<int64_t>(k.to.page) * c.Hkv + k.g;
    const int64_t first = (head * c.ps + k.to.slot0) * H + col;       // element of the cache: the block's first slot, this lane's columns
    char* cache = const_cast<char*>(k.is_v ? c.v : c.k);
    if constexpr (!kCodes) {
      T* to = reinterpret_cast<T*>(cache) + first;
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int e = p * kAtOnce + sub_row - off;
        if (e >= 0 && e < count) y[p].store(to + static_cast<int64_t>(p * kAtOnce + sub_row) * H);
      }
    } else {
      uint8_t* to = reinterpret_cast<uint8_t*>(cache) + first;
      float* scale = (k.is_v ? a.v_scale : a.k_scale) + head * (c.ps / kScaleBlock) + k.to.slot0 / kScaleBlock;
      const float before = off > 0 ? *scale : 0.f;
      uint32_t top = 0;            // bits of the largest |x|
#pragma unroll
      for (int p = 0; p < kPasses; ++p) top = y[p].largest(top);
      top = __reduce_max_sync(0xffffffffu, Eight<T>::largest_of(top));
      bool plain = top < 0x7f800000u;
      if (!plain) {                // without infinities and NaN
        top = 0;
#pragma unroll
        for (int p = 0; p < kPasses; ++p)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t z = __float_as_uint(y[p].at(i)) & 0x7fffffffu;
            top = max(top, z < 0x7f800000u ? z : 0u);
          }
        top = __reduce_max_sync(0xffffffffu, top);
      }
      const float now = fmaxf(least_scale(top), fabsf(before)), inv = 1.f / now;      // (a caller's own scale may be below 0)
      plain = plain && (__float_as_uint(now) & 0x7fffffu) == 0;      // a scale of the caller's own may be no power of two: true quotients
      uint8_t* mine = to + sub_row * H;
      auto codes = [&](int p) {
        uint32_t two[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) two[i] = code_pair(y[p].at(2 * i) * inv, y[p].at(2 * i + 1) * inv);
        return make_uint2(__byte_perm(two[0], two[1], 0x5410), __byte_perm(two[2], two[3], 0x5410));
      };
      if (plain && count == kScaleBlock) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) *reinterpret_cast<uint2*>(mine + p * kAtOnce * H) = codes(p);
      } else {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const int e = p * kAtOnce + sub_row - off;
          if (e < 0 || e >= count) continue;
          uint2 w = make_uint2(0, 0);
          if (plain) {
            w = codes(p);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t one = code(__fdiv_rn(y[p].at(i), now)) << (i & 3) * 8;
              if (i < 4) w.x |= one; else w.y |= one;
            }
          }
          *reinterpret_cast<uint2*>(mine + p * kAtOnce * H) = w;
        }
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
  };
  // the next task's rows are under way while this one's are coded
  Eight<T> y[2][kPasses];
  Task k[2];
  int task = warp;
  if (task < n_tasks) {
    k[0] = task_at(task);
    bring(k[0], y[0]);
  }
#pragma unroll 1
  for (; task < n_tasks; task += 2 * kWarps) {
    const int second = task + kWarps, third = second + kWarps;
    if (second < n_tasks) {
      k[1] = task_at(second);
      bring(k[1], y[1]);
    }
    put(k[0], y[0]);
    if (second >= n_tasks) break;
    if (third < n_tasks) {
      k[0] = task_at(third);
      bring(k[0], y[0]);
    }
    put(k[1], y[1]);
  }
}

template <typename T, int H, bool kCodes>
int launch(const PagedCache& c, const NewRows& a, cudaStream_t s) {
  constexpr uintptr_t kRow = 16 / sizeof(T);
  const bool whole = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 15) == 0 && a.k_stride % kRow == 0 && a.v_stride % kRow == 0;
  int sms = 0;
  if (paged_device(&sms) < 0) return -1;
  const auto by = [&](auto kernel, int span) {
    SLED_LAUNCH_PDL(kernel, dim3(static_cast<unsigned>((static_cast<int64_t>(a.T) + span - 1) / span)), dim3(kThreads), 0, s, c, a, whole);
  };
  // A block per row where there are few rows, or few to a request (a cache block or more then begins with nearly every row); else
  // one per 8 rows, or 32 where those still fill the GPU.  8 bits, 8 heads of 128, requests x rows, us for 1, 8, 32 rows a block:
  // 1 x 7 4.7, 7.4, 7.4, 48 x 5 5.7, 8.8, 24, 300 x 2 9.1, 13.5, 43; 64 x 8 6.8, 6.2, 16, 300 x 4 11.3, 9.0, 26, 40 x 100 18.4, 10.4,
  // 11.6, 3000 x 4 94, 60, 65; 16 x 500 28, 16.2, 15.5, 4 x 2000 28, 13.2, 12.7 (16 and 64 rows for 12 prompts of 2000 .. 16384: 112
  // and 109.5 against 109.6; for 20 chunks of 200 .. 2000 as they are 12.1 and 14.3 against 12.0).
  if (a.T <= 3LL * sms || a.T < 4LL * c.n_reqs) {
    by(append_kernel<T, H, kCodes, 1>, 1);
  } else if (a.T < 40LL * sms || a.T < 16LL * c.n_reqs) {
    by(append_kernel<T, H, kCodes, kSome>, kSome);
  } else {
    by(append_kernel<T, H, kCodes, kMany>, kMany);
  }
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
