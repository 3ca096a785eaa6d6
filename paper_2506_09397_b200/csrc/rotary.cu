// Rotary positions: pair i of a head at position p is turned by the angle p f_i.
//
//   (a, b) -> (a c - b s, a s + b c),   c, s = amplitude cos, sin of p f_i
//
// The angle is formed in fp64 and brought into (-1/2, 1/2] turns there.  It is off by 3 roundings, 3 2^-53 of its size: less than a pair's
// rounding to 32 bits for angles up to 2^26, 2^-20.4 at 2^31.  Its
// cosine and sine are taken in fp32 of the leading 24 bits and corrected by the rest (c - s d, s + c d, an angle d of less than 2^-23).
// They are computed once per row and pair, into shared memory, and serve all heads of the row.
//
// Bound by bytes for chunks (12011 rows of 40 heads of 128, bf16: 43.3 us, 87 % of the copy rate), by latency for steps (96 rows 2.6 us).
#include "kernels.h"
#include "paged_device.cuh"

namespace sled {

namespace {

constexpr int kThreads = 256;

// V elements of T as they lie in memory
template <typename T, int V>
struct Chunk {
  T x[V];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (V * sizeof(T) == 16) {
      *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = p[i];
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (V * sizeof(T) == 16) {
      *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(x);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = x[i];
    }
  }
};

template <typename T>
__device__ __forceinline__ void turn(T& a, T& b, float2 cs) {
  const float x = to_f32(a), y = to_f32(b);
  a = from_f32<T>(fmaf(x, cs.x, -y * cs.y));
  b = from_f32<T>(fmaf(x, cs.y, y * cs.x));
}

// A block has kRows rows (fewer at the end) and the heads [blockIdx.y heads_each, ...) of them.  A unit is a chunk of V
// elements of a head - or, of two halves, a chunk of either - or a chunk of dimensions that are copied.
template <typename T, int V, bool kHalves, int kRows>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryCall a, int heads_each) {
  extern __shared__ float2 turns[];       // [kRows][half]
  pdl_enter();
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kRows;
  const int rows = static_cast<int>(min(static_cast<int64_t>(kRows), a.n_rows - row0)), half = a.half;
  for (int i = threadIdx.x, r = 0, pair = threadIdx.x; i < rows * half; i += kThreads, pair += kThreads) {
    while (pair >= half) { pair -= half; ++r; }
    double t = static_cast<double>(a.positions[row0 + r]) * a.frequencies[pair] * 0.15915494309189535;   // turns: 1 / (2 pi)
    t -= rint(t);
    const float hi = static_cast<float>(t), d = static_cast<float>((t - hi) * 6.283185307179586);
    float s, c;
    sincospif(2.f * hi, &s, &c);
    const float amp = a.amplitude;
    turns[i] = make_float2(amp * fmaf(-s, d, c), a.sign * amp * fmaf(c, d, s));
  }
  __syncthreads();
  const int turned = kHalves ? half / V : 2 * half / V;
  const int copied = (a.head_dim - 2 * half) / V, units = turned + copied;
  const int head0 = blockIdx.y * heads_each, heads = min(heads_each, a.q.heads + a.k.heads - head0);
  int unit = threadIdx.x % units, head = threadIdx.x / units, r = 0;
  const int unit_step = kThreads % units, head_step = kThreads / units;
  while (true) {
    while (head >= heads) { head -= heads; ++r; }
    if (r >= rows) break;
    const bool is_q = head0 + head < a.q.heads;
    const RotaryRows& x = is_q ? a.q : a.k;
    const int h = is_q ? head0 + head : head0 + head - a.q.heads;
    const T* in = reinterpret_cast<const T*>(x.in) + (row0 + r) * x.in_row + h * x.in_head;
    T* out = reinterpret_cast<T*>(x.out) + (row0 + r) * x.out_row + h * x.out_head;
    if (unit < turned) {
      const float2* cs = turns + r * half;
      if constexpr (kHalves) {
        Chunk<T, V> lo, up;
        lo.load(in + unit * V);
        up.load(in + half + unit * V);
#pragma unroll
        for (int i = 0; i < V; ++i) turn(lo.x[i], up.x[i], cs[unit * V + i]);
        lo.store(out + unit * V);
        up.store(out + half + unit * V);
      } else {
        Chunk<T, V> c;
        c.load(in + unit * V);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) turn(c.x[2 * i], c.x[2 * i + 1], cs[unit * (V / 2) + i]);
        c.store(out + unit * V);
      }
    } else if (in != out) {
      Chunk<T, V> c;
      const int at = 2 * half + (unit - turned) * V;
      c.load(in + at);
      c.store(out + at);
    }
    unit += unit_step;
    head += head_step;
    if (unit >= units) { unit -= units; ++head; }
  }
}

template <typename T, int V, bool kHalves>
int launch(const RotaryCall& a, cudaStream_t s) {
  int sms = 0;
  if (paged_device(&sms) < 0) return -1;
  const int heads = a.q.heads + a.k.heads;
  const int units = ((kHalves ? a.half : 2 * a.half) + a.head_dim - 2 * a.half) / V;
  // Rows of a block share the work of their angles evenly: four where that still gives every SM sixteen blocks, two where it
  // gives eight (4, 2, 1 rows: 12011 rows of 40 heads of 128 43.6, 44.8, 50.6 us; 3001 rows of 8 heads of 64 in fp32 4.7, 4.3, 5.7);
  // where there are few rows, one, and a part of the heads.
  const auto many = [&](auto kernel, int n) {
    SLED_LAUNCH_PDL(kernel, dim3((a.n_rows + n - 1) / n), dim3(kThreads), n * a.half * sizeof(float2), s, a, heads);
  };
  if (a.n_rows >= 4 * 16 * sms) {
    many(rotary_kernel<T, V, kHalves, 4>, 4);
  } else if (a.n_rows >= 2 * 8 * sms) {
    many(rotary_kernel<T, V, kHalves, 2>, 2);
  } else {
    const int by_heads = max(1, min(min(heads * units / kThreads, 4 * sms / a.n_rows), 64));
    const int each = (heads + by_heads - 1) / by_heads;
    SLED_LAUNCH_PDL((rotary_kernel<T, V, kHalves, 1>), dim3(a.n_rows, (heads + each - 1) / each), dim3(kThreads), a.half * sizeof(float2), s, a, each);
  }
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T>
int launch_type(const RotaryCall& a, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  // 16 bytes at a time where every chunk is aligned
  bool whole = a.head_dim % V == 0 && (a.halves ? a.half : 2 * a.half) % V == 0;
  for (const RotaryRows* x : {&a.q, &a.k}) {
    if (!x->heads) continue;
    whole = whole && ((reinterpret_cast<uintptr_t>(x->in) | reinterpret_cast<uintptr_t>(x->out)) & 15) == 0;
    if (a.n_rows > 1) whole = whole && x->in_row % V == 0 && x->out_row % V == 0;
    if (x->heads > 1) whole = whole && x->in_head % V == 0 && x->out_head % V == 0;
  }
  if (a.halves) return whole ? launch<T, V, true>(a, s) : launch<T, 1, true>(a, s);
  return whole ? launch<T, V, false>(a, s) : launch<T, 2, false>(a, s);
}

}  // namespace

int launch_rotary(const RotaryCall& a, cudaStream_t s) {
  return a.dtype == BF16 ? launch_type<__nv_bfloat16>(a, s) : launch_type<float>(a, s);
}

}  // namespace sled
