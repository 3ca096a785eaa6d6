// What the warp-level kernels of attention over a cache of e4m3 codes share: codes and queries as fp16, a row's running
// maximum, sum and numerators' reference.
#pragma once
#include <cuda_fp16.h>

#include "paged_schedule.cuh"
#include "warp_mma.cuh"

namespace sled {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kHalfGain = 3.5f;   // numerators are at most 2^8 times 2^7

// partial results of units that were cut
struct ScaledParts {
  float* acc;      // [2 * blocks][rows of a unit][H], not normalised
  float* ml;       // [2 * blocks][rows of a unit][2]
  int4* desc;      // [blocks][2]: CutUnit
};

// two codes, exactly
__device__ __forceinline__ uint32_t half2_of(uint32_t two_codes) {
  uint32_t h;
  asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(h) : "r"(two_codes));
  return h;
}
__device__ __forceinline__ uint32_t half2_of_upper(uint32_t four_codes) {
  uint32_t h;
  asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, y;\n\t}" : "=r"(h) : "r"(four_codes));
  return h;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// (not volatile: the compiler may move products between the loads, whose order is kept)
__device__ __forceinline__ void mma_half(float c[4], const uint32_t a[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// This lane's H / 4 elements of a query row as fp16, times a power of two that brings the row's largest finite element to 2^14 .. 2^15;
// returns the factor that undoes it.  All lanes call it.
template <int H>
__device__ __forceinline__ float query_row(const __nv_bfloat16* q, bool valid, uint32_t f[H / 8]) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(q);
  uint32_t most = 0;       // |x| as bits of bf16, times 2^16
#pragma unroll
  for (int i = 0; i < H / 8; ++i) {
    f[i] = valid ? w[i] : 0u;
    const uint32_t lo = f[i] << 16 & 0x7fff0000u, hi = f[i] & 0x7fff0000u;
    most = max(most, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
  }
  most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
  most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
  const int e = min(max(268 - static_cast<int>(most >> 23), 1), 253);      // biased exponent of the factor
  const float up = __uint_as_float(static_cast<uint32_t>(e) << 23);
#pragma unroll
  for (int i = 0; i < H / 8; ++i) f[i] = pack_half(__uint_as_float(f[i] << 16) * up, __uint_as_float(f[i] & 0xffff0000u) * up);
  return __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
}

// A block's 2^(s - ref) become numerators by 2^(7 + ref - u) vs.  Scales may be any finite numbers, so that neither the power of two, 2^-129 to
// 2^164 where a row weighs anything, nor its inverse need be a float: both are kept as their square roots, and multiplied twice.
// (A row whose u lies further below its ref than 193 has results below 2^-149.)
__device__ __forceinline__ float weight_root(float ref, float u) { return exp2_approx(fminf(fmaf(ref - u, 0.5f, kHalfGain), 100.f)); }
__device__ __forceinline__ float rest_root(float m, float u) { return u == -INFINITY ? 0.f : exp2_approx(fmaf(u - (m == -INFINITY ? 0.f : m), 0.5f, -kHalfGain)); }
// What 2^(s - ref) is multiplied by, at most 2^126 in size: nothing is larger but what multiplies exponentials below 2^-111, in a
// block whose scale is above 2^(119 + u - ref); NaN stays.  plain_weight: where there is no such block.
__device__ __forceinline__ float plain_weight(float root, float vs) { return root * vs * root; }
__device__ __forceinline__ float at_most_2_126(float x) {
  float y;
  asm("min.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(0x1p126f));
  return y;
}
__device__ __forceinline__ float block_weight(float root, float vs) { return at_most_2_126(plain_weight(root, vs)); }
constexpr float kPlainRoom = -118.f;      // u - ref less a scale's log2: where plain_weight is finite

// A row's references: m of the scores, with the sum l of 2^(s - m), and u of the numerators 2^(s - u) vs.  They are raised only when
// something exceeds them by more than 2^kRaiseBy, which cancels in the end; all else goes by ref, m where that is finite.
constexpr float kRaiseBy = 8.f;
struct RowState {
  float m = -INFINITY, l = 0.f, u = -INFINITY;
  float ref = 0.f;
  float w = 0.f;              // the root of what a block's 2^(s - ref) are multiplied by beside vs
  // takes a stage's largest score s and the largest s + log2 |vs|; returns the factor of the output so far
  __device__ __forceinline__ float take(float mx, float mx_u) {
    if (mx > m + kRaiseBy || m == -INFINITY) {
      const float mn = fmaxf(m, mx);
      ref = mn == -INFINITY ? 0.f : mn;
      l *= exp2_approx(m - ref);
      m = mn;
    }
    float f = 1.f;
    if (mx_u > u + kRaiseBy || u == -INFINITY) {
      const float un = fmaxf(u, mx_u);
      f = exp2_approx(u - (un == -INFINITY ? 0.f : un));
      u = un;
    }
    w = u == -INFINITY ? 0.f : weight_root(ref, u);
    return f;
  }
  // what s - ref has to be below to need no raise, by the largest log2 |vs| of a stage; -infinity where plain_weight may not be finite
  __device__ __forceinline__ float room(float lv) const {
    const float x = (u - lv) - ref;
    return m == -INFINITY || x < kPlainRoom ? -INFINITY : kRaiseBy + fminf(0.f, x);
  }
  // the root of what the output is multiplied by at the end
  __device__ __forceinline__ float rest() const { return rest_root(m, u); }
};

}  // namespace sled
