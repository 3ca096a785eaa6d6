// Attention over a paged bf16 cache on the warp-level tensor cores.
//
// A unit is the query rows that share a KV head (a block of up to 64 of them): they are the M side of m16n8k16 products,
// so a cached key is read once for all of them.  With up to 16 (32) rows the four computing warps split every 64-key tile
// four (two) ways and merge their (maximum, sum, output) at the end of the unit; with more, every warp has 16 rows of its
// own.  A fifth warp brings the tiles in by TMA, 16 keys x head_dim per copy (128-byte swizzle, so that the matrix loads
// meet no bank conflicts), through a ring of three stages that runs on across units.  Work is handed out as
// paged_schedule.cuh says: all blocks resident, two on an SM, equal shares of the line of tiles; units that were cut leave
// partial (maximum, sum, output) for the merge kernel.
// What binds: the bytes of K and V up to about 32 rows, the tensor path above.  Measured, 8 KV heads of 128, 4 contexts of
// 32768 keys, with the merge: 4 rows (one token of 4 heads) 90 us, 6.0 TB/s; one context of 1000 keys 11.7 us, which is launches and latency.
#include <type_traits>

#include "gemm_tc.h"
#include "kernels.h"
#include "paged_schedule.cuh"
#include "warp_mma.cuh"

namespace sled {

namespace {

constexpr int kStages = 3;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

// A stage holds K, then V: four groups of 16 keys, each [H / 64][16 keys][64 columns]; the 16-byte chunk c of a row of 128
// bytes lies at c ^ (row & 7).
template <int H>
struct Smem {
  static constexpr int kGroup = 16 * H * 2;
  static constexpr int kHalf = 4 * kGroup;              // K or V of a tile
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kMergePitch = 40;                // 32 dimensions of a row; eight rows meet eight times four banks
  static constexpr int kMerge = 64 * (kMergePitch + 2) * 4;
  static constexpr int kOffMerge = kStages * kStage;
  static constexpr int kOffTree = kOffMerge + kMerge;
  static constexpr int kOffBar = kOffTree + kMaxTreeNodes * (kMaxTreeNodes / 32) * 4;
  static constexpr int kTotal = kOffBar + 16 * kStages + 1024;     // alignment slack
};
static_assert(kMaxTreeNodes == 128);   // four words per node
static_assert(Smem<128>::kTotal + 1024 + 256 <= 228 * 1024 / 2, "two blocks on an SM");

template <int H>
__device__ __forceinline__ uint32_t at(uint32_t base, int key, int chunk) {
  if constexpr (H == 32) {   // two keys to a row of 128 bytes
    const int row = (key & 15) >> 1;
    return base + (key >> 4) * Smem<H>::kGroup + row * 128 + ((((key & 1) * 4 + chunk) ^ row) << 4);
  }
  return base + (key >> 4) * Smem<H>::kGroup + (chunk >> 3) * 2048 + (key & 15) * 128 + (((chunk & 7) ^ (key & 7)) << 4);
}

struct Ring {
  uint32_t base, full, empty;
  int it;                 // tiles so far
};

struct UnitRows {
  int req, row0, m;       // the request's rows
  int group, g, j;        // j < 0: all tokens of the request, else that token
  int first, count;       // rows of the unit's block: first .. first + count - 1
  int prefix, end;        // positions below `prefix` are seen by everybody; there are `end` of them
  __device__ __forceinline__ int token(int r) const { return j >= 0 ? j : quotient(first + r, group); }
  __device__ __forceinline__ int head(int r) const { return g * group + first + r - quotient(first + r, group) * group; }
};

struct Parts {
  float* acc;      // [2 * blocks][kUnitRows][H], not normalised
  float* ml;       // [2 * blocks][kUnitRows][2]
  int4* desc;      // [blocks][2]: CutUnit
  float* scores;   // null, or [rows][Hq][keys]
  int64_t keys;
};

// One stretch of a unit: MT warps cover the rows, 4 / MT the keys of a tile.
template <int H, int MT>
__device__ __forceinline__ void consume(const PagedCache& c, const PagedRows& r, const UnitRows& u, const Segment& sg, Ring& ring,
                                        volatile int* stop, float* merge, const uint32_t* tree, const Parts& parts) {
  using S = Smem<H>;
  constexpr int KS = H / 16, DN = H / 8, NT = 2 * MT;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, tq = lane & 3;
  const int mt = warp % MT, share = warp / MT, key_off = share * 16 * MT;
  const int r_lo = mt * 16 + gq, r_hi = r_lo + 8;
  const bool active = mt * 16 < u.count, v_lo = r_lo < u.count, v_hi = r_hi < u.count;
  const int j_lo = v_lo ? u.token(r_lo) : 0, j_hi = v_hi ? u.token(r_hi) : 0;
  const int h_lo = v_lo ? u.head(r_lo) : 0, h_hi = v_hi ? u.head(r_hi) : 0;
  const float scale = r.scale * kLog2e;

  uint32_t qf[KS][4];
  {
    const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(r.q);
    const uint32_t* q_lo = reinterpret_cast<const uint32_t*>(q + (u.row0 + j_lo) * r.q_stride + static_cast<int64_t>(h_lo) * H);
    const uint32_t* q_hi = reinterpret_cast<const uint32_t*>(q + (u.row0 + j_hi) * r.q_stride + static_cast<int64_t>(h_hi) * H);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks][0] = v_lo ? q_lo[ks * 8 + tq] : 0u;
      qf[ks][1] = v_hi ? q_hi[ks * 8 + tq] : 0u;
      qf[ks][2] = v_lo ? q_lo[ks * 8 + 4 + tq] : 0u;
      qf[ks][3] = v_hi ? q_hi[ks * 8 + 4 + tq] : 0u;
    }
  }
  float o[DN][4];
#pragma unroll
  for (int i = 0; i < DN; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m_lo = -INFINITY, m_hi = -INFINITY, l_lo = 0.f, l_hi = 0.f;
  bool failed = false;

  for (int tile = sg.t0; tile < sg.t1; ++tile, ++ring.it) {
    const int st = ring.it % kStages;
    if (*stop || !mbar_wait(ring.full + 8 * st, (ring.it / kStages) & 1, stop)) { *stop = 1; failed = true; break; }
    const int k0 = tile * kTile + key_off;    // position of this warp's first key
    if (active && k0 < u.end) {
      const uint32_t kb = ring.base + st * S::kStage, vb = kb + S::kHalf;
      float sc[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int np = 0; np < MT; ++np) {
          uint32_t b0, b1, b2, b3;
          ldmatrix_x4(at<H>(kb, key_off + (np * 2 + (lane >> 4)) * 8 + (lane & 7), 2 * ks + ((lane >> 3) & 1)), b0, b1, b2, b3);
          mma_bf16(sc[np * 2], qf[ks], b0, b1);
          mma_bf16(sc[np * 2 + 1], qf[ks], b2, b3);
        }
      // Everybody sees a tile inside the prefix.  In the others a key that a row does not see, or that does not exist,
      // becomes -infinity whatever it is (a comparison, not a sum, so that NaN does not survive).
      const bool masked = k0 + 16 * MT > u.prefix;
      if (masked) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int x = k0 + nt * 8 + 2 * tq + (e & 1), j = e < 2 ? j_lo : j_hi;
            bool seen = x < u.end;
            if (x >= u.prefix && seen) {
              const int a = x - u.prefix;
              if (r.parents && u.j < 0) seen = (tree[j * (kMaxTreeNodes / 32) + (a >> 5)] >> (a & 31)) & 1u;
              else if (u.j < 0) seen = a <= j;
            }
            if (!seen) sc[nt][e] = -INFINITY;
          }
      }
      if (parts.scores) {
        float* s_lo = parts.scores + (static_cast<int64_t>(u.row0 + j_lo) * r.Hq + h_lo) * parts.keys + k0 + 2 * tq;
        float* s_hi = parts.scores + (static_cast<int64_t>(u.row0 + j_hi) * r.Hq + h_hi) * parts.keys + k0 + 2 * tq;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          if (k0 + nt * 8 + 2 * tq < u.end) {
            if (v_lo) *reinterpret_cast<float2*>(s_lo + nt * 8) = make_float2(sc[nt][0] * scale, sc[nt][1] * scale);
            if (v_hi) *reinterpret_cast<float2*>(s_hi + nt * 8) = make_float2(sc[nt][2] * scale, sc[nt][3] * scale);
          }
      }
      float mx_lo = -INFINITY, mx_hi = -INFINITY;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mx_lo = fmaxf(mx_lo, fmaxf(sc[nt][0], sc[nt][1]));
        mx_hi = fmaxf(mx_hi, fmaxf(sc[nt][2], sc[nt][3]));
      }
      mx_lo = fmaxf(mx_lo, __shfl_xor_sync(0xffffffffu, mx_lo, 1));
      mx_lo = fmaxf(mx_lo, __shfl_xor_sync(0xffffffffu, mx_lo, 2));
      mx_hi = fmaxf(mx_hi, __shfl_xor_sync(0xffffffffu, mx_hi, 1));
      mx_hi = fmaxf(mx_hi, __shfl_xor_sync(0xffffffffu, mx_hi, 2));
      const float mn_lo = fmaxf(m_lo, mx_lo * scale), mn_hi = fmaxf(m_hi, mx_hi * scale);
      const float ms_lo = mn_lo == -INFINITY ? 0.f : mn_lo, ms_hi = mn_hi == -INFINITY ? 0.f : mn_hi;
      const float al_lo = exp2_approx(m_lo - ms_lo), al_hi = exp2_approx(m_hi - ms_hi);
      m_lo = mn_lo;
      m_hi = mn_hi;
      l_lo *= al_lo;
      l_hi *= al_hi;
#pragma unroll
      for (int i = 0; i < DN; ++i) { o[i][0] *= al_lo; o[i][1] *= al_lo; o[i][2] *= al_hi; o[i][3] *= al_hi; }
      uint32_t pf[MT][4];   // the probabilities as A operand, rounded to bf16 for the second product; their sum is not
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float p0 = exp2_approx(fmaf(sc[nt][0], scale, -ms_lo)), p1 = exp2_approx(fmaf(sc[nt][1], scale, -ms_lo));
        const float p2 = exp2_approx(fmaf(sc[nt][2], scale, -ms_hi)), p3 = exp2_approx(fmaf(sc[nt][3], scale, -ms_hi));
        l_lo += p0 + p1;
        l_hi += p2 + p3;
        pf[nt >> 1][(nt & 1) * 2] = pack_bf16(p0, p1);
        pf[nt >> 1][(nt & 1) * 2 + 1] = pack_bf16(p2, p3);
      }
      if (!masked) {
#pragma unroll
        for (int kt = 0; kt < MT; ++kt)
#pragma unroll
          for (int dp = 0; dp < DN / 2; ++dp) {
            uint32_t b0, b1, b2, b3;
            ldmatrix_x4_trans(at<H>(vb, key_off + kt * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), dp * 2 + (lane >> 4)), b0, b1, b2, b3);
            mma_bf16(o[dp * 2], pf[kt], b0, b1);
            mma_bf16(o[dp * 2 + 1], pf[kt], b2, b3);
          }
      } else {
        // A probability of 0 does not silence a value that is not finite.  Values of keys that do not exist are taken as
        // 0; of the others those that are not finite are left out of the product and added afterwards, to the rows that
        // see them.
        bool odd = false;
#pragma unroll
        for (int kt = 0; kt < MT; ++kt) {
          const int x = k0 + kt * 16 + 2 * tq;
          const uint32_t there0 = (x < u.end ? 0xffffu : 0u) | (x + 1 < u.end ? 0xffff0000u : 0u);
          const uint32_t there1 = (x + 8 < u.end ? 0xffffu : 0u) | (x + 9 < u.end ? 0xffff0000u : 0u);
#pragma unroll
          for (int dp = 0; dp < DN / 2; ++dp) {
            uint32_t b[4];
            ldmatrix_x4_trans(at<H>(vb, key_off + kt * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), dp * 2 + (lane >> 4)), b[0], b[1], b[2], b[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              b[e] &= (e & 1) ? there1 : there0;
              const uint32_t off = ((b[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((b[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
              odd |= off != 0;
              b[e] &= ~off;
            }
            mma_bf16(o[dp * 2], pf[kt], b[0], b[1]);
            mma_bf16(o[dp * 2 + 1], pf[kt], b[2], b[3]);
          }
        }
        if (__any_sync(0xffffffffu, odd)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            for (int e = 0; e < 8; ++e) {
              const int src = (lane & ~3) | (e >> 1);
              const uint32_t w_lo = __shfl_sync(0xffffffffu, pf[nt >> 1][(nt & 1) * 2], src);
              const uint32_t w_hi = __shfl_sync(0xffffffffu, pf[nt >> 1][(nt & 1) * 2 + 1], src);
              const float p_lo = __uint_as_float(e & 1 ? w_lo & 0xffff0000u : w_lo << 16);
              const float p_hi = __uint_as_float(e & 1 ? w_hi & 0xffff0000u : w_hi << 16);
              const int key = key_off + nt * 8 + e;
              if (tile * kTile + key >= u.end) continue;
#pragma unroll
              for (int i = 0; i < DN; ++i) {
                uint32_t w;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at<H>(vb, key, i) + tq * 4));
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                  const float v = __uint_as_float(z ? w & 0xffff0000u : w << 16);
                  if (!(fabsf(v) < INFINITY)) {
                    if (p_lo != 0.f) o[i][z] = fmaf(p_lo, v, o[i][z]);
                    if (p_hi != 0.f) o[i][2 + z] = fmaf(p_hi, v, o[i][2 + z]);
                  }
                }
              }
            }
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(ring.empty + 8 * st);
  }

  l_lo += __shfl_xor_sync(0xffffffffu, l_lo, 1);
  l_lo += __shfl_xor_sync(0xffffffffu, l_lo, 2);
  l_hi += __shfl_xor_sync(0xffffffffu, l_hi, 1);
  l_hi += __shfl_xor_sync(0xffffffffu, l_hi, 2);
  if (r.parents && u.j < 0) {   // an unused node - it does not even see itself - sees nothing
    const uint4 b_lo = *reinterpret_cast<const uint4*>(tree + j_lo * (kMaxTreeNodes / 32));
    const uint4 b_hi = *reinterpret_cast<const uint4*>(tree + j_hi * (kMaxTreeNodes / 32));
    if (!(b_lo.x | b_lo.y | b_lo.z | b_lo.w)) {
      m_lo = -INFINITY;
      l_lo = 0.f;
#pragma unroll
      for (int i = 0; i < DN; ++i) o[i][0] = o[i][1] = 0.f;
    }
    if (!(b_hi.x | b_hi.y | b_hi.z | b_hi.w)) {
      m_hi = -INFINITY;
      l_hi = 0.f;
#pragma unroll
      for (int i = 0; i < DN; ++i) o[i][2] = o[i][3] = 0.f;
    }
  }

  if constexpr (MT < 4) {
    // The warps that shared rows lay their outputs side by side, 32 dimensions at a time, and all threads add them up: four
    // dimensions of a row (or two rows) each.
    constexpr int kShares = 4 / MT, kRowsHere = 16 * MT, kPitch = S::kMergePitch;
    float2* ml = reinterpret_cast<float2*>(merge + 64 * kPitch);
    const int mine = share * kRowsHere + r_lo, row0 = threadIdx.x >> 3, col = (threadIdx.x & 7) * 4;
    int tok[MT], hd[MT];
#pragma unroll
    for (int k = 0; k < MT; ++k) {
      tok[k] = u.token(row0 + 16 * k);
      hd[k] = u.head(row0 + 16 * k);
    }
#pragma unroll 1
    for (int part = 0; part < H / 32; ++part) {
      asm volatile("bar.sync 2, 128;" ::: "memory");      // everybody has read what was there
      if (part == 0 && tq == 0) {
        ml[mine] = make_float2(m_lo, l_lo);
        ml[mine + 8] = make_float2(m_hi, l_hi);
      }
#pragma unroll
      for (int z = 0; z < H / 32; ++z)
        if (z == part) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<float2*>(merge + mine * kPitch + i * 8 + 2 * tq) = make_float2(o[z * 4 + i][0], o[z * 4 + i][1]);
            *reinterpret_cast<float2*>(merge + (mine + 8) * kPitch + i * 8 + 2 * tq) = make_float2(o[z * 4 + i][2], o[z * 4 + i][3]);
          }
        }
      asm volatile("bar.sync 2, 128;" ::: "memory");
#pragma unroll
      for (int k = 0; k < MT; ++k) {
        const int row = row0 + 16 * k;
        float2 x[kShares];
        float top = -INFINITY, den = 0.f;
#pragma unroll
        for (int sh = 0; sh < kShares; ++sh) {
          x[sh] = ml[sh * kRowsHere + row];
          top = fmaxf(top, x[sh].x);
        }
        const float ref = top == -INFINITY ? 0.f : top;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int sh = 0; sh < kShares; ++sh) {
          const float f = exp2_approx(x[sh].x - ref);
          const float4 y = *reinterpret_cast<const float4*>(merge + (sh * kRowsHere + row) * kPitch + col);
          den = fmaf(f, x[sh].y, den);
          sum.x = fmaf(f, y.x, sum.x);
          sum.y = fmaf(f, y.y, sum.y);
          sum.z = fmaf(f, y.z, sum.z);
          sum.w = fmaf(f, y.w, sum.w);
        }
        if (row >= u.count || failed || *stop) continue;
        const int d = part * 32 + col;
        if (sg.whole) {
          const float inv = den == 0.f ? 0.f : 1.f / den;    // a row that saw nothing has a sum of 0: its output is 0
          const int64_t t = u.row0 + tok[k];
          uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(r.out) + t * r.out_stride + static_cast<int64_t>(hd[k]) * H + d);
          out[0] = pack_bf16(sum.x * inv, sum.y * inv);
          out[1] = pack_bf16(sum.z * inv, sum.w * inv);
          if (r.lse && d == 0) r.lse[t * r.Hq + hd[k]] = den == 0.f ? -INFINITY : (top + log2f(den)) * kLn2;
        } else {
          const int64_t at_row = static_cast<int64_t>(sg.slot) * kUnitRows + row;
          *reinterpret_cast<float4*>(parts.acc + at_row * H + d) = sum;
          if (d == 0) *reinterpret_cast<float2*>(parts.ml + at_row * 2) = make_float2(top, den);
        }
      }
    }
    return;
  }

  if (!active || share != 0 || failed || *stop) return;
  if (sg.whole) {
    // a row that saw nothing has a sum of 0: its output is 0
    const float i_lo = l_lo == 0.f ? 0.f : 1.f / l_lo, i_hi = l_hi == 0.f ? 0.f : 1.f / l_hi;
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(r.out);
    uint32_t* o_lo = reinterpret_cast<uint32_t*>(out + (u.row0 + j_lo) * r.out_stride + static_cast<int64_t>(h_lo) * H);
    uint32_t* o_hi = reinterpret_cast<uint32_t*>(out + (u.row0 + j_hi) * r.out_stride + static_cast<int64_t>(h_hi) * H);
#pragma unroll
    for (int i = 0; i < DN; ++i) {
      if (v_lo) o_lo[i * 4 + tq] = pack_bf16(o[i][0] * i_lo, o[i][1] * i_lo);
      if (v_hi) o_hi[i * 4 + tq] = pack_bf16(o[i][2] * i_hi, o[i][3] * i_hi);
    }
    if (r.lse && tq == 0) {
      if (v_lo) r.lse[static_cast<int64_t>(u.row0 + j_lo) * r.Hq + h_lo] = l_lo == 0.f ? -INFINITY : (m_lo + log2f(l_lo)) * kLn2;
      if (v_hi) r.lse[static_cast<int64_t>(u.row0 + j_hi) * r.Hq + h_hi] = l_hi == 0.f ? -INFINITY : (m_hi + log2f(l_hi)) * kLn2;
    }
  } else {
    const int64_t row = static_cast<int64_t>(sg.slot) * kUnitRows;
#pragma unroll
    for (int i = 0; i < DN; ++i) {
      if (v_lo) *reinterpret_cast<float2*>(parts.acc + (row + r_lo) * H + i * 8 + 2 * tq) = make_float2(o[i][0], o[i][1]);
      if (v_hi) *reinterpret_cast<float2*>(parts.acc + (row + r_hi) * H + i * 8 + 2 * tq) = make_float2(o[i][2], o[i][3]);
    }
    if (tq == 0) {
      if (v_lo) *reinterpret_cast<float2*>(parts.ml + (row + r_lo) * 2) = make_float2(m_lo, l_lo);
      if (v_hi) *reinterpret_cast<float2*>(parts.ml + (row + r_hi) * 2) = make_float2(m_hi, l_hi);
    }
  }
}

__device__ __forceinline__ UnitRows unit_rows(const PagedCache& c, const PagedRows& r, int list_len, const ReqWork& w, const Segment& sg) {
  constexpr int rows = kUnitRows;
  UnitRows u;
  u.req = sg.req;
  u.row0 = w.v.row0;
  u.m = w.v.m;
  u.group = r.group;
  u.g = sg.g;
  u.first = sg.rb * rows;
  if (list_len > 0) {
    u.j = sg.j;
    u.count = min(rows, u.group - u.first);
    const int x = w.v.n - w.v.m + sg.j, own = quotient(x, c.ps);   // the last chosen block is the token's own
    u.end = (min(list_len, own + 1) - 1) * c.ps + x - own * c.ps + 1;
    u.prefix = u.end;
  } else {
    u.j = -1;
    u.count = min(rows, w.v.m * u.group - u.first);
    u.end = w.v.n;
    u.prefix = w.v.n - w.v.m;
  }
  return u;
}

// 160 threads: warps 0-3 compute, warp 4 brings the tiles in.
template <int H>
__global__ void __launch_bounds__(160, 2) paged_mma_kernel(const PagedCache c, const PagedRows r, const int32_t* list, int list_len,
                                                           const Parts parts, const __grid_constant__ CUtensorMap map_k,
                                                           const __grid_constant__ CUtensorMap map_v) {
  using S = Smem<H>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int stop_word;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* ptr = smem_raw + (base - raw);
  volatile int* stop = &stop_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Ring ring{base, base + S::kOffBar, base + S::kOffBar + 8 * kStages, 0};
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(ring.full + 8 * s, 1);
      mbar_init(ring.empty + 8 * s, 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  __syncthreads();
  pdl_wait();
  const AttentionLine line{c, r, list_len};
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (threadIdx.x == 0) leave_none(parts.desc, blockIdx.x);
  if (share.from >= share.to) return;

  if (warp == 4) {
    const uint64_t policy = policy_evict_first();
    const int cpp = c.ps / 16;                  // 16-key groups of a page
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const UnitRows u = unit_rows(c, r, list_len, w, sg);
      const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
      const int32_t* mine = list_len > 0 ? list + (static_cast<int64_t>(w.v.row0 + sg.j) * c.Hkv + sg.g) * list_len : nullptr;
      const int groups = (u.end + 15) / 16;     // that hold any key
      const bool again = w.n_rb > 1 || list_len > 0;   // others read these keys as well: leave them in L2
      int row = 0;                              // of the group that this lane looks up: the next 32 of them at a time
      for (int t = sg.t0; t < sg.t1; ++t, ++ring.it) {
        const int ahead = (t - sg.t0) & 7;
        if (ahead == 0) {
          const int e = t * 4 + lane;
          row = 0;
          if (e < groups && e < sg.t1 * 4) {
            const int b = e / cpp;
            const int page = checked_page(c, table[mine ? checked_block(c, mine[b]) : b]);
            row = (page * c.Hkv + sg.g) * c.ps + (e - b * cpp) * 16;
          }
        }
        const int st = ring.it % kStages;
        bool ok = true;
        if (lane == 0) {
          ok = !*stop && mbar_wait(ring.empty + 8 * st, ((ring.it / kStages) & 1) ^ 1, stop);
          if (!ok) *stop = 1;
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        const int n_here = max(0, min(4, groups - t * 4));
        if (ok && lane == 0) mbar_expect(ring.full + 8 * st, n_here * 2 * S::kGroup);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int y = __shfl_sync(0xffffffffu, row, ahead * 4 + p) >> (H == 32);
          if (ok && lane == 0 && p < n_here) {
            const uint32_t dst = base + st * S::kStage + p * S::kGroup, bar = ring.full + 8 * st;
            if (again) {
              const uint64_t keep = policy_evict_last();
              tma_load_3d(dst, &map_k, 0, y, 0, bar, keep);
              tma_load_3d(dst + S::kHalf, &map_v, 0, y, 0, bar, keep);
            } else {
              tma_load_3d(dst, &map_k, 0, y, 0, bar, policy);
              tma_load_3d(dst + S::kHalf, &map_v, 0, y, 0, bar, policy);
            }
          }
        }
      }
    });
  } else {
    float* merge = reinterpret_cast<float*>(ptr + S::kOffMerge);
    uint32_t* tree = reinterpret_cast<uint32_t*>(ptr + S::kOffTree);
    int tree_of = -1;
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const UnitRows u = unit_rows(c, r, list_len, w, sg);
      if (r.parents && tree_of != sg.req) {     // what every node sees among the nodes
        tree_of = sg.req;
        asm volatile("bar.sync 2, 128;" ::: "memory");
        if (static_cast<int>(threadIdx.x) < u.m) {
          uint32_t bits[kMaxTreeNodes / 32];
          ancestors_of(r.parents + u.row0, threadIdx.x, bits, c.status);
#pragma unroll
          for (int x = 0; x < kMaxTreeNodes / 32; ++x) tree[threadIdx.x * (kMaxTreeNodes / 32) + x] = bits[x];
        }
        asm volatile("bar.sync 2, 128;" ::: "memory");
      }
      if (u.count <= 16) consume<H, 1>(c, r, u, sg, ring, stop, merge, tree, parts);
      else if (u.count <= 32) consume<H, 2>(c, r, u, sg, ring, stop, merge, tree, parts);
      else consume<H, 4>(c, r, u, sg, ring, stop, merge, tree, parts);
      if (sg.last_block >= 0 && threadIdx.x == 0) leave_cut(parts.desc, blockIdx.x, sg, u.row0, u.m, u.j, u.first, u.count);
    });
  }
  __syncthreads();
  if (*stop) {
    if (threadIdx.x == 0) set_status(c.status, SLED_ERR_DEVICE);
    const long long t0 = clock64();   // copies that were issued may still land: the shared memory stays a little longer
    while (clock64() - t0 < 2000000LL) __nanosleep(1000);
  }
}

// The partial results of the units that were cut.  Block b finishes the one that block b began, a warp per row: the first
// kAtOnce parts of a row and all parts' maxima and sums are under way before any of them is looked at.  Bound by the latency
// of two dependent loads and of its launch: 4.4 us by itself for 8 units of a few parts.
template <typename T, int H>
__global__ void __launch_bounds__(512) paged_merge_kernel(const PagedCache c, const PagedRows r, int unit, const Parts parts) {
  pdl_wait();
  const CutUnit u = cut_unit(parts.desc, blockIdx.x);
  if (u.last_block < 0) return;
  constexpr int D = H / 32, kAtOnce = 8;
  using Words = typename std::conditional<D == 4, float4, typename std::conditional<D == 2, float2, float>::type>::type;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = r.group;
  const int n_parts = u.last_block - static_cast<int>(blockIdx.x) + 1, n_warps = blockDim.x >> 5;
  auto slot = [&](int p) { return static_cast<int64_t>(p == 0 ? u.slot : 2 * (blockIdx.x + p)) * unit; };
  int row = blockIdx.y * n_warps + warp;
  float2 ml;
  float acc[kAtOnce][D];
  auto part = [&](int p, float* to) { *reinterpret_cast<Words*>(to) = *reinterpret_cast<const Words*>(parts.acc + (slot(p) + row) * H + lane * D); };
  auto load = [&] {
    ml = make_float2(-INFINITY, 0.f);
    if (row >= u.count) return;
    if (lane < n_parts) ml = *reinterpret_cast<const float2*>(parts.ml + (slot(lane) + row) * 2);
#pragma unroll
    for (int p = 0; p < kAtOnce; ++p)
      if (p < n_parts) part(p, acc[p]);
  };
  load();
  // Rows of unused nodes are 0, whatever the partial results say: a stretch of keys without nodes does not know of them.
  __shared__ signed char parents[kMaxTreeNodes];
  bool unused = false;
  if (r.parents && u.j < 0) {
    bool any = false;
    for (int i = threadIdx.x; i < u.m; i += blockDim.x) {
      const int p = r.parents[u.row0 + i];
      const bool wrong = p < -1 || p >= i;
      parents[i] = static_cast<signed char>(wrong ? -2 : p);
      any |= wrong;
    }
    unused = __syncthreads_or(any);
  }
  for (; row < u.count; row += gridDim.y * n_warps, load()) {
    float M = ml.x;
    bool nan = ml.y != ml.y;
    for (int p = 32 + lane; p < n_parts; p += 32) {
      const float2 x = *reinterpret_cast<const float2*>(parts.ml + (slot(p) + row) * 2);
      M = fmaxf(M, x.x);
      nan |= x.y != x.y;
    }
    M = warp_max(M);
    nan = __any_sync(0xffffffffu, nan);
    const float ref = M == -INFINITY ? 0.f : M;
    float f = exp2_approx(ml.x - ref), den = f * ml.y, num[D];
#pragma unroll
    for (int e = 0; e < D; ++e) num[e] = 0.f;
#pragma unroll
    for (int p = 0; p < kAtOnce; ++p) {
      const float fp = __shfl_sync(0xffffffffu, f, p);
      if (p < n_parts) {
#pragma unroll
        for (int e = 0; e < D; ++e) num[e] = fmaf(fp, acc[p][e], num[e]);
      }
    }
    for (int p0 = 0; p0 < n_parts; p0 += 32) {
      if (p0 > 0) {
        f = 0.f;
        if (p0 + lane < n_parts) {
          const float2 x = *reinterpret_cast<const float2*>(parts.ml + (slot(p0 + lane) + row) * 2);
          f = exp2_approx(x.x - ref);
          den = fmaf(f, x.y, den);
        }
      }
      const int here = min(32, n_parts - p0);
#pragma unroll 8
      for (int p = p0 > 0 ? 0 : kAtOnce; p < here; ++p) {
        const float fp = __shfl_sync(0xffffffffu, f, p);
        float x[D];
        part(p0 + p, x);
#pragma unroll
        for (int e = 0; e < D; ++e) num[e] = fmaf(fp, x[e], num[e]);
      }
    }
    den = warp_sum(den);
    bool none = M == -INFINITY && !nan;
    if (unused) {
      int a = (u.first + row) / group;
      while (a >= 0) a = parents[a];
      none |= a == -2;
    }
    const float inv = none ? 0.f : 1.f / den;
    const int of = (u.first + row) / group, t = u.row0 + (u.j >= 0 ? u.j : of), head = u.g * group + (u.first + row) - of * group;
    T* out = reinterpret_cast<T*>(r.out) + t * r.out_stride + static_cast<int64_t>(head) * H + lane * D;
    if constexpr (sizeof(T) == 2 && D == 1) {
      *out = __float2bfloat16_rn(none ? 0.f : num[0] * inv);
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < D / 2; ++e) reinterpret_cast<uint32_t*>(out)[e] = none ? 0u : pack_bf16(num[2 * e] * inv, num[2 * e + 1] * inv);
    } else {
#pragma unroll
      for (int e = 0; e < D; ++e) out[e] = none ? 0.f : num[e] * inv;
    }
    if (r.lse && lane == 0) r.lse[static_cast<int64_t>(t) * r.Hq + head] = none ? -INFINITY : (M + log2f(den)) * kLn2;
  }
}

}  // namespace

int paged_device(int* sms) {   // asked for once per device
  static std::atomic<int> known[kMaxDevices] = {};   // by any host thread
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return -1;
  int n = known[dev].load(std::memory_order_relaxed);
  if (!n) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return -1;
    known[dev].store(n, std::memory_order_relaxed);
  }
  *sms = n;
  return dev;
}

namespace {

template <int H>
int launch_h(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* scores, char* ws, cudaStream_t s) {
  static std::atomic<bool> configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!allow_shared(paged_mma_kernel<H>, Smem<H>::kTotal, dev, configured)) return -1;
  CUtensorMap map_k, map_v;
  const long long rows = static_cast<long long>(c.n_pages) * c.Hkv * c.ps;
  constexpr int kPerRow = H == 32 ? 2 : 1;      // keys of a row of the map
  if (tma_map_bf16_row_groups(&map_k, c.k, rows / kPerRow, H * kPerRow, 16 / kPerRow) ||
      tma_map_bf16_row_groups(&map_v, c.v, rows / kPerRow, H * kPerRow, 16 / kPerRow))
    return -1;
  const int blocks = min(2 * sms, kMaxPagedBlocks);
  Parts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + 2LL * kMaxPagedBlocks * kUnitRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + 2LL * kMaxPagedBlocks * kUnitRows * 2);
  parts.scores = scores;
  parts.keys = static_cast<int64_t>(c.table_cols) * c.ps;
  SLED_LAUNCH_PDL(paged_mma_kernel<H>, dim3(blocks), dim3(160), Smem<H>::kTotal, s, c, r, list, list_len, parts, map_k, map_v);
  if (cudaGetLastError() != cudaSuccess) return -1;
  const int n = launch_paged_merge(c, r, kUnitRows, blocks, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int launch_paged_merge(const PagedCache& c, const PagedRows& r, int unit_rows, int blocks, float* acc, float* ml, int4* desc, cudaStream_t s) {
  const Parts parts{acc, ml, desc, nullptr, 0};
  const dim3 grid(blocks, unit_rows > kUnitRows ? 4 : unit_rows < kUnitRows ? 1 : 2);
  const int threads = min(512, 32 * unit_rows);   // a warp for each of a small unit's rows
#define SLED_MERGE(T, H) SLED_LAUNCH_PDL((paged_merge_kernel<T, H>), grid, dim3(threads), 0, s, c, r, unit_rows, parts)
  if (c.dtype == BF16 && c.h == 128) SLED_MERGE(__nv_bfloat16, 128);
  else if (c.dtype == BF16 && c.h == 64) SLED_MERGE(__nv_bfloat16, 64);
  else if (c.dtype == BF16) SLED_MERGE(__nv_bfloat16, 32);
  else if (c.h == 128) SLED_MERGE(float, 128);
  else if (c.h == 64) SLED_MERGE(float, 64);
  else SLED_MERGE(float, 32);
#undef SLED_MERGE
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

int64_t paged_mma_workspace(int h) {
  return 2LL * kMaxPagedBlocks * kUnitRows * (h + 2) * 4 + kMaxPagedBlocks * 32LL;
}

int launch_paged_mma(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* scores, char* ws, cudaStream_t s) {
  if (c.h == 128) return launch_h<128>(c, r, list, list_len, scores, ws, s);
  return c.h == 64 ? launch_h<64>(c, r, list, list_len, scores, ws, s) : launch_h<32>(c, r, list, list_len, scores, ws, s);
}

}  // namespace sled
