// Attention over a paged cache of e4m3 codes with a scale for every block of 16 slots and KV head, on the warp-level tensor cores.
//
// For a query row r (token, head) and the keys x it sees, of block b: s_x = scale ks_b (q . c_x), o = sum p_x vs_b d_x over the
// codes c of K and d of V, p the softmax of s.  One pass over the keys with the running maximum m of s and sum l of 2^(s - m);
// scales stay out of the products' operands: ks multiplies a score, vs goes into the numerators.
//
// Codes become fp16 in registers, which is exact; queries do too, times a power of two per row that brings the row's largest
// element to 2^14, so that nothing of them is lost either.  The numerators of a row meet V as fp16(2^15 2^(s_x - u) vs_b) with a
// reference of their own, u = max (s_x + log2 vs_b) so far: they are as large as fp16 allows whatever the blocks' scales are,
// 11 bits of each down to 2^-29 of the largest.  u is joined with m at the end of a unit.
//
// A unit is the query rows that share a KV head (up to 64 of them): the M side of m16n8k16 products, so a cached key is read
// once for all.  With up to 16 (32) rows the four computing warps split every 64-key tile four (two) ways - 16 keys, one block of
// scales, each - and merge at the end of the unit; with more, every warp has 16 rows of its own.  The order of the dimensions in
// the first product is free as long as both operands agree: a lane takes H / 4 consecutive bytes of a key, whole 16-byte
// loads, and the queries are laid out to match.  V goes through transposing matrix loads of 16-bit units - two dimensions of
// a key -, a byte permutation parts them into the even and the odd dimensions of two keys.  A fifth warp brings the tiles in by
// TMA and their scales with them, looked up a round ahead.  Work is handed out as paged_schedule.cuh says.
#include "gemm_tc.h"
#include "kernels.h"
#include "paged_scaled.cuh"

namespace sled {

namespace {


// A stage holds K, then V: four groups of 16 keys, rows of 128 bytes (of one, two or four keys); the 16-byte chunk c of a row
// lies at c ^ (row & 7).
template <int H>
struct Smem {
  static constexpr int kKeysPerRow = 128 / H;
  static constexpr int kCopy = 16 * H;                              // bytes of 16 keys
  static constexpr int kGroup = kCopy < 1024 ? 1024 : kCopy;        // whole rounds of the swizzle
  static constexpr int kHalf = 4 * kGroup;
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kStages = H == 128 ? 6 : 8;
  static constexpr int kMergePitch = 48;                            // 32 dimensions of a row; four words of two rows meet 32 banks
  static constexpr int kMerge = 64 * (kMergePitch + 2) * 4;
  static constexpr int kOffMerge = kStages * kStage;
  static constexpr int kOffTree = kOffMerge + kMerge;
  static constexpr int kOffScale = kOffTree + kMaxTreeNodes * (kMaxTreeNodes / 32) * 4;     // [stage][K, V][4]
  static constexpr int kOffBar = kOffScale + kStages * 32;
  static constexpr int kTotal = kOffBar + 16 * kStages + 1024;      // alignment slack
};
static_assert(Smem<128>::kTotal + 1024 + 256 <= 228 * 1024 / 2, "two blocks on an SM");

// shared memory address of 16-byte chunk c of a key of the tile
template <int H>
__device__ __forceinline__ uint32_t at(uint32_t base, int key, int c) {
  constexpr int P = Smem<H>::kKeysPerRow;
  const int row = (key & 15) / P;
  return base + (key >> 4) * Smem<H>::kGroup + row * 128 + (((key % P * (H / 16) + c) ^ (row & 7)) << 4);
}

struct Ring {
  uint32_t base, full, empty;
  int it;                 // tiles so far
};

struct UnitRows {
  int req, row0, m;       // the request's rows
  int group, g;
  int first, count;       // rows of the unit's block: first .. first + count - 1
  int prefix, end;        // positions below `prefix` are seen by everybody; there are `end` of them
  __device__ __forceinline__ int token(int r) const { return quotient(first + r, group); }
  __device__ __forceinline__ int head(int r) const { return g * group + first + r - quotient(first + r, group) * group; }
};


// One stretch of a unit: MT warps cover the rows, 4 / MT the keys of a tile.
template <int H, int MT>
__device__ __forceinline__ void consume(const PagedRows& r, const UnitRows& u, const Segment& sg, Ring& ring, volatile int* stop,
                                        const float* scales, float* merge, const uint32_t* tree, const ScaledParts& parts) {
  using S = Smem<H>;
  constexpr int KS = H / 16, DC = H / 16, NT = 2 * MT;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, tq = lane & 3;
  const int mt = warp % MT, share = warp / MT, key_off = share * 16 * MT;
  const int r_lo = mt * 16 + gq, r_hi = r_lo + 8;
  const bool active = mt * 16 < u.count, v_lo = r_lo < u.count, v_hi = r_hi < u.count;
  const int j_lo = v_lo ? u.token(r_lo) : 0, j_hi = v_hi ? u.token(r_hi) : 0;
  const int h_lo = v_lo ? u.head(r_lo) : 0, h_hi = v_hi ? u.head(r_hi) : 0;

  uint32_t q_lo[H / 8], q_hi[H / 8];      // of product ks: words 2 ks and 2 ks + 1
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(r.q) + tq * (H / 4);
  const float f_lo = query_row<H>(q + (u.row0 + j_lo) * r.q_stride + static_cast<int64_t>(h_lo) * H, v_lo, q_lo) * (r.scale * kLog2e);
  const float f_hi = query_row<H>(q + (u.row0 + j_hi) * r.q_stride + static_cast<int64_t>(h_hi) * H, v_hi, q_hi) * (r.scale * kLog2e);
  float o[2 * DC][4];       // [2 c]: dimensions 16 c + 4 tq + {0, 2} of both rows, [2 c + 1]: + {1, 3}
#pragma unroll
  for (int i = 0; i < 2 * DC; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  RowState lo, hi;
  bool failed = false;

  for (int tile = sg.t0; tile < sg.t1; ++tile, ++ring.it) {
    const int st = ring.it % S::kStages;
    if (*stop || !mbar_wait(ring.full + 8 * st, (ring.it / S::kStages) & 1, stop)) { *stop = 1; failed = true; break; }
    const int k0 = tile * kTile + key_off;    // position of this warp's first key
    if (active && k0 < u.end) {
      const uint32_t kb = ring.base + st * S::kStage, vb = kb + S::kHalf;
      float ks[MT], vs[MT], lv = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < MT; ++kt) {
        ks[kt] = scales[st * 8 + key_off / 16 + kt];
        vs[kt] = scales[st * 8 + 4 + key_off / 16 + kt];
        lv = fmaxf(lv, __log2f(fabsf(vs[kt])));
      }
      float sc[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
        uint32_t w[H / 16];
        const int key = key_off + nt * 8 + gq;
        if constexpr (H == 32) {
          asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at<H>(kb, key, tq >> 1) + (tq & 1) * 8));
        } else {
#pragma unroll
          for (int i = 0; i < H / 64; ++i)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                         : "r"(at<H>(kb, key, tq * (H / 64) + i)));
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const uint32_t a[4] = {q_lo[2 * s], q_hi[2 * s], q_lo[2 * s + 1], q_hi[2 * s + 1]};
          mma_half(sc[nt], a, half2_of(w[s]), half2_of_upper(w[s]));
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float x = f_lo * ks[nt >> 1], y = f_hi * ks[nt >> 1];
        sc[nt][0] *= x;
        sc[nt][1] *= x;
        sc[nt][2] *= y;
        sc[nt][3] *= y;
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
              if (r.parents) seen = (tree[j * (kMaxTreeNodes / 32) + (a >> 5)] >> (a & 31)) & 1u;
              else seen = a <= j;
            }
            if (!seen) sc[nt][e] = -INFINITY;
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
      const float al_lo = lo.take(mx_lo, lv), al_hi = hi.take(mx_hi, lv);
      if (__any_sync(0xffffffffu, al_lo != 1.f || al_hi != 1.f)) {
#pragma unroll
        for (int i = 0; i < 2 * DC; ++i) { o[i][0] *= al_lo; o[i][1] *= al_lo; o[i][2] *= al_hi; o[i][3] *= al_hi; }
      }
      const float unit_lo = lo.unit_weight(), unit_hi = hi.unit_weight();
      uint32_t pf[MT][4];   // the numerators as A operand; their sum is taken before the rounding
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float p0 = exp2_approx(sc[nt][0] - lo.ref), p1 = exp2_approx(sc[nt][1] - lo.ref);
        float p2 = exp2_approx(sc[nt][2] - hi.ref), p3 = exp2_approx(sc[nt][3] - hi.ref);
        lo.l += p0 + p1;
        hi.l += p2 + p3;
        const float w_lo = lo.scaled(unit_lo, vs[nt >> 1]), w_hi = hi.scaled(unit_hi, vs[nt >> 1]);
        if (masked) {       // a scale that is no number reaches the rows that see its block, not the others
          p0 = sc[nt][0] == -INFINITY ? 0.f : p0 * w_lo;
          p1 = sc[nt][1] == -INFINITY ? 0.f : p1 * w_lo;
          p2 = sc[nt][2] == -INFINITY ? 0.f : p2 * w_hi;
          p3 = sc[nt][3] == -INFINITY ? 0.f : p3 * w_hi;
        } else {
          p0 *= w_lo;
          p1 *= w_lo;
          p2 *= w_hi;
          p3 *= w_hi;
        }
        pf[nt >> 1][(nt & 1) * 2] = pack_half(p0, p1);
        pf[nt >> 1][(nt & 1) * 2 + 1] = pack_half(p2, p3);
      }
      // V: 16 keys x 32 dimensions at a time; word: two dimensions of two keys -> the first of both, the second of both
      auto load_v = [&](int kt, int d, uint32_t b[4]) {
        ldmatrix_x4_trans(at<H>(vb, key_off + kt * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), d * 2 + (lane >> 4)), b[0], b[1], b[2], b[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = __byte_perm(b[i], 0, 0x3120);
      };
      if (!masked) {
#pragma unroll
        for (int kt = 0; kt < MT; ++kt)
#pragma unroll
          for (int d = 0; d < H / 32; ++d) {
            uint32_t b[4];
            load_v(kt, d, b);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              mma_half(o[4 * d + 2 * c], pf[kt], half2_of(b[2 * c]), half2_of(b[2 * c + 1]));
              mma_half(o[4 * d + 2 * c + 1], pf[kt], half2_of_upper(b[2 * c]), half2_of_upper(b[2 * c + 1]));
            }
          }
      } else {
        // A numerator of 0 does not silence a code that is no number.  Values of keys that do not exist are taken as 0; of the
        // others those that are no numbers are left out of the product and given afterwards to the rows that see them.
        bool odd = false;
#pragma unroll
        for (int kt = 0; kt < MT; ++kt) {
          const int x = k0 + kt * 16 + 2 * tq;
          const uint32_t there[2] = {(x < u.end ? 0xffffu : 0u) | (x + 1 < u.end ? 0xffff0000u : 0u),
                                     (x + 8 < u.end ? 0xffffu : 0u) | (x + 9 < u.end ? 0xffff0000u : 0u)};
#pragma unroll
          for (int d = 0; d < H / 32; ++d) {
            uint32_t b[4];
            load_v(kt, d, b);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int z = 0; z < 2; ++z) {
                uint32_t y[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  y[e] = (z ? half2_of_upper(b[2 * c + e]) : half2_of(b[2 * c + e])) & there[e];
                  const uint32_t off = ((y[e] & 0x7c00u) == 0x7c00u ? 0xffffu : 0u) | ((y[e] & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u);
                  odd |= off != 0;
                  y[e] &= ~off;
                }
                mma_half(o[4 * d + 2 * c + z], pf[kt], y[0], y[1]);
              }
          }
        }
        if (__any_sync(0xffffffffu, odd)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
              const int src = (lane & ~3) | (e >> 1);
              const bool see_lo = __shfl_sync(0xffffffffu, e & 1 ? sc[nt][1] : sc[nt][0], src) != -INFINITY;
              const bool see_hi = __shfl_sync(0xffffffffu, e & 1 ? sc[nt][3] : sc[nt][2], src) != -INFINITY;
              const int key = key_off + nt * 8 + e;
              if (tile * kTile + key >= u.end) continue;
#pragma unroll
              for (int c = 0; c < DC; ++c) {
                uint32_t w;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at<H>(vb, key, c) + tq * 4));
#pragma unroll
                for (int z = 0; z < 4; ++z)
                  if ((w >> 8 * z & 0x7fu) == 0x7fu) {
                    if (see_lo) o[2 * c + (z & 1)][z >> 1] = NAN;
                    if (see_hi) o[2 * c + (z & 1)][2 + (z >> 1)] = NAN;
                  }
              }
            }
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(ring.empty + 8 * st);
  }

  float l_lo = lo.l, l_hi = hi.l, m_lo = lo.m, m_hi = hi.m;
  l_lo += __shfl_xor_sync(0xffffffffu, l_lo, 1);
  l_lo += __shfl_xor_sync(0xffffffffu, l_lo, 2);
  l_hi += __shfl_xor_sync(0xffffffffu, l_hi, 1);
  l_hi += __shfl_xor_sync(0xffffffffu, l_hi, 2);
  const float e_lo = lo.rest(), e_hi = hi.rest();
#pragma unroll
  for (int i = 0; i < 2 * DC; ++i) { o[i][0] *= e_lo; o[i][1] *= e_lo; o[i][2] *= e_hi; o[i][3] *= e_hi; }
  if (r.parents) {   // an unused node - it does not even see itself - sees nothing
    const uint4 b_lo = *reinterpret_cast<const uint4*>(tree + j_lo * (kMaxTreeNodes / 32));
    const uint4 b_hi = *reinterpret_cast<const uint4*>(tree + j_hi * (kMaxTreeNodes / 32));
    if (!(b_lo.x | b_lo.y | b_lo.z | b_lo.w)) {
      m_lo = -INFINITY;
      l_lo = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * DC; ++i) o[i][0] = o[i][1] = 0.f;
    }
    if (!(b_hi.x | b_hi.y | b_hi.z | b_hi.w)) {
      m_hi = -INFINITY;
      l_hi = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * DC; ++i) o[i][2] = o[i][3] = 0.f;
    }
  }
  auto four_lo = [&](int c, float f) { return make_float4(o[2 * c][0] * f, o[2 * c + 1][0] * f, o[2 * c][1] * f, o[2 * c + 1][1] * f); };
  auto four_hi = [&](int c, float f) { return make_float4(o[2 * c][2] * f, o[2 * c + 1][2] * f, o[2 * c][3] * f, o[2 * c + 1][3] * f); };

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
          for (int c = 0; c < 2; ++c) {
            *reinterpret_cast<float4*>(merge + mine * kPitch + c * 16 + 4 * tq) = four_lo(2 * z + c, 1.f);
            *reinterpret_cast<float4*>(merge + (mine + 8) * kPitch + c * 16 + 4 * tq) = four_hi(2 * z + c, 1.f);
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
    uint32_t* to_lo = reinterpret_cast<uint32_t*>(out + (u.row0 + j_lo) * r.out_stride + static_cast<int64_t>(h_lo) * H) + 2 * tq;
    uint32_t* to_hi = reinterpret_cast<uint32_t*>(out + (u.row0 + j_hi) * r.out_stride + static_cast<int64_t>(h_hi) * H) + 2 * tq;
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      const float4 x = four_lo(c, i_lo), y = four_hi(c, i_hi);
      if (v_lo) { to_lo[8 * c] = pack_bf16(x.x, x.y); to_lo[8 * c + 1] = pack_bf16(x.z, x.w); }
      if (v_hi) { to_hi[8 * c] = pack_bf16(y.x, y.y); to_hi[8 * c + 1] = pack_bf16(y.z, y.w); }
    }
    if (r.lse && tq == 0) {
      if (v_lo) r.lse[static_cast<int64_t>(u.row0 + j_lo) * r.Hq + h_lo] = l_lo == 0.f ? -INFINITY : (m_lo + log2f(l_lo)) * kLn2;
      if (v_hi) r.lse[static_cast<int64_t>(u.row0 + j_hi) * r.Hq + h_hi] = l_hi == 0.f ? -INFINITY : (m_hi + log2f(l_hi)) * kLn2;
    }
  } else {
    const int64_t row = static_cast<int64_t>(sg.slot) * kUnitRows;
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      if (v_lo) *reinterpret_cast<float4*>(parts.acc + (row + r_lo) * H + c * 16 + 4 * tq) = four_lo(c, 1.f);
      if (v_hi) *reinterpret_cast<float4*>(parts.acc + (row + r_hi) * H + c * 16 + 4 * tq) = four_hi(c, 1.f);
    }
    if (tq == 0) {
      if (v_lo) *reinterpret_cast<float2*>(parts.ml + (row + r_lo) * 2) = make_float2(m_lo, l_lo);
      if (v_hi) *reinterpret_cast<float2*>(parts.ml + (row + r_hi) * 2) = make_float2(m_hi, l_hi);
    }
  }
}

__device__ __forceinline__ UnitRows unit_rows(const PagedRows& r, const ReqWork& w, const Segment& sg) {
  UnitRows u;
  u.req = sg.req;
  u.row0 = w.v.row0;
  u.m = w.v.m;
  u.group = r.group;
  u.g = sg.g;
  u.first = sg.rb * kUnitRows;
  u.count = min(kUnitRows, w.v.m * u.group - u.first);
  u.end = w.v.n;
  u.prefix = w.v.n - w.v.m;
  return u;
}

// 160 threads: warps 0-3 compute, warp 4 brings the tiles in.
template <int H>
__global__ void __launch_bounds__(160, 2) paged_scaled_kernel(const PagedCache c, const CacheScales sc, const PagedRows r, const ScaledParts parts,
                                                              const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = Smem<H>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int stop_word;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* ptr = smem_raw + (base - raw);
  volatile int* stop = &stop_word;
  float* scales = reinterpret_cast<float*>(ptr + S::kOffScale);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Ring ring{base, base + S::kOffBar, base + S::kOffBar + 8 * S::kStages, 0};
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = 0;
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(ring.full + 8 * s, 1);
      mbar_init(ring.empty + 8 * s, 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  __syncthreads();
  pdl_wait();
  const AttentionLine line{c, r, 0};
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (threadIdx.x == 0) leave_none(parts.desc, blockIdx.x);
  if (share.from >= share.to) return;

  if (warp == 4) {
    const uint64_t first = policy_evict_first(), last = policy_evict_last();
    const int cpp = c.ps / 16;                  // 16-key groups of a page
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const UnitRows u = unit_rows(r, w, sg);
      const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
      const int groups = min((u.end + 15) / 16, sg.t1 * 4);     // that hold any key, up to the end of the segment
      const uint64_t policy = w.n_rb > 1 ? last : first;        // others read these keys as well: leave them in L2
      // a lane looks after one of 32 groups (eight tiles): its place and its scales; those of the next round are under way
      // while this one's tiles are copied
      auto page_of = [&](int e) { return e < groups ? table[quotient(e, cpp)] : -1; };
      int block = 0, page_next = page_of(sg.t0 * 4 + lane);
      float ks = 1.f, vs = 1.f;
      auto look_up = [&](int e, int& b, float& k, float& v) {   // of the group whose page has arrived
        b = 0;
        k = v = 1.f;
        if (e < groups) {
          const int of = quotient(e, cpp);
          b = (checked_page(c, page_next) * c.Hkv + sg.g) * cpp + (e - of * cpp);
          k = sc.k[b];
          v = sc.v[b];
        }
      };
      int block_next;
      float ks_next, vs_next;
      look_up(sg.t0 * 4 + lane, block_next, ks_next, vs_next);
      page_next = page_of(sg.t0 * 4 + 32 + lane);
      for (int t = sg.t0; t < sg.t1; ++t, ++ring.it) {
        const int ahead = (t - sg.t0) & 7;
        if (ahead == 0) {
          block = block_next;
          ks = ks_next;
          vs = vs_next;
          look_up(t * 4 + 32 + lane, block_next, ks_next, vs_next);
          page_next = page_of(t * 4 + 64 + lane);
        }
        const int st = ring.it % S::kStages;
        bool ok = true;
        if (lane == 0) {
          ok = !*stop && mbar_wait(ring.empty + 8 * st, ((ring.it / S::kStages) & 1) ^ 1, stop);
          if (!ok) *stop = 1;
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        __syncwarp();
        const int n_here = max(0, min(4, groups - t * 4));
        const bool mine = lane >> 2 == ahead;
        if (ok && mine) {
          scales[st * 8 + (lane & 3)] = ks;
          scales[st * 8 + 4 + (lane & 3)] = vs;
        }
        __syncwarp();
        if (ok && lane == 0) mbar_expect(ring.full + 8 * st, n_here * 2 * S::kCopy);
        __syncwarp();
        if (ok && mine && (lane & 3) < n_here) {
          const uint32_t dst = base + st * S::kStage + (lane & 3) * S::kGroup, bar = ring.full + 8 * st;
          const int y = block * (16 / S::kKeysPerRow);
          tma_load_3d(dst, &map_k, 0, y, 0, bar, policy);
          tma_load_3d(dst + S::kHalf, &map_v, 0, y, 0, bar, policy);
        }
      }
    });
  } else {
    float* merge = reinterpret_cast<float*>(ptr + S::kOffMerge);
    uint32_t* tree = reinterpret_cast<uint32_t*>(ptr + S::kOffTree);
    int tree_of = -1;
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const UnitRows u = unit_rows(r, w, sg);
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
      if (u.count <= 16) consume<H, 1>(r, u, sg, ring, stop, scales, merge, tree, parts);
      else if (u.count <= 32) consume<H, 2>(r, u, sg, ring, stop, scales, merge, tree, parts);
      else consume<H, 4>(r, u, sg, ring, stop, scales, merge, tree, parts);
      if (sg.last_block >= 0 && threadIdx.x == 0) leave_cut(parts.desc, blockIdx.x, sg, u.row0, u.m, -1, u.first, u.count);
    });
  }
  __syncthreads();
  if (*stop) {
    if (threadIdx.x == 0) set_status(c.status, SLED_ERR_DEVICE);
    const long long t0 = clock64();   // copies that were issued may still land: the shared memory stays a little longer
    while (clock64() - t0 < 2000000LL) __nanosleep(1000);
  }
}

template <int H>
int launch_h(const PagedCache& c, const CacheScales& sc, const PagedRows& r, char* ws, cudaStream_t s) {
  static std::atomic<bool> configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!allow_shared(paged_scaled_kernel<H>, Smem<H>::kTotal, dev, configured)) return -1;
  CUtensorMap map_k, map_v;     // rows of 128 bytes, as 64 units of 16 bits
  constexpr int P = Smem<H>::kKeysPerRow;
  const long long rows = static_cast<long long>(c.n_pages) * c.Hkv * c.ps / P;
  if (tma_map_bf16_row_groups(&map_k, c.k, rows, 64, 16 / P) || tma_map_bf16_row_groups(&map_v, c.v, rows, 64, 16 / P)) return -1;
  const int blocks = min(2 * sms, kMaxPagedBlocks);
  ScaledParts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + 2LL * kMaxPagedBlocks * kUnitRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + 2LL * kMaxPagedBlocks * kUnitRows * 2);
  SLED_LAUNCH_PDL(paged_scaled_kernel<H>, dim3(blocks), dim3(160), Smem<H>::kTotal, s, c, sc, r, parts, map_k, map_v);
  if (cudaGetLastError() != cudaSuccess) return -1;
  PagedCache of = c;            // the merge goes by the results' type
  of.dtype = BF16;
  const int n = launch_paged_merge(of, r, kUnitRows, blocks, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int64_t paged_scaled_workspace(int h) {
  return max(max(paged_mma_workspace(h), scaled_few_workspace(h)), h >= 64 ? paged_tc_workspace(h) : 0);
}

int launch_paged_scaled(const PagedCache& c, const CacheScales& sc, const PagedRows& r, char* ws, cudaStream_t s) {
  // by the rows per request and KV head, on average
  const int64_t rows = static_cast<int64_t>(r.T) * r.group;
  if (rows <= 8LL * c.n_reqs) return launch_scaled_few(c, sc, r, 1, ws, s);
  if (c.h >= 64 && rows > 32LL * c.n_reqs) return launch_scaled_tc(c, sc, r, ws, s);
  if (c.h == 128) return launch_h<128>(c, sc, r, ws, s);
  return c.h == 64 ? launch_h<64>(c, sc, r, ws, s) : launch_h<32>(c, sc, r, ws, s);
}

}  // namespace sled
