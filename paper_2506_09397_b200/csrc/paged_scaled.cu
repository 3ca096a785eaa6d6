// Attention over a paged cache of e4m3 codes with a scale for every block of 16 slots and KV head, on the warp-level tensor cores:
// decoding and drafts, and every batch of head_dim 32.
//
// For a query row r (token, head) and the keys x it sees, of block b: s_x = scale ks_b (q . c_x), o = sum p_x vs_b d_x over the
// codes c of K and d of V, p the softmax of s.  One pass over the keys with the running maximum m of s and sum l of 2^(s - m);
// scales stay out of the products' operands: ks multiplies a score, vs goes into the numerators.
//
// Codes become fp16 in registers, which is exact; queries do too, times a power of two per row that brings the row's largest
// element to 2^14 .. 2^15: of them is lost what lies below 2^-39 of the largest, all of it of elements below 2^-31 of it.  The numerators of a row meet V as fp16(2^7 2^(s_x - u) vs_b) with a
// reference of their own, u = max (s_x + log2 vs_b) so far, or less by up to 8: the largest is 2^7 to 2^15 whatever the blocks'
// scales are, and what is lost of another is 2^-11 of itself, or 2^-32 of the largest where that is more.  u is joined with m at
// the end of a unit.
//
// The keys are the M side of m16n8k16 products and the rows the N side, so that eight rows cost half of what sixteen do -
// products, exponentials, registers:
//     S^T (16 keys x 8 rows) = C Q^T,    O^T (16 dimensions x 8 rows) += D^T P^T
// The order of the dimensions in the first product is free as long as both operands agree: a lane takes H / 4 consecutive bytes of
// a key, whole 16-byte loads, and the queries are laid out to match.  D^T comes from transposing matrix loads of 16-bit units (two
// dimensions of a key; a byte permutation parts them, the even and the odd dimensions become the two halves of the M side), P^T
// by a transposition in registers.
//
// A unit is the rows that share a KV head, up to 8 (kGroups 1) or 32 of them.  Its keys come in stages of 32, each read by one
// warp, or by two that have 16 rows each where the unit has more than 16; the four computing warps take stages in turn, know
// nothing of each other until the end of the unit, and merge there.  A fifth warp (and a sixth) brings the stages in by TMA, their
// scales with them, looked up a round ahead.  Work is handed out as paged_schedule.cuh says.
//
// Bound by the bytes of long caches - one token, 8 KV heads of 128: 4 x 131072 keys 172 us (6.2 TB/s), 32 x 8192 93 us (5.8),
// 32 of 128 .. 16384 45 us; 16 rows: 4 x 131072 173 us (6.2) -, between 17 and 32 rows by conversions, products and exponentials
// of two warps a stage (20 rows, 4 x 131072: 298 us), and by latency where there is little to read (one context of 64 keys 10.9 us,
// of which the merge's launch is 3).
#include "gemm_tc.h"
#include "kernels.h"
#include "paged_scaled.cuh"

namespace sled {

namespace {

constexpr int kWarps = 4;
constexpr int kStageKeys = 32;

// A stage holds K, then V: two groups of 16 keys, rows of 128 bytes (of one, two or four keys); the 16-byte chunk c of a row lies
// at c ^ (row & 7).
template <int H, int kGroups>
struct Few {
  static constexpr int kHalves = kGroups;                           // sixteen rows of a unit, or its eight
  static constexpr int kWarpRows = 8 * kGroups, kRows = kHalves * kWarpRows;
  static constexpr int kReaders = kHalves;                          // warps that may read a stage
  static constexpr int kKeysPerRow = 128 / H;
  static constexpr int kCopy = 16 * H;                              // bytes of 16 keys
  static constexpr int kGroup = kCopy < 1024 ? 1024 : kCopy;        // whole rounds of the swizzle
  static constexpr int kHalf = 2 * kGroup;
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kStages = H == 128 ? 8 : 12;
  static constexpr int kBlocks = kGroups == 1 ? 3 : 2;              // on an SM
  static constexpr int kProducers = kGroups;                        // warps that bring stages in (a third block leaves no registers for two)
  static constexpr int kThreads = 32 * (kWarps + kProducers);
  static constexpr int kDims = 32;                                  // of a round of the merge
  static constexpr int kPitch = kDims + 4;                          // four rows two apart meet 32 banks
  static constexpr int kOffQ = kStages * kStage;                    // [8 rows][two products][lane] 16 bytes
  static constexpr int kOffMerge = kOffQ + kRows / 8 * (H / 32) * 512;
  static constexpr int kOffMl = kOffMerge + kWarps * kWarpRows * kPitch * 4;
  static constexpr int kOffRow = kOffMl + kWarps * kWarpRows * 8;   // of a row: what turns products into scores, its node
  static constexpr int kOffTree = kOffRow + kRows * 8;
  static constexpr int kOffScale = kOffTree + kMaxTreeNodes * (kMaxTreeNodes / 32) * 4;     // [stage][K, V][2]
  static constexpr int kOffUnit = kOffScale + kStages * 16;         // two stretches
  static constexpr int kOffBar = kOffUnit + 2 * 96;
  static constexpr int kTotal = kOffBar + 16 * kStages + 32 + 1024; // alignment slack
};
// A place of the ring is always the same warp's within a stretch of a unit, which has then seen all its phases: the parity that it
// waits for cannot be that of the phase before the last.  (Copies need not arrive in the order in which they were issued.)
static_assert(Few<128, 1>::kStages % kWarps == 0 && Few<64, 1>::kStages % kWarps == 0, "whole rounds of the warps, and of two producers");
static_assert(3 * (Few<128, 1>::kTotal + 1024 + 512) <= 228 * 1024 && 2 * (Few<128, 2>::kTotal + 1024 + 512) <= 228 * 1024, "blocks of an SM");

template <int H, int G>
__device__ __forceinline__ uint32_t at(uint32_t base, int key, int c) {
  constexpr int P = Few<H, G>::kKeysPerRow;
  const int row = (key & 15) / P;
  return base + (key >> 4) * Few<H, G>::kGroup + row * 128 + (((key % P * (H / 16) + c) ^ (row & 7)) << 4);
}

// What a tile costs whose rows go to two warps (of others: 16), and a unit of 8 or 32 rows beside its tiles.  8 KV heads of 128, us:
// 32 contexts of 128 .. 16384 keys, 16 rows, with 16, 32, 64, 128, 192 for a unit 105, 93, 71, 58, 54, 4 rows (8 to a unit) with 16, 32,
// 64, 96, 128 57, 49.4, 42.0, 41.6, 41.8; 8 x 30000 keys of 12 to 20 rows with 16, 22, 26, 30, 34, 40 for a tile of two warps 147, 124,
// 114, 109, 115, 125.
constexpr int kSplitTile = 30, kUnit8 = 96, kUnit32 = 192;
// The line of tiles with units of up to `rows` rows.
template <int kRows>
struct FewLine : AttentionLine {
  static constexpr int kUnit = kRows == 8 ? kUnit8 : kUnit32, kSlack = kUnit;
  __device__ __forceinline__ FewLine(const PagedCache& c, const PagedRows& r) : AttentionLine{c, r, 0, kRows, kTile} {}
  __device__ __forceinline__ int min_share() const { return kMinMmaShare; }
  __device__ __forceinline__ ReqWork operator()(int i) const {
    ReqWork w = AttentionLine::operator()(i);
    if (w.units > 0) {
      const int tile = min(w.v.m * r.group, kRows) > 16 ? kSplitTile : 16;
      w.weight = unit_weight(tile, kUnit, w.tiles, tile + kUnit);
    }
    return w;
  }
};

__device__ __forceinline__ uint32_t transposed(uint32_t x) {     // of an 8 x 8 matrix of 16-bit elements
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// A stretch of a unit, as the first producer finds it and the others read it from shared memory: little of it is kept in registers.
struct FewUnit {
  Segment sg;
  int row0, m, n;         // the request's rows and keys
  int first, count;       // rows of the unit
  int more;               // 0: there are no more
};
struct FewRows {
  int group, g, first;
  __device__ __forceinline__ int token(int r) const { return quotient(first + r, group); }
  __device__ __forceinline__ int head(int r, int token) const { return g * group + first + r - token * group; }
};

// whether all of the computing threads say so
__device__ __forceinline__ bool all_of_128(bool x) {
  int y;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 2, 128, p;\n\tselp.b32 %0, 1, 0, q;\n\t}" : "=r"(y) : "r"(static_cast<int>(x)) : "memory");
  return y != 0;
}

struct FewRing {
  uint32_t base, full, empty;
  int it;                 // stages so far
};

// What a warp holds of its rows: outputs - dimensions 16 c + 2 gq (0, 1) and + 1 (2, 3) of rows 8 n + 2 tq (0, 2) and + 1 (1, 3) -
// and of rows 8 n + 2 tq, + 1 (place 2 n, 2 n + 1) maxima and sums, factors, nodes.
template <int H, int G>
struct FewState {
  float o[G][H / 16][4];
  RowState st[2 * G];
  float f[2 * G];
};

// A stage of 32 keys, k0 the position of the first.  kMasked: some row may not see some of them.
template <int H, int G, bool kMasked>
__device__ __forceinline__ void stage(FewState<H, G>& a, int prefix, int end, bool has_tree, const uint32_t* tree, const float2* of_rows, uint32_t kb, float4 blocks,
                                      const uint4* q, int k0) {
  using S = Few<H, G>;
  const uint32_t vb = kb + S::kHalf;
  const int lane = threadIdx.x & 31, gq = lane >> 2, tq = lane & 3;
  const float ks[2] = {blocks.x, blocks.y}, vs[2] = {blocks.z, blocks.w};
  const float lv[2] = {__log2f(fabsf(vs[0])), __log2f(fabsf(vs[1]))};
  float sc[2][G][4];       // keys 16 m + gq (0, 1), + 8 (2, 3)
  {
    // K, all of the stage's loads side by side where there are registers for it, 16 bytes a lane and key otherwise
    constexpr int kWords = G == 1 || H == 32 ? H / 16 : 4;
#pragma unroll
    for (int part = 0; part < H / 16 / kWords; ++part) {
      uint32_t w[2][2][kWords];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = m * 16 + e * 8 + gq;
          uint32_t* to = w[m][e];
          if constexpr (H == 32) {
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(to[0]), "=r"(to[1]) : "r"(at<H, G>(kb, key, tq >> 1) + (tq & 1) * 8));
          } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i)
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(to[4 * i]), "=r"(to[4 * i + 1]), "=r"(to[4 * i + 2]), "=r"(to[4 * i + 3])
                           : "r"(at<H, G>(kb, key, tq * (H / 64) + part * (kWords / 4) + i)));
          }
          if (part == 0) {
#pragma unroll
            for (int n = 0; n < G; ++n) sc[m][n][e] = sc[m][n][2 + e] = 0.f;
          }
        }
#pragma unroll
      for (int s = 0; s < kWords; s += 2) {
        uint4 y[G];
#pragma unroll
        for (int n = 0; n < G; ++n) y[n] = q[(n * (H / 32) + part * (kWords / 2) + s / 2) * 32];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const uint32_t x[4] = {half2_of(w[m][0][s + k]), half2_of(w[m][1][s + k]), half2_of_upper(w[m][0][s + k]), half2_of_upper(w[m][1][s + k])};
#pragma unroll
            for (int n = 0; n < G; ++n) mma_half(sc[m][n], x, k ? y[n].z : y[n].x, k ? y[n].w : y[n].y);
          }
      }
    }
  }
  // V: 16 keys x 32 dimensions a load, two loads under way
  constexpr int kLoads = 2 * (H / 32);
  uint32_t vw[2][4];
  auto load_v = [&](int i) {
    const int m = i / (H / 32), d = i % (H / 32);
    uint32_t* b = vw[i & 1];
    ldmatrix_x4_trans(at<H, G>(vb, m * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), d * 2 + (lane >> 4)), b[0], b[1], b[2], b[3]);
  };
  load_v(0);
  load_v(1);
  // The scores less their rows' references.  Where all rows see all keys and nothing exceeds a reference by much - nearly always -
  // that is all: no maximum over the warp, nothing to rescale.
  bool calm = !kMasked;
#pragma unroll
  for (int n = 0; n < G; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const RowState& r = a.st[2 * n + e];
      float top = -INFINITY;
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float x = a.f[2 * n + e] * ks[m];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          float& s = sc[m][n][2 * z + e];
          s = kMasked ? s * x : fmaf(s, x, -r.ref);
          top = fmaxf(top, s);
        }
      }
      if (!kMasked) calm = calm && top < r.room(fmaxf(lv[0], lv[1]));
    }
  // what the exponentials of a row and block are multiplied by (of more rows there are not the registers to keep it)
  constexpr bool kKept = G == 1;
  float by[kKept ? 2 * G : 1][2];
  if (!kMasked && __all_sync(0xffffffffu, calm)) {
    if constexpr (kKept) {
#pragma unroll
      for (int i = 0; i < 2 * G; ++i)
#pragma unroll
        for (int m = 0; m < 2; ++m) by[i][m] = plain_weight(a.st[i].w, vs[m]);
    }
  } else {
    float al[2 * G];
#pragma unroll
    for (int n = 0; n < G; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        RowState& r = a.st[2 * n + e];
        float top = -INFINITY, top_u = -INFINITY;
        int j = 0;
        if (kMasked) j = __float_as_int(of_rows[8 * n + 2 * tq + e].y);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            float& s = sc[m][n][2 * z + e];
            if constexpr (kMasked) {      // a key that the row does not see, or that does not exist, becomes -infinity whatever it is
              const int key = k0 + m * 16 + z * 8 + gq, of = key - prefix;
              bool seen = key < end;
              if (of >= 0 && seen) seen = has_tree ? (tree[j * (kMaxTreeNodes / 32) + (of >> 5)] >> (of & 31)) & 1u : of <= j;
              if (!seen) s = -INFINITY;
            } else {
              s += r.ref;
            }
          }
          const float here = fmaxf(sc[m][n][e], sc[m][n][2 + e]);
          top = fmaxf(top, here);
          top_u = fmaxf(top_u, here + lv[m]);
        }
#pragma unroll
        for (int o = 4; o < 32; o *= 2) {
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          top_u = fmaxf(top_u, __shfl_xor_sync(0xffffffffu, top_u, o));
        }
        al[2 * n + e] = r.take(top, top_u);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int z = 0; z < 2; ++z) sc[m][n][2 * z + e] -= r.ref;
        if constexpr (kKept) {
#pragma unroll
          for (int m = 0; m < 2; ++m) by[2 * n + e][m] = block_weight(r.w, vs[m]);
        }
      }
#pragma unroll
    for (int n = 0; n < G; ++n)
#pragma unroll
      for (int c = 0; c < H / 16; ++c) {
        a.o[n][c][0] *= al[2 * n];
        a.o[n][c][1] *= al[2 * n + 1];
        a.o[n][c][2] *= al[2 * n];
        a.o[n][c][3] *= al[2 * n + 1];
      }
  }
  uint32_t pb[2][G][2];     // the numerators as B operand; their sum is taken before the rounding
#pragma unroll
  for (int n = 0; n < G; ++n) {
    RowState &r0 = a.st[2 * n], &r1 = a.st[2 * n + 1];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float x0 = kKept ? by[kKept ? 2 * n : 0][m] : block_weight(r0.w, vs[m]), x1 = kKept ? by[kKept ? 2 * n + 1 : 0][m] : block_weight(r1.w, vs[m]);
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const float s0 = sc[m][n][2 * z], s1 = sc[m][n][2 * z + 1];
        float p0 = exp2_approx(s0), p1 = exp2_approx(s1);
        r0.l += p0;
        r1.l += p1;
        p0 *= x0;
        p1 *= x1;
        if constexpr (kMasked) {       // a scale that is no number reaches the rows that see its block, not the others
          if (s0 == -INFINITY) p0 = 0.f;
          if (s1 == -INFINITY) p1 = 0.f;
        }
        pb[m][n][z] = transposed(pack_half(p0, p1));
      }
    }
  }
  bool odd = false;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int m = i / (H / 32), d = i % (H / 32), x = k0 + m * 16 + 2 * tq;
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = __byte_perm(vw[i & 1][k], 0, 0x3120);      // the even dimension of two keys, the odd one
    if (i + 2 < kLoads) load_v(i + 2);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t v[4] = {half2_of(b[2 * c]), half2_of_upper(b[2 * c]), half2_of(b[2 * c + 1]), half2_of_upper(b[2 * c + 1])};
      if constexpr (kMasked) {
        // A numerator of 0 does not silence a code that is no number.  Values of keys that do not exist are taken as 0; of the
        // others those that are no numbers are left out and given afterwards to the rows that see them.
        const uint32_t there[2] = {(x < end ? 0xffffu : 0u) | (x + 1 < end ? 0xffff0000u : 0u),
                                   (x + 8 < end ? 0xffffu : 0u) | (x + 9 < end ? 0xffff0000u : 0u)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] &= there[e >> 1];
          const uint32_t off = ((v[e] & 0x7c00u) == 0x7c00u ? 0xffffu : 0u) | ((v[e] & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u);
          odd |= off != 0;
          v[e] &= ~off;
        }
      }
#pragma unroll
      for (int n = 0; n < G; ++n) mma_half(a.o[n][2 * d + c], v, pb[m][n][0], pb[m][n][1]);
    }
  }
  if constexpr (kMasked) {
    if (__any_sync(0xffffffffu, odd)) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll 1
          for (int e = 0; e < 8; ++e) {
            const int src = e * 4 + tq, key = m * 16 + z * 8 + e;
            bool see[2 * G];
#pragma unroll
            for (int i = 0; i < 2 * G; ++i) see[i] = __shfl_sync(0xffffffffu, sc[m][i >> 1][2 * z + (i & 1)], src) != -INFINITY;
            if (k0 + key >= end) continue;
#pragma unroll
            for (int c = 0; c < H / 16; ++c) {
              uint16_t w;
              asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(at<H, G>(vb, key, c) + gq * 2));
#pragma unroll
              for (int y = 0; y < 2; ++y)
                if ((w >> 8 * y & 0x7f) == 0x7f) {
#pragma unroll
                  for (int i = 0; i < 2 * G; ++i)
                    if (see[i]) a.o[i >> 1][c][2 * y + (i & 1)] = NAN;
                }
            }
          }
    }
  }
}

// Warps 0-3 compute, the others bring the stages in.
template <int H, int G>
__global__ void __launch_bounds__(Few<H, G>::kThreads, Few<H, G>::kBlocks) scaled_kernel(const PagedCache c, const CacheScales sc, const PagedRows r, const ScaledParts parts,
                                                                            const __grid_constant__ CUtensorMap map_k,
                                                                            const __grid_constant__ CUtensorMap map_v) {
  using S = Few<H, G>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int stop_word;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* ptr = smem_raw + (base - raw);
  volatile int* stop = &stop_word;
  float* scales = reinterpret_cast<float*>(ptr + S::kOffScale);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  FewRing ring{base, base + S::kOffBar, base + S::kOffBar + 8 * S::kStages, 0};
  const uint32_t unit_full = base + S::kOffBar + 16 * S::kStages, unit_empty = unit_full + 16;
  FewUnit* shared_units = reinterpret_cast<FewUnit*>(ptr + S::kOffUnit);
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = 0;
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(ring.full + 8 * s, 1);
      mbar_init(ring.empty + 8 * s, S::kReaders);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(unit_full + 8 * s, 1);
      mbar_init(unit_empty + 8 * s, kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  __syncthreads();
  pdl_wait();
  const FewLine<S::kRows> line(c, r);
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (threadIdx.x == 0) leave_none(parts.desc, blockIdx.x);
  if (share.from >= share.to) return;

  if (warp >= kWarps) {
    const int producer = warp - kWarps;
    const uint64_t first = policy_evict_first(), last = policy_evict_last();
    const int cpp = c.ps / 16;                  // 16-key groups of a page
    int units = 0;
    // (all lanes call it) makes a stretch known to the others once the one before the last has been dealt with
    auto publish = [&](const FewUnit& u) {
      bool ok = true;
      if (lane == 0) {
        ok = !*stop && mbar_wait(unit_empty + 8 * (units & 1), ((units >> 1) & 1) ^ 1, stop);
        if (ok) {
          shared_units[units & 1] = u;
          mbar_arrive(unit_full + 8 * (units & 1));
        } else {
          *stop = 1;
        }
      }
      ++units;
      return __shfl_sync(0xffffffffu, ok, 0) != 0;
    };
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const int row = sg.rb * S::kRows;
      if (producer == 0 && !publish(FewUnit{sg, w.v.row0, w.v.m, w.v.n, row, min(S::kRows, w.v.m * r.group - row), 1})) return;
      const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
      const int g0 = sg.t0 * (kTile / 16), g1 = min((w.v.n + 15) / 16, sg.t1 * (kTile / 16));     // groups that hold any key
      const uint64_t policy = w.n_rb > 1 ? last : first;        // others read these keys as well: leave them in L2
      // a lane looks after one of 32 groups (sixteen stages): its place and its scales; those of the next round are under way
      // while this one's stages are copied
      auto page_of = [&](int e) { return e < g1 ? table[quotient(e, cpp)] : -1; };
      int block = 0, block_next, page_next = page_of(g0 + lane);
      float ks = 1.f, vs = 1.f, ks_next, vs_next;
      auto look_up = [&](int e) {               // of the group whose page has arrived
        block_next = 0;
        ks_next = vs_next = 1.f;
        if (e < g1) {
          block_next = (checked_page(c, page_next) * c.Hkv + sg.g) * cpp + (e - quotient(e, cpp) * cpp);
          ks_next = sc.k[block_next];
          vs_next = sc.v[block_next];
        }
      };
      look_up(g0 + lane);
      page_next = page_of(g0 + 32 + lane);
      const int stages = (g1 - g0 + 1) / 2;
      int round = -1;
      // A place of the ring is always the same producer's, across stretches too: it has itself filled the place the last time, so
      // that the parity that it waits for cannot be that of the phase before the last, however far the other is behind.
      for (int k = S::kProducers == 1 ? 0 : (ring.it ^ producer) & 1; k < stages; k += S::kProducers) {
        const int e = g0 + 2 * k, ahead = (2 * k) & 31;
        if (k >> 4 != round) {
          round = k >> 4;
          block = block_next;
          ks = ks_next;
          vs = vs_next;
          look_up(g0 + ((2 * k) & ~31) + 32 + lane);
          page_next = page_of(g0 + ((2 * k) & ~31) + 64 + lane);
        }
        const int it = ring.it + k, place = it % S::kStages;
        if (!__all_sync(0xffffffffu, *stop == 0 && mbar_wait(ring.empty + 8 * place, ((it / S::kStages) & 1) ^ 1, stop))) {
          *stop = 1;
          return;
        }
        const int which = lane - ahead, n_here = min(2, g1 - e);
        if (which >= 0 && which < 2) {
          scales[place * 4 + which] = ks;
          scales[place * 4 + 2 + which] = vs;
        }
        __syncwarp();
        const uint32_t bar = ring.full + 8 * place;
        if (lane == ahead) mbar_expect(bar, n_here * 2 * S::kCopy);
        __syncwarp();
        if (which >= 0 && which < n_here) {
          const uint32_t dst = base + place * S::kStage + which * S::kGroup;
          const int y = block * (16 / S::kKeysPerRow);
          tma_load_3d(dst, &map_k, 0, y, 0, bar, policy);
          tma_load_3d(dst + S::kHalf, &map_v, 0, y, 0, bar, policy);
        }
      }
      ring.it += stages;
    });
    if (producer == 0) publish(FewUnit{});
  } else {
    float* merge = reinterpret_cast<float*>(ptr + S::kOffMerge);
    float2* ml = reinterpret_cast<float2*>(ptr + S::kOffMl);
    float2* of_rows = reinterpret_cast<float2*>(ptr + S::kOffRow);
    uint4* queries = reinterpret_cast<uint4*>(ptr + S::kOffQ);
    uint32_t* tree = reinterpret_cast<uint32_t*>(ptr + S::kOffTree);
    const int gq = lane >> 2, tq = lane & 3;
    int tree_of = -1;
    for (int units = 0;; ++units) {
      const FewUnit& at_unit = shared_units[units & 1];
      const bool known = *stop == 0 && mbar_wait(unit_full + 8 * (units & 1), (units >> 1) & 1, stop);
      if (!known) *stop = 1;
      if (!all_of_128(known && at_unit.more)) break;      // (all or none: there are barriers ahead)
      const FewRows u{r.group, at_unit.sg.g, at_unit.first};
      const int m = at_unit.m, row0 = at_unit.row0, count = at_unit.count;
      // eight rows a warp: queries as fp16 in the order of the products' operands, factors, nodes (rows that there are not: 0)
      if (warp * 8 < S::kRows) {
        const int row = warp * 8 + gq, j = row < count ? u.token(row) : 0;
        const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(r.q) + (row0 + j) * r.q_stride +
                                   static_cast<int64_t>(row < count ? u.head(row, j) : 0) * H + tq * (H / 4);
        uint32_t q[H / 8];
        const float f = query_row<H>(src, row < count, q) * (r.scale * kLog2e);
#pragma unroll
        for (int i = 0; i < H / 32; ++i) queries[(warp * (H / 32) + i) * 32 + lane] = make_uint4(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]);
        if (tq == 0) of_rows[row] = make_float2(f, __int_as_float(j));
      }
      if (r.parents && tree_of != at_unit.sg.req) {     // what every node sees among the nodes
        tree_of = at_unit.sg.req;
        if (static_cast<int>(threadIdx.x) < m) {
          uint32_t bits[kMaxTreeNodes / 32];
          ancestors_of(r.parents + row0, threadIdx.x, bits, c.status);
#pragma unroll
          for (int x = 0; x < kMaxTreeNodes / 32; ++x) tree[threadIdx.x * (kMaxTreeNodes / 32) + x] = bits[x];
        }
      }
      asm volatile("bar.sync 2, 128;" ::: "memory");
      const bool split = count > S::kWarpRows;            // two warps to a stage, with sixteen rows each
      const int half = split ? warp >> 1 : 0, turn = split ? warp & 1 : warp, turns = split ? 2 : kWarps;
      FewState<H, G> a;
#pragma unroll
      for (int n = 0; n < G; ++n) {
#pragma unroll
        for (int k = 0; k < H / 16; ++k) a.o[n][k][0] = a.o[n][k][1] = a.o[n][k][2] = a.o[n][k][3] = 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          a.f[2 * n + e] = of_rows[half * S::kWarpRows + 8 * n + 2 * tq + e].x;
        }
      }
      const uint4* mine = queries + half * G * (H / 32) * 32 + lane;
      const int end = at_unit.n, prefix = end - m, stage0 = at_unit.sg.t0 * (kTile / kStageKeys);
      const int stages = min(at_unit.sg.t1 * (kTile / kStageKeys), (end + kStageKeys - 1) / kStageKeys) - stage0;
      bool failed = false;
#pragma unroll 1
      for (int k = turn; k < stages; k += turns) {
        const int it = ring.it + k, place = it % S::kStages, k0 = (stage0 + k) * kStageKeys;
        if (*stop || !mbar_wait(ring.full + 8 * place, (it / S::kStages) & 1, stop)) { *stop = 1; failed = true; break; }
        const uint32_t kb = ring.base + place * S::kStage;
        const float4 blocks = *reinterpret_cast<const float4*>(scales + place * 4);
        if (k0 + kStageKeys <= prefix) stage<H, G, false>(a, prefix, end, false, tree, of_rows, kb, blocks, mine, k0);
        else stage<H, G, true>(a, prefix, end, r.parents != nullptr, tree, of_rows + half * S::kWarpRows, kb, blocks, mine, k0);
        __syncwarp();
        if (lane < (split ? 1 : S::kReaders)) mbar_arrive(ring.empty + 8 * place);
      }
      ring.it += stages;
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) {
        float l = a.st[i].l;
        l += __shfl_xor_sync(0xffffffffu, l, 4);
        l += __shfl_xor_sync(0xffffffffu, l, 8);
        l += __shfl_xor_sync(0xffffffffu, l, 16);
        float rest = a.st[i].rest();
        bool dead = false;
        if (r.parents) {         // an unused node - it does not even see itself - sees nothing
          const int j = __float_as_int(of_rows[half * S::kWarpRows + (i >> 1) * 8 + 2 * tq + (i & 1)].y);
          const uint4 b = *reinterpret_cast<const uint4*>(tree + j * (kMaxTreeNodes / 32));
          dead = !(b.x | b.y | b.z | b.w);
        }
        if (dead) {
          a.st[i].m = -INFINITY;
          l = rest = 0.f;
        }
#pragma unroll
        for (int k = 0; k < H / 16; ++k) {
          float* v = a.o[i >> 1][k] + (i & 1);
          v[0] = dead ? 0.f : v[0] * rest * rest;
          v[2] = dead ? 0.f : v[2] * rest * rest;
        }
        a.st[i].l = l;
      }
      // The warps lay their outputs side by side, kDims dimensions at a time, and all threads add them up, four dimensions of a row
      // (or of one of either half) each.
      constexpr int kQuads = S::kDims / 4;
      const int shares = split ? 2 : kWarps, row_of = threadIdx.x / kQuads, col = threadIdx.x % kQuads * 4;
#pragma unroll 1
      for (int part = 0; part < H / S::kDims; ++part) {
        asm volatile("bar.sync 2, 128;" ::: "memory");      // everybody has read what was there
        if (part == 0 && gq == 0) {
#pragma unroll
          for (int i = 0; i < 2 * G; ++i) ml[warp * S::kWarpRows + (i >> 1) * 8 + 2 * tq + (i & 1)] = make_float2(a.st[i].m, a.st[i].l);
        }
#pragma unroll
        for (int z = 0; z < H / S::kDims; ++z)
          if (z == part) {
#pragma unroll
            for (int n = 0; n < G; ++n)
#pragma unroll
              for (int k = 0; k < S::kDims / 16; ++k) {
                const float* v = a.o[n][z * (S::kDims / 16) + k];
                float* to = merge + (warp * S::kWarpRows + n * 8 + 2 * tq) * S::kPitch + k * 16 + 2 * gq;
                *reinterpret_cast<float2*>(to) = make_float2(v[0], v[2]);
                *reinterpret_cast<float2*>(to + S::kPitch) = make_float2(v[1], v[3]);
              }
          }
        asm volatile("bar.sync 2, 128;" ::: "memory");
        if (failed || *stop || row_of >= S::kWarpRows) continue;
#pragma unroll
        for (int hf = 0; hf < S::kHalves; ++hf) {
          const int row = hf * S::kWarpRows + row_of;
          if (row >= count) continue;
          const int from = split ? 2 * hf : 0;             // the first warp that had the row
          float top = -INFINITY, den = 0.f;
          for (int w = 0; w < shares; ++w) top = fmaxf(top, ml[(from + w) * S::kWarpRows + row_of].x);
          const float ref = top == -INFINITY ? 0.f : top;
          float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            if (w >= shares) continue;
            const float2 x = ml[(from + w) * S::kWarpRows + row_of];
            const float e = exp2_approx(x.x - ref);
            const float4 y = *reinterpret_cast<const float4*>(merge + ((from + w) * S::kWarpRows + row_of) * S::kPitch + col);
            den = fmaf(e, x.y, den);
            sum.x = fmaf(e, y.x, sum.x);
            sum.y = fmaf(e, y.y, sum.y);
            sum.z = fmaf(e, y.z, sum.z);
            sum.w = fmaf(e, y.w, sum.w);
          }
          const int d = part * S::kDims + col;
          if (at_unit.sg.whole) {
            const float inv = den == 0.f ? 0.f : 1.f / den;    // a row that saw nothing has a sum of 0: its output is 0
            const int j = __float_as_int(of_rows[row].y), head = u.head(row, j);
            const int64_t t = row0 + j;
            uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(r.out) + t * r.out_stride + static_cast<int64_t>(head) * H + d);
            out[0] = pack_bf16(sum.x * inv, sum.y * inv);
            out[1] = pack_bf16(sum.z * inv, sum.w * inv);
            if (r.lse && d == 0) r.lse[t * r.Hq + head] = den == 0.f ? -INFINITY : (top + log2f(den)) * kLn2;
          } else {
            const int64_t at_row = static_cast<int64_t>(at_unit.sg.slot) * S::kRows + row;
            *reinterpret_cast<float4*>(parts.acc + at_row * H + d) = sum;
            if (d == 0) *reinterpret_cast<float2*>(parts.ml + at_row * 2) = make_float2(top, den);
          }
        }
      }
      if (at_unit.sg.last_block >= 0 && threadIdx.x == 0) leave_cut(parts.desc, blockIdx.x, at_unit.sg, row0, m, -1, u.first, count);
      asm volatile("bar.sync 2, 128;" ::: "memory");       // the next unit's queries and tree may come
      if (lane == 0) mbar_arrive(unit_empty + 8 * (units & 1));
    }
  }
  __syncthreads();
  if (*stop) {
    if (threadIdx.x == 0) set_status(c.status, SLED_ERR_DEVICE);
    const long long t0 = clock64();   // copies that were issued may still land: the shared memory stays a little longer
    while (clock64() - t0 < 2000000LL) __nanosleep(1000);
  }
}

template <int H, int G>
int launch_h(const PagedCache& c, const CacheScales& sc, const PagedRows& r, char* ws, cudaStream_t s) {
  using S = Few<H, G>;
  static std::atomic<bool> configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!allow_shared(scaled_kernel<H, G>, S::kTotal, dev, configured)) return -1;
  CUtensorMap map_k, map_v;     // rows of 128 bytes, as 64 units of 16 bits
  constexpr int P = S::kKeysPerRow;
  const long long rows = static_cast<long long>(c.n_pages) * c.Hkv * c.ps / P;
  if (tma_map_bf16_row_groups(&map_k, c.k, rows, 64, 16 / P) || tma_map_bf16_row_groups(&map_v, c.v, rows, 64, 16 / P)) return -1;
  const int blocks = min(S::kBlocks * sms, kScaledBlocks);
  ScaledParts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + 2LL * kScaledBlocks * S::kRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + 2LL * kScaledBlocks * S::kRows * 2);
  SLED_LAUNCH_PDL((scaled_kernel<H, G>), dim3(blocks), dim3(S::kThreads), S::kTotal, s, c, sc, r, parts, map_k, map_v);
  if (cudaGetLastError() != cudaSuccess) return -1;
  PagedCache of = c;            // the merge goes by the results' type
  of.dtype = BF16;
  const int n = launch_paged_merge(of, r, S::kRows, blocks, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int64_t paged_scaled_workspace(int h) {
  const int64_t here = 2LL * kScaledBlocks * Few<128, 2>::kRows * (h + 2) * 4 + kScaledBlocks * 32LL;
  return h >= 64 ? max(here, paged_tc_workspace(h)) : here;
}

int launch_paged_scaled(const PagedCache& c, const CacheScales& sc, const PagedRows& r, char* ws, cudaStream_t s) {
  // By the rows per request and KV head, on average (head_dim 128, 8 KV heads; us).  More than 8: units of 32 rows, as several of 8
  // read the keys several times - units of 8 against 32, 8 rows: 32 x 8192 keys 94, 98, 8 x 8192 34, 37, 64 x 300 26, 28; 12 rows:
  // 179, 98; 56, 37; 40, 29.  More than 32: the products of tcgen05, which take a unit of 128 rows in the time of one - units of
  // 32 against tcgen05, 32 rows: 32 x 4096 97, 128, 8 x 8192 58, 72, 64 x 300 38, 48; 36 rows: 151, 129; 93, 73; 61, 48.  (head_dim
  // 32 has no kernel of that kind: its products would be half empty.)  What a batch has on average need not suit all of it: 31 single
  // tokens over 512 .. 8192 keys 39 us, a chunk of 100 tokens over 2000 keys 27, both in one call 70; a chunk of 500 54, with them 126.
  const int64_t rows = static_cast<int64_t>(r.T) * r.group;
  if (c.h >= 64 && rows > 32LL * c.n_reqs) return launch_scaled_tc(c, sc, r, ws, s);
  const bool few = rows <= 8LL * c.n_reqs;
  if (c.h == 128) return few ? launch_h<128, 1>(c, sc, r, ws, s) : launch_h<128, 2>(c, sc, r, ws, s);
  if (c.h == 64) return few ? launch_h<64, 1>(c, sc, r, ws, s) : launch_h<64, 2>(c, sc, r, ws, s);
  return few ? launch_h<32, 1>(c, sc, r, ws, s) : launch_h<32, 2>(c, sc, r, ws, s);
}

}  // namespace sled
