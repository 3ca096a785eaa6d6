// Attention over a paged cache of e4m3 codes, for requests with few query rows per KV head (up to 16): decoding and short drafts.
//
// The mathematics, the scales and the roundings are those of paged_scaled.cu.  Here the keys are the M side of m16n8k16 products and
// the rows the N side, so that eight rows cost half of what sixteen do - products, exponentials, registers -:
//     S^T (16 keys x 8 rows) = C Q^T,    O^T (16 dimensions x 8 rows) += D^T P^T
// C from whole 16-byte loads of a key's codes, D^T from transposing matrix loads of 16-bit units (two dimensions of a key; the
// even and the odd dimensions become the two halves of the M side), P^T by a transposition in registers.
//
// A unit is the rows that share a KV head (up to 8 kGroups of them).  Its keys come in stages of 32, each read by one warp: the four
// computing warps take stages in turn, know nothing of each other until the end of the unit, and merge there.  A fifth warp brings
// the stages in by TMA.
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
  static constexpr int kRows = 8 * kGroups;                         // of a unit
  static constexpr int kKeysPerRow = 128 / H;
  static constexpr int kCopy = 16 * H;                              // bytes of 16 keys
  static constexpr int kGroup = kCopy < 1024 ? 1024 : kCopy;        // whole rounds of the swizzle
  static constexpr int kHalf = 2 * kGroup;
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kStages = H == 128 ? (kGroups == 1 ? 7 : 8) : 12;
  static constexpr int kBlocks = kGroups == 1 ? 3 : 2;              // on an SM
  static constexpr int kDims = H < 64 / kGroups ? H : 64 / kGroups; // of a round of the merge: all threads have four
  static constexpr int kPitch = kDims + 4;                          // four rows two apart meet 32 banks
  static constexpr int kOffMerge = kStages * kStage;
  static constexpr int kOffMl = kOffMerge + kWarps * kRows * kPitch * 4;
  static constexpr int kOffTree = kOffMl + kWarps * kRows * 8;
  static constexpr int kOffScale = kOffTree + kMaxTreeNodes * (kMaxTreeNodes / 32) * 4;     // [stage][K, V][2]
  static constexpr int kOffBar = kOffScale + kStages * 16;
  static constexpr int kTotal = kOffBar + 16 * kStages + 1024;      // alignment slack
};
static_assert(3 * (Few<128, 1>::kTotal + 1280) <= 228 * 1024 && 2 * (Few<128, 2>::kTotal + 1280) <= 228 * 1024, "blocks of an SM");

template <int H, int G>
__device__ __forceinline__ uint32_t at(uint32_t base, int key, int c) {
  constexpr int P = Few<H, G>::kKeysPerRow;
  const int row = (key & 15) / P;
  return base + (key >> 4) * Few<H, G>::kGroup + row * 128 + (((key % P * (H / 16) + c) ^ (row & 7)) << 4);
}

// The line of tiles with units of up to `rows` rows.
struct FewLine : AttentionLine {
  __device__ __forceinline__ FewLine(const PagedCache& c, const PagedRows& r, int rows) : AttentionLine{c, r, 0, rows, kTile} {}
  __device__ __forceinline__ int min_share() const { return kMinMmaShare; }
  __device__ __forceinline__ ReqWork operator()(int i) const {
    ReqWork w = AttentionLine::operator()(i);
    if (w.units > 0) w.weight = unit_weight(16, 64, w.tiles, 80);
    return w;
  }
};

__device__ __forceinline__ uint32_t transposed(uint32_t x) {     // of an 8 x 8 matrix of 16-bit elements
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

struct FewRows {
  int req, row0, group, g, first, count, prefix, end;
  __device__ __forceinline__ int token(int r) const { return quotient(first + r, group); }
};

struct FewRing {
  uint32_t base, full, empty;
  int it;                 // stages so far
};

// The stages of one stretch of a unit that are this warp's, and the merge.
template <int H, int G>
__device__ __forceinline__ void consume(const PagedRows& r, const FewRows& u, const Segment& sg, FewRing& ring, volatile int* stop,
                                        const float* scales, float* merge, float2* ml, const uint32_t* tree, const ScaledParts& parts) {
  using S = Few<H, G>;
  constexpr int KS = H / 16, DC = H / 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, tq = lane & 3;
  uint32_t q[G][H / 8];                  // row 8 n + gq: words 2 s, 2 s + 1 of product s
  float f[2 * G];                        // what turns products into scores, of rows 8 n + 2 tq, 8 n + 2 tq + 1
  int node[2 * G];
#pragma unroll
  for (int n = 0; n < G; ++n) {
    const int row = 8 * n + gq, j = row < u.count ? u.token(row) : 0;
    const int head = row < u.count ? u.g * u.group + u.first + row - j * u.group : 0;
    const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(r.q) + (u.row0 + j) * r.q_stride + static_cast<int64_t>(head) * H + tq * (H / 4);
    const float mine = query_row<H>(src, row < u.count, q[n]) * (r.scale * kLog2e);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      f[2 * n + e] = __shfl_sync(0xffffffffu, mine, (2 * tq + e) * 4);
      node[2 * n + e] = __shfl_sync(0xffffffffu, j, (2 * tq + e) * 4);
    }
  }
  float o[G][DC][4];       // dimensions 16 c + 2 gq (0, 1) and + 1 (2, 3) of rows 8 n + 2 tq (0, 2) and + 1 (1, 3)
#pragma unroll
  for (int n = 0; n < G; ++n)
#pragma unroll
    for (int c = 0; c < DC; ++c) o[n][c][0] = o[n][c][1] = o[n][c][2] = o[n][c][3] = 0.f;
  RowState st[2 * G];
  bool failed = false;
  const int stage0 = sg.t0 * (kTile / kStageKeys), stages = min(sg.t1 * (kTile / kStageKeys), (u.end + kStageKeys - 1) / kStageKeys) - stage0;

#pragma unroll 1
  for (int k = warp; k < stages; k += kWarps) {
    const int it = ring.it + k, place = it % S::kStages;
    if (*stop || !mbar_wait(ring.full + 8 * place, (it / S::kStages) & 1, stop)) { *stop = 1; failed = true; break; }
    const int k0 = (stage0 + k) * kStageKeys;
    const uint32_t kb = ring.base + place * S::kStage, vb = kb + S::kHalf;
    const float4 blocks = *reinterpret_cast<const float4*>(scales + place * 4);
    const float ks[2] = {blocks.x, blocks.y}, vs[2] = {blocks.z, blocks.w};
    const float lv = fmaxf(__log2f(fabsf(vs[0])), __log2f(fabsf(vs[1])));
    float sc[2][G][4];       // keys 16 m + gq (0, 1), + 8 (2, 3)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      uint32_t w[2][H / 16];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = m * 16 + e * 8 + gq;
        if constexpr (H == 32) {
          asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[e][0]), "=r"(w[e][1]) : "r"(at<H, G>(kb, key, tq >> 1) + (tq & 1) * 8));
        } else {
#pragma unroll
          for (int i = 0; i < H / 64; ++i)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[e][4 * i]), "=r"(w[e][4 * i + 1]), "=r"(w[e][4 * i + 2]), "=r"(w[e][4 * i + 3])
                         : "r"(at<H, G>(kb, key, tq * (H / 64) + i)));
        }
      }
#pragma unroll
      for (int n = 0; n < G; ++n) sc[m][n][0] = sc[m][n][1] = sc[m][n][2] = sc[m][n][3] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const uint32_t a[4] = {half2_of(w[0][s]), half2_of(w[1][s]), half2_of_upper(w[0][s]), half2_of_upper(w[1][s])};
#pragma unroll
        for (int n = 0; n < G; ++n) mma_half(sc[m][n], a, q[n][2 * s], q[n][2 * s + 1]);
      }
    }
    const bool masked = k0 + kStageKeys > u.prefix;
    float mx[2 * G];
#pragma unroll
    for (int n = 0; n < G; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float top = -INFINITY;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const float x = f[2 * n + e] * ks[m];
          sc[m][n][e] *= x;
          sc[m][n][2 + e] *= x;
          if (masked) {      // a key that the row does not see, or that does not exist, becomes -infinity whatever it is
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const int key = k0 + m * 16 + z * 8 + gq, a = key - u.prefix, j = node[2 * n + e];
              bool seen = key < u.end;
              if (a >= 0 && seen) seen = r.parents ? (tree[j * (kMaxTreeNodes / 32) + (a >> 5)] >> (a & 31)) & 1u : a <= j;
              if (!seen) sc[m][n][2 * z + e] = -INFINITY;
            }
          }
          top = fmaxf(top, fmaxf(sc[m][n][e], sc[m][n][2 + e]));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        mx[2 * n + e] = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
      }
    float al[2 * G];
    bool change = false;
#pragma unroll
    for (int i = 0; i < 2 * G; ++i) {
      al[i] = st[i].take(mx[i], lv);
      change |= al[i] != 1.f;
    }
    if (__any_sync(0xffffffffu, change)) {
#pragma unroll
      for (int n = 0; n < G; ++n)
#pragma unroll
        for (int c = 0; c < DC; ++c) {
          o[n][c][0] *= al[2 * n];
          o[n][c][1] *= al[2 * n + 1];
          o[n][c][2] *= al[2 * n];
          o[n][c][3] *= al[2 * n + 1];
        }
    }
    uint32_t pb[2][G][2];     // the numerators as B operand; their sum is taken before the rounding
#pragma unroll
    for (int n = 0; n < G; ++n) {
      const float w0 = st[2 * n].unit_weight(), w1 = st[2 * n + 1].unit_weight();
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float x0 = st[2 * n].scaled(w0, vs[m]), x1 = st[2 * n + 1].scaled(w1, vs[m]);
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const float s0 = sc[m][n][2 * z], s1 = sc[m][n][2 * z + 1];
          float p0 = exp2_approx(s0 - st[2 * n].ref), p1 = exp2_approx(s1 - st[2 * n + 1].ref);
          st[2 * n].l += p0;
          st[2 * n + 1].l += p1;
          p0 *= x0;
          p1 *= x1;
          if (masked) {       // a scale that is no number reaches the rows that see its block, not the others
            if (s0 == -INFINITY) p0 = 0.f;
            if (s1 == -INFINITY) p1 = 0.f;
          }
          pb[m][n][z] = transposed(pack_half(p0, p1));
        }
      }
    }
    bool odd = false;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int x = k0 + m * 16 + 2 * tq;
      const uint32_t there[2] = {(x < u.end ? 0xffffu : 0u) | (x + 1 < u.end ? 0xffff0000u : 0u),
                                 (x + 8 < u.end ? 0xffffu : 0u) | (x + 9 < u.end ? 0xffff0000u : 0u)};
#pragma unroll
      for (int d = 0; d < H / 32; ++d) {
        uint32_t b[4];
        ldmatrix_x4_trans(at<H, G>(vb, m * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), d * 2 + (lane >> 4)), b[0], b[1], b[2], b[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = __byte_perm(b[i], 0, 0x3120);      // the even dimension of two keys, the odd one
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t a[4] = {half2_of(b[2 * c]), half2_of_upper(b[2 * c]), half2_of(b[2 * c + 1]), half2_of_upper(b[2 * c + 1])};
          if (masked) {
            // A numerator of 0 does not silence a code that is no number.  Values of keys that do not exist are taken as 0; of
            // the others those that are no numbers are left out and given afterwards to the rows that see them.
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              a[e] &= there[e >> 1];
              const uint32_t off = ((a[e] & 0x7c00u) == 0x7c00u ? 0xffffu : 0u) | ((a[e] & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u);
              odd |= off != 0;
              a[e] &= ~off;
            }
          }
#pragma unroll
          for (int n = 0; n < G; ++n) mma_half(o[n][2 * d + c], a, pb[m][n][0], pb[m][n][1]);
        }
      }
    }
    if (masked && __any_sync(0xffffffffu, odd)) {
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
            if (k0 + key >= u.end) continue;
#pragma unroll
            for (int c = 0; c < DC; ++c) {
              uint16_t w;
              asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(at<H, G>(vb, key, c) + gq * 2));
#pragma unroll
              for (int y = 0; y < 2; ++y)
                if ((w >> 8 * y & 0x7f) == 0x7f) {
#pragma unroll
                  for (int i = 0; i < 2 * G; ++i)
                    if (see[i]) o[i >> 1][c][2 * y + (i & 1)] = NAN;
                }
            }
          }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(ring.empty + 8 * place);
  }
  ring.it += stages;

#pragma unroll
  for (int i = 0; i < 2 * G; ++i) {
    float l = st[i].l;
    l += __shfl_xor_sync(0xffffffffu, l, 4);
    l += __shfl_xor_sync(0xffffffffu, l, 8);
    l += __shfl_xor_sync(0xffffffffu, l, 16);
    float rest = st[i].rest(), m = st[i].m;
    if (r.parents) {         // an unused node - it does not even see itself - sees nothing
      const uint4 b = *reinterpret_cast<const uint4*>(tree + node[i] * (kMaxTreeNodes / 32));
      if (!(b.x | b.y | b.z | b.w)) {
        m = -INFINITY;
        l = rest = 0.f;
#pragma unroll
        for (int c = 0; c < DC; ++c) o[i >> 1][c][i & 1] = o[i >> 1][c][2 + (i & 1)] = 0.f;
      }
    }
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      o[i >> 1][c][i & 1] *= rest;
      o[i >> 1][c][2 + (i & 1)] *= rest;
    }
    st[i].l = l;
    st[i].m = m;
  }
  // The warps lay their outputs side by side, kDims dimensions at a time, and all threads add them up, four dimensions of a row each.
  constexpr int kQuads = S::kDims / 4;
  const int row = threadIdx.x / kQuads, col = threadIdx.x % kQuads * 4;
  const bool writes = row < u.count && row < S::kRows;
  const int j = writes ? u.token(row) : 0, head = u.g * u.group + u.first + row - j * u.group;
#pragma unroll 1
  for (int part = 0; part < H / S::kDims; ++part) {
    asm volatile("bar.sync 2, 128;" ::: "memory");      // everybody has read what was there
    if (part == 0 && gq == 0) {
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) ml[warp * S::kRows + (i >> 1) * 8 + 2 * tq + (i & 1)] = make_float2(st[i].m, st[i].l);
    }
#pragma unroll
    for (int z = 0; z < H / S::kDims; ++z)
      if (z == part) {
#pragma unroll
        for (int n = 0; n < G; ++n)
#pragma unroll
          for (int c = 0; c < S::kDims / 16; ++c) {
            const float* v = o[n][z * (S::kDims / 16) + c];
            float* to = merge + (warp * S::kRows + n * 8 + 2 * tq) * S::kPitch + c * 16 + 2 * gq;
            *reinterpret_cast<float2*>(to) = make_float2(v[0], v[2]);
            *reinterpret_cast<float2*>(to + S::kPitch) = make_float2(v[1], v[3]);
          }
      }
    asm volatile("bar.sync 2, 128;" ::: "memory");
    if (!writes || failed || *stop) continue;
    float2 x[kWarps];
    float top = -INFINITY, den = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      x[w] = ml[w * S::kRows + row];
      top = fmaxf(top, x[w].x);
    }
    const float ref = top == -INFINITY ? 0.f : top;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float e = exp2_approx(x[w].x - ref);
      const float4 y = *reinterpret_cast<const float4*>(merge + (w * S::kRows + row) * S::kPitch + col);
      den = fmaf(e, x[w].y, den);
      sum.x = fmaf(e, y.x, sum.x);
      sum.y = fmaf(e, y.y, sum.y);
      sum.z = fmaf(e, y.z, sum.z);
      sum.w = fmaf(e, y.w, sum.w);
    }
    const int d = part * S::kDims + col;
    if (sg.whole) {
      const float inv = den == 0.f ? 0.f : 1.f / den;    // a row that saw nothing has a sum of 0: its output is 0
      const int64_t t = u.row0 + j;
      uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(r.out) + t * r.out_stride + static_cast<int64_t>(head) * H + d);
      out[0] = pack_bf16(sum.x * inv, sum.y * inv);
      out[1] = pack_bf16(sum.z * inv, sum.w * inv);
      if (r.lse && d == 0) r.lse[t * r.Hq + head] = den == 0.f ? -INFINITY : (top + log2f(den)) * kLn2;
    } else {
      const int64_t at_row = static_cast<int64_t>(sg.slot) * S::kRows + row;
      *reinterpret_cast<float4*>(parts.acc + at_row * H + d) = sum;
      if (d == 0) *reinterpret_cast<float2*>(parts.ml + at_row * 2) = make_float2(top, den);
    }
  }
}

// 160 threads: warps 0-3 compute, warp 4 brings the stages in.
template <int H, int G>
__global__ void __launch_bounds__(160, Few<H, G>::kBlocks) scaled_few_kernel(const PagedCache c, const CacheScales sc, const PagedRows r, const ScaledParts parts,
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
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = 0;
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(ring.full + 8 * s, 1);
      mbar_init(ring.empty + 8 * s, 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  __syncthreads();
  pdl_wait();
  const FewLine line(c, r, S::kRows);
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (threadIdx.x == 0) leave_none(parts.desc, blockIdx.x);
  if (share.from >= share.to) return;

  if (warp == 4) {
    const uint64_t first = policy_evict_first(), last = policy_evict_last();
    const int cpp = c.ps / 16;                  // 16-key groups of a page
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
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
      for (int e = g0; e < g1; e += 2, ++ring.it) {
        const int ahead = (e - g0) & 31;
        if (ahead == 0) {
          block = block_next;
          ks = ks_next;
          vs = vs_next;
          look_up(e + 32 + lane);
          page_next = page_of(e + 64 + lane);
        }
        const int place = ring.it % S::kStages;
        bool ok = true;
        if (lane == 0) {
          ok = !*stop && mbar_wait(ring.empty + 8 * place, ((ring.it / S::kStages) & 1) ^ 1, stop);
          if (!ok) *stop = 1;
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        __syncwarp();
        const int which = lane - ahead, n_here = min(2, g1 - e);
        const bool mine = which >= 0 && which < 2;
        if (ok && mine) {
          scales[place * 4 + which] = ks;
          scales[place * 4 + 2 + which] = vs;
        }
        __syncwarp();
        if (ok && lane == 0) mbar_expect(ring.full + 8 * place, n_here * 2 * S::kCopy);
        __syncwarp();
        if (ok && mine && which < n_here) {
          const uint32_t dst = base + place * S::kStage + which * S::kGroup, bar = ring.full + 8 * place;
          const int y = block * (16 / S::kKeysPerRow);
          tma_load_3d(dst, &map_k, 0, y, 0, bar, policy);
          tma_load_3d(dst + S::kHalf, &map_v, 0, y, 0, bar, policy);
        }
      }
    });
  } else {
    float* merge = reinterpret_cast<float*>(ptr + S::kOffMerge);
    float2* ml = reinterpret_cast<float2*>(ptr + S::kOffMl);
    uint32_t* tree = reinterpret_cast<uint32_t*>(ptr + S::kOffTree);
    int tree_of = -1;
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const int first = sg.rb * S::kRows;
      const FewRows u{sg.req, w.v.row0, r.group, sg.g, first, min(S::kRows, w.v.m * r.group - first), w.v.n - w.v.m, w.v.n};
      if (r.parents && tree_of != sg.req) {     // what every node sees among the nodes
        tree_of = sg.req;
        asm volatile("bar.sync 2, 128;" ::: "memory");
        if (static_cast<int>(threadIdx.x) < w.v.m) {
          uint32_t bits[kMaxTreeNodes / 32];
          ancestors_of(r.parents + u.row0, threadIdx.x, bits, c.status);
#pragma unroll
          for (int x = 0; x < kMaxTreeNodes / 32; ++x) tree[threadIdx.x * (kMaxTreeNodes / 32) + x] = bits[x];
        }
        asm volatile("bar.sync 2, 128;" ::: "memory");
      }
      consume<H, G>(r, u, sg, ring, stop, scales, merge, ml, tree, parts);
      if (sg.last_block >= 0 && threadIdx.x == 0) leave_cut(parts.desc, blockIdx.x, sg, u.row0, w.v.m, -1, u.first, u.count);
    });
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
  if (!allow_shared(scaled_few_kernel<H, G>, S::kTotal, dev, configured)) return -1;
  CUtensorMap map_k, map_v;     // rows of 128 bytes, as 64 units of 16 bits
  constexpr int P = S::kKeysPerRow;
  const long long rows = static_cast<long long>(c.n_pages) * c.Hkv * c.ps / P;
  if (tma_map_bf16_row_groups(&map_k, c.k, rows, 64, 16 / P) || tma_map_bf16_row_groups(&map_v, c.v, rows, 64, 16 / P)) return -1;
  const int blocks = min(S::kBlocks * sms, kFewBlocks);
  ScaledParts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + 2LL * kFewBlocks * S::kRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + 2LL * kFewBlocks * S::kRows * 2);
  SLED_LAUNCH_PDL((scaled_few_kernel<H, G>), dim3(blocks), dim3(160), S::kTotal, s, c, sc, r, parts, map_k, map_v);
  if (cudaGetLastError() != cudaSuccess) return -1;
  PagedCache of = c;            // the merge goes by the results' type
  of.dtype = BF16;
  const int n = launch_paged_merge(of, r, S::kRows, blocks, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int64_t scaled_few_workspace(int h) { return 2LL * kFewBlocks * 16 * (h + 2) * 4 + kFewBlocks * 32LL; }

int launch_scaled_few(const PagedCache& c, const CacheScales& sc, const PagedRows& r, int groups, char* ws, cudaStream_t s) {
  if (groups == 1) {
    if (c.h == 128) return launch_h<128, 1>(c, sc, r, ws, s);
    return c.h == 64 ? launch_h<64, 1>(c, sc, r, ws, s) : launch_h<32, 1>(c, sc, r, ws, s);
  }
  if (c.h == 128) return launch_h<128, 2>(c, sc, r, ws, s);
  return c.h == 64 ? launch_h<64, 2>(c, sc, r, ws, s) : launch_h<32, 2>(c, sc, r, ws, s);
}

}  // namespace sled
