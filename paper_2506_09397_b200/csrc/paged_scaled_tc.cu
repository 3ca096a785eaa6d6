// Attention over a paged cache of e4m3 codes on the 5th-generation tensor cores (tcgen05), head_dim 64 and 128: for batches whose
// requests bring many query rows (drafted trees under grouped-query attention, prompts).
//
// Formulas, scales and roundings are those of paged_scaled.cu; units, their sharing out and the two softmax groups are those
// of paged_tc.cu: a unit is up to 256 query rows that share a KV head, the M side of the products, a row per tensor-memory lane; with
// more than 128 rows both groups of four warps take every 128-key tile, with fewer they take the tiles in turn and join at
// the end.
//     S = Q C^T      (M 128 x N 128 keys, contraction over H)      -> tensor memory, fp32
//     O += P D       (M 128 x N H, contraction over 128 keys)      P from tensor memory (fp16, over S)
// The products take 16-bit operands, so four warps turn the codes into fp16: from a ring of pieces of 64 keys, K and V of a tile in
// turn, into operand tiles.  Each warp brings its sixteen keys of a piece itself, with asynchronous 16-byte
// copies, and needs nobody to tell it that they have arrived.  They bring the queries too, as fp16 times a power of two per row.  A
// score meets its block's scale ks where it leaves tensor memory, a numerator its vs before it is rounded.  The references of a row - m of the scores, u of the numerators - are raised only when something exceeds them
// by more than 2^8; raising u means rescaling the row of O in tensor memory, which happens in a unit's first tiles.
// Scores are read from tensor memory twice, for the maximum and for the exponentials: no thread holds a row of them.
//   warps 0-3, 4-7 : softmax and output of the two groups
//   warps 8-11     : K, V and Q to fp16, scales
//   warp 12        : tensor-memory allocation, products (one thread); 13-15 only complete the warpgroup
// Every wait is bounded; when one runs out the block says so in *status, lets what is under way land, frees its tensor
// memory and returns.
#include "kernels.h"
#include "paged_scaled.cuh"
#include "tcgen05_ptx.cuh"

namespace sled {

namespace {

constexpr int kKeys = 128;                 // keys per tile
constexpr int kGroupRows = 128;            // rows of a softmax group
constexpr int kScaleSlots = 16;            // tiles whose scales are kept: more than copies, K, V and S are ahead of a softmax
constexpr int kScaleWords = 20;            // ks [8], vs [8], the largest log2 |vs|
constexpr int kPieceKeys = 64;

// Operands lie in groups of eight rows, [H / 64][8 rows][64 columns] (K, V), or as [H / 64][128 rows][64 columns] (Q); rows of
// 128 bytes, 16-byte chunk c at c ^ (row & 7).
template <int H, int kGroups>
struct ScaledTc {
  static constexpr int kHalves = H / 64;
  static constexpr int kOctet = kHalves * 1024;          // eight rows
  static constexpr int kTileBytes = 16 * kOctet;         // K, V or 128 rows of Q
  static constexpr int kKStages = H == 64 ? 3 : 2, kVStages = H == 64 ? 3 : 2;
  static constexpr int kOffQ = 0;
  static constexpr int kOffK = kGroups * kTileBytes;
  static constexpr int kOffV = kOffK + kKStages * kTileBytes;
  static constexpr int kPieces = H == 64 || kGroups == 1 ? 7 : 3, kPieceBytes = kPieceKeys * H;
  static constexpr int kOffRaw = kOffV + kVStages * kTileBytes;
  static constexpr int kOffBar = kOffRaw + kPieces * kPieceBytes;
  static constexpr int kOffTree = kOffBar + 384;         // parents of the nodes, one byte each, for either group
  static constexpr int kOffTop = kOffTree + 2 * kMaxTreeNodes;     // what the groups tell each other about a row
  static constexpr int kOffScale = kOffTop + kGroupRows * 16;      // [slot][kScaleWords]
  static constexpr int kOffFactor = kOffScale + kScaleSlots * kScaleWords * 4;  // of the rows of Q
  static constexpr int kTotal = kOffFactor + kGroups * kGroupRows * 4 + 1024;     // alignment slack
};
static_assert(kMaxTreeNodes == 128);
static_assert(ScaledTc<128, 1>::kTotal + 512 <= 227 * 1024 && ScaledTc<128, 2>::kTotal + 512 <= 227 * 1024 && ScaledTc<64, 2>::kTotal + 512 <= 227 * 1024,
              "shared memory of one block");

// barriers, 8 bytes each
enum { B_KFULL = 0, B_KEMPTY = 4, B_VFULL = 8, B_VEMPTY = 12, B_QFULL = 16, B_QEMPTY = 17, B_SFULL = 18, B_PFULL = 20, B_ODONE = 24, B_SCALE = 26,
       B_COUNT = B_SCALE + kScaleSlots };
static_assert(B_COUNT * 8 + 4 <= 384);

// what a row sees of the request's own nodes
struct SeenNodes {
  uint32_t bits[kMaxTreeNodes / 32];
  int last;        // chains: the last position it sees
  bool tree;
  __device__ __forceinline__ uint32_t word(int w) const {
    uint32_t x = 0;
#pragma unroll
    for (int i = 0; i < kMaxTreeNodes / 32; ++i)
      if (w == i) x = bits[i];
    return x;
  }
  // positions x .. x + 31 as a bit set
  __device__ __forceinline__ uint32_t seen(int x, int prefix, int end) const {
    uint32_t v;
    if (!tree) {
      const int n = last + 1 - x;
      v = n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1;
    } else {
      const int a = x - prefix;
      if (a <= -32) v = 0xffffffffu;
      else if (a < 0) v = ((1u << -a) - 1) | (bits[0] << -a);
      else v = __funnelshift_r(word(a >> 5), word((a >> 5) + 1), a & 31);
    }
    const int n = end - x;
    return n <= 0 ? 0u : n >= 32 ? v : v & ((1u << n) - 1);
  }
};

__device__ __forceinline__ void mul2(float& a, float& b, float f) {
  asm("{\n\t.reg .b64 x, y;\n\t"
      "mov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\t"
      "mul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(a), "+f"(b) : "f"(f));
}
__device__ __forceinline__ void copy_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void prefetch_line(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// a unit, or the stretch of it that the block works on
struct TcUnit {
  Segment sg;
  int row0, m, n;
};

template <int H, int kGroups>
__global__ void __launch_bounds__(512, 1) scaled_tc_kernel(const PagedCache c, const CacheScales sc, const PagedRows r, const ScaledParts parts,
                                                           bool whole_q, bool whole_out) {
  using L = ScaledTc<H, kGroups>;
  constexpr int kUnit = kGroups * kGroupRows;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int stop_word;
  __shared__ int odd_words[2];           // the last units in which a key of the masked tiles had a value that is no number
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* ptr = smem_raw + (base - raw);
  volatile int* stop = &stop_word;
  volatile int* odd = odd_words;
  signed char* parents = reinterpret_cast<signed char*>(ptr + L::kOffTree) + (threadIdx.x >> 7 & 1) * kMaxTreeNodes;
  float4* tops = reinterpret_cast<float4*>(ptr + L::kOffTop);
  float* scales = reinterpret_cast<float*>(ptr + L::kOffScale);
  float* factors = reinterpret_cast<float*>(ptr + L::kOffFactor);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ptr + L::kOffBar + 8 * B_COUNT);
  auto bar = [&](int i) { return base + L::kOffBar + 8u * static_cast<uint32_t>(i); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = r.group;
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = odd[0] = odd[1] = 0;
    for (int s = 0; s < L::kKStages; ++s) { mbar_init(bar(B_KFULL + s), 4); mbar_init(bar(B_KEMPTY + s), 1); }
    for (int s = 0; s < L::kVStages; ++s) { mbar_init(bar(B_VFULL + s), 4); mbar_init(bar(B_VEMPTY + s), 1); }
    mbar_init(bar(B_QFULL), 4);
    mbar_init(bar(B_QEMPTY), 8);
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(B_SFULL + s), 1);
      mbar_init(bar(B_PFULL + 2 * s), 4);
      mbar_init(bar(B_PFULL + 2 * s + 1), 4);
      mbar_init(bar(B_ODONE + s), 1);
    }
    for (int s = 0; s < kScaleSlots; ++s) mbar_init(bar(B_SCALE + s), 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {   // S of the two groups at columns 0 and 128, O at 256 and 384
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  const AttentionLine line{c, r, 0, kUnit, kKeys};
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (threadIdx.x == 0) leave_none(parts.desc, blockIdx.x);

  // The registers of the block, 512 x 128, go where they are needed: 8 warps x 152, 4 x 128, 4 x 80 (all 65,536).
  if (warp >= 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 12 && lane == 0) {
      // ------------------------------------------------------------------------------------------------ products
      constexpr uint32_t kFormat = (1u << 4) | (static_cast<uint32_t>(128 >> 4) << 24);   // fp32 += fp16 x fp16, M 128
      constexpr uint32_t idesc_s = kFormat | (static_cast<uint32_t>(kKeys >> 3) << 17);
      constexpr uint32_t idesc_o = kFormat | (static_cast<uint32_t>(H >> 3) << 17) | (1u << 16);   // V is MN-major
      int kst = 0, kphase = 0, vst = 0, vphase = 0, units = 0, ip[2] = {0, 0};
      for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
        if (*stop) return;
        const bool both = kGroups == 2 && w.v.m * group - sg.rb * kUnit > kGroupRows;   // both groups have rows of their own
        const int n_tiles = sg.t1 - sg.t0;
        const uint32_t q0 = base + L::kOffQ;
        bool ok = mbar_wait(bar(B_QFULL), units & 1, stop);
        ++units;
        // K tiles and V tiles are used in order; a tile that both groups take is given back by the second
        auto scores = [&](int s, bool last_reader) {
          if (!mbar_wait(bar(B_KFULL + kst), kphase, stop)) return false;
          fence_after();
          const uint64_t q = operand_desc(q0 + (both ? s : 0) * L::kTileBytes, 1, 1024);
          const uint64_t k = operand_desc(base + L::kOffK + kst * L::kTileBytes, 1, L::kOctet);
#pragma unroll
          for (int ks = 0; ks < H / 16; ++ks) {
            const uint32_t within = (ks & 3) * 32;
            umma_ss(tmem + s * 128, q + (((ks >> 2) * kGroupRows * 128 + within) >> 4), k + (((ks >> 2) * 1024 + within) >> 4), idesc_s, ks != 0);
          }
          umma_commit(bar(B_SFULL + s));
          if (last_reader) {
            umma_commit(bar(B_KEMPTY + kst));
            if (++kst == L::kKStages) { kst = 0; kphase ^= 1; }
          }
          return true;
        };
        auto output = [&](int s, bool first, bool last_reader) {
          if (!mbar_wait(bar(B_VFULL + vst), vphase, stop)) return false;
          const uint64_t v = operand_desc(base + L::kOffV + vst * L::kTileBytes, 1024 >> 4, L::kOctet);
#pragma unroll
          for (int half = 0; half < 2; ++half) {     // the second half of P is still being made under the first half's products
            if (!mbar_wait(bar(B_PFULL + 2 * s + half), ip[s] & 1, stop)) return false;
            fence_after();
#pragma unroll
            for (int kt = half * (kKeys / 32); kt < (half + 1) * (kKeys / 32); ++kt)
              umma_ts(tmem + 256 + s * 128, tmem + s * 128 + kt * 8, v + ((kt * 2 * L::kOctet) >> 4), idesc_o, !first || kt != 0);
          }
          ++ip[s];
          if (last_reader) {
            umma_commit(bar(B_VEMPTY + vst));
            if (++vst == L::kVStages) { vst = 0; vphase ^= 1; }
          }
          return true;
        };
        if (both) {
          ok = ok && scores(0, false) && scores(1, true);
          for (int t = 0; ok && t < n_tiles; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              ok = ok && output(s, t == 0, s == 1);
              if (!ok) break;
              if (t + 1 < n_tiles) ok = scores(s, s == 1);
              else umma_commit(bar(B_ODONE + s));
            }
        } else {
          ok = ok && scores(0, true);
          if (n_tiles > 1) ok = ok && scores(1, true);
          for (int t = 0; ok && t < n_tiles; ++t) {
            const int s = t & 1;
            ok = output(s, t < 2, true);
            if (!ok) break;
            if (t + 2 < n_tiles) ok = scores(s, true);
            else umma_commit(bar(B_ODONE + s));
          }
        }
        if (!ok) *stop = 1;
      });
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ------------------------------------------------------------------------------------------- codes to fp16: Q, K, V
    constexpr int kLanes = H / 8, kAtOnce = 32 / kLanes;      // lanes of a key, keys at a time: a warp has 16 of a piece
    const int part = warp & 3, chunk = lane % kLanes, sub = lane / kLanes, cpp = c.ps / 16;
    const uint8_t *k_codes = reinterpret_cast<const uint8_t*>(c.k), *v_codes = reinterpret_cast<const uint8_t*>(c.v);
    int tiles_issued = 0;
    int kst = 0, kphase = 1, vst = 0, vphase = 1, units = 0, tiles = 0;
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const int first = sg.rb * kUnit, total = w.v.m * group, rows = min(kUnit, total - first);
      ++units;
      const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
      const int groups = min((w.v.n + 15) / 16, sg.t1 * 8);     // 16-key groups up to the end of the segment
      // lane l looks after group l of four tiles: the block's place among all and (one warp) its scales; those of the next round
      // and the table's entries of the one after are under way
      auto page_of = [&](int e) { return e < groups ? table[quotient(e, cpp)] : 0; };
      auto block_of = [&](int e, int page) { return e < groups ? (checked_page(c, page) * c.Hkv + sg.g) * cpp + (e - quotient(e, cpp) * cpp) : 0; };
      int block, page_next = page_of(sg.t0 * 8 + lane), block_next = block_of(sg.t0 * 8 + lane, page_next);
      float ks, vs, ks_next = 1.f, vs_next = 1.f;
      auto scales_of = [&](int e) {
        if (warp == 8 && e < groups) {
          ks_next = sc.k[block_next];
          vs_next = sc.v[block_next];
        }
      };
      scales_of(sg.t0 * 8 + lane);
      page_next = page_of(sg.t0 * 8 + 32 + lane);
      // piece i of the segment: keys 64 (i % 2) .. of K (i % 4 < 2) or V of tile t0 + i / 4; this warp: 16 of them
      const int n_pieces = (sg.t1 - sg.t0) * 4;
      int issued = 0, into = 0;
      auto issue = [&]() {
        if (issued < n_pieces) {
          const int t = sg.t0 + (issued >> 2), ahead = (issued >> 2) & 3;
          if ((issued & 3) == 0) {
            if (ahead == 0) {
              block = block_next;
              ks = ks_next;
              vs = vs_next;
              block_next = block_of((t + 4) * 8 + lane, page_next);
              ks_next = vs_next = 1.f;
              scales_of((t + 4) * 8 + lane);
              page_next = page_of((t + 8) * 8 + lane);
            }
            if (warp == 8) {
              float* to = scales + ((tiles_issued) % kScaleSlots) * kScaleWords;
              const bool mine = lane >> 3 == ahead;
              const float lv = warp_max(mine ? __log2f(fabsf(vs)) : -INFINITY);
              if (mine) {
                to[lane & 7] = ks;
                to[8 + (lane & 7)] = vs;
                if ((lane & 7) == 0) to[16] = lv;
              }
            }
            ++tiles_issued;
            // what comes four tiles later is asked into L2: two groups a warp, a line a lane
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int which = part * 2 + i;
              const int64_t at = static_cast<int64_t>(__shfl_sync(0xffffffffu, block_next, ahead * 8 + which)) * 16 * H + (lane & 15) * H;
              if ((t + 4) * 8 + which < groups && (H == 128 || !(lane & 1))) prefetch_line((lane < 16 ? k_codes : v_codes) + at);
            }
          }
          const int which = (issued & 1) * 4 + part;
          const int64_t b = __shfl_sync(0xffffffffu, block, ahead * 8 + which);
          if (t * 8 + which < groups) {
            const uint8_t* from = (issued & 2 ? v_codes : k_codes) + b * 16 * H + lane * 16;
            const uint32_t to = base + L::kOffRaw + into * L::kPieceBytes + part * 16 * H + lane * 16;
#pragma unroll
            for (int i = 0; i < H / 32; ++i) copy_16(to + i * 512, from + i * 512);
          }
          ++issued;
          if (++into == L::kPieces) into = 0;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
#pragma unroll 1
      for (int i = 0; i < L::kPieces - 1; ++i) issue();
      // the unit's Q: a row per thread
      if (!__all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_QEMPTY), (units & 1), stop))) { *stop = 1; return; }
      for (int s = 0; s < (rows > kGroupRows ? kGroups : 1); ++s) {
        const int mine = threadIdx.x & 127, at = first + s * kGroupRows + mine;
        uint4 x[H / 8];
        if (at < total) {
          const int j = quotient(at, group);
          const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(r.q) + (w.v.row0 + j) * r.q_stride + (static_cast<int64_t>(sg.g) * group + (at - j * group)) * H;
          if (whole_q) {
#pragma unroll
            for (int i = 0; i < H / 8; ++i) x[i] = reinterpret_cast<const uint4*>(q)[i];
          } else {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(q);
#pragma unroll
            for (int i = 0; i < H / 8; ++i) x[i] = make_uint4(p[4 * i], p[4 * i + 1], p[4 * i + 2], p[4 * i + 3]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < H / 8; ++i) x[i] = make_uint4(0, 0, 0, 0);
        }
        uint32_t most = 0;       // |x| as bits of bf16, times 2^16: the largest finite one
#pragma unroll
        for (int i = 0; i < H / 2; ++i) {
          const uint32_t v = reinterpret_cast<const uint32_t*>(x)[i], lo = v << 16 & 0x7fff0000u, hi = v & 0x7fff0000u;
          most = max(most, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
        }
        const int e = min(max(268 - static_cast<int>(most >> 23), 1), 253);
        const float up = __uint_as_float(static_cast<uint32_t>(e) << 23);
        factors[s * kGroupRows + mine] = __uint_as_float(static_cast<uint32_t>(254 - e) << 23) * (r.scale * kLog2e);
        const uint32_t to = base + L::kOffQ + s * L::kTileBytes + mine * 128;
#pragma unroll
        for (int i = 0; i < H / 8; ++i) {
          uint32_t y[4];
          const uint32_t v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] = pack_half(__uint_as_float(v[k] << 16) * up, __uint_as_float(v[k] & 0xffff0000u) * up);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (i >> 3) * kGroupRows * 128 + (((i & 7) ^ (mine & 7)) << 4)), "r"(y[0]), "r"(y[1]),
                       "r"(y[2]), "r"(y[3]) : "memory");
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_QFULL));

      const int end = w.v.n, prefix = end - w.v.m + (r.parents ? 0 : first / group + 1);
      // a tile of K or V: clean(key, codes) changes what may not become part of a product
      int piece = 0;
      auto convert = [&](uint32_t tile, auto clean) {
#pragma unroll 1
        for (int p = 0; p < kKeys / kPieceKeys; ++p) {
          asm volatile("cp.async.wait_group %0;" ::"n"(L::kPieces - 2) : "memory");
          __syncwarp();
          const uint32_t from = base + L::kOffRaw + piece * L::kPieceBytes + part * 16 * H + lane * 8, to = tile + (p * 8 + part * 2) * L::kOctet + (chunk >> 3) * 1024;
          uint2 x[16 / kAtOnce];
#pragma unroll
          for (int i = 0; i < 16 / kAtOnce; ++i)
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x[i].x), "=r"(x[i].y) : "r"(from + i * 256));
#pragma unroll
          for (int i = 0; i < 16 / kAtOnce; ++i) {
            const int key = i * kAtOnce + sub, row = key & 7;
            clean(p * kPieceKeys + part * 16 + key, x[i]);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (key >> 3) * L::kOctet + row * 128 + (((chunk & 7) ^ row) << 4)), "r"(half2_of(x[i].x)),
                         "r"(half2_of_upper(x[i].x)), "r"(half2_of(x[i].y)), "r"(half2_of_upper(x[i].y)) : "memory");
          }
          issue();       // into the place of the piece before this one, which all lanes have read
          if (++piece == L::kPieces) piece = 0;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      };
      for (int t = sg.t0; t < sg.t1; ++t, ++tiles) {
        bool ok = __all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_KEMPTY + kst), kphase, stop));
        if (!ok) { *stop = 1; break; }
        convert(base + L::kOffK + kst * L::kTileBytes, [](int, uint2&) {});
        if (lane == 0) mbar_arrive(bar(B_KFULL + kst));
        if (++kst == L::kKStages) { kst = 0; kphase ^= 1; }

        ok = __all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_VEMPTY + vst), vphase, stop));
        if (!ok) { *stop = 1; break; }
        const uint32_t to = base + L::kOffV + vst * L::kTileBytes;
        const int x0 = t * kKeys;
        if (x0 + kKeys <= prefix) {
          convert(to, [](int, uint2&) {});
        } else {
          // A numerator of 0 does not silence a value that is no number: values of positions that hold no key become 0, and so
          // do those that are no numbers, which the rows that see them get back at the end.
          uint32_t found = 0;
          convert(to, [&](int key, uint2& x) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t y = x0 + key < end ? (i ? x.y : x.x) : 0u;
              const uint32_t none = ((y & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;      // in the bytes 0x7f and 0xff
              found |= none;
              y &= ~((none >> 7) * 0xffu);
              if (i) x.y = y; else x.x = y;
            }
          });
          if (found) odd[units & 1] = units;
          __syncwarp();
        }
        if (lane == 0) {
          mbar_arrive(bar(B_SCALE + tiles % kScaleSlots));
          mbar_arrive(bar(B_VFULL + vst));
        }
        if (++vst == L::kVStages) { vst = 0; vphase ^= 1; }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");      // (copies are still under way only where the segment was given up)
      __syncwarp();
    });
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
    // ------------------------------------------------------------------------------------------------ softmax, output
    const int s = warp >> 2, row_in_group = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tmem_s = tmem + lanes + s * 128, tmem_o = tmem + lanes + 256 + s * 128;
    int is = 0, units = 0, tiles = 0;
    Walk<AttentionLine> walk(line, share, blockIdx.x);
    TcUnit next;
    auto advance = [&]() {
      if (!walk.next(next.sg)) return false;
      next.row0 = walk.w.v.row0;
      next.m = walk.w.v.m;
      next.n = walk.w.v.n;
      return true;
    };
    int done[2] = {0, 0};       // units that either group has finished
    for (bool have = advance(); have;) {
      const TcUnit u = next;
      ++units;
      const int first = u.sg.rb * kUnit, rows = min(kUnit, u.m * group - first);
      const bool both = kGroups == 2 && rows > kGroupRows;
      // positions below `prefix` are seen by all rows of the unit: those of a chain end with its first row's own
      const int n_tiles = u.sg.t1 - u.sg.t0, prefix = u.n - u.m + (r.parents ? 0 : first / group + 1), end = u.n;
      const int row = (both ? s * kGroupRows : 0) + row_in_group;      // of the unit
      const bool valid = row < rows, active = (row & ~31) < rows;      // whole warps without rows only keep up
      const int j = valid ? (first + row) / group : 0, head = u.sg.g * group + (valid ? (first + row) % group : 0);
      const int64_t t_row = u.row0 + j;
      // What the row sees of the nodes.  (A stretch without any of them need not know of unused ones: the merge leaves
      // those out.)  Either group has its own copy of the parents, so that neither waits for the other.
      SeenNodes view;
      view.tree = r.parents != nullptr;
      view.last = u.n - u.m + j;
#pragma unroll
      for (int i = 0; i < kMaxTreeNodes / 32; ++i) view.bits[i] = 0;
      bool dead = false;
      if (view.tree && u.sg.t1 * kKeys > prefix) {
        if (row_in_group < u.m) {
          int p = r.parents[u.row0 + row_in_group];
          if (p < -2 || p >= row_in_group) {
            set_status(c.status, SLED_ERR_ARG);
            p = -2;
          }
          parents[row_in_group] = static_cast<signed char>(p);
        }
        if (s == 0) asm volatile("bar.sync 2, 128;" ::: "memory");
        else asm volatile("bar.sync 3, 128;" ::: "memory");
        int a = j;
        while (a >= 0) {     // a parent is an earlier node: this ends
#pragma unroll
          for (int i = 0; i < kMaxTreeNodes / 32; ++i)
            if (i == (a >> 5)) view.bits[i] |= 1u << (a & 31);
          a = parents[a];
        }
        dead = a == -2;
        if (dead) {
#pragma unroll
          for (int i = 0; i < kMaxTreeNodes / 32; ++i) view.bits[i] = 0;
        }
        // (the next unit's parents are written after every thread has been through this unit's tiles)
      }
      float m = -INFINITY, l = 0.f, top_u = -INFINITY;
      const int step = both ? 1 : 2, t_first = both ? 0 : s;
      bool ok = __all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_QFULL), (units & 1) ^ 1, stop));
      const float factor = factors[row];
      if (t_first >= n_tiles && lane == 0) mbar_arrive(bar(B_QEMPTY));      // nothing to do for this group
      for (int t = 0; t < n_tiles; ++t, ++tiles) {
        if (!ok || t < t_first || (step == 2 && ((t ^ s) & 1))) continue;
        // (every decision to give up is the whole warp's: the instructions that follow need all lanes)
        const int slot = tiles % kScaleSlots;
        if (!__all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_SCALE + slot), (tiles / kScaleSlots) & 1, stop) &&
                                         mbar_wait(bar(B_SFULL + s), is & 1, stop))) { ok = false; continue; }
        ++is;
        fence_after();
        if (t + step >= n_tiles && lane == 0) mbar_arrive(bar(B_QEMPTY));    // the group is done with Q
        const int x0 = (u.sg.t0 + t) * kKeys;
        const bool masked = x0 + kKeys > prefix;
        if (active) {
          const float* ks = scales + slot * kScaleWords;
          const float* vs = ks + 8;
          // Scores of tiles that some row does not see all of are scaled and masked in tensor memory, in a pass of its own: the code
          // that every tile runs through stays short.
          if (masked) {
#pragma unroll 1
            for (int q = 0; q < kKeys / 32; ++q) {
              const uint32_t see = view.seen(x0 + q * 32, prefix, end);
              float x[32];
              tmem_ld32(tmem_s + q * 32, x);
              const float f0 = factor * ks[2 * q], f1 = factor * ks[2 * q + 1];
              uint32_t y[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) y[i] = (see >> i) & 1u ? __float_as_uint(x[i] * (i < 16 ? f0 : f1)) : 0xff800000u;
              tmem_st16(tmem_s + q * 32, y);
              tmem_st16(tmem_s + q * 32 + 16, y + 16);
            }
            tmem_st_wait();
          }
          const float by = masked ? 1.f : factor;
          float mx = -INFINITY;
          const float lv = ks[16];
          float v[2][32];
          tmem_ld32_nowait(tmem_s, v[0]);
#pragma unroll
          for (int q = 0; q < kKeys / 32; ++q) {
            float* x = v[q & 1];
            tmem_ld_wait<32>(x);
            if (q + 1 < kKeys / 32) tmem_ld32_nowait(tmem_s + (q + 1) * 32, v[(q + 1) & 1]);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              const float f = by * (masked ? 1.f : ks[2 * q + b]);
              float top = x[b * 16];
              if (f >= 0.f) {      // (the same for all rows: a row's own factor is positive)
#pragma unroll
                for (int i = 1; i < 16; ++i) top = fmaxf(top, x[b * 16 + i]);
              } else {
#pragma unroll
                for (int i = 1; i < 16; ++i) top = fminf(top, x[b * 16 + i]);
              }
              mx = fmaxf(mx, top * f);
            }
          }
          const bool raise = mx > m + kRaiseBy || (m == -INFINITY && mx > -INFINITY);
          const bool raise_u = mx + lv > top_u + kRaiseBy || (top_u == -INFINITY && mx + lv > -INFINITY);
          if (__any_sync(0xffffffffu, raise || raise_u)) {
            if (raise) {
              l *= exp2_approx(m - mx);     // 0 where nothing had been seen before
              m = mx;
            }
            const float f = raise_u ? exp2_approx(top_u - (mx + lv)) : 1.f;
            if (raise_u) top_u = mx + lv;
            if (t != t_first) {   // the products so far are complete: they came before these scores
#pragma unroll 1
              for (int q = 0; q < H / 32; ++q) {
                float o[32];
                tmem_ld32(tmem_o + q * 32, o);
                uint32_t x[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(o[i] * f);
                tmem_st16(tmem_o + q * 32, x);
                tmem_st16(tmem_o + q * 32 + 16, x + 16);
              }
              tmem_st_wait();
            }
          }
          const float ref = m == -INFINITY ? 0.f : m;
          const float weight = top_u == -INFINITY ? 0.f : kGain * exp2_approx(fminf(ref - top_u, 110.f));
          float sum0 = 0.f, sum1 = 0.f;
          tmem_ld32_nowait(tmem_s, v[0]);
#pragma unroll
          for (int q = 0; q < kKeys / 32; ++q) {
            float* x = v[q & 1];
            tmem_ld_wait<32>(x);
            if (q + 1 < kKeys / 32) tmem_ld32_nowait(tmem_s + (q + 1) * 32, v[(q + 1) & 1]);
            uint32_t p[16];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float f = by * (masked ? 1.f : ks[2 * q + e]), wb = top_u == -INFINITY ? 0.f : weight * vs[2 * q + e];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float a = x[e * 16 + 2 * i], b = x[e * 16 + 2 * i + 1];
                fma2(a, b, f, -ref);
                a = exp2_approx(a);
                b = exp2_approx(b);
                add2(sum0, sum1, a, b);
                mul2(a, b, wb);
                p[e * 8 + i] = pack_half(a, b);
              }
            }
            tmem_st16(tmem_s + q * 16, p);     // P lies over the scores
            if (q == kKeys / 64 - 1) {
              tmem_st_wait();
              fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(B_PFULL + 2 * s));
            }
          }
          l += sum0 + sum1;
          tmem_st_wait();
        }
        fence_before();
        __syncwarp();
        if (lane == 0) {
          if (!active) mbar_arrive(bar(B_PFULL + 2 * s));
          mbar_arrive(bar(B_PFULL + 2 * s + 1));
        }
      }
      have = advance();
      // The groups' results.  With rows of their own each writes its own; groups that shared rows also share the writing,
      // half of the columns each: both results of a row are in the same lane of tensor memory, only maximum, sum and the
      // numerators' reference have to be exchanged.
      const bool joint = !both && n_tiles > 1;
      const float rest = top_u == -INFINITY ? 0.f : exp2_approx(top_u - (m == -INFINITY ? 0.f : m)) * (1.f / kGain);     // of the output
      if (joint) {
        if (s == 1) tops[row_in_group] = make_float4(m, l, rest, 0.f);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(B_ODONE), done[0] & 1, stop) && mbar_wait(bar(B_ODONE + 1), done[1] & 1, stop));
      } else if (t_first < n_tiles && ok) {
        ok = __all_sync(0xffffffffu, mbar_wait(bar(B_ODONE + s), done[s] & 1, stop));
      }
      ++done[0];
      if (both || joint) ++done[1];
      if (!ok) *stop = 1;
      fence_after();
      float f_mine = rest, f_other = 0.f;      // factors of the group's own result and of the other's
      if (!joint || s == 0) {
        if (joint) {
          const float4 x = tops[row_in_group];
          const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
          const float a = exp2_approx(m - ref), b = exp2_approx(x.x - ref);
          f_mine = a * rest;
          f_other = b * x.z;
          l = l * a + x.y * b;
          m = top;
        }
        if (dead) { m = -INFINITY; l = 0.f; }
        if (u.sg.whole) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          f_mine *= inv;
          f_other *= inv;
        }
        if (joint) tops[row_in_group] = make_float4(f_other, f_mine, 0.f, 0.f);
      }
      if (joint) {
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (s == 1) {
          const float4 x = tops[row_in_group];
          f_mine = x.x;
          f_other = x.y;
        }
      }
      // codes that were left out of a group's products, for the rows that see them (of a chain few keys of the masked tiles
      // are: a prompt's unit goes through its own last keys only)
      auto add_odd = [&](float* v, int d0, int whose) {
        const int behind = min(view.tree ? end : min(end, view.last + 1), u.sg.t1 * kKeys);
        for (int x = max(prefix & ~(kKeys - 1), u.sg.t0 * kKeys); x < behind; ++x) {
          if (!both && ((x / kKeys - u.sg.t0) & 1) != whose) continue;
          if (!(view.seen(x & ~31, prefix, end) >> (x & 31) & 1u)) continue;
          const int page = checked_page(c, c.table[static_cast<int64_t>(u.sg.req) * c.table_stride + x / c.ps]);
          const uint8_t* src = reinterpret_cast<const uint8_t*>(c.v) + ((static_cast<int64_t>(page) * c.Hkv + u.sg.g) * c.ps + x % c.ps) * H + d0;
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if ((src[i] & 0x7f) == 0x7f) v[i] = NAN;
        }
      };
      const bool writes = ok && active && (both || joint || s == 0);
      const int q0 = joint ? s * (H / 64) : 0, q1 = joint ? q0 + H / 64 : H / 32;      // chunks of 32 columns
      if (writes) {
#pragma unroll 1
        for (int q = q0; q < q1; ++q) {
          float v[32];
          tmem_ld32(tmem_o + q * 32, v);
          if (odd[units & 1] == units) add_odd(v, q * 32, s);
          if (joint) {
            float o[32];
            tmem_ld32(tmem + lanes + 256 + (s ^ 1) * 128 + q * 32, o);
            if (odd[units & 1] == units) add_odd(o, q * 32, s ^ 1);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = v[i] * f_mine + o[i] * f_other;
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= f_mine;
          }
          if (valid && u.sg.whole) {
            uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(r.out) + t_row * r.out_stride + static_cast<int64_t>(head) * H + q * 32);
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = dead ? 0u : pack_bf16(v[2 * i], v[2 * i + 1]);
            if (whole_out) {
              store32(out, p);
              store32(out + 8, p + 8);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) out[i] = p[i];
            }
          } else if (valid) {
            char* acc = reinterpret_cast<char*>(parts.acc + (static_cast<int64_t>(u.sg.slot) * kUnit + row) * H + q * 32);
            uint32_t x[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = dead ? 0u : __float_as_uint(v[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i) store32(acc + 32 * i, x + 8 * i);
          }
        }
        if (valid && (both || s == 0)) {
          if (!u.sg.whole) {
            *reinterpret_cast<float2*>(parts.ml + (static_cast<int64_t>(u.sg.slot) * kUnit + row) * 2) = make_float2(m, l);
          } else if (r.lse) {
            r.lse[t_row * r.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
          }
        }
      }
      fence_before();        // O has been read: the next unit's products may overwrite it
      if (joint) asm volatile("bar.sync 1, 256;" ::: "memory");     // by both
      if (u.sg.last_block >= 0 && threadIdx.x == 0)
        leave_cut(parts.desc, blockIdx.x, u.sg, u.row0, u.m, -1, u.sg.rb * kUnit, min(kUnit, u.m * (r.group) - u.sg.rb * kUnit));
    }
  }

  fence_before();
  __syncthreads();
  if (*stop) {
    if (threadIdx.x == 0) set_status(c.status, SLED_ERR_DEVICE);
    const long long t0 = clock64();   // products that were issued may still land
    while (clock64() - t0 < 2000000LL) __nanosleep(1000);
  }
  if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int H, int kGroups>
int launch_h(const PagedCache& c, const CacheScales& sc, const PagedRows& r, char* ws, cudaStream_t s) {
  static std::atomic<bool> configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!allow_shared(scaled_tc_kernel<H, kGroups>, ScaledTc<H, kGroups>::kTotal, dev, configured)) return -1;
  const int blocks = min(sms, kMaxPagedBlocks / 2);
  ScaledParts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + static_cast<int64_t>(kMaxPagedBlocks) * 2 * kGroupRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + static_cast<int64_t>(kMaxPagedBlocks) * 2 * kGroupRows * 2);
  const bool whole_q = (reinterpret_cast<uintptr_t>(r.q) & 15) == 0 && r.q_stride % 8 == 0;
  const bool whole_out = (reinterpret_cast<uintptr_t>(r.out) & 31) == 0 && r.out_stride % 16 == 0;      // results go out a sector at a time
  SLED_LAUNCH_PDL((scaled_tc_kernel<H, kGroups>), dim3(blocks), dim3(512), (ScaledTc<H, kGroups>::kTotal), s, c, sc, r, parts, whole_q, whole_out);
  if (cudaGetLastError() != cudaSuccess) return -1;
  PagedCache of = c;            // the merge goes by the results' type
  of.dtype = BF16;
  const int n = launch_paged_merge(of, r, kGroups * kGroupRows, blocks, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int launch_scaled_tc(const PagedCache& c, const CacheScales& sc, const PagedRows& r, char* ws, cudaStream_t s) {
  int sms = 0;
  if (paged_device(&sms) < 0) return -1;
  const int64_t rows = static_cast<int64_t>(r.T) * r.group / c.n_reqs, keys = static_cast<int64_t>(c.table_cols) * c.ps;
  const bool wide = rows > kGroupRows && (rows + kGroupRows - 1) / (2 * kGroupRows) * c.n_reqs * c.Hkv * ((keys + kKeys - 1) / kKeys) >= 32LL * sms;
  if (c.h == 128) return wide ? launch_h<128, 2>(c, sc, r, ws, s) : launch_h<128, 1>(c, sc, r, ws, s);
  return wide ? launch_h<64, 2>(c, sc, r, ws, s) : launch_h<64, 1>(c, sc, r, ws, s);
}

}  // namespace sled
