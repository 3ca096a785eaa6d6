// Attention over a paged bf16 cache on the 5th-generation tensor cores (tcgen05), head_dim 64 and 128: for batches whose
// requests bring many query rows (drafted trees under grouped-query attention).
//
// A unit is up to 256 query rows that share a KV head.  They are the M side of the products, a row per tensor-memory lane,
// so that the softmax of a row stays in one thread: two groups of four warps have 128 rows each.  With more than 128
// rows both groups take every 128-key tile (its K and V are read once for all rows); with up to 128 rows the groups take
// the tiles in turn, for the same rows, and merge at the end of the unit.  Either way one group's softmax runs under the
// other's products:
//     S = Q K^T      (M 128 x N 128 keys, contraction over H)      -> tensor memory, fp32
//     O += P V       (M 128 x N H, contraction over 128 keys)      P from tensor memory (bf16, over S), V as it lies
// K and V pages arrive by TMA as 128-byte swizzled rows of 64 dimensions: K is a K-major operand of the first product, V
// an MN-major operand of the second; nothing is transposed.  A row's reference maximum is raised only when a score exceeds
// it by more than 8 (in units of log2: harmless for bf16 probabilities and fp32 sums, and it cancels in the end), which
// means rescaling the row of O in tensor memory and happens in a unit's first tiles.
//   warps 0-3, 4-7 : softmax and output of the two groups
//   warps 8, 10    : TMA of K and of V (one block per SM)
//   warp 9         : tensor-memory allocation, products (one thread); warp 11 only completes the warpgroup
// The work is shared out as paged_schedule.cuh says.  What binds: a unit's begin and end (about 20,000 cycles) where units
// have few tiles; in long ones the bytes of K and V up to about 64 rows, then the products, which one thread issues in
// order (a 128 x 128 x 16 step takes about 100 cycles of the second and 64 of the first).  Measured, 8 KV heads of 128, 4
// contexts of 32768 keys: 120 rows 126 us, 4.3 TB/s; 256 rows 178 us, 770 TFLOP/s; 512 rows 315 us, 870 TFLOP/s.  A row's
// scores and what outlives a tile do not fit the 168 registers that the compiler may use: 364 - 458 bytes a thread are
// spilled.  Every wait is bounded; when one runs out the block says so in *status, lets what is under way land, frees its
// tensor memory and returns.
#include "gemm_tc.h"
#include "kernels.h"
#include "paged_schedule.cuh"
#include "tcgen05_ptx.cuh"

namespace sled {

namespace {

constexpr int kKeys = 128;                 // keys per tile
constexpr int kGroupRows = 128;            // rows of a softmax group
constexpr float kRaiseBy = 8.f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

// kGroups: softmax groups that have rows of their own in the largest unit (1: units of up to 128 rows, 2: up to 256).
// K and V lie in groups of eight rows, [H / 64][8 rows][64 columns], as a copy of 16 cached keys leaves them; 128 rows of Q
// as [H / 64][128 rows][64 columns].
template <int H, int kGroups>
struct Tc {
  static constexpr int kHalves = H / 64;
  static constexpr int kOctet = kHalves * 1024;          // eight rows
  static constexpr int kTileBytes = 16 * kOctet;         // K, V or 128 rows of Q
  static constexpr int kKStages = H == 64 ? 5 : 3, kVStages = H == 64 ? 4 : kGroups == 1 ? 3 : 2;
  static constexpr int kOffQ = 0;
  static constexpr int kOffK = kGroups * kTileBytes;
  static constexpr int kOffV = kOffK + kKStages * kTileBytes;
  static constexpr int kOffBar = kOffV + kVStages * kTileBytes;
  static constexpr int kOffTree = kOffBar + 256;         // parents of the nodes, one byte each, for either group
  static constexpr int kOffTop = kOffTree + 2 * kMaxTreeNodes;   // what the groups tell each other about a row
  static constexpr int kTotal = kOffTop + kGroupRows * 8 + 1024;       // alignment slack
};
static_assert(kMaxTreeNodes == 128);
static_assert(Tc<128, 1>::kTotal + 512 <= 227 * 1024 && Tc<128, 2>::kTotal + 512 <= 227 * 1024 && Tc<64, 2>::kTotal + 512 <= 227 * 1024, "shared memory of one block");

// barriers, 8 bytes each
enum { B_KFULL = 0, B_KEMPTY = 5, B_VFULL = 10, B_VEMPTY = 14, B_QFULL = 18, B_QEMPTY = 19, B_SFULL = 20, B_PFULL = 22, B_ODONE = 26, B_COUNT = 28 };
static_assert(B_COUNT * 8 + 4 <= 256);

struct TcParts {
  float* acc;      // [2 * blocks][rows of a unit][H], not normalised
  float* ml;       // [2 * blocks][rows of a unit][2]
  int4* desc;      // [blocks][2]: CutUnit
};

// what a row sees of the request's own nodes
struct RowView {
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

// a unit, or the stretch of it that the block works on
struct TcUnit {
  Segment sg;
  int row0, m, n;
};

template <int H, int kGroups>
__global__ void __launch_bounds__(384, 1) paged_tc_kernel(const PagedCache c, const PagedRows r, const TcParts parts,
                                                          const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                          const __grid_constant__ CUtensorMap map_v) {
  using L = Tc<H, kGroups>;
  constexpr int kUnit = kGroups * kGroupRows;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int stop_word;
  __shared__ int odd_words[2];           // the last units in which a key of the masked tiles had a value that is not finite
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* ptr = smem_raw + (base - raw);
  volatile int* stop = &stop_word;
  volatile int* odd = odd_words;
  signed char* parents = reinterpret_cast<signed char*>(ptr + L::kOffTree) + (threadIdx.x >> 7 & 1) * kMaxTreeNodes;
  float2* tops = reinterpret_cast<float2*>(ptr + L::kOffTop);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ptr + L::kOffBar + 8 * B_COUNT);
  auto bar = [&](int i) { return base + L::kOffBar + 8u * static_cast<uint32_t>(i); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = r.group;
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = odd[0] = odd[1] = 0;
    for (int s = 0; s < L::kKStages; ++s) { mbar_init(bar(B_KFULL + s), 1); mbar_init(bar(B_KEMPTY + s), 1); }
    for (int s = 0; s < L::kVStages; ++s) { mbar_init(bar(B_VFULL + s), 1); mbar_init(bar(B_VEMPTY + s), 1); }
    mbar_init(bar(B_QFULL), 1);
    mbar_init(bar(B_QEMPTY), 8);
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(B_SFULL + s), 1);
      mbar_init(bar(B_PFULL + 2 * s), 4);
      mbar_init(bar(B_PFULL + 2 * s + 1), 4);
      mbar_init(bar(B_ODONE + s), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_q);
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  if (warp == 9) {   // S of the two groups at columns 0 and 128, O at 256 and 384
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

  // The registers of the block, 384 x 168, go where they are needed: 4 warps x 88, 8 warps x 200 (62,464 of 64,512).
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 8 || warp == 10) {
      // ------------------------------------------------------------------------------------------------ TMA: K, V
      const bool is_k = warp == 8;
      const CUtensorMap* map = is_k ? &map_k : &map_v;
      const uint32_t ring = base + (is_k ? L::kOffK : L::kOffV);
      const int stages = is_k ? L::kKStages : L::kVStages, b_full = is_k ? B_KFULL : B_VFULL, b_empty = is_k ? B_KEMPTY : B_VEMPTY;
      const uint64_t policy = policy_evict_first();
      const int cpp = c.ps / 16;
      int st = 0, phase = 1, units = 0;
      for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
        const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
        const int groups = min((w.v.n + 15) / 16, sg.t1 * 8);     // 16-key groups up to the end of the segment
        auto octet_of = [&](int e) {                              // where group e begins, in rows / 8
          if (e >= groups) return 0;
          const int b = e / cpp;
          return ((checked_page(c, table[b]) * c.Hkv + sg.g) * c.ps + (e - b * cpp) * 16) >> 3;
        };
        if (is_k) {     // the unit's Q first
          const int left = w.v.m * group - sg.rb * kUnit;
          const bool both = kGroups == 2 && left > kGroupRows;
          bool ok = true;
          if (lane == 0) {
            ok = !*stop && mbar_wait(bar(B_QEMPTY), (units & 1) ^ 1, stop);
            if (ok) {
              mbar_expect(bar(B_QFULL), (both ? 2 : 1) * L::kTileBytes);
              for (int s = 0; s < (both ? 2 : 1); ++s)
                tma_load_rows(base + L::kOffQ + s * L::kTileBytes, &map_q, sg.g * group,
                              w.v.row0 + (sg.rb * kUnit + s * kGroupRows) / group, bar(B_QFULL), policy);
            }
          }
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) { *stop = 1; return; }
          ++units;
        }
        // lane l looks after group l of four tiles; what comes after them is asked into L2, since shared memory holds too
        // little to cover the latency of DRAM while tiles wait for their softmax
        int octet = octet_of(sg.t0 * 8 + lane), later = 0;
        for (int t = sg.t0; t < sg.t1; ++t) {
          const int ahead = (t - sg.t0) & 3;
          if (ahead == 0) {
            if (t > sg.t0) octet = later;
            if (t == sg.t0 && (lane >> 3) >= 2 && sg.t0 * 8 + lane < groups) tma_prefetch_4d(map, octet);
            later = octet_of((t + 4) * 8 + lane);
            if ((t + 4) * 8 + lane < groups) tma_prefetch_4d(map, later);
          }
          bool ok = true;
          if (lane == 0) ok = !*stop && mbar_wait(bar(b_empty + st), phase, stop);
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) { *stop = 1; return; }
          const int n_here = min(8, groups - t * 8);
          if (lane == 0) mbar_expect(bar(b_full + st), n_here * 16 * H * 2);
          __syncwarp();
          if ((lane >> 3) == ahead && (lane & 7) < n_here)
            tma_load_4d(ring + st * L::kTileBytes + (lane & 7) * 2 * L::kOctet, map, octet, bar(b_full + st), policy);
          if (++st == stages) { st = 0; phase ^= 1; }
        }
      });
    } else if (warp == 9 && lane == 0) {
      // ------------------------------------------------------------------------------------------------ products
      constexpr uint32_t kFormat = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(128 >> 4) << 24);   // fp32 += bf16 x bf16, M 128
      constexpr uint32_t idesc_s = kFormat | (static_cast<uint32_t>(kKeys >> 3) << 17);
      constexpr uint32_t idesc_o = kFormat | (static_cast<uint32_t>(H >> 3) << 17) | (1u << 16);                    // V is MN-major
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
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // ------------------------------------------------------------------------------------------------ softmax, output
    const int s = warp >> 2, row_in_group = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tmem_s = tmem + lanes + s * 128, tmem_o = tmem + lanes + 256 + s * 128;
    const float scale = r.scale * kLog2e;
    int is = 0, vst = 0, vphase = 0, units = 0;
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
      RowView view;
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
      }
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      const int step = both ? 1 : 2, t_first = both ? 0 : s;
      if (t_first >= n_tiles) {   // nothing to do for this group; but it must not give back the Q of a unit that has not begun
        ok = __all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_QFULL), (units & 1) ^ 1, stop));
        if (lane == 0) mbar_arrive(bar(B_QEMPTY));
      }
      for (int t = 0; t < n_tiles; ++t) {
        const int my_vst = vst, my_vphase = vphase;
        if (++vst == L::kVStages) { vst = 0; vphase ^= 1; }
        if (!ok || t < t_first || (step == 2 && ((t ^ s) & 1))) continue;
        // (every decision to give up is the whole warp's: the instructions that follow need all lanes)
        if (!__all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_SFULL + s), is & 1, stop))) { ok = false; continue; }
        ++is;
        fence_after();
        if (t + step >= n_tiles && lane == 0) mbar_arrive(bar(B_QEMPTY));    // the group is done with Q
        const int x0 = (u.sg.t0 + t) * kKeys;
        const bool masked = x0 + kKeys > prefix;
        if (masked && (s == 0 || !both)) {
          // A probability of 0 does not silence a value that is not finite: values of positions that hold no key become
          // 0 here, and so do those that are not finite, which the rows that see them get back at the end.
          const int x = x0 + row_in_group;
          if (!__all_sync(0xffffffffu, mbar_wait(bar(B_VFULL + my_vst), my_vphase, stop))) { ok = false; continue; }
          const uint32_t v = base + L::kOffV + my_vst * L::kTileBytes + (row_in_group >> 3) * L::kOctet + (row_in_group & 7) * 128;
          // (the eight lanes of a quarter warp take different sixteenths of their rows: eight rows, eight banks)
          auto piece = [&](int k) { return v + (k >> 3) * 1024 + (((k & 7) ^ (row_in_group & 7)) << 4); };
          if (x >= end) {
#pragma unroll
            for (int k = 0; k < H / 8; ++k) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(piece(k)), "r"(0) : "memory");
          } else {
            uint32_t found = 0;      // all ones in an exponent carry into bit 15 or 31
#pragma unroll
            for (int k = 0; k < H / 8; ++k) {
              uint32_t y[4];
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(piece(k)));
#pragma unroll
              for (int e = 0; e < 4; ++e) found |= (y[e] & 0x7f807f80u) + 0x00800080u;
            }
            if (found & 0x80008000u) {
              odd[units & 1] = units;
#pragma unroll 1
              for (int k = 0; k < H / 8; ++k)
#pragma unroll 1
                for (int e = 0; e < 4; ++e) {
                  uint32_t y;
                  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(y) : "r"(piece(k) + 4 * e));
                  const uint32_t off = ((y & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((y & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                  asm volatile("st.shared.b32 [%0], %1;" ::"r"(piece(k) + 4 * e), "r"(y & ~off) : "memory");
                }
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (active) {
          // What a row does not see becomes -infinity in tensor memory, in a pass of its own: the code that every tile runs
          // through stays short (a tile's first run waits for its instructions).
          if (masked) {
#pragma unroll 1
            for (int q = 0; q < kKeys / 32; ++q) {
              const uint32_t see = view.seen(x0 + q * 32, prefix, end);
              if (__all_sync(0xffffffffu, see == 0xffffffffu)) continue;
              float x[32];
              tmem_ld32(tmem_s + q * 32, x);
              uint32_t y[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) y[i] = (see >> i) & 1u ? __float_as_uint(x[i]) : 0xff800000u;
              tmem_st16(tmem_s + q * 32, y);
              tmem_st16(tmem_s + q * 32 + 16, y + 16);
            }
            tmem_st_wait();
          }
          float v[kKeys];
#pragma unroll
          for (int q = 0; q < kKeys / 32; ++q) tmem_ld32_nowait(tmem_s + q * 32, v + q * 32);
          tmem_ld_wait<kKeys>(v);
          float top[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int i = 4; i < kKeys; i += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) top[e] = fmaxf(top[e], i + 4 < kKeys ? fmaxf(v[i + e], v[i + 4 + e]) : v[i + e]);
          float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
          mx *= scale;
          const bool raise = mx > m + kRaiseBy || (m == -INFINITY && mx > -INFINITY);
          if (__any_sync(0xffffffffu, raise)) {
            const float f = raise ? exp2_approx(m - mx) : 1.f;     // 0 where nothing had been seen before
            if (raise) m = mx;
            l *= f;
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
          float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
          for (int q = 0; q < kKeys / 32; ++q) {
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float a = v[q * 32 + 2 * i], b = v[q * 32 + 2 * i + 1];
              fma2(a, b, scale, -ref);
              a = exp2_approx(a);
              b = exp2_approx(b);
              add2(sum0, sum1, a, b);
              p[i] = pack_bf16(a, b);
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
      // half of the columns each: both results of a row are in the same lane of tensor memory, only maximum and sum have
      // to be exchanged.
      const bool joint = !both && n_tiles > 1;
      if (joint) {
        if (s == 1) tops[row_in_group] = make_float2(m, l);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(B_ODONE), done[0] & 1, stop) && mbar_wait(bar(B_ODONE + 1), done[1] & 1, stop));
      } else if (t_first < n_tiles && ok) {
        ok = __all_sync(0xffffffffu, mbar_wait(bar(B_ODONE + s), done[s] & 1, stop));
      }
      ++done[0];
      if (both || joint) ++done[1];
      if (!ok) *stop = 1;
      fence_after();
      float f_mine = 1.f, f_other = 0.f;      // factors of the group's own result and of the other's
      if (!joint || s == 0) {
        if (joint) {
          const float2 x = tops[row_in_group];
          const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
          f_mine = exp2_approx(m - ref);
          f_other = exp2_approx(x.x - ref);
          l = l * f_mine + x.y * f_other;
          m = top;
        }
        if (dead) { m = -INFINITY; l = 0.f; }
        if (u.sg.whole) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          f_mine *= inv;
          f_other *= inv;
        }
        if (joint) tops[row_in_group] = make_float2(f_other, f_mine);
      }
      if (joint) {
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (s == 1) {
          const float2 x = tops[row_in_group];
          f_mine = x.x;
          f_other = x.y;
        }
      }
      // values that were left out of a group's products, for the rows that see them (of a chain few keys of the masked tiles
      // are: a prompt's unit goes through its own last keys only)
      auto add_odd = [&](float* v, int d0, int whose) {
        const int behind = min(view.tree ? end : min(end, view.last + 1), u.sg.t1 * kKeys);
        for (int x = max(prefix & ~(kKeys - 1), u.sg.t0 * kKeys); x < behind; ++x) {
          if (!both && ((x / kKeys - u.sg.t0) & 1) != whose) continue;
          if (!(view.seen(x & ~31, prefix, end) >> (x & 31) & 1u)) continue;
          const int page = checked_page(c, c.table[static_cast<int64_t>(u.sg.req) * c.table_stride + x / c.ps]);
          const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(c.v) + ((static_cast<int64_t>(page) * c.Hkv + u.sg.g) * c.ps + x % c.ps) * H + d0;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float y = __bfloat162float(src[i]);
            if (!(fabsf(y) < INFINITY)) v[i] += y;
          }
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
            char* out = reinterpret_cast<char*>(reinterpret_cast<__nv_bfloat16*>(r.out) + t_row * r.out_stride + static_cast<int64_t>(head) * H + q * 32);
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = dead ? 0u : pack_bf16(v[2 * i], v[2 * i + 1]);
            store32(out, p);
            store32(out + 32, p + 8);
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
    const long long t0 = clock64();   // copies and products that were issued may still land
    while (clock64() - t0 < 2000000LL) __nanosleep(1000);
  }
  if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int H, int kGroups>
int launch_h(const PagedCache& c, const PagedRows& r, char* ws, cudaStream_t s) {
  static std::atomic<bool> configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!allow_shared(paged_tc_kernel<H, kGroups>, Tc<H, kGroups>::kTotal, dev, configured)) return -1;
  CUtensorMap map_q, map_k, map_v;
  if (tma_map_bf16_heads(&map_q, r.q, r.T, r.Hq, H, r.q_stride, r.group, kGroupRows / (r.group))) return -1;
  const long long rows = static_cast<long long>(c.n_pages) * c.Hkv * c.ps;
  if (tma_map_bf16_row_octets(&map_k, c.k, rows, H) || tma_map_bf16_row_octets(&map_v, c.v, rows, H)) return -1;
  const int blocks = min(sms, kMaxPagedBlocks / 2);
  TcParts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + static_cast<int64_t>(kMaxPagedBlocks) * 2 * kGroupRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + static_cast<int64_t>(kMaxPagedBlocks) * 2 * kGroupRows * 2);
  SLED_LAUNCH_PDL((paged_tc_kernel<H, kGroups>), dim3(blocks), dim3(384), (Tc<H, kGroups>::kTotal), s, c, r, parts, map_q, map_k, map_v);
  if (cudaGetLastError() != cudaSuccess) return -1;
  const int n = launch_paged_merge(c, r, kGroups * kGroupRows, blocks, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int64_t paged_tc_workspace(int h) {
  return static_cast<int64_t>(kMaxPagedBlocks) * 2 * kGroupRows * (h + 2) * 4 + kMaxPagedBlocks * 32LL;
}

// Q comes in by TMA, heads of whole tokens, and results go out a sector at a time
bool paged_tc_serves(const PagedCache& c, const PagedRows& r) {
  const int group = r.group;
  return c.dtype == BF16 && (c.h == 64 || c.h == 128) && kGroupRows % group == 0 && r.q_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(r.q) & 15) == 0 &&
         r.out_stride % 16 == 0 && (reinterpret_cast<uintptr_t>(r.out) & 31) == 0;
}

int launch_paged_tc(const PagedCache& c, const PagedRows& r, char* ws, cudaStream_t s) {
  // Units of 256 rows where the requests have more than 128 on average and, as far as the page table allows, there are 32
  // such tiles to an SM: the keys are read once for all rows, but a unit is longer.  64 nodes of 4 heads, 8 KV heads of 128,
  // wide and narrow: 4 contexts of 32768 keys (55 tiles to an SM) 179 and 211 us, 64 of 2048 (55) 229 and 253, 8 of 8192
  // (28) 118 and 118, one of 1000 (0.4) 28 and 23.
  int sms = 0;
  if (paged_device(&sms) < 0) return -1;
  const int64_t rows = static_cast<int64_t>(r.T) * r.group / c.n_reqs, keys = static_cast<int64_t>(c.table_cols) * c.ps;
  const bool wide = rows > kGroupRows && (rows + kGroupRows - 1) / (2 * kGroupRows) * c.n_reqs * c.Hkv * ((keys + kKeys - 1) / kKeys) >= 32LL * sms;
  if (c.h == 128) return wide ? launch_h<128, 2>(c, r, ws, s) : launch_h<128, 1>(c, r, ws, s);
  return wide ? launch_h<64, 2>(c, r, ws, s) : launch_h<64, 1>(c, r, ws, s);
}

}  // namespace sled
