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
//   warp 8         : TMA, three K and two V tiles under way (one block per SM)
//   warp 9         : tensor-memory allocation, products (one thread)
// The work is shared out as paged_schedule.cuh says.  What binds: the bytes of K and V up to 128 rows, the exponentials
// (16 a clock and SM) above.  Every wait is bounded; when one runs out the block says so in *status, lets what is under
// way land, frees its tensor memory and returns.
#include "gemm_tc.h"
#include "paged_schedule.cuh"
#include "warp_mma.cuh"

namespace sled {

namespace {

constexpr int kKeys = 128;                 // keys per tile
constexpr int kGroupRows = 128;            // rows of a softmax group
constexpr float kRaiseBy = 8.f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

template <int H>
struct Tc {
  static constexpr int kHalves = H / 64;
  static constexpr int kHalf = kKeys * 128;              // [128 rows][64 columns]: 16 KB
  static constexpr int kTileBytes = kHalves * kHalf;     // K, V or 128 rows of Q
  static constexpr int kKStages = H == 128 ? 3 : 5, kVStages = H == 128 ? 2 : 4;
  static constexpr int kOffQ = 0;                        // two groups of rows; the second also carries the merge
  static constexpr int kOffK = 2 * kTileBytes;
  static constexpr int kOffV = kOffK + kKStages * kTileBytes;
  static constexpr int kOffBar = kOffV + kVStages * kTileBytes;
  static constexpr int kTotal = kOffBar + 256 + 1024;    // alignment slack
};
static_assert(Tc<128>::kTotal + 1024 <= 227 * 1024 && Tc<64>::kTotal + 1024 <= 227 * 1024, "shared memory of one block");

// barriers, 8 bytes each
enum { B_KFULL = 0, B_KEMPTY = 5, B_VFULL = 10, B_VEMPTY = 14, B_QFULL = 18, B_SFULL = 19, B_PFULL = 21, B_ODONE = 23, B_COUNT = 25 };
static_assert(B_COUNT * 8 + 4 <= 256);

// bounded wait of the single-thread roles: they share their schedulers with softmax warps and sleep between polls
__device__ __forceinline__ bool mbar_wait_idle(uint32_t bar, uint32_t parity, volatile int* stop) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  for (;;) {
    __nanosleep(20);
    if (mbar_try_wait(bar, parity)) return true;
    if (*stop != 0 || clock64() - t0 > kWaitCycles) return false;
  }
}

// Operand descriptors, 128-byte swizzle, rows of 128 bytes, groups of 8 rows 1024 bytes apart.  K-major: the contraction
// runs along a row (Q, K).  MN-major: down the rows (V); the leading offset is the distance to the next 64 columns.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t leading) {
  return static_cast<uint64_t>((addr & 0x3ffff) >> 4) | (static_cast<uint64_t>(leading) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
         (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}
__device__ __forceinline__ uint64_t desc_k_major(uint32_t addr) { return operand_desc(addr, 1); }
__device__ __forceinline__ uint64_t desc_mn_major(uint32_t addr, uint32_t leading_bytes) { return operand_desc(addr, leading_bytes >> 4); }

__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(0u)
      : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {   // A in tensor memory
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(0u)
      : "memory");
}
__device__ __forceinline__ void umma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%3, %4}], [%2], %5;"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "l"(policy)
      : "memory");
}

// 32 consecutive columns of this warp's 32 lanes (thread = lane)
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15,"
      " %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

struct TcParts {
  float* acc;      // [2 * blocks][256][H], not normalised
  float* ml;       // [2 * blocks][256][2]
  int4* desc;      // [blocks] {last block or -1, first slot, request, unit of the request}
  float* scores;   // null, or [rows][Hq][keys]
  int64_t keys;
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

template <int H>
__global__ void __launch_bounds__(320, 1) paged_tc_kernel(const PagedCache c, const PagedRows r, const TcParts parts,
                                                          const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using L = Tc<H>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int stop_word, odd_word;                // odd: a key of this unit's last tiles has a value that is not finite
  __shared__ int32_t parent[kMaxTreeNodes];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* ptr = smem_raw + (base - raw);
  volatile int* stop = &stop_word;
  volatile int* odd = &odd_word;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ptr + L::kOffBar + 8 * B_COUNT);
  auto bar = [&](int i) { return base + L::kOffBar + 8u * static_cast<uint32_t>(i); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = r.Hq / c.Hkv;
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = 0;
    for (int s = 0; s < L::kKStages; ++s) { mbar_init(bar(B_KFULL + s), 1); mbar_init(bar(B_KEMPTY + s), 1); }
    for (int s = 0; s < L::kVStages; ++s) { mbar_init(bar(B_VFULL + s), 1); mbar_init(bar(B_VEMPTY + s), 1); }
    mbar_init(bar(B_QFULL), 8);
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(B_SFULL + s), 1);
      mbar_init(bar(B_PFULL + s), 4);
      mbar_init(bar(B_ODONE + s), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
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
  const AttentionLine line{c, r, 0, 2 * kGroupRows, kKeys};
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (threadIdx.x == 0) parts.desc[blockIdx.x] = make_int4(-1, 0, 0, 0);

  if (warp == 8) {
    // ------------------------------------------------------------------------------------------------ TMA
    const uint64_t policy = policy_evict_first();
    const int cpp = c.ps / 16;
    int ik = 0, iv = 0;
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
      const int groups = (w.v.n + 15) / 16, n_tiles = sg.t1 - sg.t0;
      // lane l looks up the 16-key groups l & 7 of the tiles (l >> 3), four tiles at a time
      auto rows_of = [&](int t) {
        const int e = t * 8 + lane;
        if (e >= groups || e >= sg.t1 * 8) return 0;
        const int b = e / cpp;
        return (checked_page(c, table[b]) * c.Hkv + sg.g) * c.ps + (e - b * cpp) * 16;
      };
      auto load = [&](int t, int rows, int t_rows, const CUtensorMap* map, uint32_t dst, uint32_t full) {
        const int n_here = min(8, groups - t * 8);
        if (lane == 0) mbar_expect(full, n_here * 16 * H * 2);
#pragma unroll
        for (int p = 0; p < 8; ++p) {
          const int y = __shfl_sync(0xffffffffu, rows, (t - t_rows) * 8 + p);
          if (lane == 0 && p < n_here)
#pragma unroll
            for (int hh = 0; hh < L::kHalves; ++hh) tma_load_2d(dst + hh * L::kHalf + p * 2048, map, hh * 64, y, full, policy);
        }
      };
      auto wait = [&](uint32_t b, uint32_t parity) {
        bool ok = true;
        if (lane == 0) ok = !*stop && mbar_wait_idle(b, parity, stop);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) *stop = 1;
        return ok;
      };
      // K runs one tile ahead of V: the order in which they are needed
      int k_rows = 0, v_rows = 0, k_at = -4, v_at = -4;
      for (int t = 0; t <= n_tiles; ++t) {
        if (t < n_tiles) {
          if (t - k_at >= 4) { k_at = t; k_rows = rows_of(sg.t0 + t); }
          const int st = ik % L::kKStages;
          if (!wait(bar(B_KEMPTY + st), ((ik / L::kKStages) & 1) ^ 1)) return;
          load(sg.t0 + t, k_rows, sg.t0 + k_at, &map_k, base + L::kOffK + st * L::kTileBytes, bar(B_KFULL + st));
          ++ik;
        }
        if (t > 0) {
          if (t - 1 - v_at >= 4) { v_at = t - 1; v_rows = rows_of(sg.t0 + t - 1); }
          const int st = iv % L::kVStages;
          if (!wait(bar(B_VEMPTY + st), ((iv / L::kVStages) & 1) ^ 1)) return;
          load(sg.t0 + t - 1, v_rows, sg.t0 + v_at, &map_v, base + L::kOffV + st * L::kTileBytes, bar(B_VFULL + st));
          ++iv;
        }
      }
    });
  } else if (warp == 9) {
    // ------------------------------------------------------------------------------------------------ products
    if (lane == 0) {
      constexpr uint32_t kFormat = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(128 >> 4) << 24);   // fp32 += bf16 x bf16, M 128
      constexpr uint32_t idesc_s = kFormat | (static_cast<uint32_t>(kKeys >> 3) << 17);
      constexpr uint32_t idesc_o = kFormat | (static_cast<uint32_t>(H >> 3) << 17) | (1u << 16);                    // V is MN-major
      int ik = 0, iv = 0, units = 0, ip[2] = {0, 0};
      for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
        if (*stop) return;
        const bool both = w.v.m * group - sg.rb * 2 * kGroupRows > kGroupRows;   // both groups have rows of their own
        const int n_tiles = sg.t1 - sg.t0;
        bool ok = mbar_wait_idle(bar(B_QFULL), units & 1, stop);
        ++units;
        const int ik0 = ik, iv0 = iv;
        auto scores = [&](int s, int t, bool last_reader) {
          const int st = (ik0 + t) % L::kKStages;
          if (!mbar_wait_idle(bar(B_KFULL + st), ((ik0 + t) / L::kKStages) & 1, stop)) return false;
          fence_after();
          const uint32_t q = base + L::kOffQ + (both ? s * L::kTileBytes : 0), k = base + L::kOffK + st * L::kTileBytes;
#pragma unroll
          for (int ks = 0; ks < H / 16; ++ks)
            umma_ss(tmem + s * 128, desc_k_major(q + (ks >> 2) * L::kHalf + (ks & 3) * 32), desc_k_major(k + (ks >> 2) * L::kHalf + (ks & 3) * 32),
                    idesc_s, ks != 0);
          umma_commit(bar(B_SFULL + s));
          if (last_reader) umma_commit(bar(B_KEMPTY + st));
          return true;
        };
        auto output = [&](int s, int t, bool first, bool last_reader) {
          const int st = (iv0 + t) % L::kVStages;
          if (!mbar_wait_idle(bar(B_VFULL + st), ((iv0 + t) / L::kVStages) & 1, stop)) return false;
          if (!mbar_wait_idle(bar(B_PFULL + s), ip[s] & 1, stop)) return false;
          ++ip[s];
          fence_after();
          const uint32_t v = base + L::kOffV + st * L::kTileBytes;
#pragma unroll
          for (int kt = 0; kt < kKeys / 16; ++kt)
            umma_ts(tmem + 256 + s * 128, tmem + s * 128 + kt * 8, desc_mn_major(v + kt * 2048, L::kHalf), idesc_o, !first || kt != 0);
          if (last_reader) umma_commit(bar(B_VEMPTY + st));
          return true;
        };
        if (both) {
          if (ok) ok = scores(0, 0, false) && scores(1, 0, true);
          for (int t = 0; ok && t < n_tiles; ++t)
            for (int s = 0; ok && s < 2; ++s) {
              ok = output(s, t, t == 0, s == 1);
              if (!ok) break;
              if (t + 1 < n_tiles) ok = scores(s, t + 1, s == 1);
              else umma_commit(bar(B_ODONE + s));
            }
        } else {
          if (ok) ok = scores(0, 0, true);
          if (ok && n_tiles > 1) ok = scores(1, 1, true);
          for (int t = 0; ok && t < n_tiles; ++t) {
            const int s = t & 1;
            ok = output(s, t, t < 2, true);
            if (!ok) break;
            if (t + 2 < n_tiles) ok = scores(s, t + 2, true);
            else umma_commit(bar(B_ODONE + s));
          }
        }
        ik += n_tiles;
        iv += n_tiles;
        if (!ok) *stop = 1;
      });
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------------------------------------ softmax, output
    const int s = warp >> 2, row_in_group = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tmem_s = tmem + lanes + s * 128, tmem_o = tmem + lanes + 256 + s * 128;
    const float scale = r.scale * kLog2e;
    int is = 0, io = 0, iv = 0;
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const int first = sg.rb * 2 * kGroupRows, rows = min(2 * kGroupRows, w.v.m * group - first);
      const bool both = rows > kGroupRows;
      const int n_tiles = sg.t1 - sg.t0, prefix = w.v.n - w.v.m, end = w.v.n;
      const int row = (both ? s * kGroupRows : 0) + row_in_group;      // of the unit
      const bool valid = row < rows, active = (row & ~31) < rows;      // whole warps without rows only keep up
      const int j = valid ? (first + row) / group : 0, head = sg.g * group + (valid ? (first + row) % group : 0);
      const int64_t t_row = w.v.row0 + j;
      // the last unit's Q, merge area, parents and flag are done with
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (threadIdx.x == 0) *odd = 0;
      if (r.parents && static_cast<int>(threadIdx.x) < w.v.m) parent[threadIdx.x] = r.parents[w.v.row0 + threadIdx.x];
      {
        // Q: with two groups a thread brings in its row, else two threads share one
        const int q_row = both ? row : (threadIdx.x & 255) >> 1;
        constexpr int kChunks = H / 8;
        const int c0 = both ? 0 : (threadIdx.x & 1) * (kChunks / 2), c1 = both ? kChunks : c0 + kChunks / 2;
        const bool there = q_row < rows;
        const int qj = there ? (first + q_row) / group : 0, qh = sg.g * group + (there ? (first + q_row) % group : 0);
        const uint32_t* src = reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(r.q) + (w.v.row0 + qj) * r.q_stride +
                                                                static_cast<int64_t>(qh) * H);
        const uint32_t dst = base + L::kOffQ + (q_row >> 7) * L::kTileBytes + (q_row & 127) * 128;
#pragma unroll 4
        for (int k = c0; k < c1; ++k) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (there) x = make_uint4(src[4 * k], src[4 * k + 1], src[4 * k + 2], src[4 * k + 3]);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                       ::"r"(dst + (k >> 3) * L::kHalf + (((k & 7) ^ (q_row & 7)) << 4)), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_QFULL));
      }
      RowView view;
      view.tree = r.parents != nullptr;
      view.last = prefix + j;
#pragma unroll
      for (int i = 0; i < kMaxTreeNodes / 32; ++i) view.bits[i] = 0;
      bool dead = false;
      if (view.tree) {
        asm volatile("bar.sync 1, 256;" ::: "memory");   // the parents are there
        ancestors_of(parent, j, view.bits, c.status);
        dead = !(view.bits[0] | view.bits[1] | view.bits[2] | view.bits[3]);
      }
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      const int step = both ? 1 : 2;
      const int t_first = both ? 0 : s;
      for (int t = t_first; t < n_tiles; t += step) {
        // (every decision to give up is the whole warp's: the instructions that follow need all lanes)
        if (!__all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_SFULL + s), is & 1, stop))) { ok = false; break; }
        ++is;
        fence_after();
        const int x0 = (sg.t0 + t) * kKeys;
        const bool masked = x0 + kKeys > prefix;
        if (active) {
          float mx = -INFINITY;
#pragma unroll
          for (int q = 0; q < kKeys / 32; ++q) {
            float v[32];
            tmem_ld32(tmem_s + q * 32, v);
            if (masked) {
              const uint32_t see = view.seen(x0 + q * 32, prefix, end);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = (see >> i) & 1u ? v[i] : -INFINITY;
            }
            float a = v[0], b = v[1], d = v[2], e = v[3];
#pragma unroll
            for (int i = 4; i < 32; i += 4) { a = fmaxf(a, v[i]); b = fmaxf(b, v[i + 1]); d = fmaxf(d, v[i + 2]); e = fmaxf(e, v[i + 3]); }
            mx = fmaxf(mx, fmaxf(fmaxf(a, b), fmaxf(d, e)));
          }
          mx *= scale;
          const bool raise = mx > m + kRaiseBy || (m == -INFINITY && mx > -INFINITY);
          if (__any_sync(0xffffffffu, raise)) {
            const float f = raise ? exp2_approx(m - mx) : 1.f;     // 0 where nothing had been seen before
            if (raise) m = mx;
            l *= f;
            if (t != t_first) {   // the products so far are complete: they came before these scores
#pragma unroll
              for (int q = 0; q < H / 32; ++q) {
                float v[32];
                tmem_ld32(tmem_o + q * 32, v);
                uint32_t u[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) u[i] = __float_as_uint(v[i] * f);
                tmem_st16(tmem_o + q * 32, u);
                tmem_st16(tmem_o + q * 32 + 16, u + 16);
              }
              tmem_st_wait();
            }
          }
          const float ref = m == -INFINITY ? 0.f : m;
          float sum0 = 0.f, sum1 = 0.f;
          float* sc = parts.scores && valid ? parts.scores + (t_row * r.Hq + head) * parts.keys + x0 : nullptr;
#pragma unroll
          for (int q = 0; q < kKeys / 32; ++q) {
            float v[32];
            tmem_ld32(tmem_s + q * 32, v);
            if (masked) {
              const uint32_t see = view.seen(x0 + q * 32, prefix, end);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = (see >> i) & 1u ? v[i] : -INFINITY;
            }
            if (sc) {
#pragma unroll
              for (int i = 0; i < 32; i += 4)
                if (x0 + q * 32 + i < end)
                  *reinterpret_cast<float4*>(sc + q * 32 + i) = make_float4(v[i] * scale, v[i + 1] * scale, v[i + 2] * scale, v[i + 3] * scale);
            }
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float a = exp2_approx(fmaf(v[2 * i], scale, -ref)), b = exp2_approx(fmaf(v[2 * i + 1], scale, -ref));
              sum0 += a;
              sum1 += b;
              p[i] = pack_bf16(a, b);
            }
            tmem_st16(tmem_s + q * 16, p);     // P lies over the scores that have been read
          }
          l += sum0 + sum1;
          tmem_st_wait();
        }
        if (masked && (s == 0 || !both)) {
          // A probability of 0 does not silence a value that is not finite: values of positions that hold no key become
          // 0 here, and so do those that are not finite, which the rows that see them get back at the end.
          const int st = (iv + t) % L::kVStages, x = x0 + row_in_group;
          if (!__all_sync(0xffffffffu, mbar_wait(bar(B_VFULL + st), ((iv + t) / L::kVStages) & 1, stop))) { ok = false; break; }
          const uint32_t v = base + L::kOffV + st * L::kTileBytes + row_in_group * 128;
          bool found = false;
#pragma unroll
          for (int hh = 0; hh < L::kHalves; ++hh)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const uint32_t a = v + hh * L::kHalf + k * 16;
              uint32_t y[4];
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(a));
              bool change = x >= end;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t off = ((y[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((y[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                found |= off != 0 && x < end;
                change |= off != 0;
                y[e] = x >= end ? 0u : y[e] & ~off;
              }
              if (change) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
            }
          if (found) *odd = 1;
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PFULL + s));
      }
      const bool worked = t_first < n_tiles;
      if (ok && worked) {
        ok = __all_sync(0xffffffffu, mbar_wait(bar(B_ODONE + s), io & 1, stop));
        ++io;
      }
      iv += n_tiles;
      if (!ok) *stop = 1;
      fence_after();
      // values that were left out, for the rows that see them
      auto add_odd = [&](float* v, int d0) {
        for (int x = max(prefix & ~(kKeys - 1), sg.t0 * kKeys); x < min(end, sg.t1 * kKeys); ++x) {
          if (!both && ((x / kKeys - sg.t0) & 1) != s) continue;
          if (!(view.seen(x & ~31, prefix, end) >> (x & 31) & 1u)) continue;
          const int page = checked_page(c, c.table[static_cast<int64_t>(sg.req) * c.table_stride + x / c.ps]);
          const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(c.v) + ((static_cast<int64_t>(page) * c.Hkv + sg.g) * c.ps + x % c.ps) * H + d0;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float y = __bfloat162float(src[i]);
            if (!(fabsf(y) < INFINITY)) v[i] += y;
          }
        }
      };
      auto read_o = [&](int q, float* v) {       // 32 columns of the row's output
        if (worked && ok) {
          tmem_ld32(tmem_o + q * 32, v);
          if (*odd) add_odd(v, q * 32);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = 0.f;
        }
      };
      // 32 columns of a row of this unit's result
      auto write_o = [&](int q, const float* v, float inv) {
        if (!valid || !ok || *stop) return;
        if (sg.whole) {
          uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(r.out) + t_row * r.out_stride + static_cast<int64_t>(head) * H) + q * 16;
#pragma unroll
          for (int i = 0; i < 16; ++i) out[i] = dead ? 0u : pack_bf16(v[2 * i] * inv, v[2 * i + 1] * inv);
        } else {
          float4* acc = reinterpret_cast<float4*>(parts.acc + (static_cast<int64_t>(sg.slot) * 2 * kGroupRows + row) * H + q * 32);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] = dead ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
      };
      if (!both && n_tiles > 1) {
        // the second group hands its half of the keys over, [columns][128 rows], as many columns at a time as the area holds
        float* area = reinterpret_cast<float*>(ptr + L::kOffQ + L::kTileBytes);
        float2* ml = reinterpret_cast<float2*>(ptr + L::kOffQ);                    // Q is done with: every product of the unit is complete
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (s == 1) ml[row_in_group] = make_float2(m, l);
        constexpr int kAtOnce = L::kTileBytes / (128 * 4) / 32;                    // chunks of 32 columns
        float f_mine = 1.f, f_other = 0.f, inv = 0.f;
#pragma unroll 1
        for (int q0 = 0; q0 < H / 32; q0 += kAtOnce) {
          if (s == 1) {
#pragma unroll 1
            for (int q = 0; q < kAtOnce; ++q) {
              float v[32];
              read_o(q0 + q, v);
#pragma unroll
              for (int i = 0; i < 32; ++i) area[(q * 32 + i) * 128 + row_in_group] = v[i];
            }
          }
          asm volatile("bar.sync 1, 256;" ::: "memory");
          if (s == 0) {
            if (q0 == 0) {
              const float2 x = ml[row_in_group];
              const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
              f_mine = exp2_approx(m - ref);
              f_other = exp2_approx(x.x - ref);
              l = l * f_mine + x.y * f_other;
              m = top;
              if (dead) { m = -INFINITY; l = 0.f; }
              inv = l == 0.f ? 0.f : 1.f / l;
            }
#pragma unroll 1
            for (int q = 0; q < kAtOnce; ++q) {
              float v[32];
              read_o(q0 + q, v);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = v[i] * f_mine + area[(q * 32 + i) * 128 + row_in_group] * f_other;
              write_o(q0 + q, v, inv);
            }
          }
          asm volatile("bar.sync 1, 256;" ::: "memory");
        }
      } else if ((both || s == 0) && active) {
        if (dead) { m = -INFINITY; l = 0.f; }
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
        for (int q = 0; q < H / 32; ++q) {
          float v[32];
          read_o(q, v);
          write_o(q, v, inv);
        }
      }
      if (valid && (both || s == 0) && ok && !*stop) {
        if (!sg.whole) {
          *reinterpret_cast<float2*>(parts.ml + (static_cast<int64_t>(sg.slot) * 2 * kGroupRows + row) * 2) = make_float2(m, l);
        } else if (r.lse) {
          r.lse[t_row * r.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
        }
      }
      fence_before();        // O has been read: the next unit's products may overwrite it
      if (sg.last_block >= 0 && threadIdx.x == 0)
        parts.desc[blockIdx.x] = make_int4(sg.last_block, sg.slot, sg.req, sg.g * w.n_rb + sg.rb);
    });
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

constexpr int kMaxDevices = 64;

template <int H>
int launch_h(const PagedCache& c, const PagedRows& r, float* scores, char* ws, cudaStream_t s) {
  static bool configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!configured[dev]) {
    if (cudaFuncSetAttribute(paged_tc_kernel<H>, cudaFuncAttributeMaxDynamicSharedMemorySize, Tc<H>::kTotal) != cudaSuccess) return -1;
    configured[dev] = true;
  }
  CUtensorMap map_k, map_v;
  const long long rows = static_cast<long long>(c.n_pages) * c.Hkv * c.ps;
  if (tma_map_bf16_rows(&map_k, c.k, rows, H, 16) || tma_map_bf16_rows(&map_v, c.v, rows, H, 16)) return -1;
  const int blocks = min(sms, kMaxPagedBlocks / 2);
  TcParts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + static_cast<int64_t>(kMaxPagedBlocks) * 2 * kGroupRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + static_cast<int64_t>(kMaxPagedBlocks) * 2 * kGroupRows * 2);
  parts.scores = scores;
  parts.keys = static_cast<int64_t>(c.table_cols) * c.ps;
  SLED_LAUNCH_PDL(paged_tc_kernel<H>, dim3(blocks), dim3(320), Tc<H>::kTotal, s, c, r, parts, map_k, map_v);
  if (cudaGetLastError() != cudaSuccess) return -1;
  const int n = launch_paged_merge(c, r, 0, 2 * kGroupRows, kKeys, blocks, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int64_t paged_tc_workspace(int h) {
  return static_cast<int64_t>(kMaxPagedBlocks) * 2 * kGroupRows * (h + 2) * 4 + kMaxPagedBlocks * 16LL;
}

int launch_paged_tc(const PagedCache& c, const PagedRows& r, float* scores, char* ws, cudaStream_t s) {
  return c.h == 128 ? launch_h<128>(c, r, scores, ws, s) : launch_h<64>(c, r, scores, ws, s);
}

}  // namespace sled
