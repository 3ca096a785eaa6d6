// Attention weight of every cached key, for requests with many query rows (bf16, head_dim 64 and 128): the scores are
// computed once more from the keys, S^T = K Q^T, with the KEYS on the M side, one per tensor-memory lane, so that a thread
// has one key and sums exp2(s - lse) over the rows, which are its columns, by itself; one addition per key, no atomics.
// (Keeping the scores instead costs 8 bytes per row and key, which is more than the 2 H bytes of a key from about 16 rows
// on.)
//   warps 0-3, 4-7 : sums, for every second tile each
//   warp 8         : TMA: the rows of Q a unit has, tiles of 128 keys through a ring
//   warp 9         : tensor-memory allocation, products (one thread)
// A unit is (request, KV head); rows beyond 256 are gone through 256 at a time within a tile.  What binds: the bytes of K
// (from L2 where the attention before it has left them there) up to about 128 rows, the exponentials above.  Measured, 8 KV
// heads of 128, 4 contexts of 32768 keys: 96 us on top of the attention's 126 for 120 rows, 78 on top of 118 for 36.
#include "gemm_tc.h"
#include "kernels.h"
#include "paged_schedule.cuh"
#include "tcgen05_ptx.cuh"

namespace sled {

namespace {

constexpr int kKeys = 128, kRows = 256;    // of a tile; query rows at a time
constexpr float kLog2e = 1.4426950408889634f;

template <int H>
struct Wg {
  static constexpr int kOctet = H / 64 * 1024;
  static constexpr int kTileBytes = 16 * kOctet;           // 128 keys, or 128 rows of Q as [H / 64][128 rows][64 columns]
  static constexpr int kStages = H == 128 ? 4 : 6;
  static constexpr int kOffK = 2 * kTileBytes;
  static constexpr int kOffBar = kOffK + kStages * kTileBytes;
  static constexpr int kOffLse = kOffBar + 256;            // of the rows at hand, in units of log2, for either group
  static constexpr int kOffToken = kOffLse + 2 * kRows * 4; // token of each of them, one byte, for either group
  static constexpr int kOffNone = kOffToken + 2 * kRows;    // which of them saw nothing, 32 to a word, for either group
  static constexpr int kOffDown = kOffNone + 2 * kRows / 8; // who sees a node: a set of nodes each
  static constexpr int kOffParent = kOffDown + kMaxTreeNodes * 16;
  static constexpr int kTotal = kOffParent + kMaxTreeNodes + 1024;
};
static_assert(Wg<128>::kTotal + 512 <= 227 * 1024);

enum { B_KFULL = 0, B_KEMPTY = 6, B_QFULL = 12, B_QEMPTY = 13, B_SFULL = 14, B_SEMPTY = 16, B_COUNT = 18 };

template <int H>
__global__ void __launch_bounds__(320, 1) paged_weigh_kernel(const PagedCache c, const PagedRows r, float* key_weights,
                                                             const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k) {
  using L = Wg<H>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int stop_word;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* ptr = smem_raw + (base - raw);
  volatile int* stop = &stop_word;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ptr + L::kOffBar + 8 * B_COUNT);
  auto bar = [&](int i) { return base + L::kOffBar + 8u * static_cast<uint32_t>(i); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = r.group;
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = 0;
    for (int s = 0; s < L::kStages; ++s) { mbar_init(bar(B_KFULL + s), 1); mbar_init(bar(B_KEMPTY + s), 1); }
    mbar_init(bar(B_QFULL), 1);
    mbar_init(bar(B_QEMPTY), 1);
    for (int s = 0; s < 2; ++s) { mbar_init(bar(B_SFULL + s), 1); mbar_init(bar(B_SEMPTY + s), 4); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_q);
    prefetch_map(&map_k);
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  const AttentionLine line{c, r, kWholeRows, kRows, kKeys};
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  const int tokens = kRows / group;        // of a block of rows

  if (warp == 8) {
    const uint64_t policy = policy_evict_first(), keep = policy_evict_last();
    const int cpp = c.ps / 16;
    int st = 0, phase = 1, blocks = 0;
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
      const int groups = min((w.v.n + 15) / 16, sg.t1 * 8), n_rb = (w.v.m + tokens - 1) / tokens;
      auto wait = [&](uint32_t b, uint32_t parity) {
        bool ok = true;
        if (lane == 0) ok = !*stop && mbar_wait(b, parity, stop);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) *stop = 1;
        return ok;
      };
      auto bring_q = [&](int rb) {
        if (!wait(bar(B_QEMPTY), (blocks & 1) ^ 1)) return false;
        if (lane == 0) {
          const int parts = min(w.v.m - rb * tokens, tokens) * group > kRows / 2 ? 2 : 1;
          mbar_expect(bar(B_QFULL), parts * L::kTileBytes);
          for (int p = 0; p < parts; ++p)
            tma_load_rows(base + p * L::kTileBytes, &map_q, sg.g * group, w.v.row0 + rb * tokens + p * (tokens / 2), bar(B_QFULL), keep);
        }
        ++blocks;
        return true;
      };
      if (n_rb == 1 && !bring_q(0)) return;
      int octet = 0;
      for (int t = sg.t0; t < sg.t1; ++t) {
        const int ahead = (t - sg.t0) & 3;
        if (ahead == 0) {
          const int e = t * 8 + lane;
          octet = 0;
          if (e < groups) {
            const int b = e / cpp;
            octet = ((checked_page(c, table[b]) * c.Hkv + sg.g) * c.ps + (e - b * cpp) * 16) >> 3;
          }
        }
        if (!wait(bar(B_KEMPTY + st), phase)) return;
        const int n_here = min(8, groups - t * 8);
        if (lane == 0) mbar_expect(bar(B_KFULL + st), n_here * 16 * H * 2);
        __syncwarp();
        if ((lane >> 3) == ahead && (lane & 7) < n_here)
          tma_load_4d(base + L::kOffK + st * L::kTileBytes + (lane & 7) * 2 * L::kOctet, &map_k, octet, bar(B_KFULL + st), policy);
        if (++st == L::kStages) { st = 0; phase ^= 1; }
        if (n_rb > 1)
          for (int rb = 0; rb < n_rb; ++rb)
            if (!bring_q(rb)) return;
      }
    });
  } else if (warp == 9) {
    if (lane == 0) {
      int st = 0, phase = 0, blocks = 0, made = 0;
      for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
        if (*stop) return;
        const int n_rb = (w.v.m + tokens - 1) / tokens;
        bool ok = true;
        if (n_rb == 1) ok = mbar_wait(bar(B_QFULL), blocks++ & 1, stop);
        for (int t = sg.t0; ok && t < sg.t1; ++t) {
          ok = mbar_wait(bar(B_KFULL + st), phase, stop);
          for (int rb = 0; ok && rb < n_rb; ++rb) {
            if (n_rb > 1) ok = mbar_wait(bar(B_QFULL), blocks++ & 1, stop);
            const int s = made & 1;
            ok = ok && mbar_wait(bar(B_SEMPTY + s), ((made >> 1) & 1) ^ 1, stop);
            if (!ok) break;
            ++made;
            fence_after();
            const int n = (min(w.v.m - rb * tokens, tokens) * group + 15) / 16 * 16;
            // M 128 keys, N 16 .. 256 rows; more than 128 lie in two pieces
            constexpr uint32_t kFormat = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(128 >> 4) << 24);
            const uint64_t k = operand_desc(base + L::kOffK + st * L::kTileBytes, 1, L::kOctet);
            for (int p = 0; p * 128 < n; ++p) {
              const uint32_t idesc = kFormat | (static_cast<uint32_t>(min(128, n - p * 128) >> 3) << 17);
              const uint64_t q = operand_desc(base + p * L::kTileBytes, 1, 1024);
#pragma unroll
              for (int ks = 0; ks < H / 16; ++ks) {
                const uint32_t within = (ks & 3) * 32;
                umma_ss(tmem + s * 256 + p * 128, k + (((ks >> 2) * 1024 + within) >> 4), q + (((ks >> 2) * 128 * 128 + within) >> 4), idesc, ks != 0);
              }
            }
            umma_commit(bar(B_SFULL + s));
            if (n_rb > 1) umma_commit(bar(B_QEMPTY));
          }
          if (ok) umma_commit(bar(B_KEMPTY + st));
          if (++st == L::kStages) { st = 0; phase ^= 1; }
        }
        if (ok && n_rb == 1) umma_commit(bar(B_QEMPTY));
        if (!ok) *stop = 1;
      });
    }
    __syncwarp();
  } else {
    const int s = warp >> 2, key = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tmem_s = tmem + lanes + s * 256;
    float* lse = reinterpret_cast<float*>(ptr + L::kOffLse) + s * kRows;
    uint8_t* token = ptr + L::kOffToken + s * kRows;
    uint32_t* none = reinterpret_cast<uint32_t*>(ptr + L::kOffNone) + s * (kRows / 32);
    uint32_t* down = reinterpret_cast<uint32_t*>(ptr + L::kOffDown);
    signed char* parents = reinterpret_cast<signed char*>(ptr + L::kOffParent);
    const float scale = r.scale * kLog2e;
    int made = 0;
    auto group_sync = [&]() {
      if (s == 0) asm volatile("bar.sync 2, 128;" ::: "memory");
      else asm volatile("bar.sync 3, 128;" ::: "memory");
    };
    for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
      const int n_rb = (w.v.m + tokens - 1) / tokens, prefix = w.v.n - w.v.m;
      auto bring_lse = [&](int rb) {
        group_sync();
        const int rows = min(w.v.m - rb * tokens, tokens) * group;
        for (int i = key; i < (rows + 31) / 32 * 32; i += 128) {    // whole warps
          float x = INFINITY;        // a row that saw nothing, or is none, adds nothing
          if (i < rows) {
            const float y = r.lse[static_cast<int64_t>(w.v.row0 + rb * tokens + i / group) * r.Hq + sg.g * group + i % group];
            if (y != -INFINITY) x = y * kLog2e;
          }
          const uint32_t empty = __ballot_sync(0xffffffffu, x == INFINITY);
          if (lane == 0) none[i >> 5] = empty;
          lse[i] = x;
          token[i] = static_cast<uint8_t>(i / group);
        }
        group_sync();
      };
      // the nodes that see a node, itself and its descendants: every node enters itself with all its ancestors
      if (r.parents && sg.t1 * kKeys > prefix) {
        asm volatile("bar.sync 1, 256;" ::: "memory");
        for (int i = threadIdx.x; i < kMaxTreeNodes * 4; i += 256) down[i] = 0;
        if (static_cast<int>(threadIdx.x) < w.v.m) {
          const int p = r.parents[w.v.row0 + threadIdx.x];
          parents[threadIdx.x] = static_cast<signed char>(p < -1 || p >= static_cast<int>(threadIdx.x) ? -2 : p);
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (static_cast<int>(threadIdx.x) < w.v.m) {
          const int j = threadIdx.x;
          int a = j;
          while (a >= 0) a = parents[a];
          for (int b = j; a == -1 && b >= 0; b = parents[b]) atomicOr(&down[b * 4 + (j >> 5)], 1u << (j & 31));
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
      }
      if (n_rb == 1) bring_lse(0);
      for (int t = sg.t0; t < sg.t1; ++t) {
        const int x = t * kKeys + key;
        const bool node_tile = (t + 1) * kKeys > prefix;
        float sum = 0.f, old = 0.f;
        float* to = nullptr;
        // the tiles, or the blocks of rows of a tile, are taken in turn; with several blocks both groups have a part of a tile
        const bool mine = n_rb > 1 || (made & 1) == s;
        if (mine && x < w.v.n && (n_rb == 1 || s == 0)) {
          const int page = c.table[static_cast<int64_t>(sg.req) * c.table_stride + x / c.ps];
          if (page_exists(c, page)) {
            to = key_weights + (static_cast<int64_t>(page) * c.Hkv + sg.g) * c.ps + x % c.ps;
            old = *to;
          }
        }
        uint4 seen = make_uint4(0, 0, 0, 0);
        if (node_tile && x >= prefix && x < w.v.n && r.parents) seen = *reinterpret_cast<const uint4*>(down + (x - prefix) * 4);
        for (int rb = 0; rb < n_rb; ++rb, ++made) {
          if ((made & 1) != s) continue;
          const int rows = min(w.v.m - rb * tokens, tokens) * group;
          if (n_rb > 1) bring_lse(rb);
          if (!__all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_SFULL + s), (made >> 1) & 1, stop))) { *stop = 1; continue; }
          fence_after();
#pragma unroll 1
          for (int q = 0; q * 32 < rows; ++q) {
            float v[32];
            tmem_ld32(tmem_s + q * 32, v);
            const uint32_t empty = none[q];
            if (empty) {          // scores of rows that saw nothing, and columns beyond the rows, may be no numbers
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = (empty >> i) & 1u ? 0.f : v[i];
            }
            if (node_tile && x >= prefix) {
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const int j = rb * tokens + token[q * 32 + i];
                const uint32_t word = j < 32 ? seen.x : j < 64 ? seen.y : j < 96 ? seen.z : seen.w;
                const bool see = r.parents ? (word >> (j & 31)) & 1u : x - prefix <= j;
                if (see) sum += exp2_approx(fmaf(v[i], scale, -lse[q * 32 + i]));
              }
            } else {
              float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 z = *reinterpret_cast<const float4*>(lse + q * 32 + i);
                part[0] += exp2_approx(fmaf(v[i], scale, -z.x));
                part[1] += exp2_approx(fmaf(v[i + 1], scale, -z.y));
                part[2] += exp2_approx(fmaf(v[i + 2], scale, -z.z));
                part[3] += exp2_approx(fmaf(v[i + 3], scale, -z.w));
              }
              sum += (part[0] + part[1]) + (part[2] + part[3]);
            }
          }
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_SEMPTY + s));
        }
        if (n_rb > 1) {
          // the groups' parts of the tile's sums meet in the space of the descendants' neighbour, one float a key
          float* meet = reinterpret_cast<float*>(ptr + L::kOffLse) + kRows;    // the second group's rows: written again before their next use
          asm volatile("bar.sync 1, 256;" ::: "memory");
          if (s == 1) meet[key] = sum;
          asm volatile("bar.sync 1, 256;" ::: "memory");
          if (s == 0) sum += meet[key];
          asm volatile("bar.sync 1, 256;" ::: "memory");
        }
        if (to && !*stop) *to = old + sum;
      }
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

template <int H>
int launch_h(const PagedCache& c, const PagedRows& r, float* key_weights, cudaStream_t s) {
  static std::atomic<bool> configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!allow_shared(paged_weigh_kernel<H>, Wg<H>::kTotal, dev, configured)) return -1;
  CUtensorMap map_q, map_k;
  const int group = r.group;
  if (tma_map_bf16_heads(&map_q, r.q, r.T, r.Hq, H, r.q_stride, group, 128 / group)) return -1;
  if (tma_map_bf16_row_octets(&map_k, c.k, static_cast<long long>(c.n_pages) * c.Hkv * c.ps, H)) return -1;
  SLED_LAUNCH_PDL(paged_weigh_kernel<H>, dim3(sms), dim3(320), Wg<H>::kTotal, s, c, r, key_weights, map_q, map_k);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace

int launch_paged_weigh(const PagedCache& c, const PagedRows& r, float* key_weights, cudaStream_t s) {
  return c.h == 128 ? launch_h<128>(c, r, key_weights, s) : launch_h<64>(c, r, key_weights, s);
}

}  // namespace sled
