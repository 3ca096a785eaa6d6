// Attention over a paged fp32 cache (CUDA cores; sums, products and probabilities all in fp32).
//
// Every warp has a share of the line of key tiles to itself and meets no other: a unit is up to 4 query rows of a KV head,
// a tile 32 keys.  K and V come in through two buffers of the warp's own, 32 keys x 32 dimensions at a time, by
// 16-byte asynchronous copies, the next one under the current one's arithmetic.  Scores: a lane has a key and all rows
// (its key's row is padded against bank conflicts, the queries are broadcast).  Output: a lane has one of
// a piece's dimensions of all rows, the probabilities are broadcast.  With R rows a byte of cache meets R / 4 multiply-adds: the
// bytes bind for single tokens, shared memory and the multiply-adds from about eight rows on.
#include "kernels.h"
#include "paged_schedule.cuh"
#include "warp_mma.cuh"

namespace sled {

namespace {

constexpr int kWarps = 4;
constexpr int kRows = 4;           // of a unit at most (with more a warp's code is longer than its first run is worth, and there are fewer warps)
constexpr int kKeys = 32;          // of a tile
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

template <int H>
struct F32 {
  static constexpr int kDims = 32;                   // of a piece of K or V
  static constexpr int kPieces = H / kDims;
  static constexpr int kPitch = kDims + 4;
  static constexpr int kBuffer = kKeys * kPitch;     // floats
  static constexpr int kQ = kRows * H, kP = kRows * kKeys;
  static constexpr int kTree = kRows * (kMaxTreeNodes / 32) + kMaxTreeNodes / 4;
  static constexpr int kWarp = 2 * kBuffer + kQ + kP + kTree;
  static constexpr int kBytes = kWarps * kWarp * 4;
};

struct F32Parts {
  float* acc;      // [2 * shares][kRows][H]
  float* ml;       // [2 * shares][kRows][2]
  int4* desc;      // [shares]
  float* scores;   // null, or [rows][Hq][keys]
  int64_t keys;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {   // 0 where there is nothing
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// One stretch of a unit.
template <int H>
__device__ __forceinline__ void work_on(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, const ReqWork& w,
                                        const Segment& sg, const F32Parts& parts, float* mem) {
  using L = F32<H>;
  constexpr int R = kRows, PER = 1;              // dimensions of a lane in a piece
  const int lane = threadIdx.x & 31, group = r.Hq / c.Hkv;
  float* buffers = mem;
  float* q = mem + 2 * L::kBuffer;
  float* p = q + L::kQ;
  uint32_t* tree = reinterpret_cast<uint32_t*>(p + L::kP);
  signed char* parents = reinterpret_cast<signed char*>(tree + kRows * (kMaxTreeNodes / 32));
  const int first = sg.rb * kRows;
  int rows, prefix, end;
  if (list_len > 0) {
    rows = min(kRows, group - first);
    const int x = w.v.n - w.v.m + sg.j, own = x / c.ps;
    end = (min(list_len, own + 1) - 1) * c.ps + x - own * c.ps + 1;
    prefix = end;
  } else {
    rows = min(kRows, w.v.m * group - first);
    end = w.v.n;
    prefix = w.v.n - w.v.m;
  }
  auto token = [&](int i) { return list_len > 0 ? sg.j : (first + i) / group; };
  auto head = [&](int i) { return sg.g * group + (first + i) % group; };
  __syncwarp();
#pragma unroll 1
  for (int i = 0; i < R; ++i) {
    const float* src = reinterpret_cast<const float*>(r.q) + (w.v.row0 + token(min(i, rows - 1))) * r.q_stride + static_cast<int64_t>(head(min(i, rows - 1))) * H;
#pragma unroll
    for (int d = 0; d < H / 32; ++d) q[i * H + d * 32 + lane] = i < rows ? src[d * 32 + lane] : 0.f;
  }
  const bool nodes = r.parents && list_len <= 0;
  bool dead = false;         // of row `lane`
  if (nodes) {
    for (int i = lane; i < w.v.m; i += 32) {
      const int x = r.parents[w.v.row0 + i];
      if (x < -2 || x >= i) set_status(c.status, SLED_ERR_ARG);
      parents[i] = static_cast<signed char>(x < -1 || x >= i ? -2 : x);
    }
    __syncwarp();
    if (lane < rows) {
      uint32_t bits[kMaxTreeNodes / 32] = {};
      int a = token(lane);
      while (a >= 0) {
#pragma unroll
        for (int k = 0; k < kMaxTreeNodes / 32; ++k)
          if (k == (a >> 5)) bits[k] |= 1u << (a & 31);
        a = parents[a];
      }
      dead = a == -2;
#pragma unroll
      for (int k = 0; k < kMaxTreeNodes / 32; ++k) tree[lane * (kMaxTreeNodes / 32) + k] = dead ? 0u : bits[k];
    }
  }
  __syncwarp();
  const uint32_t dead_rows = __ballot_sync(0xffffffffu, dead);

  const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
  const int32_t* mine = list_len > 0 ? list + (static_cast<int64_t>(w.v.row0 + sg.j) * c.Hkv + sg.g) * list_len : nullptr;
  const int cpp = c.ps / 16, groups = (end + 15) / 16;
  // where the tile's two groups of 16 keys begin, in keys of the pool; found by lanes 0 and 1
  auto locate = [&](int t) {
    int at = 0;
    const int e = t * 2 + (lane & 1);
    if (e < groups) {
      const int b = e / cpp;
      at = (checked_page(c, table[mine ? mine[b] : b]) * c.Hkv + sg.g) * c.ps + (e - b * cpp) * 16;
    }
    return at;
  };
  int at = locate(sg.t0), at_next = 0;
  // piece n of tile t: the pieces of K, then those of V
  auto fetch = [&](int t, int n, int where, int buffer) {
    const float* pool = reinterpret_cast<const float*>(n < L::kPieces ? c.k : c.v) + n % L::kPieces * L::kDims;
    const uint32_t dst = smem_u32(buffers + buffer * L::kBuffer);
    constexpr int kChunks = L::kDims / 4;        // 16-byte pieces of a row
#pragma unroll 4
    for (int i = 0; i < kChunks; ++i) {
      const int e = i * 32 + lane, key = e / kChunks, ch = e % kChunks;
      const int g0 = __shfl_sync(0xffffffffu, where, 0), g1 = __shfl_sync(0xffffffffu, where, 1);
      const int64_t row = static_cast<int64_t>(key < 16 ? g0 : g1) + (key & 15);
      copy16(dst + (key * L::kPitch + ch * 4) * 4, pool + row * H + ch * 4, t * kKeys + key < end);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  float m[R], l[R], o[R][H / 32];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < H / 32; ++d) o[i][d] = 0.f;
  }
  const float scale = r.scale * kLog2e;
  int buffer = 0;
  fetch(sg.t0, 0, at, 0);
  for (int t = sg.t0; t < sg.t1; ++t) {
    if (t + 1 < sg.t1) at_next = locate(t + 1);
    float s[R];
#pragma unroll
    for (int i = 0; i < R; ++i) s[i] = 0.f;
    const int x = t * kKeys + lane;
    const bool masked = (t + 1) * kKeys > prefix;
#pragma unroll
    for (int n = 0; n < 2 * L::kPieces; ++n) {
      // the next piece goes into the other buffer, which everybody has left
      __syncwarp();
      const bool last = n + 1 == 2 * L::kPieces;
      if (!last) fetch(t, n + 1, at, buffer ^ 1);
      else if (t + 1 < sg.t1) fetch(t + 1, 0, at_next, buffer ^ 1);
      else asm volatile("cp.async.commit_group;" ::: "memory");
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      __syncwarp();
      const float* piece = buffers + buffer * L::kBuffer;
      if (n < L::kPieces) {
        const float* qn = q + n * L::kDims;
#pragma unroll 2
        for (int d = 0; d < L::kDims; d += 4) {
          const float4 k4 = *reinterpret_cast<const float4*>(piece + lane * L::kPitch + d);
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float4 q4 = *reinterpret_cast<const float4*>(qn + i * H + d);
            s[i] = fmaf(q4.x, k4.x, s[i]);
            s[i] = fmaf(q4.y, k4.y, s[i]);
            s[i] = fmaf(q4.z, k4.z, s[i]);
            s[i] = fmaf(q4.w, k4.w, s[i]);
          }
        }
        if (n + 1 == L::kPieces) {
#pragma unroll
          for (int i = 0; i < R; ++i) {
            s[i] *= scale;
            if (masked) {
              bool see = x < end;
              if (see && x >= prefix) {
                const int a = x - prefix;
                if (nodes) see = (tree[i * (kMaxTreeNodes / 32) + (a >> 5)] >> (a & 31)) & 1u;
                else if (list_len <= 0) see = a <= token(i);
              }
              if (!see) s[i] = -INFINITY;
            }
            if (parts.scores && i < rows && x < end)
              parts.scores[(static_cast<int64_t>(w.v.row0 + token(i)) * r.Hq + head(i)) * parts.keys + x] = s[i];
            const float top = fmaxf(m[i], warp_max(s[i])), ref = top == -INFINITY ? 0.f : top;
            const float f = exp2f(m[i] - ref), pi = exp2f(s[i] - ref);
            m[i] = top;
            l[i] = l[i] * f + pi;              // of this lane's keys
#pragma unroll
            for (int d = 0; d < H / 32; ++d) o[i][d] *= f;
            p[i * kKeys + lane] = pi;
          }
          __syncwarp();
        }
      } else {
#pragma unroll 1
        for (int key = 0; key < kKeys; key += 4) {
          float v[4][PER];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e][0] = piece[(key + e) * L::kPitch + lane];
          }
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float4 p4 = *reinterpret_cast<const float4*>(p + i * kKeys + key);
            const float pe[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int d = 0; d < PER; ++d) {
                // (n is a constant of the unrolled loop: so is the place in o)
                float& y = o[i][(n - L::kPieces) * PER + d];
                // a probability of 0 does not silence a value that is not finite
                if (masked) y = pe[e] != 0.f ? fmaf(pe[e], v[e][d], y) : y;
                else y = fmaf(pe[e], v[e][d], y);
              }
          }
        }
      }
      buffer ^= 1;
    }
    at = at_next;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");

#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i >= rows) break;
    float sum = warp_sum(l[i]), top = m[i];
    const bool none = (dead_rows >> i) & 1u;
    if (none) { sum = 0.f; top = -INFINITY; }
    const int64_t t_row = w.v.row0 + token(i);
    float* dst;
    float f = 1.f;
    if (sg.whole) {
      dst = reinterpret_cast<float*>(r.out) + t_row * r.out_stride + static_cast<int64_t>(head(i)) * H;
      f = sum == 0.f ? 0.f : 1.f / sum;
      if (r.lse && lane == 0) r.lse[t_row * r.Hq + head(i)] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    } else {
      dst = parts.acc + (static_cast<int64_t>(sg.slot) * kRows + i) * H;
      if (lane == 0) *reinterpret_cast<float2*>(parts.ml + (static_cast<int64_t>(sg.slot) * kRows + i) * 2) = make_float2(top, sum);
    }
#pragma unroll
    for (int n = 0; n < L::kPieces; ++n)
#pragma unroll
      for (int d = 0; d < PER; ++d) dst[n * L::kDims + lane * PER + d] = none ? 0.f : o[i][n * PER + d] * f;
  }
}

template <int H>
__global__ void __launch_bounds__(32 * kWarps) paged_f32_kernel(const PagedCache c, const PagedRows r, const int32_t* list, int list_len,
                                                                const F32Parts parts) {
  extern __shared__ __align__(16) float smem[];
  __shared__ Share shares[kWarps];
  pdl_launch_dependents();
  pdl_wait();
  const AttentionLine line{c, r, list_len, kRows, kKeys};
  block_shares<kWarps>(line, blockIdx.x * kWarps, gridDim.x * kWarps, shares);
  const int warp = threadIdx.x >> 5, mine = blockIdx.x * kWarps + warp;
  if ((threadIdx.x & 31) == 0) parts.desc[mine] = make_int4(-1, 0, 0, 0);
  float* mem = smem + warp * F32<H>::kWarp;
  for_segments(line, shares[warp], mine, [&](const ReqWork& w, const Segment& sg) {
    work_on<H>(c, r, list, list_len, w, sg, parts, mem);
    if (sg.last_block >= 0 && (threadIdx.x & 31) == 0) {
      const int unit = (list_len > 0 ? sg.j * c.Hkv + sg.g : sg.g) * w.n_rb + sg.rb;
      parts.desc[mine] = make_int4(sg.last_block, sg.slot, sg.req, unit);
    }
  });
}

constexpr int kMaxDevices = 64;
constexpr int kPerSm = 4;                     // blocks (shared memory holds five, or four with head_dim 128)
constexpr int kMaxShares = kMaxPagedBlocks / 2 * kPerSm * kWarps;

template <int H>
int launch_h(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* scores, char* ws, cudaStream_t s) {
  static bool configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!configured[dev]) {
    if (cudaFuncSetAttribute(paged_f32_kernel<H>, cudaFuncAttributeMaxDynamicSharedMemorySize, F32<H>::kBytes) != cudaSuccess) return -1;
    configured[dev] = true;
  }
  const int blocks = min(kPerSm * sms, kMaxShares / kWarps);
  F32Parts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + 2LL * kMaxShares * kRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + 2LL * kMaxShares * kRows * 2);
  parts.scores = scores;
  parts.keys = static_cast<int64_t>(c.table_cols) * c.ps;
  SLED_LAUNCH_PDL(paged_f32_kernel<H>, dim3(blocks), dim3(32 * kWarps), F32<H>::kBytes, s, c, r, list, list_len, parts);
  if (cudaGetLastError() != cudaSuccess) return -1;
  const int n = launch_paged_merge(c, r, list_len, kRows, kKeys, blocks * kWarps, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int64_t paged_f32_workspace(int h) { return 2LL * kMaxShares * kRows * (h + 2) * 4 + kMaxShares * 16LL; }

int launch_paged_f32(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* scores, char* ws, cudaStream_t s) {
  if (c.h == 128) return launch_h<128>(c, r, list, list_len, scores, ws, s);
  return c.h == 64 ? launch_h<64>(c, r, list, list_len, scores, ws, s) : launch_h<32>(c, r, list, list_len, scores, ws, s);
}

}  // namespace sled
