// Attention over a paged fp32 cache (CUDA cores; sums, products and probabilities all in fp32).
//
// Every warp has a share of the line of key tiles to itself and meets no other: a unit is up to 4 query rows of a KV head,
// a tile 32 keys.  K and V come in through a ring of the warp's own, 4 KB at a time, by 16-byte asynchronous copies, the next
// ones under the current one's arithmetic: K as 32 dimensions of the tile's keys, V as whole rows of some of them, so that
// neither loop knows which piece it has and the code stays short (a warp runs it a handful of times).  Scores: a lane has a
// key and all rows (the key's 16-byte parts are permuted against bank conflicts, the queries are broadcast).  Output: a lane
// has H / 32 neighbouring dimensions of all rows, the probabilities are broadcast.  With R rows a byte of cache meets R / 4
// multiply-adds: the bytes bind for single tokens, shared memory and the multiply-adds from about eight rows on.  Measured, 8
// KV heads of 128, 4 contexts of 16384 keys: 4 rows 110 us, 4.9 TB/s; 36 rows 699 us.
#include <algorithm>

#include "kernels.h"
#include "paged_schedule.cuh"
#include "warp_mma.cuh"

namespace sled {

namespace {

constexpr int kWarps = 4;
// Rows of a unit at most.  With 8: 24 short trees 34.8 us against 29.3, 4 contexts of 16384 keys with one token (4 rows) 187
// against 110, with 9 tokens 753 against 699.
constexpr int kRows = 4;
constexpr int kKeys = 32;          // of a tile
constexpr int kBuffers = 2;        // pieces under way or in use (with 3 the short trees took 30.4 us)
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

template <int H>
struct F32 {
  static constexpr int kDims = 32;                   // of a piece of K
  static constexpr int kPieces = H / kDims;          // of a tile's K, and of its V
  static constexpr int kVKeys = kKeys / kPieces;     // of a piece of V
  static constexpr int kBuffer = kKeys * kDims;      // floats
  static constexpr int kQ = kRows * H, kP = kRows * kKeys;
  static constexpr int kTree = kRows * (kMaxTreeNodes / 32) + kMaxTreeNodes / 4;
  static constexpr int kWarp = kBuffers * kBuffer + kQ + kP + kTree;
  static constexpr int kBytes = kWarps * kWarp * 4;
};

struct F32Parts {
  float* acc;      // [2 * shares][kRows][H]
  float* ml;       // [2 * shares][kRows][2]
  int4* desc;      // [shares][2]
  float* scores;   // null, or [rows][Hq][keys]
  int64_t keys;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {   // 0 where there is nothing
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}

// One stretch of a unit.
template <int H>
__device__ __forceinline__ void work_on(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, const ReqWork& w,
                                        const Segment& sg, const F32Parts& parts, float* mem) {
  using L = F32<H>;
  constexpr int R = kRows, PER = H / 32;         // dimensions of a lane
  const int lane = threadIdx.x & 31, group = r.group;
  float* buffers = mem;
  float* q = mem + kBuffers * L::kBuffer;
  float* p = q + L::kQ;
  uint32_t* tree = reinterpret_cast<uint32_t*>(p + L::kP);
  signed char* parents = reinterpret_cast<signed char*>(tree + kRows * (kMaxTreeNodes / 32));
  const int first = sg.rb * kRows;
  int rows, prefix, end;
  if (list_len > 0) {
    rows = min(kRows, group - first);
    const int x = w.v.n - w.v.m + sg.j, own = quotient(x, c.ps);
    end = (min(list_len, own + 1) - 1) * c.ps + x - own * c.ps + 1;
    prefix = end;
  } else {
    rows = min(kRows, w.v.m * group - first);
    end = w.v.n;
    prefix = w.v.n - w.v.m;
  }
  // row i's token and head within the group, from row to row
  const int token0 = list_len > 0 ? sg.j : first / group, head0 = list_len > 0 ? first : first - token0 * group;
  auto next_row = [&](int& token, int& head) {
    if (++head == group) {
      head = 0;
      ++token;
    }
  };
  const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
  const int32_t* mine = list_len > 0 ? list + (static_cast<int64_t>(w.v.row0 + sg.j) * c.Hkv + sg.g) * list_len : nullptr;
  const int cpp = c.ps / 16, groups = (end + 15) / 16, shift = (cpp & (cpp - 1)) == 0 ? __ffs(cpp) - 1 : -1;
  // where a tile's two groups of 16 keys begin, in keys of the pool, is found by lanes 0 and 1; the page's number is read a
  // tile before it is looked at
  auto block_of = [&](int t) {
    const int e = min(t * 2 + (lane & 1), groups - 1);
    return shift >= 0 ? e >> shift : e / cpp;
  };
  auto page_of = [&](int t) {
    const int b = block_of(t);
    return table[mine ? checked_block(c, mine[b]) : b];
  };
  auto locate = [&](int t, int page) {
    const int e = min(t * 2 + (lane & 1), groups - 1);
    return (checked_page(c, page) * c.Hkv + sg.g) * c.ps + (e - block_of(t) * cpp) * 16;
  };
  // the pieces in order, tile by tile those of K and then those of V, are fetched kBuffers - 1 ahead
  int ft = sg.t0, fn = 0, fbuf = 0, page = page_of(ft), next_page = page_of(ft + 1), at = 0;
  const bool nodes = r.parents && list_len <= 0;
  const int parent = nodes && lane < w.v.m ? r.parents[w.v.row0 + lane] : 0;
  __syncwarp();              // the segment before is done with this warp's memory
#pragma unroll 1
  for (int i = 0, token = token0, head = head0; i < R; ++i) {
    const float* src = reinterpret_cast<const float*>(r.q) + (w.v.row0 + token) * r.q_stride + static_cast<int64_t>(sg.g * group + head) * H;
#pragma unroll
    for (int d = 0; d < H; d += 32) copy4(smem_u32(q + i * H + d + lane), src + d + lane, i < rows);
    if (i + 1 < rows) next_row(token, head);
  }
  auto fetch = [&] {
    if (ft < sg.t1) {
      if (fn == 0) {
        at = locate(ft, page);
        page = next_page;
        next_page = page_of(ft + 2);
      }
      const bool is_v = fn >= L::kPieces;
      constexpr int kVShift = H == 128 ? 5 : H == 64 ? 4 : 3;
      const int chunk_shift = is_v ? kVShift : 3, key0 = is_v ? (fn - L::kPieces) * L::kVKeys : 0;   // 16-byte parts of a row
      const float* pool = reinterpret_cast<const float*>(is_v ? c.v : c.k) + (is_v ? 0 : fn * L::kDims);
      const uint32_t dst = smem_u32(buffers + fbuf * L::kBuffer);
      const int ch = lane & ((1 << chunk_shift) - 1), step = 32 >> chunk_shift;
      const int64_t g0 = __shfl_sync(0xffffffffu, at, 0), g1 = __shfl_sync(0xffffffffu, at, 1) - 16;
      int key = key0 + (lane >> chunk_shift);
#pragma unroll 4
      for (int i = 0; i < L::kBuffer / 128; ++i) {
        const int part = is_v ? i * 32 + lane : (i * 32 + lane) ^ (key & 7);
        copy16(dst + part * 16, pool + ((key < 16 ? g0 : g1) + key) * H + ch * 4, ft * kKeys + key < end);
        key += step;
      }
      if (++fn == 2 * L::kPieces) {
        fn = 0;
        ++ft;
      }
      if (++fbuf == kBuffers) fbuf = 0;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll 1
  for (int i = 0; i < kBuffers - 1; ++i) fetch();
  bool dead = false;         // of row `lane`
  if (nodes) {
    for (int i = lane; i < w.v.m; i += 32) {
      const int x = i == lane ? parent : r.parents[w.v.row0 + i];
      if (x < -2 || x >= i) set_status(c.status, SLED_ERR_ARG);
      parents[i] = static_cast<signed char>(x < -1 || x >= i ? -2 : x);
    }
    __syncwarp();
    if (lane < rows) {
      uint32_t bits[kMaxTreeNodes / 32] = {};
      int a = (first + lane) / group;
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
#pragma unroll 1
  for (int t = sg.t0; t < sg.t1; ++t) {
    float s[R];
#pragma unroll
    for (int i = 0; i < R; ++i) s[i] = 0.f;
    const int x = t * kKeys + lane;
    const bool masked = (t + 1) * kKeys > prefix;
#pragma unroll 1
    for (int n = 0; n < 2 * L::kPieces; ++n) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kBuffers - 2) : "memory");
      __syncwarp();
      fetch();             // into the buffer of the piece before, which everybody has left
      const float* piece = buffers + buffer * L::kBuffer;
      if (++buffer == kBuffers) buffer = 0;
      if (n < L::kPieces) {
        const float* qn = q + n * L::kDims;
#pragma unroll 2
        for (int d = 0; d < L::kDims / 4; ++d) {
          const float4 k4 = *reinterpret_cast<const float4*>(piece + lane * L::kDims + (d ^ (lane & 7)) * 4);
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float4 q4 = *reinterpret_cast<const float4*>(qn + i * H + d * 4);
            s[i] = fmaf(q4.x, k4.x, s[i]);
            s[i] = fmaf(q4.y, k4.y, s[i]);
            s[i] = fmaf(q4.z, k4.z, s[i]);
            s[i] = fmaf(q4.w, k4.w, s[i]);
          }
        }
        if (n + 1 == L::kPieces) {
          int token = token0, head = head0;
#pragma unroll
          for (int i = 0; i < R; ++i) {
            s[i] *= scale;
            if (masked) {
              bool see = x < end;
              if (see && x >= prefix) {
                const int a = x - prefix;
                if (nodes) see = (tree[i * (kMaxTreeNodes / 32) + (a >> 5)] >> (a & 31)) & 1u;
                else if (list_len <= 0) see = a <= token;
              }
              if (!see) s[i] = -INFINITY;
            }
            if (parts.scores && i < rows && x < end)
              parts.scores[(static_cast<int64_t>(w.v.row0 + token) * r.Hq + sg.g * group + head) * parts.keys + x] = s[i];
            next_row(token, head);
            const float top = fmaxf(m[i], warp_max(s[i])), ref = top == -INFINITY ? 0.f : top;
            const float f = exp2f(m[i] - ref), pi = exp2f(s[i] - ref);
            m[i] = top;
            l[i] = l[i] * f + pi;              // of this lane's keys
#pragma unroll
            for (int d = 0; d < PER; ++d) o[i][d] *= f;
            p[i * kKeys + lane] = pi;
          }
          __syncwarp();
        }
      } else {
        const float* pn = p + (n - L::kPieces) * L::kVKeys;
#pragma unroll 1
        for (int key = 0; key < L::kVKeys; key += 4) {
          float v[4][PER];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float* src = piece + (key + e) * H + lane * PER;
            if constexpr (PER == 4) {
              const float4 y = *reinterpret_cast<const float4*>(src);
              v[e][0] = y.x; v[e][1] = y.y; v[e][2] = y.z; v[e][3] = y.w;
            } else if constexpr (PER == 2) {
              const float2 y = *reinterpret_cast<const float2*>(src);
              v[e][0] = y.x; v[e][1] = y.y;
            } else {
              v[e][0] = *src;
            }
          }
          // a probability of 0 does not silence a value that is not finite: such keys are left out where they are masked
          bool finite = true;
          if (masked)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int d = 0; d < PER; ++d) finite = finite && fabsf(v[e][d]) < INFINITY;
          if (finite) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
              const float4 p4 = *reinterpret_cast<const float4*>(pn + i * kKeys + key);
#pragma unroll
              for (int d = 0; d < PER; ++d) {
                o[i][d] = fmaf(p4.x, v[0][d], o[i][d]);
                o[i][d] = fmaf(p4.y, v[1][d], o[i][d]);
                o[i][d] = fmaf(p4.z, v[2][d], o[i][d]);
                o[i][d] = fmaf(p4.w, v[3][d], o[i][d]);
              }
            }
          } else {
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll 1
              for (int e = 0; e < 4; ++e) {
                const float pe = pn[i * kKeys + key + e];
                if (pe == 0.f) continue;
#pragma unroll
                for (int d = 0; d < PER; ++d) o[i][d] = fmaf(pe, piece[(key + e) * H + lane * PER + d], o[i][d]);
              }
          }
        }
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");

  int token = token0, head = head0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i >= rows) break;
    float sum = warp_sum(l[i]), top = m[i];
    const bool none = (dead_rows >> i) & 1u;
    if (none) { sum = 0.f; top = -INFINITY; }
    const int64_t t_row = w.v.row0 + token;
    const int h_row = sg.g * group + head;
    next_row(token, head);
    float* dst;
    float f = 1.f;
    if (sg.whole) {
      dst = reinterpret_cast<float*>(r.out) + t_row * r.out_stride + static_cast<int64_t>(h_row) * H;
      f = sum == 0.f ? 0.f : 1.f / sum;
      if (r.lse && lane == 0) r.lse[t_row * r.Hq + h_row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    } else {
      dst = parts.acc + (static_cast<int64_t>(sg.slot) * kRows + i) * H;
      if (lane == 0) *reinterpret_cast<float2*>(parts.ml + (static_cast<int64_t>(sg.slot) * kRows + i) * 2) = make_float2(top, sum);
    }
#pragma unroll
    for (int d = 0; d < PER; ++d) dst[lane * PER + d] = none ? 0.f : o[i][d] * f;
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
  if ((threadIdx.x & 31) == 0) leave_none(parts.desc, mine);
  float* mem = smem + warp * F32<H>::kWarp;
  for_segments(line, shares[warp], mine, [&](const ReqWork& w, const Segment& sg) {
    work_on<H>(c, r, list, list_len, w, sg, parts, mem);
    if (sg.last_block >= 0 && (threadIdx.x & 31) == 0) {
      const int first = sg.rb * kRows, group = r.group;
      leave_cut(parts.desc, mine, sg, w.v.row0, w.v.m, list_len > 0 ? sg.j : -1, first, min(kRows, (list_len > 0 ? group : w.v.m * group) - first));
    }
  });
}

constexpr int kPerSm = 4;                     // blocks at most
constexpr int kMaxShares = kMaxPagedBlocks / 2 * kPerSm * kWarps;

template <int H>
int launch_h(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* scores, char* ws, cudaStream_t s) {
  static std::atomic<bool> configured[kMaxDevices] = {};
  int sms = 0;
  const int dev = paged_device(&sms);
  if (dev < 0) return -1;
  if (!allow_shared(paged_f32_kernel<H>, F32<H>::kBytes, dev, configured)) return -1;
  constexpr int kResident = std::min(kPerSm, 227 * 1024 / (F32<H>::kBytes + 1024));   // as many as shared memory holds
  const int blocks = min(kResident * sms, kMaxShares / kWarps);
  F32Parts parts;
  parts.acc = reinterpret_cast<float*>(ws);
  parts.ml = parts.acc + 2LL * kMaxShares * kRows * H;
  parts.desc = reinterpret_cast<int4*>(parts.ml + 2LL * kMaxShares * kRows * 2);
  parts.scores = scores;
  parts.keys = static_cast<int64_t>(c.table_cols) * c.ps;
  SLED_LAUNCH_PDL(paged_f32_kernel<H>, dim3(blocks), dim3(32 * kWarps), F32<H>::kBytes, s, c, r, list, list_len, parts);
  if (cudaGetLastError() != cudaSuccess) return -1;
  const int n = launch_paged_merge(c, r, kRows, blocks * kWarps, parts.acc, parts.ml, parts.desc, s);
  return n < 0 ? n : n + 1;
}

}  // namespace

int64_t paged_f32_workspace(int h) { return 2LL * kMaxShares * kRows * (h + 2) * 4 + kMaxShares * 32LL; }

int launch_paged_f32(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* scores, char* ws, cudaStream_t s) {
  if (c.h == 128) return launch_h<128>(c, r, list, list_len, scores, ws, s);
  return c.h == 64 ? launch_h<64>(c, r, list, list_len, scores, ws, s) : launch_h<32>(c, r, list, list_len, scores, ws, s);
}

}  // namespace sled
