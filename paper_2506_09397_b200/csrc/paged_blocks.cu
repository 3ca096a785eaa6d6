// Bounds of the keys of every block (page) of a cache, and the choice of the blocks that a query attends to.
//
// bounds[page][kv head][0/1][d] = smallest / largest k_d over the block's keys.  For a query q every key of the block has
// q.k <= sum_d max(q_d low_d, q_d high_d) (= sum_d max(q_d, 0) high_d + min(q_d, 0) low_d where all of them are finite):
// the block's score for that query, the largest over the heads that share the KV head.  A query reads the n_local blocks
// that end with its own and, of the earlier ones, those of largest score, the lower block first among equals.  Scores are
// fp32 sums.
#include <algorithm>

#include "paged_schedule.cuh"
#include "warp_mma.cuh"

namespace sled {

namespace {

// Blocks whose bounds are asked for, for units of a KV head: a tile is a block.
struct BoundsLine {
  const PagedCache& c;
  const int32_t* first;
  __device__ __forceinline__ int32_t fault(const ReqView&) const { return SLED_ERR_ARG; }
  __device__ __forceinline__ int min_share() const { return 8; }   // a block gets work for all its warps, at least
  __device__ __forceinline__ int from(int i) const { return first ? max(0, first[i]) / c.ps : 0; }
  __device__ __forceinline__ ReqWork operator()(int i) const {
    ReqWork w;
    w.v.n = c.n_kv[i];
    w.v.m = w.v.row0 = 0;
    w.v.ok = w.v.n >= 0 && w.v.n <= static_cast<int64_t>(c.table_cols) * c.ps;
    w.n_rb = 1;
    w.tiles = w.v.ok ? max(0, (w.v.n + c.ps - 1) / c.ps - from(i)) : 0;
    w.units = w.tiles && !(first && first[i] >= w.v.n) ? c.Hkv : 0;     // nothing where there are no new keys, in a page partly filled either
    w.weight = 1;
    return w;
  }
};

template <typename T> struct Vec;           // 16 bytes of keys
template <> struct Vec<float> {
  static constexpr int kElems = 4, kWords = 4;
  static __device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) {
    const float x = __uint_as_float(a), y = __uint_as_float(b);
    return __float_as_uint(x != x || y != y ? NAN : fminf(x, y));
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    const float x = __uint_as_float(a), y = __uint_as_float(b);
    return __float_as_uint(x != x || y != y ? NAN : fmaxf(x, y));
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int kElems = 8, kWords = 4;
  static __device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmin2_nan(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
};

// A warp per (block, KV head): the lanes take 16 bytes each, kRows rows at a time, four such loads under way; every key is
// read once, which is what bounds it: 24 prompts of 2000 .. 16384 keys, 8 KV heads of 128, 65 us, 88 % of the copy rate, with
// four blocks an SM (two 85 us, six 74, eight 68).
template <typename T, int H>
__global__ void __launch_bounds__(256) block_bounds_kernel(PagedCache c, const int32_t* first, T* bounds) {
  using V = Vec<T>;
  constexpr int kLanes = H / V::kElems, kRows = 32 / kLanes;   // lanes of a key row; rows that a warp reads at once
  pdl_launch_dependents();
  pdl_wait();
  const BoundsLine line{c, first};
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (share.from >= share.to) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = lane % kLanes, sub = lane / kLanes;
  for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
    const int from = line.from(sg.req);
    for (int t = sg.t0 + warp; t < sg.t1; t += 8) {
      const int b = from + t, page = c.table[static_cast<int64_t>(sg.req) * c.table_stride + b];
      if (!page_exists(c, page)) {
        if (lane == 0) set_status(c.status, SLED_ERR_ARG);
        continue;
      }
      const int count = min(c.ps, w.v.n - b * c.ps);
      const uint4* k = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(c.k) + (static_cast<int64_t>(page) * c.Hkv + sg.g) * c.ps * H) + col;
      uint32_t lo[4], hi[4];
      {
        const uint4 x = k[min(sub, count - 1) * kLanes];      // rows behind the last key repeat it
        lo[0] = hi[0] = x.x; lo[1] = hi[1] = x.y; lo[2] = hi[2] = x.z; lo[3] = hi[3] = x.w;
      }
      for (int e = 0; e < count; e += 4 * kRows) {
        uint4 x[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) x[z] = k[min(e + z * kRows + sub, count - 1) * kLanes];
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          lo[0] = V::smaller(lo[0], x[z].x); lo[1] = V::smaller(lo[1], x[z].y); lo[2] = V::smaller(lo[2], x[z].z); lo[3] = V::smaller(lo[3], x[z].w);
          hi[0] = V::larger(hi[0], x[z].x); hi[1] = V::larger(hi[1], x[z].y); hi[2] = V::larger(hi[2], x[z].z); hi[3] = V::larger(hi[3], x[z].w);
        }
      }
#pragma unroll
      for (int o = kLanes; o < 32; o <<= 1)
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          lo[z] = V::smaller(lo[z], __shfl_xor_sync(0xffffffffu, lo[z], o));
          hi[z] = V::larger(hi[z], __shfl_xor_sync(0xffffffffu, hi[z], o));
        }
      if (sub == 0) {
        uint4* out = reinterpret_cast<uint4*>(bounds + (static_cast<int64_t>(page) * c.Hkv + sg.g) * 2 * H) + col;
        out[0] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        out[kLanes] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      }
    }
  });
}

// the larger of two scores; a NaN is the largest
__device__ __forceinline__ float larger(float a, float b) { return a != a || b != b ? NAN : fmaxf(a, b); }

// The score by its definition, for one query and block: bounds or queries that are not finite take this way, since on the
// tensor cores the zeros of min(q, 0) and max(q, 0) meet the bound that does not count, and 0 times infinity is no number.
template <typename T, int H>
__device__ __noinline__ float score_of(const T* q, const T* low) {
  float s = 0.f;
#pragma unroll 1
  for (int d = 0; d < H; ++d) {
    const float x = to_f32(q[d]);
    s += larger(x * to_f32(low[d]), x * to_f32(low[H + d]));
  }
  return s;
}

constexpr int kScoreRows = 48;

// Earlier blocks of a request's tokens, in tiles of 64, for units of (KV head, up to 48 rows); nothing where all blocks of
// the request's last token are read anyway.
struct ScoreLine {
  const PagedCache& c;
  const PagedRows& r;
  int n_blocks, n_local;
  __device__ __forceinline__ int32_t fault(const ReqView& v) const { return req_fault(r, v); }
  __device__ __forceinline__ int min_share() const { return 1; }
  __device__ __forceinline__ int tokens() const { return max(1, kScoreRows / (r.group)); }   // of a unit
  __device__ __forceinline__ ReqWork operator()(int i) const {
    ReqWork w;
    w.v = req_view(c, r, i);
    w.tiles = w.units = w.n_rb = 0;
    w.weight = 1;
    if (!w.v.ok || w.v.m == 0) return w;
    const int blocks = (w.v.n - 1) / c.ps + 1;
    if (blocks <= n_blocks || n_blocks == n_local) return w;
    w.tiles = (blocks - n_local + 63) / 64;
    w.n_rb = (w.v.m + tokens() - 1) / tokens();
    w.units = w.n_rb * c.Hkv;
    w.weight = 1;
    return w;
  }
};

// Scores on the tensor cores: rows [min(q, 0), max(q, 0)] against the bounds as they lie in memory, [low, high], a
// contraction over 2 H.  The order of the terms is free, so a thread takes 16 consecutive bytes of a row as two
// instructions' operands (both sides alike) and the bounds go from memory straight into registers, a tile ahead.  A warp
// has 16 of the tile's 64 blocks and all the unit's rows; the maximum over a group's heads is taken in shared memory.
// Bound by the bytes of the bounds, 4 H per block and KV head, and by how little there is: 60 MB in 25 us (2.4 TB/s), one
// context of 30000 keys in 9 us.
template <int H>
__global__ void __launch_bounds__(128, 3) block_score_kernel(PagedCache c, PagedRows r, const __nv_bfloat16* bounds, int n_blocks,
                                                             int n_local, float* scores) {
  constexpr int kRow = 2 * H + 8;                  // padded: eight rows' 16-byte pieces meet no bank twice
  constexpr int kPieces = H / 16;                  // 32 terms each
  __shared__ __align__(16) __nv_bfloat16 qs[kScoreRows * kRow];
  __shared__ float tile[kScoreRows][65];
  pdl_launch_dependents();
  pdl_wait();
  const ScoreLine line{c, r, n_blocks, n_local};
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (share.from >= share.to) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, tq = lane & 3, group = r.group;
  const bool wide_q = (reinterpret_cast<uintptr_t>(r.q) & 15) == 0 && r.q_stride % 8 == 0;
  for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) {
    const int j0 = sg.rb * line.tokens(), nj = min(line.tokens(), w.v.m - j0), rows = nj * group;
    const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
    const int early = (w.v.n - 1) / c.ps + 1 - n_local;
    uint4 bb[2][kPieces];                          // this thread's quarters of the bounds of two blocks
    auto fetch = [&](int t) {
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
        const int b = t * 64 + warp * 16 + nt * 8 + gq;
        const bool there = b < early;
        const uint4* src = reinterpret_cast<const uint4*>(bounds) + tq;
        if (there) src += (static_cast<int64_t>(checked_page(c, table[b])) * c.Hkv + sg.g) * (2 * H / 8);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) bb[nt][k] = there ? src[4 * k] : make_uint4(0, 0, 0, 0);
      }
    };
    fetch(sg.t0);
    __syncthreads();
    uint32_t found = 0;        // all ones in an exponent carry into bit 15 or 31
    {
      // the rows as the two halves of the contraction, all loads under way at once
      constexpr int kVecs = kScoreRows * (H / 8) / 128;
      uint4 x[kVecs];
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int e = i * 128 + threadIdx.x, row = e / (H / 8), d = e % (H / 8);
        x[i] = make_uint4(0, 0, 0, 0);
        if (row < rows) {
          const uint32_t* src = reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(r.q) + (w.v.row0 + j0 + row / group) * r.q_stride +
                                                                  static_cast<int64_t>(sg.g * group + row % group) * H) + 4 * d;
          if (wide_q) x[i] = *reinterpret_cast<const uint4*>(src);
          else x[i] = make_uint4(src[0], src[1], src[2], src[3]);
        }
      }
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int e = i * 128 + threadIdx.x, row = e / (H / 8), d = e % (H / 8);
        const uint32_t in[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        uint32_t low[4], high[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          found |= (in[k] & 0x7f807f80u) + 0x00800080u;
          low[k] = Vec<__nv_bfloat16>::smaller(in[k], 0u);
          high[k] = Vec<__nv_bfloat16>::larger(in[k], 0u);
        }
        *reinterpret_cast<uint4*>(qs + row * kRow + 8 * d) = make_uint4(low[0], low[1], low[2], low[3]);
        *reinterpret_cast<uint4*>(qs + row * kRow + H + 8 * d) = make_uint4(high[0], high[1], high[2], high[3]);
      }
    }
    const bool odd = __syncthreads_or((found & 0x80008000u) != 0);   // a query that is not finite
    for (int t = sg.t0; t < sg.t1; ++t) {
#pragma unroll 1
      for (int mt = 0; mt * 16 < rows; ++mt) {
        float s[2][4] = {};
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
          const uint4 lo = *reinterpret_cast<const uint4*>(qs + (mt * 16 + gq) * kRow + k * 32 + tq * 8);
          const uint4 hi = *reinterpret_cast<const uint4*>(qs + (mt * 16 + gq + 8) * kRow + k * 32 + tq * 8);
          const uint32_t a0[4] = {lo.x, hi.x, lo.y, hi.y}, a1[4] = {lo.z, hi.z, lo.w, hi.w};
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            mma_bf16(s[nt], a0, bb[nt][k].x, bb[nt][k].y);
            mma_bf16(s[nt], a1, bb[nt][k].z, bb[nt][k].w);
          }
        }
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          const int col = warp * 16 + nt * 8 + 2 * tq;
          tile[mt * 16 + gq][col] = s[nt][0];
          tile[mt * 16 + gq][col + 1] = s[nt][1];
          tile[mt * 16 + gq + 8][col] = s[nt][2];
          tile[mt * 16 + gq + 8][col + 1] = s[nt][3];
        }
      }
      if (t + 1 < sg.t1) fetch(t + 1);
      __syncthreads();
      for (int e = threadIdx.x; e < nj * 64; e += 128) {
        const int j = e >> 6, col = e & 63, b = t * 64 + col;
        float best = tile[j * group][col];
        for (int hh = 1; hh < group; ++hh) best = larger(best, tile[j * group + hh][col]);
        if ((odd || best != best) && b < early) {                     // infinite bounds leave a NaN as well
          const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(r.q) + (w.v.row0 + j0 + j) * r.q_stride + static_cast<int64_t>(sg.g * group) * H;
          const __nv_bfloat16* low = bounds + (static_cast<int64_t>(checked_page(c, table[b])) * c.Hkv + sg.g) * 2 * H;
          best = -INFINITY;
          for (int hh = 0; hh < group; ++hh) best = larger(best, score_of<__nv_bfloat16, H>(q + hh * H, low));
        }
        if (b < early) scores[(static_cast<int64_t>(w.v.row0 + j0 + j) * c.Hkv + sg.g) * c.table_cols + b] = best;
      }
      __syncthreads();
    }
  });
}

// The same without tensor cores (fp32 caches and small or odd shapes): a warp per block and row, the lanes share the head.
template <typename T, int H>
__global__ void __launch_bounds__(256) block_score_row_kernel(PagedCache c, PagedRows r, const T* bounds, int n_blocks, int n_local, float* scores) {
  constexpr int D = H / 32;
  pdl_launch_dependents();
  pdl_wait();
  const int t = blockIdx.x, g = blockIdx.y, group = r.group;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = req_of_row(r.cu_q, c.n_reqs, t);
  const ReqView v = req_view(c, r, i);
  const int j = t - v.row0;
  if (!v.ok || j < 0 || j >= v.m) return;
  const int own = (v.n - v.m + j) / c.ps, early = own + 1 - n_local;
  if (own + 1 <= n_blocks) return;
  float* sc = scores + (static_cast<int64_t>(t) * c.Hkv + g) * c.table_cols;
  for (int b = blockIdx.z * 8 + warp; b < early; b += gridDim.z * 8) {
    const int page = checked_page(c, c.table[static_cast<int64_t>(i) * c.table_stride + b]);
    const T* lo = bounds + (static_cast<int64_t>(page) * c.Hkv + g) * 2 * H + lane * D;
    float low[D], high[D], best = -INFINITY;
    float zero = 0.f;                                    // a NaN where a bound is not finite
#pragma unroll
    for (int d = 0; d < D; ++d) {
      low[d] = to_f32(lo[d]);
      high[d] = to_f32(lo[H + d]);
      zero = fmaf(0.f, low[d], fmaf(0.f, high[d], zero));
    }
    for (int hh = 0; hh < group; ++hh) {
      const T* q = reinterpret_cast<const T*>(r.q) + t * r.q_stride + static_cast<int64_t>(g * group + hh) * H + lane * D;
      float s = zero;
#pragma unroll
      for (int d = 0; d < D; ++d) {
        const float x = to_f32(q[d]);
        s = fmaf(x, x < 0.f ? low[d] : high[d], s);      // the larger of the two products, where everything is finite
      }
      s = warp_sum(s);
      if (!(fabsf(s) < INFINITY)) {                      // bounds, or a query, that are not: the definition
        s = 0.f;
#pragma unroll
        for (int d = 0; d < D; ++d) s += larger(to_f32(q[d]) * low[d], to_f32(q[d]) * high[d]);
        s = warp_sum(s);
      }
      best = larger(best, s);
    }
    if (lane == 0) sc[b] = best;
  }
}

// The choice: one block per (token, KV head); the scores of up to kMostCached blocks stay in shared memory (with twice as
// many the 872 choices of 109 tokens did not run all at once: 20 us against 16).
constexpr int kMostCached = 4096;
__global__ void __launch_bounds__(1024) block_choice_kernel(PagedCache c, PagedRows r, int n_blocks, int n_local, const float* scores,
                                                           int32_t* list) {
  __shared__ int hist[2048], scratch[36];
  __shared__ uint32_t cached[kMostCached];
  pdl_launch_dependents();
  pdl_wait();
  const int t = blockIdx.x, g = blockIdx.y;
  const int i = req_of_row(r.cu_q, c.n_reqs, t);
  const ReqView v = req_view(c, r, i);
  const int j = t - v.row0;
  if (!v.ok || j < 0 || j >= v.m) return;
  const int own = (v.n - v.m + j) / c.ps;
  int32_t* mine = list + (static_cast<int64_t>(t) * c.Hkv + g) * n_blocks;
  if (own + 1 <= n_blocks) {   // everything is read
    for (int b = threadIdx.x; b <= own; b += blockDim.x) mine[b] = b;
    return;
  }
  const int early = own + 1 - n_local, want = n_blocks - n_local;   // early > want
  const float* sc = scores + (static_cast<int64_t>(t) * c.Hkv + g) * c.table_cols;
  if (want > 0) {
    for (int b = threadIdx.x; b < min(early, kMostCached); b += blockDim.x) cached[b] = rank_bits(sc[b]);
    __syncthreads();
    auto rank = [&](int b) { return b < kMostCached ? cached[b] : rank_bits(sc[b]); };
    int greater = 0, total;
    const uint32_t edge = select_largest(rank, early, want, hist, scratch, &greater);
    const int missing = want - greater;
    // a thread goes through a stretch of blocks, in order; before its first one come so many greater ones and equals
    const int per = (early + blockDim.x - 1) / blockDim.x, b0 = min(static_cast<int>(threadIdx.x) * per, early), b1 = min(b0 + per, early);
    int above = 0, ties = 0;
    for (int b = b0; b < b1; ++b) {
      const uint32_t x = rank(b);
      above += x > edge;
      ties += x == edge;
    }
    above = block_scan(above, scratch, &total);
    ties = block_scan(ties, scratch, &total);
    for (int b = b0; b < b1; ++b) {
      const uint32_t x = rank(b);
      if (x > edge || (x == edge && ties < missing)) mine[above + min(ties, missing)] = b;
      above += x > edge;
      ties += x == edge;
    }
  }
  for (int b = threadIdx.x; b < n_local; b += blockDim.x) mine[want + b] = early + b;
}

template <typename T, int H>
int bounds_typed(const PagedCache& c, const int32_t* first, void* bounds, cudaStream_t s) {
  int sms = 0;
  if (paged_device(&sms) < 0) return -1;
  SLED_LAUNCH_PDL((block_bounds_kernel<T, H>), dim3(4 * sms), dim3(256), 0, s, c, first, static_cast<T*>(bounds));
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}
template <typename T, int H>
int choice_typed(const PagedCache& c, const PagedRows& r, const void* bounds, int n_blocks, int n_local, float* scores, int32_t* list, cudaStream_t s) {
  int sms = 0;
  if (paged_device(&sms) < 0) return -1;
  // few choices among many blocks: a large block each; many choices share an SM (a whole call, one token of 30000 keys: 27 us,
  // with 256 threads 36; 109 tokens of 24 contexts: 154 us, with 1024 threads 162)
  const int threads = c.table_cols > 512 && static_cast<int64_t>(r.T) * c.Hkv <= 2 * sms ? 1024 : 256;
  if constexpr (sizeof(T) == 2 && H >= 64) {
    if (r.group <= kScoreRows) {
      SLED_LAUNCH_PDL(block_score_kernel<H>, dim3(3 * sms), dim3(128), 0, s, c, r, static_cast<const T*>(bounds), n_blocks, n_local, scores);
      SLED_LAUNCH_PDL(block_choice_kernel, dim3(r.T, c.Hkv), dim3(threads), 0, s, c, r, n_blocks, n_local, static_cast<const float*>(scores), list);
      return cudaGetLastError() == cudaSuccess ? 2 : -1;
    }
  }
  // enough blocks per row to fill the machine with few rows
  const int z = std::max(1, std::min((c.table_cols + 7) / 8, static_cast<int>(8LL * sms / (static_cast<long long>(r.T) * c.Hkv))));
  SLED_LAUNCH_PDL((block_score_row_kernel<T, H>), dim3(r.T, c.Hkv, z), dim3(256), 0, s, c, r, static_cast<const T*>(bounds), n_blocks, n_local, scores);
  SLED_LAUNCH_PDL(block_choice_kernel, dim3(r.T, c.Hkv), dim3(threads), 0, s, c, r, n_blocks, n_local, static_cast<const float*>(scores), list);
  return cudaGetLastError() == cudaSuccess ? 2 : -1;
}

}  // namespace

int launch_block_bounds(const PagedCache& c, const int32_t* first, void* bounds, cudaStream_t s) {
  if (c.dtype == 1) {
    if (c.h == 32) return bounds_typed<__nv_bfloat16, 32>(c, first, bounds, s);
    if (c.h == 64) return bounds_typed<__nv_bfloat16, 64>(c, first, bounds, s);
    if (c.h == 128) return bounds_typed<__nv_bfloat16, 128>(c, first, bounds, s);
  } else {
    if (c.h == 32) return bounds_typed<float, 32>(c, first, bounds, s);
    if (c.h == 64) return bounds_typed<float, 64>(c, first, bounds, s);
    if (c.h == 128) return bounds_typed<float, 128>(c, first, bounds, s);
  }
  return -1;
}

int launch_block_choice(const PagedCache& c, const PagedRows& r, const void* bounds, int n_blocks, int n_local, float* scores,
                        int32_t* list, cudaStream_t s) {
  if (c.dtype == 1) {
    if (c.h == 32) return choice_typed<__nv_bfloat16, 32>(c, r, bounds, n_blocks, n_local, scores, list, s);
    if (c.h == 64) return choice_typed<__nv_bfloat16, 64>(c, r, bounds, n_blocks, n_local, scores, list, s);
    if (c.h == 128) return choice_typed<__nv_bfloat16, 128>(c, r, bounds, n_blocks, n_local, scores, list, s);
  } else {
    if (c.h == 32) return choice_typed<float, 32>(c, r, bounds, n_blocks, n_local, scores, list, s);
    if (c.h == 64) return choice_typed<float, 64>(c, r, bounds, n_blocks, n_local, scores, list, s);
    if (c.h == 128) return choice_typed<float, 128>(c, r, bounds, n_blocks, n_local, scores, list, s);
  }
  return -1;
}

}  // namespace sled
