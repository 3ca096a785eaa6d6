// How the attention kernels over a paged cache share their work out: on the device, from the lengths alone.
//
// The work of a call is a line of key tiles.  Request by request, a request's units - (KV head, block of up to kUnitRows
// query rows), or with chosen blocks (token, KV head, block of rows) - follow each other, and a unit is `tiles` tiles of
// kTile keys.  A tile weighs what it costs (a number that depends on how many rows meet it); block c of G takes the tiles
// that begin in [c C / G, (c + 1) C / G) of the total weight C; G is no larger than leaves every block a
// tile.  All blocks are resident and end together, whatever the lengths are, a long context spreads over as many of them as
// it takes, and nothing has to be known on the host.  A unit that is cut leaves one partial result per block; only a
// block's first and last unit can be cut, so two places per block hold them.
#pragma once
#include "paged_device.cuh"

namespace sled {

// Quotients of what is not negative.  The code around them runs once or twice per kernel, so that fetching instructions is
// most of its time: small numbers take a handful.  (a + 1/2) / b lies at least 1 / (2 b) from a whole number, and
// __fdividef is off by 2 units in the last place, 2^-22 of its result, which is less while a < 2^20 (a divisor that a float
// does not hold is larger than a).
__device__ __forceinline__ int quotient(int a, int b) {
  if (__builtin_expect(a < (1 << 20), 1)) return static_cast<int>(__fdividef(static_cast<float>(a) + 0.5f, static_cast<float>(b)));
  return static_cast<int>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b));
}
__device__ __forceinline__ long long divide(long long a, long long b) {
  if (__builtin_expect((a | b) < (1 << 20), 1))
    return static_cast<int>(__fdividef(static_cast<float>(static_cast<int>(a)) + 0.5f, static_cast<float>(static_cast<int>(b))));
  return a / b;
}

constexpr int kTile = 64;        // keys per tile
constexpr int kUnitRows = 64;    // query rows of a unit at most (tensor cores)

// one request's share of the line
struct ReqWork {
  ReqView v;
  int tiles;        // of a unit
  int n_rb;         // row blocks
  int units;
  int weight;       // of a tile
  __device__ __forceinline__ long long count() const { return static_cast<long long>(units) * tiles; }
  __device__ __forceinline__ long long cost() const { return count() * weight; }
};

// Time of a 64-key tile with up to 16, 32, 64 rows: 1.0 / 1.15 / 1.93 (measured per tile with two blocks on an SM), in
// sixteenths.  Beginning and ending a unit costs a number of tiles as well; it is spread over the unit's tiles.
// A share is no smaller than this and no smaller than a tile.  Two tiles of few rows for the warp-level tensor cores (one
// context of 1000 keys: 12 us, with four tiles 15), one of tcgen05 (700 keys: 13 us, with two 16.5), a warp of the fp32
// kernel a tile of a long unit or two (24 trees: 29.2 us, without a minimum 30.5).
constexpr int kMinShare = 64;       // where a unit has whole requests
constexpr int kMinMmaShare = 32;
constexpr int kMinWarpShare = 24;
__device__ __forceinline__ int unit_weight(int tile, int unit, int tiles, int most = kMinShare - 1) { return min(tile + quotient(unit, tiles), most); }
__device__ __forceinline__ int tile_weight(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 18 : 31; }

// The work of attention.  list_len > 0: units attend to chosen blocks, at most list_len per token.  kWholeRows: a unit has
// all rows of its request (kernels that work key by key); a tile then weighs what its rows do, up to the largest weight.
constexpr int kWholeRows = -1;
struct AttentionLine {
  const PagedCache& c;
  const PagedRows& r;
  int list_len;
  int unit_rows = kUnitRows, tile = kTile;
  __device__ __forceinline__ int32_t fault(const ReqView& v) const { return req_fault(r, v); }
  __device__ __forceinline__ int min_share() const {
    return list_len == kWholeRows ? kMinShare : unit_rows == kUnitRows ? kMinMmaShare : unit_rows < kUnitRows ? kMinWarpShare : 1;
  }
  __device__ __forceinline__ ReqWork operator()(int i) const {
    ReqWork w;
    w.v = req_view(c, r, i);
    const int group = r.group;
    w.tiles = w.units = w.n_rb = 0;
    w.weight = 1;
    if (!w.v.ok || w.v.m == 0) return w;
    const int rows = list_len > 0 ? group : w.v.m * group;
    int keys = w.v.n;
    if (list_len > 0) keys = min(list_len, quotient(w.v.n - 1, c.ps) + 1) * c.ps;
    w.tiles = (keys + tile - 1) / tile;
    w.n_rb = list_len == kWholeRows ? 1 : (rows + unit_rows - 1) / unit_rows;
    w.units = w.n_rb * c.Hkv * (list_len > 0 ? w.v.m : 1);
    if (list_len == kWholeRows) w.weight = min(16 + rows, kMinShare - 1);
    // tcgen05, in cycles by regression over the blocks: 2200 a tile and 15,000 a unit up to 128 rows, 4000 and 18,500 above
    else if (unit_rows > kUnitRows) w.weight = rows > kUnitRows * 2 ? unit_weight(38, 175, w.tiles, 38 + 175) : unit_weight(16, 160, w.tiles);
    // warp-level tensor cores, likewise: 2100 a tile and 8100 a unit with up to 16 rows (32 contexts of 128 .. 16384 keys with
    // weights 127 us; half as much for a unit, and capped at 63, 139)
    else if (unit_rows == kUnitRows) w.weight = unit_weight(tile_weight(min(rows, kUnitRows)), 64, w.tiles, tile_weight(kUnitRows) + 64);
    else w.weight = unit_weight(12, 24, w.tiles, kMinWarpShare - 1);
    return w;
  }
};

struct Share {
  int req;               // first request
  long long at;          // where it begins on the line
  long long from, to;    // this share's part of the line
  long long each;        // its length, but that the first `rest` shares are one longer
  int rest;
  ReqWork w;             // of the first request
};


// Shares `first`, .. `first` + kShares - 1 of at most `most`, into out[] (shared memory).  All threads of the block call it
// (blockDim.x a multiple of 32, at most 32 * kMostWarps).  The block with share 0 reports the requests that are left out.
constexpr int kMostWarps = 12;
template <int kShares, typename Line>
__device__ __forceinline__ void block_shares(const Line& line, int first, int most, Share* out) {
  __shared__ long long sums[kMostWarps];   // (little, so that attention blocks still share an SM)
  __shared__ int2 weights[kMostWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const int n_reqs = line.c.n_reqs, per = (n_reqs + blockDim.x - 1) / blockDim.x;
  const int i0 = min(static_cast<int>(threadIdx.x) * per, n_reqs), i1 = min(i0 + per, n_reqs);
  long long own = 0;
  ReqWork w;
  int heaviest = 1, lightest = 1 << 30;        // tile
#pragma unroll 1
  for (int i = i0; i < i1; ++i) {
    w = line(i);
    own += w.cost();
    if (w.units > 0) {
      heaviest = max(heaviest, w.weight);
      lightest = min(lightest, w.weight);
    }
    if (first == 0 && !w.v.ok) set_status(line.c.status, line.fault(w.v));
  }
  long long x = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  heaviest = __reduce_max_sync(0xffffffffu, heaviest);
  lightest = __reduce_min_sync(0xffffffffu, lightest);
  if (lane == 31) {
    sums[warp] = x;
    weights[warp] = make_int2(heaviest, lightest);
  }
  if (threadIdx.x < kShares) out[threadIdx.x].from = out[threadIdx.x].to = out[threadIdx.x].at = 0;
  __syncthreads();
  long long before = 0, total = 0;
  for (int k = 0; k < nw; ++k) {
    if (k < warp) before += sums[k];
    total += sums[k];
    heaviest = max(heaviest, weights[k].x);
    lightest = min(lightest, weights[k].y);
  }
  // A part of the line that is no shorter than any tile holds the beginning of one.  Whole tiles to a share: the longest
  // share is no longer for it, there are fewer of them, and units are cut in the same places where they are alike.
  const long long least = max(divide(total + most - 1, most), static_cast<long long>(max(line.min_share(), heaviest)));
  const long long whole = divide(least + lightest - 1, lightest) * lightest;
  long long many = divide(total + whole - 1, whole);
  if (many * heaviest > total) --many;
  const int count = static_cast<int>(max(1LL, many));
  const long long each = divide(total, count), rest = total - each * count;
  long long at = before + x - own;
  const long long end = at + own;
#pragma unroll 1
  for (int k = 0; k < kShares; ++k) {
    const int mine = first + k;
    const long long from = each * mine + min(static_cast<long long>(mine), rest), to = from + each + (mine < rest);
    if (mine < count && from < to && at <= from && from < end) {
      long long begin = at;
      int i = i0;
      if (per > 1) {         // (a thread that has one request knows it already)
#pragma unroll 1
        for (;; ++i) {
          w = line(i);
          if (from < begin + w.cost()) break;
          begin += w.cost();
        }
      }
      out[k] = Share{i, begin, from, to, each, static_cast<int>(rest), w};
    }
  }
  __syncthreads();
}
template <typename Line>
__device__ __forceinline__ Share block_share(const Line& line, int block, int most) {
  __shared__ Share mine;
  block_shares<1>(line, block, most, &mine);
  return mine;
}

// the share that owns the tile which begins at `at`
__device__ __forceinline__ int owner_of(long long at, const Share& s) {
  const long long longer = (s.each + 1) * s.rest;
  const bool early = at < longer;
  return static_cast<int>(divide(early ? at : at - longer, early ? s.each + 1 : s.each)) + (early ? 0 : s.rest);
}

// A stretch of one unit that a block works on.
struct Segment {
  int req, j, g, rb;     // j: the token (chosen blocks), otherwise unused
  int t0, t1;            // tiles
  bool whole;            // the unit is not cut
  int slot;              // place of the partial result: 2 * block for the block's first tile, 2 * block + 1 otherwise
  int last_block;        // cut units, where t0 == 0: the block that ends the unit; -1 otherwise
};

// What the merge has to know of a cut unit, left by the share that begins it at its own place (two int4 of `desc`).
struct CutUnit {
  int last_block, slot;        // the share that ends the unit, or -1 where this share begins none; place of the first partial result
  int row0, m, g, j;           // the request's rows; KV head; the token, or -1: all of them
  int first, count;            // rows of the unit
};
__device__ __forceinline__ void leave_none(int4* desc, int block) { desc[2 * block].x = -1; }
__device__ __forceinline__ void leave_cut(int4* desc, int block, const Segment& sg, int row0, int m, int j, int first, int count) {
  desc[2 * block] = make_int4(sg.last_block, sg.slot, row0, m);
  desc[2 * block + 1] = make_int4(sg.g, j, first, count);
}
__device__ __forceinline__ CutUnit cut_unit(const int4* desc, int block) {
  const int4 a = desc[2 * block], b = desc[2 * block + 1];
  return CutUnit{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

// The segments of a share, in order.
template <typename Line>
struct Walk {
  const Line& line;
  const Share& s;
  int block, i;
  long long at, lt = 0, lt_end = 0;
  ReqWork w;               // of the current segment's request
  bool first = true, fresh = true;
  __device__ __forceinline__ Walk(const Line& l, const Share& share, int b) : line(l), s(share), block(b), i(share.req), at(share.at), w(share.w) {}
  __device__ __forceinline__ bool next(Segment& g) {
    while (lt >= lt_end) {
      if (!fresh) {
        at += w.cost();
        ++i;
      }
      if (at >= s.to) return false;
      if (!fresh) w = line(i);
      fresh = false;
      lt_end = min(w.count(), divide(s.to - at + w.weight - 1, w.weight));
      lt = s.from > at ? divide(s.from - at + w.weight - 1, w.weight) : 0;
    }
    const int u = static_cast<int>(divide(lt, w.tiles));
    g.req = i;
    g.t0 = static_cast<int>(lt - static_cast<long long>(u) * w.tiles);
    g.t1 = static_cast<int>(min(static_cast<long long>(w.tiles), g.t0 + (lt_end - lt)));
    const int of_rb = w.n_rb == 1 ? u : quotient(u, w.n_rb);
    g.rb = u - of_rb * w.n_rb;
    g.j = quotient(of_rb, line.c.Hkv);
    g.g = of_rb - g.j * line.c.Hkv;
    g.whole = g.t0 == 0 && g.t1 == w.tiles;
    g.slot = 2 * block + (first ? 0 : 1);
    g.last_block = -1;
    if (g.t0 == 0 && !g.whole) g.last_block = owner_of(at + ((static_cast<long long>(u) + 1) * w.tiles - 1) * w.weight, s);
    first = false;
    lt += g.t1 - g.t0;
    return true;
  }
};

// Calls f(work of the request, segment) for every segment of the share.
template <typename Line, typename F>
__device__ __forceinline__ void for_segments(const Line& line, const Share& s, int block, F f) {
  Walk<Line> walk(line, s, block);
  Segment g;
  while (walk.next(g)) f(walk.w, g);
}

}  // namespace sled
