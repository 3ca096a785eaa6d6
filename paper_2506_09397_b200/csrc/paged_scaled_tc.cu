// Attention over a paged cache of e4m3 codes on the 5th-generation tensor cores (tcgen05), head_dim 64 and 128: for batches whose
// requests bring many query rows (drafted trees under grouped-query attention, prompts).
//
// Formulas, scales and roundings are those of paged_scaled.cu.  A unit is up to 256 query rows that share a KV head, the M side of
// the products, a row per tensor-memory lane; two groups of four warps have the softmax of 128 rows each.  With more than 128
// rows both groups take every 64-key tile; with fewer they take the tiles in turn, for the same rows, and join at the end.
//     S = Q C^T      (M 128 x N 64 keys, contraction over H)       -> tensor memory, fp32, two buffers a group
//     O += P D       (M 128 x N H, contraction over 64 keys)       P from tensor memory (fp16, over S)
// A group's next scores are formed while it is at the softmax of the present ones.  The products take 16-bit operands, so four warps
// turn the codes into fp16, from a ring of three tiles, into operand tiles.  Each warp brings its
// sixteen keys of a tile itself, with asynchronous 16-byte copies, and needs nobody to tell it that they have arrived.  They
// bring the queries too, as fp16 times a power of two per row.  A score meets its block's scale ks where it leaves tensor memory, a
// numerator its vs before it is rounded.  The references of a row - m of the scores, u of the numerators - are raised only when
// something exceeds them by more than 2^8; raising u means rescaling the row of O in tensor memory, which happens in a unit's
// first tiles.  So a tile's exponentials are formed by the references that there are, beside the search for its largest scores, and
// once more where those call for others.
//
// 64 trees of 48 - 64 nodes over 512 - 4096 keys, 8 KV heads of 128 for 32: 226 us; 512 rows over four contexts of 32768 keys 321 us
// (857 TFLOP/s), 128 rows 128 us.  A 64-key tile of 256 rows takes about 2400 cycles: 1900 of them are a softmax warp's own (load of
// the scores 180, exponentials and maxima, vote, store and arrival 270, in one chain, two such warps on a scheduler), products
// and their waits 1500 beside them, conversion 1150.  A unit costs about 17,000 cycles more (Q, first scores, last output, results
// to memory), which is what short contexts pay.
//   warps 0-3, 4-7 : softmax and output of the two groups
//   warps 8-11     : K, V and Q to fp16, scales
//   warps 12, 13   : products of either group (one thread each: a product takes about 70 cycles to issue), tensor-memory allocation
//   warp 14        : the block's stretches of units, for all others; 15 only completes the warpgroup
// Every wait is bounded; when one runs out the block says so in *status, lets what is under way land, frees its tensor
// memory and returns.
#include "kernels.h"
#include "paged_scaled.cuh"
#include "tcgen05_ptx.cuh"

namespace sled {

namespace {

constexpr int kKeys = 64;                  // keys per tile
constexpr int kGroupRows = 128;            // rows of a softmax group
constexpr int kScaleSlots = 16;            // tiles whose scales are kept (written before a tile's K): more than copies, K and S are ahead of a softmax
constexpr int kScaleWords = 12;            // ks, vs, log2 |vs| of four blocks
constexpr int kUnitSlots = 4;              // stretches of units that are known ahead

// Operands lie in groups of eight rows, [H / 64][8 rows][64 columns] (K, V), or as [H / 64][128 rows][64 columns] (Q); rows of
// 128 bytes, 16-byte chunk c at c ^ (row & 7).
template <int H, int kGroups>
struct ScaledTc {
  static constexpr int kHalves = H / 64;
  static constexpr int kOctet = kHalves * 1024;          // eight rows
  static constexpr int kTileBytes = kKeys / 8 * kOctet;  // K or V
  static constexpr int kQBytes = kGroupRows / 8 * kOctet;
  static constexpr int kStages = kGroups == 1 ? 4 : 3;    // of K and V each
  static constexpr int kOffQ = 0;
  static constexpr int kOffK = kGroups * kQBytes;
  static constexpr int kOffV = kOffK + kStages * kTileBytes;
  static constexpr int kPieces = 3, kPieceBytes = 2 * kKeys * H;      // codes of K and V of a tile
  static constexpr int kOffRaw = kOffV + kStages * kTileBytes;
  static constexpr int kOffBar = kOffRaw + kPieces * kPieceBytes;
  static constexpr int kOffTree = kOffBar + 512;         // parents of the nodes, one byte each, for either group
  static constexpr int kOffTop = kOffTree + 2 * kMaxTreeNodes;     // what the groups tell each other about a row
  static constexpr int kOffScale = kOffTop + kGroupRows * 16;      // [slot][kScaleWords]
  static constexpr int kOffUnit = kOffScale + kScaleSlots * kScaleWords * 4;
  static constexpr int kOffFactor = kOffUnit + kUnitSlots * 64;    // of the rows of Q
  static constexpr int kTotal = kOffFactor + kGroups * kGroupRows * 4 + 1024;     // alignment slack
};
static_assert(kMaxTreeNodes == 128);
static_assert(ScaledTc<128, 1>::kTotal + 512 <= 227 * 1024 && ScaledTc<128, 2>::kTotal + 512 <= 227 * 1024 && ScaledTc<64, 2>::kTotal + 512 <= 227 * 1024,
              "shared memory of one block");

// barriers, 8 bytes each
enum { B_KFULL = 0, B_KEMPTY = 4, B_VFULL = 8, B_VEMPTY = 12, B_QFULL = 16, B_QEMPTY = 17, B_SFULL = 18, B_PFULL = 22, B_PVDONE = 26, B_ODONE = 28, B_UFULL = 30,
       B_UEMPTY = B_UFULL + kUnitSlots, B_COUNT = B_UEMPTY + kUnitSlots };
static_assert(B_COUNT * 8 + 4 <= 512);

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

// A unit, or the stretch of it that the block works on, as warp 14 leaves it in shared memory.
struct TcUnit {
  Segment sg;
  int row0, m, n;
  int more;        // 0: there are no more
};
static_assert(sizeof(TcUnit) <= 64);
constexpr int kUnitReaders = 14;       // warps 0 - 13

// The line of 64-key tiles with units of up to unit_rows rows.  A tile costs about as much with few rows as with many, a unit 7.5
// times that (8 KV heads of 128, us, with 16 : 130, 20 : 160, 28 : 200, 28 : 220, 28 : 260 for them: 64 trees of 48 - 64 nodes - , - , - ,
// 224.6, 225.6; 32 contexts of 128 .. 16384 keys, 64 rows 103, 103, 103, - , - ; 8 to 60 tokens each, where units of up to 128 rows
// weigh 16 : 190, 20 : 160, 25 : 200, 28 : 200 beside 28 : 220 for the others, 231, 198, 170, 161).
struct TcLine : AttentionLine {
  static constexpr int kSlack = 210;
  __device__ __forceinline__ TcLine(const PagedCache& c, const PagedRows& r, int unit_rows) : AttentionLine{c, r, 0, unit_rows, kKeys} {}
  __device__ __forceinline__ int min_share() const { return 1; }
  __device__ __forceinline__ ReqWork operator()(int i) const {
    ReqWork w = AttentionLine::operator()(i);
    if (w.units > 0) w.weight = unit_weight(28, 210, w.tiles, 28 + 210);
    return w;
  }
};

// whether all threads of the two softmax groups say so
__device__ __forceinline__ bool all_of_256(bool x) {
  int y;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 256, p;\n\tselp.b32 %0, 1, 0, q;\n\t}" : "=r"(y) : "r"(static_cast<int>(x)) : "memory");
  return y != 0;
}

// of sixteen, three at a time
__device__ __forceinline__ float largest16(const float* v) {
  const auto of3 = [](float x, float y, float z) { return fmaxf(fmaxf(x, y), z); };
  const float a = of3(of3(v[0], v[1], v[2]), of3(v[3], v[4], v[5]), of3(v[6], v[7], v[8]));
  return fmaxf(a, of3(of3(v[9], v[10], v[11]), of3(v[12], v[13], v[14]), v[15]));
}

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
  const TcUnit* unit_slots = reinterpret_cast<const TcUnit*>(ptr + L::kOffUnit);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ptr + L::kOffBar + 8 * B_COUNT);
  auto bar = [&](int i) { return base + L::kOffBar + 8u * static_cast<uint32_t>(i); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = r.group;
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    *stop = odd[0] = odd[1] = 0;
    for (int s = 0; s < L::kStages; ++s) { mbar_init(bar(B_KFULL + s), 4); mbar_init(bar(B_KEMPTY + s), 2); }
    for (int s = 0; s < L::kStages; ++s) { mbar_init(bar(B_VFULL + s), 4); mbar_init(bar(B_VEMPTY + s), 2); }
    mbar_init(bar(B_QFULL), 4);
    mbar_init(bar(B_QEMPTY), 10);       // the softmax warps and the two product threads
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(B_SFULL + 2 * s), 1);
      mbar_init(bar(B_SFULL + 2 * s + 1), 1);
      mbar_init(bar(B_PFULL + 2 * s), 4);
      mbar_init(bar(B_PFULL + 2 * s + 1), 4);
      mbar_init(bar(B_PVDONE + s), 1);
      mbar_init(bar(B_ODONE + s), 1);
    }
    for (int s = 0; s < kUnitSlots; ++s) { mbar_init(bar(B_UFULL + s), 1); mbar_init(bar(B_UEMPTY + s), kUnitReaders); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {   // S of the two groups at columns 0, 64 and 128, 192, O at 256 and 384
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  const TcLine line(c, r, kUnit);
  const Share share = block_share(line, blockIdx.x, gridDim.x);
  if (threadIdx.x == 0) leave_none(parts.desc, blockIdx.x);

  // The registers of the block, 512 x 128, go where they are needed: 8 warps x 152, 4 x 128, 4 x 80 (all 65,536).
  if (warp >= 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp < 14 && lane == 0) {
      // ------------------------------------------------------------------------------------------------ products
      constexpr uint32_t kFormat = (1u << 4) | (static_cast<uint32_t>(128 >> 4) << 24);   // fp32 += fp16 x fp16, M 128
      constexpr uint32_t idesc_s = kFormat | (static_cast<uint32_t>(kKeys >> 3) << 17);
      constexpr uint32_t idesc_o = kFormat | (static_cast<uint32_t>(H >> 3) << 17) | (1u << 16);   // V is MN-major
      const int s = warp - 12;
      int before = 0, n_s = 0, n_p = 0;       // tiles of earlier units, scores and outputs of the group so far
      for (int units = 0;; ++units) {
        if (*stop || !mbar_wait(bar(B_UFULL + units % kUnitSlots), (units / kUnitSlots) & 1, stop)) { *stop = 1; break; }
        const TcUnit& u = unit_slots[units % kUnitSlots];
        if (!u.more) break;
        const bool both = kGroups == 2 && u.m * group - u.sg.rb * kUnit > kGroupRows;   // both groups have rows of their own
        const int n_tiles = u.sg.t1 - u.sg.t0, step = both ? 1 : 2, t_first = both ? 0 : s, mine = (n_tiles - t_first + step - 1) / step;
        // (in every unit, also where the group has no tile: then all K and V of earlier units have been there, and the parity of a
        // stage that the other group has used last cannot be taken for that of the phase before.  Q is given back by this thread
        // too, by now: without it the others could be through with units of one tile, two phases of this barrier, before a group
        // without tiles has looked at the first)
        bool ok = mbar_wait(bar(B_QFULL), units & 1, stop);
        mbar_arrive(bar(B_QEMPTY));
        const uint64_t q = operand_desc(base + L::kOffQ + (both ? s : 0) * L::kQBytes, 1, 1024);
        // scores go two tiles ahead of the outputs, into the buffer that those have left (products of a thread run in order)
        for (int i = 0; ok && i < mine + 2; ++i) {
          if (i >= 2) {
            const int at = before + t_first + (i - 2) * step, st = at % L::kStages, b = n_p & 1;
            ok = mbar_wait(bar(B_VFULL + st), (at / L::kStages) & 1, stop) && mbar_wait(bar(B_PFULL + 2 * s + b), (n_p >> 1) & 1, stop);
            if (!ok) break;
            fence_after();
            const uint64_t v = operand_desc(base + L::kOffV + st * L::kTileBytes, 1024 >> 4, L::kOctet);
            const uint32_t p = tmem + s * 128 + b * 64;
#pragma unroll
            for (int kt = 0; kt < kKeys / 16; ++kt) umma_ts(tmem + 256 + s * 128, p + kt * 8, v + ((kt * 2 * L::kOctet) >> 4), idesc_o, i != 2 || kt != 0);
            umma_commit(bar(i == mine + 1 ? B_ODONE + s : B_PVDONE + s));
            umma_commit(bar(B_VEMPTY + st));
            if (!both) mbar_arrive(bar(B_VEMPTY + st));      // for the other group
            ++n_p;
          }
          if (i < mine) {
            const int at = before + t_first + i * step, st = at % L::kStages, b = n_s & 1;
            ok = mbar_wait(bar(B_KFULL + st), (at / L::kStages) & 1, stop);
            if (!ok) break;
            fence_after();
            const uint64_t k = operand_desc(base + L::kOffK + st * L::kTileBytes, 1, L::kOctet);
#pragma unroll
            for (int ks = 0; ks < H / 16; ++ks) {
              const uint32_t within = (ks & 3) * 32;
              umma_ss(tmem + s * 128 + b * 64, q + (((ks >> 2) * kGroupRows * 128 + within) >> 4), k + (((ks >> 2) * 1024 + within) >> 4), idesc_s, ks != 0);
            }
            umma_commit(bar(B_SFULL + 2 * s + b));
            umma_commit(bar(B_KEMPTY + st));
            if (!both) mbar_arrive(bar(B_KEMPTY + st));
            ++n_s;
          }
        }
        before += n_tiles;
        if (!ok) *stop = 1;
        mbar_arrive(bar(B_UEMPTY + units % kUnitSlots));
      }
    } else if (warp == 14) {
      // -------------------------------------------------------------------------------------------- stretches of units
      int units = 0;
      auto publish = [&](const TcUnit& u) {
        if (lane == 0) {
          // (a slot becomes free when its stretch is done with, which may take many times what other waits do: as long as nobody
          // else gives up, up to a minute; 2^31 keys take half of that)
          bool free = false;
          for (int tries = 0; !free && tries < 600 && *stop == 0; ++tries) free = mbar_wait(bar(B_UEMPTY + units % kUnitSlots), ((units / kUnitSlots) & 1) ^ 1, stop);
          if (free) {
            const_cast<TcUnit*>(unit_slots)[units % kUnitSlots] = u;
            mbar_arrive(bar(B_UFULL + units % kUnitSlots));
          } else {
            *stop = 1;
          }
        }
        ++units;
      };
      for_segments(line, share, blockIdx.x, [&](const ReqWork& w, const Segment& sg) { publish(TcUnit{sg, w.v.row0, w.v.m, w.v.n, 1}); });
      publish(TcUnit{});
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ------------------------------------------------------------------------------------------- codes to fp16: Q, K, V
    constexpr int kLanes = H / 8, kAtOnce = 32 / kLanes;      // lanes of a key, keys at a time: a warp has 16 of a piece
    const int part = warp & 3, chunk = lane % kLanes, sub = lane / kLanes, cpp = c.ps / 16;
    const uint8_t *k_codes = reinterpret_cast<const uint8_t*>(c.k), *v_codes = reinterpret_cast<const uint8_t*>(c.v);
    int tiles_issued = 0;
    int st = 0, phase = 1, units = 0;
    for (;; ++units) {
      if (!__all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_UFULL + units % kUnitSlots), (units / kUnitSlots) & 1, stop))) { *stop = 1; break; }
      const TcUnit u = unit_slots[units % kUnitSlots];
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_UEMPTY + units % kUnitSlots));
      if (!u.more) break;
      const Segment& sg = u.sg;
      const int first = sg.rb * kUnit, total = u.m * group, rows = min(kUnit, total - first);
      const int32_t* table = c.table + static_cast<int64_t>(sg.req) * c.table_stride;
      const int groups = min((u.n + 15) / 16, sg.t1 * 4);       // 16-key groups up to the end of the segment
      // lane l looks after group l of eight tiles: the block's place among all and (one warp) its scales; those of the next round
      // and the table's entries of the one after are under way
      auto page_of = [&](int e) { return e < groups ? table[quotient(e, cpp)] : 0; };
      auto block_of = [&](int e, int page) { return e < groups ? (checked_page(c, page) * c.Hkv + sg.g) * cpp + (e - quotient(e, cpp) * cpp) : 0; };
      int block, page_next = page_of(sg.t0 * 4 + lane), block_next = block_of(sg.t0 * 4 + lane, page_next);
      float ks, vs, ks_next = 1.f, vs_next = 1.f;
      auto scales_of = [&](int e) {
        if (warp == 8 && e < groups) {
          ks_next = sc.k[block_next];
          vs_next = sc.v[block_next];
        }
      };
      scales_of(sg.t0 * 4 + lane);
      page_next = page_of(sg.t0 * 4 + 32 + lane);
      // the codes of the next tile, this warp's 16 keys of K and V
      int issued = sg.t0, into = 0;
      auto issue = [&]() {
        if (issued < sg.t1) {
          const int t = issued, ahead = (t - sg.t0) & 7;
          if (ahead == 0) {
            block = block_next;
            ks = ks_next;
            vs = vs_next;
            block_next = block_of((t + 8) * 4 + lane, page_next);
            ks_next = vs_next = 1.f;
            scales_of((t + 8) * 4 + lane);
            page_next = page_of((t + 16) * 4 + lane);
          }
          if (warp == 8) {
            float* to = scales + (tiles_issued % kScaleSlots) * kScaleWords;
            if (lane >> 2 == ahead) {
              to[lane & 3] = ks;
              to[4 + (lane & 3)] = vs;
              to[8 + (lane & 3)] = __log2f(fabsf(vs));
            }
          }
          ++tiles_issued;
          const int64_t at = static_cast<int64_t>(__shfl_sync(0xffffffffu, block, ahead * 4 + part)) * 16 * H + lane * 16;
          if (t * 4 + part < groups) {
            const uint32_t to = base + L::kOffRaw + into * L::kPieceBytes + part * 32 * H + lane * 16;
#pragma unroll
            for (int i = 0; i < H / 32; ++i) {
              copy_16(to + i * 512, k_codes + at + i * 512);
              copy_16(to + 16 * H + i * 512, v_codes + at + i * 512);
            }
          }
          ++issued;
          if (++into == L::kPieces) into = 0;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
#pragma unroll 1
      for (int i = 0; i < L::kPieces - 1; ++i) issue();
      // the unit's Q: a row per thread
      if (!__all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_QEMPTY), (units & 1) ^ 1, stop))) { *stop = 1; break; }
      for (int s = 0; s < (rows > kGroupRows ? kGroups : 1); ++s) {
        const int mine = threadIdx.x & 127, at = first + s * kGroupRows + mine;
        uint4 x[H / 8];
        if (at < total) {
          const int j = quotient(at, group);
          const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(r.q) + (u.row0 + j) * r.q_stride + (static_cast<int64_t>(sg.g) * group + (at - j * group)) * H;
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
        uint32_t two = 0;        // the largest |x|, in pairs
#pragma unroll
        for (int i = 0; i < H / 8; ++i) {
          two = __vimax3_u16x2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu, two);
          two = __vimax3_u16x2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu, two);
        }
        uint32_t most = max(two << 16, two & 0xffff0000u);
        if (most >= 0x7f800000u) {        // of the finite ones
          most = 0;
#pragma unroll
          for (int i = 0; i < H / 8; ++i) {
            const uint32_t v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t lo = v[k] << 16 & 0x7fff0000u, hi = v[k] & 0x7fff0000u;
              most = max(most, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
            }
          }
        }
        const int e = min(max(268 - static_cast<int>(most >> 23), 1), 253);
        const float up = __uint_as_float(static_cast<uint32_t>(e) << 23);
        factors[s * kGroupRows + mine] = __uint_as_float(static_cast<uint32_t>(254 - e) << 23) * (r.scale * kLog2e);
        const uint32_t to = base + L::kOffQ + s * L::kQBytes + mine * 128;
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

      const int end = u.n, prefix = end - u.m + (r.parents ? 0 : first / group + 1);
      int piece = 0;
      for (int t = sg.t0; t < sg.t1; ++t) {
        const bool ok = __all_sync(0xffffffffu, *stop == 0 && mbar_wait(bar(B_KEMPTY + st), phase, stop) && mbar_wait(bar(B_VEMPTY + st), phase, stop));
        if (!ok) { *stop = 1; break; }
        asm volatile("cp.async.wait_group %0;" ::"n"(L::kPieces - 2) : "memory");
        __syncwarp();
        const uint32_t from = base + L::kOffRaw + piece * L::kPieceBytes + part * 32 * H + lane * 8, within = st * L::kTileBytes + part * 2 * L::kOctet + (chunk >> 3) * 1024;
        constexpr int kLoads = 16 / kAtOnce;
        uint2 x[2 * kLoads];       // K, then V
#pragma unroll
        for (int i = 0; i < 2 * kLoads; ++i)
          asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x[i].x), "=r"(x[i].y) : "r"(from + i * 256));
        issue();       // into the place of the tile before this one, which all lanes have read
        if (++piece == L::kPieces) piece = 0;
        // A numerator of 0 does not silence a value that is no number: values of positions that hold no key become 0, and so do
        // those that are no numbers, which the rows that see them get back at the end.
        const int x0 = t * kKeys;
        if (x0 + kKeys > prefix) {
          uint32_t found = 0;
#pragma unroll
          for (int i = kLoads; i < 2 * kLoads; ++i) {
            const bool there = x0 + part * 16 + (i - kLoads) * kAtOnce + sub < end;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint32_t y = there ? (k ? x[i].y : x[i].x) : 0u;
              const uint32_t none = ((y & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;      // in the bytes 0x7f and 0xff
              found |= none;
              y &= ~((none >> 7) * 0xffu);
              if (k) x[i].y = y; else x[i].x = y;
            }
          }
          if (found) odd[(units + 1) & 1] = units + 1;
        }
#pragma unroll
        for (int i = 0; i < 2 * kLoads; ++i) {
          const int key = i % kLoads * kAtOnce + sub, row = key & 7;
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                       ::"r"(base + (i < kLoads ? L::kOffK : L::kOffV) + within + (key >> 3) * L::kOctet + row * 128 + (((chunk & 7) ^ row) << 4)), "r"(half2_of(x[i].x)),
                       "r"(half2_of_upper(x[i].x)), "r"(half2_of(x[i].y)), "r"(half2_of_upper(x[i].y)) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(B_KFULL + st));
          mbar_arrive(bar(B_VFULL + st));
        }
        if (++st == L::kStages) { st = 0; phase ^= 1; }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");      // (copies are still under way only where the segment was given up)
      __syncwarp();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
    // ------------------------------------------------------------------------------------------------ softmax, output
    const int s = warp >> 2, row_in_group = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tmem_s = tmem + lanes + s * 128, tmem_o = tmem + lanes + 256 + s * 128;
    int is = 0, units = 0, tiles = 0;
    int done[2] = {0, 0};       // units that either group has finished
    int n_pv = 0;               // outputs of the group, but for the last of every unit
    for (;;) {
      const bool known = *stop == 0 && mbar_wait(bar(B_UFULL + units % kUnitSlots), (units / kUnitSlots) & 1, stop);
      if (!known) *stop = 1;
      const TcUnit u = unit_slots[units % kUnitSlots];
      if (!all_of_256(known && u.more)) break;       // (all or none: there are barriers ahead)
      if (lane == 0) mbar_arrive(bar(B_UEMPTY + units % kUnitSlots));
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
        const int slot = tiles % kScaleSlots, b = is & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(bar(B_SFULL + 2 * s + b), (is >> 1) & 1, stop))) { ok = false; continue; }
        ++is;
        fence_after();
        if (t + step >= n_tiles && lane == 0) mbar_arrive(bar(B_QEMPTY));    // the group is done with Q
        const int x0 = (u.sg.t0 + t) * kKeys;
        const bool masked = x0 + kKeys > prefix;
        const uint32_t tmem_b = tmem_s + b * 64;
        if (active) {
          float4 ks = *reinterpret_cast<const float4*>(scales + slot * kScaleWords);
          float4 vs = *reinterpret_cast<const float4*>(scales + slot * kScaleWords + 4);
          const float4 lv = *reinterpret_cast<const float4*>(scales + slot * kScaleWords + 8);
          ks.x *= factor;
          ks.y *= factor;
          ks.z *= factor;
          ks.w *= factor;
          const bool below = fminf(fminf(ks.x, ks.y), fminf(ks.z, ks.w)) < 0.f;      // (the same for all rows: a row's own factor is positive)
          // Exponentials by the references that there are, and the largest scores beside them; where those call for other references -
          // in a unit's first tiles - once more.
          uint32_t p[kKeys / 2];
          float sum0, sum1;
#pragma unroll 1
          for (int pass = 0;; ++pass) {
            float v[kKeys];
            tmem_ld32_nowait(tmem_b, v);
            tmem_ld32_nowait(tmem_b + 32, v + 32);
            tmem_ld_wait<kKeys>(v);
            float4 by = ks;
            // Scores of tiles that some row does not see all of are scaled and masked first; so are those of scales below 0.
            if (masked || below) {
              const uint32_t see0 = view.seen(x0, prefix, end), see1 = view.seen(x0 + 32, prefix, end);
#pragma unroll
              for (int i = 0; i < kKeys; ++i) {
                const float f = i < 16 ? ks.x : i < 32 ? ks.y : i < 48 ? ks.z : ks.w;
                v[i] = ((i < 32 ? see0 : see1) >> (i & 31)) & 1u ? v[i] * f : -INFINITY;
              }
              by = make_float4(1.f, 1.f, 1.f, 1.f);
              // a scale that is no number reaches the rows that see something of its block, not the others
              if (!(see0 & 0xffffu)) vs.x = 0.f;
              if (!(see0 >> 16)) vs.y = 0.f;
              if (!(see1 & 0xffffu)) vs.z = 0.f;
              if (!(see1 >> 16)) vs.w = 0.f;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            const float weight = top_u == -INFINITY ? 0.f : weight_root(ref, top_u);
            float wx = vs.x, wy = vs.y, wz = vs.z, ww = vs.w;
            mul2(wx, wy, weight);
            mul2(wz, ww, weight);
            mul2(wx, wy, weight);
            mul2(wz, ww, weight);
            float mx = -INFINITY, mx_u = -INFINITY;      // of the scores, of those plus log2 |vs|
            sum0 = sum1 = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float f = q == 0 ? by.x : q == 1 ? by.y : q == 2 ? by.z : by.w;
              const float wb = at_most_2_126(q == 0 ? wx : q == 1 ? wy : q == 2 ? wz : ww);
              const float top = largest16(v + q * 16) * f;
              mx = fmaxf(mx, top);
              mx_u = fmaxf(mx_u, top + (q == 0 ? lv.x : q == 1 ? lv.y : q == 2 ? lv.z : lv.w));
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float a = v[q * 16 + 2 * i], y = v[q * 16 + 2 * i + 1];
                fma2(a, y, f, -ref);
                a = exp2_approx(a);
                y = exp2_approx(y);
                add2(sum0, sum1, a, y);
                mul2(a, y, wb);
                p[q * 8 + i] = pack_half(a, y);
              }
            }
            const bool raise = mx > m + kRaiseBy || (m == -INFINITY && mx > -INFINITY);
            const bool raise_u = mx_u > top_u + kRaiseBy || (top_u == -INFINITY && mx_u > -INFINITY);
            if (pass == 1 || !__any_sync(0xffffffffu, raise || raise_u)) break;
            if (raise) {
              l *= exp2_approx(m - mx);     // 0 where nothing had been seen before
              m = mx;
            }
            const float f = raise_u ? exp2_approx(top_u - mx_u) : 1.f;
            if (raise_u) top_u = mx_u;
            // The output of the group's tile before may be under way; of the one before that it is complete, since these scores came
            // after it.
            if (t != t_first && ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(B_PVDONE + s), (n_pv - 1) & 1, stop));
            if (t != t_first && ok) {
              fence_after();
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
          tmem_st16(tmem_b, p);     // P lies over the scores
          tmem_st16(tmem_b + 16, p + 16);
          l += sum0 + sum1;
          tmem_st_wait();
        }
        if (t + step < n_tiles) ++n_pv;
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PFULL + 2 * s + b));
      }
      // The groups' results.  With rows of their own each writes its own; groups that shared rows also share the writing,
      // half of the columns each: both results of a row are in the same lane of tensor memory, only maximum, sum and the
      // numerators' reference have to be exchanged.
      const bool joint = !both && n_tiles > 1;
      const float rest = rest_root(m, top_u);     // its square is the output's
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
      float f_mine = rest, f_other = 0.f, rest_other = 0.f;      // factors of the group's own result and of the other's, beside `rest`
      if (!joint || s == 0) {
        if (joint) {
          const float4 x = tops[row_in_group];
          const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
          const float a = exp2_approx(m - ref), b = exp2_approx(x.x - ref);
          f_mine = a * rest;
          f_other = b * x.z;
          rest_other = x.z;
          l = l * a + x.y * b;
          m = top;
        }
        if (dead) { m = -INFINITY; l = 0.f; }
        if (u.sg.whole) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          f_mine *= inv;
          f_other *= inv;
        }
        if (joint) tops[row_in_group] = make_float4(f_other, f_mine, rest, 0.f);
      }
      if (joint) {
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (s == 1) {
          const float4 x = tops[row_in_group];
          f_mine = x.x;
          f_other = x.y;
          rest_other = x.z;
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
            for (int i = 0; i < 32; ++i) v[i] = v[i] * f_mine * rest + o[i] * f_other * rest_other;
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = v[i] * f_mine * rest;
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
  // 256 rows a unit turn every tile into fp16 once for both halves, and pay where there are enough units and tiles to keep all SMs
  // at it (head_dim 128, 8 KV heads; units of 128 against 256 rows, us): 132 rows, 64 x 300 keys 87, 69, 16 x 1000 49, 39, 20 x 2000
  // 103, 90, 8 x 8192 129, 105; 256 rows, 64 x 300 87, 77, 16 x 1000 50, 42, 20 x 2000 111, 107, 8 x 8192 135, 115 (64 x 1000, where
  // units of 256 do not share out as well: 153, 165).  With few tiles, or up to 128 rows, they lose: 132 rows, 8 x 1000 30, 34,
  // 1 x 1000 23, 24, 1 x 4096 27, 32; 256 rows, 30, 42; 23, 31; 27, 40; 64 rows, 8 x 8192 75, 107, 64 x 300 50, 56.  How many tiles there
  // are the host knows only from the table's width: with columns for 131072 keys the calls with few tiles take the longer of their two.
  const int64_t rows = static_cast<int64_t>(r.T) * r.group / c.n_reqs, keys = static_cast<int64_t>(c.table_cols) * c.ps;
  const bool wide = rows > kGroupRows && (rows + kGroupRows - 1) / (2 * kGroupRows) * c.n_reqs * c.Hkv * ((keys + kKeys - 1) / kKeys) >= 12LL * sms;
  if (c.h == 128) return wide ? launch_h<128, 2>(c, sc, r, ws, s) : launch_h<128, 1>(c, sc, r, ws, s);
  return wide ? launch_h<64, 2>(c, sc, r, ws, s) : launch_h<64, 1>(c, sc, r, ws, s);
}

}  // namespace sled
