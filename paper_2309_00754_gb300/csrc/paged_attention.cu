// Attention of each sequence's new tokens over a paged key/value cache (kv_cache.cuh):
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp2(s_j - m),  s_j = scale log2(e) q.k_j,  j <= cached + t
//
// in one pass over the cache. The query rows of a key/value head (its tokens times its query heads) are the columns of
// two products by mma.m16n8k16, a tile of 16 cached tokens each: S^T = K q^T (tokens x rows) and O^T += V^T P^T (channels x
// rows), so that a decode step's one to eight rows waste nothing but a tile's eight columns, scores of a token lie in the
// lanes that hold its scales, and P^T is S^T's own fragment turned by movmatrix. Both operands lie in the cache as the
// fragments want them.
//
// In 4 bits a code enters as the fp16 integer code - zero: its bits over those of 1024 (or 16 times it over 1024, for the
// upper nibble of a byte) are a float, less 1024 + zero, all exact; what is 16 times too large is undone in q and at
// the end. So keys' products are exact up to the sums, their scale is multiplied in fp32 after, and a value's scale goes
// into its probability, which is the one thing that is rounded: to fp16, 2^-11, which adds a hundredth to the error that the
// output's own rounding makes. (bf16's 2^-8 would add as much again; what the rounding leaves as a second fp16 number is 10 to
// 15 % of the time: 53.7, 38.2 and 71.2 us for 64 sequences of 800 tokens, 16 of 4096 and 3 of 131,072, against 47.4, 34.6 and
// 61.8.) To keep that in fp16's range, each row has a power of two for each group of channels (`lift`) by which the group's
// weights are held, so that a group's precision is its own, whatever the other's scales are. m, a whole number, and the lifts
// are moved only when a row's weights pass the range, which a vote finds: the pass would spend its time on maxima else. A bf16
// cache takes the probability as two bf16.
//
// A bf16 cache is bound by its bytes (8 sequences of up to 32,768 tokens, 8 heads: 580 MB in 92 us, 6.3 TB/s). In 4 bits the
// copies are hidden and what a tile costs to unpack and multiply, 360 instructions of a warp for 2304 bytes, is as much as
// its bytes or more: 3 sequences of up to 131,072 tokens, 8 heads: 283 MB in 62 us, 4.5 TB/s; 64 sequences of up to 800, 32
// heads: 146 MB in 47 us. Half of the issue slots are used, the rest goes to dependent instructions and their fetch.
//
// Work is cut evenly: the tiles of all (sequence, eight rows, head) items in a row, a contiguous part for each warp, which
// copies its tiles into a ring of its own (cp.async: a bulk copy and its barrier cost a warp some hundred clocks a stage)
// and needs no other warp on the way: it writes the items that it has whole. What it has of an item that others share it
// leaves until the CTA's end, where the parts of the CTA's warps are added up, and what CTAs share a second kernel adds up,
// both in the order of the parts. (Sixteen to 32 rows an item, which unpack a tile once for all of them, want registers:
// with half or a quarter of the warps they took 43 and 46 us for 16 sequences x 20 rows over 4096 tokens, eight rows 36. Codes
// as fp16 numbers below the normal range, whose zero points come off the sums, are 295 instructions a tile and no faster.)
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "kv_cache.cuh"

namespace hydra {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxCtas = 320;     // of a grid; parts of items lie in the workspace, two a CTA and one a warp
constexpr int kRows = 8;          // query rows of an item: the columns of a product
// Tiles of a warp, where there are more warps than that fills (one sequence of 300 tokens, 32 heads: 7.8 us with one or two,
// 8.5 with four, which leave warps idle).
constexpr int kMinUnits = 2;
// Tokens of a table up to which a CTA takes an item alone, without the second kernel, where there are CTAs for all (one sequence, 32
// heads: 300 tokens 7.8 us against 12.0, 1100 tokens 11.9 against 13.2, 2200 tokens 17.5 against 14.4). Twice as many where a quarter
// of the CTAs have an item and a tile costs less than in 4 bits with 128 channels (bf16, 13 sequences of 2000 tokens, 156 items of 64
// channels, 15.1 us against 16.6; 4 of 2000, 128 of 128 channels, 20.7 against 22.8; one of 2200, 32 items, 18.2 against 15.9;
// 4 bits with 128 channels, 8 of 2400, 256 items, 26.2 against 23.7).
constexpr int64_t kAlignedTokens = 1280;
// What an item costs beside its tiles, in tiles (16 sequences x 20 rows over up to 4096 tokens: 35 us with 6 or 12, 36 with 3, 52
// with 0; 64 sequences of up to 800, 32 heads: 47, 48, 48, 65).
constexpr int kItemUnits = 6;
constexpr float kLowest = -FLT_MAX;      // a maximum of nothing yet, which the least finite score does not lie below
constexpr float kNothing = -INFINITY;    // mass of a part whose scores are all -inf
// Exponents: of a probability relative to m up to 2^8; in 4 bits of probability times scale times the group's lift, of which the
// largest is put between 2^6 and 2^7 when the lift is set, up to 2^14 (fp16 ends at 2^16, and keeps 11 bits down to 2^-14). A
// lift is at most 2^118, so that its product with a probability is finite, and at least 2^-126.
constexpr float kSlack = 8.f, kMost = 14.f;
constexpr int kTop = 7, kLiftMost = 118, kLiftLeast = -126;

// What a CTA leaves for the second kernel.
struct Desc {
  int s, rt, h;   // the item that its last segment begins and does not end, if slot >= 0
  int slot;       // where that segment's part lies, or -1
  int ends;       // its first segment (slot 0) ends an item that an earlier CTA began
  int live;       // rows of the item that have a token
  int pad[2];
};

// Part of an item's rows, normalised, with log2 of the sum of exp2(s) that it stands for (NaN: unusable).
template <int kDh>
struct Part {
  float o[kRows][kDh];
  float mass[kRows];
};

template <int kDh, bool kInt4>
struct Config {
  using Tile = KvTile<kDh, kInt4>;
  using Parts = Part<kDh>;
  using Vec = std::conditional_t<kDh == 128, float4, float2>;  // a lane's channels where a warp has a row
  static constexpr int kMTiles = kDh / 16;
  static constexpr int kCtasPerSm = kInt4 || kDh == 64 ? 2 : 1;
  static constexpr int kStageTiles = kInt4 ? 2 : 1;  // that are copied and taken together
  static constexpr int kStageBytes = kStageTiles * Tile::kBytes;
  static constexpr int kStages = 2;  // a power of two
  static_assert(kRows * kDh * 4 <= kStages * kStageBytes, "a warp's ring takes its last part at the end");
  static constexpr int kRing = kWarps * kStages * kStageBytes;
  static constexpr int kQ = kRows * kDh * 2;  // a warp's queries, as rows and then as fragments
  static constexpr int kSmem = kRing + kWarps * kQ;
};

// A warp's last part (in its ring) and the one before it that does not begin its item (in the workspace), by what becomes
// of them at the CTA's end.
struct WarpEnd {
  int s, rt, h;     // item of the last segment
  int first_rt;     // (the first segment's item: only its rows matter)
  bool first;       // there is a first part, of an item that an earlier warp began
  bool first_last;  // it is the last segment as well, and lies in the ring
  bool first_ends;  // it ends its item
  bool tail;        // the last segment begins an item and does not end it
  int live;         // rows with a token of that item
};

// (not volatile: the compiler interleaves them)
__device__ __forceinline__ void first_mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t turned(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// (-inf below 2^-126)
__device__ __forceinline__ float lg2_or_none(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t max_f16(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// whether one of two fp16 is above 2^14, or an infinity (not: NaN)
__device__ __forceinline__ bool above_f16(uint32_t a) {
  uint32_t r;
  asm("{\n\t.reg .pred p, q;\n\tsetp.gt.f16x2 p|q, %1, %2;\n\tor.pred p, p, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"(a), "r"(0x74007400u));
  return r != 0;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t add_f16(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
        "l"(reinterpret_cast<unsigned long long&>(c)));
  return r;
}
// 2^e, e in [-126, 127]
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ float pow2_or_0(int e) { return pow2(max(e, -127)); }  // 0 below 2^-126

// (w & mask) | bits in one instruction: `bits` comes from a register, as two constants in one would take two instructions
template <uint32_t kMask>
__device__ __forceinline__ uint32_t merged(uint32_t w, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w), "n"(kMask), "r"(bits));
  return r;
}
__device__ __forceinline__ uint32_t held(uint32_t constant) {
  uint32_t r;
  asm volatile("mov.b32 %0, %1;" : "=r"(r) : "r"(constant));
  return r;
}
constexpr uint32_t kFp16Of1024 = 0x64006400u, kFp16OfMinus1024 = 0xe400e400u;
// code - zero of the low nibbles of the bytes 0 and 2 (16 (code - zero) of the high ones), as fp16; `of`: kFp16Of1024
__device__ __forceinline__ uint32_t low_nibbles(uint32_t w, uint32_t minus, uint32_t of) { return add_f16(merged<0x000f000fu>(w, of), minus); }
__device__ __forceinline__ uint32_t high_nibbles(uint32_t w, uint32_t minus, uint32_t of) { return add_f16(merged<0x00f000f0u>(w, of), minus); }
// -(1024 + zero), -(1024 + 16 zero) from two zero points as the cache holds them; `of`: kFp16OfMinus1024
__device__ __forceinline__ uint32_t minus_low(uint32_t z, uint32_t of) { return merged<0x000f000fu>(z, of); }
// (the second from the first, exactly, as a multiplication and addition: logic has half the rate, and is what a tile waits for)
__device__ __forceinline__ uint32_t minus_high(uint32_t low) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(low), "r"(0x4c004c00u), "r"(0x73807380u));  // 16 low + 15360
  return r;
}

// ---------------------------------------------------------------- what is whose

struct Geometry {
  int group, rows, row_tiles, kv_heads;  // query heads of a kv head; rows of a kv head; passes over its rows
};
__device__ __forceinline__ Geometry geometry(const PagedAttentionArgs& p) {
  Geometry g;
  g.kv_heads = p.cache.kv_heads;
  g.group = static_cast<int>(p.n_heads) / g.kv_heads;
  g.rows = g.group * static_cast<int>(p.batch.L);
  g.row_tiles = (g.rows + kRows - 1) / kRows;
  return g;
}

// Tiles of cached tokens that rows [8 rt, ...) of a sequence see; 0 where there is nothing to compute.
__device__ __forceinline__ int tiles_of(const Geometry& g, const KvSeq& seq, int rt) {
  if (!seq.ok || seq.n == 0) return 0;
  if (g.row_tiles == 1) return (seq.cached + seq.n - 1) / kKvTile + 1;
  const int live = g.group * seq.n, first = rt * kRows;
  if (first >= live) return 0;
  const int last = (min(first + kRows, live) - 1) / g.group;
  return (seq.cached + last) / kKvTile + 1;
}
// Units of an item: its tiles, at least one (an item without tiles has rows to fill), and behind them what it costs besides.
__device__ __forceinline__ int units_of_item(int tiles) { return max(1, tiles) + kItemUnits; }
__device__ __forceinline__ long long units_of(const Geometry& g, const KvSeq& seq) {
  long long n = 0;
  for (int rt = 0; rt < g.row_tiles; ++rt) n += units_of_item(tiles_of(g, seq, rt));
  return n;
}

__device__ __forceinline__ KvSeq seq_of(const PagedAttentionArgs& p, int s, int* err) {
  return kv_seq(p.batch, s, p.batch.max_pages << p.cache.page_bits, err);
}

// A place in the units: an item, and a tile of it.
struct Place {
  KvSeq seq;
  int s, rt, h, tile, tiles;
  __device__ __forceinline__ void next_item(const PagedAttentionArgs& p, const Geometry& g) {
    tile = 0;
    if (++h < g.kv_heads) return;
    h = 0;
    if (++rt == g.row_tiles) {
      rt = 0;
      ++s;
      seq = seq_of(p, s, nullptr);
    }
    tiles = tiles_of(g, seq, rt);
  }
};

// The exclusive prefix of a value over the warp's or the block's threads, and its sum.
struct Scan {
  long long before, total;
};
__device__ __forceinline__ Scan warp_scan(long long v) {
  const int lane = threadIdx.x & 31;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return Scan{x - v, __shfl_sync(0xffffffffu, x, 31)};
}
__device__ __forceinline__ Scan block_scan(long long v, long long* sh) {
  const int warp = threadIdx.x >> 5;
  const Scan own = warp_scan(v);
  if ((threadIdx.x & 31) == 31) sh[warp] = own.total;
  __syncthreads();
  Scan r{own.before, 0};
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) r.before += sh[w];
    r.total += sh[w];
  }
  __syncthreads();
  return r;
}

struct Shared {
  Place load[kWarps], take[kWarps];  // items that a warp copies and computes
  int load_left[kWarps];
  long long scan[kWarps];
  long long offset[kWarps];
  int s[kWarps];
  WarpEnd end[kWarps];
  float mass[kWarps][kRows];  // of the parts in the rings
};
// Where the warp's part begins, and how many units it has; `active` is how many of a CTA's warps have one. Two ways:
//  - aligned (the host knows that there are no more items than CTAs, and short ones): a CTA an item, which is joined there.
//  - else the units in a row, a contiguous part for each warp. (Few items cut in equal parts, so that a warp has one part of one
//    item, took 1 us longer: the parts are counted first.)
__device__ __forceinline__ int begin(const PagedAttentionArgs& p, const Geometry& g, bool aligned, Place& c, int& active, Shared& sh) {
  const int S = static_cast<int>(p.batch.S), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int* const err = blockIdx.x == 0 ? p.err : nullptr;
  if (aligned) {
    const int items_of_s = g.kv_heads * g.row_tiles;
    c.s = static_cast<int>(blockIdx.x) / items_of_s;
    const int i = static_cast<int>(blockIdx.x) - c.s * items_of_s;
    c.rt = i / g.kv_heads;
    c.h = i - c.rt * g.kv_heads;
    c.seq = seq_of(p, c.s, i == 0 ? p.err : nullptr);
    c.tiles = tiles_of(g, c.seq, c.rt);
    active = min(kWarps, max(1, (c.tiles + kMinUnits - 1) / kMinUnits));
    c.tile = c.tiles * warp / active;
    return warp >= active ? 0 : max(1, c.tiles) * (warp + 1) / active - c.tile;
  }
  const bool few = S <= 32;  // each warp looks for itself, a lane a sequence
  long long mine = 0, total = 0;
  Scan scan{0, 0};
  for (int at = 0; at < S; at += kThreads) {
    const int s = few ? lane : at + static_cast<int>(threadIdx.x);
    mine = s < S ? units_of(g, seq_of(p, s, err)) * g.kv_heads : 0;
    scan = few ? warp_scan(mine) : block_scan(mine, sh.scan);
    total += scan.total;
  }
  const int most = gridDim.x * kWarps;
  auto ratio = [](long long x, int y) -> long long {  // (a division of 64 bits takes as long as a read of memory)
    if (x < (1LL << 31)) return static_cast<unsigned>(x) / static_cast<unsigned>(y);
    return x / y;
  };
  const int all = static_cast<int>(min((total + kMinUnits - 1) / kMinUnits, static_cast<long long>(most)));
  active = (all + gridDim.x - 1) / gridDim.x;
  const int warps = min(all, static_cast<int>(gridDim.x) * active), first_warp = blockIdx.x * active;
  const long long each = ratio(total, warps);
  const int over = static_cast<int>(total - each * warps);
  auto from = [&](int w) { return w >= warps ? total : each * w + min(w, over); };
  // the sequence that a warp's first unit (part) is in
  long long before = 0;
  for (int at = 0; at < S; at += kThreads) {
    if (S > kThreads) {
      const int s = at + static_cast<int>(threadIdx.x);
      mine = s < S ? units_of(g, seq_of(p, s, nullptr)) * g.kv_heads : 0;
      scan = block_scan(mine, sh.scan);
    }
    const long long start = before + scan.before;
    if (few) {
      const long long first = from(first_warp + warp);
      const unsigned found = __ballot_sync(0xffffffffu, first >= start && first < start + mine);
      const int s = found == 0 ? 0 : __ffs(found) - 1;
      const long long offset = first - __shfl_sync(0xffffffffu, start, s);
      if (lane == 0) {
        sh.s[warp] = s;
        sh.offset[warp] = offset;
      }
      break;
    }
    for (int w = 0; w < active; ++w) {
      const long long first = from(first_warp + w);
      if (first >= start && first < start + mine) {
        sh.s[w] = at + static_cast<int>(threadIdx.x);
        sh.offset[w] = first - start;
      }
    }
    before += scan.total;
  }
  if (few) __syncwarp(); else __syncthreads();
  if (warp >= active || first_warp + warp >= warps) return 0;
  c.s = sh.s[warp];
  long long rest = sh.offset[warp];
  c.seq = seq_of(p, c.s, nullptr);
  int each_item;
  for (c.rt = 0;; ++c.rt) {
    c.tiles = tiles_of(g, c.seq, c.rt);
    each_item = units_of_item(c.tiles);
    const long long units = static_cast<long long>(each_item) * g.kv_heads;
    if (rest < units) break;
    rest -= units;
  }
  c.h = static_cast<int>(ratio(rest, each_item));
  c.tile = static_cast<int>(rest - static_cast<long long>(c.h) * each_item);
  int left = static_cast<int>(from(first_warp + warp + 1) - from(first_warp + warp));
  if (c.tile >= max(1, c.tiles)) {  // behind an item's tiles
    left -= units_of_item(c.tiles) - c.tile;
    if (left > 0) c.next_item(p, g);
  }
  return left;
}

// ---------------------------------------------------------------- a warp's copies

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there = true) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(there ? 16 : 0)
               : "memory");  // (zeros where there is nothing)
}
__device__ __forceinline__ void copy16_if(bool there, uint32_t dst, const void* src) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %0, 0;\n\t@p cp.async.cg.shared.global [%1], [%2], 16;\n\t}" ::"r"(
                   static_cast<uint32_t>(there)),
               "r"(dst), "l"(reinterpret_cast<uint64_t>(src))
               : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until at most kGroups of the warp's groups are on their way
template <int kGroups>
__device__ __forceinline__ void wait_copies() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kGroups) : "memory");
  __syncwarp();
}

// Tiles of a stage, the first at `tile`: two from an even one on, so that they lie in one page or in two neighbours of a
// batch (below).
template <typename C>
__device__ __forceinline__ int stage_tiles(int tile, int end) {
  return C::kStageTiles == 1 || (tile & 1) != 0 ? 1 : min(2, end - tile);
}

// What a warp copies next. Every lane holds where one of 32 neighbouring tiles lies (a batch).
template <int kDh, bool kInt4>
struct Loader {
  using C = Config<kDh, kInt4>;
  const uint8_t* mine = nullptr;  // the lane's tile
  long long head = 0;             // offset of the item's head
  int s = -1, tile = 0, end = 0;  // sequence, next tile to copy, end of the warp's part of the item
  int base = -1;                  // of the batch
  int issued = 0;                 // stages
  bool bad = false;               // a page was none of the cache's

  __device__ __forceinline__ void batch(const PagedAttentionArgs& p, int lane) {
    base = tile & ~31;
    const int at = base + lane;
    int page = 0;
    if (at < end) page = p.batch.table[static_cast<long long>(s) * p.batch.ld_table + ((at * kKvTile) >> p.cache.page_bits)];
    const bool ok = page >= 0 && page < p.cache.n_pages;
    if (__any_sync(0xffffffffu, !ok)) {
      bad = true;
      if (lane == 0) record_error(p.err, kDevBadPage);
    }
    mine = kv_tile<typename C::Tile>(p.cache, ok ? page : 0, 0, at * kKvTile) + head;
  }
  // The item that `at` says, `left` units from its tile on; those without tiles are passed over. `at` goes on to the next.
  // (The lanes read the shared copies, compute the same, and write them again.)
  __device__ __forceinline__ void item(const PagedAttentionArgs& p, const Geometry& g, Place& at, int& left) {
    Place now = at;
    int n = left;
    while (n > 0 && now.tiles == 0) {
      n -= units_of_item(0);
      if (n > 0) now.next_item(p, g);
    }
    if (n > 0) {
      // a sequence's next head of up to 32 tiles lies in the batch that is there, the same way on
      const long long to = static_cast<long long>(now.h) * ((1 << (p.cache.page_bits - 4)) * C::Tile::kBytes);
      if (now.s != s || now.h == 0 || now.tiles > 32) base = -1;
      mine += to - head;
      head = to;
      s = now.s;
      tile = now.tile;
      end = min(now.tiles, tile + n);
      n -= units_of_item(now.tiles) - tile;
      if (n > 0) now.next_item(p, g);
    }
    __syncwarp();
    at = now;
    left = n;
    __syncwarp();
  }
  // The next stage: a group of copies, empty where nothing is left.
  __device__ __forceinline__ void issue(const PagedAttentionArgs& p, const Geometry& g, Place& at, int& left, int lane,
                                        uint32_t ring) {
    if (tile >= end && left > 0) item(p, g, at, left);
    int n = 0;
    if (tile < end) {
      if ((tile & ~31) != base) batch(p, lane);
      n = stage_tiles<C>(tile, end);
    }
    fill(p, n, lane, ring);
  }
  // n tiles of the batch into the next stage
  __device__ __forceinline__ void fill(const PagedAttentionArgs& p, int n, int lane, uint32_t ring) {
    const uint32_t dst = ring + (issued & (C::kStages - 1)) * C::kStageBytes + lane * 16;
    const uint8_t* src = from_lane(tile & 31) + lane * 16;
    if (n > 0) copy(dst, src, lane);
    if (C::kStageTiles == 2 && n == 2)
      copy(dst + C::Tile::kBytes, p.cache.page_bits == 4 ? from_lane((tile + 1) & 31) + lane * 16 : src + C::Tile::kBytes, lane);
    tile += n;
    ++issued;
    commit_copies();
  }
  __device__ __forceinline__ const uint8_t* from_lane(int from) const {
    return reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), from));
  }
  // A tile; dst and src are the lane's first 16 bytes of it.
  __device__ __forceinline__ static void copy(uint32_t dst, const uint8_t* src, int lane) {
    constexpr int kWhole = C::Tile::kBytes / 512, kRest = C::Tile::kBytes % 512 / 16;
#pragma unroll
    for (int i = 0; i < kWhole; ++i) copy16(dst + i * 512, src + i * 512);
    if (kRest != 0) copy16_if(lane < kRest, dst + kWhole * 512, src + kWhole * 512);
  }
};

// ---------------------------------------------------------------- a tile

// What a warp knows of its item's rows, and what it has added up.
template <int kDh, bool kInt4>
struct Rows {
  using C = Config<kDh, kInt4>;
  float factor[2];
  int limit[2];             // last position that rows 2t and 2t + 1 see
  int first_limit, last_limit;  // the least and the largest of the rows'
  // fragments of 16 channels; in 4 bits fp16, of which the second word is a sixteenth
  const uint2* q;
  static constexpr int kGroups = kInt4 ? kDh / kKvGroup : 1;  // of channels that have a scale of their own
  float o[C::kMTiles][4], m[2], l[2];
  float lift[2][kGroups];  // 4 bits: powers of two by which a group's weights are held (o with them) for fp16's range
  uint32_t plus1024, minus1024;  // kFp16Of1024, kFp16OfMinus1024 in registers

  __device__ __forceinline__ uint2 query(int step, int lane) const { return q[step * 32 + lane]; }

  __device__ __forceinline__ static int live_rows(const Geometry& geo, const Place& c) {
    return c.tiles == 0 ? 0 : min(kRows, c.seq.n * geo.group - c.rt * kRows);
  }
  // The queries' rows to where their fragments will be, zeros for rows without a token.
  __device__ __forceinline__ static void fetch(const PagedAttentionArgs& p, const Geometry& geo, const Place& c, int lane, uint32_t to) {
    constexpr int kPieces = kDh / 8, kRowsAtOnce = 32 / kPieces;  // of 16 bytes a row
    const int live = live_rows(geo, c);
#pragma unroll
    for (int i = 0; i < kRows / kRowsAtOnce; ++i) {
      const int r = i * kRowsAtOnce + lane / kPieces, row = c.rt * kRows + r, tok = geo.group == geo.rows ? 0 : row / geo.group;
      const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q);
      if (r < live)
        src += (static_cast<long long>(c.s) * p.batch.L + tok) * p.ld_q + (c.h * geo.group + row - tok * geo.group) * kDh + lane % kPieces * 8;
      copy16(to + (i * 32 + lane) * 16, src, r < live);
    }
  }

  // The queries' fragments; in 4 bits each row times a power of two that makes its largest 2^14 to 2^15 (fp16 holds all bits of a
  // bf16 down to 2^-28 of that, of the part that is a sixteenth, too; a row with an infinity or NaN is NaN).
  __device__ __forceinline__ void begin(const PagedAttentionArgs& p, const Geometry& geo, const Place& c, int live, int lane,
                                        uint2* shared) {
    const int g = lane >> 2, t = lane & 3;
    q = shared;
    uint4 raw[kDh / 32];
#pragma unroll
    for (int i = 0; i < kDh / 32; ++i)
      raw[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(shared) + g * kDh +
                                               (kInt4 ? 64 * (i >> 1) + 16 * t + 8 * (i & 1) : 32 * i + 8 * t));
    __syncwarp();  // (these eight rows' fragments take these eight rows' place)
    auto put = [&](int step, uint2 f) { shared[step * 32 + lane] = f; };
    float by_row = p.scale * 1.4426950408889634f;
    if constexpr (kInt4) {
      float x[kDh / 32][8], top = 0.f;
#pragma unroll
      for (int i = 0; i < kDh / 32; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[i][2 * e] = bf16_lo(w[e]);
          x[i][2 * e + 1] = bf16_hi(w[e]);
          top = fmaxf(top, fmaxf(fabsf(x[i][2 * e]), fabsf(x[i][2 * e + 1])));
        }
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int exponent = (__float_as_int(top) >> 23) - 127;  // -127 for 0 and what is below 2^-126
      const int by = min(126, 14 - exponent);
      by_row = exponent > 127 ? __int_as_float(0x7fffffff) : by_row * pow2(max(-by, -126));
      const float up = pow2(by);
#pragma unroll
      for (int i = 0; i < kDh / 32; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          put(2 * i + h, make_uint2(pack_f16(x[i][2 * h] * up, x[i][2 * h + 4] * up),
                                    pack_f16(x[i][2 * h + 1] * (up * 0.0625f), x[i][2 * h + 5] * (up * 0.0625f))));
    } else {
#pragma unroll
      for (int i = 0; i < kDh / 32; ++i) {
        put(2 * i, make_uint2(raw[i].x, raw[i].y));
        put(2 * i + 1, make_uint2(raw[i].z, raw[i].w));
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      factor[e] = __shfl_sync(0xffffffffu, by_row, (2 * t + e) * 4);
      limit[e] = c.seq.cached +
                    (geo.group == geo.rows ? 0 : min((c.rt * kRows + 2 * t + e) / geo.group, c.seq.n - 1));
      m[e] = kLowest;
      l[e] = 0.f;
#pragma unroll
      for (int gr = 0; gr < kGroups; ++gr) lift[e][gr] = 1.f;
    }
#pragma unroll
    for (int j = 0; j < C::kMTiles; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    first_limit = c.seq.cached + c.rt * kRows / geo.group;
    last_limit = c.seq.cached + (min(kRows, live) + c.rt * kRows - 1) / geo.group;
    __syncwarp();
  }

  // kN neighbouring tiles, the first at position `pos`; kMasked: some of their tokens may lie behind what some rows see.
  template <int kN, bool kMasked>
  __device__ __forceinline__ void take(const uint8_t* first_tile, int pos, int lane) {
    using Tile = typename C::Tile;
    constexpr int kWords = kDh / 32;
    const int g = lane >> 2, t = lane & 3;
    // ---- scores: S^T = K q^T
    // (as exponents of 2, and numbers of their own: a product that is rounded only when the maximum comes off lies, beyond 2^25,
    // further from the maximum than the range that follows)
    float sc[kN][4], sv[kN][2][kGroups];  // values' scales of tokens g and g + 8
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const uint8_t* tp = first_tile + i * Tile::kBytes;
      float part[kGroups][4];
      if constexpr (kInt4) {
        float sk[2][kGroups];
        uint32_t zk[2][kGroups], kw[2][kWords];
        if constexpr (kDh == 128) {
          const uint4 s4 = *reinterpret_cast<const uint4*>(tp + Tile::kScales + g * 16);
          const uint2 z2 = *reinterpret_cast<const uint2*>(tp + Tile::kZerosK + g * 8);
          const uint32_t kk[2] = {s4.x, s4.z}, vv[2] = {s4.y, s4.w}, zz[2] = {z2.x, z2.y};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            sk[h][0] = bf16_lo(kk[h]);
            sk[h][kGroups - 1] = bf16_hi(kk[h]);
            sv[i][h][0] = bf16_lo(vv[h]);
            sv[i][h][kGroups - 1] = bf16_hi(vv[h]);
            zk[h][0] = __byte_perm(zz[h], 0, 0x1010);
            zk[h][kGroups - 1] = __byte_perm(zz[h], 0, 0x3232);
            const uint4 w = *reinterpret_cast<const uint4*>(tp + (g + 8 * h) * 64 + t * 16);
            kw[h][0] = w.x;
            kw[h][1] = w.y;
            kw[h][kWords - 2] = w.z;
            kw[h][kWords - 1] = w.w;
          }
        } else {
          const uint2 s2 = *reinterpret_cast<const uint2*>(tp + Tile::kScales + g * 8);
          const uint32_t z1 = *reinterpret_cast<const uint32_t*>(tp + Tile::kZerosK + g * 4);
          const uint32_t kv[2] = {s2.x, s2.y};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            sk[h][0] = bf16_lo(kv[h]);
            sv[i][h][0] = bf16_hi(kv[h]);
            zk[h][0] = __byte_perm(z1, 0, h == 0 ? 0x1010 : 0x3232);
            const uint2 w = *reinterpret_cast<const uint2*>(tp + (g + 8 * h) * 32 + t * 8);
            kw[h][0] = w.x;
            kw[h][1] = w.y;
          }
        }
        uint32_t minus[2][kGroups][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            minus[h][gr][0] = minus_low(zk[h][gr], minus1024);
            minus[h][gr][1] = minus_high(minus[h][gr][0]);
          }
#pragma unroll
        for (int step = 0; step < 4; ++step)
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {  // (groups in turn: their sums are chains)
            const int w = 2 * gr + step / 2, x = step % 2;
            const uint32_t w0 = x == 0 ? kw[0][w] : kw[0][w] >> 8, w1 = x == 0 ? kw[1][w] : kw[1][w] >> 8;
            const uint32_t a[4] = {low_nibbles(w0, minus[0][gr][0], plus1024), low_nibbles(w1, minus[1][gr][0], plus1024),
                                   high_nibbles(w0, minus[0][gr][1], plus1024), high_nibbles(w1, minus[1][gr][1], plus1024)};
            const uint2 f = query(2 * w + x, lane);
            if (step == 0) first_mma_f16(part[gr], a, f.x, f.y); else mma_f16(part[gr], a, f.x, f.y);
          }
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // (the row's factor before the keys' scales: the sums of large keys alone would pass fp32)
          const float2 f = make_float2(factor[0], factor[1]);
          float2 s = mul2(mul2(make_float2(part[0][2 * h], part[0][2 * h + 1]), f), make_float2(sk[h][0], sk[h][0]));
          if constexpr (kGroups == 2)
            s = fma2(mul2(make_float2(part[1][2 * h], part[1][2 * h + 1]), f), make_float2(sk[h][1], sk[h][1]), s);
          sc[i][2 * h] = s.x;
          sc[i][2 * h + 1] = s.y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) part[0][e] = 0.f;
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          const uint4 k0 = *reinterpret_cast<const uint4*>(tp + (w * kKvTile + g) * 64 + t * 16);
          const uint4 k1 = *reinterpret_cast<const uint4*>(tp + (w * kKvTile + g + 8) * 64 + t * 16);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t a[4] = {x == 0 ? k0.x : k0.z, x == 0 ? k1.x : k1.z, x == 0 ? k0.y : k0.w, x == 0 ? k1.y : k1.w};
            const uint2 f = query(2 * w + x, lane);
            mma_bf16(part[0], a, f.x, f.y);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[i][e] = __fmul_rn(part[0][e], factor[e & 1]);
      }
    }

    // ---- relative to m: a score's exponent, -inf where the row does not see the token; probabilities, turned into the
    // second product's fragments (4 bits: by group of channels; bf16: the probability and what its rounding left)
    float pr[kN][4];
    uint32_t pf[kN][2][2];
    auto hidden = [&](int i, int e) { return kMasked && pos + kKvTile * i + g + 8 * (e >> 1) > limit[e & 1]; };
    auto probabilities = [&]() {
      bool far = false;
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < kN; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float ex = sc[i][e] - m[e & 1];
          if (hidden(i, e)) ex = -INFINITY;
          far |= ex > kSlack;
          pr[i][e] = ex2(ex);
        }
        if constexpr (kInt4) {
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // (both rows at once: 64 sequences of up to 800 tokens 47.4 us, singly 48.8)
              float2 w = mul2(mul2(make_float2(pr[i][2 * h], pr[i][2 * h + 1]), make_float2(lift[0][gr], lift[1][gr])),
                              make_float2(sv[i][h][gr], sv[i][h][gr]));
              if (hidden(i, 2 * h)) w.x = 0.f;  // whatever its scale is
              if (hidden(i, 2 * h + 1)) w.y = 0.f;
              pf[i][gr][h] = pack_f16(w.x, w.y);
            }
            most = max_f16(most, max_f16(pf[i][gr][0], pf[i][gr][1]));
          }
        }
      }
      if constexpr (kInt4) far |= above_f16(most);
      return far;
    };
    if (__any_sync(0xffffffffu, probabilities())) {
      // (both rows at once: this runs at every item's start)
      float score[kN][4], top[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < kN; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          score[i][e] = hidden(i, e) ? -INFINITY : sc[i][e];
          top[e & 1] = fmaxf(top[e & 1], score[i][e]);
        }
#pragma unroll
      for (int off = 4; off < 32; off <<= 1)
#pragma unroll
        for (int e = 0; e < 2; ++e) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], off));
      // (a row of which nothing passes its range keeps what it has: what it does not see must not change it; whole exponents, so
      // that what is added up is scaled without a rounding)
      int up[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bool moves = top[e] - m[e] > kSlack;
        const float now = moves ? ceilf(top[e]) : m[e];
        up[e] = moves ? static_cast<int>(fminf(now - m[e], 1000.f)) : 0;
        m[e] = now;
        l[e] *= pow2_or_0(-up[e]);
      }
      if constexpr (kInt4) {
        float most[2][kGroups];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            most[e][gr] = -INFINITY;
#pragma unroll
            for (int i = 0; i < kN; ++i)
#pragma unroll
              for (int h = 0; h < 2; ++h) most[e][gr] = fmaxf(most[e][gr], score[i][e + 2 * h] - m[e] + lg2_or_none(sv[i][h][gr]));
          }
#pragma unroll
        for (int off = 4; off < 32; off <<= 1)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int gr = 0; gr < kGroups; ++gr) most[e][gr] = fmaxf(most[e][gr], __shfl_xor_sync(0xffffffffu, most[e][gr], off));
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            // what is held stays what it is when m moves, as far as the lift reaches
            const int was = (__float_as_int(lift[e][gr]) >> 23) - 127 + up[e];
            const int by = min(most[e][gr] + static_cast<float>(was) > kMost ? max(kTop - static_cast<int>(ceilf(most[e][gr])), kLiftLeast) : was,
                               kLiftMost);
            lift[e][gr] = pow2(by);
            const float held = pow2_or_0(by - was);
#pragma unroll
            for (int j = gr * 4; j < gr * 4 + 4; ++j) {
              o[j][e] *= held;
              o[j][e + 2] *= held;
            }
          }
      } else {
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int j = 0; j < C::kMTiles; ++j) {
            o[j][e] *= pow2_or_0(-up[e]);
            o[j][e + 2] *= pow2_or_0(-up[e]);
          }
      }
      probabilities();
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      l[0] += pr[i][0] + pr[i][2];
      l[1] += pr[i][1] + pr[i][3];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (kInt4) {
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) pf[i][gr][h] = turned(pf[i][gr][h]);
        } else {
          const uint32_t top = pack_bf16x2(pr[i][2 * h], pr[i][2 * h + 1]);
          pf[i][0][h] = turned(top);
          pf[i][1][h] = turned(pack_bf16x2(pr[i][2 * h] - bf16_lo(top), pr[i][2 * h + 1] - bf16_hi(top)));
        }
      }
    }

    // ---- O^T += V^T P^T
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const uint8_t* tp = first_tile + i * Tile::kBytes;
      if constexpr (kInt4) {
        uint32_t zv[2][kGroups], vw[2][kWords];
        if constexpr (kDh == 128) {
          const uint4 z4 = *reinterpret_cast<const uint4*>(tp + Tile::kZerosV + t * 16);
          zv[0][0] = z4.x;
          zv[0][kGroups - 1] = z4.y;
          zv[1][0] = z4.z;
          zv[1][kGroups - 1] = z4.w;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 w = *reinterpret_cast<const uint4*>(tp + Tile::kValues + h * 512 + lane * 16);
            vw[h][0] = w.x;
            vw[h][1] = w.y;
            vw[h][kWords - 2] = w.z;
            vw[h][kWords - 1] = w.w;
          }
        } else {
          const uint2 z2 = *reinterpret_cast<const uint2*>(tp + Tile::kZerosV + t * 8);
          zv[0][0] = z2.x;
          zv[1][0] = z2.y;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint2 w = *reinterpret_cast<const uint2*>(tp + Tile::kValues + h * 256 + lane * 8);
            vw[h][0] = w.x;
            vw[h][1] = w.y;
          }
        }
        uint32_t minus[2][kGroups][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            minus[h][gr][0] = minus_low(zv[h][gr], minus1024);
            minus[h][gr][1] = minus_high(minus[h][gr][0]);
          }
#pragma unroll
        for (int j = 0; j < C::kMTiles; ++j) {
          const int w = j / 2, gr = w / 2;
          const uint32_t w0 = j % 2 == 0 ? vw[0][w] : vw[0][w] >> 8, w1 = j % 2 == 0 ? vw[1][w] : vw[1][w] >> 8;
          const uint32_t a[4] = {low_nibbles(w0, minus[0][gr][0], plus1024), high_nibbles(w0, minus[0][gr][1], plus1024),
                                 low_nibbles(w1, minus[1][gr][0], plus1024), high_nibbles(w1, minus[1][gr][1], plus1024)};
          mma_f16(o[j], a, pf[i][gr][0], pf[i][gr][1]);
        }
      } else {
        // bytes behind the last token count as zeros, an infinity or NaN that some rows may see too, at first
        uint32_t keep[2];
        if constexpr (kMasked) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int first = pos + kKvTile * i + 8 * h + 2 * t;
            keep[h] = (first <= last_limit ? 0x0000ffffu : 0u) | (first + 1 <= last_limit ? 0xffff0000u : 0u);
          }
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          const uint4 v0 = *reinterpret_cast<const uint4*>(tp + Tile::kValues + (w * 32 + lane) * 16);
          const uint4 v1 = *reinterpret_cast<const uint4*>(tp + Tile::kValues + ((kWords + w) * 32 + lane) * 16);
          uint32_t v[2][4] = {{v0.x, v0.y, v0.z, v0.w}, {v1.x, v1.y, v1.z, v1.w}}, sick[2][4];
          bool any = false;
          if constexpr (kMasked) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                v[h][x] &= keep[h];
                sick[h][x] = ((v[h][x] & 0x7f80u) == 0x7f80u ? v[h][x] & 0xffffu : 0u) |
                             ((v[h][x] & 0x7f800000u) == 0x7f800000u ? v[h][x] & 0xffff0000u : 0u);
                v[h][x] ^= sick[h][x];
                any |= sick[h][x] != 0;
              }
            }
            any = __any_sync(0xffffffffu, any);
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int j = 2 * w + x;
            const uint32_t a[4] = {v[0][2 * x], v[0][2 * x + 1], v[1][2 * x], v[1][2 * x + 1]};
            mma_bf16(o[j], a, pf[i][0][0], pf[i][0][1]);
            mma_bf16(o[j], a, pf[i][1][0], pf[i][1][1]);
            if constexpr (kMasked) {
              if (any) {  // a token at a time, for the rows that see it
#pragma unroll 1
                for (int tok = 0; tok < kKvTile; ++tok) {
                  const uint32_t half = t == (tok & 7) / 2 ? ((tok & 1) == 0 ? 0x0000ffffu : 0xffff0000u) : 0u;
                  uint32_t b[4];
#pragma unroll
                  for (int y = 0; y < 2; ++y) {
                    b[y] = tok < 8 ? sick[0][2 * x + y] & half : 0u;
                    b[2 + y] = tok < 8 ? 0u : sick[1][2 * x + y] & half;
                  }
                  float d[4] = {0.f, 0.f, 0.f, 0.f};
                  mma_bf16(d, b, pf[i][0][0], pf[i][0][1]);
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    if (pos + kKvTile * i + tok <= limit[e & 1]) o[j][e] += d[e];
                }
              }
            }
          }
        }
      }
    }
  }

  // What the lane has of row 2t + e, normalised: f(first channel, values) for every four neighbouring channels.
  template <typename F>
  __device__ __forceinline__ void each(int e, float by, int lane, F f) const {
    const int g = lane >> 2;
    const float high = kInt4 ? by * 0.0625f : by;
#pragma unroll
    for (int j = 0; j < C::kMTiles; j += 2) {
      float4 v = make_float4(o[j][e] * by, o[j][e + 2] * high, o[j + 1][e] * by, o[j + 1][e + 2] * high);
      if constexpr (kInt4) {
        const float held = pow2(127 - (__float_as_int(lift[e][j >> 2]) >> 23));  // its reciprocal
        v = make_float4(v.x * held, v.y * held, v.z * held, v.w * held);
      }
      f(kInt4 ? 64 * (j >> 2) + 8 * g + 2 * (j & 3) : 32 * (j >> 1) + 4 * g, v);
    }
  }
};

// ---------------------------------------------------------------- the kernel

// Parts in the workspace: of each CTA two (what Desc says), then of each warp one.
template <int kDh>
__device__ __forceinline__ Part<kDh>* cta_part(const PagedAttentionArgs& p, int cta, int slot) {
  return reinterpret_cast<Part<kDh>*>(static_cast<uint8_t*>(p.ws) + sizeof(Desc) * kMaxCtas) + 2 * cta + slot;
}
template <int kDh>
__device__ __forceinline__ Part<kDh>* warp_part(const PagedAttentionArgs& p, int warp) {
  return cta_part<kDh>(p, kMaxCtas, 0) + blockIdx.x * kWarps + warp;
}

__device__ __forceinline__ __nv_bfloat16* out_row(const PagedAttentionArgs& p, const Geometry& geo, int s, int row, int h, int head_dim) {
  const int tok = row / geo.group;
  return static_cast<__nv_bfloat16*>(p.out) + (static_cast<long long>(s) * p.batch.L + tok) * p.ld_out +
         (h * geo.group + row - tok * geo.group) * head_dim;
}

template <int kDh, bool kInt4>
__global__ void __launch_bounds__(kThreads, Config<kDh, kInt4>::kCtasPerSm)
    paged_attention_kernel(const PagedAttentionArgs p, bool aligned) {
  using C = Config<kDh, kInt4>;
  using Tile = typename C::Tile;
  using Parts = Part<kDh>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Shared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint8_t* const ring = smem + warp * (C::kStages * C::kStageBytes);
  pdl_wait();
  pdl_launch_dependents();
  const Geometry geo = geometry(p);
  Place c;
  int active;
  int left = begin(p, geo, aligned, c, active, sh);
  WarpEnd end{0, 0, 0, 0, false, false, false, false, 0};
  if (left > 0) {
    Place& load = sh.load[warp];
    Place& take = sh.take[warp];
    int& load_left = sh.load_left[warp];
    const uint32_t ring_at = smem_u32(ring);
    uint2* const queries = reinterpret_cast<uint2*>(smem + C::kRing + warp * C::kQ);
    using R = Rows<kDh, kInt4>;
    R::fetch(p, geo, c, lane, smem_u32(queries));
    Loader<kDh, kInt4> loader;
    load = c;
    take = c;
    load_left = left;
    __syncwarp();
    Rows<kDh, kInt4> rows;
    rows.plus1024 = held(kFp16Of1024);
    rows.minus1024 = held(kFp16OfMinus1024);
    int used = 0;  // stages
    int lo = 0, tile = 0, hi = 0, live = 0;  // the warp's part of the present item, the next tile; rows with a token
    bool open = false;
    int bad_from = INT_MAX;  // first position of the item whose page is none of the cache's
    // (one place each where a stage is filled, an item begun and ended: what runs rarely runs from a cold instruction cache)
    int fast = 0;  // stages that need no second look, neither when taken nor (copying) when filled again
    bool copying = false;
#pragma unroll 1
    for (;;) {
      if (fast == 0) {
      if (loader.issued - used < C::kStages) {
        loader.issue(p, geo, load, load_left, lane, ring_at);
        if (loader.issued - used < C::kStages) continue;
      }
      if (tile >= hi) {
        c = take;
        const int row0 = c.rt * kRows;
        if (open) {
          // ---- an item as a whole goes out, a part of one waits: the last segment's in the ring, an earlier one's in memory
          const bool last = left <= 0, ended = hi == max(1, c.tiles), whole = lo == 0 && ended;
          Place next = c;
          if (!last) {  // the next item's queries come while this one is finished
            next.next_item(p, geo);
            R::fetch(p, geo, next, lane, smem_u32(queries));
          }
          float* part_o = last ? reinterpret_cast<float*>(ring) : &warp_part<kDh>(p, warp)->o[0][0];
          float* part_mass = last ? sh.mass[warp] : warp_part<kDh>(p, warp)->mass;
          const int slots = min(kRows, geo.rows - row0);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int row = 2 * t + e;
            float sum = rows.l[e];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            const bool poison = rows.limit[e] >= bad_from;  // (a row that ends before it is what it is)
            const float by = poison ? __int_as_float(0x7fffffff) : 1.f / sum;  // (NaN where all scores are -inf)
            if (whole) {
              if (row < slots) {
                __nv_bfloat16* dst = out_row(p, geo, c.s, row0 + row, c.h, kDh);
                // an empty slot, or positions that cannot be (NaN)
                const uint32_t fill = !c.seq.ok && row0 + row < c.seq.n * geo.group ? 0x7fff7fffu : 0u;
                rows.each(e, by, lane, [&](int d, const float4& v) {
                  *reinterpret_cast<uint2*>(dst + d) =
                      row < live ? make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)) : make_uint2(fill, fill);
                });
              }
            } else if (row < live) {
              rows.each(e, by, lane, [&](int d, const float4& v) { *reinterpret_cast<float4*>(part_o + row * kDh + d) = v; });
              if (g == 0)
                part_mass[row] = poison ? __int_as_float(0x7fffffff) : sum == 0.f ? kNothing : rows.m[e] + log2f(sum);
            }
          }
          if (!whole) {
            if (lo > 0) {
              end.first = true;
              end.first_rt = c.rt;
              end.first_last = last;
              end.first_ends = ended;
            } else {
              end.tail = true;
              end.live = live;
            }
          }
          end.s = c.s;
          end.rt = c.rt;
          end.h = c.h;
          if (last) break;
          c = next;
          __syncwarp();
          take = c;
          __syncwarp();
        }
        // ---- the next item
        lo = tile = c.tile;
        hi = min(max(1, c.tiles), lo + left);
        left -= units_of_item(c.tiles) - lo;
        live = R::live_rows(geo, c);
        open = true;
        bad_from = INT_MAX;
        commit_copies();
        wait_copies<0>();
        rows.begin(p, geo, c, live, lane, queries);
        if (c.tiles == 0) {
          tile = hi;
          continue;
        }
      }
      constexpr int kT = C::kStageTiles;
      const int clear = min(hi, (rows.first_limit + 1) / kKvTile) - tile;
      if (!loader.bad && (tile & (kT - 1)) == 0 && clear >= kT) {
        const int same = min(loader.end, (loader.tile | 31) + 1) - loader.tile;
        copying = (loader.tile & (kT - 1)) == 0 && (loader.tile & ~31) == loader.base && same >= kT;
        fast = copying ? min(clear, same) / kT : 1;
      } else {
        const int n = stage_tiles<C>(tile, hi), pos = tile * kKvTile;
        const uint8_t* const at = ring + (used & (C::kStages - 1)) * C::kStageBytes;
        wait_copies<C::kStages - 1>();
        if (loader.bad)  // rare: whether it is these tiles' pages
          for (int i = 0; i < n; ++i)
            if (kv_page(p.batch, p.cache, take.s, pos + i * kKvTile, nullptr) < 0) bad_from = min(bad_from, pos + i * kKvTile);
#pragma unroll 1
        for (int i = 0; i < n; ++i) rows.template take<1, true>(at + i * Tile::kBytes, pos + i * kKvTile, lane);
        __syncwarp();
        ++used;
        tile += n;
        continue;
      }
      }
      --fast;
      const uint8_t* const at = ring + (used & (C::kStages - 1)) * C::kStageBytes;
      wait_copies<C::kStages - 1>();
      rows.template take<C::kStageTiles, false>(at, tile * kKvTile, lane);
      __syncwarp();
      ++used;
      tile += C::kStageTiles;
      if (copying) loader.fill(p, C::kStageTiles, lane, ring_at);
    }
  }
  if (lane == 0) sh.end[warp] = end;
  __syncthreads();

  // ---- chains of parts of one item: from what an earlier CTA began, or from a warp's tail, over the following warps' first
  // parts to the one that ends it. A warp a row of a chain; a lane holds a part's mass, and all parts are read at once.
  const WarpEnd& my_end = sh.end[lane & (kWarps - 1)];
  const unsigned have = (1u << active) - 1;
  const unsigned firsts = __ballot_sync(0xffffffffu, my_end.first) & have, enders = __ballot_sync(0xffffffffu, my_end.first_ends) & have;
  const unsigned tails = __ballot_sync(0xffffffffu, my_end.tail) & have, ringed = __ballot_sync(0xffffffffu, my_end.first_last) & have;
  int turn = 0, tail_warp = -1;
  bool ends = false;
  for (unsigned starts = (firsts & 1u) | tails << 1; starts != 0; starts &= starts - 1) {
    const int start = __ffs(starts) - 2, next = start + 1;  // start -1: an earlier CTA's
    // the run of first parts from `next` on, up to the one that ends the item
    const unsigned run = ~(firsts >> next), stop_at = enders >> next;
    const int length = __ffs(run) - 1, end_at = __ffs(stop_at);
    const bool done = end_at > 0 && end_at <= length;
    const int stop = next + (done ? end_at : length);
    if (start < 0) ends = done;
    else if (!done) tail_warp = start;
    const WarpEnd& item = sh.end[max(start, 0)];
    const int rt = start < 0 ? item.first_rt : item.rt, shown = min(kRows, geo.rows - rt * kRows);
    constexpr int kE = kDh / 32;
    // (rows past the last token hold nothing; what is made of them is not read)
    for (int row = (warp - turn) & (kWarps - 1); row < shown; row += kWarps) {
      using Vec = typename C::Vec;
      const bool there = lane < stop && lane >= max(start, 0), near = lane == start || (ringed >> (lane & 31) & 1) != 0;
      const int w0 = there ? lane : 0;
      const Parts* far_part = warp_part<kDh>(p, w0);
      const float* row_at = there && !near ? far_part->o[row]
                                           : reinterpret_cast<const float*>(smem + w0 * (C::kStages * C::kStageBytes)) + row * kDh;
      const float mass = !there ? kNothing : near ? sh.mass[w0][row] : far_part->mass[row];
      Vec in[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w)
        in[w] = reinterpret_cast<const Vec*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row_at), w))[lane];
      float top = mass;
#pragma unroll
      for (int off = 4; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
      const float weight = mass == kNothing ? 0.f : ex2(mass - top);
      float sum = weight;
#pragma unroll
      for (int off = 4; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      const float share = weight / sum;  // (0 / 0 where all scores are -inf: NaN, which the mass keeps from counting beside others)
      float out[kE];
#pragma unroll
      for (int i = 0; i < kE; ++i) out[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float by = __shfl_sync(0xffffffffu, share, w);
        if (by == 0.f) continue;
        const float* x = reinterpret_cast<const float*>(&in[w]);
#pragma unroll
        for (int i = 0; i < kE; ++i) out[i] = fmaf(x[i], by, out[i]);
      }
      if (start >= 0 && done) {
        __nv_bfloat16* dst = out_row(p, geo, item.s, rt * kRows + row, item.h, kDh) + lane * kE;
#pragma unroll
        for (int i = 0; i < kE; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = row < item.live ? pack_bf16x2(out[i], out[i + 1]) : 0u;
      } else {
        Parts* to = cta_part<kDh>(p, blockIdx.x, start < 0 ? 0 : 1);
#pragma unroll
        for (int i = 0; i < kE; ++i) to->o[row][lane * kE + i] = out[i];
        const float total = __shfl_sync(0xffffffffu, sum, 0), highest = __shfl_sync(0xffffffffu, top, 0);
        if (lane == 0) to->mass[row] = total == 0.f ? kNothing : highest + log2f(total);
      }
    }
    turn += shown;
  }
  if (threadIdx.x == 0) {
    Desc d{0, 0, 0, -1, ends, 0, {0, 0}};
    if (tail_warp >= 0) {
      d.s = sh.end[tail_warp].s;
      d.rt = sh.end[tail_warp].rt;
      d.h = sh.end[tail_warp].h;
      d.live = sh.end[tail_warp].live;
      d.slot = 1;
    }
    static_cast<Desc*>(p.ws)[blockIdx.x] = d;
  }
}

// Items that several CTAs have parts of: the CTA that holds an item's first part adds up all of them, a row in y.
template <int kDh>
__global__ void __launch_bounds__(kThreads) paged_attention_join_kernel(const PagedAttentionArgs p, int ctas) {
  __shared__ float sh_o[kWarps][kDh], sh_sum[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  const Desc* desc = static_cast<const Desc*>(p.ws);
  const int b = blockIdx.x, row = blockIdx.y;
  const Desc mine = desc[b];
  int more = b + 1 + lane < ctas && desc[b + 1 + lane].ends != 0;  // (read beside it)
  if (mine.slot < 0) return;
  const Geometry geo = geometry(p);
  const int q_row = mine.rt * kRows + row;
  if (q_row >= geo.rows) return;
  int end = ctas;  // parts: this CTA's, then slot 0 of those up to the first that ends the item
  for (int at = b + 1; at < ctas; at += 32) {
    const unsigned found = __ballot_sync(0xffffffffu, more);
    if (found != 0) {
      end = at + __ffs(found);
      break;
    }
    more = at + 32 + lane < ctas && desc[at + 32 + lane].ends != 0;
  }
  // a lane a part's mass; a warp adds up every eighth part, its loads independent of each other
  using Vec = std::conditional_t<kDh == 128, float4, float2>;
  constexpr int kE = kDh / 32;
  const int n = end - b;
  float mass = kNothing, top, sum = 0.f, out[kE];
  for (int i = lane; i < n; i += 32) mass = fmaxf(mass, cta_part<kDh>(p, b + i, i == 0 ? mine.slot : 0)->mass[row]);
  top = mass;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
#pragma unroll
  for (int i = 0; i < kE; ++i) out[i] = 0.f;
#pragma unroll 4
  for (int i = warp; i < n; i += kWarps) {
    const Part<kDh>* part = cta_part<kDh>(p, b + i, i == 0 ? mine.slot : 0);
    const Vec x = reinterpret_cast<const Vec*>(part->o[row])[lane];
    const float m = part->mass[row], weight = m == kNothing ? 0.f : ex2(m - top);
    sum += weight;
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (weight != 0.f) out[e] = fmaf(reinterpret_cast<const float*>(&x)[e], weight, out[e]);
  }
#pragma unroll
  for (int i = 0; i < kE; ++i) sh_o[warp][lane * kE + i] = out[i];
  if (lane == 0) sh_sum[warp] = sum;
  __syncthreads();
  if (threadIdx.x < kDh) {
    float total = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      total += sh_sum[w];
      acc += sh_o[w][threadIdx.x];
    }
    __nv_bfloat16* dst = out_row(p, geo, mine.s, q_row, mine.h, kDh);
    dst[threadIdx.x] = __float2bfloat16_rn(row >= mine.live ? 0.f : acc / total);
  }
}

template <int kDh, bool kInt4>
int launch(const PagedAttentionArgs& a, cudaStream_t st) {
  using C = Config<kDh, kInt4>;
  static_assert(C::kSmem * C::kCtasPerSm <= 227 * 1024, "shared memory of an SM");
  static std::atomic<bool> attr_set[64];  // the shared-memory limit is a per-device attribute; host threads may ask at once
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return -3;
  if (!attr_set[dev]) {
    if (cudaFuncSetAttribute(paged_attention_kernel<kDh, kInt4>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) !=
        cudaSuccess)
      return -3;
    attr_set[dev] = true;
  }
  const int ctas = std::min(kMaxCtas, std::max(1, sm_count()) * C::kCtasPerSm);
  const int64_t rows = a.n_heads / a.cache.kv_heads * a.batch.L;
  const int64_t items = a.batch.S * a.cache.kv_heads * ((rows + kRows - 1) / kRows);
  const int64_t tokens = (!kInt4 || kDh == 64) && 4 * items >= ctas ? 2 * kAlignedTokens : kAlignedTokens;
  const bool aligned = items <= ctas && (a.batch.max_pages << a.cache.page_bits) <= tokens;
  if (aligned)
    return launch_pdl(paged_attention_kernel<kDh, kInt4>, dim3(static_cast<unsigned>(items)), dim3(kThreads), C::kSmem, st, a, true) ==
                   cudaSuccess
               ? 0
               : -3;
  if (launch_pdl(paged_attention_kernel<kDh, kInt4>, dim3(ctas), dim3(kThreads), C::kSmem, st, a, false) != cudaSuccess) return -3;
  const dim3 grid(ctas, static_cast<unsigned>(std::min<int64_t>(rows, kRows)));
  return launch_pdl(paged_attention_join_kernel<kDh>, grid, dim3(kThreads), 0, st, a, ctas) == cudaSuccess ? 0 : -3;
}

}  // namespace

size_t paged_attention_workspace_bytes(int64_t head_dim) {
  return sizeof(Desc) * kMaxCtas + (2 + kWarps) * kMaxCtas * (head_dim == 128 ? sizeof(Part<128>) : sizeof(Part<64>));
}

int launch_paged_attention(const PagedAttentionArgs& a, cudaStream_t st) {
  if (a.cache.head_dim == 128) return a.cache.int4 ? launch<128, true>(a, st) : launch<128, false>(a, st);
  return a.cache.int4 ? launch<64, true>(a, st) : launch<64, false>(a, st);
}

}  // namespace hydra
