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
// into its probability, which is the one thing that is rounded (to fp16, 2^-12; bf16's 2^-9 would add as much again to the
// error as the output's own rounding). To keep that in fp16's range, m is not the largest score but that of probability
// times scale, and moved only when a row's passes the range, which a vote finds: the pass would spend its time on
// maxima else. A bf16 cache takes the probability as two bf16.
//
// Bound by the cache's bytes. Work is cut evenly: the tiles of all (sequence, rows, head) items in a row, a contiguous part for
// each warp, which copies its tiles into a ring of its own (cp.async.bulk) and needs no other warp on the way: it writes the
// items that it has whole. What it has of an item that others share it leaves until the CTA's end, where the parts of the
// CTA's warps are added up, and what CTAs share a second kernel adds up, both in the order of the parts.
#include <algorithm>
#include <climits>

#include "kv_cache.cuh"

namespace hydra {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxCtas = 320;     // of a grid; parts of items lie in the workspace, two a CTA and one a warp
constexpr int kMaxRowTiles = 4;   // of 8 query rows that share a pass
constexpr int kMinUnits = 4;      // tiles of a warp, where there are more warps than that fills
constexpr float kFar = -1e30f;    // a maximum of nothing
// Exponents relative to m. bf16: a probability up to 2^8. 4 bits: probability times scale from 2^6, when m is set, up to
// 2^14 (fp16 ends at 2^16, and keeps 11 bits down to 2^-14); the probability alone, whose scale may be 0, up to 2^108.
constexpr float kSlack = 8.f, kTop = 6.f, kMost = 14.f, kAlone = 100.f;

// What a CTA leaves for the second kernel.
struct Desc {
  int s, rt, h;   // the item that its last segment begins and does not end, if slot >= 0
  int slot;       // where that segment's part lies, or -1
  int ends;       // its first segment (slot 0) ends an item that an earlier CTA began
  int pad[3];
};

// Part of an item's rows, normalised, with log2 of the sum of exp2(s) that it stands for (NaN: unusable).
template <int kDh, int kR>
struct Part {
  float o[8 * kR][kDh];
  float mass[8 * kR];
};

template <int kDh, bool kInt4, int kR>
struct Config {
  using Tile = KvTile<kDh, kInt4>;
  using Parts = Part<kDh, kR>;
  static constexpr int kMTiles = kDh / 16;
  static constexpr int kCtasPerSm = kInt4 && kR == 1 ? 2 : 1;
  static constexpr bool kQShared = kR > 2;  // the queries' fragments: shared memory, else registers
  static constexpr int kPair = kInt4 && kR <= 2 ? 2 : 1;  // tiles that are taken together
  // a warp's ring also takes its last part at the end
  static constexpr int kLeast = (8 * kR * kDh * 4 + Tile::kBytes - 1) / Tile::kBytes;
  static constexpr int kWant = kInt4 ? 6 : kDh == 64 ? 4 : kR <= 2 ? 3 : 2;
  static constexpr int kStages = kWant > kLeast ? kWant : kLeast;
  static constexpr int kRing = kWarps * kStages * Tile::kBytes;
  static constexpr int kQ = kQShared ? kWarps * kR * kMTiles * 32 * 8 : 0;
  static constexpr int kSmem = kRing + kQ + kWarps * kStages * 8;
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
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool kInt4>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kInt4) mma_f16(d, a, b0, b1); else mma_bf16(d, a, b0, b1);
}
__device__ __forceinline__ uint32_t turned(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));  // (with subnormals: m may lie far above the scores)
  return y;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
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
// 2^e, e in [-126, 127]
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }

// code - zero of the low nibbles of the bytes 0 and 2 (16 (code - zero) of the high ones), as fp16.
__device__ __forceinline__ uint32_t low_nibbles(uint32_t w, uint32_t minus) { return add_f16((w & 0x000f000fu) | 0x64006400u, minus); }
__device__ __forceinline__ uint32_t high_nibbles(uint32_t w, uint32_t minus) { return add_f16((w & 0x00f000f0u) | 0x64006400u, minus); }
// -(1024 + zero), -(1024 + 16 zero) from two zero points as the cache holds them
__device__ __forceinline__ uint32_t minus_low(uint32_t z) { return (z & 0x000f000fu) | 0xe400e400u; }
__device__ __forceinline__ uint32_t minus_high(uint32_t z) { return (z & 0x00f000f0u) | 0xe400e400u; }

// ---------------------------------------------------------------- what is whose

struct Geometry {
  int group, rows, row_tiles, kv_heads;  // query heads of a kv head; rows of a kv head; passes over its rows
};
template <int kR>
__device__ __forceinline__ Geometry geometry(const PagedAttentionArgs& p) {
  Geometry g;
  g.kv_heads = p.cache.kv_heads;
  g.group = static_cast<int>(p.n_heads) / g.kv_heads;
  g.rows = g.group * static_cast<int>(p.batch.L);
  g.row_tiles = (g.rows + 8 * kR - 1) / (8 * kR);
  return g;
}

// Tiles of cached tokens that rows [8 kR rt, ...) of a sequence see; 0 where there is nothing to compute.
template <int kR>
__device__ __forceinline__ int tiles_of(const Geometry& g, const KvSeq& seq, int rt) {
  const int live = g.group * seq.n, first = rt * 8 * kR;
  if (!seq.ok || first >= live) return 0;
  const int last = (min(first + 8 * kR, live) - 1) / g.group;
  return (seq.cached + last) / kKvTile + 1;
}
// Units of a sequence's items of one head, at least one each: an item without tiles has rows to fill.
template <int kR>
__device__ __forceinline__ long long units_of(const Geometry& g, const KvSeq& seq) {
  long long n = 0;
  for (int rt = 0; rt < g.row_tiles; ++rt) n += max(1, tiles_of<kR>(g, seq, rt));
  return n;
}

__device__ __forceinline__ KvSeq seq_of(const PagedAttentionArgs& p, int s, int* err) {
  return kv_seq(p.batch, s, p.batch.max_pages << p.cache.page_bits, err);
}

// A place in the units: an item, and a tile of it.
template <int kR>
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
    tiles = tiles_of<kR>(g, seq, rt);
  }
};

// The exclusive prefix of a value over the block's threads, and its sum.
struct Scan {
  long long before, total;
};
__device__ __forceinline__ Scan block_scan(long long v, long long* sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sh[warp] = x;
  __syncthreads();
  Scan r{x - v, 0};
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) r.before += sh[w];
    r.total += sh[w];
  }
  __syncthreads();
  return r;
}

// Where the warp's part of the units begins, and how many they are. As few warps as have kMinUnits each, over all CTAs;
// `active` is how many of a CTA's warps these are.
struct Shared {
  long long scan[kWarps];
  long long offset[kWarps];
  int s[kWarps];
  WarpEnd end[kWarps];
  float mass[kWarps][8 * kMaxRowTiles];  // of the parts in the rings
  int abort;
};
template <int kR>
__device__ __forceinline__ int begin(const PagedAttentionArgs& p, const Geometry& g, Place<kR>& c, int& active, Shared& sh) {
  const int S = static_cast<int>(p.batch.S), warp = threadIdx.x >> 5;
  int* const err = blockIdx.x == 0 ? p.err : nullptr;
  long long mine = 0, total = 0;
  Scan scan{0, 0};
  for (int at = 0; at < S; at += kThreads) {
    const int s = at + static_cast<int>(threadIdx.x);
    mine = s < S ? units_of<kR>(g, seq_of(p, s, err)) * g.kv_heads : 0;
    scan = block_scan(mine, sh.scan);
    total += scan.total;
  }
  const long long want = (total + kMinUnits - 1) / kMinUnits;
  active = static_cast<int>(min(static_cast<long long>(kWarps), (want + gridDim.x - 1) / gridDim.x));
  const long long warps = min(want, static_cast<long long>(gridDim.x) * active);
  const long long first_warp = static_cast<long long>(blockIdx.x) * active;
  auto from = [&](long long w) { return w >= warps ? total : total * w / warps; };
  // the sequence that a warp's first unit is in
  long long before = 0;
  for (int at = 0; at < S; at += kThreads) {
    if (S > kThreads) {
      const int s = at + static_cast<int>(threadIdx.x);
      mine = s < S ? units_of<kR>(g, seq_of(p, s, nullptr)) * g.kv_heads : 0;
      scan = block_scan(mine, sh.scan);
    }
    const long long start = before + scan.before;
    for (int w = 0; w < active; ++w) {
      const long long first = from(first_warp + w);
      if (first >= start && first < start + mine) {
        sh.s[w] = at + static_cast<int>(threadIdx.x);
        sh.offset[w] = first - start;
      }
    }
    before += scan.total;
  }
  __syncthreads();
  if (warp >= active || first_warp + warp >= warps) return 0;
  c.s = sh.s[warp];
  long long rest = sh.offset[warp];
  c.seq = seq_of(p, c.s, nullptr);
  for (c.rt = 0;; ++c.rt) {
    c.tiles = tiles_of<kR>(g, c.seq, c.rt);
    const long long units = max(1, c.tiles);
    if (rest < units * g.kv_heads) {
      c.h = static_cast<int>(rest / units);
      c.tile = static_cast<int>(rest % units);
      break;
    }
    rest -= units * g.kv_heads;
  }
  return static_cast<int>(from(first_warp + warp + 1) - from(first_warp + warp));
}

// ---------------------------------------------------------------- a warp's copies

template <int kDh, bool kInt4, int kR>
struct Loader {
  using C = Config<kDh, kInt4, kR>;
  Place<kR> at;
  int left;                  // units not copied yet
  const int32_t* row;        // of the page table
  int page;                  // of the next tile, loaded a tile ahead
  const uint8_t* src;        // of the next tile, unless a page begins with it
  bool turn;                 // a page begins with it
  int stage = 0, issued = 0;
  uint32_t bad = 0;          // stages whose page is none of the cache's

  __device__ __forceinline__ void find(const PagedAttentionArgs& p, const Geometry& g) {
    while (left > 0 && at.tiles == 0)
      if (--left > 0) at.next_item(p, g);
    if (left <= 0) return;
    row = p.batch.table + static_cast<long long>(at.s) * p.batch.ld_table;
    page = row[(at.tile * kKvTile) >> p.cache.page_bits];
    turn = true;
  }
  __device__ __forceinline__ void issue(const PagedAttentionArgs& p, const Geometry& g, int lane, uint8_t* ring, uint32_t bars) {
    if (left <= 0) return;
    if (turn) {
      const bool ok = page >= 0 && page < p.cache.n_pages;
      if (!ok && lane == 0) record_error(p.err, kDevBadPage);
      src = kv_tile<typename C::Tile>(p.cache, ok ? page : 0, at.h, at.tile * kKvTile);
      page = ok ? page : -1;
      turn = false;
    }
    bad = page >= 0 ? bad & ~(1u << stage) : bad | (1u << stage);
    if (lane == 0) {
      const uint32_t bar = bars + 8 * stage;
      mbar_arrive_expect_tx(bar, C::Tile::kBytes);
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                       smem_u32(ring + stage * C::Tile::kBytes)),
                   "l"(reinterpret_cast<uint64_t>(src)), "r"(C::Tile::kBytes), "r"(bar)
                   : "memory");
    }
    stage = stage + 1 == C::kStages ? 0 : stage + 1;
    ++issued;
    --left;
    if (++at.tile == at.tiles) {
      if (left > 0) {
        at.next_item(p, g);
        find(p, g);
      }
    } else {
      src += C::Tile::kBytes;
      if ((at.tile & ((1 << (p.cache.page_bits - 4)) - 1)) == 0 && left > 0) {
        page = row[(at.tile * kKvTile) >> p.cache.page_bits];
        turn = true;
      }
    }
  }
};

// ---------------------------------------------------------------- a tile

// What a warp knows of its item's rows, and what it has added up.
template <int kDh, bool kInt4, int kR>
struct Rows {
  using C = Config<kDh, kInt4, kR>;
  float factor[kR][2];
  int limit[kR][2];             // last position that rows 2t and 2t + 1 of each eight see
  int first_limit, last_limit;  // the least and the largest of the rows'
  uint2 q[C::kQShared ? 1 : kR][C::kQShared ? 1 : kDh / 16];
  const uint2* q_shared;
  float o[C::kMTiles][kR][4], m[kR][2], l[kR][2];

  __device__ __forceinline__ uint2 query(int n, int step, int lane) const {
    if constexpr (C::kQShared) return q_shared[(n * C::kMTiles + step) * 32 + lane];
    else return q[n][step];
  }

  // The queries' fragments; in 4 bits (fp16) each row times a power of two that makes its largest 2^7.
  __device__ __forceinline__ void begin(const PagedAttentionArgs& p, const Geometry& geo, const Place<kR>& c, int live, int lane,
                                        uint2* to_shared) {
    const int g = lane >> 2, t = lane & 3;
    q_shared = to_shared;
#pragma unroll
    for (int n = 0; n < kR; ++n) {
      const int r = n * 8 + g, row = c.rt * 8 * kR + r;
      uint4 raw[kDh / 32];
#pragma unroll
      for (int i = 0; i < kDh / 32; ++i) raw[i] = make_uint4(0, 0, 0, 0);
      if (r < live) {
        const int tok = row / geo.group;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q) +
                                   (static_cast<long long>(c.s) * p.batch.L + tok) * p.ld_q +
                                   (c.h * geo.group + row - tok * geo.group) * kDh;
#pragma unroll
        for (int i = 0; i < kDh / 32; ++i)
          raw[i] = *reinterpret_cast<const uint4*>(src + (kInt4 ? 64 * (i >> 1) + 16 * t + 8 * (i & 1) : 32 * i + 8 * t));
      }
      auto put = [&](int step, uint2 f) {
        if constexpr (C::kQShared) to_shared[(n * C::kMTiles + step) * 32 + lane] = f; else q[n][step] = f;
      };
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
        const int by = exponent > 127 ? 0 : min(126, 7 - exponent);
        by_row *= pow2(max(-by, -126));
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
        factor[n][e] = __shfl_sync(0xffffffffu, by_row, (2 * t + e) * 4);
        limit[n][e] = c.seq.cached + min((c.rt * 8 * kR + n * 8 + 2 * t + e) / geo.group, c.seq.n - 1);
        m[n][e] = kFar;
        l[n][e] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < C::kMTiles; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][n][e] = 0.f;
    }
    first_limit = c.seq.cached + c.rt * 8 * kR / geo.group;
    last_limit = c.seq.cached + (min(8 * kR, live) + c.rt * 8 * kR - 1) / geo.group;
    if constexpr (C::kQShared) __syncwarp();
  }

  // kN neighbouring tiles, the first at position `pos`; kMasked: some of their tokens may lie behind what some rows see.
  template <int kN, bool kMasked>
  __device__ __forceinline__ void take(const uint8_t* const (&tiles)[kN], int pos, int lane) {
    using Tile = typename C::Tile;
    constexpr int kGroups = kInt4 ? kDh / kKvGroup : 1;  // that have a scale of their own
    constexpr int kWords = kDh / 32;
    const int g = lane >> 2, t = lane & 3;
    // ---- scores: S^T = K q^T
    float sc[kN][kR][4], sv[kN][2][kGroups];  // values' scales of tokens g and g + 8
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const uint8_t* tp = tiles[i];
      float part[kGroups][kR][4];
#pragma unroll
      for (int gr = 0; gr < kGroups; ++gr)
#pragma unroll
        for (int n = 0; n < kR; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) part[gr][n][e] = 0.f;
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
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          const int gr = w / 2;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t w0 = x == 0 ? kw[0][w] : kw[0][w] >> 8, w1 = x == 0 ? kw[1][w] : kw[1][w] >> 8;
            const uint32_t a[4] = {low_nibbles(w0, minus_low(zk[0][gr])), low_nibbles(w1, minus_low(zk[1][gr])),
                                   high_nibbles(w0, minus_high(zk[0][gr])), high_nibbles(w1, minus_high(zk[1][gr]))};
#pragma unroll
            for (int n = 0; n < kR; ++n) {
              const uint2 f = query(n, 2 * w + x, lane);
              mma<true>(part[gr][n], a, f.x, f.y);
            }
          }
        }
#pragma unroll
        for (int n = 0; n < kR; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sc[i][n][e] = part[0][n][e] * sk[e >> 1][0];
            if constexpr (kGroups == 2) sc[i][n][e] = fmaf(part[1][n][e], sk[e >> 1][1], sc[i][n][e]);
          }
      } else {
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          const uint4 k0 = *reinterpret_cast<const uint4*>(tp + (w * kKvTile + g) * 64 + t * 16);
          const uint4 k1 = *reinterpret_cast<const uint4*>(tp + (w * kKvTile + g + 8) * 64 + t * 16);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t a[4] = {x == 0 ? k0.x : k0.z, x == 0 ? k1.x : k1.z, x == 0 ? k0.y : k0.w, x == 0 ? k1.y : k1.w};
#pragma unroll
            for (int n = 0; n < kR; ++n) {
              const uint2 f = query(n, 2 * w + x, lane);
              mma<false>(part[0][n], a, f.x, f.y);
            }
          }
        }
#pragma unroll
        for (int n = 0; n < kR; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[i][n][e] = part[0][n][e];
      }
    }

    // ---- relative to m: a score's exponent, -inf where the row does not see the token; probabilities, turned into the
    // second product's fragments (4 bits: by group of channels; bf16: the probability and what its rounding left)
    float pr[kN][kR][4];
    uint32_t pf[kN][2][kR][2];
    auto hidden = [&](int i, int n, int e) { return kMasked && pos + kKvTile * i + g + 8 * (e >> 1) > limit[n][e & 1]; };
    auto probabilities = [&]() {
      bool far = false;
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < kN; ++i)
#pragma unroll
        for (int n = 0; n < kR; ++n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float ex = fmaf(sc[i][n][e], factor[n][e & 1], -m[n][e & 1]);
            if (hidden(i, n, e)) ex = -INFINITY;
            far |= ex > (kInt4 ? kAlone + kSlack : kSlack);
            pr[i][n][e] = ex2(ex);
          }
          if constexpr (kInt4) {
#pragma unroll
            for (int gr = 0; gr < kGroups; ++gr) {
              float w[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                w[e] = pr[i][n][e] * sv[i][e >> 1][gr];
                if (hidden(i, n, e)) w[e] = 0.f;  // whatever its scale is
              }
              pf[i][gr][n][0] = pack_f16(w[0], w[1]);
              pf[i][gr][n][1] = pack_f16(w[2], w[3]);
              most = max_f16(most, max_f16(pf[i][gr][n][0], pf[i][gr][n][1]));
            }
          }
        }
      if constexpr (kInt4) far |= above_f16(most);
      return far;
    };
    if (__any_sync(0xffffffffu, probabilities())) {
#pragma unroll
      for (int n = 0; n < kR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = -INFINITY, top_w = -INFINITY;
#pragma unroll
          for (int i = 0; i < kN; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float x = hidden(i, n, e + 2 * h) ? -INFINITY : sc[i][n][e + 2 * h] * factor[n][e];
              top = fmaxf(top, x);
              if constexpr (kInt4) top_w = fmaxf(top_w, x + lg2(fmaxf(sv[i][h][0], sv[i][h][kGroups - 1])));
            }
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            if constexpr (kInt4) top_w = fmaxf(top_w, __shfl_xor_sync(0xffffffffu, top_w, off));
          }
          // (the other rows keep theirs: what a row does not see must not change it)
          if (kInt4 ? top_w - m[n][e] > kMost || top - m[n][e] > kAlone + kSlack : top - m[n][e] > kSlack) {
            const float now = kInt4 ? fmaxf(top_w - kTop, top - kAlone) : top, by = ex2(m[n][e] - now);
            m[n][e] = now;
            l[n][e] *= by;
#pragma unroll
            for (int j = 0; j < C::kMTiles; ++j) {
              o[j][n][e] *= by;
              o[j][n][e + 2] *= by;
            }
          }
        }
      probabilities();
    }
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int n = 0; n < kR; ++n) {
        l[n][0] += pr[i][n][0] + pr[i][n][2];
        l[n][1] += pr[i][n][1] + pr[i][n][3];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if constexpr (kInt4) {
#pragma unroll
            for (int gr = 0; gr < kGroups; ++gr) pf[i][gr][n][h] = turned(pf[i][gr][n][h]);
          } else {
            const uint32_t top = pack_bf16x2(pr[i][n][2 * h], pr[i][n][2 * h + 1]);
            pf[i][0][n][h] = turned(top);
            pf[i][1][n][h] = turned(pack_bf16x2(pr[i][n][2 * h] - bf16_lo(top), pr[i][n][2 * h + 1] - bf16_hi(top)));
          }
        }
      }

    // ---- O^T += V^T P^T
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const uint8_t* tp = tiles[i];
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
#pragma unroll
        for (int j = 0; j < C::kMTiles; ++j) {
          const int w = j / 2, gr = w / 2;
          const uint32_t w0 = j % 2 == 0 ? vw[0][w] : vw[0][w] >> 8, w1 = j % 2 == 0 ? vw[1][w] : vw[1][w] >> 8;
          const uint32_t a[4] = {low_nibbles(w0, minus_low(zv[0][gr])), high_nibbles(w0, minus_high(zv[0][gr])),
                                 low_nibbles(w1, minus_low(zv[1][gr])), high_nibbles(w1, minus_high(zv[1][gr]))};
#pragma unroll
          for (int n = 0; n < kR; ++n) mma<true>(o[j][n], a, pf[i][gr][n][0], pf[i][gr][n][1]);
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
#pragma unroll
            for (int n = 0; n < kR; ++n) {
              mma<false>(o[j][n], a, pf[i][0][n][0], pf[i][0][n][1]);
              mma<false>(o[j][n], a, pf[i][1][n][0], pf[i][1][n][1]);
            }
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
#pragma unroll
                  for (int n = 0; n < kR; ++n) {
                    float d[4] = {0.f, 0.f, 0.f, 0.f};
                    mma<false>(d, b, pf[i][0][n][0], pf[i][0][n][1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                      if (pos + kKvTile * i + tok <= limit[n][e & 1]) o[j][n][e] += d[e];
                  }
                }
              }
            }
          }
        }
      }
    }
  }

  // What the lane has of row n * 8 + 2t + e, normalised: f(first channel, values) for every four neighbouring channels.
  template <typename F>
  __device__ __forceinline__ void each(int n, int e, float by, int lane, F f) const {
    const int g = lane >> 2;
    const float high = kInt4 ? by * 0.0625f : by;
#pragma unroll
    for (int j = 0; j < C::kMTiles; j += 2)
      f(kInt4 ? 64 * (j >> 2) + 8 * g + 2 * (j & 3) : 32 * (j >> 1) + 4 * g,
        make_float4(o[j][n][e] * by, o[j][n][e + 2] * high, o[j + 1][n][e] * by, o[j + 1][n][e + 2] * high));
  }
};

// ---------------------------------------------------------------- the kernel

// Parts in the workspace: of each CTA two (what Desc says), then of each warp one.
template <int kDh, int kR>
__device__ __forceinline__ Part<kDh, kR>* cta_part(const PagedAttentionArgs& p, int cta, int slot) {
  return reinterpret_cast<Part<kDh, kR>*>(static_cast<uint8_t*>(p.ws) + sizeof(Desc) * kMaxCtas) + 2 * cta + slot;
}
template <int kDh, int kR>
__device__ __forceinline__ Part<kDh, kR>* warp_part(const PagedAttentionArgs& p, int warp) {
  return cta_part<kDh, kR>(p, kMaxCtas, 0) + blockIdx.x * kWarps + warp;
}

template <int kR>
__device__ __forceinline__ __nv_bfloat16* out_row(const PagedAttentionArgs& p, const Geometry& geo, int s, int row, int h, int head_dim) {
  const int tok = row / geo.group;
  return static_cast<__nv_bfloat16*>(p.out) + (static_cast<long long>(s) * p.batch.L + tok) * p.ld_out +
         (h * geo.group + row - tok * geo.group) * head_dim;
}

template <int kDh, bool kInt4, int kR>
__global__ void __launch_bounds__(kThreads, Config<kDh, kInt4, kR>::kCtasPerSm)
    paged_attention_kernel(const PagedAttentionArgs p) {
  using C = Config<kDh, kInt4, kR>;
  using Tile = typename C::Tile;
  using Parts = Part<kDh, kR>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Shared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint8_t* const ring = smem + warp * (C::kStages * Tile::kBytes);
  const uint32_t bars = smem_u32(smem + C::kRing + C::kQ) + warp * C::kStages * 8;
  if (lane == 0)
    for (int i = 0; i < C::kStages; ++i) mbar_init(bars + 8 * i, 1);
  if (threadIdx.x == 0) sh.abort = 0;
  fence_mbar_init();
  pdl_wait();
  pdl_launch_dependents();
  const Geometry geo = geometry<kR>(p);
  Place<kR> c;
  int active;
  int left = begin(p, geo, c, active, sh);  // (synchronises the block)
  WarpEnd end{0, 0, 0, 0, false, false, false, false};
  if (left > 0) {
    Loader<kDh, kInt4, kR> loader;
    loader.at = c;
    loader.left = left;
    loader.find(p, geo);
#pragma unroll 1
    for (int i = 0; i < C::kStages; ++i) loader.issue(p, geo, lane, ring, bars);
    int stage = 0, used = 0;  // of the ring
    uint32_t phase = 0;
    Rows<kDh, kInt4, kR> rows;
#pragma unroll 1
    while (left > 0) {
      const int lo = c.tile, units = max(1, c.tiles), hi = min(units, lo + left);
      left -= hi - lo;
      const bool whole = lo == 0 && hi == units;
      const int row0 = c.rt * 8 * kR;
      const int live = c.tiles == 0 ? 0 : min(8 * kR, c.seq.n * geo.group - row0);  // rows with a token
      bool poison = false;
      if (c.tiles > 0) {
        rows.begin(p, geo, c, live, lane, reinterpret_cast<uint2*>(smem + C::kRing) + warp * (C::kQ / kWarps / 8));
        auto wait = [&]() {
          const bool there = warp_wait_bounded(bars + 8 * stage, phase, &sh.abort, p.err, kDevTimeoutProducer);
          poison |= !there || ((loader.bad >> stage) & 1) != 0;
          const uint8_t* at = ring + stage * Tile::kBytes;
          if (there) {
            ++used;
            if (++stage == C::kStages) {
              stage = 0;
              phase ^= 1;
            }
          }
          return at;
        };
#pragma unroll 1
        for (int tile = lo; tile < hi;) {
          const int pos = tile * kKvTile;
          int taken = 1;
          if (C::kPair == 2 && tile + 2 <= hi && pos + 2 * kKvTile - 1 <= rows.first_limit) {
            const uint8_t* const at0 = wait();
            const uint8_t* const at[2] = {at0, wait()};
            rows.template take<2, false>(at, pos, lane);
            taken = 2;
          } else if (C::kPair == 1 && pos + kKvTile - 1 <= rows.first_limit) {
            const uint8_t* const at[1] = {wait()};
            rows.template take<1, false>(at, pos, lane);
          } else {
            const uint8_t* const at[1] = {wait()};
            rows.template take<1, true>(at, pos, lane);
          }
          tile += taken;
          __syncwarp();
          if (sh.abort == 0)
            for (; taken > 0; --taken) loader.issue(p, geo, lane, ring, bars);
        }
      }

      // ---- an item as a whole goes out, a part of one waits: the last segment's in the ring, an earlier one's in memory
      const bool last = left == 0;
      if (last) {
        for (; used < loader.issued; ++used) {  // copies that a wait has given up are not left behind
          int alone = 0;
          mbar_wait_bounded(bars + 8 * stage, phase, &alone, p.err, kDevTimeoutDrain);
          if (++stage == C::kStages) {
            stage = 0;
            phase ^= 1;
          }
        }
        __syncwarp();
      }
      float* part_o = last ? reinterpret_cast<float*>(ring) : &warp_part<kDh, kR>(p, warp)->o[0][0];
      float* part_mass = last ? sh.mass[warp] : warp_part<kDh, kR>(p, warp)->mass;
      const int slots = min(8 * kR, geo.rows - row0);
#pragma unroll
      for (int n = 0; n < kR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = n * 8 + 2 * t + e;
          float sum = 0.f, by = 0.f;
          if (c.tiles > 0) {
            sum = rows.l[n][e];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            by = poison ? __int_as_float(0x7fffffff) : sum == 0.f ? 0.f : 1.f / sum;
          }
          if (whole) {
            if (row < slots) {
              __nv_bfloat16* dst = out_row<kR>(p, geo, c.s, row0 + row, c.h, kDh);
              if (row < live) {
                rows.each(n, e, by, lane, [&](int d, const float4& v) {
                  *reinterpret_cast<uint2*>(dst + d) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
                });
              } else {
                // an empty slot, or positions that cannot be (NaN)
                const uint32_t fill = !c.seq.ok && row0 + row < c.seq.n * geo.group ? 0x7fff7fffu : 0u;
                for (int d = 4 * g; d < kDh; d += 32) *reinterpret_cast<uint2*>(dst + d) = make_uint2(fill, fill);
              }
            }
          } else if (row < live) {
            rows.each(n, e, by, lane, [&](int d, const float4& v) { *reinterpret_cast<float4*>(part_o + row * kDh + d) = v; });
            if (g == 0)
              part_mass[row] = poison ? __int_as_float(0x7fffffff) : sum == 0.f ? kFar : rows.m[n][e] + log2f(sum);
          }
        }
      if (!whole) {
        if (lo > 0) {
          end.first = true;
          end.first_rt = c.rt;
          end.first_last = last;
          end.first_ends = hi == units;
        } else {
          end.tail = true;
        }
      }
      end.s = c.s;
      end.rt = c.rt;
      end.h = c.h;
      c.tile = hi;
      if (left > 0) c.next_item(p, geo);
    }
  }
  if (lane == 0) sh.end[warp] = end;
  __syncthreads();

  // ---- chains of parts of one item: from what an earlier CTA began, or from a warp's tail, over the following warps' first
  // parts to the one that ends it. A warp a row of a chain.
  int chain = 0, tail_warp = -1, ends = 0;
  for (int start = -1; start < active; ++start) {
    const bool from_before = start < 0;
    if (from_before ? !sh.end[0].first : !sh.end[start].tail) continue;
    const WarpEnd& item = sh.end[from_before ? 0 : start];
    int stop = from_before ? 0 : start + 1;  // one past its last warp
    bool done = false;
    while (stop < active && sh.end[stop].first && !done) done = sh.end[stop++].first_ends;
    if (from_before) ends = done;
    if (!from_before && !done) tail_warp = start;
    const int rt = from_before ? item.first_rt : item.rt;
    const int shown = min(8 * kR, geo.rows - rt * 8 * kR);
    Parts* to = cta_part<kDh, kR>(p, blockIdx.x, from_before ? 0 : 1);
    const int base = from_before ? 0 : start;
    constexpr int kE = kDh / 32;
    // (rows past the last token hold nothing; what is made of them is not read)
    for (int row = (warp + kWarps - chain % kWarps) % kWarps; row < shown; row += kWarps) {
      float mass[kWarps], top = kFar, sum = 0.f, out[kE];
      const float* part[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        mass[w] = kFar;
        part[w] = nullptr;
        if (w >= base && w < stop) {
          const bool ringed = w == start || sh.end[w].first_last;
          const Parts* kept = warp_part<kDh, kR>(p, w);
          part[w] = ringed ? reinterpret_cast<const float*>(smem + w * (C::kStages * Tile::kBytes)) + row * kDh : kept->o[row];
          mass[w] = ringed ? sh.mass[w][row] : kept->mass[row];
        }
        top = fmaxf(top, mass[w]);
      }
#pragma unroll
      for (int i = 0; i < kE; ++i) out[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        mass[w] = mass[w] == kFar ? 0.f : ex2(mass[w] - top);
        sum += mass[w];
      }
      const float norm = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int w = 0; w < kWarps; ++w)
        if (mass[w] != 0.f) {
#pragma unroll
          for (int i = 0; i < kE; ++i) out[i] = fmaf(part[w][lane * kE + i], mass[w] * norm, out[i]);
        }
      if (!from_before && done) {
        const KvSeq seq = seq_of(p, item.s, nullptr);
        const int q_row = rt * 8 * kR + row;
        __nv_bfloat16* dst = out_row<kR>(p, geo, item.s, q_row, item.h, kDh) + lane * kE;
#pragma unroll
        for (int i = 0; i < kE; i += 2)
          *reinterpret_cast<uint32_t*>(dst + i) = q_row < seq.n * geo.group ? pack_bf16x2(out[i], out[i + 1]) : 0u;
      } else {
#pragma unroll
        for (int i = 0; i < kE; ++i) to->o[row][lane * kE + i] = out[i];
        if (lane == 0) to->mass[row] = sum == 0.f ? kFar : top + log2f(sum);
      }
    }
    chain += shown;
  }
  if (threadIdx.x == 0) {
    Desc d{0, 0, 0, -1, ends, {0, 0, 0}};
    if (tail_warp >= 0) {
      d.s = sh.end[tail_warp].s;
      d.rt = sh.end[tail_warp].rt;
      d.h = sh.end[tail_warp].h;
      d.slot = 1;
    }
    static_cast<Desc*>(p.ws)[blockIdx.x] = d;
  }
}

// Items that several CTAs have parts of: the CTA that holds an item's first part adds up all of them, a row in y.
template <int kDh, int kR>
__global__ void __launch_bounds__(kThreads) paged_attention_join_kernel(const PagedAttentionArgs p, int ctas) {
  __shared__ float sh_o[kWarps][kDh], sh_top[kWarps], sh_sum[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  const Desc* desc = static_cast<const Desc*>(p.ws);
  const int b = blockIdx.x, row = blockIdx.y;
  const Desc mine = desc[b];
  if (mine.slot < 0) return;
  const Geometry geo = geometry<kR>(p);
  const int q_row = mine.rt * 8 * kR + row;
  if (q_row >= geo.rows) return;
  int end = ctas;  // parts: this CTA's, then slot 0 of those up to the first that ends the item
  for (int at = b + 1; at < ctas; at += 32) {
    const unsigned found = __ballot_sync(0xffffffffu, at + lane < ctas && desc[at + lane].ends != 0);
    if (found != 0) {
      end = at + __ffs(found);
      break;
    }
  }
  constexpr int kE = kDh / 32;
  float top = kFar, sum = 0.f, out[kE];
#pragma unroll
  for (int i = 0; i < kE; ++i) out[i] = 0.f;
  for (int at = b + warp; at < end; at += kWarps) {
    const Part<kDh, kR>& part = *cta_part<kDh, kR>(p, at, at == b ? mine.slot : 0);
    const float mass = part.mass[row];
    const float now = fmaxf(top, mass), by = ex2(top - now), weight = mass == kFar ? 0.f : ex2(mass - now);
    top = now;
    sum = sum * by + weight;
#pragma unroll
    for (int i = 0; i < kE; ++i) out[i] = out[i] * by + (weight == 0.f ? 0.f : weight * part.o[row][lane * kE + i]);
  }
#pragma unroll
  for (int i = 0; i < kE; ++i) sh_o[warp][lane * kE + i] = out[i];
  if (lane == 0) {
    sh_top[warp] = top;
    sh_sum[warp] = sum;
  }
  __syncthreads();
  if (threadIdx.x < kDh) {
    float all = kFar, total = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all = fmaxf(all, sh_top[w]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float by = ex2(sh_top[w] - all);
      total += sh_sum[w] * by;
      acc += sh_o[w][threadIdx.x] * by;
    }
    const KvSeq seq = seq_of(p, mine.s, nullptr);
    __nv_bfloat16* dst = out_row<kR>(p, geo, mine.s, q_row, mine.h, kDh);
    dst[threadIdx.x] = __float2bfloat16_rn(q_row >= seq.n * geo.group ? 0.f : acc / total);
  }
}

template <int kDh, bool kInt4, int kR>
int launch(const PagedAttentionArgs& a, cudaStream_t st) {
  using C = Config<kDh, kInt4, kR>;
  static_assert(C::kSmem * C::kCtasPerSm <= 227 * 1024, "shared memory of an SM");
  if (cudaFuncSetAttribute(paged_attention_kernel<kDh, kInt4, kR>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) !=
      cudaSuccess)
    return -3;
  const int ctas = std::min(kMaxCtas, std::max(1, sm_count()) * C::kCtasPerSm);
  if (launch_pdl(paged_attention_kernel<kDh, kInt4, kR>, dim3(ctas), dim3(kThreads), C::kSmem, st, a) != cudaSuccess) return -3;
  const int64_t rows = a.n_heads / a.cache.kv_heads * a.batch.L;
  const dim3 grid(ctas, static_cast<unsigned>(std::min<int64_t>(rows, 8 * kR)));
  return launch_pdl(paged_attention_join_kernel<kDh, kR>, grid, dim3(kThreads), 0, st, a, ctas) == cudaSuccess ? 0 : -3;
}

// Passes over the rows of a kv head, 8 to 32 rows each: as few as can be, then the narrowest that do.
int row_tiles_of(int64_t rows) {
  const int64_t eights = (rows + 7) / 8, passes = (eights + kMaxRowTiles - 1) / kMaxRowTiles;
  return static_cast<int>((eights + passes - 1) / passes);
}

template <int kDh, bool kInt4>
int launch_rows(const PagedAttentionArgs& a, cudaStream_t st) {
  switch (row_tiles_of(a.n_heads / a.cache.kv_heads * a.batch.L)) {
    case 1: return launch<kDh, kInt4, 1>(a, st);
    case 2: return launch<kDh, kInt4, 2>(a, st);
    case 3: return launch<kDh, kInt4, 3>(a, st);
    default: return launch<kDh, kInt4, 4>(a, st);
  }
}

}  // namespace

size_t paged_attention_workspace_bytes(int64_t S, int64_t L, int64_t n_heads, int64_t kv_heads, int64_t head_dim) {
  const int64_t rows = 8 * row_tiles_of(std::max<int64_t>(1, n_heads / kv_heads * L));
  return sizeof(Desc) * kMaxCtas + static_cast<size_t>((2 + kWarps) * kMaxCtas * rows * (head_dim + 1) * 4);
}

int launch_paged_attention(const PagedAttentionArgs& a, cudaStream_t st) {
  if (a.cache.head_dim == 128) return a.cache.int4 ? launch_rows<128, true>(a, st) : launch_rows<128, false>(a, st);
  return a.cache.int4 ? launch_rows<64, true>(a, st) : launch_rows<64, false>(a, st);
}

}  // namespace hydra
