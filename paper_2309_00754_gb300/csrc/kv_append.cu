// New tokens' keys and values into a paged cache, rotated on the way, and cached rows read back dense.
//
//   r_i = x_i cos a - x_{i + D/2} sin a,  r_{i + D/2} = x_i sin a + x_{i + D/2} cos a   (queries and keys)
//
// with every product and sum rounded to fp32 as hydra_rope rounds them. A bf16 cache takes bf16(r). A cache in 4 bits
// takes, for each group of 64 channels, lo = min(0, r), hi = max(0, r), scale = bf16((hi / 2 - lo / 2) 2/15), the
// zero point rint(-lo / scale) and the codes rint(r / scale) + zero, both within 0..15.
//
// Bound by bytes for prompts, by latency for a step's few tokens. 8 prompts of up to 512 tokens with 32 query heads and 32 for
// keys and values of 128 channels: 25.0 us to append (4 bits), 14.5 us to read back; one token of 64 sequences 3.7 us, of one
// 2.8 us.
#include "kv_cache.cuh"

namespace hydra {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
// Heads of a warp where there are many: it reads the rotation once for them and has the next head on its way while it works
// (the 8 prompts above: 25.0 us with four heads, 28.6 with two, 39.1 with one; 2 such prompts, 12,000 blocks times heads, 10.2
// with four and 13.1 with one; 4 of 128 tokens in bf16, 6500, are the faster singly, 7.6 against 8.1).
constexpr int kPer = 4;
constexpr int64_t kManyUnits = 10000;  // blocks of eight tokens times heads
constexpr int kBlock = 8;  // tokens of a warp, from a multiple of 8 on: half of a tile

__device__ __forceinline__ void unpack8(const uint4& v, float* f) {
  const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = unpack_bf16x2(r[i]);
    f[2 * i] = x.x;
    f[2 * i + 1] = x.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

__device__ __forceinline__ float max_or_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Of a group of channels: the least and the largest value (0 among them); `hi` is NaN where one of them is.
struct Range {
  float lo = 0.f, hi = 0.f;
  __device__ __forceinline__ void take(float x) {
    lo = fminf(lo, x);
    hi = max_or_nan(hi, x);
  }
};
// over the lanes that differ in the bit `off`: of one range, and of two, of which the lane goes on with the one of its bit
__device__ __forceinline__ Range met(const Range& mine, const Range& sent, int off) {
  Range r;
  r.lo = fminf(mine.lo, __shfl_xor_sync(0xffffffffu, sent.lo, off));
  r.hi = max_or_nan(mine.hi, __shfl_xor_sync(0xffffffffu, sent.hi, off));
  return r;
}
__device__ __forceinline__ Range met(const Range& r, int off) { return met(r, r, off); }
__device__ __forceinline__ Range halved(const Range& zero, const Range& one, int off) {
  const bool bit = (threadIdx.x & off) != 0;
  return met(bit ? one : zero, bit ? zero : one, off);
}

struct Quant {
  float scale, zero;  // scale 0 or NaN: all codes are 0
  float inv;          // 1 / scale, or NaN where codes are not to come from it
  __device__ __forceinline__ explicit Quant(const Range& r) {
    // (halves: the difference of two large values passes fp32)
    scale = __bfloat162float(__float2bfloat16_rn(__fmul_rn(__fsub_rn(r.hi * 0.5f, r.lo * 0.5f), 2.0f / 15.0f)));
    scale = fmaf(scale, 0.f, scale);  // infinite only with an infinity among the channels: NaN then, too
    zero = scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(-r.lo, scale)), 0.f), 15.f) : 0.f;
    inv = scale > 1e-30f && scale < 1e30f ? __frcp_rn(scale) : __int_as_float(0x7fffffff);
  }
  // that of another lane
  __device__ __forceinline__ Quant(const Quant& q, int lane)
      : scale(__shfl_sync(0xffffffffu, q.scale, lane)), zero(__shfl_sync(0xffffffffu, q.zero, lane)), inv(__shfl_sync(0xffffffffu, q.inv, lane)) {}
  __device__ __forceinline__ uint32_t code(float x) const {
    if (!(scale > 0.f)) return 0;
    return static_cast<uint32_t>(fminf(fmaxf(rintf(__fdiv_rn(x, scale)) + zero, 0.f), 15.f));
  }
  // Codes of 8 channels, the first in the lowest bits. By the reciprocal, x / scale is off by less than 2^-19 (it is at
  // most 16); where that could turn the rounding, by the division.
  __device__ __forceinline__ uint32_t codes(const float* x) const {
    constexpr float kMagic = 12582912.f;  // 1.5 2^23: what is added to it is rounded to an integer in the low bits
    constexpr uint32_t kMagicBits = 0x4b400000u;
    const bool usual = inv == inv;
    const float magic = kMagic + zero;
    uint32_t w = 0;
    float off = 0.f;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
      const float t = fmaf(x[i], inv, magic);
      off = fmaxf(off, fabsf(fmaf(x[i], inv, magic - t)));
      w = w * 16 + __float_as_uint(fminf(fmaxf(t, kMagic), kMagic + 15.f));
    }
    w -= kMagicBits * 0x11111111u;
    if (!usual || off > 0.49999f) {
      uint32_t close = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float t = fmaf(x[i], inv, magic);
        if (!usual || fabsf(fmaf(x[i], inv, magic - t)) > 0.49999f) close |= 1u << i;
      }
#pragma unroll 1
      for (; close != 0; close &= close - 1) {  // (one copy of the division: a short call waits for its instructions)
        const int at = __ffs(close) - 1;
        float one = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) one = at == i ? x[i] : one;
        w = (w & ~(15u << (4 * at))) | code(one) << (4 * at);
      }
    }
    return w;
  }
  __device__ __forceinline__ uint32_t scale_bits() const { return __bfloat16_as_ushort(__float2bfloat16_rn(scale)); }
  __device__ __forceinline__ uint32_t zero_bits() const { return 17u * static_cast<uint32_t>(zero); }
};

// The tokens of a warp: `slot` of the first (maybe below 0), and what the call says of their sequence.
struct Block {
  int s, first;
  KvSeq seq;
  __device__ __forceinline__ Block(const KvBatch& b, int blocks, long long positions, int* err) {
    s = static_cast<int>(blockIdx.x) / blocks;
    seq = kv_seq(b, s, positions, err);
    first = (static_cast<int>(blockIdx.x) - s * blocks) * kBlock - (seq.cached & (kBlock - 1));
  }
};

// The warps of a block of tokens: up to `per` heads of a kind for each; where there is a single token, a head for each of the
// lanes' tokens (64 sequences of 32 + 64 heads: 3.7 us; with 7 of 8 lanes idle 7.6).
struct Units {
  int per, v_per, q, k, v;
  __host__ __device__ Units(int heads, int kv, bool single, int per_)
      : per(single ? kBlock : per_), v_per(single ? kBlock / 2 : per_), q((heads + per - 1) / per), k((kv + per - 1) / per),
        v((kv + v_per - 1) / v_per) {}
};

// A warp has 8 tokens of up to `per` heads of a kind. Queries and keys: lane (token lane / 4, part t = lane % 4) has channels
// D/8 t .. and D/2 + D/8 t .., which rotate together. Values: lane (g = lane / 4, t = lane % 4) has tokens 2 t and 2 t + 1,
// channels 8 g .. of each 64. So a lane's codes are 16 bytes of the tile (D = 64: 8) where it has both tokens, and a warp's
// lie side by side.
template <int kDh, bool kInt4>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const KvAppendArgs p, int blocks, int per) {
  using Tile = KvTile<kDh, kInt4>;
  constexpr int kGroups = kDh / kKvGroup, kRun = kDh / 8, kRaw = 2 * kGroups;
  const int lane = threadIdx.x & 31, quad = lane >> 2, t = lane & 3;
  const int heads = p.q_out != nullptr ? static_cast<int>(p.n_heads) : 0, kv = p.cache.kv_heads;
  const int L = static_cast<int>(p.batch.L);
  const bool single = L == 1;
  const Units units(heads, kv, single, per);
  const int unit = blockIdx.y * kWarps + (threadIdx.x >> 5);
  pdl_wait();
  pdl_launch_dependents();
  if (unit >= units.v + units.k + units.q) return;
  const bool value = unit < units.v, query = unit >= units.v + units.k;  // (what takes longest first)
  const int head0 = value ? unit * units.v_per : (query ? unit - units.v - units.k : unit - units.v) * units.per;
  const int end = min(head0 + (value ? units.v_per : units.per), query ? heads : kv), steps = single ? 1 : end - head0;
  const long long positions = p.batch.max_pages << p.cache.page_bits;
  const Block at(p.batch, blocks, p.rope != nullptr ? min(positions, static_cast<long long>(p.rope_len)) : positions, p.err);
  const int n = at.seq.ok ? at.seq.n : 0;
  const long long row0 = static_cast<long long>(at.s) * L;

  if (!value) {
    const int slot = single ? 0 : at.first + quad, pos = at.seq.cached + slot;
    int head = single ? head0 + quad : head0;
    const long long row = row0 + slot;
    const bool there = slot >= 0 && slot < n && head < end;
    __nv_bfloat16* q_out = static_cast<__nv_bfloat16*>(p.q_out) + row * p.ld_q_out + kRun * t;
    if (query && !there && slot >= 0 && slot < L) {
      const uint32_t fill = slot < at.seq.n ? 0x7fff7fffu : 0u;  // NaN, or an empty slot
      for (int h = head; h < min(head + steps, end); ++h)
#pragma unroll
        for (int i = 0; i < kRaw; ++i)
          *reinterpret_cast<uint4*>(q_out + h * kDh + (i / kGroups) * (kDh / 2) + (i % kGroups) * 8) = make_uint4(fill, fill, fill, fill);
    }
    if (!__any_sync(0xffffffffu, there)) return;
    const __nv_bfloat16* x = query ? static_cast<const __nv_bfloat16*>(p.q) + row * p.ld_q : static_cast<const __nv_bfloat16*>(p.k) + row * p.ld_kv;
    x += kRun * t;
    uint4 raw[kRaw] = {};
    auto load = [&](int h) {
      if (there)
#pragma unroll
        for (int i = 0; i < kRaw; ++i)
          raw[i] = *reinterpret_cast<const uint4*>(x + h * kDh + (i / kGroups) * (kDh / 2) + (i % kGroups) * 8);
    };
    load(head);
    float4 rope[kRun / 2] = {};
    if (p.rope != nullptr && there) {
      const float4* r = reinterpret_cast<const float4*>(p.rope + (static_cast<long long>(pos) * (kDh / 2) + kRun * t) * 2);
#pragma unroll
      for (int i = 0; i < kRun / 2; ++i) rope[i] = r[i];
    }
    const int page = there && !query ? kv_page(p.batch, p.cache, at.s, pos, p.err) : -1;
#pragma unroll 1
    for (int step = 1; step <= steps; ++step, ++head) {
      float a[kRun], b[kRun];
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        unpack8(raw[i], a + 8 * i);
        unpack8(raw[kGroups + i], b + 8 * i);
      }
      if (step < steps) load(head + 1);
      if (p.rope != nullptr) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          const float c = i & 1 ? rope[i / 2].z : rope[i / 2].x, sn = i & 1 ? rope[i / 2].w : rope[i / 2].y;
          const float x1 = a[i], x2 = b[i];
          a[i] = __fsub_rn(__fmul_rn(x1, c), __fmul_rn(x2, sn));
          b[i] = __fadd_rn(__fmul_rn(x1, sn), __fmul_rn(x2, c));
        }
      }
      if (query) {
        if (there)
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            *reinterpret_cast<uint4*>(q_out + head * kDh + 8 * i) = pack8(a + 8 * i);
            *reinterpret_cast<uint4*>(q_out + head * kDh + kDh / 2 + 8 * i) = pack8(b + 8 * i);
          }
        continue;
      }
      const int token = pos & (kKvTile - 1);
      uint8_t* tile = page >= 0 ? kv_tile<Tile>(p.cache, page, head, pos) : nullptr;
      if constexpr (!kInt4) {
        if (tile != nullptr)
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            *reinterpret_cast<uint4*>(tile + Tile::key(token, kRun * t + 8 * i)) = pack8(a + 8 * i);
            *reinterpret_cast<uint4*>(tile + Tile::key(token, kDh / 2 + kRun * t + 8 * i)) = pack8(b + 8 * i);
          }
      } else {
        Range range[kGroups];
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          range[0].take(a[i]);
          range[kGroups - 1].take(b[i]);
        }
        // (D = 128: a lane works out one of the two groups; the other comes from its neighbour)
        const Quant own(met(kGroups == 2 ? halved(range[0], range[kGroups - 1], 1) : met(range[0], 1), 2));
        const Quant qa(kGroups == 2 ? Quant(own, lane & ~1) : own), qb(kGroups == 2 ? Quant(own, lane | 1) : own);
        if (tile != nullptr && t < kGroups) {
          *reinterpret_cast<uint16_t*>(tile + Tile::scale(token, false, t)) = static_cast<uint16_t>(own.scale_bits());
          *reinterpret_cast<uint16_t*>(tile + Tile::zero(token, false, t)) = static_cast<uint16_t>(own.zero_bits());
        }
        if (tile != nullptr) {
          if constexpr (kGroups == 2) {
            *reinterpret_cast<uint4*>(tile + Tile::key(token, kRun * t)) = make_uint4(qa.codes(a), qa.codes(a + 8), qb.codes(b), qb.codes(b + 8));
          } else {
            *reinterpret_cast<uint32_t*>(tile + Tile::key(token, kRun * t)) = qa.codes(a);
            *reinterpret_cast<uint32_t*>(tile + Tile::key(token, kDh / 2 + kRun * t)) = qa.codes(b);
          }
        }
      }
    }
    return;
  }

  const int slot = single ? -(at.seq.cached & 1) : at.first + 2 * t, pos = at.seq.cached + slot;  // of the first of two tokens (even)
  int head = single ? head0 + t : head0;
  const bool there[2] = {slot >= 0 && slot < n && head < end, slot + 1 >= 0 && slot + 1 < n && head < end};
  const bool any[2] = {__any_sync(0xffffffffu, there[0]) != 0, __any_sync(0xffffffffu, there[1]) != 0};  // of the warp's
  if (!any[0] && !any[1]) return;
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(p.v) + (row0 + slot) * p.ld_kv + 8 * quad;
  uint4 raw[2][kGroups] = {};
  auto load = [&](int h) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
      if (there[b])
#pragma unroll
        for (int g = 0; g < kGroups; ++g) raw[b][g] = *reinterpret_cast<const uint4*>(x + b * p.ld_kv + h * kDh + g * kKvGroup);
  };
  load(head);
  const int page = there[0] || there[1] ? kv_page(p.batch, p.cache, at.s, pos + (there[0] ? 0 : 1), p.err) : -1;
  const int token = pos & (kKvTile - 1);
#pragma unroll 1
  for (int step = 1; step <= steps; ++step, ++head) {
    uint8_t* tile = page >= 0 ? kv_tile<Tile>(p.cache, page, head, pos) : nullptr;
    if constexpr (!kInt4) {
      if (tile != nullptr) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          const uint32_t r[2][4] = {{raw[0][g].x, raw[0][g].y, raw[0][g].z, raw[0][g].w}, {raw[1][g].x, raw[1][g].y, raw[1][g].z, raw[1][g].w}};
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // 4 channels
            uint8_t* to = tile + Tile::value(token, g * kKvGroup + 8 * quad + 4 * h);
            if (there[0] && there[1]) {
              *reinterpret_cast<uint4*>(to) = make_uint4(
                  __byte_perm(r[0][2 * h], r[1][2 * h], 0x5410), __byte_perm(r[0][2 * h], r[1][2 * h], 0x7632),
                  __byte_perm(r[0][2 * h + 1], r[1][2 * h + 1], 0x5410), __byte_perm(r[0][2 * h + 1], r[1][2 * h + 1], 0x7632));
            } else {
              const int b = there[0] ? 0 : 1;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t two = b == 0 ? r[0][2 * h + i / 2] : r[1][2 * h + i / 2];
                reinterpret_cast<uint16_t*>(to)[2 * i + b] = static_cast<uint16_t>(i & 1 ? two >> 16 : two);
              }
            }
          }
        }
      }
      if (step < steps) load(head + 1);
    } else {
      float v[2][kGroups][8];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int g = 0; g < kGroups; ++g) unpack8(raw[b][g], v[b][g]);
      if (step < steps) load(head + 1);
      Range range[2][kGroups];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int i = 0; i < 8; ++i) range[b][g].take(v[b][g][i]);
      // a lane works out the token of bit 2 of its number and (D = 128) the group of bit 3; the others come from their lanes
      Range mine = halved(range[0][0], range[1][0], 4);
      if constexpr (kGroups == 2)
        mine = halved(mine, halved(range[0][1], range[1][1], 4), 8);
      else
        mine = met(mine, 8);
      const Quant own(met(mine, 16));
      uint32_t w[2][kGroups] = {};
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (!(b == 0 ? any[0] : any[1])) continue;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) w[b][g] = Quant(own, t + 4 * b + 8 * g).codes(v[b][g]);
      }
      if (tile != nullptr) {
        uint8_t* to = tile + Tile::value(token, 8 * quad);
        if (there[0] && there[1]) {
          uint32_t piece[2 * kGroups];
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            piece[2 * g] = __byte_perm(w[0][g], w[1][g], 0x5410);
            piece[2 * g + 1] = __byte_perm(w[0][g], w[1][g], 0x7632);
          }
          if constexpr (kGroups == 2)
            *reinterpret_cast<uint4*>(to) = make_uint4(piece[0], piece[1], piece[2], piece[3]);
          else
            *reinterpret_cast<uint2*>(to) = make_uint2(piece[0], piece[1]);
        } else {
          const int b = there[0] ? 0 : 1;
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            const uint32_t one = b == 0 ? w[0][g] : w[1][g];
            reinterpret_cast<uint16_t*>(to)[4 * g + b] = static_cast<uint16_t>(one);
            reinterpret_cast<uint16_t*>(to)[4 * g + 2 + b] = static_cast<uint16_t>(one >> 16);
          }
        }
        if (quad < 2 * kGroups && there[quad & 1]) {  // a lane a token and group
          *reinterpret_cast<uint16_t*>(tile + Tile::scale(token + (quad & 1), true, quad >> 1)) = static_cast<uint16_t>(own.scale_bits());
          *reinterpret_cast<uint16_t*>(tile + Tile::zero(token + (quad & 1), true, quad >> 1)) = static_cast<uint16_t>(own.zero_bits());
        }
      }
    }
  }
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* x) { *reinterpret_cast<uint4*>(p) = pack8(x); }
__device__ __forceinline__ void store8(float* p, const float* x) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// What 8 codes stand for, from a group's scale and zero point (17 times it).
__device__ __forceinline__ void values8(uint32_t w, uint32_t scale_bits, uint32_t zero_bits, float* x) {
  const float scale = __uint_as_float(scale_bits << 16), minus = -8388608.f - static_cast<float>(zero_bits & 15);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = scale * (__uint_as_float(0x4b000000u | ((w >> (4 * i)) & 15)) + minus);  // 2^23 + code
}

// A warp has 8 tokens of a head's keys or values, four lanes a key, eight two values.
template <int kDh, bool kInt4, typename Out>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const KvReadArgs p, int blocks) {
  using Tile = KvTile<kDh, kInt4>;
  constexpr int kGroups = kDh / kKvGroup;
  const int lane = threadIdx.x & 31, quad = lane >> 2, t = lane & 3;
  const int kv = p.cache.kv_heads;
  const int unit = blockIdx.y * kWarps + (threadIdx.x >> 5);
  pdl_wait();
  pdl_launch_dependents();
  if (unit >= 2 * kv) return;
  const bool value = unit >= kv;
  const int head = value ? unit - kv : unit;
  Out* out = static_cast<Out*>(value ? p.v : p.k);
  if (out == nullptr) return;
  const Block at(p.batch, blocks, p.batch.max_pages << p.cache.page_bits, p.err);
  const int L = static_cast<int>(p.batch.L);
  const int slot = at.first + (value ? 2 * t : quad), pos = at.seq.cached + slot, tokens = value ? 2 : 1;
  bool any = false, in[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    in[b] = b < tokens && slot + b >= 0 && slot + b < L;
    any |= in[b] && slot + b < at.seq.n;
  }
  const int valid = slot < 0 ? pos + 1 : pos;  // a position that is the sequence's
  const int page = any && at.seq.ok ? kv_page(p.batch, p.cache, at.s, valid, p.err) : -1;
  const uint8_t* tile = page >= 0 ? kv_tile<Tile>(p.cache, page, head, valid) : nullptr;
  out += (static_cast<long long>(at.s) * L + slot) * p.ld + head * kDh;
  const int token = pos & (kKvTile - 1);
  // a token's 8 channels from d on
  auto put = [&](int b, int d, float* x) {
    if (!in[b]) return;
    if (slot + b >= at.seq.n || tile == nullptr) {
      const float fill = slot + b >= at.seq.n ? 0.f : __int_as_float(0x7fffffff);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fill;
    }
    store8(out + b * p.ld + d, x);
  };
  if (!value) {
    uint32_t scale = 0, zero = 0;
    if (kInt4 && tile != nullptr) {
      if constexpr (kGroups == 2) {
        scale = *reinterpret_cast<const uint32_t*>(tile + Tile::scale(token, false, 0));
        zero = *reinterpret_cast<const uint32_t*>(tile + Tile::zero(token, false, 0));
      } else {
        scale = *reinterpret_cast<const uint16_t*>(tile + Tile::scale(token, false, 0));
        zero = *reinterpret_cast<const uint16_t*>(tile + Tile::zero(token, false, 0));
      }
    }
#pragma unroll
    for (int i = 0; i < kDh / 32; ++i) {  // 8 channels of each 32, so that four lanes write a row's bytes in order
      const int d = 32 * i + 8 * t;
      float x[8] = {};
      if (tile != nullptr) {
        if constexpr (kInt4)
          values8(*reinterpret_cast<const uint32_t*>(tile + Tile::key(token, d)), (scale >> (16 * (i / 2))) & 0xffff,
                  zero >> (16 * (i / 2)), x);
        else
          unpack8(*reinterpret_cast<const uint4*>(tile + Tile::key(token, d)), x);
      }
      put(0, d, x);
    }
  } else {
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int d = g * kKvGroup + 8 * quad;
      float x[2][8] = {};
      if (tile != nullptr) {
        if constexpr (kInt4) {
          const uint2 v = *reinterpret_cast<const uint2*>(tile + Tile::value(token, d));
          const uint32_t zero = *reinterpret_cast<const uint32_t*>(tile + Tile::zero(token, true, g));
#pragma unroll
          for (int b = 0; b < 2; ++b)
            values8(__byte_perm(v.x, v.y, b == 0 ? 0x5410 : 0x7632),
                    *reinterpret_cast<const uint16_t*>(tile + Tile::scale(token + b, true, g)), zero >> (16 * b), x[b]);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // 4 channels
            const uint4 v = *reinterpret_cast<const uint4*>(tile + Tile::value(token, d + 4 * h));
            const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 two = unpack_bf16x2(r[i]);
              x[0][4 * h + i] = two.x;
              x[1][4 * h + i] = two.y;
            }
          }
        }
      }
      put(0, d, x[0]);
      put(1, d, x[1]);
    }
  }
}

// Blocks of 8 positions that L tokens can touch.
int64_t blocks_of(int64_t L) { return (L + 2 * kBlock - 2) / kBlock; }

template <int kDh, bool kInt4>
cudaError_t append(const KvAppendArgs& a, cudaStream_t st) {
  const int64_t blocks = blocks_of(a.batch.L);
  const int heads = a.q_out != nullptr ? static_cast<int>(a.n_heads) : 0, kv = a.cache.kv_heads;
  const int per = a.batch.S * blocks * (heads + 2 * kv) >= kManyUnits ? kPer : 1;
  const Units u(heads, kv, a.batch.L == 1, per);
  return launch_pdl(kv_append_kernel<kDh, kInt4>, dim3(static_cast<unsigned>(a.batch.S * blocks), static_cast<unsigned>((u.q + u.k + u.v + kWarps - 1) / kWarps)),
                    dim3(kThreads), 0, st, a, static_cast<int>(blocks), per);
}
template <int kDh, bool kInt4>
cudaError_t read(const KvReadArgs& a, cudaStream_t st) {
  const int64_t blocks = blocks_of(a.batch.L);
  const dim3 grid(static_cast<unsigned>(a.batch.S * blocks), static_cast<unsigned>((2 * a.cache.kv_heads + kWarps - 1) / kWarps));
  return a.f32 ? launch_pdl(kv_read_kernel<kDh, kInt4, float>, grid, dim3(kThreads), 0, st, a, static_cast<int>(blocks))
               : launch_pdl(kv_read_kernel<kDh, kInt4, __nv_bfloat16>, grid, dim3(kThreads), 0, st, a, static_cast<int>(blocks));
}

}  // namespace

int launch_kv_append(const KvAppendArgs& a, cudaStream_t st) {
  const auto f = a.cache.head_dim == 128 ? (a.cache.int4 ? append<128, true> : append<128, false>)
                                         : (a.cache.int4 ? append<64, true> : append<64, false>);
  return f(a, st) == cudaSuccess ? 0 : -3;
}

int launch_kv_read(const KvReadArgs& a, cudaStream_t st) {
  const auto f = a.cache.head_dim == 128 ? (a.cache.int4 ? read<128, true> : read<128, false>)
                                         : (a.cache.int4 ? read<64, true> : read<64, false>);
  return f(a, st) == cudaSuccess ? 0 : -3;
}

}  // namespace hydra
