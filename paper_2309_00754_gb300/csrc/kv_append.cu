// New tokens' keys and values into a paged cache, rotated on the way, and cached rows read back dense.
//
//   r_i = x_i cos a - x_{i + D/2} sin a,  r_{i + D/2} = x_i sin a + x_{i + D/2} cos a   (queries and keys)
//
// with every product and sum rounded to fp32 as hydra_rope rounds them. A bf16 cache takes bf16(r). A cache in 4 bits
// takes, for each group of 64 channels, lo = min(0, r), hi = max(0, r), scale = bf16((hi / 2 - lo / 2) 2/15), the
// zero point rint(-lo / scale) and the codes rint(r / scale) + zero, both within 0..15.
#include "kv_cache.cuh"

namespace hydra {
namespace {

constexpr int kThreads = 256;

// The 16 channels of a lane: 8 from 8 j on, and 8 from D/2 + 8 j on.
template <int kDh>
struct Half {
  static constexpr int kLanes = kDh / 16;  // of a head
};

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = unpack_bf16x2(r[i]);
    f[2 * i] = x.x;
    f[2 * i + 1] = x.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// Of a group of channels, from the least and the largest value (0 among them).
struct Quant {
  float scale, zero;
  __device__ __forceinline__ Quant(float lo, float hi) {
    // (halves: the difference of two large values passes fp32)
    scale = __bfloat162float(__float2bfloat16_rn(__fmul_rn(__fsub_rn(hi * 0.5f, lo * 0.5f), 2.0f / 15.0f)));
    zero = scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(-lo, scale)), 0.f), 15.f) : 0.f;
  }
  __device__ __forceinline__ uint32_t code(float x) const {
    if (!(scale > 0.f)) return 0;
    return static_cast<uint32_t>(fminf(fmaxf(rintf(__fdiv_rn(x, scale)) + zero, 0.f), 15.f));
  }
};

// A token's head to its place in the tile. `a`, `b`: the lane's channels from 8 j and D/2 + 8 j on.
template <int kDh, bool kInt4>
__device__ __forceinline__ void store_head(uint8_t* tile, int token, bool value, int j, const float (&a)[8],
                                           const float (&b)[8], bool there) {
  using Tile = KvTile<kDh, kInt4>;
  constexpr int kLanes = Half<kDh>::kLanes;
  if constexpr (kInt4) {
    constexpr int kGroups = Tile::kGroups;
    // NaN, which fmin and fmax drop, and infinities make the scale NaN
    float lo[2] = {0.f, 0.f}, hi[2] = {0.f, 0.f}, sick[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[0] = fminf(lo[0], a[i]);
      hi[0] = fmaxf(hi[0], a[i]);
      lo[1] = fminf(lo[1], b[i]);
      hi[1] = fmaxf(hi[1], b[i]);
      sick[0] += a[i] * 0.f;
      sick[1] += b[i] * 0.f;
    }
    if constexpr (kGroups == 1) {
      lo[0] = fminf(lo[0], lo[1]);
      hi[0] = fmaxf(hi[0], hi[1]);
      sick[0] += sick[1];
    }
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        lo[g] = fminf(lo[g], __shfl_xor_sync(0xffffffffu, lo[g], off));
        hi[g] = fmaxf(hi[g], __shfl_xor_sync(0xffffffffu, hi[g], off));
        sick[g] += __shfl_xor_sync(0xffffffffu, sick[g], off);
      }
    if (!there) return;
    Quant qa(lo[0], hi[0]), qb(lo[kGroups - 1], hi[kGroups - 1]);
    qa.scale += sick[0];
    qb.scale += sick[kGroups - 1];
    uint32_t wa = 0, wb = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      wa |= qa.code(a[i]) << (4 * i);
      wb |= qb.code(b[i]) << (4 * i);
    }
    const int da = 8 * j, db = kDh / 2 + 8 * j;
    if (!value) {
      *reinterpret_cast<uint32_t*>(tile + Tile::key(token, da)) = wa;
      *reinterpret_cast<uint32_t*>(tile + Tile::key(token, db)) = wb;
    } else {
      *reinterpret_cast<uint16_t*>(tile + Tile::value(token, da)) = static_cast<uint16_t>(wa);
      *reinterpret_cast<uint16_t*>(tile + Tile::value(token, da + 4)) = static_cast<uint16_t>(wa >> 16);
      *reinterpret_cast<uint16_t*>(tile + Tile::value(token, db)) = static_cast<uint16_t>(wb);
      *reinterpret_cast<uint16_t*>(tile + Tile::value(token, db + 4)) = static_cast<uint16_t>(wb >> 16);
    }
    if (j < kGroups) {
      const Quant& q = j == 0 ? qa : qb;
      *reinterpret_cast<__nv_bfloat16*>(tile + Tile::scale(token, value, j)) = __float2bfloat16_rn(q.scale);
      *reinterpret_cast<uint16_t*>(tile + Tile::zero(token, value, j)) =
          static_cast<uint16_t>(17u * static_cast<uint32_t>(q.scale > 0.f ? q.zero : 0.f));
    }
  } else {
    if (!there) return;
    const int d[2] = {8 * j, kDh / 2 + 8 * j};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float(&x)[8] = h == 0 ? a : b;
      if (!value) {
        *reinterpret_cast<uint4*>(tile + Tile::key(token, d[h])) = pack8(x);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<__nv_bfloat16*>(tile + Tile::value(token, d[h] + (i & 4)) + 4 * (i & 3)) = __float2bfloat16_rn(x[i]);
      }
    }
  }
}

// One row (token slot) a CTA in x, kThreads / kLanes heads in y: the queries', then the keys' and values'.
template <int kDh, bool kInt4>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const KvAppendArgs p) {
  constexpr int kLanes = Half<kDh>::kLanes;
  const int j = threadIdx.x % kLanes;
  const int head = blockIdx.y * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int heads = static_cast<int>(p.n_heads), kv = p.cache.kv_heads;
  const long long row = blockIdx.x;
  const int s = static_cast<int>(row / p.batch.L), t = static_cast<int>(row % p.batch.L);
  pdl_wait();
  pdl_launch_dependents();
  const bool there = head < heads + 2 * kv;
  const bool query = head < heads, value = head >= heads + kv;
  const long long positions = p.batch.max_pages << p.cache.page_bits;
  const KvSeq seq = kv_seq(p.batch, s, p.rope != nullptr ? min(positions, static_cast<long long>(p.rope_len)) : positions, p.err);
  if (t >= seq.n || !seq.ok) {
    if (there && query && p.q_out != nullptr) {
      const uint32_t fill = t < seq.n ? 0x7fff7fffu : 0u;  // NaN, or an empty slot
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.q_out) + row * p.ld_q_out + head * kDh + 8 * j;
      *reinterpret_cast<uint4*>(out) = make_uint4(fill, fill, fill, fill);
      *reinterpret_cast<uint4*>(out + kDh / 2) = make_uint4(fill, fill, fill, fill);
    }
    return;
  }
  const int pos = seq.cached + t;
  float a[8] = {}, b[8] = {};
  if (there) {
    const __nv_bfloat16* x = query   ? static_cast<const __nv_bfloat16*>(p.q) + row * p.ld_q + head * kDh
                             : value ? static_cast<const __nv_bfloat16*>(p.v) + row * p.ld_kv + (head - heads - kv) * kDh
                                     : static_cast<const __nv_bfloat16*>(p.k) + row * p.ld_kv + (head - heads) * kDh;
    unpack8(*reinterpret_cast<const uint4*>(x + 8 * j), a);
    unpack8(*reinterpret_cast<const uint4*>(x + kDh / 2 + 8 * j), b);
  }
  if (p.rope != nullptr && there && !value) {
    const float4* r = reinterpret_cast<const float4*>(p.rope + (static_cast<long long>(pos) * (kDh / 2) + 8 * j) * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 cs = r[i];
      const float c[2] = {cs.x, cs.z}, sn[2] = {cs.y, cs.w};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float x1 = a[2 * i + e], x2 = b[2 * i + e];
        a[2 * i + e] = __fsub_rn(__fmul_rn(x1, c[e]), __fmul_rn(x2, sn[e]));
        b[2 * i + e] = __fadd_rn(__fmul_rn(x1, sn[e]), __fmul_rn(x2, c[e]));
      }
    }
  }
  if (there && query && p.q_out != nullptr) {
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.q_out) + row * p.ld_q_out + head * kDh + 8 * j;
    *reinterpret_cast<uint4*>(out) = pack8(a);
    *reinterpret_cast<uint4*>(out + kDh / 2) = pack8(b);
  }
  const int page = there && !query ? kv_page(p.batch, p.cache, s, pos, p.err) : -1;
  uint8_t* tile = page < 0 ? nullptr
                           : kv_tile<KvTile<kDh, kInt4>>(p.cache, page, value ? head - heads - kv : head - heads, pos);
  store_head<kDh, kInt4>(tile, pos % kKvTile, value, j, a, b, page >= 0);  // (shuffles: by every lane)
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) { *reinterpret_cast<uint4*>(p) = pack8(x); }
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Eight channels a thread, a row a CTA in x.
template <int kDh, bool kInt4, typename Out>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const KvReadArgs p) {
  using Tile = KvTile<kDh, kInt4>;
  constexpr int kLanes = kDh / 8;
  const int j = threadIdx.x % kLanes;
  const int unit = blockIdx.y * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int kv = p.cache.kv_heads;
  const long long row = blockIdx.x;
  const int s = static_cast<int>(row / p.batch.L), t = static_cast<int>(row % p.batch.L);
  pdl_wait();
  pdl_launch_dependents();
  if (unit >= 2 * kv) return;
  const bool value = unit >= kv;
  const int head = value ? unit - kv : unit;
  Out* out = static_cast<Out*>(value ? p.v : p.k);
  if (out == nullptr) return;
  out += row * p.ld + head * kDh + 8 * j;
  const KvSeq seq = kv_seq(p.batch, s, p.batch.max_pages << p.cache.page_bits, p.err);
  float x[8] = {};
  if (t < seq.n) {
    const int pos = seq.cached + t, token = pos & (kKvTile - 1);
    const int page = seq.ok ? kv_page(p.batch, p.cache, s, pos, p.err) : -1;
    if (page < 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __int_as_float(0x7fffffff);
    } else {
      const uint8_t* tile = kv_tile<Tile>(p.cache, page, head, pos);
      if constexpr (kInt4) {
        const uint32_t w = !value ? *reinterpret_cast<const uint32_t*>(tile + Tile::key(token, 8 * j))
                                  : *reinterpret_cast<const uint16_t*>(tile + Tile::value(token, 8 * j)) |
                                        static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(tile + Tile::value(token, 8 * j + 4))) << 16;
        const float scale = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(tile + Tile::scale(token, value, j / 8)));
        const int zero = *reinterpret_cast<const uint16_t*>(tile + Tile::zero(token, value, j / 8)) & 15;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = scale * static_cast<float>(static_cast<int>((w >> (4 * i)) & 15) - zero);
      } else if (!value) {
        unpack8(*reinterpret_cast<const uint4*>(tile + Tile::key(token, 8 * j)), x);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[i] = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(tile + Tile::value(token, 8 * j + (i & 4)) + 4 * (i & 3)));
      }
    }
  }
  store8(out, x);
}

template <int kDh, bool kInt4>
cudaError_t append(const KvAppendArgs& a, cudaStream_t st) {
  const int64_t heads = a.n_heads + 2 * a.cache.kv_heads, per = kThreads / Half<kDh>::kLanes;
  return launch_pdl(kv_append_kernel<kDh, kInt4>, dim3(static_cast<unsigned>(a.batch.S * a.batch.L), static_cast<unsigned>((heads + per - 1) / per)),
                    dim3(kThreads), 0, st, a);
}
template <int kDh, bool kInt4>
cudaError_t read(const KvReadArgs& a, cudaStream_t st) {
  const int per = kThreads / (kDh / 8);
  const dim3 grid(static_cast<unsigned>(a.batch.S * a.batch.L), static_cast<unsigned>((2 * a.cache.kv_heads + per - 1) / per));
  return a.f32 ? launch_pdl(kv_read_kernel<kDh, kInt4, float>, grid, dim3(kThreads), 0, st, a)
               : launch_pdl(kv_read_kernel<kDh, kInt4, __nv_bfloat16>, grid, dim3(kThreads), 0, st, a);
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
