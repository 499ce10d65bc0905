// Attention of each sequence's new tokens over a paged key/value cache (kv_cache.cuh):
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(a q.k_j - m),  j <= cached + t
//
// in one pass over the keys and values, with the running maximum m and sum. A warp takes every eighth token, a lane D / 32
// channels of it.
#include <cfloat>

#include "kv_cache.cuh"

namespace hydra {
namespace {

constexpr int kWarps = 8;

template <int kDh, bool kInt4>
__global__ void __launch_bounds__(kWarps * 32) paged_attention_kernel(const PagedAttentionArgs p) {
  using Tile = KvTile<kDh, kInt4>;
  constexpr int kE = kDh / 32;  // channels of a lane
  __shared__ float sh_o[kWarps][kDh], sh_m[kWarps], sh_l[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d0 = lane * kE;
  const int head = blockIdx.y, group = static_cast<int>(p.n_heads) / p.cache.kv_heads;
  const long long row = blockIdx.x;
  const int s = static_cast<int>(row / p.batch.L), t = static_cast<int>(row % p.batch.L);
  pdl_wait();
  pdl_launch_dependents();
  const KvSeq seq = kv_seq(p.batch, s, p.batch.max_pages << p.cache.page_bits, p.err);
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + row * p.ld_out + head * kDh;
  if (t >= seq.n || !seq.ok) {
    for (int d = threadIdx.x; d < kDh; d += kWarps * 32) out[d] = __float2bfloat16_rn(t < seq.n ? __int_as_float(0x7fffffff) : 0.f);
    return;
  }
  float q[kE], o[kE] = {};
  for (int e = 0; e < kE; ++e)
    q[e] = __bfloat162float((static_cast<const __nv_bfloat16*>(p.q) + row * p.ld_q + head * kDh)[d0 + e]) * p.scale;
  float m = -FLT_MAX, l = 0.f;
  for (int pos = warp; pos <= seq.cached + t; pos += kWarps) {
    const int page = kv_page(p.batch, p.cache, s, pos, p.err);
    if (page < 0) {
      l = __int_as_float(0x7fffffff);
      break;
    }
    const uint8_t* tile = kv_tile<Tile>(p.cache, page, head / group, pos);
    const int token = pos & (kKvTile - 1);
    float k[kE], v[kE];
    for (int e = 0; e < kE; ++e) {
      const int d = d0 + e;
      if constexpr (kInt4) {
        const uint32_t kw = *reinterpret_cast<const uint32_t*>(tile + Tile::key(token, d & ~7));
        const uint16_t vw = *reinterpret_cast<const uint16_t*>(tile + Tile::value(token, d & ~3));
        const int zk = *reinterpret_cast<const uint16_t*>(tile + Tile::zero(token, false, d >> 6)) & 15;
        const int zv = *reinterpret_cast<const uint16_t*>(tile + Tile::zero(token, true, d >> 6)) & 15;
        k[e] = (static_cast<int>((kw >> (4 * (d & 7))) & 15) - zk) *
               __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(tile + Tile::scale(token, false, d >> 6)));
        v[e] = (static_cast<int>((vw >> (4 * (d & 3))) & 15) - zv) *
               __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(tile + Tile::scale(token, true, d >> 6)));
      } else {
        k[e] = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(tile + Tile::key(token, d & ~7))[d & 7]);
        v[e] = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(tile + Tile::value(token, d & ~3) + 4 * (d & 3)));
      }
    }
    float x = 0.f;
    for (int e = 0; e < kE; ++e) x = fmaf(q[e], k[e], x);
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    const float m_new = fmaxf(m, x), by = expf(m - m_new), pj = expf(x - m_new);
    m = m_new;
    l = l * by + pj;
    for (int e = 0; e < kE; ++e) o[e] = o[e] * by + pj * v[e];
  }
  for (int e = 0; e < kE; ++e) sh_o[warp][d0 + e] = o[e];
  if (lane == 0) {
    sh_m[warp] = m;
    sh_l[warp] = l;
  }
  __syncthreads();
  if (threadIdx.x < kDh) {
    float top = -FLT_MAX, sum = 0.f, acc = 0.f;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh_m[w]);
    for (int w = 0; w < kWarps; ++w) {
      const float by = expf(sh_m[w] - top);
      sum += sh_l[w] * by;
      acc += sh_o[w][threadIdx.x] * by;
    }
    out[threadIdx.x] = __float2bfloat16_rn(acc / sum);
  }
}

}  // namespace

size_t paged_attention_workspace_bytes(int64_t, int64_t, int64_t, int64_t, int64_t) { return 16; }

int launch_paged_attention(const PagedAttentionArgs& a, cudaStream_t st) {
  const auto f = a.cache.head_dim == 128 ? (a.cache.int4 ? paged_attention_kernel<128, true> : paged_attention_kernel<128, false>)
                                         : (a.cache.int4 ? paged_attention_kernel<64, true> : paged_attention_kernel<64, false>);
  return launch_pdl(f, dim3(static_cast<unsigned>(a.batch.S * a.batch.L), static_cast<unsigned>(a.n_heads)), dim3(kWarps * 32), 0,
                    st, a) == cudaSuccess
             ? 0
             : -3;
}

}  // namespace hydra
