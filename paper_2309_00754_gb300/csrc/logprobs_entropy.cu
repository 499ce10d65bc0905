// Token statistics of rows of logits and their gradient (§2 "Stage 3: PPO": the probability ratio
// needs each sampled token's log-probability, its gradient goes back into the logits).
//
// Forward, per row z of V logits, one pass with a running maximum (Milakov & Gimelshein 2018):
//     m = max z,  s = sum exp(z - m),  w = sum exp(z - m) (z - m)
//     logp = (z[id] - m) - log s,  entropy = log s - w / s
// Both terms of the entropy are at least 0, so nothing cancels; keeping m and log s apart keeps
// log-probabilities exact where |m| is large (a vocabulary masked with the type's lowest value).
//
// The k likeliest tokens, in the order (logit descending, index ascending): every thread keeps the
// best of the slots (16-byte groups of logits) that it read. The k best elements of the row lie in
// the k threads whose best come first in that order: an element of another thread has k better
// ones before it. Those threads' slots alone are read again, and the few elements not behind the
// k-th best thread's best are ranked by counting.
//
// Backward, with p = exp((z - m) - log s):
//     dz[v] = g_logp (1[v = id] - p_v) - g_entropy p_v (log p_v + entropy)
#include "common.cuh"
#include "kernels.h"

namespace hydra {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCandidates = 512;  // elements ranked at once
constexpr float kInf = __builtin_huge_valf(), kNan = __builtin_nanf("");
constexpr float kLog2e = 1.4426950408889634f;
// exp of anything below is 0 in fp32; a finite stand-in keeps 0 * (z - m) from being 0 * -inf
constexpr float kFloor = -256.f;

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float exp_fast(float x) {  // 2 ulp of ex2, x <= 0
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * kLog2e));
  return r;
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A row's elements in slots of 16 bytes on the address grid: slot j holds elements
// [j E - a, j E - a + E), the first and the last of them possibly in part.
template <typename T>
struct Row {
  static constexpr int E = 16 / sizeof(T);
  const T* p;
  int a, V, n_slots, full_lo, full_hi;  // slots [full_lo, full_hi) are whole

  __device__ __forceinline__ Row(const T* row, int v) : p(row), V(v) {
    a = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    n_slots = static_cast<int>((static_cast<long long>(v) + a + E - 1) / E);
    full_lo = a > 0 ? 1 : 0;
    full_hi = static_cast<int>((static_cast<long long>(v) + a) / E);
  }
  // index of a slot's first element (below 0 in the first slot)
  __device__ __forceinline__ int first(int j) const { return j * E - a; }
  __device__ __forceinline__ uint4 load_full(int j) const {
    return *reinterpret_cast<const uint4*>(p + first(j));
  }
  __device__ __forceinline__ void load(int j, float (&f)[E]) const {
    if (j >= full_lo && j < full_hi) {
      unpack(load_full(j), f);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = first(j) + e;
        f[e] = i >= 0 && i < V ? to_f(p[i]) : -kInf;
      }
    }
  }
  __device__ static __forceinline__ void unpack(const uint4& v, float (&f)[E]) {
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (E == 4) {
        f[q] = __uint_as_float(r[q]);
      } else {
        const float2 x = unpack_bf16x2(r[q]);
        f[2 * q] = x.x;
        f[2 * q + 1] = x.y;
      }
    }
  }
};

// Order of logits as unsigned integers: NaN first, then descending, -0 equal to 0. No value maps to 0.
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0xffffffffu;
  const int b = __float_as_int(v + 0.f);
  return b < 0 ? ~static_cast<uint32_t>(b) : static_cast<uint32_t>(b) | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) {
  if (k == 0xffffffffu) return kNan;
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// larger: better value, or the same at a lower index
__device__ __forceinline__ uint64_t rank_key(uint32_t key, int index) {
  return static_cast<uint64_t>(key) << 32 | static_cast<uint32_t>(~index);
}

struct Stats {  // running maximum, sum of exp(z - m), sum of exp(z - m) (z - m)
  float m = -kInf, s = 0.f, w = 0.f;

  // nm is the new maximum (NaN if there is a NaN)
  __device__ __forceinline__ void rescale(float nm) {
    const float d = max_nan(m - nm, kFloor);
    const float c = exp_fast(d);
    w = c * (w + s * d);
    s *= c;
    m = nm;
  }
  __device__ __forceinline__ void merge(float m2, float s2, float w2) {
    const float nm = max_nan(m, m2);
    // both -inf: the difference is NaN, the sums 0
    const float d1 = fmaxf(m - nm, kFloor), d2 = fmaxf(m2 - nm, kFloor);
    const float c1 = exp_fast(d1), c2 = exp_fast(d2);
    w = c1 * (w + s * d1) + c2 * (w2 + s2 * d2);
    s = s * c1 + s2 * c2;
    m = nm;
  }
};

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int mask) {
  return __shfl_xor_sync(0xffffffffu, static_cast<unsigned long long>(v), mask);
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t min64(uint64_t a, uint64_t b) { return a < b ? a : b; }

// Bitonic network over a warp, one key a lane, lane 0 the largest.
__device__ __forceinline__ uint64_t bitonic_merge(uint64_t v, int lane) {
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const uint64_t o = shfl_xor64(v, j);
    v = lane & j ? min64(v, o) : max64(v, o);
  }
  return v;
}
__device__ __forceinline__ uint64_t sort_warp(uint64_t v, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
    for (int j = size >> 1; j > 0; j >>= 1) {
      const uint64_t o = shfl_xor64(v, j);
      const bool descending = (lane & size) == 0;
      v = ((lane & j) == 0) == descending ? max64(v, o) : min64(v, o);
    }
  }
  return v;
}

struct TopShared {
  uint64_t list[kWarps][32];
  uint64_t cand[kCandidates];
  uint64_t floor;  // elements behind it are not among the k best
  int count;
};

template <typename T, bool kTop>
__global__ void __launch_bounds__(kThreads)
    token_stats_kernel(const T* __restrict__ logits, long long ld, int L, int V,
                       const int32_t* __restrict__ ids, const int32_t* __restrict__ lengths, int k,
                       float* __restrict__ logp, float* __restrict__ entropy, float* __restrict__ norm,
                       int32_t* __restrict__ top_ids, float* __restrict__ top_logp, int* err) {
  constexpr int E = Row<T>::E;
  constexpr int U = 4;
  pdl_wait();
  pdl_launch_dependents();
  const long long row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sq = static_cast<int>(row / L);
  const int t = static_cast<int>(row - static_cast<long long>(sq) * L);
  int n = lengths ? lengths[sq] : L;
  if (n < 0 || n > L) {
    if (tid == 0) record_error(err, kDevBadLength);
    n = n < 0 ? 0 : L;
  }
  if (t >= n) {
    if (tid == 0) {
      if (logp) logp[row] = 0.f;
      if (entropy) entropy[row] = 0.f;
      if (norm) norm[2 * row] = norm[2 * row + 1] = 0.f;
    }
    if (kTop && tid < k) {
      top_ids[row * k + tid] = -1;
      top_logp[row * k + tid] = 0.f;
    }
    return;
  }
  const Row<T> r(logits + row * ld, V);
  Stats st;
  uint32_t best = 0;
  int best_slot = 0;
  for (int j0 = tid; j0 < r.n_slots; j0 += U * kThreads) {
    float f[U][E], vm[U];
    const bool whole = j0 >= r.full_lo && j0 + (U - 1) * kThreads < r.full_hi;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kThreads;
      if (whole) {
        Row<T>::unpack(r.load_full(j), f[u]);
      } else if (j < r.n_slots) {
        r.load(j, f[u]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) f[u][e] = -kInf;
      }
    }
    float cm = -kInf;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      vm[u] = f[u][0];
#pragma unroll
      for (int e = 1; e < E; ++e) vm[u] = max_nan(vm[u], f[u][e]);
      cm = max_nan(cm, vm[u]);
    }
    if (!(cm <= st.m) || (kTop && best == 0)) {
      if (kTop) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t key = order_key(vm[u]);
          if (key > best && j0 + u * kThreads < r.n_slots) {
            best = key;
            best_slot = j0 + u * kThreads;
          }
        }
      }
      if (!(cm <= st.m)) st.rescale(max_nan(st.m, cm));
    }
    const float base = st.m == -kInf ? 0.f : st.m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = max_nan(f[u][e] - base, kFloor);
        const float x = exp_fast(d);
        st.s += x;
        st.w += x * d;
      }
    }
  }

  __shared__ float red[3][kWarps];
  __shared__ float row_norm[2];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, st.m, off), s2 = __shfl_xor_sync(0xffffffffu, st.s, off),
                w2 = __shfl_xor_sync(0xffffffffu, st.w, off);
    st.merge(m2, s2, w2);
  }
  if (lane == 0) {
    red[0][warp] = st.m;
    red[1][warp] = st.s;
    red[2][warp] = st.w;
  }
  __shared__ TopShared top;
  uint64_t mine = 0;
  if (kTop) {
    mine = sort_warp(best == 0 ? 0 : rank_key(best, best_slot), lane);
    top.list[warp][lane] = mine;
  }
  __syncthreads();
  if (tid == 0) {
    st = Stats();
    for (int q = 0; q < kWarps; ++q) st.merge(red[0][q], red[1][q], red[2][q]);
    const bool empty = st.m == -kInf;  // nothing but -inf
    const float ls = empty ? 0.f : logf(st.s);
    row_norm[0] = st.m;
    row_norm[1] = ls;
    if (norm) {
      norm[2 * row] = st.m;
      norm[2 * row + 1] = ls;
    }
    if (entropy) entropy[row] = empty ? 0.f : ls - st.w / st.s;
    if (logp) {
      const int id = ids[row];
      if (id < 0 || id >= V) {
        record_error(err, kDevBadTokenId);
        logp[row] = kNan;
      } else {
        logp[row] = empty ? -kInf : (to_f(r.p[id]) - st.m) - ls;
      }
    }
  }
  if constexpr (kTop) {

    // the 32 best of the threads' bests, in warp 0
    for (int half = kWarps / 2; half > 0; half >>= 1) {
      if (warp < half) {
        mine = bitonic_merge(max64(mine, top.list[warp + half][31 - lane]), lane);
        top.list[warp][lane] = mine;
      }
      __syncthreads();
    }
    const uint64_t slot_floor = top.list[0][k - 1];  // 0 where fewer threads than k hold anything
    if (tid == 0) top.floor = 0;
    for (;;) {
      if (tid == 0) top.count = 0;
      __syncthreads();
      const uint64_t floor = top.floor;
      for (int g = warp; g < k; g += kWarps) {
        const uint64_t key = top.list[0][g];
        if (key == 0) break;
        const int owner = static_cast<int>(~static_cast<uint32_t>(key)) % kThreads;
        for (int j = owner + lane * kThreads; j < r.n_slots; j += 32 * kThreads) {
          float f[E];
          r.load(j, f);
  #pragma unroll
          for (int e = 0; e < E; ++e) {
            const int i = r.first(j) + e;
            const uint32_t key_e = order_key(f[e]);
            if (i >= 0 && i < V && rank_key(key_e, j) >= slot_floor && rank_key(key_e, i) >= floor) {
              const int at = atomicAdd(&top.count, 1);
              if (at < kCandidates) top.cand[at] = rank_key(key_e, i);
            }
          }
        }
      }
      __syncthreads();
      const int count = top.count, held = min(count, kCandidates);
      for (int c = tid; c < held; c += kThreads) {
        const uint64_t key = top.cand[c];
        int rank = 0;
        for (int o = 0; o < held; ++o) rank += top.cand[o] > key;
        if (count > kCandidates) {
          // more than fit: the k-th best of those held is a higher floor, which leaves out the rest
          if (rank == k - 1) top.floor = key;
        } else if (rank < k) {
          const float v = order_value(static_cast<uint32_t>(key >> 32));
          const float m = row_norm[0];
          top_ids[row * k + rank] = static_cast<int>(~static_cast<uint32_t>(key));
          top_logp[row * k + rank] = m == -kInf ? -kInf : (v - m) - row_norm[1];
        }
      }
      if (count <= kCandidates) return;
      __syncthreads();
    }
  }
}

constexpr int kUnit = 8;      // elements a thread turns at once
constexpr int kUnitsEach = 2;
constexpr int kTile = kThreads * kUnit * kUnitsEach;

template <typename T>
__device__ __forceinline__ void load_unit(const T* p, float (&f)[kUnit]) {
  constexpr int E = 16 / sizeof(T);
#pragma unroll
  for (int q = 0; q < kUnit / E; ++q) {
    float part[E];
    Row<T>::unpack(*reinterpret_cast<const uint4*>(p + q * E), part);
#pragma unroll
    for (int e = 0; e < E; ++e) f[q * E + e] = part[e];
  }
}
__device__ __forceinline__ void store_unit(float* p, const float (&f)[kUnit]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store_unit(__nv_bfloat16* p, const float (&f)[kUnit]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                            pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// One CTA per tile of a row. Units lie on the 16-byte grid of both arrays where their rows start
// alike on it (`a` elements before the row); else every element goes by itself.
template <typename TI, typename TO>
__global__ void __launch_bounds__(kThreads)
    token_stats_grad_kernel(const TI* logits, long long ld, int L, int V, int tiles,
                            const int32_t* __restrict__ ids, const int32_t* __restrict__ lengths,
                            const float* __restrict__ norm, const float* __restrict__ entropy,
                            const float* __restrict__ grad_logp, const float* __restrict__ grad_entropy,
                            TO* dlogits, long long ld_d, int* err) {
  pdl_wait();
  pdl_launch_dependents();
  const long long row = blockIdx.x / tiles;
  const int tile = static_cast<int>(blockIdx.x - row * tiles);
  const int tid = threadIdx.x;
  const int sq = static_cast<int>(row / L);
  const int t = static_cast<int>(row - static_cast<long long>(sq) * L);
  int n = lengths ? lengths[sq] : L;
  if (n < 0 || n > L) {
    if (tid == 0) record_error(err, kDevBadLength);
    n = n < 0 ? 0 : L;
  }
  const TI* z = logits + row * ld;
  TO* d = dlogits + row * ld_d;
  const float m = norm[2 * row], ls = norm[2 * row + 1];
  const bool live = t < n && m != -kInf;  // an empty row has no gradient
  float gl = 0.f, gh = 0.f, h = 0.f;
  int id = -1;
  if (live) {
    if (grad_logp) gl = grad_logp[row];
    if (grad_entropy) {
      gh = grad_entropy[row];
      h = entropy[row];
    }
    id = grad_logp ? ids[row] : 0;
    if (id < 0 || id >= V) {
      if (tid == 0) record_error(err, kDevBadTokenId);
      gl = kNan;
    }
  }
  const float c0 = gl + gh * h;
  auto value = [&](float x, int i) {
    const float lp = max_nan((x - m) - ls, kFloor);
    const float p = exp_fast(lp);
    // 1 - p of a token that is nearly certain
    return i == id && grad_logp ? -gl * expm1f(lp) - p * (gh * (lp + h)) : -p * (c0 + gh * lp);
  };
  const int phase_i = static_cast<int>(reinterpret_cast<uintptr_t>(z) / sizeof(TI) % kUnit);
  const int phase_o = static_cast<int>(reinterpret_cast<uintptr_t>(d) / sizeof(TO) % kUnit);
  const int a = sizeof(TO) == 2 ? phase_o : phase_i;
  const bool together = (phase_i - a) % static_cast<int>(16 / sizeof(TI)) == 0 &&
                        (phase_o - a) % static_cast<int>(16 / sizeof(TO)) == 0;
  if (together) {
#pragma unroll
    for (int u = 0; u < kUnitsEach; ++u) {
      const long long i0 = static_cast<long long>(tile) * kTile + (u * kThreads + tid) * kUnit - a;
      if (i0 >= V) return;
      const int i = static_cast<int>(i0);
      if (i >= 0 && i0 + kUnit <= V) {
        float f[kUnit] = {};
        if (live) {
          load_unit(z + i, f);
#pragma unroll
          for (int e = 0; e < kUnit; ++e) f[e] = value(f[e], i + e);
        }
        store_unit(d + i, f);
      } else {
        for (int e = max(i, 0); e < min(i0 + kUnit, static_cast<long long>(V)); ++e)
          d[e] = from_f<TO>(live ? value(to_f(z[e]), e) : 0.f);
      }
    }
  } else {
    const long long i0 = static_cast<long long>(tile) * kTile - a;
    const int hi = static_cast<int>(min(i0 + kTile, static_cast<long long>(V)));
    for (int i = static_cast<int>(max(i0, 0LL)) + tid; i < hi; i += kThreads)
      d[i] = from_f<TO>(live ? value(to_f(z[i]), i) : 0.f);
  }
}

template <typename T>
int launch_stats(const TokenStatsArgs& a, cudaStream_t stream) {
  const auto kernel = a.top_k > 0 ? token_stats_kernel<T, true> : token_stats_kernel<T, false>;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(a.S * a.L)), dim3(kThreads), 0, stream,
                    static_cast<const T*>(a.logits), static_cast<long long>(a.ld), static_cast<int>(a.L),
                    static_cast<int>(a.V), a.ids, a.lengths, static_cast<int>(a.top_k), a.logp, a.entropy,
                    a.norm, a.top_ids, a.top_logp, a.err) == cudaSuccess
             ? 0
             : -3;
}

template <typename TI, typename TO>
int launch_grad(const TokenStatsGradArgs& a, cudaStream_t stream) {
  const int64_t tiles = token_stats_grad_tiles(a.V);
  return launch_pdl(token_stats_grad_kernel<TI, TO>, dim3(static_cast<unsigned>(a.S * a.L * tiles)),
                    dim3(kThreads), 0, stream, static_cast<const TI*>(a.logits), static_cast<long long>(a.ld),
                    static_cast<int>(a.L), static_cast<int>(a.V), static_cast<int>(tiles), a.ids, a.lengths,
                    a.norm, a.entropy, a.grad_logp, a.grad_entropy, static_cast<TO*>(a.dlogits),
                    static_cast<long long>(a.ld_d), a.err) == cudaSuccess
             ? 0
             : -3;
}

}  // namespace

int launch_token_stats(const TokenStatsArgs& a, cudaStream_t stream) {
  return a.bf16 ? launch_stats<__nv_bfloat16>(a, stream) : launch_stats<float>(a, stream);
}

// the row's first unit may start up to kUnit - 1 elements before it
int64_t token_stats_grad_tiles(int64_t V) { return (V + kUnit - 1 + kTile - 1) / kTile; }

int launch_token_stats_grad(const TokenStatsGradArgs& a, cudaStream_t stream) {
  if (a.bf16)
    return a.grad_bf16 ? launch_grad<__nv_bfloat16, __nv_bfloat16>(a, stream)
                       : launch_grad<__nv_bfloat16, float>(a, stream);
  return a.grad_bf16 ? launch_grad<float, __nv_bfloat16>(a, stream) : launch_grad<float, float>(a, stream);
}

}  // namespace hydra
