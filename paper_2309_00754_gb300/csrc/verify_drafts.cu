// Drafted tokens accepted or refused by the target's probabilities, and the token that follows them (speculative
// sampling: Leviathan, Kalman and Matias 2023, "Fast inference from transformers via speculative decoding"):
//
//   a_i = min(1, p_i(x_i) / q_i(x_i));  x_i is kept while u_i < a_i
//   then argmax_v (log max(p_j - q_j, 0)[v] + noise[v]) at the first refusal j, or argmax_v (z_n[v] + noise[v])
//
// with p, q the target's and the draft model's probabilities and the noise standard Gumbel, so that the argmax is a
// draw from the distribution whose logarithm it perturbs. Without random numbers a token is kept while it is the target's
// argmax.
//
// Bound by the reads of the logits. A cluster of CTAs has a sequence: each CTA takes a slice of the vocabulary of all its
// rows, a warp a share of that, in one pass with a running maximum and sum; the shares' (maximum, sum) pairs are all that
// the CTAs exchange before every one of them knows where the drafts end. The row that the last token is drawn from is
// read a second time, from L2 as a rule.
#include <algorithm>
#include <cfloat>
#include <climits>

#include "common.cuh"
#include "kernels.h"

namespace hydra {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kMaxRows = 2 * kVerifyMaxDrafts + 1;  // target rows 0..n, then draft rows 0..n-1

// A value with its index; the larger one, of equal ones the lower index.
struct Best {
  float v = -INFINITY;
  int i = INT_MAX;
  __device__ __forceinline__ void take(float ov, int oi) {
    if (ov > v || (ov == v && oi < i)) {
      v = ov;
      i = oi;
    }
  }
};

// Part of a row: maximum (-FLT_MAX where there is none), sum of exp(z - maximum); greedy: its argmax.
struct Part {
  float m = -FLT_MAX, s = 0.f;
  Best best;
};

struct Shared {
  Part part[kMaxRows][kWarps];
  Part cta[kMaxRows];              // this CTA's, read by the cluster
  float m[kMaxRows], c[kMaxRows];  // of whole rows: maximum, log of the sum
  int top[kMaxRows];
  Best best[2][kWarps];
  Best cta_best[2];  // drawn from the residual, from the row; read by the cluster
  int kept;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ void unpack(const uint4& v, float (&f)[16 / sizeof(T)]) {
  const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (sizeof(T) == 4) {
      f[q] = __uint_as_float(r[q]);
    } else {
      const float2 x = unpack_bf16x2(r[q]);
      f[2 * q] = x.x;
      f[2 * q + 1] = x.y;
    }
  }
}

__device__ __forceinline__ float exp_fast(float x) { return exp2f(x * 1.4426950408889634f); }

// N neighbouring logits more, the first at index `first`.
template <bool kArg, int N>
__device__ __forceinline__ void add(Part& p, const float (&x)[N], int first) {
  float top = x[0];
#pragma unroll
  for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
  if constexpr (kArg) {
    if (top > p.best.v || p.best.i == INT_MAX)
#pragma unroll
      for (int e = 0; e < N; ++e) p.best.take(x[e], first + e);
  }
  const float now = fmaxf(p.m, top);
  p.s *= exp_fast(p.m - now);
  p.m = now;
#pragma unroll
  for (int e = 0; e < N; ++e) p.s += exp_fast(x[e] - now);
}

template <bool kArg>
__device__ __forceinline__ void merge(Part& p, const Part& o) {
  if constexpr (kArg) p.best.take(o.best.v, o.best.i);
  const float now = fmaxf(p.m, o.m);
  p.s = p.s * exp_fast(p.m - now) + o.s * exp_fast(o.m - now);
  p.m = now;
}

// [lo, hi) of a row by a warp.
template <typename T, bool kArg>
__device__ __forceinline__ Part scan(const T* row, int lo, int hi, int lane) {
  constexpr int E = 16 / sizeof(T), kDeep = 4;
  Part p;
  const int off = static_cast<int>((reinterpret_cast<uintptr_t>(row + lo) & 15) / sizeof(T));
  const int head = min(off == 0 ? 0 : E - off, hi - lo);
  const int vecs = (hi - lo - head) / E, body = lo + head;
  if (lane < head) {
    const float x[1] = {to_f(row[lo + lane])};
    add<kArg>(p, x, lo + lane);
  }
  for (int v = lane; v < vecs; v += 32 * kDeep) {
    uint4 raw[kDeep];
#pragma unroll
    for (int d = 0; d < kDeep; ++d)
      if (v + 32 * d < vecs) raw[d] = *reinterpret_cast<const uint4*>(row + body + (v + 32 * d) * E);
#pragma unroll
    for (int d = 0; d < kDeep; ++d)
      if (v + 32 * d < vecs) {
        float x[E];
        unpack<T>(raw[d], x);
        add<kArg>(p, x, body + (v + 32 * d) * E);
      }
  }
  const int tail = body + vecs * E + lane;
  if (tail < hi) {
    const float x[1] = {to_f(row[tail])};
    add<kArg>(p, x, tail);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Part other;
    other.m = __shfl_xor_sync(0xffffffffu, p.m, o);
    other.s = __shfl_xor_sync(0xffffffffu, p.s, o);
    if constexpr (kArg) {
      other.best.v = __shfl_xor_sync(0xffffffffu, p.best.v, o);
      other.best.i = __shfl_xor_sync(0xffffffffu, p.best.i, o);
    }
    merge<kArg>(p, other);
  }
  return p;
}

// (the address of `local` in another CTA)
__device__ __forceinline__ float ld_cluster(const float* local, unsigned rank) { return ld_cluster_f32(local, rank); }
__device__ __forceinline__ int ld_cluster(const int* local, unsigned rank) {
  return __float_as_int(ld_cluster_f32(reinterpret_cast<const float*>(local), rank));
}

template <typename T, bool kGreedy>
__global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyArgs p, int cs) {
  extern __shared__ uint8_t raw_shared[];
  Shared& sh = *reinterpret_cast<Shared*>(raw_shared);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = cs > 1 ? static_cast<int>(cluster_rank()) : 0;
  const long long s = blockIdx.x / cs;
  const int V = static_cast<int>(p.V), D = static_cast<int>(p.D);
  pdl_wait();
  pdl_launch_dependents();
  const int given = p.n_draft != nullptr ? p.n_draft[s] : D;
  const int n = min(max(given, 0), D);
  if (n != given && threadIdx.x == 0 && rank == 0) record_error(p.err, kDevBadLength);
  const T* target = static_cast<const T*>(p.target) + s * (D + 1) * p.ld;
  const T* draft = p.draft != nullptr ? static_cast<const T*>(p.draft) + s * D * p.ld_draft : nullptr;
  const int rows = n + 1 + (draft != nullptr ? n : 0);

  // this CTA's slice, and the warp's share of it, whole vectors of a row that starts at one
  const int step = ((V + cs * kWarps - 1) / (cs * kWarps) + 7) & ~7;
  const int lo = min(V, (rank * kWarps + warp) * step), hi = min(V, lo + step);
  for (int r = 0; r < rows; ++r) {
    const T* row = r <= n ? target + r * p.ld : draft + (r - n - 1) * p.ld_draft;
    const Part part = scan<T, kGreedy>(row, lo, hi, lane);
    if (lane == 0) sh.part[r][warp] = part;
  }
  __syncthreads();
  for (int r = threadIdx.x; r < rows; r += kThreads) {
    Part all = sh.part[r][0];
    for (int w = 1; w < kWarps; ++w) merge<kGreedy>(all, sh.part[r][w]);
    sh.cta[r] = all;
  }
  if (cs > 1) cluster_sync_all(); else __syncthreads();
  for (int r = threadIdx.x; r < rows; r += kThreads) {
    Part all = sh.cta[r];
    if (cs > 1)
      for (int c = 0; c < cs; ++c) {
        Part o;
        o.m = ld_cluster(&sh.cta[r].m, c);
        o.s = ld_cluster(&sh.cta[r].s, c);
        if (kGreedy) {
          o.best.v = ld_cluster(&sh.cta[r].best.v, c);
          o.best.i = ld_cluster(&sh.cta[r].best.i, c);
        }
        if (c == 0) all = o; else merge<kGreedy>(all, o);
      }
    // a row of nothing but -inf: its sum is 0
    sh.m[r] = all.s == 0.f ? -INFINITY : all.m;
    sh.c[r] = all.s == 0.f ? 0.f : logf(all.s);
    sh.top[r] = all.best.i == INT_MAX ? 0 : all.best.i;  // (nothing but NaN)
  }
  __syncthreads();

  // log-probability of token x in row r (the sums are in fp32; what is made of them here in 64 bits)
  auto log_p = [&](const T* row, int r, int x) {
    return static_cast<double>(to_f(row[x])) - sh.m[r] - sh.c[r];
  };
  if (warp == 0) {
    float a = 0.f;
    bool keep = false;
    if (lane < n) {
      const int x = p.ids[s * D + lane];
      if (x < 0 || x >= V) {
        a = __int_as_float(0x7fffffff);
        if (rank == 0) record_error(p.err, kDevBadTokenId);
      } else if (kGreedy) {
        keep = sh.top[lane] == x;
        a = keep ? 1.f : 0.f;
      } else {
        const T* row = target + lane * p.ld;
        if (sh.m[lane] == -INFINITY || to_f(row[x]) == -INFINITY) {
          a = 0.f;
        } else {
          double d = log_p(row, lane, x);
          if (draft != nullptr) {
            const T* q = draft + lane * p.ld_draft;
            d = sh.m[n + 1 + lane] == -INFINITY ? INFINITY : d - log_p(q, n + 1 + lane, x);
          }
          a = d >= 0.0 ? 1.f : expf(static_cast<float>(d));
        }
        keep = p.uniform[s * D + lane] < a;
      }
    }
    const unsigned refused = __ballot_sync(0xffffffffu, !keep);
    const int kept = min(n, refused == 0 ? 32 : __ffs(refused) - 1);
    if (lane == 0) sh.kept = kept;
    if (rank == 0 && p.accept != nullptr && lane < D) p.accept[s * D + lane] = a;
  }
  __syncthreads();
  const int kept = sh.kept;
  const T* last = target + kept * p.ld;
  int next = sh.top[kept];

  if constexpr (!kGreedy) {
    const float* noise = p.gumbel + s * p.ld_gumbel;
    const bool refused = kept < n;
    const T* q = refused && draft != nullptr ? draft + kept * p.ld_draft : nullptr;
    const int x = refused ? p.ids[s * D + kept] : -1;
    const float pm = sh.m[kept], pc = sh.c[kept];
    const float qm = q != nullptr ? sh.m[n + 1 + kept] : 0.f, qc = q != nullptr ? sh.c[n + 1 + kept] : 0.f;
    Best rest, whole;
    const int mine = (V + cs - 1) / cs, from = min(V, rank * mine), to = min(V, from + mine);
    for (int v = from + threadIdx.x; v < to; v += kThreads) {
      const float z = to_f(last[v]), g = noise[v];
      whole.take(z + g, v);
      if (q != nullptr) {
        const float pv = z == -INFINITY ? 0.f : expf((z - pm) - pc);
        const float w = to_f(q[v]);
        const float r = pv - (w == -INFINITY ? 0.f : expf((w - qm) - qc));
        if (r > 0.f) rest.take(logf(r) + g, v);
      } else if (refused && v != x && z > -INFINITY) {
        rest.take(z + g, v);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      rest.take(__shfl_xor_sync(0xffffffffu, rest.v, o), __shfl_xor_sync(0xffffffffu, rest.i, o));
      whole.take(__shfl_xor_sync(0xffffffffu, whole.v, o), __shfl_xor_sync(0xffffffffu, whole.i, o));
    }
    if (lane == 0) {
      sh.best[0][warp] = rest;
      sh.best[1][warp] = whole;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
      Best b = sh.best[threadIdx.x][0];
      for (int w = 1; w < kWarps; ++w) b.take(sh.best[threadIdx.x][w].v, sh.best[threadIdx.x][w].i);
      sh.cta_best[threadIdx.x] = b;
    }
    if (cs > 1) cluster_sync_all(); else __syncthreads();
    rest = sh.cta_best[0];
    whole = sh.cta_best[1];
    if (cs > 1 && rank == 0)
      for (int c = 1; c < cs; ++c) {
        rest.take(ld_cluster(&sh.cta_best[0].v, c), ld_cluster(&sh.cta_best[0].i, c));
        whole.take(ld_cluster(&sh.cta_best[1].v, c), ld_cluster(&sh.cta_best[1].i, c));
      }
    // nothing of the residual is left: from the row itself
    next = refused && rest.i != INT_MAX ? rest.i : whole.i != INT_MAX ? whole.i : 0;
  }
  if (rank == 0) {
    for (int i = threadIdx.x; i <= D; i += kThreads) {
      const int tok = i < kept ? p.ids[s * D + i] : i == kept ? next : -1;
      p.tokens[s * (D + 1) + i] = tok;
      if (p.logp != nullptr)
        p.logp[s * (D + 1) + i] = i > kept                ? 0.f
                                  : sh.m[i] == -INFINITY ? -INFINITY
                                                          : static_cast<float>(log_p(target + i * p.ld, i, tok));
    }
    if (threadIdx.x == 0) p.accepted[s] = kept;
  }
  if (cs > 1) cluster_sync_all();  // nobody leaves while its memory is read
}

template <typename T, bool kGreedy>
cudaError_t launch(const VerifyArgs& a, cudaStream_t st) {
  // the fewest CTAs a sequence that fill the device, none with under 1000 tokens
  int cs = 1;
  while (cs < kMaxCluster && a.S * cs < 2 * std::max(1, sm_count()) && a.V >= 2000 * cs) cs *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.S * cs));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Shared);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(cs);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_kernel<T, kGreedy>, a, cs);
}

}  // namespace

int launch_verify_drafts(const VerifyArgs& a, cudaStream_t st) {
  const bool greedy = a.gumbel == nullptr;
  const auto f = a.bf16 ? (greedy ? launch<__nv_bfloat16, true> : launch<__nv_bfloat16, false>)
                        : (greedy ? launch<float, true> : launch<float, false>);
  return f(a, st) == cudaSuccess ? 0 : -3;
}

}  // namespace hydra
