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
// Bound by the reads of the logits. A cluster of CTAs has a sequence. Every row is cut in the same number of slices, which its
// warps take in turn, each in one pass with a running maximum and sum; the slices' (maximum, sum) pairs are all that the CTAs
// exchange before every one of them knows where the drafts end. (Cut alike, equal rows have equal sums: a draft model that
// is the target is never refused.) The row that the last token is drawn from is read a second time, from L2 as a rule.
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

// A value with its index, and a logit beside it; the larger value, of equal ones the lower index.
struct Best {
  float v = -INFINITY;
  int i = INT_MAX;
  float z = -INFINITY;
  __device__ __forceinline__ void take(float ov, int oi, float oz) {
    if (ov > v || (ov == v && oi < i)) {
      v = ov;
      i = oi;
      z = oz;
    }
  }
  __device__ __forceinline__ void take_lanes(int most) {
    for (int o = most / 2; o > 0; o >>= 1)
      take(__shfl_xor_sync(0xffffffffu, v, o), __shfl_xor_sync(0xffffffffu, i, o), __shfl_xor_sync(0xffffffffu, z, o));
  }
};

// Part of a row: maximum (-FLT_MAX where there is none), sum of exp(z - maximum); greedy: its argmax.
struct Part {
  float m = -FLT_MAX, s = 0.f, best = -INFINITY;
  int i = INT_MAX;
  __device__ __forceinline__ void take(float ov, int oi) {
    if (ov > best || (ov == best && oi < i)) {
      best = ov;
      i = oi;
    }
  }
};

constexpr int kRounds = 4;  // slices of a warp, where there are not many more warps than rows
constexpr int kMaxSlices = kMaxRows / kWarps + 1;
static_assert(kMaxSlices >= kRounds, "a warp's slices");

struct Shared {
  Part part[kWarps][kMaxSlices];  // read by the cluster
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
    if (top > p.best || p.i == INT_MAX)
#pragma unroll
      for (int e = 0; e < N; ++e) p.take(x[e], first + e);
  }
  const float now = fmaxf(p.m, top);
  p.s *= exp_fast(p.m - now);
  p.m = now;
#pragma unroll
  for (int e = 0; e < N; ++e) p.s += exp_fast(x[e] - now);
}

template <bool kArg>
__device__ __forceinline__ void merge(Part& p, const Part& o) {
  if constexpr (kArg) p.take(o.best, o.i);
  const float now = fmaxf(p.m, o.m);
  p.s = p.s * exp_fast(p.m - now) + o.s * exp_fast(o.m - now);
  p.m = now;
}

template <bool kArg>
__device__ __forceinline__ Part warp_merge(Part p) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Part other;
    other.m = __shfl_xor_sync(0xffffffffu, p.m, o);
    other.s = __shfl_xor_sync(0xffffffffu, p.s, o);
    if constexpr (kArg) {
      other.best = __shfl_xor_sync(0xffffffffu, p.best, o);
      other.i = __shfl_xor_sync(0xffffffffu, p.i, o);
    }
    merge<kArg>(p, other);
  }
  return p;
}

// [lo, hi) of a row by a warp, kDeep vectors a lane on their way.
template <typename T, bool kArg, int kDeep>
__device__ __forceinline__ Part scan(const T* row, int lo, int hi, int lane) {
  constexpr int E = 16 / sizeof(T);
  Part p;
  const int off = static_cast<int>((reinterpret_cast<uintptr_t>(row + lo) & 15) / sizeof(T));
  const int head = min(off == 0 ? 0 : E - off, hi - lo);
  const int vecs = (hi - lo - head) / E, body = lo + head;
  if (lane < head) {
    const float x[1] = {to_f(row[lo + lane])};
    add<kArg>(p, x, lo + lane);
  }
  const uint4* at = reinterpret_cast<const uint4*>(row + body);
  int v = lane;
#pragma unroll 1
  for (; v + 32 * (kDeep - 1) < vecs; v += 32 * kDeep) {
    uint4 raw[kDeep];
#pragma unroll
    for (int d = 0; d < kDeep; ++d) raw[d] = at[v + 32 * d];
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      float x[E];
      unpack<T>(raw[d], x);
      add<kArg>(p, x, body + (v + 32 * d) * E);
    }
  }
  uint4 raw[kDeep];
#pragma unroll
  for (int d = 0; d < kDeep; ++d)
    if (v + 32 * d < vecs) raw[d] = at[v + 32 * d];
#pragma unroll
  for (int d = 0; d < kDeep; ++d)
    if (v + 32 * d < vecs) {
      float x[E];
      unpack<T>(raw[d], x);
      add<kArg>(p, x, body + (v + 32 * d) * E);
    }
  const int tail = body + vecs * E + lane;
  if (tail < hi) {
    const float x[1] = {to_f(row[tail])};
    add<kArg>(p, x, tail);
  }
  return warp_merge<kArg>(p);
}

// (the address of `local` in another CTA)
__device__ __forceinline__ float ld_cluster(const float* local, unsigned rank) { return ld_cluster_f32(local, rank); }
__device__ __forceinline__ int ld_cluster(const int* local, unsigned rank) {
  return __float_as_int(ld_cluster_f32(reinterpret_cast<const float*>(local), rank));
}

// kAlone: a CTA has an SM for itself, and twice the loads on their way.
template <typename T, bool kGreedy, bool kAlone>
__global__ void __launch_bounds__(kThreads, kAlone ? 1 : 2) verify_kernel(const VerifyArgs p, int cs) {
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
  auto row_at = [&](int r) { return r <= n ? target + r * p.ld : draft + (r - n - 1) * p.ld_draft; };

  // a draft's token and its logits (lane: draft), on their way while the sums are made
  int x = -1;
  float zx = 0.f, wx = 0.f, u = 0.f;
  if (warp == 0 && lane < n) {
    x = p.ids[s * D + lane];
    if (!kGreedy) u = p.uniform[s * D + lane];
    if (x >= 0 && x < V) {
      zx = to_f(target[lane * p.ld + x]);
      if (draft != nullptr) wx = to_f(draft[lane * p.ld_draft + x]);
    }
  }

  // slices of a row: one for a warp of the cluster, or kRounds where they would not come out even, with all drafts there
  const int warps = cs * kWarps, most = p.draft != nullptr ? 2 * D + 1 : D + 1;
  const int slices = max(1, (warps >= 8 * most ? warps : kRounds * warps) / most);
  for (int i = rank * kWarps + warp, k = 0; i < rows * slices; i += warps, ++k) {
    const int r = i / slices, j = i - r * slices;
    const int lo = static_cast<int>(static_cast<long long>(V) * j / slices), hi = static_cast<int>(static_cast<long long>(V) * (j + 1) / slices);
    const Part part = scan<T, kGreedy, kAlone ? 8 : 4>(row_at(r), lo, hi, lane);
    if (lane == 0) sh.part[warp][k] = part;
  }
  if (cs > 1) cluster_sync_all(); else __syncthreads();
  // a warp a row, a lane a slice of it
  for (int r = warp; r < rows; r += kWarps) {
    Part all;
    for (int j = lane; j < slices; j += 32) {
      const int i = r * slices + j, w = i % warps;
      const Part* from = &sh.part[w % kWarps][i / warps];
      Part o;
      const int c = w / kWarps;
      o.m = c == rank ? from->m : ld_cluster(&from->m, c);
      o.s = c == rank ? from->s : ld_cluster(&from->s, c);
      if (kGreedy) {
        o.best = c == rank ? from->best : ld_cluster(&from->best, c);
        o.i = c == rank ? from->i : ld_cluster(&from->i, c);
      }
      merge<kGreedy>(all, o);
    }
    all = warp_merge<kGreedy>(all);
    if (lane == 0) {
      // a row of nothing but -inf: its sum is 0
      sh.m[r] = all.s == 0.f ? -INFINITY : all.m;
      sh.c[r] = all.s == 0.f ? 0.f : logf(all.s);
      sh.top[r] = all.i == INT_MAX ? 0 : all.i;  // (nothing but NaN)
    }
  }
  __syncthreads();

  // log-probability of logit z in row r (the sums are in fp32; what is made of them here in 64 bits)
  auto log_p = [&](float z, int r) { return static_cast<double>(z) - sh.m[r] - sh.c[r]; };
  if (warp == 0) {
    float a = 0.f;
    bool keep = false;
    if (lane < n) {
      if (x < 0 || x >= V) {
        a = __int_as_float(0x7fffffff);
        if (rank == 0) record_error(p.err, kDevBadTokenId);
      } else if (kGreedy) {
        keep = sh.top[lane] == x;
        a = keep ? 1.f : 0.f;
      } else {
        if (sh.m[lane] == -INFINITY || zx == -INFINITY) {
          a = 0.f;
        } else {
          double d = log_p(zx, lane);
          if (draft != nullptr) d = sh.m[n + 1 + lane] == -INFINITY ? INFINITY : d - log_p(wx, n + 1 + lane);
          a = d >= 0.0 ? 1.f : expf(static_cast<float>(d));
        }
        keep = u < a;
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
  float next_z = 0.f;

  if constexpr (!kGreedy) {
    const float* noise = p.gumbel + s * p.ld_gumbel;
    const bool refused = kept < n;
    const T* q = refused && draft != nullptr ? draft + kept * p.ld_draft : nullptr;
    const int gone = refused ? p.ids[s * D + kept] : -1;
    const float pm = sh.m[kept], pc = sh.c[kept];
    const float qm = q != nullptr ? sh.m[n + 1 + kept] : 0.f, qc = q != nullptr ? sh.c[n + 1 + kept] : 0.f;
    Best rest, whole;
    const int mine = (V + cs - 1) / cs, from = min(V, rank * mine), to = min(V, from + mine);
    constexpr int kDeep = 8;  // of a thread, on their way (rows start anywhere: element by element)
    // log r is at most log p: where that does not reach the warp's best so far, r is not worked out (it takes as long as all
    // else). The slack covers the roundings of the bound.
    float reach = -INFINITY;
#pragma unroll 1
    for (int first = from + (threadIdx.x & ~31); first < to; first += kThreads * kDeep) {
      float z[kDeep], g[kDeep], w[kDeep];
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        const int v = first + lane + kThreads * i;
        z[i] = v < to ? to_f(last[v]) : -INFINITY;
        g[i] = v < to ? noise[v] : 0.f;
        w[i] = q != nullptr && v < to ? to_f(q[v]) : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        const int v = first + lane + kThreads * i;
        const float t = z[i] + g[i];
        if (v < to) whole.take(t, v, z[i]);
        if (q != nullptr) {
          if (t - pm - pc + 1e-3f + 1e-6f * (fabsf(t) + fabsf(pm)) > reach) {  // (not in a row's end: -inf)
            const float r = expf((z[i] - pm) - pc) - (w[i] == -INFINITY ? 0.f : expf((w[i] - qm) - qc));
            if (r > 0.f) rest.take(logf(r) + g[i], v, z[i]);
          }
        } else if (refused && v != gone && z[i] > -INFINITY) {
          rest.take(t, v, z[i]);
        }
      }
      if (q != nullptr) {
        reach = rest.v;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) reach = fmaxf(reach, __shfl_xor_sync(0xffffffffu, reach, o));
      }
    }
    rest.take_lanes(32);
    whole.take_lanes(32);
    if (lane == 0) {
      sh.best[0][warp] = rest;
      sh.best[1][warp] = whole;
    }
    __syncthreads();
    if (warp < 2) {  // one each
      Best b = sh.best[warp][lane & (kWarps - 1)];
      b.take_lanes(kWarps);
      if (lane == 0) sh.cta_best[warp] = b;
    }
    if (cs > 1) cluster_sync_all(); else __syncthreads();
    if (rank == 0 && warp == 0) {
      const int c = lane & (cs - 1);
      auto of = [&](const Best& b) {
        Best o;
        o.v = c == 0 ? b.v : ld_cluster(&b.v, c);
        o.i = c == 0 ? b.i : ld_cluster(&b.i, c);
        o.z = c == 0 ? b.z : ld_cluster(&b.z, c);
        o.take_lanes(cs);
        return o;
      };
      const Best r = of(sh.cta_best[0]), all = of(sh.cta_best[1]);
      // nothing of the residual is left: from the row itself
      const Best& b = refused && r.i != INT_MAX ? r : all;
      next = b.i != INT_MAX ? b.i : 0;  // (nothing but NaN)
      next_z = b.i != INT_MAX ? b.z : to_f(last[0]);
    }
  }
  if (rank == 0 && warp == 0) {
    if constexpr (kGreedy) next_z = to_f(last[next]);
    for (int i = lane; i <= D; i += 32) {  // (lane: the draft that it has, and D beyond 31)
      const bool draft_kept = i < kept;
      p.tokens[s * (D + 1) + i] = draft_kept ? x : i == kept ? next : -1;
      if (p.logp != nullptr)
        p.logp[s * (D + 1) + i] = i > kept                ? 0.f
                                  : sh.m[i] == -INFINITY ? -INFINITY
                                                          : static_cast<float>(log_p(draft_kept ? zx : next_z, i));
    }
    if (lane == 0) p.accepted[s] = kept;
  }
  if (cs > 1) cluster_sync_all();  // nobody leaves while its memory is read
}

template <typename T, bool kGreedy>
cudaError_t launch(const VerifyArgs& a, cudaStream_t st) {
  // as many CTAs a sequence as the device holds at once, none with under 1000 tokens of a row: one an SM, or where that leaves
  // SMs idle two
  const int sms = std::max(1, sm_count());
  int cs = 1;
  while (cs < kMaxCluster && a.S * cs <= sms && a.V >= 2000 * cs) cs *= 2;
  const bool alone = a.S * cs <= sms;
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
  return alone ? cudaLaunchKernelEx(&cfg, verify_kernel<T, kGreedy, true>, a, cs)
               : cudaLaunchKernelEx(&cfg, verify_kernel<T, kGreedy, false>, a, cs);
}

}  // namespace

int launch_verify_drafts(const VerifyArgs& a, cudaStream_t st) {
  const bool greedy = a.gumbel == nullptr;
  const auto f = a.bf16 ? (greedy ? launch<__nv_bfloat16, true> : launch<__nv_bfloat16, false>)
                        : (greedy ? launch<float, true> : launch<float, false>);
  return f(a, st) == cudaSuccess ? 0 : -3;
}

}  // namespace hydra
