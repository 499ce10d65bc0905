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
// exchange before every one of them knows where the drafts end. (Cut alike, equal rows that start alike modulo 16 bytes have
// equal sums: a draft model that is the target is never refused.) The row that the last token is drawn from is read a second
// time, from L2 as a rule.
//
// Measured: 64 sequences of up to 4 drafts and 32,000 fp32 logits (49 MB) in 18.4 us, 2.7 TB/s: a cluster has its rows in 6 to 8
// us of that and what follows is a chain of latencies (the pairs' exchange, the second read, the exchange of what it found),
// 9 us where a single sequence is all there is.
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>

#include "common.cuh"
#include "kernels.h"

namespace hydra {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
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

constexpr int kMaxSlices = 6;  // of a warp
static_assert(kMaxSlices * kWarps >= kMaxRows, "a warp's slices");

struct alignas(16) Shared {
  Part part[kWarps][kMaxSlices];  // read by the cluster
  float m[kMaxRows], c[kMaxRows];  // of whole rows: maximum, log of the sum
  int top[kMaxRows];
  Best best[kWarps];
  Best cta_best[2];  // of the first draw, of a second; read by the cluster
  int kept;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
// (off by two units in the last place at most, and zero below 2^-126, which no sum of at least 1 sees)
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float exp_fast(float x) { return exp2_fast(x * kLog2e); }

// Largest of a vector's logits, in their own type for two at once.
template <typename T>
__device__ __forceinline__ float top_of(const uint4& v) {
  if constexpr (sizeof(T) == 4) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  } else {
    const auto h = [](const uint32_t& r) { return reinterpret_cast<const __nv_bfloat162&>(r); };
    const __nv_bfloat162 m = __hmax2(__hmax2(h(v.x), h(v.y)), __hmax2(h(v.z), h(v.w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
}

// The sum of exp(z - m) of a vector's logits, in two halves.
template <typename T>
__device__ __forceinline__ float2 exp_sum(const uint4& v, float m, float2 sum) {
  const uint32_t r[4] = {v.x, v.y, v.z, v.w};
  const float2 minus = {-m, -m}, log2e = {kLog2e, kLog2e};
  auto two = [&](float2 z) {
    const float2 e = mul2(add2(z, minus), log2e);
    sum = add2(sum, make_float2(exp2_fast(e.x), exp2_fast(e.y)));
  };
  if constexpr (sizeof(T) == 4) {
    two(make_float2(__uint_as_float(r[0]), __uint_as_float(r[1])));
    two(make_float2(__uint_as_float(r[2]), __uint_as_float(r[3])));
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) two(unpack_bf16x2(r[q]));
  }
  return sum;
}

// kN vectors more, that of x[q] from index first + q stride on. Of the largest logit only the vector is kept.
template <typename T, bool kArg, int kN>
__device__ __forceinline__ void add(Part& p, const uint4 (&x)[kN], int first, int stride) {
  float top = p.m;
#pragma unroll
  for (int q = 0; q < kN; ++q) {
    const float t = top_of<T>(x[q]);
    top = fmaxf(top, t);
    if constexpr (kArg) {
      if (t > p.best) {
        p.best = t;
        p.i = first + q * stride;
      }
    }
  }
  float2 sum = {0.f, 0.f};
#pragma unroll
  for (int q = 0; q < kN; ++q) sum = exp_sum<T>(x[q], top, sum);
  p.s = p.s * exp_fast(p.m - top) + (sum.x + sum.y);
  p.m = top;
}

template <bool kArg>
__device__ __forceinline__ void merge(Part& p, const Part& o) {
  if constexpr (kArg) p.take(o.best, o.i);
  const float now = fmaxf(p.m, o.m);
  p.s = p.s * exp_fast(p.m - now) + o.s * exp_fast(o.m - now);
  p.m = now;
}

template <bool kArg>
__device__ __forceinline__ Part warp_merge(const Part& p) {
  Part all = p;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all.m = fmaxf(all.m, __shfl_xor_sync(0xffffffffu, all.m, o));
  all.s = p.s * exp_fast(p.m - all.m);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    all.s += __shfl_xor_sync(0xffffffffu, all.s, o);
    if constexpr (kArg) {
      const float best = __shfl_xor_sync(0xffffffffu, all.best, o);
      all.take(best, __shfl_xor_sync(0xffffffffu, all.i, o));
    }
  }
  return all;
}

// A warp's slices as a stream of rounds: kVecs 16-byte vectors for each of 32 lanes, kAhead rounds on their way in a ring in
// shared memory, over the ends of slices, too. A lane reads what it put there itself: -inf behind a row's last vector.
// (Two rounds ahead: 19.9 us for the 64 sequences above, three 25.6; rounds of half the size 19.2.)
constexpr int kVecs = 4, kAhead = 1, kStages = kAhead + 1;
constexpr int kRoundVecs = kVecs * 32, kRoundBytes = kRoundVecs * 16;

// A row as 16-byte vectors, with the logits before the first of them and behind the last.
template <typename T>
struct Row {
  static constexpr int E = 16 / sizeof(T);
  const T* at;
  int head, vecs, tail;
  __device__ __forceinline__ Row(const T* row, int V) : at(row) {
    const int off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = min(off == 0 ? 0 : E - off, V);
    vecs = (V - head) / E;
    tail = V - head - vecs * E;
  }
};

template <typename T>
__device__ __forceinline__ void fetch(bool there, uint8_t* dst, const T* src) {
  constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %0, 0;\n\t@p cp.async.cg.shared.global [%1], [%2], 16;\n\t"
      "@!p st.shared.v4.b32 [%1], {%3, %3, %3, %3};\n\t}" ::"r"(static_cast<uint32_t>(there)),
      "r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(src)), "r"(kNone)
      : "memory");
}

// Slices first, first + step, ... below `total` by a warp, `slices` of `rounds` rounds a row (the last one shorter);
// done(k, part) for the k-th of them.
template <typename T, bool kArg, typename RowAt, typename Done>
__device__ __forceinline__ void scan(int first, int step, int total, int slices, int rounds, int V, uint8_t* ring, int lane,
                                     RowAt row_at, Done done) {
  constexpr int E = 16 / sizeof(T);
  ring += lane * 16;
  // what is fetched next: a round of slice `next`, from this lane's `from` with `left` vectors to the row's end
  int next = first, left = 0, ahead = 0, fill = 0;
  const T* from = nullptr;
  auto open = [&]() {
    for (ahead = 0; next < total; next += step) {
      const int r = next / slices, skip = (next - r * slices) * rounds * kRoundVecs;
      const Row<T> row(row_at(r), V);
      left = row.vecs - skip;
      ahead = min(rounds, (left + kRoundVecs - 1) / kRoundVecs);
      if (ahead > 0) {
        left -= lane;
        from = row.at + row.head + static_cast<long long>(skip + lane) * E;
        break;
      }
    }
  };
  auto produce = [&]() {
    if (ahead > 0) {
#pragma unroll
      for (int q = 0; q < kVecs; ++q) fetch(q * 32 < left, ring + fill * kRoundBytes + q * 512, from + q * 32 * E);
      from += kRoundVecs * E;
      left -= kRoundVecs;
      if (--ahead == 0) {
        next += step;
        open();
      }
    }
    fill = fill + 1 == kStages ? 0 : fill + 1;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  open();
#pragma unroll 1
  for (int i = 0; i < kAhead; ++i) produce();
  int take = 0;
#pragma unroll 1
  for (int i = first, k = 0; i < total; i += step, ++k) {
    const int r = i / slices, j = i - r * slices, skip = j * rounds * kRoundVecs;
    const Row<T> row(row_at(r), V);
    // the logits before the first vector with the first slice, those behind the last with the last
    int edge = -1;
    if (j == 0 && lane < row.head) edge = lane;
    if (j == slices - 1 && lane >= 16 && lane - 16 < row.tail) edge = V - row.tail + lane - 16;
    const float edge_z = edge >= 0 ? to_f(row.at[edge]) : -INFINITY;
    const int mine = min(rounds, (row.vecs - skip + kRoundVecs - 1) / kRoundVecs);
    Part p;
#pragma unroll 1
    for (int v = 0; v < mine; ++v) {
      produce();
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
      uint4 x[kVecs];
#pragma unroll
      for (int q = 0; q < kVecs; ++q) x[q] = *reinterpret_cast<const uint4*>(ring + take * kRoundBytes + q * 512);
      take = take + 1 == kStages ? 0 : take + 1;
      add<T, kArg>(p, x, row.head + (skip + v * kRoundVecs + lane) * E, 32 * E);
    }
    if (edge >= 0) {
      if (kArg && edge_z > -INFINITY) p.take(edge_z, edge);  // (a row of nothing else has no largest)
      const float now = fmaxf(p.m, edge_z);
      p.s = p.s * exp_fast(p.m - now) + exp_fast(edge_z - now);
      p.m = now;
    }
    done(k, warp_merge<kArg>(p));
  }
}

// (the address of `local` in another CTA)
__device__ __forceinline__ float ld_cluster(const float* local, unsigned rank) { return ld_cluster_f32(local, rank); }
__device__ __forceinline__ int ld_cluster(const int* local, unsigned rank) {
  return __float_as_int(ld_cluster_f32(reinterpret_cast<const float*>(local), rank));
}

template <typename T, bool kGreedy>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const VerifyArgs p, int cs) {
  extern __shared__ __align__(16) uint8_t raw_shared[];
  Shared& sh = *reinterpret_cast<Shared*>(raw_shared);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = cs > 1 ? static_cast<int>(cluster_rank()) : 0;
  const long long s = blockIdx.x / cs;
  const int V = static_cast<int>(p.V), D = static_cast<int>(p.D);
  // (nothing behind it is let in early: its CTAs would take the SMs that clusters are spread over; calls in a row took 26 us
  // instead of 16 with 24 sequences of 8 drafts, 30 instead of 25 with 37 of 7)
  pdl_wait();
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

  // Slices of a row: t for each of the cluster's warps, t such that they come out with the fewest rounds, a slice's end counted
  // as one (a lane a t). By the drafts that are there: cut for all D, a sequence of few leaves most warps idle.
  const int warps = cs * kWarps, all = (V + kRoundVecs * Row<T>::E - 1) / (kRoundVecs * Row<T>::E);  // rounds of a row
  const int t = lane + 1, least = max(1, t * warps / rows), mine_rounds = (all + least - 1) / least;
  const unsigned cost = t <= kMaxSlices && t * warps >= rows ? static_cast<unsigned>(t * (mine_rounds + 1)) : UINT_MAX / 2;
  const int best_t = __ffs(__ballot_sync(0xffffffffu, cost == __reduce_min_sync(0xffffffffu, cost))) - 1;
  const int rounds = __shfl_sync(0xffffffffu, mine_rounds, best_t), slices = (all + rounds - 1) / rounds;
  scan<T, kGreedy>(
      rank * kWarps + warp, warps, rows * slices, slices, rounds, V,
      raw_shared + sizeof(Shared) + warp * kStages * kRoundBytes, lane, row_at, [&](int k, const Part& part) {
        if (lane == 0) sh.part[warp][k] = part;
      });
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
    if (kGreedy && all.i != INT_MAX) {  // which one of the vector
      const int i = all.i + lane;
      all.i += __ffs(__ballot_sync(0xffffffffu, lane < 16 / static_cast<int>(sizeof(T)) && i < V && to_f(row_at(r)[min(i, V - 1)]) == all.best)) - 1;
    }
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
      } else if (isnan(sh.c[lane]) || (draft != nullptr && isnan(sh.c[n + 1 + lane]))) {
        a = __int_as_float(0x7fffffff);  // a NaN or +inf logit, which makes its row's sum NaN: refused, whatever the draft's own is
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
    const float pm = sh.m[kept], pc = sh.c[kept];
    const float qm = q != nullptr ? sh.m[n + 1 + kept] : 0.f, qc = q != nullptr ? sh.c[n + 1 + kept] : 0.f;
    const int mine = (V + cs - 1) / cs, from = min(V, rank * mine), to = min(V, from + mine);
    constexpr int kDeep = 8;  // of a thread, on their way (rows start anywhere: element by element)
    // from the residual; where nothing is left of it, once more from the row itself
    Best b;
    for (bool residual = refused;; residual = false) {
      b = Best();
      if (residual && q != nullptr) {
        // log r is at most log p: where that does not reach the warp's best so far, r is not worked out (it takes as long as
        // all else). The slack covers the roundings of the bound.
        auto bound = [&](float t) { return t - pm - pc + 1e-3f + 1e-6f * (fabsf(t) + fabsf(pm)); };
        auto draw = [&](float z, float g, float w, int v) {
          const float r = expf((z - pm) - pc) - (w == -INFINITY ? 0.f : expf((w - qm) - qc));
          if (r > 0.f) b.take(logf(r) + g, v, z);
        };
        float reach = -INFINITY;
#pragma unroll 1
        for (int first = from + (threadIdx.x & ~31); first < to; first += kThreads * kDeep) {
          float z[kDeep], g[kDeep], w[kDeep];
#pragma unroll
          for (int i = 0; i < kDeep; ++i) {
            const int v = first + lane + kThreads * i;
            z[i] = v < to ? to_f(last[v]) : -INFINITY;
            g[i] = v < to ? noise[v] : 0.f;
            w[i] = v < to ? to_f(q[v]) : -INFINITY;
          }
          // a lane's likeliest first
          float top = -INFINITY, top_z = -INFINITY, top_w = 0.f, top_g = 0.f;
          int top_i = -1;
#pragma unroll
          for (int i = 0; i < kDeep; ++i)
            if (z[i] + g[i] > top) {
              top = z[i] + g[i];
              top_z = z[i];
              top_g = g[i];
              top_w = w[i];
              top_i = i;
            }
          if (bound(top) > reach) draw(top_z, top_g, top_w, first + lane + kThreads * top_i);
          reach = fmaxf(reach, b.v);
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) reach = fmaxf(reach, __shfl_xor_sync(0xffffffffu, reach, o));
#pragma unroll
          for (int i = 0; i < kDeep; ++i)
            if (i != top_i && bound(z[i] + g[i]) > reach) draw(z[i], g[i], w[i], first + lane + kThreads * i);
        }
      } else {
        const int gone = residual ? p.ids[s * D + kept] : -1;
#pragma unroll 1
        for (int first = from + static_cast<int>(threadIdx.x); first < to; first += kThreads * kDeep) {
          float z[kDeep], g[kDeep];
#pragma unroll
          for (int i = 0; i < kDeep; ++i) {
            const int v = first + kThreads * i;
            z[i] = v < to ? to_f(last[v]) : -INFINITY;
            g[i] = v < to ? noise[v] : 0.f;
          }
#pragma unroll
          for (int i = 0; i < kDeep; ++i) {
            // (the maximum off first: beside logits of 10^5 noise would be left with steps of 1/128)
            const float score = (z[i] - pm) + g[i];
            if (const int v = first + kThreads * i; score > b.v && v != gone) {
              b.v = score;
              b.i = v;
              b.z = z[i];
            }
          }
        }
      }
      b.take_lanes(32);
      if (lane == 0) sh.best[warp] = b;
      __syncthreads();
      if (warp == 0) {
        b = sh.best[lane & (kWarps - 1)];
        b.take_lanes(kWarps);
        if (lane == 0) sh.cta_best[residual] = b;
      }
      if (cs > 1) cluster_sync_all(); else __syncthreads();
      if (residual || (rank == 0 && warp == 0)) {
        const int c = lane & (cs - 1);
        const Best& of = sh.cta_best[residual];
        b.v = c == rank ? of.v : ld_cluster(&of.v, c);
        b.i = c == rank ? of.i : ld_cluster(&of.i, c);
        b.z = c == rank ? of.z : ld_cluster(&of.z, c);
        b.take_lanes(cs);
      }
      if (!residual || b.i != INT_MAX) break;
    }
    next = b.i != INT_MAX ? b.i : 0;  // (nothing but NaN and -inf)
    next_z = b.i != INT_MAX ? b.z : to_f(last[0]);
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

constexpr int kSmem = sizeof(Shared) + kWarps * kStages * kRoundBytes;

cudaLaunchConfig_t config(int64_t clusters, int cs, cudaStream_t st, cudaLaunchAttribute (&attr)[2]) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(clusters * cs));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(cs);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cfg;
}

// Clusters of 1 << bits CTAs that the device holds at once (0: none, or it does not say, which is not kept).
template <typename T, bool kGreedy>
int clusters_held(int dev, int bits) {
  static std::atomic<int> held[64][4];  // and one more; host threads may ask at once
  if (const int known = held[dev][bits]; known > 0) return known - 1;
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = config(1, 1 << bits, nullptr, attr);
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, verify_kernel<T, kGreedy>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  held[dev][bits] = n + 1;
  return n;
}

template <typename T, bool kGreedy>
cudaError_t launch(const VerifyArgs& a, cudaStream_t st) {
  static std::atomic<bool> attr_set[64];  // the shared-memory limit is a per-device attribute; host threads may ask at once
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess || dev < 0 || dev >= 64) return e == cudaSuccess ? cudaErrorInvalidDevice : e;
  if (!attr_set[dev]) {
    if (cudaError_t e = cudaFuncSetAttribute(verify_kernel<T, kGreedy>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); e != cudaSuccess)
      return e;
    attr_set[dev] = true;
  }
  // As many CTAs a sequence as the device holds for all at once, none with under 1000 tokens of a row (64 sequences of 4 drafts and
  // 32,000 tokens: 18.4 us by fours, 22.0 by twos, 24.9 by eights, of which 35 fit).
  int bits = 3;
  while (bits > 0 && (a.V < (1000LL << bits) || a.S > clusters_held<T, kGreedy>(dev, bits))) --bits;
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = config(a.S, 1 << bits, st, attr);
  return cudaLaunchKernelEx(&cfg, verify_kernel<T, kGreedy>, a, 1 << bits);
}

}  // namespace

int launch_verify_drafts(const VerifyArgs& a, cudaStream_t st) {
  const bool greedy = a.gumbel == nullptr;
  const auto f = a.bf16 ? (greedy ? launch<__nv_bfloat16, true> : launch<__nv_bfloat16, false>)
                        : (greedy ? launch<float, true> : launch<float, false>);
  return f(a, st) == cudaSuccess ? 0 : -3;
}

}  // namespace hydra
