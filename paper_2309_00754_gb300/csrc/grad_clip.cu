// Global gradient norm over many tensors, and clipping to a largest norm (the update that follows
// the gradients of §2 "Stage 3: PPO": one LoRA set is hundreds of tensors of a few KB to a few MB).
//
//     norm = sqrt(sum over all tensors and elements of g^2)
//     coef = min(1, max_norm / (norm + 1e-6)), 1 where the norm is not finite;  out = g coef
//
// Two launches: every CTA sums the squares of a contiguous range of chunks and writes one
// partial sum; every CTA of the second pass adds all partials in the same fixed order and scales its
// range, from its end, whose chunks L2 still holds. The tensors' addresses travel as a kernel parameter, so
// that a captured call stands by itself.
//
// Squares are summed in fp32 over a thread's elements of a chunk, and these sums as pairs of fp32 numbers with
// their rounding errors (Knuth 1969): fp64 runs at a sixty-fourth of the fp32 rate here (393 chunks of fp32: 21 us
// with fp64 sums over CTAs). A chunk whose fp32 sum leaves [2^-80, 2^90] while its elements are not all
// zero is summed again in fp64, where no square of an fp32 value overflows or vanishes, and only then is anything
// beyond it done in fp64.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace hydra {
namespace {

constexpr int kThreads = 256;
constexpr int kCtasPerSm = 4;  // (two: 205 MB of fp32 103 us, six 140, eight 163, for 94)
// Chunks of 16 KB, of a large list 32 KB. Small / large, us in a graph, 20 tensors, fp32 and bf16: 50 MB 24.6 / 25.8 and
// 25.5 / 28.1, 100 MB 47.8 / 48.6 and 49.5 / 51.3, 130 MB 62.1 / 61.9 and 65.5 / 64.4, 155 MB 74.5 / 72.8 and 78.9 / 76.1,
// 205 MB 97.9 / 96.9 and 104.4 / 99.6; 400 tensors cross at the same size. The large ones are scaled by two CTAs an SM at a
// time (registers; held to 64 of them 126 us for 205 MB).
constexpr int kChunkSmall = 16384, kChunkLarge = 32768;
constexpr int64_t kLargeBytes = 120 << 20;
// Of a longer list the last of every CTA's range, where the second pass begins, is to stay in L2; the rest and the outputs
// leave it first (102 MB of fp32 53 -> 49 us, 205 MB 110 -> 94, 822 MB 411 -> 376; 16 or 32 MB of it 53, 99 and 96, 376).
constexpr int kKeepBytes = 64 << 20;
constexpr int kTableMax = 880;  // tensors of one launch: 30 KB of parameters
constexpr float kEps = 1e-6f, kEpsLo = static_cast<float>(1e-6 - static_cast<double>(kEps));

struct Entry {
  const void* src;
  void* dst;
  long long numel;
  int first;  // first chunk
  int bf16;
};
// A launch's parameters. A search for a CTA's first tensor would be a chain of constant-cache misses.
template <int kCap>
struct Table {
  uint16_t start[kGradMaxBlocks];  // of each CTA, the tensor of its first chunk
  Entry e[kCap];
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A chunk's elements, from `src` on.
template <typename T, int kBytes>
struct Chunk {
  static constexpr int E = 16 / sizeof(T);
  static constexpr int kElems = kBytes / sizeof(T);
  static constexpr int kVecs = kBytes / 16 / kThreads;  // of a thread in a whole chunk
  const T* src;
  int n, head, vecs;  // elements, elements before the first vector, vectors
  __device__ __forceinline__ Chunk(const Entry& e, int c) {
    const long long lo = static_cast<long long>(c - e.first) * kElems;
    src = static_cast<const T*>(e.src) + lo;
    n = static_cast<int>(min(e.numel - lo, static_cast<long long>(kElems)));
    const int off = static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
    head = min(off == 0 ? 0 : E - off, n);
    vecs = (n - head) / E;
  }
};

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

// (not volatile: then the compiler holds them in registers that the loads want)
__device__ __forceinline__ uint64_t policy_first() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t policy_normal() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint4 load16(const void* p, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p), "l"(policy)
               : "memory");
  return v;
}
__device__ __forceinline__ void store16(void* p, const uint4& v, uint64_t policy) {
  asm volatile("st.global.L2::cache_hint.v4.u32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z),
               "r"(v.w), "l"(policy)
               : "memory");
}

// A sum hi + lo, exact to twice the bits of fp32; the order of two does not change what they add up to.
struct Sum {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float v, float v_lo) {
    const float sum = hi + v, part = sum - hi;
    lo = (lo + v_lo) + ((hi - (sum - part)) + (v - part));
    hi = sum;
  }
};

// A thread's sum of squares, and those that would not do in fp32.
struct Squares {
  Sum sum;
  double d = 0.0;

  template <typename T, int kBytes>
  __device__ __forceinline__ void add(const Chunk<T, kBytes>& c, uint64_t policy) {
    constexpr int E = 16 / sizeof(T), kVecs = Chunk<T, kBytes>::kVecs;
    const int t = threadIdx.x, tail = c.head + c.vecs * E;
    uint4 v[kVecs];
    float ends[2] = {0.f, 0.f};  // up to E - 1 elements at either end
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
      v[q] = make_uint4(0, 0, 0, 0);
      if (t + q * kThreads < c.vecs) v[q] = load16(c.src + c.head + (t + q * kThreads) * E, policy);
    }
    if (t < c.head) ends[0] = to_f(c.src[t]);
    if (t < c.n - tail) ends[1] = to_f(c.src[tail + t]);
    float s = ends[0] * ends[0] + ends[1] * ends[1];
    uint32_t any = __float_as_uint(ends[0]) | __float_as_uint(ends[1]);
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
      float x[E];
      unpack<T>(v[q], x);
#pragma unroll
      for (int e = 0; e < E; ++e) s = fmaf(x[e], x[e], s);
      any |= v[q].x | v[q].y | v[q].z | v[q].w;
    }
    const uint32_t signs = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
    if ((any & ~signs) == 0 || (s >= 0x1p-80f && s <= 0x1p90f)) {
      sum.add(s, 0.f);
      return;
    }
    d += static_cast<double>(ends[0]) * ends[0] + static_cast<double>(ends[1]) * ends[1];
#pragma unroll 1
    for (int q = 0; q < kVecs; ++q) {
      if (t + q * kThreads >= c.vecs) break;
      const T* p = c.src + c.head + (t + q * kThreads) * E;
#pragma unroll 1
      for (int e = 0; e < E; ++e) d += static_cast<double>(to_f(p[e])) * to_f(p[e]);
    }
  }
};

// A CTA's sum, or another part of it: `d` is 0 but where fp32 would not do.
struct alignas(16) Partial {
  Sum sum;
  double d;
};

struct BlockShared {
  Sum sum[kThreads / 32];
  double d[kThreads / 32];
};
// The threads' parts added up, in every thread; their order is fixed.
__device__ __forceinline__ Partial block_sum(Sum s, double d, BlockShared& sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
    s.add(__shfl_xor_sync(0xffffffffu, s.hi, off), __shfl_xor_sync(0xffffffffu, s.lo, off));
  if (lane == 0) sh.sum[warp] = s;
  const bool wide = __syncthreads_or(__double_as_longlong(d) != 0);
  Partial r{sh.sum[0], 0.0};
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) r.sum.add(sh.sum[w].hi, sh.sum[w].lo);
  if (wide) {
    for (int off = 16; off > 0; off >>= 1) d += __shfl_xor_sync(0xffffffffu, d, off);
    if (lane == 0) sh.d[warp] = d;
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w) r.d += sh.d[w];
  }
  return r;
}

// chunks [b chunks / grid, (b + 1) chunks / grid) of a launch
__device__ __forceinline__ int range_at(int chunks, unsigned b) {
  return static_cast<int>(static_cast<long long>(chunks) * b / gridDim.x);
}

// partial[b] = (add: +=) sum of the squares of CTA b's chunks
template <int kCap, int kBytes>
__global__ void __launch_bounds__(kThreads)
    grad_square_kernel(const __grid_constant__ Table<kCap> table, int n, int chunks, int add,
                       Partial* __restrict__ partial) {
  __shared__ BlockShared sh;
  const int c0 = range_at(chunks, blockIdx.x), c1 = range_at(chunks, blockIdx.x + 1);
  int i = table.start[blockIdx.x];
  pdl_wait();
  pdl_launch_dependents();
  Squares squares;
  const int keep = kKeepBytes / kBytes / gridDim.x;
  const uint64_t first = policy_first();
  for (int c = c0; c < c1; ++c) {
    while (i + 1 < n && table.e[i + 1].first <= c) ++i;
    const Entry& e = table.e[i];
    const uint64_t policy = c >= c1 - keep ? policy_normal() : first;
    if (e.bf16) squares.add(Chunk<__nv_bfloat16, kBytes>(e, c), policy); else squares.add(Chunk<float, kBytes>(e, c), policy);
  }
  Partial p = block_sum(squares.sum, squares.d, sh);
  if (threadIdx.x == 0) {
    if (add) {
      const Partial before = partial[blockIdx.x];
      p.sum.add(before.sum.hi, before.sum.lo);
      p.d += before.d;
    }
    partial[blockIdx.x] = p;
  }
}

// A coefficient of 1 copies: a product would give NaN another bit pattern.
template <typename T>
__device__ __forceinline__ T scaled(T v, float coef) {
  return coef == 1.f ? v : from_f<T>(to_f(v) * coef);
}
template <typename T>
__device__ __forceinline__ uint4 scaled(const uint4& v, float coef) {
  if (coef == 1.f) return v;
  float x[16 / sizeof(T)];
  unpack<T>(v, x);
  if constexpr (sizeof(T) == 4)
    return make_uint4(__float_as_uint(x[0] * coef), __float_as_uint(x[1] * coef), __float_as_uint(x[2] * coef),
                      __float_as_uint(x[3] * coef));
  else
    return make_uint4(pack_bf16x2(x[0] * coef, x[1] * coef), pack_bf16x2(x[2] * coef, x[3] * coef),
                      pack_bf16x2(x[4] * coef, x[5] * coef), pack_bf16x2(x[6] * coef, x[7] * coef));
}

template <typename T, int kBytes>
__device__ __forceinline__ void scale_chunk(const Entry& e, int ci, float coef) {
  constexpr int E = 16 / sizeof(T), kVecs = Chunk<T, kBytes>::kVecs;
  const Chunk<T, kBytes> c(e, ci);
  T* dst = static_cast<T*>(e.dst) + (c.src - static_cast<const T*>(e.src));
  const int t = threadIdx.x;
  if (((reinterpret_cast<uintptr_t>(dst) ^ reinterpret_cast<uintptr_t>(c.src)) & 15) == 0) {
    uint4 x[kVecs];
#pragma unroll
    for (int q = 0; q < kVecs; ++q)
      if (t + q * kThreads < c.vecs) x[q] = load16(c.src + c.head + (t + q * kThreads) * E, policy_first());
#pragma unroll
    for (int q = 0; q < kVecs; ++q)
      if (t + q * kThreads < c.vecs)
        store16(dst + c.head + (t + q * kThreads) * E, scaled<T>(x[q], coef), policy_first());
    const int tail = c.head + c.vecs * E;
    if (t < c.head) dst[t] = scaled(c.src[t], coef);
    if (t < c.n - tail) dst[tail + t] = scaled(c.src[tail + t], coef);
  } else {
    for (int i = t; i < c.n; i += kThreads) dst[i] = scaled(c.src[i], coef);
  }
}

struct Norm {
  float norm, coef;
};
// The root of a sum and the coefficient, each rounded once at the end: the residuals of root, sum and quotient are
// taken along as second terms (Dekker 1971, "A floating-point technique for extending the available precision"). In fp32 as
// it is, the coefficient, and every clipped value with it, would be off by more than half a step; fp64 takes longer
// than a small list. (The second terms' own quotients want few bits: __fdividef, 0.05 us of a small list's 3.9 less.)
__device__ __forceinline__ Norm norm_of(const Sum& s, float max_norm) {
  const float sum = s.hi + s.lo;
  const float root = sqrtf(sum), rest = (s.hi - sum) + s.lo;  // 0 or in [2^-40, 2^63]: nothing below vanishes
  const float root_lo = sum == 0.f ? 0.f : __fdividef(fmaf(-root, root, sum) + rest, 2.f * root);
  const float norm = root + root_lo;
  const float d = root + kEps, part = d - root;  // root + eps = d + d_lo
  const float d_lo = ((root - (d - part)) + (kEps - part)) + (root_lo + kEpsLo);
  const float q = max_norm / d;
  if (!(q < 2.f)) return Norm{norm, 1.f};
  return Norm{norm, fminf(1.f, q + __fdividef(fmaf(-q, d, max_norm) - q * d_lo, d))};
}
__device__ __forceinline__ Norm norm_of(const Partial* partial, int n, float max_norm, BlockShared& sh) {
  Sum s;
  double d = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const Partial p = partial[i];
    s.add(p.sum.hi, p.sum.lo);
    if (__double_as_longlong(p.d) != 0) d += p.d;
  }
  const Partial all = block_sum(s, d, sh);
  if (__double_as_longlong(all.d) == 0) return norm_of(all.sum, max_norm);
  const double norm = sqrt(all.d + all.sum.hi + all.sum.lo);
  return Norm{static_cast<float>(norm),
              isfinite(norm) ? static_cast<float>(fmin(1.0, max_norm / (norm + 1e-6))) : 1.f};
}

template <int kCap, int kBytes>
__global__ void __launch_bounds__(kThreads)
    grad_scale_kernel(const __grid_constant__ Table<kCap> table, int n, int chunks,
                      const Partial* __restrict__ partial, int n_partials, float max_norm,
                      float* __restrict__ norm_out) {
  __shared__ BlockShared sh;
  const int c0 = range_at(chunks, blockIdx.x), c1 = range_at(chunks, blockIdx.x + 1);
  // from the range's end: the last of its tensors is found while the sums are under way
  int i = table.start[blockIdx.x];
  while (i + 1 < n && table.e[i + 1].first < c1) ++i;
  pdl_wait();
  pdl_launch_dependents();
  const Norm r = norm_of(partial, n_partials, max_norm, sh);
  if (blockIdx.x == 0 && threadIdx.x == 0 && norm_out != nullptr) {
    norm_out[0] = r.norm;
    norm_out[1] = r.coef;
  }
  for (int c = c1 - 1; c >= c0; --c) {
    while (table.e[i].first > c) --i;
    const Entry& e = table.e[i];
    if (r.coef == 1.f && e.dst == e.src) continue;  // nothing changes
    if (e.bf16) scale_chunk<__nv_bfloat16, kBytes>(e, c, r.coef); else scale_chunk<float, kBytes>(e, c, r.coef);
  }
}

__global__ void __launch_bounds__(kThreads)
    grad_norm_kernel(const Partial* __restrict__ partial, int n, float max_norm, float* __restrict__ norm_out) {
  __shared__ BlockShared sh;
  pdl_wait();
  pdl_launch_dependents();
  const Norm r = norm_of(partial, n, max_norm, sh);
  if (threadIdx.x == 0) {
    norm_out[0] = r.norm;
    norm_out[1] = r.coef;
  }
}

int grid_of(int64_t chunks) {
  const int64_t most = std::min(kGradMaxBlocks, kCtasPerSm * std::max(1, sm_count()));
  return static_cast<int>(std::min(std::max<int64_t>(chunks, 1), most));
}

// One launch's part of the list: up to kTableMax tensors from `i` on, and under 2^31 chunks, for a grid of CTAs.
struct ListPart {
  Table<kTableMax> table;
  int n = 0, chunks = 0, grid = 0;
  int64_t next;
  ListPart(const GradTensor* t, int64_t count, int64_t i, int chunk_bytes) {
    for (; i < count && n < kTableMax; ++i) {
      const int64_t elems = chunk_bytes / (t[i].bf16 ? 2 : 4);
      const int64_t c = (t[i].numel + elems - 1) / elems;
      if (chunks + c >= (1LL << 31)) break;
      table.e[n++] = Entry{t[i].grad, t[i].out, t[i].numel, chunks, t[i].bf16};
      chunks += static_cast<int>(c);
    }
    next = i;
  }
  // the first tensor of each CTA's range; range_at without a division a CTA
  void deal(int ctas) {
    grid = ctas;
    const int each = chunks / grid, rest = chunks % grid;
    for (int b = 0, c = 0, part = 0, i = 0; b < grid; ++b) {
      while (i + 1 < n && table.e[i + 1].first <= c) ++i;
      table.start[b] = static_cast<uint16_t>(i);
      c += each;
      part += rest;
      if (part >= grid) {
        part -= grid;
        ++c;
      }
    }
  }
  // Table<kCap>'s layout is the front of every larger one's
  template <int kCap>
  const Table<kCap>& parameters() const { return *reinterpret_cast<const Table<kCap>*>(&table); }
};

template <int kCap, int kBytes>
cudaError_t launch_square(const ListPart& p, bool add, Partial* partial, cudaStream_t st) {
  return launch_pdl(grad_square_kernel<kCap, kBytes>, dim3(p.grid), dim3(kThreads), 0, st, p.parameters<kCap>(), p.n,
                    p.chunks, static_cast<int>(add), partial);
}
template <int kCap, int kBytes>
cudaError_t launch_scale(const ListPart& p, const Partial* partial, int n_partials, float max_norm, float* norm_out,
                         cudaStream_t st) {
  return launch_pdl(grad_scale_kernel<kCap, kBytes>, dim3(p.grid), dim3(kThreads), 0, st, p.parameters<kCap>(), p.n,
                    p.chunks, partial, n_partials, max_norm, norm_out);
}
// A launch carries a table of 32, 224 or 880 tensors: it is copied twice on its way, in full. A call's enqueueing of 20 / 100
// / 194 tensors takes 7.5 / 9.3 / 10.7 us so, 9.5 / 10.7 / 12.3 with the table of 880 alone; the kernels take the same.
// 224 hold the LoRA gradients of 32 layers (six a layer) and some more.
constexpr int kTableSmall = 32, kTableMiddle = 224;

}  // namespace

size_t grad_norm_workspace_bytes() { return sizeof(Partial) * kGradMaxBlocks; }

int launch_grad_norm(const GradTensor* t, int64_t n, float max_norm, float* norm_out, bool scale, void* ws,
                     cudaStream_t st) {
  Partial* partial = static_cast<Partial*>(ws);
  int64_t bytes = 0;
  for (int64_t i = 0; i < n; ++i) bytes += t[i].numel * (t[i].bf16 ? 2 : 4);
  const bool large = bytes >= kLargeBytes;
  const int chunk_bytes = large ? kChunkLarge : kChunkSmall;
  int n_partials = 0;
  ListPart p(t, n, 0, chunk_bytes);
  const bool whole = p.next == n;  // then both launches take the same part
  for (int64_t i = 0; i < n; i = p.next) {
    if (i > 0) p = ListPart(t, n, i, chunk_bytes);
    // a list of several launches: each adds to the partials of the one before it
    p.deal(grid_of(whole ? p.chunks : INT64_MAX));
    const auto launch = large ? (p.n <= kTableMiddle ? launch_square<kTableMiddle, kChunkLarge>
                                                     : launch_square<kTableMax, kChunkLarge>)
                        : p.n <= kTableSmall  ? launch_square<kTableSmall, kChunkSmall>
                        : p.n <= kTableMiddle ? launch_square<kTableMiddle, kChunkSmall>
                                              : launch_square<kTableMax, kChunkSmall>;
    if (launch(p, i > 0, partial, st) != cudaSuccess) return -3;
    n_partials = p.grid;
  }
  if (!scale || n == 0)
    return launch_pdl(grad_norm_kernel, dim3(1), dim3(kThreads), 0, st, static_cast<const Partial*>(partial),
                      n_partials, max_norm, norm_out) == cudaSuccess
               ? 0
               : -3;
  for (int64_t i = 0; i < n; i = p.next) {
    if (!whole) {
      p = ListPart(t, n, i, chunk_bytes);
      p.deal(grid_of(p.chunks));
    }
    const auto launch = large ? (p.n <= kTableMiddle ? launch_scale<kTableMiddle, kChunkLarge>
                                                     : launch_scale<kTableMax, kChunkLarge>)
                        : p.n <= kTableSmall  ? launch_scale<kTableSmall, kChunkSmall>
                        : p.n <= kTableMiddle ? launch_scale<kTableMiddle, kChunkSmall>
                                              : launch_scale<kTableMax, kChunkSmall>;
    if (launch(p, partial, n_partials, max_norm, i == 0 ? norm_out : nullptr, st) != cudaSuccess) return -3;
  }
  return 0;
}

}  // namespace hydra
