// Global gradient norm over many tensors, and clipping to a largest norm (the update that follows
// the gradients of §2 "Stage 3: PPO": one LoRA set is hundreds of tensors of a few KB to a few MB).
//
//     norm = sqrt(sum over all tensors and elements of g^2)
//     coef = min(1, max_norm / (norm + 1e-6)), 1 where the norm is not finite;  out = g coef
//
// Two launches: every CTA sums the squares of a contiguous range of chunks and writes one fp64
// partial; every CTA of the second pass adds all partials in the same fixed order and scales its
// range. The tensors' addresses travel as a kernel parameter, so that a captured call stands by itself.
//
// Squares are summed in fp32 over a thread's elements of a chunk and in fp64 beyond. A chunk whose
// fp32 sum leaves [2^-80, 2^120] while its elements are not all zero is summed again in fp64,
// where no square of an fp32 value overflows or vanishes.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace hydra {
namespace {

constexpr int kThreads = 256;
constexpr int kChunkBytes = 16384;
constexpr int kTableMax = 960;  // tensors of one launch: 30 KB of parameters
constexpr double kEps = 1e-6;

struct Entry {
  const void* src;
  void* dst;
  long long numel;
  int first;  // first chunk
  int bf16;
};
template <int kCap>
struct Table {
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

// A chunk's elements: [lo, hi) of its tensor, of which those of whole 16-byte vectors are [v0, v1).
template <typename T>
struct Chunk {
  static constexpr int E = 16 / sizeof(T);
  static constexpr int kElems = kChunkBytes / sizeof(T);
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

// f(value) over this thread's elements of a chunk
template <typename T, typename F>
__device__ __forceinline__ void for_each(const Chunk<T>& c, F f) {
  constexpr int E = Chunk<T>::E;
#pragma unroll
  for (int q = 0; q < kChunkBytes / 16 / kThreads; ++q) {
    const int v = threadIdx.x + q * kThreads;
    if (v < c.vecs) {
      float x[E];
      unpack<T>(*reinterpret_cast<const uint4*>(c.src + c.head + v * E), x);
#pragma unroll
      for (int e = 0; e < E; ++e) f(x[e]);
    }
  }
  // up to E - 1 elements at either end
  const int t = threadIdx.x;
  const int tail = c.head + c.vecs * E;
  if (t < c.head) f(to_f(c.src[t]));
  if (t < c.n - tail) f(to_f(c.src[tail + t]));
}

template <typename T>
__device__ __forceinline__ double square_sum(const Chunk<T>& c) {
  float s = 0.f;
  uint32_t any = 0;
  for_each(c, [&](float x) {
    s = fmaf(x, x, s);
    any |= __float_as_uint(x) << 1;
  });
  if (any == 0 || (s >= 0x1p-80f && s <= 0x1p120f)) return s;
  double d = 0.0;
  for_each(c, [&](float x) { d += static_cast<double>(x) * x; });
  return d;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) v += red[w];
  return v;
}

// the tensor that chunk c belongs to: the last one that starts at or before it (empty ones have no chunk)
template <int kCap>
__device__ __forceinline__ int find(const Table<kCap>& t, int n, int c) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (t.e[mid].first <= c) lo = mid; else hi = mid;
  }
  return lo;
}

// chunks [b chunks / grid, (b + 1) chunks / grid) of a launch
__device__ __forceinline__ int range_at(int chunks, unsigned b) {
  return static_cast<int>(static_cast<long long>(chunks) * b / gridDim.x);
}

// partial[b] = (add: +=) sum of the squares of CTA b's chunks
template <int kCap>
__global__ void __launch_bounds__(kThreads)
    grad_square_kernel(const __grid_constant__ Table<kCap> table, int n, int chunks, int add,
                       double* __restrict__ partial) {
  __shared__ double red[kThreads / 32];
  pdl_wait();
  pdl_launch_dependents();
  const int c0 = range_at(chunks, blockIdx.x), c1 = range_at(chunks, blockIdx.x + 1);
  double sum = 0.0;
  for (int c = c0, i = find(table, n, c0); c < c1; ++c) {
    while (i + 1 < n && table.e[i + 1].first <= c) ++i;
    const Entry& e = table.e[i];
    sum += e.bf16 ? square_sum(Chunk<__nv_bfloat16>(e, c)) : square_sum(Chunk<float>(e, c));
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + sum : sum;
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

template <typename T>
__device__ __forceinline__ void scale_chunk(const Entry& e, int ci, float coef) {
  constexpr int E = Chunk<T>::E;
  const Chunk<T> c(e, ci);
  T* dst = static_cast<T*>(e.dst) + (c.src - static_cast<const T*>(e.src));
  const int t = threadIdx.x;
  if (((reinterpret_cast<uintptr_t>(dst) ^ reinterpret_cast<uintptr_t>(c.src)) & 15) == 0) {
#pragma unroll
    for (int q = 0; q < kChunkBytes / 16 / kThreads; ++q) {
      const int v = t + q * kThreads;
      if (v < c.vecs)
        *reinterpret_cast<uint4*>(dst + c.head + v * E) =
            scaled<T>(*reinterpret_cast<const uint4*>(c.src + c.head + v * E), coef);
    }
    const int tail = c.head + c.vecs * E;
    if (t < c.head) dst[t] = scaled(c.src[t], coef);
    if (t < c.n - tail) dst[tail + t] = scaled(c.src[tail + t], coef);
  } else {
    for (int i = t; i < c.n; i += kThreads) dst[i] = scaled(c.src[i], coef);
  }
}

__device__ __forceinline__ double norm_of(const double* partial, int n, double* red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) s += partial[i];
  return sqrt(block_sum(s, red));
}
__device__ __forceinline__ float coef_of(double norm, float max_norm) {
  if (!isfinite(norm)) return 1.f;
  return static_cast<float>(fmin(1.0, static_cast<double>(max_norm) / (norm + kEps)));
}

template <int kCap>
__global__ void __launch_bounds__(kThreads)
    grad_scale_kernel(const __grid_constant__ Table<kCap> table, int n, int chunks,
                      const double* __restrict__ partial, int n_partials, float max_norm,
                      float* __restrict__ norm_out) {
  __shared__ double red[kThreads / 32];
  pdl_wait();
  pdl_launch_dependents();
  const double norm = norm_of(partial, n_partials, red);
  const float coef = coef_of(norm, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0 && norm_out != nullptr) {
    norm_out[0] = static_cast<float>(norm);
    norm_out[1] = coef;
  }
  const int c0 = range_at(chunks, blockIdx.x), c1 = range_at(chunks, blockIdx.x + 1);
  for (int c = c0, i = find(table, n, c0); c < c1; ++c) {
    while (i + 1 < n && table.e[i + 1].first <= c) ++i;
    const Entry& e = table.e[i];
    if (coef == 1.f && e.dst == e.src) continue;  // nothing changes
    if (e.bf16) scale_chunk<__nv_bfloat16>(e, c, coef); else scale_chunk<float>(e, c, coef);
  }
}

__global__ void __launch_bounds__(kThreads)
    grad_norm_kernel(const double* __restrict__ partial, int n, float max_norm, float* __restrict__ norm_out) {
  __shared__ double red[kThreads / 32];
  pdl_wait();
  pdl_launch_dependents();
  const double norm = norm_of(partial, n, red);
  if (threadIdx.x == 0) {
    norm_out[0] = static_cast<float>(norm);
    norm_out[1] = coef_of(norm, max_norm);
  }
}

int grid_of(int64_t chunks) {
  const int64_t most = std::min(kGradMaxBlocks, std::max(1, 4 * sm_count()));
  return static_cast<int>(std::min(std::max<int64_t>(chunks, 1), most));
}

// One launch's part of the list: up to kTableMax tensors from `i` on, and under 2^31 chunks.
struct Part {
  Table<kTableMax> table;
  int n = 0, chunks = 0;
  int64_t next;
  Part(const GradTensor* t, int64_t count, int64_t i) {
    for (; i < count && n < kTableMax; ++i) {
      if (t[i].numel == 0) continue;
      const int64_t elems = kChunkBytes / (t[i].bf16 ? 2 : 4);
      const int64_t c = (t[i].numel + elems - 1) / elems;
      if (chunks + c >= (1LL << 31)) break;
      table.e[n++] = Entry{t[i].grad, t[i].out, t[i].numel, chunks, t[i].bf16};
      chunks += static_cast<int>(c);
    }
    next = i;
  }
};

}  // namespace

size_t grad_norm_workspace_bytes() { return sizeof(double) * kGradMaxBlocks; }

int launch_grad_norm(const GradTensor* t, int64_t n, float max_norm, float* norm_out, bool scale, void* ws,
                     cudaStream_t st) {
  double* partial = static_cast<double*>(ws);
  int n_partials = 0;
  for (int64_t i = 0; i < n;) {
    const Part p(t, n, i);
    const bool only = i == 0 && p.next == n;
    i = p.next;
    if (p.n == 0) break;
    // a list of several launches: each adds to the partials of the one before it
    const int grid = grid_of(only ? p.chunks : INT64_MAX);
    if (launch_pdl(grad_square_kernel<kTableMax>, dim3(grid), dim3(kThreads), 0, st, p.table, p.n, p.chunks,
                   static_cast<int>(n_partials != 0), partial) != cudaSuccess)
      return -3;
    n_partials = grid;
  }
  if (!scale || n_partials == 0)
    return launch_pdl(grad_norm_kernel, dim3(1), dim3(kThreads), 0, st, static_cast<const double*>(partial),
                      n_partials, max_norm, norm_out) == cudaSuccess
               ? 0
               : -3;
  bool first = true;
  for (int64_t i = 0; i < n;) {
    const Part p(t, n, i);
    i = p.next;
    if (p.n == 0) break;
    if (launch_pdl(grad_scale_kernel<kTableMax>, dim3(grid_of(p.chunks)), dim3(kThreads), 0, st, p.table, p.n,
                   p.chunks, static_cast<const double*>(partial), n_partials, max_norm,
                   first ? norm_out : static_cast<float*>(nullptr)) != cudaSuccess)
      return -3;
    first = false;
  }
  return 0;
}

}  // namespace hydra
