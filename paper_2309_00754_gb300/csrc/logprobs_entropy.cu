// Token statistics of rows of logits and their gradient (§2 "Stage 3: PPO": the probability ratio
// needs each sampled token's log-probability, its gradient goes back into the logits).
//
// Forward, per row z of V logits, one pass with a running maximum (Milakov & Gimelshein 2018):
//     m = max z,  s = sum exp(z - m),  w = sum exp(z - m) (z - m)
//     logp = (z[id] - m) - log s,  entropy = log s - w / s
// Both terms of the entropy are at least 0; keeping m and log s apart keeps log-probabilities exact
// where |m| is large (a vocabulary masked with the type's lowest value).
//
// The rows come through a ring of 16 KB stages that one warp fills with bulk copies, rows ahead of the
// eight warps that sum them: 256 threads with a maximum and two sums each, whose parts one warp puts
// together. Four CTAs an SM take every 608th row. HBM bounds it where the logits are fp32 (4096 x 32000: 77 to 80 us,
// 97 to 101 % of the measured rate), and nearly so the 8.4 instructions an element of bf16 (8192 x 32000: 82.3 us,
// 94 %). Few rows are shared by clusters, which meet in the first CTA's memory; short ones take a warp each.
//
// The k likeliest tokens, in the order (logit descending, index ascending): every thread keeps its best
// value of each eighth of the row. A bound that k of the 256 threads reach holds for the k-th best element,
// too; the eighths that reach it, about k, are read again, and the few elements not behind it are ranked by
// counting. Three warps of a CTA do that, a row each, while the others are in the next rows, as it takes
// 3 to 8 us, most of it one step waiting for the one before. Two such CTAs fit an SM (4096 x 32000 fp32, k = 8:
// 81 us; 8192 x 32000 bf16 99; when that was 97, three CTAs of fewer registers took 113, and selection by the summing
// threads themselves 130).
//
// Backward, with p = exp((z - m) - log s):
//     dz[v] = g_logp (1[v = id] - p_v) - g_entropy p_v (log p_v + entropy)
#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "kernels.h"

namespace hydra {
namespace {

constexpr int kSummers = 256;  // threads of a CTA that sum a row; one more warp fetches it
constexpr int kWarps = kSummers / 32;
constexpr int kSlotsEach = 4;  // slots a thread takes of a stage
constexpr int kStageSlots = kSummers * kSlotsEach;
constexpr int kClusterMax = 8;
constexpr int kEvenMax = 128;     // sequences whose live rows are counted
constexpr int kEnders = 3;        // warps of a CTA that finish rows where tokens are selected
constexpr int kSegments = 8;      // of a row's stages, with a best value of each thread
constexpr int kCandidates = 252;  // elements ranked at once
constexpr float kInf = __builtin_huge_valf(), kNan = __builtin_nanf("");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// exp of anything below is 0 in fp32; a finite stand-in keeps 0 * (z - m) from being 0 * -inf
constexpr float kFloor = -256.f;

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {  // 2 ulp
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// two fp32 values an instruction
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
// v twice, kept: the compiler would build it again for every pair
__device__ __forceinline__ uint64_t twice(float v) {
  uint64_t r;
  asm volatile("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
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

// Order of logits as unsigned integers: NaN first, then descending, -0 equal to 0. No value maps to 0.
constexpr uint32_t kNanKey = 0xffffffffu;
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return kNanKey;
  const int b = __float_as_int(v + 0.f);
  return b < 0 ? ~static_cast<uint32_t>(b) : static_cast<uint32_t>(b) | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) {
  if (k == kNanKey) return kNan;
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// Whether a value's order_key is not below `least`, without working the key out.
struct AtLeast {
  float value;    // not below it
  bool nan_only;  // least is beyond +inf
  __device__ __forceinline__ explicit AtLeast(uint32_t least)
      : value(order_value(least)), nan_only(least > order_key(kInf)) {}
  __device__ __forceinline__ bool operator()(float v) const { return nan_only ? v != v : !(v < value); }
};

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
  __device__ __forceinline__ uint4 load_full(int j) const { return *reinterpret_cast<const uint4*>(p + first(j)); }
  // a slot from memory, -inf in the places before and behind the row
  __device__ __forceinline__ uint4 load(int j) const {
    if (j >= full_lo && j < full_hi) return load_full(j);
    alignas(16) T v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = first(j) + e;
      v[e] = i >= 0 && i < V ? p[i] : from_f<T>(-kInf);
    }
    return *reinterpret_cast<uint4*>(v);
  }
  __device__ static __forceinline__ void unpack(const uint4& v, float (&f)[E]) {
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (E == 4) {
        f[q] = __uint_as_float(r[q]);
      } else {
        f[2 * q] = __uint_as_float(r[q] << 16);
        f[2 * q + 1] = __uint_as_float(r[q] & 0xffff0000u);
      }
    }
  }
  // a bit for each element of slot j that is `enough`
  __device__ __forceinline__ uint32_t which(const uint4& v, int j, const AtLeast& enough) const {
    float f[E];
    unpack(v, f);
    uint32_t mask = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) mask |= (enough(f[e]) ? 1u : 0u) << e;
    const int i = first(j);
    if (i < 0) mask &= ~0u << -i;
    if (i + E > V) mask &= (1u << (V - i)) - 1;
    return mask;
  }
  __device__ static __forceinline__ float max_of(const uint4& v) {
    if constexpr (E == 4) {
      return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)),
                     max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
    } else {
      const uint32_t m = max_nan_bf16x2(max_nan_bf16x2(v.x, v.y), max_nan_bf16x2(v.z, v.w));
      return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
  }
};

// larger: better value, or the same at a lower index
__device__ __forceinline__ uint64_t rank_key(uint32_t key, int index) {
  return static_cast<uint64_t>(key) << 32 | static_cast<uint32_t>(~index);
}

__device__ __forceinline__ float warp_max_nan(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// m = max z, s = sum 2^x, w = sum 2^x x with x = (z - m) log2 e, of parts of a row
struct Stats {
  float m, s, w;
  // over the first `lanes` lanes of a warp, whose others hold (-inf, 0, 0); every one of them has the result
  __device__ __forceinline__ void merge_lanes(int lanes) {
    const float nm = warp_max_nan(m);
    const float d = fmaxf(m - nm, kFloor) * kLog2e;  // -inf less -inf is NaN: the sums are 0
    const float c = exp2_fast(d);
    w = c * (w + s * d);
    s *= c;
    m = nm;
#pragma unroll
    for (int off = lanes / 2; off > 0; off >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, off);
      w += __shfl_xor_sync(0xffffffffu, w, off);
    }
  }
};

// A thread's running statistics. One fma gives x: z log2 e - ref with ref = m' log2 e rounded, m' a maximum of the
// row so far that is not raised before another passes it by kAhead: a row has few stages, and one that has just
// begun raises its maximum in nearly every one (for some lane of a warp). What ref is beside m log2 e, its rounding among
// it, is taken out at the end (rebase).
constexpr float kAhead = 8.f;  // of log2: sums of 2^8 times the terms, and 8 steps of 2^-24 in the entropy
template <typename T>
struct Running {
  float m = -kInf;      // the maximum
  float from = -kInf;   // m'
  float limit = -kInf;  // above it m' is raised
  bool huge = true;     // ref's rounding would not be small beside 1, or m' is -inf: (z - m') log2 e instead
  uint64_t nref = 0;    // -ref twice; huge: -m', 0 for -inf
  uint32_t low = 0;     // not huge: values below it (fp32, or bf16 twice) count as it, which is 0: 0 * x stays 0
  uint64_t s = 0, w = 0;

  __device__ __forceinline__ void raise(float nm) {  // m' to nm, NaN if there is a NaN
    const bool h = fabsf(nm) >= 0x1p20f;
    const float ref = h ? nm : nm * kLog2e;
    // From the old reference to the new one, each with its own rounding, which may be 2^-4 near 2^20 and is in every term
    // so far: (of a huge one: none) one fma takes the other from it.
    const float old = -unpack2(nref).x;
    const float d = max_nan(huge ? (h ? (from - nm) * kLog2e : fmaf(from, kLog2e, -ref))
                                 : (h ? fmaf(-nm, kLog2e, old) : old - ref), kFloor * kLog2e);
    const float c = exp2_fast(d);
    w = fma2(s, pack2(d, d), w);
    s = fma2(s, pack2(c, c), 0);
    w = fma2(w, pack2(c, c), 0);
    from = nm;
    nref = pack2(-ref, -ref);
    huge = h;
    limit = h ? nm : nm + kAhead * kLn2;
    const float l = nm + kFloor - 0x1p-6f * fabsf(nm);
    low = sizeof(T) == 4 ? __float_as_uint(l) : pack_bf16x2(l, l);
  }

  __device__ __forceinline__ static float max_of(const uint32_t* r, int n) {  // of 4 n registers
    if constexpr (sizeof(T) == 4) {
      float x = __uint_as_float(r[0]);
#pragma unroll
      for (int i = 1; i < 4 * n; ++i) x = max_nan(x, __uint_as_float(r[i]));
      return x;
    } else {
      uint32_t x = r[0];
#pragma unroll
      for (int i = 1; i < 4 * n; ++i) x = max_nan_bf16x2(x, r[i]);
      return max_nan(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    }
  }

  __device__ __forceinline__ static bool all_are(const uint32_t* r, int n, float v) {
    const uint32_t want = sizeof(T) == 4 ? __float_as_uint(v) : pack_bf16x2(v, v);
    uint32_t other = 0;
#pragma unroll
    for (int i = 0; i < 4 * n; ++i) other |= r[i] ^ want;
    return other == 0;
  }

  __device__ __forceinline__ void add_pair(uint64_t z2, uint64_t log2e) {
    const uint64_t x2 = fma2(z2, log2e, nref);
    const float2 x = unpack2(x2);
    const uint64_t e2 = pack2(exp2_fast(x.x), exp2_fast(x.y));
    s = add2(s, e2);
    w = fma2(e2, x2, w);
  }
  // 4 n registers of values, whose largest is cm
  template <int n>
  __device__ __forceinline__ void add(const uint32_t* r, float cm, uint64_t log2e) {
    if (cm == -kInf) return;  // nothing but masked logits
    if (!(cm <= limit)) raise(cm);
    m = max_nan(m, cm);
    if (!huge) {
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4 * n; i += 2)
          add_pair(pack2(max_nan(__uint_as_float(r[i]), __uint_as_float(low)),
                         max_nan(__uint_as_float(r[i + 1]), __uint_as_float(low))), log2e);
      } else {
#pragma unroll
        for (int i = 0; i < 4 * n; ++i) {
          const uint32_t c = max_nan_bf16x2(r[i], low);
          add_pair(pack2(__uint_as_float(c << 16), __uint_as_float(c & 0xffff0000u)), log2e);
        }
      }
    } else if (from < kInf && all_are(r, n, from)) {
      // masked with the type's lowest value, and nothing above it yet: x = 0 (420 x 32000 bf16, k = 20: 14 us, 104
      // with the terms below and all elements of a row collected before the top is found to be too many)
      const float count = n * (Row<T>::E / 2);
      s = add2(s, pack2(count, count));
    } else {
      const float base = -unpack2(nref).x;
#pragma unroll 1
      for (int u = 0; u < n; ++u) {
        float f[Row<T>::E];
        uint4 v;
        if constexpr (n == 1) {
          v = make_uint4(r[0], r[1], r[2], r[3]);
        } else {  // without indexing registers
          v = make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < n; ++i)
            if (i == u) v = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
        }
        Row<T>::unpack(v, f);
#pragma unroll
        for (int e = 0; e < Row<T>::E; e += 2) {
          const float x0 = max_nan(f[e] - base, kFloor) * kLog2e, x1 = max_nan(f[e + 1] - base, kFloor) * kLog2e;
          const uint64_t e2 = pack2(exp2_fast(x0), exp2_fast(x1));
          s = add2(s, e2);
          w = fma2(e2, pack2(x0, x1), w);
        }
      }
    }
  }
  // the sums relative to m itself
  __device__ __forceinline__ Stats rebase() const {
    const float2 sp = unpack2(s), wp = unpack2(w);
    Stats r{m, sp.x + sp.y, wp.x + wp.y};
    if (!huge) {
      const float d = fmaf(m, kLog2e, unpack2(nref).x);  // one rounding, of a number up to kAhead
      const float c = exp2_fast(-d);
      r.w = c * (r.w - r.s * d);
      r.s *= c;
    }
    return r;
  }
};

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int mask) {
  return __shfl_xor_sync(0xffffffffu, static_cast<unsigned long long>(v), mask);
}
__device__ __forceinline__ uint32_t shfl(uint32_t v, int from) { return __shfl_sync(0xffffffffu, v, from); }
__device__ __forceinline__ uint64_t shfl(uint64_t v, int from) {
  return __shfl_sync(0xffffffffu, static_cast<unsigned long long>(v), from);
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t min64(uint64_t a, uint64_t b) { return a < b ? a : b; }

// Bitonic networks over a warp, one key a lane, lane 0 the largest.
__device__ __forceinline__ uint64_t bitonic_merge(uint64_t v, int lane) {
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const uint64_t o = shfl_xor64(v, j);
    v = lane & j ? min64(v, o) : max64(v, o);
  }
  return v;
}
// The same over 32-bit keys.
__device__ __forceinline__ uint32_t bitonic_merge(uint32_t v, int lane) {
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const uint32_t o = __shfl_xor_sync(0xffffffffu, v, j);
    v = lane & j ? min(v, o) : max(v, o);
  }
  return v;
}
__device__ __forceinline__ uint32_t sort_warp(uint32_t v, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
    for (int j = size >> 1; j > 0; j >>= 1) {
      const uint32_t o = __shfl_xor_sync(0xffffffffu, v, j);
      v = ((lane & j) == 0) == ((lane & size) == 0) ? max(v, o) : min(v, o);
    }
  }
  return v;
}
// warp_wait_bounded whose loop the whole warp takes together, without lanes that branch off (8 x 1024 ragged rows of 32000
// bf16, k = 8: 66.8 us, 67.8 with that)
__device__ __forceinline__ bool warp_wait_converged(uint32_t bar, uint32_t parity, volatile int* abort, int* err, int code) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  const long long t0 = clock64();
  for (uint32_t i = 1;; ++i) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((i & 255u) != 0u) continue;
    const bool late = clock64() - t0 > kWaitBudgetCycles;
    if (__any_sync(0xffffffffu, late || *abort)) {
      if (late) {
        *abort = 1;
        record_error(err, code);
      }
      return false;
    }
  }
}

// A barrier of the summing threads. A warp that leaves early is excused from the next one: it arrives there without
// waiting, so that a wait that has run out in one warp keeps none of the others.
__device__ __forceinline__ void summers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kSummers) : "memory"); }
__device__ __forceinline__ void summers_excuse() { asm volatile("bar.arrive 1, %0;" ::"n"(kSummers) : "memory"); }

// A bound that at least k of 256 keys reach, or 0 where fewer than k are not 0: the k-th largest of the best of 64
// groups of four. list[w] holds a key a lane.
__device__ __forceinline__ uint32_t kth_bound(const uint32_t (*list)[32], int k, int lane) {
  uint32_t a = 0, b = 0;
#pragma unroll
  for (int w = 0; w < kWarps / 2; ++w) {
    a = max(a, list[w][lane]);
    b = max(b, list[w + kWarps / 2][lane]);
  }
  a = sort_warp(a, lane);
  b = sort_warp(b, lane);
  a = bitonic_merge(max(a, shfl(b, 31 - lane)), lane);
  return shfl(a, k - 1);
}

// A value to the address of `local` in another CTA of the cluster; its bytes arrive on that CTA's `bar`
__device__ __forceinline__ void send(const float* local, const uint64_t* bar, uint32_t rank, float v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(
                   map_to_rank(smem_u32(local), rank)),
               "f"(v), "r"(map_to_rank(smem_u32(bar), rank))
               : "memory");
}
__device__ __forceinline__ void send(const uint64_t* local, const uint64_t* bar, uint32_t rank, uint64_t v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.u64 [%0], %1, [%2];" ::"r"(
                   map_to_rank(smem_u32(local), rank)),
               "l"(v), "r"(map_to_rank(smem_u32(bar), rank))
               : "memory");
}
// This thread's stores to shared memory before the bulk copies that it issues from here on
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// [p, p + bytes) to shared memory at dst, all on 16-byte boundaries; its bytes arrive on `bar`
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* p, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(p)), "r"(bytes), "r"(bar)
               : "memory");
}

// What a stage holds: slots [j0, j0 + n) of a row; n < 0 ends the work.
struct alignas(16) Stage {
  unsigned row;
  int j0, n_flags, id;
};
// beside n: the row's first and last stage in this CTA, the last of a segment, and which one
constexpr int kFirst = 1 << 16, kLast = 1 << 17, kSegmentEnd = 1 << 18, kSegmentShift = 20;

template <bool kTop>
constexpr int stages_of() { return kTop ? 4 : 3; }

template <bool kTop>
struct Shared {
  static constexpr int kStages = stages_of<kTop>();
  unsigned char ring[kStages][kStageSlots * 16];
  Stage stage[kStages];
  uint64_t full[kStages], drained[kStages], others;
  float red[kEnders][3][kWarps];
  float cluster_stats[kClusterMax][3];
  int before[kEvenMax];  // live rows of the sequences before one
  int abort_flag;
};
// What the summers leave of a row for one of the enders, and what that warp works with.
struct End {
  uint4 hit[128];                         // slots that hold candidates: four a lane
  uint64_t cand[kCandidates + 4];         // elements that may be among the best
  uint64_t best[32];                      // this CTA's k best elements
  alignas(8) __nv_bfloat16 segment[kSegments][kSummers];  // each summer's best value of a segment, rounded up
  uint32_t key[kWarps][32];               // order_key of its best value of all, 0 where it has none
  int hit_slot[128];
  uint16_t asked[kSummers];               // summers that hold candidates
  uint16_t owner[kSegments * kSummers];   // segments that do
  unsigned row;
  int id;                                 // the row's token
  bool end;                               // no row is left
  uint64_t done, free;
};
struct SharedTop {
  End end[kEnders];
  // a cluster has one row, for the first ender: another's segments hold what its CTAs send
  __device__ __forceinline__ uint64_t* cluster_best(unsigned rank) {
    return reinterpret_cast<uint64_t*>(end[1].segment) + rank * 32;
  }
};
static_assert(kClusterMax * 32 * sizeof(uint64_t) <= sizeof(End::segment), "the keys of a cluster");
template <bool kTop>
constexpr size_t shared_bytes() { return sizeof(Shared<kTop>) + (kTop ? sizeof(SharedTop) : 0); }
template <bool kTop>
constexpr int block_threads() { return kSummers + 32 + (kTop ? kEnders * 32 : 0); }
template <bool kTop>
constexpr int ctas_per_sm() { return kTop ? 2 : 4; }
static_assert(2 * (shared_bytes<true>() + 1024) <= 228 * 1024 && 4 * (shared_bytes<false>() + 1024) <= 228 * 1024,
              "CTAs an SM");

// A row's slots in this CTA of a cluster of 1 << bits.
struct Part {
  int lo, hi;
  __device__ __forceinline__ Part(int n_slots, unsigned rank, unsigned bits) {
    lo = static_cast<int>(static_cast<unsigned>(n_slots) * static_cast<unsigned long long>(rank) >> bits);
    hi = static_cast<int>(static_cast<unsigned>(n_slots) * static_cast<unsigned long long>(rank + 1) >> bits);
  }
};

// Stages of a segment of a row's part.
__device__ __forceinline__ int segment_stages(const Part& part) {
  return ((part.hi - part.lo + kStageSlots - 1) / kStageSlots + kSegments - 1) / kSegments;
}

// The sum of v over the lanes below, and over all of them. Mostly no lane has more than one.
__device__ __forceinline__ int scan(int v, int lane, int& total) {
  const uint32_t some = __ballot_sync(0xffffffffu, v != 0);
  if (!__any_sync(0xffffffffu, v > 1)) {
    total = __popc(some);
    return __popc(some & ((1u << lane) - 1));
  }
  int sum = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, sum, off);
    sum += lane >= off ? o : 0;
  }
  total = __shfl_sync(0xffffffffu, sum, 31);
  return sum - v;
}

// The k best of the row's slots [part.lo, part.hi), best first, one a lane (0 behind the last). By one warp, whose
// every step waits for the one before it: a vote or a branch for each of many things would cost more than
// their loads (8 us a row instead of 3), so each lane works out what it adds and one scan places it.
template <typename T>
__device__ __forceinline__ uint64_t select_top(End& e, const Row<T>& r, const Part& part, int k, int lane) {
  constexpr int G = 4;
  const int stages = segment_stages(part), each = stages * kSlotsEach;
  // a summer's slots of a segment by as many lanes, up to 32
  const int bits = each <= 4 ? 2 : each <= 8 ? 3 : each <= 16 ? 4 : 5, at_once = 32 >> bits;
  const int full_hi = min(part.hi, r.full_hi);
  const uint32_t lowest = order_key(-kInf);
  uint32_t bound = max(kth_bound(e.key, k, lane), 1u);  // at least k values are not below it
  // Every value from the bound on is taken, or, where more equal the bound than can be ranked (masked logits often do),
  // every value above it; those that equal it then follow by index. Where more than fit are above it, too, the best of
  // those seen give a higher bound, and the range of keys in which the k-th lies is halved until few enough reach its
  // middle: 33 more passes at most, whatever the order of the values. (Raised bounds alone took a pass for every 220 values
  // in the worst order: 160 x 262144 fp32 7.8 ms, 0.22 so, and above that a time that grew with V^2.)
  uint32_t step = bound == lowest ? 1 : 0;  // what is taken is beyond the bound by this much
  uint32_t top = 0;  // the k-th is not above it (0: not asked yet)
  for (;;) {
    const bool above = step != 0;
    const uint32_t least = bound + step;
    const bool none = least == 0;  // nothing is above NaN
    const AtLeast enough(least);
    e.best[lane] = 0;
    int asked, found = 0;
    uint32_t is = 0;  // a bit for each warp's summer of this lane
#pragma unroll
    for (int w = 0; w < kWarps; ++w) is |= (!none && e.key[w][lane] >= least ? 1u : 0u) << w;
    for (int at = scan(__popc(is), lane, asked); is != 0; is &= is - 1)
      e.asked[at++] = static_cast<uint16_t>((__ffs(is) - 1) * 32 + lane);
    __syncwarp();
    // their segments that hold candidates, up to kSegments a lane; all of them first, or batches of the loads below
    // would go half empty (8192 x 32000 bf16, k = 32: 131 us, 125 so)
    int owners = 0;
    for (int x0 = 0; x0 < asked && (above || owners <= kCandidates); x0 += 32) {
      const int summer = x0 + lane < asked ? e.asked[x0 + lane] : 0;
      is = 0;
#pragma unroll
      for (int q = 0; q < kSegments; ++q)
        if (part.lo + q * stages * kStageSlots + summer < part.hi)
          is |= (enough(__bfloat162float(e.segment[q][summer])) ? 1u : 0u) << q;
      if (x0 + lane >= asked) is = 0;
      int more;
      int at = owners + scan(__popc(is), lane, more);
      for (; is != 0; is &= is - 1) e.owner[at++] = static_cast<uint16_t>((__ffs(is) - 1) << 10 | summer);
      owners += more;
    }
    if (!above && owners > kCandidates) {  // with a candidate each, too many of them
      step = 1;
      continue;
    }
    __syncwarp();
#pragma unroll 1
    for (int i0 = 0; i0 < each && found <= kCandidates; i0 += 1 << bits) {
      const int i = i0 + (lane & ((1 << bits) - 1));
#pragma unroll 1
      for (int g0 = 0; g0 < owners && found <= kCandidates; g0 += G * at_once) {  // more than fit: enough is known
        uint4 v[G];
        int j[G];
        bool in_part = false;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const int o = g0 + g * at_once + (lane >> bits);
          j[g] = part.hi;
          if (o < owners && i < each)
            j[g] = part.lo + (e.owner[o] >> 10) * stages * kStageSlots + (e.owner[o] & 1023) + i * kSummers;
          if (j[g] >= r.full_lo && j[g] < full_hi) v[g] = r.load_full(j[g]); else in_part |= j[g] < part.hi;
        }
        // the row's first and last slot, where it has them in part
        if (__any_sync(0xffffffffu, in_part)) {
#pragma unroll
          for (int g = 0; g < G; ++g)
            if (j[g] < part.hi && (j[g] < r.full_lo || j[g] >= full_hi)) v[g] = r.load(j[g]);
        }
        // the slots that hold some, in a row; then their elements, a slot a lane
        int hits = 0;
#pragma unroll
        for (int g = 0; g < G; ++g)
          if (j[g] >= part.hi || !enough(Row<T>::max_of(v[g]))) j[g] = -1; else ++hits;
        int slots;
        int at = scan(hits, lane, slots);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          if (j[g] < 0) continue;
          e.hit[at] = v[g];
          e.hit_slot[at++] = j[g];
        }
        __syncwarp();
        for (int h0 = 0; h0 < slots; h0 += 32) {
          const int slot = h0 + lane < slots ? e.hit_slot[h0 + lane] : 0;
          uint32_t mask = 0;
          if (h0 + lane < slots) mask = r.which(e.hit[h0 + lane], slot, enough);
          int more;
          int c = found + scan(__popc(mask), lane, more);
          found += more;
          for (; mask != 0; mask &= mask - 1, ++c) {
            const int q = __ffs(mask) - 1;
            if (c < kCandidates)
              e.cand[c] = rank_key(order_key(to_f(reinterpret_cast<const T*>(&e.hit[h0 + lane])[q])), r.first(slot) + q);
          }
        }
        __syncwarp();
      }
    }
    if (found > kCandidates && !above) {
      step = 1;
      continue;
    }
    const int held = min(found, kCandidates);
    if (lane < 4) e.cand[held + lane] = 0;
    __syncwarp();
    uint64_t kth = 0;
    for (int c = lane; c < held; c += 32) {
      const uint64_t mine = e.cand[c];
      int place = 0;
#pragma unroll 2
      for (int o = 0; o < held; o += 4) {
        const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(&e.cand[o]),
                         y = *reinterpret_cast<const ulonglong2*>(&e.cand[o + 2]);
        place += (x.x > mine) + (x.y > mine) + (y.x > mine) + (y.y > mine);
      }
      if (place < k && found <= kCandidates) e.best[place] = mine;
      if (place == k - 1) kth = mine;
    }
    __syncwarp();
    if (found <= kCandidates) {
      if (!above || found >= k) return e.best[lane];
      if (step == 1) break;
      top = least - 1;
    } else {
      // more than fit: the k-th best of those held is a higher bound
      const uint32_t who = __ballot_sync(0xffffffffu, kth != 0);
      bound = static_cast<uint32_t>(shfl(kth, __ffs(who) - 1) >> 32);
      if (top == 0) {
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = max(top, e.key[w][lane]);
        top = __reduce_max_sync(0xffffffffu, top);
      }
    }
    step = max((top - bound + 1) / 2, 1u);
  }
  // the first values that equal the bound, in the segments that may hold some
  int place = __popc(__ballot_sync(0xffffffffu, e.best[lane] != 0));
  const AtLeast equal(bound);  // or above, where no more are
  for (int j0 = part.lo; j0 < part.hi && place < k; j0 += 32) {
    const int j = j0 + lane, in = j - part.lo;
    const bool may = j < part.hi && equal(__bfloat162float(e.segment[in / (stages * kStageSlots)][in % kSummers]));
    if (!__any_sync(0xffffffffu, may)) continue;
    uint32_t mask = 0;
    if (may) {
      const uint4 v = r.load(j);
      mask = r.which(v, j, equal);
      if (bound != kNanKey) mask &= ~r.which(v, j, AtLeast(bound + 1));
    }
    int more;
    int at = place + scan(__popc(mask), lane, more);
    for (; mask != 0 && at < k; mask &= mask - 1, ++at) e.best[at] = rank_key(bound, r.first(j) + __ffs(mask) - 1);
    place += more;
  }
  __syncwarp();
  return e.best[lane];
}

// What a call gives for a row.
struct Outputs {
  float* logp;
  float* entropy;
  float* norm;
  int32_t* top_ids;
  float* top_logp;
  int k;

  __device__ __forceinline__ void dead(unsigned row) const {
    if (logp) logp[row] = 0.f;
    if (entropy) entropy[row] = 0.f;
    if (norm) norm[2ll * row] = norm[2ll * row + 1] = 0.f;
    for (int x = 0; x < k; ++x) {
      top_ids[static_cast<long long>(row) * k + x] = -1;
      top_logp[static_cast<long long>(row) * k + x] = 0.f;
    }
  }
  // by a warp; st.m in every lane, the rest in lane 0, `top` one of the best a lane
  template <bool kTop>
  __device__ __forceinline__ void live(unsigned row, const Stats& st, float z_id, uint64_t top, int lane) const {
    const float m = st.m, sum = __shfl_sync(0xffffffffu, st.s, 0);
    const bool empty = m == -kInf;  // nothing but -inf
    const float ls = empty ? 0.f : logf(sum);
    if (lane == 0) {
      if (norm) {
        norm[2ll * row] = m;
        norm[2ll * row + 1] = ls;
      }
      if (entropy) entropy[row] = empty ? 0.f : ls - kLn2 * (st.w / sum);
      if (logp) logp[row] = empty && z_id == z_id ? -kInf : (z_id - m) - ls;
    }
    if (kTop && lane < k) {
      const float x = order_value(static_cast<uint32_t>(top >> 32));
      top_ids[static_cast<long long>(row) * k + lane] = static_cast<int>(~static_cast<uint32_t>(top));
      top_logp[static_cast<long long>(row) * k + lane] = empty ? -kInf : (x - m) - ls;
    }
  }
};

// What a CTA sends to the first of its cluster.
template <bool kTop>
constexpr uint32_t sent_bytes() { return 3 * sizeof(float) + (kTop ? 32 * sizeof(uint64_t) : 0); }

// A warp of a cluster's first CTA that has given up a wait stays until nothing more can arrive in its memory: until
// the peers' threads have ended (the barrier counts those as arrived) and what they sent has come, or cannot come any
// more. Without an expiry none is needed: the CTA that ends a row has waited for all of it.
// (A call: in line it makes the kernels of clusters 0.1 to 0.2 us longer.)
__device__ __noinline__ void outlive_peers(uint32_t others, int* err) {
  cluster_sync_all();
  int never = 0;
  warp_wait_cluster_bounded(others, 0, &never, err, kDevTimeoutEpilogue);
}

// A CTA's part of a row, by a warp: written out, or in a cluster sent to its first CTA, which writes the whole.
// (Bytes that arrive by themselves: plain stores, a fence and an arrival took 0.5 us more.)
template <bool kTop>
__device__ __forceinline__ void finish(Shared<kTop>& sh, SharedTop& top, const Outputs& out, unsigned row, Stats st, float z_id,
                                       uint64_t best, unsigned rank, unsigned cs, int lane, int* err) {
  if (cs > 1) {
    if (rank != 0) {
      if (lane < 3) send(&sh.cluster_stats[rank][lane], &sh.others, 0, lane == 0 ? st.m : lane == 1 ? st.s : st.w);
      if constexpr (kTop) send(top.cluster_best(rank) + lane, &sh.others, 0, best);
      return;
    }
    if (!warp_wait_cluster_bounded(smem_u32(&sh.others), 0, &sh.abort_flag, err, kDevTimeoutEpilogue)) {
      outlive_peers(smem_u32(&sh.others), err);
      st.m = kNan;
    }
    if (lane > 0) {
      st = Stats{-kInf, 0.f, 0.f};
      if (lane < static_cast<int>(cs)) st = Stats{sh.cluster_stats[lane][0], sh.cluster_stats[lane][1], sh.cluster_stats[lane][2]};
    }
    st.merge_lanes(kClusterMax);
    if constexpr (kTop) {
      uint64_t list[kClusterMax] = {best};
#pragma unroll
      for (int c = 1; c < kClusterMax; ++c) list[c] = c < static_cast<int>(cs) ? top.cluster_best(c)[c % 2 ? 31 - lane : lane] : 0;
#pragma unroll
      for (int half = kClusterMax / 2; half > 0; half >>= 1) {
        if (half >= static_cast<int>(cs)) continue;
#pragma unroll
        for (int c = 0; c < half; ++c) {
          // the second of a pair backwards
          list[c] = bitonic_merge(max64(list[2 * c], list[2 * c + 1]), lane);
          if (half > 1 && c % 2) list[c] = shfl(list[c], 31 - lane);
        }
      }
      best = list[0];
    }
  }
  out.live<kTop>(row, st, z_id, best, lane);
}

// Clusters of one CTA take every gridDim.x-th row in turn, larger ones one row that their CTAs share. The last
// warp of a CTA fetches the slots of its rows, stage by stage, and the others sum them.
template <typename T, bool kTop, bool kCluster>
__global__ void __launch_bounds__(block_threads<kTop>(), ctas_per_sm<kTop>())
    token_stats_kernel(const T* __restrict__ logits, long long ld, unsigned rows, unsigned L, int V,
                       const int32_t* __restrict__ ids, const int32_t* __restrict__ lengths, unsigned cluster_bits,
                       const Outputs out, int* err) {
  extern __shared__ __align__(16) unsigned char raw[];
  constexpr int kStages = stages_of<kTop>();
  Shared<kTop>& sh = *reinterpret_cast<Shared<kTop>*>(raw);
  SharedTop& top = *reinterpret_cast<SharedTop*>(raw + sizeof(Shared<kTop>));  // with kTop
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned bits = kCluster ? cluster_bits : 0, cs = 1u << bits, rank = kCluster ? cluster_rank() : 0;
  if (tid == 0) {
    for (int q = 0; q < kStages; ++q) {
      mbar_init(smem_u32(&sh.full[q]), 1);
      mbar_init(smem_u32(&sh.drained[q]), kWarps);
    }
    mbar_init(smem_u32(&sh.others), 1);
    if constexpr (kTop)
      for (int f = 0; f < kEnders; ++f) {
        mbar_init(smem_u32(&top.end[f].done), kWarps);
        mbar_init(smem_u32(&top.end[f].free), 1);
      }
    sh.abort_flag = 0;
    fence_mbar_init();
    if (cs > 1 && rank == 0) mbar_arrive_expect_tx(smem_u32(&sh.others), (cs - 1) * sent_bytes<kTop>());
  }
  if (cs > 1) cluster_sync_all(); else __syncthreads();
  pdl_wait();
  pdl_launch_dependents();

  auto give_up = [&]() {
    if (kCluster && rank == 0) outlive_peers(smem_u32(&sh.others), err);
  };
  if (warp == kWarps) {
    // ------------------------------------------------------------------ fetch
    const unsigned step = gridDim.x >> bits;
    int q = 0;
    uint32_t parity = 1;  // of a stage's last release; none in the first round
    bool wrapped = false;
    auto acquire = [&]() {
      return !wrapped || warp_wait_bounded(smem_u32(&sh.drained[q]), parity, &sh.abort_flag, err, kDevTimeoutProducer);
    };
    auto advance = [&]() {
      __syncwarp();
      if (++q == kStages) {
        q = 0;
        parity ^= 1;
        wrapped = true;
      }
    };
    // Of few sequences the rows that hold a token are dealt evenly, by their number among these: a CTA's every 608th
    // row may hold one each time, or never (1000 live rows of 4 x 400, 32000 fp32: 29.2 us, 25.1 so).
    const unsigned seqs = rows / L;
    const bool even = bits == 0 && lengths != nullptr && seqs <= kEvenMax && gridDim.x < rows;
    unsigned items = rows;
    if (even) {
      int len[kEvenMax / 32], sum = 0, all;
#pragma unroll
      for (int x = 0; x < kEvenMax / 32; ++x) {
        const unsigned sq = lane * (kEvenMax / 32) + x;
        len[x] = 0;
        if (sq < seqs) {
          const int n = lengths[sq];
          if (n < 0 || n > static_cast<int>(L)) record_error(err, kDevBadLength);
          len[x] = min(max(n, 0), static_cast<int>(L));
        }
        sum += len[x];
      }
      int before = scan(sum, lane, all);
#pragma unroll
      for (int x = 0; x < kEvenMax / 32; ++x) {
        sh.before[lane * (kEvenMax / 32) + x] = before;
        before += len[x];
      }
      items = all;
      __syncwarp();
    }
    auto live_row = [&](unsigned row, bool report) {
      if (lengths == nullptr) return true;
      const unsigned sq = row / L, t = row - sq * L;
      const int n = lengths[sq];
      if ((n < 0 || n > static_cast<int>(L)) && report) record_error(err, kDevBadLength);
      return n > static_cast<int>(L) || static_cast<int>(t) < n;
    };
    // 32 of the rows at a time, one a lane: whether it holds a token, and which
    auto fetch = [&]() {  // false where a wait has run out
      for (unsigned long long base = blockIdx.x >> bits; base < items; base += 32ull * step) {
        const unsigned long long item = base + static_cast<unsigned long long>(lane) * step;
        unsigned row_l = static_cast<unsigned>(item);
        bool live = item < items;
        int id = 0;
        if (live) {
          if (even) {  // the last sequence with no more rows before it
            int lo = 0, hi = kEvenMax;
            while (hi - lo > 1) {
              const int mid = (lo + hi) / 2;
              if (sh.before[mid] <= static_cast<int>(item)) lo = mid; else hi = mid;
            }
            row_l = lo * L + static_cast<unsigned>(item) - sh.before[lo];
          }
          if (out.logp) id = ids[row_l];
          if (!even) {
            live = live_row(row_l, rank == 0);
            if (!live && rank == 0) out.dead(row_l);
          }
        }
        for (uint32_t todo = __ballot_sync(0xffffffffu, live); todo != 0; todo &= todo - 1) {
          const int l = __ffs(todo) - 1;
          const unsigned row = __shfl_sync(0xffffffffu, row_l, l);
          const int row_id = __shfl_sync(0xffffffffu, id, l);
          const Row<T> r(logits + row * ld, V);
          const Part part(r.n_slots, rank, bits);
          int j0 = part.lo, segment = 0, left = segment_stages(part);
          do {  // a part without slots has a stage, too
            if (!acquire()) return false;
            if (lane == 0) {
              const int j1 = min(j0 + kStageSlots, part.hi), lo = max(j0, r.full_lo), hi = min(j1, r.full_hi);
              unsigned char* dst = sh.ring[q];
              // The row's first and last slot, where it has them in part. Whole stages that lie there later are written by
              // bulk copies: a proxy of their own, before which these stores have to be done.
              const bool head = j0 < min(lo, j1), tail = hi < j1 && j1 > lo;
              if (head) *reinterpret_cast<uint4*>(dst) = r.load(j0);
              if (tail) *reinterpret_cast<uint4*>(dst + (j1 - 1 - j0) * 16) = r.load(j1 - 1);
              if (head || tail) fence_proxy_async();
              sh.stage[q] = Stage{row, j0,
                                  (j1 - j0) | (j0 == part.lo ? kFirst : 0) | (j1 == part.hi ? kLast : 0) |
                                      (left <= 1 || j1 == part.hi ? kSegmentEnd : 0) | segment << kSegmentShift,
                                  row_id};
              const uint32_t bytes = hi > lo ? static_cast<uint32_t>(hi - lo) * 16 : 0;
              mbar_arrive_expect_tx(smem_u32(&sh.full[q]), bytes);
              if (bytes > 0) bulk_load(smem_u32(dst + (lo - j0) * 16), r.p + r.first(lo), bytes, smem_u32(&sh.full[q]));
            }
            advance();
            j0 += kStageSlots;
            if (--left == 0) {
              left = segment_stages(part);
              ++segment;
            }
          } while (j0 < part.hi);
        }
      }
      if (!acquire()) return false;
      if (lane == 0) {
        sh.stage[q] = Stage{0, 0, -1, 0};
        mbar_arrive(smem_u32(&sh.full[q]));
      }
      return true;
    };
    if (!fetch()) {  // the copies under way come before this CTA's memory goes
      int never = 0;
      for (int x = 0; x < kStages; ++x)
        if (x < q || wrapped)
          warp_wait_bounded(smem_u32(&sh.full[x]), x < q ? parity ^ 1 : parity, &never, err, kDevTimeoutProducer);
      give_up();
      return;
    }
    if (even)
      for (unsigned long long row = blockIdx.x + static_cast<unsigned long long>(lane) * step; row < rows; row += 32ull * step)
        if (!live_row(static_cast<unsigned>(row), false)) out.dead(static_cast<unsigned>(row));
    return;
  }

  if (kTop && warp > kWarps) {
    // ------------------------------------------------------------------ ends of rows
    const int f = warp - kWarps - 1;
    End& e = top.end[f];
    for (uint32_t parity = 0;; parity ^= 1) {
      if (!warp_wait_bounded(smem_u32(&e.done), parity, &sh.abort_flag, err, kDevTimeoutEpilogue)) {
        give_up();
        return;
      }
      if (e.end) return;
      const unsigned row = e.row;
      const Row<T> r(logits + row * ld, V);
      float z_id = kNan;
      if (lane == 0 && rank == 0 && out.logp) {
        if (e.id < 0 || e.id >= V) record_error(err, kDevBadTokenId); else z_id = to_f(r.p[e.id]);
      }
      Stats st = lane < kWarps ? Stats{sh.red[f][0][lane], sh.red[f][1][lane], sh.red[f][2][lane]} : Stats{-kInf, 0.f, 0.f};
      st.merge_lanes(kWarps);
      const uint64_t best = select_top<T>(e, r, Part(r.n_slots, rank, bits), out.k, lane);
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&e.free));
      finish<kTop>(sh, top, out, row, st, z_id, best, rank, cs, lane, err);
    }
  }

  // -------------------------------------------------------------------- sums
  int q = 0, buf = 0;
  uint32_t parity = 0, used = 0;  // used: bit 0 of how often both buffers were filled, bit 1 whether they were
  float z_id = 0.f;
  const uint64_t log2e = twice(kLog2e);
  Running<T> run;
  float segment = -kInf;  // the thread's maximum of the segment so far
  bool holds = false;     // whether it has any slot
  for (;;) {
    if (!warp_wait_converged(smem_u32(&sh.full[q]), parity, &sh.abort_flag, err, kDevTimeoutEpilogue)) {
      if constexpr (!kTop) summers_excuse();
      give_up();
      return;
    }
    const Stage in = sh.stage[q];
    if (in.n_flags < 0) break;
    const int n = in.n_flags & (kFirst - 1);
    if (in.n_flags & kFirst) {
      run = Running<T>();
      holds = tid < n;  // a summer without a slot in the first stage has none
      if (kTop && (used & 2) && !warp_wait_bounded(smem_u32(&top.end[buf].free), used & 1, &sh.abort_flag, err, kDevTimeoutDrain))
        return;  // (not in a cluster: it has one row)
      if (!kTop && tid == 0 && rank == 0 && out.logp) {
        z_id = kNan;
        if (in.id < 0 || in.id >= V) record_error(err, kDevBadTokenId); else z_id = to_f(logits[in.row * ld + in.id]);
      }
    }
    const uint4* src = reinterpret_cast<const uint4*>(sh.ring[q]) + tid;
    float cm = -kInf;
    if (n > kStageSlots / 2) {  // a stage that is not full with -inf behind its slots
      uint32_t v[4 * kSlotsEach];
#pragma unroll
      for (int u = 0; u < kSlotsEach; ++u) {
        const uint32_t fill = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
        uint4 x = make_uint4(fill, fill, fill, fill);
        if (u < kSlotsEach / 2 || tid + u * kSummers < n) x = src[u * kSummers];
        v[4 * u] = x.x;
        v[4 * u + 1] = x.y;
        v[4 * u + 2] = x.z;
        v[4 * u + 3] = x.w;
      }
      cm = run.max_of(v, kSlotsEach);
      run.template add<kSlotsEach>(v, cm, log2e);
    } else {
#pragma unroll 1
      for (int u = 0; tid + u * kSummers < n; ++u) {
        const uint4 x = src[u * kSummers];
        const uint32_t v[4] = {x.x, x.y, x.z, x.w};
        const float slot_max = run.max_of(v, 1);
        run.template add<1>(v, slot_max, log2e);
        cm = max_nan(cm, slot_max);
      }
    }
    if constexpr (kTop) {
      segment = max_nan(segment, cm);
      if (in.n_flags & kSegmentEnd) {
        top.end[buf].segment[in.n_flags >> kSegmentShift][tid] = __float2bfloat16_ru(segment);
        segment = -kInf;
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sh.drained[q]));
    if (++q == kStages) {
      q = 0;
      parity ^= 1;
    }
    if (!(in.n_flags & kLast)) continue;

    Stats st = run.rebase();
    const float value = run.m;
    st.merge_lanes(32);
    if constexpr (kTop) {
      End& e = top.end[buf];
      e.key[warp][lane] = holds ? order_key(value) : 0;
      if (tid == 0) {
        e.row = in.row;
        e.id = in.id;
        e.end = false;
      }
    }
    if (lane == 0) {
      sh.red[buf][0][warp] = st.m;
      sh.red[buf][1][warp] = st.s;
      sh.red[buf][2][warp] = st.w;
    }
    if constexpr (kTop) {
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&top.end[buf].done));
    } else {
      summers_sync();
      if (warp == 0) {
        st = lane < kWarps ? Stats{sh.red[buf][0][lane], sh.red[buf][1][lane], sh.red[buf][2][lane]} : Stats{-kInf, 0.f, 0.f};
        st.merge_lanes(kWarps);
        finish<kTop>(sh, top, out, in.row, st, z_id, 0, rank, cs, lane, err);
      }
      // one that missed this barrier has raised the flag before it; all the others see that here or at the next
      if (!kCluster && *static_cast<volatile int*>(&sh.abort_flag)) {
        summers_excuse();
        return;
      }
    }
    if (++buf == kEnders) {
      buf = 0;
      used = used == 0 ? 2 : used ^ 1;
    }
  }
  if constexpr (kTop) {
    for (int f = 0; f < kEnders; ++f) {  // the enders may go
      End& e = top.end[buf];
      if ((used & 2) && !warp_wait_bounded(smem_u32(&e.free), used & 1, &sh.abort_flag, err, kDevTimeoutDrain)) return;
      if (tid == 0) e.end = true;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&e.done));
      if (++buf == kEnders) {
        buf = 0;
        used = used == 0 ? 2 : used ^ 1;
      }
    }
  }
}

// Short rows without alternatives, a warp each: nothing passes between warps, where a row of the kernel above
// takes the summing threads' meeting and one of their warps' end, about 2 us a row for a CTA.
constexpr int kShortWarps = 8, kShortSlots = 8;  // of a CTA; of a lane under way
template <typename T>
__global__ void __launch_bounds__(kShortWarps * 32)
    token_stats_short_kernel(const T* __restrict__ logits, long long ld, unsigned rows, unsigned L, int V,
                             const int32_t* __restrict__ ids, const int32_t* __restrict__ lengths, const Outputs out,
                             int* err) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const unsigned row = blockIdx.x * kShortWarps + (threadIdx.x >> 5);
  if (row >= rows) return;
  if (lengths != nullptr) {
    const unsigned sq = row / L;
    const int n = lengths[sq];
    if ((n < 0 || n > static_cast<int>(L)) && lane == 0) record_error(err, kDevBadLength);
    if (static_cast<int>(row - sq * L) >= n) {
      if (lane == 0) out.dead(row);
      return;
    }
  }
  const Row<T> r(logits + row * ld, V);
  float z_id = kNan;
  if (lane == 0 && out.logp) {
    const int id = ids[row];
    if (id < 0 || id >= V) record_error(err, kDevBadTokenId); else z_id = to_f(r.p[id]);
  }
  const uint64_t log2e = twice(kLog2e);
  Running<T> run;
  for (int j0 = lane; j0 < r.n_slots; j0 += 32 * kShortSlots) {
    uint32_t v[4 * kShortSlots];
#pragma unroll
    for (int u = 0; u < kShortSlots; ++u) {
      const int j = j0 + u * 32;
      const uint32_t fill = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;  // -inf
      uint4 x = make_uint4(fill, fill, fill, fill);
      if (j < r.n_slots) x = r.load(j);
      v[4 * u] = x.x;
      v[4 * u + 1] = x.y;
      v[4 * u + 2] = x.z;
      v[4 * u + 3] = x.w;
    }
    run.template add<kShortSlots>(v, run.max_of(v, kShortSlots), log2e);
  }
  Stats st = run.rebase();
  st.merge_lanes(32);
  out.live<false>(row, st, z_id, 0, lane);
}

constexpr int kUnit = 8;  // elements a lane turns at once
constexpr int kTileUnits = 8;  // units a lane takes of a tile
constexpr int kTile = 32 * kUnit * kTileUnits;
constexpr int kGradWarps = 8;

template <typename T>
__device__ __forceinline__ void load_unit(const T* p, uint4 (&v)[sizeof(T) / 2]) {
#pragma unroll
  for (int q = 0; q < static_cast<int>(sizeof(T) / 2); ++q) v[q] = reinterpret_cast<const uint4*>(p)[q];
}
__device__ __forceinline__ void store_unit(float* p, const uint64_t (&d)[kUnit / 2]) {
  reinterpret_cast<ulonglong2*>(p)[0] = make_ulonglong2(d[0], d[1]);
  reinterpret_cast<ulonglong2*>(p)[1] = make_ulonglong2(d[2], d[3]);
}
__device__ __forceinline__ void store_unit(__nv_bfloat16* p, const uint64_t (&d)[kUnit / 2]) {
  uint32_t r[kUnit / 2];
#pragma unroll
  for (int q = 0; q < kUnit / 2; ++q) {
    const float2 x = unpack2(d[q]);
    r[q] = pack_bf16x2(x.x, x.y);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(r[0], r[1], r[2], r[3]);
}

// Element e of a unit, e known to the compiler.
template <typename T>
__device__ __forceinline__ float element(const uint4 (&v)[sizeof(T) / 2], int e) {
  const uint4& x = v[sizeof(T) == 4 ? e / 4 : 0];
  const int r = sizeof(T) == 4 ? e % 4 : e / 2;
  const uint32_t w = r == 0 ? x.x : r == 1 ? x.y : r == 2 ? x.z : x.w;
  return sizeof(T) == 4 ? __uint_as_float(w) : __uint_as_float(e % 2 ? w & 0xffff0000u : w << 16);
}

// A row's gradient. With x = (z - m) log2 e - c log2 e (c the row's log-sum), p = 2^x and
//     d = -p (g_logp + g_entropy (c' + x ln 2)),  c' the entropy, and g_logp more at the token
struct RowGrad {
  float m, c, gl, gh, h;
  int id;
  bool logp;

  // an element that is not the token's, for any m
  __device__ __forceinline__ float other(float z) const {
    const float lp = max_nan((z - m) - c, kFloor);
    return -exp2_fast(lp * kLog2e) * ((gl + gh * h) + gh * lp);
  }
  // one element: 1 - p of a token that is nearly certain, and any m
  __device__ __forceinline__ float value(float z, int i) const {
    const float lp = max_nan((z - m) - c, kFloor);
    const float p = exp2_fast(lp * kLog2e);
    return i == id && logp ? -gl * expm1f(lp) - p * (gh * (lp + h)) : -p * ((gl + gh * h) + gh * lp);
  }
};

// A tile of a row whose x would be rounded apart, or of rows that do not lie alike on the grid: a call, as its registers
// would slow the kernel down (2048 x 32000 bf16: 42.3 us, 44.9 with it in line).
template <typename TI, typename TO>
__device__ __noinline__ void tile_apart(const TI* z, TO* d, int i0, int V, bool together, bool live, const RowGrad& g,
                                        int lane) {
  const int hi = min(i0 + kTile, V);
  if (together) {  // mostly a row of which a mask of the type's lowest value leaves nothing (7092 x 1736, a third of the
                   // rows such: 43 us an element at a time, 21 so)
#pragma unroll 2
    for (int i = i0 + lane * kUnit; i < hi; i += 32 * kUnit) {
      if (i >= 0 && i <= V - kUnit && (!g.logp || g.id < i || g.id >= i + kUnit)) {
        uint4 v[sizeof(TI) / 2];
        uint64_t o[kUnit / 2];
        load_unit(z + i, v);
#pragma unroll
        for (int q = 0; q < kUnit / 2; ++q)
          o[q] = pack2(g.other(element<TI>(v, 2 * q)), g.other(element<TI>(v, 2 * q + 1)));
        store_unit(d + i, o);
      } else {
        for (int e = max(i, 0); e < min(i + kUnit, V); ++e) d[e] = from_f<TO>(g.value(to_f(z[e]), e));
      }
    }
  } else {
    // eight elements a lane under way (2048 x 32001 into rows of 32008: fp32 104 us, 230 one after another; bf16 77, 180)
    constexpr int G = 8;
    const int lo = max(i0, 0);
    int i = lo + lane;
#pragma unroll 1
    for (; i + 32 * (G - 1) < hi; i += 32 * G) {
      TI x[G];
      if (live) {
#pragma unroll
        for (int q = 0; q < G; ++q) x[q] = z[i + 32 * q];
      }
#pragma unroll
      for (int q = 0; q < G; ++q) d[i + 32 * q] = from_f<TO>(live ? g.other(to_f(x[q])) : 0.f);
    }
#pragma unroll 1
    for (; i < hi; i += 32) d[i] = from_f<TO>(live ? g.other(to_f(z[i])) : 0.f);
    if (live && g.logp && g.id >= lo && g.id < hi && (g.id - lo) % 32 == lane)  // by the lane that wrote it
      d[g.id] = from_f<TO>(g.value(to_f(z[g.id]), g.id));
  }
}

// A warp takes a tile of a row. Units lie on the 16-byte grid of both arrays where their rows start alike on it
// (`a` elements before the row); else every element goes by itself.
// Memory bounds it: 2048 x 32000 fp32 80 us (96 % of measured HBM), fp32 to bf16 58 (99 %), bf16 42 (92 %; 62.8
// when every element was turned by itself, with a CTA a tile of 4096; so were 8000 x 1001, 22 us, 12.4 now), bf16 to fp32
// 65 (89 %).
template <typename TI, typename TO>
__global__ void __launch_bounds__(kGradWarps * 32, 4)
    token_stats_grad_kernel(const TI* logits, long long ld, unsigned L, int V, unsigned tiles, unsigned items,
                            const int32_t* __restrict__ ids, const int32_t* __restrict__ lengths,
                            const float* __restrict__ norm, const float* __restrict__ entropy,
                            const float* __restrict__ grad_logp, const float* __restrict__ grad_entropy,
                            TO* dlogits, long long ld_d, int* err) {
  constexpr int G = sizeof(TI) + sizeof(TO) == 4 ? 8 : 4;  // units under way at once (bf16 to bf16: 44.3 us with four)
  pdl_wait();
  pdl_launch_dependents();
  const unsigned item = blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5);
  if (item >= items) return;
  const int lane = threadIdx.x & 31;
  const unsigned row = item / tiles;
  const int tile = static_cast<int>(item - row * tiles);
  const unsigned sq = row / L;
  int n = static_cast<int>(L);
  if (lengths != nullptr) n = lengths[sq];
  RowGrad g;
  g.m = norm[2ll * row];
  g.c = norm[2ll * row + 1];
  g.logp = grad_logp != nullptr;
  g.gl = g.gh = g.h = 0.f;
  g.id = 0;
  if (g.logp) {
    g.gl = grad_logp[row];
    g.id = ids[row];
  }
  if (grad_entropy != nullptr) {
    g.gh = grad_entropy[row];
    g.h = entropy[row];
  }
  if (n < 0 || n > static_cast<int>(L)) {
    if (lane == 0) record_error(err, kDevBadLength);
    n = n < 0 ? 0 : static_cast<int>(L);
  }
  const bool live = static_cast<int>(row - sq * L) < n && g.m != -kInf;  // an empty row has no gradient
  if (live && (g.id < 0 || g.id >= V)) {
    if (lane == 0) record_error(err, kDevBadTokenId);
    g.gl = kNan;
  }
  const TI* z = logits + row * ld;
  TO* d = dlogits + row * ld_d;
  const int phase_i = static_cast<int>(reinterpret_cast<uintptr_t>(z) / sizeof(TI) % kUnit);
  const int phase_o = static_cast<int>(reinterpret_cast<uintptr_t>(d) / sizeof(TO) % kUnit);
  const int a = sizeof(TO) == 2 ? phase_o : phase_i;
  const bool together = (phase_i - a) % static_cast<int>(16 / sizeof(TI)) == 0 &&
                        (phase_o - a) % static_cast<int>(16 / sizeof(TO)) == 0;
  const int i0 = tile * kTile - a;  // the tile's first element (below 0 in a first one)
  // beyond, z log2 e and the rest of x are rounded apart
  const bool huge = live && !(fabsf(g.m) < 0x1p20f);
  if (!together || huge) {
    tile_apart<TI, TO>(z, d, i0, V, together, live, g, lane);
    return;
  }
  const float mref = g.m * kLog2e;
  const float rest = fmaf(g.m, kLog2e, -mref) + g.c * kLog2e;
  const float low = g.m + kFloor - 0x1p-6f * fabsf(g.m);  // values below it count as it: p = 0
  const uint32_t low2 = pack_bf16x2(low, low);
  const uint64_t log2e = twice(kLog2e), nref = twice(-mref), nrest = twice(-rest);
  const uint64_t slope = twice(-g.gh * kLn2), base = twice(-(g.gl + g.gh * g.h));
  const int unit = g.logp ? g.id - i0 : -1;  // the token's place in the tile
#pragma unroll 1
  for (int u0 = 0; u0 < kTileUnits; u0 += G) {
    if (i0 + u0 * 32 * kUnit >= V) return;
    uint4 v[G][sizeof(TI) / 2];
#pragma unroll
    for (int u = 0; u < G; ++u) {
      const int i = i0 + ((u0 + u) * 32 + lane) * kUnit;
      if (live && i >= 0 && i <= V - kUnit) load_unit(z + i, v[u]);
    }
#pragma unroll
    for (int u = 0; u < G; ++u) {
      const int i = i0 + ((u0 + u) * 32 + lane) * kUnit;
      if (i0 + (u0 + u) * 32 * kUnit >= V) return;
      if (i >= 0 && i <= V - kUnit) {
        uint64_t o[kUnit / 2] = {};
        if (live) {
#pragma unroll
          for (int q = 0; q < kUnit / 2; ++q) {
            uint64_t z2;
            if constexpr (sizeof(TI) == 4) {
              const uint4& x = v[u][q / 2];
              z2 = pack2(max_nan(__uint_as_float(q % 2 ? x.z : x.x), low), max_nan(__uint_as_float(q % 2 ? x.w : x.y), low));
            } else {
              const uint4& x = v[u][0];
              const uint32_t c = max_nan_bf16x2(q == 0 ? x.x : q == 1 ? x.y : q == 2 ? x.z : x.w, low2);
              z2 = pack2(__uint_as_float(c << 16), __uint_as_float(c & 0xffff0000u));
            }
            const uint64_t x2 = add2(fma2(z2, log2e, nref), nrest);
            const float2 x = unpack2(x2);
            o[q] = mul2(pack2(exp2_fast(x.x), exp2_fast(x.y)), fma2(x2, slope, base));
          }
          if (unit >= 0 && unit / kUnit == (u0 + u) * 32 + lane) {
#pragma unroll
            for (int q = 0; q < kUnit / 2; ++q) {
              float2 x = unpack2(o[q]);
              if (g.id == i + 2 * q) x.x = g.value(element<TI>(v[u], 2 * q), g.id);
              if (g.id == i + 2 * q + 1) x.y = g.value(element<TI>(v[u], 2 * q + 1), g.id);
              o[q] = pack2(x.x, x.y);
            }
          }
        }
        store_unit(d + i, o);
      } else if (i < V) {
        for (int e = max(i, 0); e < min(i + kUnit, V); ++e) d[e] = from_f<TO>(live ? g.value(to_f(z[e]), e) : 0.f);
      }
    }
  }
}

template <typename T, bool kTop>
cudaLaunchConfig_t stats_config(unsigned clusters, int cs, cudaStream_t stream, cudaLaunchAttribute (&attr)[2]) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(clusters * static_cast<unsigned>(cs));
  cfg.blockDim = dim3(block_threads<kTop>());
  cfg.dynamicSmemBytes = shared_bytes<kTop>();
  cfg.stream = stream;
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
template <typename T, bool kTop>
int clusters_held(int dev, int bits) {
  static std::atomic<int> held[64][4];  // and one more; host threads may ask at once
  if (const int known = held[dev][bits]; known > 0) return known - 1;
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = stats_config<T, kTop>(1, 1 << bits, nullptr, attr);
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, token_stats_kernel<T, kTop, true>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  held[dev][bits] = n + 1;
  return n;
}

// How many CTAs share a row (as a power of two): the most of which the device holds a cluster for every row, where a row
// is long enough. Of one / two / four / eight CTAs, us in a graph, 32 KB a row: 1 x 8000 fp32 3.3 / 3.3 / 3.3 / 3.1,
// 75 rows 3.4 / 3.3 / 3.9 / -; 64 KB: 1 x 32000 bf16 4.5 / 3.9 / 3.4 / 3.3, 75 rows 5.8 / 5.0 / 5.3 / -; 512 KB: 37 x
// 128001 fp32 18.0 / 11.5 / 8.5 / 7.6. With eight tokens, whose lists are merged: 32 KB 5.8 / 6.1 / 6.1 / 6.3, 64 KB 7.2 /
// 6.9 / 6.4 / 6.7, 125 KB 8.2 / 7.4 / 6.6 / 6.4; 75 rows of 64 KB (fp32) 7.5 / 7.7 / -, of 125 KB 9.2 / 8.9 / -.
template <typename T, bool kTop>
int cluster_bits(int64_t rows, int64_t V, int dev) {
  constexpr int64_t kLeast[] = {0, (kTop ? 120 : 48) * 1024, 48 * 1024, (kTop ? 96 : 31) * 1024};
  for (int bits = 3; bits > 0; --bits)
    if (V * static_cast<int64_t>(sizeof(T)) >= kLeast[bits] && rows <= clusters_held<T, kTop>(dev, bits)) return bits;
  return 0;
}

template <typename T>
int launch_short(const TokenStatsArgs& a, cudaStream_t stream) {
  const int64_t rows = a.S * a.L;
  return launch_pdl(token_stats_short_kernel<T>, dim3(static_cast<unsigned>((rows + kShortWarps - 1) / kShortWarps)),
                    dim3(kShortWarps * 32), 0, stream, static_cast<const T*>(a.logits), static_cast<long long>(a.ld),
                    static_cast<unsigned>(rows), static_cast<unsigned>(a.L), static_cast<int>(a.V), a.ids, a.lengths,
                    Outputs{a.logp, a.entropy, a.norm, nullptr, nullptr, 0}, a.err) == cudaSuccess
             ? 0
             : -3;
}

// Whether rows go to a warp each: those that it has under way at once (600 x 1000 fp32 3.4 -> 2.5 us, 8000 x 1000
// 20.0 -> 9.9, 30000 x 500 bf16 69 -> 30), and of many rows longer ones (2000 x 4000 fp32 10.5 -> 9.1 us, 30000 x 2000
// 79 -> 41, 2000 x 6000 13.5 -> 11.9; but 2000 x 12000 19.3 and 20.4, 600 x 4000 5.3 and 7.0).
template <typename T>
bool rows_are_short(int64_t rows, int64_t V) {
  const int64_t bytes = V * static_cast<int64_t>(sizeof(T));
  if (bytes <= 32 * kShortSlots * 16) return true;
  // (and no lane adds more than 128 terms one after another)
  return bytes <= 24 * 1024 && V <= 8192 && rows > 2 * static_cast<int64_t>(ctas_per_sm<false>()) * std::max(1, sm_count());
}

template <typename T, bool kTop>
int launch_stats(const TokenStatsArgs& a, cudaStream_t stream) {
  static std::atomic<bool> attr_set[64];  // the shared-memory limit is a per-device attribute
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return -1;
  if (!attr_set[dev]) {
    for (auto* kernel : {token_stats_kernel<T, kTop, false>, token_stats_kernel<T, kTop, true>})
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(shared_bytes<kTop>())) !=
          cudaSuccess)
        return -1;
    attr_set[dev] = true;
  }
  const int64_t rows = a.S * a.L;
  const int bits = cluster_bits<T, kTop>(rows, a.V, dev);
  const int64_t resident = static_cast<int64_t>(ctas_per_sm<kTop>()) * std::max(1, sm_count());
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg =
      stats_config<T, kTop>(static_cast<unsigned>(bits > 0 ? rows : std::min(rows, resident)), 1 << bits, stream, attr);
  const auto kernel = bits > 0 ? token_stats_kernel<T, kTop, true> : token_stats_kernel<T, kTop, false>;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<const T*>(a.logits),
                            static_cast<long long>(a.ld), static_cast<unsigned>(rows), static_cast<unsigned>(a.L),
                            static_cast<int>(a.V), a.ids, a.lengths, static_cast<unsigned>(bits),
                            Outputs{a.logp, a.entropy, a.norm, a.top_ids, a.top_logp, static_cast<int>(a.top_k)},
                            a.err) == cudaSuccess
             ? 0
             : -3;
}

template <typename TI, typename TO>
int launch_grad(const TokenStatsGradArgs& a, cudaStream_t stream) {
  const int64_t tiles = token_stats_grad_tiles(a.V), items = a.S * a.L * tiles;
  // few tiles: on as many multiprocessors as there are
  const int64_t warps = std::min<int64_t>(kGradWarps, (items - 1) / std::max(1, sm_count()) + 1);
  return launch_pdl(token_stats_grad_kernel<TI, TO>, dim3(static_cast<unsigned>((items + warps - 1) / warps)),
                    dim3(static_cast<unsigned>(warps * 32)), 0, stream, static_cast<const TI*>(a.logits), static_cast<long long>(a.ld),
                    static_cast<unsigned>(a.L), static_cast<int>(a.V), static_cast<unsigned>(tiles),
                    static_cast<unsigned>(items), a.ids, a.lengths, a.norm, a.entropy, a.grad_logp, a.grad_entropy,
                    static_cast<TO*>(a.dlogits), static_cast<long long>(a.ld_d), a.err) == cudaSuccess
             ? 0
             : -3;
}

}  // namespace

int launch_token_stats(const TokenStatsArgs& a, cudaStream_t stream) {
  if (a.top_k > 0) return a.bf16 ? launch_stats<__nv_bfloat16, true>(a, stream) : launch_stats<float, true>(a, stream);
  const int64_t rows = a.S * a.L;
  if (a.bf16)
    return rows_are_short<__nv_bfloat16>(rows, a.V) ? launch_short<__nv_bfloat16>(a, stream)
                                                    : launch_stats<__nv_bfloat16, false>(a, stream);
  return rows_are_short<float>(rows, a.V) ? launch_short<float>(a, stream) : launch_stats<float, false>(a, stream);
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
