// Distillation from search results.  For a row z of n student scores and the
// teacher's k results (id_j, s_j), at temperature T:
//   t = softmax over the results that take part of s_j / T,
//   p = softmax over the n chunks of z / T,
//   loss = sum_j t_j (log t_j - log p[id_j]),   dloss/dz = (p - t) / T.
// A result takes part if its id is a chunk's, its score is above -inf and the
// student's score of that chunk is above its type's lowest value (this value and -inf
// hide a chunk from the row).  A row without such a result has loss 0 and no gradient.
//
// Bound by HBM: a row is read once and its gradient written once.  A row belongs to a
// cluster of 1 to 16 CTAs.  Each thread copies its own 16-byte groups with cp.async into its
// own places in shared memory and reads them itself, so that no barrier guards them; with
// the maximum m_i that thread i saw and its sum s_i of e^((z - m_i) / T), one reduction of
// the pairs (m, s), through distributed shared memory where a cluster has several CTAs,
// gives the row's.  The gradient then goes backwards over the row: the last batches are
// still in shared memory, the ones before come from L2, where the most recent are
// likeliest to be.  256 rows of 2^20 bf16 scores: 228 us, 4.7 TB/s of the bytes that are
// needed (DRAM reads 1.2 times the rows), the loss alone 110; 1024 x 32768 fp32 60 us (38);
// 300 x 50021 bf16 19 to 22 us (15): one wave that fills half of the places, whose CTAs all
// read first and all write last.  About 90 instructions per group keep the issue slots half
// busy; barriers and first loads of many small CTAs are the rest.
//
// Tried: rows kept whole in one CTA per SM (26 groups a thread), the next row's copies
// flying meanwhile: 433 us for the first, 103 for the second line; persistent CTAs that
// fetch the next row's first batches: 249 and 63 us; the teacher's results by a warp
// of their own: 249 and 64; scalar instead of packed fp32 arithmetic: 244 and 64.
#include <cooperative_groups.h>

#include <cmath>

#include "common.cuh"
#include "internal.h"
#include "values.cuh"

namespace cg = cooperative_groups;

namespace oprag {

namespace {

constexpr float kLog2e = 1.44269504088896341f;

// e^((z - m) / T) = 2^((z - m) c): a difference, a product and the approximation of 2^x
// (2^-22 relatively).  The difference comes first, so that scores near the end of the range
// and their maximum cancel.
__device__ __forceinline__ float exp_diff(float z, float m, float c) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"((z - m) * c));
  return r;
}

// Two floats in a 64-bit register, for the packed fp32 instructions.
using Two = uint64_t;

__device__ __forceinline__ Two two(float lo, float hi) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split(Two v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ Two add2(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// exp_diff of both, with (-m, -m) and (c, c).
__device__ __forceinline__ Two exp_diff2(Two z, Two minus_m, Two c) {
  float lo, hi;
  split(mul2(add2(z, minus_m), c), lo, hi);
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(lo));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(hi));
  return two(lo, hi);
}

// A 16-byte group of scores as pairs, and a running maximum of groups.
template <typename T>
struct Group;
template <>
struct Group<uint16_t> {
  static constexpr int kPairs = 4;
  using Max = __nv_bfloat162;
  __device__ __forceinline__ static void unpack(const uint4& g, Two (&v)[4]) {
    const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = two(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
  __device__ __forceinline__ static uint4 pack(const Two (&v)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      split(v[i], lo, hi);
      const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ static Max lowest() {
    return __halves2bfloat162(__ushort_as_bfloat16(0xFF7F), __ushort_as_bfloat16(0xFF7F));
  }
  __device__ __forceinline__ static void raise(Max& m, const uint4& g) {
    const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __hmax2(m, *reinterpret_cast<const __nv_bfloat162*>(&w[i]));
  }
  __device__ __forceinline__ static float value(const Max& m) {
    return fmaxf(__low2float(m), __high2float(m));
  }
};
template <>
struct Group<float> {
  static constexpr int kPairs = 2;
  using Max = float;
  __device__ __forceinline__ static void unpack(const uint4& g, Two (&v)[2]) {
    v[0] = two(__uint_as_float(g.x), __uint_as_float(g.y));
    v[1] = two(__uint_as_float(g.z), __uint_as_float(g.w));
  }
  __device__ __forceinline__ static uint4 pack(const Two (&v)[2]) {
    float a, b, c, d;
    split(v[0], a, b);
    split(v[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
  __device__ __forceinline__ static Max lowest() { return Values<float>::kLowest; }
  __device__ __forceinline__ static void raise(Max& m, const uint4& g) {
    m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(g.x)), __uint_as_float(g.y)),
              fmaxf(__uint_as_float(g.z), __uint_as_float(g.w)));
  }
  __device__ __forceinline__ static float value(const Max& m) { return m; }
};

// A maximum (no less than the lowest finite value, so that -inf less it is -inf) and
// the sum of e^((z - max) / T).
struct MaxSum {
  float m, s;
};

__device__ __forceinline__ MaxSum warp_join(MaxSum x, float c) {
  float m = x.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float s = x.s * exp_diff(x.m, m, c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return {m, s};
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// The part of a row that a CTA of a cluster has: `head` single values before the first
// 16-byte boundary (rank 0), groups [g0, g1) and `tail` single values behind the last
// (last rank); elements [from, to) of the row.
struct Part {
  int head, tail;           // of this CTA
  int groups;
  int body;                 // element of the first group
  int from, to;
};

template <typename T>
__device__ __forceinline__ Part part_of(const T* z, int n, int rank, int ctas) {
  constexpr int N = Values<T>::kN;
  const int misaligned = static_cast<int>(reinterpret_cast<uintptr_t>(z) & 15) / static_cast<int>(sizeof(T));
  const int head = min(n, misaligned == 0 ? 0 : N - misaligned);
  const int groups = (n - head) / N;
  const int each = static_cast<int>(static_cast<uint32_t>(groups + ctas - 1) / static_cast<uint32_t>(ctas));
  const int g0 = min(groups, rank * each), g1 = min(groups, g0 + each);
  Part p;
  p.head = rank == 0 ? head : 0;
  p.tail = rank == ctas - 1 ? n - head - groups * N : 0;
  p.groups = g1 - g0;
  p.body = head + g0 * N;
  p.from = rank == 0 ? 0 : p.body;
  p.to = rank == ctas - 1 ? n : head + g1 * N;
  return p;
}

// Stores a group of the gradient, whose rows may lie on other boundaries than the scores'.
template <typename T>
__device__ __forceinline__ void store_group(T* dst, const uint4& v, bool aligned) {
  if (aligned) {
    __stcs(reinterpret_cast<uint4*>(dst), v);
  } else {
    const T* one = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int i = 0; i < Values<T>::kN; ++i) dst[i] = one[i];
  }
}

constexpr int kBatch = 4;                         // groups of a thread that are copied together
constexpr int kMaxCluster = 16;
constexpr int64_t kShare = 96 << 10;              // bytes of a row that a CTA takes at most ...
constexpr int64_t kSmallRow = 1 << 20;            // ... up to this many bytes of a row

__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(src)
               : "memory");
}
__device__ __forceinline__ void copies_begin() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All copies are there but those of the last N batches.
template <int N>
__device__ __forceinline__ void copies_but() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A cluster per row.  kCtas CTAs share an SM; a thread has kRing batches in shared memory
// and E of the teacher's results.
template <typename T, int Threads, int kCtas, int kRing, int E>
__global__ void __launch_bounds__(Threads, kCtas) distill_kernel(DistillArgs a) {
  constexpr int N = Values<T>::kN, P = Group<T>::kPairs, kWarps = Threads / 32;
  constexpr int kPlaces = 2 * E * Threads;
  constexpr unsigned short kNone = 0xFFFF;
  extern __shared__ __align__(16) uint4 ring[];
  __shared__ int ids[E * Threads];        // of the results that take part, else -1
  __shared__ float shares[E * Threads];
  // By hashing: a result that has the id, or kNone (cleared as words).
  __shared__ __align__(16) unsigned short met[kPlaces];
  __shared__ MaxSum warps[kWarps], teachers[kWarps], parts[kMaxCluster];
  __shared__ float terms[kWarps];
  __shared__ int repeated;                // an id that two results have
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = static_cast<int>(cluster.num_blocks());
  const int rank = static_cast<int>(cluster.block_rank());
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (ctas > 1) cluster.barrier_arrive(); // (this CTA has begun: its peers may write to parts)
  const float c = kLog2e / a.temperature;
  const Two c2 = two(c, c);
  const int64_t row = blockIdx.x / static_cast<unsigned>(ctas);
  const T* z = static_cast<const T*>(a.logits) + row * a.row_stride;
  const Part p = part_of(z, a.n, rank, ctas);
  const bool has_extra = tid < p.head + p.tail;
  const int extra_at = tid < p.head ? tid : p.to - p.tail + tid - p.head;
  // This thread's groups tid, tid + Threads, ..., in batches; batch b is in place b mod kRing.
  const int count = tid < p.groups ? (p.groups - tid + Threads - 1) / Threads : 0;
  const int batches = (count + kBatch - 1) / kBatch;
  const uint4* body = reinterpret_cast<const uint4*>(z + p.body) + tid;
  auto place = [&](int b) { return ring + (b % kRing) * (kBatch * Threads) + tid; };
  auto fetch = [&](int b, uint4* to) {
    const uint4* from = body + b * (kBatch * Threads);
    if (b >= 0 && (b + 1) * kBatch <= count) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) copy_async(to + u * Threads, from + u * Threads);
    } else if (b >= 0) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (b * kBatch + u < count) copy_async(to + u * Threads, from + u * Threads);
    }
    copies_begin();
  };
#pragma unroll
  for (int b = 0; b < kRing; ++b) fetch(b, place(b));

  // The teacher's results, E for a thread; the other warps have none.
  const bool teaches = warp * 32 < a.k;
  const float weight = a.weight != nullptr ? a.weight[row] : 1.f;
  const float extra = has_extra ? Values<T>::one(z[extra_at]) : -INFINITY;
  int id[E];
  float s[E], zt[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    id[e] = -1;
    s[e] = zt[e] = 0.f;
  }
  if (teaches) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = e * Threads + tid;
      const int64_t v = j < a.k ? a.ids[row * a.k + j] : -1;
      s[e] = j < a.k ? a.scores[row * a.k + j] : 0.f;
      id[e] = v >= 0 && v < a.n && !(s[e] == -INFINITY) ? static_cast<int>(v) : -1;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (id[e] >= 0) zt[e] = Values<T>::one(z[id[e]]);
  }
  for (int i = tid; i < kPlaces / 2; i += Threads) reinterpret_cast<uint32_t*>(met)[i] = 0xFFFFFFFFu;
  if (tid == 0) repeated = 0;

  // The row's maximum and sum.
  float m = fmaxf(Values<T>::kLowest, extra);
  Two total = two(0.f, 0.f);
  auto add_batch = [&](const uint4* at, int groups) {
    auto top = Group<T>::lowest();
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (u < groups) Group<T>::raise(top, at[u * Threads]);
    const float higher = fmaxf(m, Group<T>::value(top)), by = exp_diff(m, higher, c);
    total = mul2(total, two(by, by));
    m = higher;
    const Two minus_m = two(-m, -m);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (u >= groups) continue;
      Two v[P];
      Group<T>::unpack(at[u * Threads], v);
#pragma unroll
      for (int l = 0; l < P; ++l) total = add2(total, exp_diff2(v[l], minus_m, c2));
    }
  };
  for (int b = 0; b < batches; ++b) {
    uint4* at = place(b);
    copies_but<kRing - 1>();
    if ((b + 1) * kBatch <= count)
      add_batch(at, kBatch);
    else
      add_batch(at, count - b * kBatch);
    // (the last kRing batches stay)
    fetch(b + kRing < batches ? b + kRing : -1, at);
  }
  float lo, hi;
  split(total, lo, hi);
  MaxSum x = warp_join({m, lo + hi + exp_diff(extra, m, c)}, c);
  MaxSum y{Values<float>::kLowest, 0.f};  // the same of the teacher's scores
  if (teaches) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (id[e] >= 0 && zt[e] <= Values<T>::kLowest) id[e] = -1;
      ids[e * Threads + tid] = id[e];
      if (id[e] >= 0) y.m = fmaxf(y.m, s[e]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (id[e] >= 0) y.s += exp_diff(s[e], y.m, c);
    y = warp_join(y, c);
  }
  if (lane == 0) {
    warps[warp] = x;
    teachers[warp] = y;
  }
  __syncthreads();
  x = warp_join(lane < kWarps ? warps[lane] : MaxSum{Values<T>::kLowest, 0.f}, c);
  y = warp_join(lane < kWarps ? teachers[lane] : MaxSum{Values<float>::kLowest, 0.f}, c);
  if (ctas > 1) {
    cluster.barrier_wait();               // long past: all CTAs of the cluster have begun
    if (warp == 0 && lane < ctas) *cluster.map_shared_rank(&parts[rank], lane) = x;
    cluster.sync();
    x = warp_join(lane < ctas ? parts[lane] : MaxSum{Values<T>::kLowest, 0.f}, c);
  }

  // The results' shares, their part of the loss, and the ids that repeat.
  float share[E];
  bool first[E];
  if (teaches) {
    const float log_mass = logf(y.s), log_sum = logf(x.s);
    float term = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = e * Threads + tid;
      share[e] = 0.f;
      first[e] = id[e] >= 0;
      if (id[e] >= 0) {
        share[e] = exp_diff(s[e], y.m, c) / y.s;
        if (share[e] != 0.f)                // (not a number: the loss is none)
          term += share[e] * (((s[e] - y.m) / a.temperature - log_mass) -
                              ((zt[e] - x.m) / a.temperature - log_sum));
        int h = static_cast<int>((static_cast<uint32_t>(id[e]) * 2654435761u >> 16) % kPlaces);
        while (true) {                    // (ends: half of the places stay free)
          const unsigned short old = atomicCAS(&met[h], kNone, static_cast<unsigned short>(j));
          if (old == kNone) break;
          if (ids[old] == id[e]) {
            first[e] = false;
            repeated = 1;
            break;
          }
          h = (h + 1) % kPlaces;
        }
      }
      shares[j] = share[e];
    }
    term = warp_sum(term);
    if (lane == 0) terms[warp] = term;
  }

  // The gradient, backwards: the last batches are still here, the ones before them
  // the likeliest in L2.
  T* g = static_cast<T*>(a.grad) + row * a.grad_stride;
  const float w = a.grad != nullptr && y.s != 0.f ? weight / a.temperature : 0.f;
  const float by = w != 0.f ? w / x.s : 0.f;
  if (a.grad != nullptr) {
    const bool aligned = (reinterpret_cast<uintptr_t>(g + p.body) & 15) == 0;
    const Two by2 = two(by, by), minus_m = two(-x.m, -x.m);
    T* dst = g + p.body + tid * N;
    auto put_batch = [&](const uint4* at, T* to, int groups) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (u >= groups) continue;
        Two v[P];
        Group<T>::unpack(at[u * Threads], v);
#pragma unroll
        for (int l = 0; l < P; ++l) v[l] = mul2(exp_diff2(v[l], minus_m, c2), by2);
        store_group(to + u * (Threads * N), Group<T>::pack(v), aligned);
      }
    };
    for (int b = batches - 1; b >= 0; --b) {
      uint4* at = place(b);
      T* to = dst + static_cast<int64_t>(b) * (kBatch * Threads * N);
      copies_but<kRing - 1>();
      if (w == 0.f) {                     // (whatever the scores are)
        for (int u = 0; u < kBatch && b * kBatch + u < count; ++u)
          store_group(to + u * (Threads * N), make_uint4(0, 0, 0, 0), aligned);
      } else if ((b + 1) * kBatch <= count) {
        put_batch(at, to, kBatch);
      } else {
        put_batch(at, to, count - b * kBatch);
      }
      if (b >= kRing)
        fetch(b - kRing, at);
      else
        copies_begin();
    }
    if (has_extra) g[extra_at] = Values<T>::pack_one(w != 0.f ? exp_diff(extra, x.m, c) * by : 0.f);
  }
  __syncthreads();
  if (tid == 0 && rank == 0) {
    float loss = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i)
      if (i * 32 < a.k) loss += terms[i];
    a.loss[row] = y.s != 0.f ? loss : 0.f;
  }
  if (w == 0.f || !teaches) return;
  // The results' chunks, over what was just written.
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (!first[e] || id[e] < p.from || id[e] >= p.to) continue;
    if (repeated != 0) {                  // the shares of the id, in order
      share[e] = 0.f;
      for (int j = 0; j < a.k; ++j)
        if (ids[j] == id[e]) share[e] += shares[j];
    }
    g[id[e]] = Values<T>::pack_one(exp_diff(zt[e], x.m, c) * by - w * share[e]);
  }
}

template <typename T, int Threads, int kCtas, int kRing, int E>
cudaError_t launch_rows(const DistillArgs& a, int ctas, cudaStream_t st) {
  constexpr size_t kBytes = static_cast<size_t>(kRing) * kBatch * Threads * 16;
  auto* kernel = distill_kernel<T, Threads, kCtas, kRing, E>;
  cudaLaunchConfig_t cfg{};
  cfg.blockDim = dim3(Threads);
  cfg.dynamicSmemBytes = kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  static DeviceOnce once, largest;
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  e = once.run(device, [&] {
    const cudaError_t r = cudaFuncSetAttribute(
        kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kBytes));
    return r != cudaSuccess ? r : cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
  if (e != cudaSuccess) return e;
  if (ctas > 8) {                         // eight where the device runs no larger cluster
    e = largest.run(device, [&] {
      attr[0].val.clusterDim.x = kMaxCluster;
      cfg.gridDim = dim3(kMaxCluster);
      int n = 0;
      const cudaError_t r = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
      if (r != cudaSuccess) cudaGetLastError();
      return r == cudaSuccess && n < 1 ? cudaErrorNotSupported : r;
    });
    if (e != cudaSuccess) ctas = 8;
  }
  attr[0].val.clusterDim.x = ctas;
  cfg.numAttrs = ctas > 1 ? 1 : 0;
  cfg.gridDim = dim3(static_cast<unsigned>(a.q) * ctas);
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

// CTAs of 128 threads, eight on an SM with 24 KB of a row each, take up to 96 KB of a
// row; a row of more than 1 MB is split over 16 CTAs of 256 threads, four on an SM with
// 48 KB each, so that the rows under way fit into L2 (some 50 MB hold).  Measured, us:
// 2048 rows of 31 KB 128 threads 30, 256 threads 34; 300 of 98 KB in 1 / 2 / 4 CTAs 23 / 17 / 21;
// 1024 of 128 KB 1 / 2 / 4 / 8 CTAs 71 / 61 / 59 / 70 (the limit of 96 KB favours the former); 2000 of 195 KB 4 / 8 CTAs 149 / 166; 256 of
// 586 KB 8 / 16 CTAs 72 / 77; 256 of 800 KB 4 / 8 / 16 CTAs 113 / 101 / 92; 256 of 2 MB 16 CTAs of 128
// and 256 threads 236 and 229, 8 of 512 threads 241.  16 KB of a row in a CTA's shared
// memory instead of 24: 195 KB rows 156, 800 KB rows 96.  Few rows are spread further, down
// to 16 KB a CTA: 4 rows of 2 MB with 1 / 4 / 16 CTAs of 256 threads 148 / 42 / 17.
template <typename T>
cudaError_t launch_typed(const DistillArgs& a, cudaStream_t st) {
  const int64_t bytes = static_cast<int64_t>(a.n) * sizeof(T);
  int dev = 0, sms = 1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  if (bytes > kSmallRow) return launch_rows<T, 256, 4, 3, 1>(a, kMaxCluster, st);
  int ctas = 1;
  while (ctas < kMaxCluster && bytes > ctas * kShare) ctas *= 2;
  while (ctas < 8 && 2 * static_cast<int64_t>(a.q) * ctas <= sms && bytes >= ctas * (32 << 10)) ctas *= 2;
  if (a.k > 128) return launch_rows<T, 128, 8, 3, 2>(a, ctas, st);
  return launch_rows<T, 128, 8, 3, 1>(a, ctas, st);
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, cudaStream_t st) {
  if (a.q <= 0) return cudaSuccess;
  return a.dtype == kBF16 ? launch_typed<uint16_t>(a, st) : launch_typed<float>(a, st);
}

}  // namespace oprag
