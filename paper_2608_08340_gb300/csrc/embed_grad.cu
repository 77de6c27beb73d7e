// Gradient of the embedding tail y = m / |m|, m = the mean of a text's real hidden
// states: dm = (g - y (y . g)) / |m| for the gradient g of y, and dm / c for each of
// the text's c real tokens, 0 for its padding.  A text without real tokens, or with
// m = 0, has no gradient; a mean that is infinite or not a number has one that is not a
// number.
//
// Bound by HBM writes: batch x tokens x dim values from two rows per text.  A CTA forms
// the text's row in shared memory, rounded, and copies it to a chunk of its tokens; the
// sums over the row are formed again by every chunk's CTA (its rows come from L2).
// 256 x 512 x 4096 bf16: 156 us, 6.9 TB/s; values formed again per token took 258.
#include <cmath>

#include "internal.h"
#include "values.cuh"

namespace oprag {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxDim = 16384;
// Squared norms between which neither the squares nor the products with a gradient lose
// what counts: a value whose square is lost is below 2^-54 of the norm.
constexpr float kLeast = 0x1p-40f, kMost = 0x1p40f;

template <typename T>
__device__ __forceinline__ void load4(const T* src, float (&v)[4]) {
  if constexpr (sizeof(T) == 2) {
    const uint2 w = __ldg(reinterpret_cast<const uint2*>(src));
    v[0] = __uint_as_float(w.x << 16);
    v[1] = __uint_as_float(w.x & 0xFFFF0000u);
    v[2] = __uint_as_float(w.y << 16);
    v[3] = __uint_as_float(w.y & 0xFFFF0000u);
  } else {
    const float4 w = __ldg(reinterpret_cast<const float4*>(src));
    v[0] = w.x;
    v[1] = w.y;
    v[2] = w.z;
    v[3] = w.w;
  }
}

template <typename TIn, typename TOut>
__global__ void __launch_bounds__(kThreads)
embed_pool_grad_kernel(const TIn* __restrict__ grad, const float* __restrict__ mean, int tokens,
                       int dim, const uint8_t* __restrict__ mask, TOut* __restrict__ out,
                       int chunk, bool per_token) {
  extern __shared__ __align__(16) unsigned char shared[];
  TOut* row = reinterpret_cast<TOut*>(shared);
  __shared__ float sums[3][kWarps];
  __shared__ uint32_t tops[kWarps];
  const int64_t b = blockIdx.x;
  const float* m = mean + b * dim;
  const TIn* g = grad + b * dim;
  const uint8_t* mrow = mask + b * tokens;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // (m / 2^e) . (m / 2^e), (m / 2^e) . g and the real tokens.
  float part[3];
  auto add_up = [&](int e) {
    part[0] = part[1] = part[2] = 0.f;
    for (int i = 4 * threadIdx.x; i < dim; i += 4 * kThreads) {
      float x[4], y[4];
      load4(m + i, x);
      load4(g + i, y);
#pragma unroll
      for (int l = 0; l < 4; ++l) {
        if (e != 0) x[l] = scalbnf(x[l], -e);
        part[0] = fmaf(x[l], x[l], part[0]);
        part[1] = fmaf(x[l], y[l], part[1]);
      }
    }
    for (int t = threadIdx.x; t < tokens; t += kThreads) part[2] += mrow[t] != 0 ? 1.f : 0.f;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) part[k] += __shfl_xor_sync(0xffffffffu, part[k], o);
      if (lane == 0) sums[k][warp] = part[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      part[k] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) part[k] += sums[k][w];
    }
  };
  add_up(0);
  // A mean whose squares may leave the range is taken as 2^e (m / 2^e), its largest
  // magnitude being in [2^e, 2^(e + 1)): no rounding, so the same bits as without.
  int e = 0;
  if (part[2] > 0.f && !(part[0] >= kLeast && part[0] <= kMost)) {
    uint32_t top = 0;                             // (ordered as the magnitudes are)
    for (int i = threadIdx.x; i < dim; i += kThreads) top = max(top, __float_as_uint(fabsf(m[i])));
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) tops[warp] = top;
    __syncthreads();                              // (the sums are read)
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = max(top, tops[w]);
    if (top >= __float_as_uint(INFINITY)) {       // infinite, or not a number: no direction
      part[0] = NAN;
    } else if (top != 0) {
      e = ilogbf(__uint_as_float(top));
      add_up(e);
    }
  }
  const float mm = part[0], mg = part[1], real = part[2];
  const bool there = real > 0.f && mm != 0.f;     // (what is not a number is passed on)
  const float by = there ? 1.f / (real * sqrtf(mm)) : 0.f;
  const float along = there ? mg / mm : 0.f;      // (y . g) / (|m| / 2^e)
  for (int i = 4 * threadIdx.x; i < dim; i += 4 * kThreads) {
    float x[4], y[4];
    load4(m + i, x);
    load4(g + i, y);
#pragma unroll
    for (int l = 0; l < 4; ++l) {
      if (e != 0) x[l] = scalbnf(x[l], -e);
      y[l] = there ? (y[l] - x[l] * along) * by : 0.f;
      if (e != 0) y[l] = scalbnf(y[l], -e);
    }
    store_values(row + i, y);
  }
  __syncthreads();
  constexpr int N = 16 / sizeof(TOut);
  const int groups = dim / N;
  const uint4* src = reinterpret_cast<const uint4*>(row);
  if (!per_token) {
    uint4* dst = reinterpret_cast<uint4*>(out + b * dim);
    for (int i = threadIdx.x; i < groups; i += kThreads) dst[i] = src[i];
    return;
  }
  // The chunk's (token, group) pairs, one after the other.
  const int t0 = blockIdx.y * chunk, t1 = min(tokens, t0 + chunk);
  uint4* dst = reinterpret_cast<uint4*>(out + (b * tokens + t0) * dim);
  int t = t0 + threadIdx.x / groups, i = threadIdx.x % groups;
  const int step_t = kThreads / groups, step_i = kThreads % groups;
#pragma unroll 4
  for (int64_t at = threadIdx.x; t < t1; at += kThreads) {
    const bool is_real = __ldg(mrow + t) != 0;
    __stcs(dst + at, is_real ? src[i] : make_uint4(0, 0, 0, 0));
    t += step_t;
    i += step_i;
    if (i >= groups) {
      i -= groups;
      ++t;
    }
  }
}

template <typename TIn, typename TOut>
cudaError_t launch_typed(const void* grad, const float* mean, int batch, int tokens, int dim,
                         const uint8_t* mask, void* out, bool per_token, cudaStream_t st) {
  static DeviceOnce once;
  const cudaError_t e = allow_smem(once, embed_pool_grad_kernel<TIn, TOut>, kMaxDim * sizeof(TOut));
  if (e != cudaSuccess) return e;
  // Chunks of 8 to 64 tokens: eight CTAs for each of 152 SMs where there are enough.
  const int64_t share = (static_cast<int64_t>(batch) * tokens + 8 * 152 - 1) / (8 * 152);
  int chunk = static_cast<int>(share < 8 ? 8 : share > 64 ? 64 : share);
  // (a grid has at most 65535 chunks)
  if ((tokens + chunk - 1) / chunk > 65535) chunk = (tokens + 65534) / 65535;
  const dim3 grid(batch, per_token ? (tokens + chunk - 1) / chunk : 1);
  embed_pool_grad_kernel<TIn, TOut><<<grid, kThreads, dim * sizeof(TOut), st>>>(
      static_cast<const TIn*>(grad), mean, tokens, dim, mask, static_cast<TOut*>(out), chunk,
      per_token);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_embed_pool_grad(const void* grad, int grad_dtype, const float* mean, int batch,
                                   int tokens, int dim, const uint8_t* mask, void* out,
                                   int out_dtype, bool per_token, cudaStream_t st) {
  if (batch <= 0) return cudaSuccess;
  const bool in16 = grad_dtype == kBF16, out16 = out_dtype == kBF16;
  if (in16)
    return out16 ? launch_typed<uint16_t, uint16_t>(grad, mean, batch, tokens, dim, mask, out, per_token, st)
                 : launch_typed<uint16_t, float>(grad, mean, batch, tokens, dim, mask, out, per_token, st);
  return out16 ? launch_typed<float, uint16_t>(grad, mean, batch, tokens, dim, mask, out, per_token, st)
               : launch_typed<float, float>(grad, mean, batch, tokens, dim, mask, out, per_token, st);
}

}  // namespace oprag
