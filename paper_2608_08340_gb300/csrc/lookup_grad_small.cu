// Gradient of an embedding lookup of few tokens (lookup_grad.cu holds the
// formula): nearly all of the work is writing zeros, so one launch does it without a sort.
// A CTA owns every C-th row of the table, for C CTAs (so that the common tokens' rows,
// which are often neighbours, fall to different ones), and 1024 columns.  It reads all
// ids, lists those of its rows in the tokens' order, and a warp takes a row at a time: the
// row's tokens are picked from the list by ballots and added in order.  Rows with more
// than four tokens are split over the CTA's warps and joined in shared memory, in order.
//
// Bound by the table's bytes and one launch: 256 tokens into 30522 x 768 fp32 rows (94 MB,
// 13.9 us of HBM) 24 us.  One CTA adds up a row, however many tokens it has: 1024 of one row
// of 768 columns take 103 us, which is one reason for the limit (few_tokens), and 16 texts of
// 64 tokens padded with one id of the table 72 us, with -1 36.
#include "lookup_grad.cuh"
#include "values.cuh"

namespace oprag {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kColumns = kSmallColumns;           // of a CTA
constexpr int kSpan = 2;                          // blocks of 128 columns that a warp adds together
constexpr int kMaxRows = 256;                     // of a CTA
constexpr int kSplitFrom = 4;                     // tokens of a row that one warp adds
constexpr int kPerThread = kSmallTokens / kThreads;

template <typename TIn, typename TOut, typename TId>
__global__ void __launch_bounds__(kThreads, 3) small_grad_kernel(LookupGradArgs a) {
  using Raw = typename Four<TIn>::Raw;
  constexpr int E = sizeof(TIn) == 2 ? 8 : 4;     // tokens whose rows fly together
  __shared__ uint32_t list[kSmallTokens];         // the CTA's row << 16 | token
  __shared__ int count[kMaxRows];
  __shared__ int warp_total[kWarps];
  __shared__ float4 part[kWarps][kColumns / 4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t vocab = static_cast<uint32_t>(a.vocab), ctas = gridDim.x;
  const int rows = static_cast<int>((vocab - blockIdx.x + ctas - 1) / ctas);
  const int n = static_cast<int>(a.count);
  const int group0 = blockIdx.y * (kColumns / 4);
  const int limit = min(a.dim / 4, group0 + kColumns / 4);        // of this CTA's groups
  const int blocks = (limit - group0 + 31) / 32;
  const TId* ids = static_cast<const TId*>(a.ids);

  // The list: thread i has tokens i * each ... + each - 1.
  for (int r = tid; r < kMaxRows; r += kThreads) count[r] = 0;
  const int each = (n + kThreads - 1) / kThreads;
  uint32_t mine[kPerThread];
  int found = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int t = tid * each + i;
    mine[i] = 0xFFFFFFFFu;
    if (i < each && t < n) {
      const int64_t id = ids[t];
      const uint32_t v = id >= 0 && id < vocab ? static_cast<uint32_t>(id) : 0xFFFFFFFFu;
      const uint32_t r = v / ctas;
      if (v < vocab && v - r * ctas == blockIdx.x) {
        mine[i] = r << 16 | static_cast<uint32_t>(t);
        ++found;
      }
    }
  }
  int at = found;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, at, o);
    if (lane >= o) at += y;
  }
  if (lane == 31) warp_total[warp] = at;
  __syncthreads();
  int listed = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) at += warp_total[w];
    listed += warp_total[w];
  }
  at -= found;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i)
    if (mine[i] != 0xFFFFFFFFu) {
      list[at++] = mine[i];
      atomicAdd(&count[mine[i] >> 16], 1);
    }
  __syncthreads();

  // Adds the tokens of row r with ordinals [from, to) to this lane's 4 columns of blocks
  // b0 ... b0 + kSpan - 1.
  const TIn* grad = static_cast<const TIn*>(a.grad);
  auto add = [&](int r, int from, int to, int b0, float (&acc)[kSpan][4]) {
    const int g0 = group0 + b0 * 32 + lane;
    int seen = 0;
    for (int base = 0; base < listed && seen < to; base += 32) {
      const uint32_t e = base + lane < listed ? list[base + lane] : 0xFFFFFFFFu;
      const bool is_row = static_cast<int>(e >> 16) == r;
      uint32_t m = __ballot_sync(0xffffffffu, is_row);
      const int matches = __popc(m);
      if (seen + matches > from) {
        int64_t offset = 0;
        if (is_row) {
          const uint32_t t = e & 0xFFFFu, tokens = static_cast<uint32_t>(a.tokens);
          offset = t / tokens * a.text_stride + t % tokens * a.token_stride;
        }
        for (int skip = from - seen; skip > 0; --skip) m &= m - 1;
        int left = min(__popc(m), to - max(seen, from));
        while (left > 0) {
          Raw v[E][kSpan];
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const int64_t o = __shfl_sync(0xffffffffu, offset, m != 0 ? __ffs(m) - 1 : 0);
            m &= m - 1;
            const Raw* src = reinterpret_cast<const Raw*>(grad + o);
#pragma unroll
            for (int b = 0; b < kSpan; ++b)
              if (k < left && g0 + 32 * b < limit) v[k][b] = __ldg(src + g0 + 32 * b);
          }
#pragma unroll
          for (int k = 0; k < E; ++k)
#pragma unroll
            for (int b = 0; b < kSpan; ++b)
              if (k < left && g0 + 32 * b < limit) Four<TIn>::add(v[k][b], acc[b]);
          left -= E;
        }
      }
      seen += matches;
    }
  };
  auto put = [&](int r, int g, float (&acc)[4]) {
    if (g >= limit) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] *= a.scale;
    const int64_t v = blockIdx.x + static_cast<int64_t>(r) * ctas;
    store_values(static_cast<TOut*>(a.out) + v * a.dim + 4 * g, acc);
  };

  bool split = false;
  for (int r = warp; r < rows; r += kWarps) {
    const int c = count[r];
    if (c == 0) continue;
    if (c > kSplitFrom) {
      split = true;
      continue;
    }
    for (int b0 = 0; b0 < blocks; b0 += kSpan) {
      float acc[kSpan][4] = {};
      add(r, 0, c, b0, acc);
#pragma unroll
      for (int b = 0; b < kSpan; ++b) put(r, group0 + (b0 + b) * 32 + lane, acc[b]);
    }
  }
  split = __syncthreads_or(split);
  for (int r = 0; split && r < rows; ++r) {
    const int c = count[r];
    if (c <= kSplitFrom) continue;
    for (int b0 = 0; b0 < blocks; b0 += kSpan) {
      float acc[kSpan][4] = {};
      add(r, c * warp / kWarps, c * (warp + 1) / kWarps, b0, acc);
#pragma unroll
      for (int b = 0; b < kSpan; ++b)
        part[warp][(b0 + b) * 32 + lane] = make_float4(acc[b][0], acc[b][1], acc[b][2], acc[b][3]);
    }
    __syncthreads();
    if (tid < blocks * 32) {
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 v = part[w][tid];
        acc[0] += v.x;
        acc[1] += v.y;
        acc[2] += v.z;
        acc[3] += v.w;
      }
      put(r, group0 + tid, acc);
    }
    __syncthreads();
  }
  // Rows without tokens, at the end: their stores keep HBM busy while other CTAs wait.
  {
    constexpr int N = 16 / sizeof(TOut);
    const int per_row = (limit - group0) * 4 / N;         // 16-byte stores
    for (int r = warp; r < rows; r += kWarps) {
      if (count[r] != 0) continue;
      uint4* dst = reinterpret_cast<uint4*>(
          static_cast<TOut*>(a.out) + (blockIdx.x + static_cast<int64_t>(r) * ctas) * a.dim + 4 * group0);
      for (int i = lane; i < per_row; i += 32) dst[i] = make_uint4(0, 0, 0, 0);
    }
  }
}

template <typename TIn, typename TOut>
cudaError_t launch_typed(const LookupGradArgs& a, cudaStream_t st) {
  const int64_t slabs = (a.dim + kColumns - 1) / kColumns;
  // Three CTAs (all that fit) for each of 152 SMs, as far as there are rows.
  int64_t ctas = 3 * 152 / slabs;
  if (ctas < (a.vocab + kMaxRows - 1) / kMaxRows) ctas = (a.vocab + kMaxRows - 1) / kMaxRows;
  if (ctas > a.vocab) ctas = a.vocab;
  const dim3 grid(static_cast<unsigned>(ctas), static_cast<unsigned>(slabs));
  if (a.ids64)
    small_grad_kernel<TIn, TOut, int64_t><<<grid, kThreads, 0, st>>>(a);
  else
    small_grad_kernel<TIn, TOut, int32_t><<<grid, kThreads, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_lookup_grad_small(const LookupGradArgs& a, cudaStream_t st) {
  const bool in16 = a.grad_dtype == kBF16, out16 = a.out_dtype == kBF16;
  if (in16)
    return out16 ? launch_typed<uint16_t, uint16_t>(a, st) : launch_typed<uint16_t, float>(a, st);
  return out16 ? launch_typed<float, uint16_t>(a, st) : launch_typed<float, float>(a, st);
}

}  // namespace oprag
