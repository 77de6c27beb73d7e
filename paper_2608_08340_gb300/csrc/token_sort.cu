// Stable sort of tokens by id (token_sort.cuh), a tile of 1024 or 4096 tokens per CTA.  A pass
// ranks every token among the tokens of its digit: a warp's 32 tokens by matching, the
// warps of a CTA by their counts per digit, the tiles by theirs.  One kernel counts
// the first digit per tile; a kernel per pass ranks and scatters, and counts the next digit
// of every token in the tile where it goes.  The first pass drops tokens whose id is
// outside the table.  Up to kSumTiles tiles a CTA of the second kernel adds the tiles'
// counts up itself; beyond, one more kernel per pass does.
//
// Bound by latency: the tokens' ids are a few hundred KB.  131072 tokens take three
// launches of 4, 10 and 8 us.  The same sort in one launch of one 16-CTA cluster, tokens
// exchanged through distributed shared memory, took 27 us (shared-memory latency on
// 16 of 152 SMs).
#include "internal.h"
#include "token_sort.cuh"

namespace oprag {

namespace {

constexpr int kItems = 8;                         // tokens of a thread
constexpr int kMaxDigits = 1 << kMaxDigitBits;
constexpr uint32_t kSumTiles = 128;
constexpr int kSumThreads = 512;

constexpr uint32_t kGone = 0xFFFFFFFFu;           // key of a token that is not sorted

// Token i of the first pass as (id, position).
__device__ __forceinline__ uint2 token(const SortArgs& a, uint32_t i) {
  if (i >= a.count) return make_uint2(kGone, i);
  const int64_t id = a.ids64 ? static_cast<const int64_t*>(a.ids)[i]
                             : static_cast<int64_t>(static_cast<const int32_t*>(a.ids)[i]);
  return make_uint2(id >= 0 && id < a.vocab ? static_cast<uint32_t>(id) : kGone, i);
}

// Sum of x over the threads before this one (all threads of the CTA take part).
template <int Threads>
__device__ __forceinline__ uint32_t sum_before(uint32_t* sums, uint32_t x, uint32_t* all) {
  constexpr int kWarps = Threads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) sums[warp] = incl;
  __syncthreads();
  const uint32_t s = lane < kWarps ? sums[lane] : 0;
  *all = __reduce_add_sync(0xffffffffu, s);
  return __reduce_add_sync(0xffffffffu, lane < warp ? s : 0) + incl - x;
}

// Counts the first digit per tile and clears what later passes count into.
template <int Threads>
__global__ void __launch_bounds__(Threads) count_kernel(SortArgs a) {
  __shared__ uint32_t count[kMaxDigits];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t digits = 1u << a.digit_bits, tiles = gridDim.x;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.zero = 0;
  uint32_t key[kItems];
#pragma unroll
  for (int r = 0; r < kItems; ++r)
    key[r] = token(a, (blockIdx.x * kItems + r) * Threads + threadIdx.x).x;
  for (uint32_t d = threadIdx.x; d < digits; d += Threads) count[d] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kItems; ++r)
    if (key[r] != kGone) atomicAdd(&count[key[r] & (digits - 1)], 1u);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += Threads) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * digits + d;
    a.counts[at] = count[d];
    for (int pass = 1; pass < a.passes; ++pass)
      a.counts[at + static_cast<int64_t>(pass) * (tiles + 1) * digits] = 0;
  }
}

// A digit's counts, added up over the tiles before each; its total behind them all.
__global__ void __launch_bounds__(kSumThreads) count_sums_kernel(uint32_t* counts, uint32_t tiles) {
  __shared__ uint32_t sums[kSumThreads / 32];
  const uint32_t digits = gridDim.x;
  uint32_t so_far = 0;
  for (uint32_t t0 = 0; t0 < tiles; t0 += kSumThreads) {
    const uint32_t t = t0 + threadIdx.x;
    uint32_t* at = counts + static_cast<int64_t>(t) * digits + blockIdx.x;
    const uint32_t c = t < tiles ? *at : 0;
    uint32_t all;
    const uint32_t before = sum_before<kSumThreads>(sums, c, &all);
    if (t < tiles) *at = so_far + before;
    so_far += all;
    __syncthreads();                      // sums are read
  }
  if (threadIdx.x == 0) counts[static_cast<int64_t>(tiles) * digits + blockIdx.x] = so_far;
}

// kSummed: the counts are sums over the tiles before each, with totals behind.
template <int Threads, bool kSummed>
__global__ void __launch_bounds__(Threads)
scatter_kernel(SortArgs a, const uint2* in, uint2* out, int pass) {
  constexpr int kWarps = Threads / 32;
  constexpr int kTile = kItems * Threads;
  constexpr int kOwn = Threads < kMaxDigits ? kMaxDigits / Threads : 1;   // digits of a thread, at most
  // Counts per warp, then tokens before (cleared as words).
  __shared__ __align__(16) uint16_t hist[kWarps][kMaxDigits];
  __shared__ uint32_t base[kMaxDigits], sums[kWarps];
  __shared__ uint4 part[2][Threads];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int shift = pass * a.digit_bits;
  const uint32_t digits = 1u << a.digit_bits, tiles = gridDim.x;
  const uint32_t* counts = a.counts + static_cast<int64_t>(pass) * (tiles + 1) * digits;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t first_item = blockIdx.x * kTile + warp * (32 * kItems) + lane;
  uint2 item[kItems];
  if (pass == 0) {
#pragma unroll
    for (int r = 0; r < kItems; ++r) item[r] = token(a, first_item + r * 32);
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (pass > 0) {
    const uint32_t count = *a.sorted_count;
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
      const uint32_t i = first_item + r * 32;
      item[r] = i < count ? in[i] : make_uint2(kGone, i);
    }
  }
  // Tokens per digit, all of them and those in the tiles before: a thread adds up
  // four digits of every step-th tile.
  const uint32_t quads = digits / 4, step = Threads / quads;
  if constexpr (!kSummed) {
    uint4 all = make_uint4(0, 0, 0, 0), early = all;
    const uint32_t q = threadIdx.x & (quads - 1);
#pragma unroll 8
    for (uint32_t t = threadIdx.x / quads; t < tiles; t += step) {
      const uint4 n = reinterpret_cast<const uint4*>(counts + t * digits)[q];
      all.x += n.x;
      all.y += n.y;
      all.z += n.z;
      all.w += n.w;
      if (t < blockIdx.x) {
        early.x += n.x;
        early.y += n.y;
        early.z += n.z;
        early.w += n.w;
      }
    }
    part[0][threadIdx.x] = all;
    part[1][threadIdx.x] = early;
  }
  uint32_t* words = reinterpret_cast<uint32_t*>(&hist[warp][0]);
  for (uint32_t d = lane; d < digits / 2; d += 32) words[d] = 0;
  __syncwarp();
  uint16_t rank[kItems];
#pragma unroll
  for (int r = 0; r < kItems; ++r) {
    const bool there = item[r].x != kGone;
    const uint32_t d = there ? item[r].x >> shift & (digits - 1) : kMaxDigits;
    const uint32_t peers = __match_any_sync(0xffffffffu, d);
    const uint32_t prev = there ? hist[warp][d] : 0;
    __syncwarp();
    if (there && lane == __ffs(peers) - 1) hist[warp][d] = static_cast<uint16_t>(prev + __popc(peers));
    __syncwarp();
    rank[r] = static_cast<uint16_t>(prev + __popc(peers & ((1u << lane) - 1u)));
  }
  __syncthreads();
  // This thread's digits own * per ... + per - 1.
  const uint32_t per = digits > Threads ? digits / Threads : 1, own = threadIdx.x * per;
  uint32_t total[kOwn], before[kOwn], mine = 0;
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    total[k] = before[k] = 0;
    const uint32_t d = own + k;
    if (k >= per || d >= digits) continue;
    uint32_t at = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t c = hist[w][d];
      hist[w][d] = static_cast<uint16_t>(at);
      at += c;
    }
    if constexpr (kSummed) {
      total[k] = counts[static_cast<int64_t>(tiles) * digits + d];
      before[k] = counts[static_cast<int64_t>(blockIdx.x) * digits + d];
    } else {
      const uint32_t parts = min(step, tiles);
      for (uint32_t t = 0; t < parts; ++t) {
        total[k] += reinterpret_cast<const uint32_t*>(&part[0][t * quads])[d];
        before[k] += reinterpret_cast<const uint32_t*>(&part[1][t * quads])[d];
      }
    }
    mine += total[k];
  }
  uint32_t all;
  uint32_t at = sum_before<Threads>(sums, mine, &all);
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    if (k < per && own + k < digits) base[own + k] = at + before[k];
    at += total[k];
  }
  if (pass == 0 && blockIdx.x == 0 && threadIdx.x == 0) *a.sorted_count = all;
  __syncthreads();
  uint32_t* next = pass + 1 < a.passes
                       ? a.counts + static_cast<int64_t>(pass + 1) * (tiles + 1) * digits
                       : nullptr;
#pragma unroll
  for (int r = 0; r < kItems; ++r) {
    if (item[r].x == kGone) continue;
    const uint32_t d = item[r].x >> shift & (digits - 1);
    const uint32_t to = base[d] + hist[warp][d] + rank[r];
    out[to] = item[r];
    if (next != nullptr)
      atomicAdd(next + static_cast<int64_t>(to / kTile) * digits +
                    (item[r].x >> (shift + a.digit_bits) & (digits - 1)), 1u);
  }
}

// A launch that may start while the kernel before it ends.
template <typename Kernel, typename... Args>
cudaError_t launch_after(Kernel* kernel, unsigned grid, int threads, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int Threads>
cudaError_t launch_sort(const SortArgs& a, cudaStream_t st) {
  const uint32_t tiles = static_cast<uint32_t>(sort_tiles(a.count)), digits = 1u << a.digit_bits;
  count_kernel<Threads><<<tiles, Threads, 0, st>>>(a);
  cudaError_t e = cudaGetLastError();
  for (int pass = 0; pass < a.passes && e == cudaSuccess; ++pass) {
    uint2* to = (a.passes - pass) & 1 ? a.out : a.other;     // the last pass: out
    const uint2* from = pass == 0 ? nullptr : to == a.out ? a.other : a.out;
    if (tiles <= kSumTiles) {
      e = launch_after(scatter_kernel<Threads, false>, tiles, Threads, st, a, from, to, pass);
    } else {
      count_sums_kernel<<<digits, kSumThreads, 0, st>>>(
          a.counts + static_cast<int64_t>(pass) * (tiles + 1) * digits, tiles);
      scatter_kernel<Threads, true><<<tiles, Threads, 0, st>>>(a, from, to, pass);
      e = cudaGetLastError();
    }
  }
  return e;
}

}  // namespace

cudaError_t launch_token_sort(const SortArgs& a, cudaStream_t st) {
  static_assert(kSmallTile == 128 * kItems && kLargeTile == 512 * kItems, "tiles of the two kernels");
  return sort_tile(a.count) == kSmallTile ? launch_sort<128>(a, st) : launch_sort<512>(a, st);
}

}  // namespace oprag
