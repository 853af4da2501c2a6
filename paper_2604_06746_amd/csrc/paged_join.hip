// The chunks of an attend call over pages joined, and the single tokens' weights gathered by page, in one launch.
//
// Rows as in cache_join.h.  The first launch also left each row's weight of each block of 16 slots, in the log2 domain: a page's mass takes 2^(x - lse2) of its
// blocks and all heads, or, of weights in units of 2^u, 2^((u - M) + (x - log2 Z)), large numbers and small
// ones apart.  Few bytes, so what counts is the chain of loads; the workgroups that gather form the rows' norms themselves, beside
// those that join the rows, and have the blocks' weights on their way meanwhile.  2081 slots 6.2 us (by two launches 4.3 + 11.2), eight of 64K to 128K 12.
#include "cache_join.h"
#include "paged.h"

#include <algorithm>

namespace skv {
namespace {

constexpr int64_t kLaunchBlocks = (int64_t)1 << 23;
constexpr int kStretch = 64;    // blocks whose weights a workgroup gathers: whole pages of any size

template <class TAB, class T, int DP>
__global__ __launch_bounds__(256) void paged_join_kernel(TAB tab, PagedView c, AttendWork w, int row_blocks, int first_block) {
  short_kernel_priority();
  __shared__ __attribute__((aligned(16))) float sh[256 * 4];
  __shared__ float zs[4];
  extern __shared__ float norms[];   // of the heads: M + log2 Z, and behind them each apart
  PagedUnit* apart_norms = reinterpret_cast<PagedUnit*>(norms + w.H);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, place = first_block + (int)blockIdx.x;
  if (place < row_blocks) {   // a row: lane groups on shares of its chunks
    const int r = (int)((uint32_t)place / (uint32_t)w.H), head = place - r * w.H;
    const int b = sequence_of(tab, r);
    const int4 share = w.shares[b];
    const int g = token_of(w, head), mine = head - g * w.gs;   // (a single token's rows are its heads)
    const int64_t part0 = ((int64_t)(share.x + mine / 16) * c.G + g) * 16 + mine % 16, step = (int64_t)(tab.units[b + 1] - tab.units[b]) * c.G * 16;
    join_row<T, DP>(w, c.d, (int64_t)r * w.H + head, reinterpret_cast<const joined_t*>(w.ml) + part0, w.o + part0 * DP + threadIdx.x % (DP / 4) * 4, step, share.z, sh, zs);
    return;
  }
  // Blocks i0 .. i0 + 63 of sequence b, one in each lane; a wave takes every fourth head.
  const int lb = c.shift - 4, per = (int)((((int64_t)c.max_pages << lb) + kStretch - 1) / kStretch);
  const int b = (place - row_blocks) / per, i0 = (place - row_blocks - b * per) * kStretch;
  const int4 share = w.shares[b];
  const int n = share.w, blocks = (n + kBlock - 1) / kBlock;   // (0 where the fresh token is not there)
  if (tab.cu_new[b + 1] - tab.cu_new[b] != 1 || i0 >= blocks) return;
  const int block = i0 + lane, live = share.z;
  const bool there = block < blocks && (uint32_t)c.pages[b * c.pst + (block >> lb)] < (uint32_t)c.n_pages;
  const float* x = w.x + ((int64_t)b * c.max_pages << lb) + block;
  float ahead[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) ahead[k] = there && wave + 4 * k < w.H ? x[(wave + 4 * k) * w.xs] : -INFINITY;
  const int page = (i0 >> lb) + (int)threadIdx.x;
  const bool mine = (int)threadIdx.x < kStretch >> lb && (int64_t)page << c.shift < n;
  const float old = mine ? c.mass[b * c.pst + page] : 0.f;
  const int64_t chunk_step = (int64_t)(tab.units[b + 1] - tab.units[b]) * c.G * 16;
  for (int h0 = wave; h0 < w.H; h0 += 4 * kAhead) {   // norms: a lane a chunk
    joined_t a[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int h = h0 + 4 * j, g = token_of(w, h), r = h - g * w.gs;
      a[j] = joined_stat(reinterpret_cast<const joined_t*>(w.ml) + ((int64_t)(share.x + r / 16) * c.G + g) * 16 + r % 16, chunk_step, live, h < w.H);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (h0 + 4 * j >= w.H) break;
      const float top = wave_top(a[j][0]), z = wave_total(a[j][1] * __builtin_amdgcn_exp2f(a[j][0] - top));
      if (lane == 0) {
        const float log_z = z != 0.f ? __builtin_amdgcn_logf(z) : INFINITY;
        norms[h0 + 4 * j] = top + log_z;
        apart_norms[h0 + 4 * j] = PagedUnit{top, log_z};
      }
    }
  }
  __syncthreads();   // (a wave reads its own heads' norms; the barrier is for the wave's own writes too)
  float sum = 0.f;
  for (int h0 = wave; h0 < w.H; h0 += 4 * kAhead) {
    float now[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) now[k] = ahead[k];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int h = h0 + 4 * (kAhead + k);
      ahead[k] = there && h < w.H ? x[h * w.xs] : -INFINITY;
    }
    float exponent[kAhead];
    bool apart = false;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      exponent[k] = h0 + 4 * k < w.H ? now[k] - norms[h0 + 4 * k] : -INFINITY;
      apart |= now[k] == kApart;
    }
    if (__any(apart)) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (now[k] == kApart) {
          const PagedUnit pair = reinterpret_cast<const PagedUnit*>(w.x + w.H * w.xs)[x - w.x + (h0 + 4 * k) * w.xs], norm = apart_norms[h0 + 4 * k];
          exponent[k] = (pair.unit - norm.unit) + (pair.weight - norm.weight);
        }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) sum += there ? __builtin_amdgcn_exp2f(exponent[k]) : 0.f;
  }
  sh[threadIdx.x] = sum;
  __syncthreads();
  if (mine) {
    float total = 0.f;
    for (int i = 0; i < 1 << lb; ++i) {
      const int at = ((int)threadIdx.x << lb) + i;
      total += (sh[at] + sh[64 + at]) + (sh[128 + at] + sh[192 + at]);
    }
    c.mass[b * c.pst + page] = w.lambda * old + total;
  }
}

}  // namespace

hipError_t launch_paged_join(const CacheTable& t, const PagedView& c, const AttendWork& w, bool bf16, hipStream_t st) {
  const int64_t stretches = ceil_div((int64_t)c.max_pages << (c.shift - 4), kStretch);
  const int64_t blocks = w.rows + stretches * c.batch;
  const auto launch = [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    with_cache_table(t, [&](const auto& tab) {
      using TAB = std::decay_t<decltype(tab)>;
      const size_t lds = (sizeof(float) + sizeof(PagedUnit)) * w.H;
      for (int64_t first = 0; first < blocks; first += kLaunchBlocks) {   // (a launch takes fewer than 2^32 threads)
        const unsigned now = (unsigned)std::min<int64_t>(kLaunchBlocks, blocks - first);
        if (bf16) paged_join_kernel<TAB, uint16_t, DP><<<now, 256, lds, st>>>(tab, c, w, (int)w.rows, (int)first);
        else paged_join_kernel<TAB, float, DP><<<now, 256, lds, st>>>(tab, c, w, (int)w.rows, (int)first);
      }
    });
    return hipGetLastError();
  };
  if (c.d <= 64) return launch(std::integral_constant<int, 64>{});
  if (c.d <= 128) return launch(std::integral_constant<int, 128>{});
  return launch(std::integral_constant<int, 256>{});
}

}  // namespace skv
