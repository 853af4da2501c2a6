// The chunks of an attend call joined, and the single tokens' weights gathered.
//
// A workgroup per row (cache_join.h).  The workgroups behind the rows' add the weights of a stretch of slots of one plane, 2^(x - lse) from the scores that
// the first launch left, so that the cache is read once.  Few bytes, so what counts is the chain of loads: the sequence's shares, which the
// first launch left; then the chunks' M and Z beside the sums or the scores themselves, all at once; nothing is loaded after the norms are known.
#include "cache_join.h"

namespace skv {
namespace {

constexpr int kSplitHeads = 16;   // from so many heads of a plane on, the waves share them

// What joining a row needs to know; n: its slots.
struct Row {
  int live;
  int64_t part0, step;   // its first chunk's partial result, and how far the next one's is
  bool written;          // by the first launch
};
template <class TAB>
__device__ __forceinline__ Row row_of(const TAB& tab, const CacheView& c, const AttendWork& w, int64_t at, int rows_wg) {
  const int r = (int)((uint32_t)at / (uint32_t)w.H), head = (int)(at - (int64_t)r * w.H);   // (rows stay below 2^31)
  Row row;
  int b = 0;
  while (b + 1 < tab.batch && r >= tab.cu_new[b + 1]) ++b;
  const int4 share = w.shares[b];
  const int rcs = tab.units[b + 1] - tab.units[b];
  const int g = token_of(w, head), mine = (r - tab.cu_new[b]) * w.gs + head - g * w.gs, rc = mine >> __builtin_ctz(rows_wg);
  row.live = share.z;
  row.part0 = ((int64_t)(share.x + rc) * c.G + g) * rows_wg + (mine & (rows_wg - 1));
  row.step = (int64_t)rcs * c.G * rows_wg;
  row.written = share.y == 1 && !w.x;
  return row;
}
// FEW: a lane group of DP / 4 a row, for sequences that have some kFewChunks chunks when all are full (more, in rounds, where the others are
// short); else a workgroup a row, its lane groups on shares of the chunks
constexpr int kFewChunks = 8;
template <class TAB, class T, int DP, bool FEW, int V>
__global__ __launch_bounds__(256) void cache_combine_kernel(TAB tab, CacheView c, AttendWork w, int rows_wg, int row_blocks, int stretch) {
  short_kernel_priority();
  constexpr int LANES = DP / 4, PARTS = 256 / LANES;
  __shared__ __attribute__((aligned(16))) float sh[256 * (V > 1 ? 2 * V : 4)];
  __shared__ float zs[4];
  extern __shared__ float norms[];   // of a plane's heads
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = threadIdx.x / LANES, col = threadIdx.x % LANES * 4;
  if ((int)blockIdx.x < row_blocks) {
    const int64_t at = FEW ? (int64_t)blockIdx.x * PARTS + part : blockIdx.x;
    if (at >= w.rows) return;
    const Row row = row_of(tab, c, w, at, rows_wg);
    if (row.written) return;
    const joined_t* ml = reinterpret_cast<const joined_t*>(w.ml) + row.part0;
    const float* po = w.o + row.part0 * DP + col;
    if (FEW) {
      float top = kNothingSeen, z = 0.f;
      floatx4 o = {0.f, 0.f, 0.f, 0.f};
      Chunks some;
      for (int i0 = 0; i0 < row.live; i0 += kAhead) {
        some.load(ml, po, row.step, DP, row.live, col < c.d, i0, 1);
        const float old = top;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) top = fmaxf(top, some.stat[k][0]);
        const float shrink = __builtin_amdgcn_exp2f(old - top);
        z *= shrink;
        o *= shrink;
        some.add(top, z, o);
      }
      if (col < c.d) put_row<T>(w, at, c.d, col, o, top, z);
    } else {
      join_row<T, DP>(w, c.d, at, ml, po, row.step, row.live, sh, zs);
    }
    return;
  }
  // weights
  const int u = ((int)blockIdx.x - row_blocks) / c.planes, plane = ((int)blockIdx.x - row_blocks) % c.planes;
  int b = 0;
  while (b + 1 < tab.batch && u >= tab.reach[b + 1]) ++b;
  const int4 share = w.shares[b];
  const int first = share.x, live = share.z;
  const int s0 = (u - tab.reach[b]) * stretch, s1 = min(s0 + stretch, share.w);
  if (tab.cu_new[b + 1] - tab.cu_new[b] != 1 || s0 >= s1) return;
  const int64_t chunk_step = (int64_t)(tab.units[b + 1] - tab.units[b]) * c.G * rows_wg;
  const int heads = w.H / c.planes;
  const float* x = w.x + plane * heads * w.xs + tab.cu[b] + kScorePad * b;
  float* mass = c.mass + plane * c.slots + tab.cu[b];
  // V consecutive slots a thread.  Many heads: a wave's lanes' slots at a time, a wave every fourth head of them; few: the workgroup's threads'
  // slots at a time, all heads of a slot in its thread.  (x has room behind a sequence's scores, mass does not.)
  const bool split = heads >= kSplitHeads;
  const int first_head = split ? wave : 0, step = split ? 4 : 1, slots = (split ? 64 : 256) * V;
  int s = s0 + (split ? lane : (int)threadIdx.x) * V;
  typedef float __attribute__((ext_vector_type(V), aligned(4))) some;
  typedef float __attribute__((ext_vector_type(V))) held_some;
  held_some ahead[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    ahead[k] = s < s1 && first_head + k * step < heads ? (held_some)*reinterpret_cast<const some*>(x + (first_head + k * step) * w.xs + s) : (held_some)(-INFINITY);
  for (int i0 = wave; i0 < heads; i0 += 4 * kAhead) {   // norms: a lane a chunk, the wave's heads at once
    joined_t a[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + 4 * j;
      const int head = plane * heads + i, g = token_of(w, head), r = head - g * w.gs;
      a[j] = joined_stat(reinterpret_cast<const joined_t*>(w.ml) + ((int64_t)(first + (r >> __builtin_ctz(rows_wg))) * c.G + g) * rows_wg + (r & (rows_wg - 1)), chunk_step, live,
                         i < heads);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i0 + 4 * j >= heads) break;
      const float top = wave_top(a[j][0]), z = wave_total(a[j][1] * __builtin_amdgcn_exp2f(a[j][0] - top));
      if (lane == 0) norms[i0 + 4 * j] = z != 0.f ? top + __builtin_amdgcn_logf(z) : INFINITY;
    }
  }
  __syncthreads();
  for (int t0 = s0; t0 < s1; t0 += slots, s += slots) {
    const bool whole = s + V <= s1, writes = s < s1 && (!split || wave == 0);
    held_some old = (held_some)(0.f);
    if (writes && whole) old = *reinterpret_cast<const some*>(mass + s);
    held_some sum = (held_some)(0.f);
    for (int i0 = first_head; i0 < heads; i0 += kAhead * step) {
      held_some now[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) now[k] = ahead[k];
      // the next heads, or the first ones of the next slots
      const bool same = i0 + kAhead * step < heads;
      const int sn = same ? s : s + slots, in = same ? i0 + kAhead * step : first_head;
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        ahead[k] = sn < s1 && in + k * step < heads ? (held_some)*reinterpret_cast<const some*>(x + (in + k * step) * w.xs + sn) : (held_some)(-INFINITY);
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + k * step < heads) {
          const float norm = norms[i0 + k * step];
#pragma unroll
          for (int e = 0; e < V; ++e) sum[e] += __builtin_amdgcn_exp2f(now[k][e] - norm);
        }
    }
    if (split) {   // (two halves of sh in turns: a wave is at most one barrier ahead)
      float* part = sh + ((t0 - s0) / slots & 1) * 256 * V;
      *reinterpret_cast<held_some*>(part + threadIdx.x * V) = sum;
      __syncthreads();
      if (wave != 0) continue;
      const held_some* parts = reinterpret_cast<const held_some*>(part);
      sum = (parts[lane] + parts[64 + lane]) + (parts[128 + lane] + parts[192 + lane]);
    }
    if (whole && writes) {
      *reinterpret_cast<some*>(mass + s) = w.lambda * old + sum;
    } else if (writes) {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (s + e < s1) mass[s + e] = w.lambda * mass[s + e] + sum[e];
    }
  }
}

}  // namespace

hipError_t launch_cache_combine(const CacheTable& t, const CacheView& c, const AttendPlan& p, const AttendWork& w, bool bf16,
                                hipStream_t st) {
  const auto launch = [&](auto dp, auto few, auto some) {
    constexpr int DP = decltype(dp)::value, V = decltype(some)::value;
    constexpr bool FEW = decltype(few)::value;
    const int64_t row_blocks = FEW ? ceil_div(w.rows, 256 / (DP / 4)) : w.rows;
    // slots of a workgroup: as many as it takes at a time, or twice that, where four workgroups a CU are left
    CacheTable u = t;
    int64_t blocks = row_blocks;
    int stretch = (w.H / c.planes >= kSplitHeads ? 64 : 256) * V;
    if (p.gather) {
      if (t.cu[t.batch] * c.planes / (2 * stretch) >= 4 * 256) stretch *= 2;
      u.reach[0] = 0;
      for (int b = 0; b < t.batch; ++b) u.reach[b + 1] = u.reach[b] + (int32_t)ceil_div(t.cu[b + 1] - t.cu[b], stretch);
      blocks += (int64_t)u.reach[t.batch] * c.planes;
    }
    const size_t lds = p.gather ? sizeof(float) * (w.H / c.planes) : 0;
    with_cache_table(u, [&](const auto& tab) {
      using TAB = std::decay_t<decltype(tab)>;
      const dim3 grid((unsigned)blocks);
      if (bf16) cache_combine_kernel<TAB, uint16_t, DP, FEW, V><<<grid, 256, lds, st>>>(tab, c, w, p.rows, (int)row_blocks, stretch);
      else cache_combine_kernel<TAB, float, DP, FEW, V><<<grid, 256, lds, st>>>(tab, c, w, p.rows, (int)row_blocks, stretch);
    });
    return hipGetLastError();
  };
  // four slots a thread where that leaves the weights two workgroups a CU
  const int64_t slots = t.cu[t.batch] * c.planes;
  const bool wide = p.gather && slots / (4 * (w.H / c.planes >= kSplitHeads ? 64 : 256)) >= 2 * 256;
  const auto by_slots = [&](auto dp, auto few) {
    return wide ? launch(dp, few, std::integral_constant<int, 4>{}) : launch(dp, few, std::integral_constant<int, 1>{});
  };
  const auto by_chunks = [&](auto dp) { return p.most_chunks <= kFewChunks ? by_slots(dp, std::true_type{}) : by_slots(dp, std::false_type{}); };
  if (c.d <= 64) return by_chunks(std::integral_constant<int, 64>{});
  if (c.d <= 128) return by_chunks(std::integral_constant<int, 128>{});
  return by_chunks(std::integral_constant<int, 256>{});
}

}  // namespace skv
