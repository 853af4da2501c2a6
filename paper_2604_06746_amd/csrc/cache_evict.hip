// Eviction from a cache in use: per sequence and plane the slots that stay, found by an exact radix select on order-preserving keys
// (recent slots above all), then kept slots from behind the budget move into the holes before it.  The holes lie below the budget and
// the slots that fill them from it on, so rows move in place, each once, whatever the order of the workgroups.
#include "cache.h"

#include <algorithm>

namespace skv {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;

__device__ __forceinline__ uint32_t lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// A workgroup per sequence and plane.  Its keys are read once per digit (11, 11 and 10 bits) and once to place the slots.
template <class TAB>
__global__ __launch_bounds__(kThreads) void cache_evict_kernel(TAB tab, CacheView c, EvictWork w) {
  short_kernel_priority();
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t part[3][kWaves];
  __shared__ int32_t top_pos;
  __shared__ uint32_t found[2];
  const int b = blockIdx.x, plane = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t lo = tab.cu[b];
  const int n = max(0, (int)min((int64_t)c.lens[b], tab.cu[b + 1] - lo)), budget = tab.units[b];
  if (tid == 0) {
    if (plane == 0) w.lens_out[b] = min(n, budget);
    if (n <= budget) w.count[plane * tab.batch + b] = 0;
    top_pos = 0;
  }
  if (n <= budget) return;
  const float* scores = w.scores + plane * c.slots + lo;
  int32_t* pos = c.pos ? c.pos + plane * c.slots + lo : nullptr;
  float* mass = c.mass ? c.mass + plane * c.slots + lo : nullptr;
  __syncthreads();
  if (w.keep_tail > 0) {
    int32_t top = 0;
    for (int s = tid; s < n; s += kThreads) top = max(top, pos[s]);
    for (int m = 1; m < 64; m <<= 1) top = max(top, __shfl_xor(top, m));
    if (lane == 0) atomicMax(&top_pos, top);
    __syncthreads();
  }
  const int64_t recent = w.keep_tail > 0 ? (int64_t)top_pos - w.keep_tail : 0;
  auto key_of = [&](int s) { return w.keep_tail > 0 && pos[s] > recent ? ~0u : score_key(scores[s]); };
  // the budget-th largest key, and how many of those equal to it stay
  uint32_t prefix = 0, left = (uint32_t)budget;
  for (int digit = 0; digit < 3 && budget > 0; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
    for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
    for (int s = tid; s < n; s += kThreads) {
      const uint32_t key = key_of(s);
      if (digit == 0 || key >> (shift + bits) == prefix) atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    // two bins a thread, from the top
    const uint32_t hi = hist[kBins - 1 - 2 * tid], under = hist[kBins - 2 - 2 * tid];
    uint32_t run = hi + under;
    for (int m = 1; m < 64; m <<= 1) {
      const uint32_t x = __shfl_up(run, m);
      if (lane >= m) run += x;
    }
    if (lane == 63) part[0][wave] = run;
    __syncthreads();
    for (int i = 0; i < wave; ++i) run += part[0][i];
    const uint32_t before = run - hi - under;
    if (before < left && run >= left) {
      const bool second = before + hi < left;
      found[0] = (uint32_t)(kBins - 1 - 2 * tid - second);
      found[1] = left - before - (second ? hi : 0);
    }
    __syncthreads();
    prefix = prefix << bits | found[0];
    left = found[1];
  }
  // holes and the slots that fill them, in ascending order: a block of consecutive slots at a time
  int32_t* holes = w.holes + plane * c.slots + lo;
  int32_t* moved = w.moved + plane * c.slots + lo;
  uint32_t ties = 0, n_holes = 0, n_moved = 0;
  for (int s0 = 0; s0 < n; s0 += kThreads) {
    const int s = s0 + tid;
    const uint32_t key = s < n ? key_of(s) : 0;
    const bool tie = budget > 0 && s < n && key == prefix;
    const uint64_t tie_mask = __ballot(tie);
    if (lane == 0) part[0][wave] = __popcll(tie_mask);
    __syncthreads();
    uint32_t rank = ties;
    for (int i = 0; i < kWaves; ++i) { ties += part[0][i]; rank += i < wave ? part[0][i] : 0; }
    rank += lanes_before(tie_mask);
    const bool kept = budget > 0 && s < n && (key > prefix || (tie && rank < left));
    const bool hole = s < budget && !kept, move = s >= budget && kept;
    const uint64_t hole_mask = __ballot(hole), move_mask = __ballot(move);
    if (lane == 0) { part[1][wave] = __popcll(hole_mask); part[2][wave] = __popcll(move_mask); }
    __syncthreads();
    uint32_t hr = n_holes, mr = n_moved;
    for (int i = 0; i < kWaves; ++i) {
      n_holes += part[1][i]; hr += i < wave ? part[1][i] : 0;
      n_moved += part[2][i]; mr += i < wave ? part[2][i] : 0;
    }
    if (hole) holes[hr + lanes_before(hole_mask)] = s;
    if (move) moved[mr + lanes_before(move_mask)] = s;
  }
  if (tid == 0) w.count[plane * tab.batch + b] = (int32_t)n_moved;
  __syncthreads();
  for (uint32_t j = tid; j < n_moved; j += kThreads) {
    if (mass) mass[holes[j]] = mass[moved[j]];
    if (pos) pos[holes[j]] = pos[moved[j]];
  }
}

// blockIdx.y: KV head and tensor, blockIdx.z: sequence; a thread per unit of a moved row
template <class TAB, class V>
__global__ __launch_bounds__(256) void cache_evict_rows_kernel(TAB tab, CacheView c, EvictWork w, int elem_bytes, int units_per_row) {
  short_kernel_priority();
  const int b = blockIdx.z, g = blockIdx.y >> 1, plane = c.planes > 1 ? g : 0;
  const int64_t lo = tab.cu[b], e = (int64_t)blockIdx.x * 256 + threadIdx.x, j = e / units_per_row;
  if (j >= w.count[plane * tab.batch + b]) return;
  const int64_t u = (e - j * units_per_row) * (int64_t)sizeof(V);
  uint8_t* rows = (uint8_t*)((blockIdx.y & 1) ? c.v : c.k) + ((int64_t)g * c.sh + lo * c.ss) * elem_bytes;
  const int64_t at = plane * c.slots + lo + j, step = c.ss * elem_bytes;
  *reinterpret_cast<V*>(rows + w.holes[at] * step + u) = load_once<V>(rows + w.moved[at] * step + u);
}

}  // namespace

hipError_t launch_cache_evict(const CacheTable& t, const CacheView& c, const EvictWork& w, int elem_bytes, hipStream_t st) {
  int64_t most = 0;   // rows that may move
  for (int b = 0; b < t.batch; ++b) {
    const int64_t over = t.cu[b + 1] - t.cu[b] - t.units[b];
    most = std::max(most, std::min<int64_t>(over, t.units[b]));
  }
  const uintptr_t bits = (uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)((c.sh | c.ss | c.d) * elem_bytes);
  with_cache_table(t, [&](const auto& tab) {
    using TAB = std::decay_t<decltype(tab)>;
    cache_evict_kernel<TAB><<<dim3((unsigned)t.batch, (unsigned)c.planes), kThreads, 0, st>>>(tab, c, w);
    if (most <= 0) return;
    auto rows = [&](auto unit) {
      using V = decltype(unit);
      const int upr = c.d * elem_bytes / (int)sizeof(V);
      cache_evict_rows_kernel<TAB, V><<<dim3((unsigned)ceil_div(most * upr, 256), 2 * (unsigned)c.G, (unsigned)t.batch), 256, 0, st>>>(
          tab, c, w, elem_bytes, upr);
    };
    if (bits % 16 == 0) rows(uint4{});
    else if (bits % 4 == 0) rows(uint32_t{});
    else rows(uint16_t{});
  });
  return hipGetLastError();
}

}  // namespace skv
