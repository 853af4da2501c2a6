// Eviction from a cache in use: per sequence and plane the slots that stay -- recent ones above all, then by score, ties to the lower slot --
// found by exact selection on order-preserving keys, then kept slots from behind the budget move into the holes before it.  The holes
// lie below the budget and the slots that fill them from it on, so rows move in place, each once, whatever the order of the workgroups.
//
// Scores and positions are a few bytes a slot; launches, dependent loads and barriers are what a selection costs.  Two forms, by the largest
// capacity:
//   short (up to 32768 slots): a workgroup per sequence and plane holds all keys in registers.  The range between the smallest and the
//     largest key is cut into 2048 bins, the bin with the last slot that stays again, or, once it holds few keys, these are ranked against
//     each other.  Where at most kFusedRows slots can move, and few bytes, it moves them too: a full cache that evicts one token a step.
//     From 16385 slots on a thread has 32 keys and spills 8 to 11 registers: a call on an idle queue that evicts one of 16385 30 us, of 16384 17,
//     of 32768 33; by digits, one of 32769 39.
//   long: three digits of the keys (11, 11 and 10 bits) by all workgroups of a sequence, one launch each, then each workgroup's counts,
//     then the lists.
// Stream order is the only synchronisation between launches, and the histograms' integer additions the only atomics.
#include "cache.h"

#include <algorithm>

namespace skv {
namespace {

__device__ __forceinline__ uint32_t lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t x, uint32_t without) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)without, (int)x, CTRL, ROWS, 0xF, false);
}
// over the 64 lanes: inclusive sums, and the largest in the last lane, by moves inside the rows of 16 and then between them
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {
  x += moved<0x111, 0xF>(x, 0u);
  x += moved<0x112, 0xF>(x, 0u);
  x += moved<0x114, 0xF>(x, 0u);
  x += moved<0x118, 0xF>(x, 0u);
  x += moved<0x142, 0xA>(x, 0u);
  x += moved<0x143, 0xC>(x, 0u);
  return x;
}
__device__ __forceinline__ uint32_t wave_largest(uint32_t x) {
  x = max(x, moved<0x111, 0xF>(x, 0u));
  x = max(x, moved<0x112, 0xF>(x, 0u));
  x = max(x, moved<0x114, 0xF>(x, 0u));
  x = max(x, moved<0x118, 0xF>(x, 0u));
  x = max(x, moved<0x142, 0xA>(x, 0u));
  x = max(x, moved<0x143, 0xC>(x, 0u));
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
// over the workgroup's WAVES waves' values v (the same in all lanes of a wave); sh: WAVES words, not written again before another barrier.
// The sum, and in *before that of the waves before the calling one.
template <int WAVES>
__device__ __forceinline__ uint32_t waves_sum(uint32_t v, uint32_t* sh, uint32_t* before) {
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  if (lane == 0) sh[wave] = v;
  __syncthreads();
  const uint32_t s = wave_sums(lane < WAVES ? sh[lane] : 0u);
  *before = wave ? (uint32_t)__builtin_amdgcn_readlane((int)s, wave - 1) : 0u;
  return (uint32_t)__builtin_amdgcn_readlane((int)s, WAVES - 1);
}
template <int WAVES>
__device__ __forceinline__ uint32_t waves_largest(uint32_t v, uint32_t* sh) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (lane == 0) sh[wave] = v;
  __syncthreads();
  return wave_largest(lane < WAVES ? sh[lane] : 0u);
}

constexpr int kBins = 2048;
// From the top of kBins bins in LDS, the one with the left-th key: its number in res[0], the rank left in it in res[1], its keys in res[2].
template <int THREADS>
__device__ __forceinline__ void find_bin(const uint32_t* hist, uint32_t left, uint32_t* sh, uint32_t* res) {
  constexpr int PER = kBins / THREADS;
  uint32_t own[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) { own[i] = hist[kBins - 1 - (int)(threadIdx.x * PER + i)]; sum += own[i]; }
  const uint32_t scan = wave_sums(sum);
  uint32_t before;
  waves_sum<THREADS / 64>((uint32_t)__builtin_amdgcn_readlane((int)scan, 63), sh, &before);
  uint32_t run = before + scan - sum;
  if (run < left && run + sum >= left) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (run < left && run + own[i] >= left) {
        res[0] = (uint32_t)(kBins - 1 - (int)(threadIdx.x * PER + i));
        res[1] = left - run;
        res[2] = own[i];
      }
      run += own[i];
    }
  }
  __syncthreads();
}

// ---- short ----------------------------------------------------------------------------------------------------------------------
constexpr int kRanked = 256;      // most keys that are ranked against each other
constexpr int kFusedRows = 64;    // most slots of a plane, ...
constexpr int kFusedBytes = 1 << 17;   // ... and bytes of K and V that the selecting workgroup moves itself

// PER keys a thread; a wave has consecutive slots, its lanes neighbouring ones.
template <class TAB, int THREADS, int PER, bool FUSED>
__global__ __launch_bounds__(THREADS) void cache_evict_short_kernel(TAB tab, CacheView c, EvictWork w, int elem_bytes) {
  short_kernel_priority();
  constexpr int WAVES = THREADS / 64;
  static_assert(PER <= 32, "a bit a slot");
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t sh[8][WAVES];
  __shared__ uint32_t res[4], listed, list[kRanked];
  __shared__ int32_t from[FUSED ? kFusedRows : 1], to[FUSED ? kFusedRows : 1];
  const int b = blockIdx.x, plane = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t lo = tab.cu[b], plane0 = plane * c.slots + lo;
  const int n = max(0, (int)min((int64_t)c.lens[b], tab.cu[b + 1] - lo)), budget = tab.units[b];
  if (tid == 0) {
    if (plane == 0) w.lens_out[b] = min(n, budget);
    if (!FUSED && n <= budget) w.count[plane * tab.batch + b] = 0;
  }
  if (n <= budget) return;
  const float* scores = w.scores + plane0;
  const int s0 = wave * 64 * PER + lane;
  uint32_t key[PER], recent = 0;   // recent: a bit a slot
  int32_t at[PER], top = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = s0 + i * 64;
    key[i] = s < n ? __float_as_uint(scores[s]) : 0u;
    at[i] = w.keep_tail > 0 && s < n ? c.pos[plane0 + s] : -1;
  }
  for (int i = tid; i < kBins; i += THREADS) hist[i] = 0;
  if (tid == 0) listed = 0;
  if (w.keep_tail > 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) top = max(top, at[i]);
    top = (int32_t)waves_largest<WAVES>(wave_largest((uint32_t)top), sh[0]);
#pragma unroll
    for (int i = 0; i < PER; ++i) recent |= at[i] >= 0 && (int64_t)at[i] > (int64_t)top - w.keep_tail ? 1u << i : 0u;
  }
  uint32_t most = 0, least = ~0u;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    key[i] = score_key(__uint_as_float(key[i]));
    if (s0 + i * 64 < n && !(recent >> i & 1)) { most = max(most, key[i]); least = min(least, key[i]); }
  }
  uint32_t ignored;
  const uint32_t recents = waves_sum<WAVES>((uint32_t)__builtin_amdgcn_readlane((int)wave_sums(__popc(recent)), 63), sh[1], &ignored);
  const uint32_t hi0 = waves_largest<WAVES>(wave_largest(most), sh[2]), lo0 = ~waves_largest<WAVES>(wave_largest(~least), sh[3]);
  // The last key that stays, and how many of those equal to it do; all recent ones above it.  More recent ones than the budget: the
  // first of them.
  const bool crowd = recents >= (uint32_t)budget;
  uint32_t tau = 0, need = (uint32_t)budget, equal = recents;
  if (!crowd) {
    uint32_t first = lo0, last = hi0, left = (uint32_t)budget - recents;
    equal = ~0u;
    for (;;) {
      if (first == last) { tau = first; need = left; break; }
      const uint32_t span = last - first, shift = span < kBins ? 0 : 32 - __builtin_clz(span) - 11;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (s0 + i * 64 < n && !(recent >> i & 1) && key[i] >= first && key[i] <= last) atomicAdd(&hist[(key[i] - first) >> shift], 1u);
      __syncthreads();
      find_bin<THREADS>(hist, left, sh[4], res);
      first += res[0] << shift;
      last = first + min(last - first, (1u << shift) - 1);
      left = res[1];
      const uint32_t held = res[2];
      if (shift == 0) { tau = first; need = left; equal = held; break; }
      if (held <= kRanked) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (s0 + i * 64 < n && !(recent >> i & 1) && key[i] >= first && key[i] <= last) list[atomicAdd(&listed, 1u)] = key[i];
        __syncthreads();
        if (tid < (int)held) {
          const uint32_t mine = list[tid];
          uint32_t above = 0, same = 0;
          for (uint32_t k = 0; k < held; ++k) { above += list[k] > mine; same += list[k] == mine; }
          if (above < left && above + same >= left) { res[0] = mine; res[1] = left - above; res[2] = same; }
        }
        __syncthreads();
        tau = res[0]; need = res[1]; equal = res[2];
        break;
      }
      for (int i = tid; i < kBins; i += THREADS) hist[i] = 0;   // (all have read it: find_bin ends with a barrier)
      __syncthreads();
    }
  }
  uint32_t kept = crowd ? 0u : recent, ties = crowd ? recent : 0u;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (s0 + i * 64 < n && !crowd && !(recent >> i & 1)) {
      kept |= key[i] > tau ? 1u << i : 0u;
      ties |= key[i] == tau ? 1u << i : 0u;
    }
  if (need >= equal) {
    kept |= ties;
  } else {   // the lower slots of those that are equal
    uint32_t rank;
    waves_sum<WAVES>((uint32_t)__builtin_amdgcn_readlane((int)wave_sums(__popc(ties)), 63), sh[5], &rank);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint64_t all = __ballot(ties >> i & 1);
      if ((ties >> i & 1) && rank + lanes_before(all) < need) kept |= 1u << i;
      rank += __popcll(all);
    }
  }
  // holes below the budget and kept slots from it on, in ascending order
  uint32_t holes = 0, moves = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = s0 + i * 64;
    holes += __popcll(__ballot(s < budget && !(kept >> i & 1)));
    moves += __popcll(__ballot(s >= budget && (kept >> i & 1)));
  }
  uint32_t hole_at, move_at;
  waves_sum<WAVES>(holes, sh[6], &hole_at);
  const uint32_t moving = waves_sum<WAVES>(moves, sh[7], &move_at);
  int32_t* hole_list = FUSED ? to : w.holes + plane0;
  int32_t* move_list = FUSED ? from : w.moved + plane0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = s0 + i * 64;
    const bool hole = s < budget && !(kept >> i & 1), move = s >= budget && (kept >> i & 1);
    const uint64_t all_holes = __ballot(hole), all_moves = __ballot(move);
    if (hole) hole_list[hole_at + lanes_before(all_holes)] = s;
    if (move) move_list[move_at + lanes_before(all_moves)] = s;
    hole_at += __popcll(all_holes);
    move_at += __popcll(all_moves);
  }
  if (!FUSED) {
    if (tid == 0) w.count[plane * tab.batch + b] = (int32_t)moving;
    return;
  }
  __syncthreads();
  if (tid < (int)moving) {
    if (c.mass) c.mass[plane0 + to[tid]] = c.mass[plane0 + from[tid]];
    if (c.pos) c.pos[plane0 + to[tid]] = c.pos[plane0 + from[tid]];
  }
  const uint32_t upr = (uint32_t)(c.d * elem_bytes) / 16, heads = c.planes > 1 ? 1 : (uint32_t)c.G, units = moving * heads * 2 * upr;
  const int64_t step = c.ss * elem_bytes;
  for (uint32_t e = tid; e < units; e += THREADS) {
    const uint32_t q = e / upr, u = e - q * upr, head = (q >> 1) % heads, j = (q >> 1) / heads;
    const int64_t g = c.planes > 1 ? plane : (int64_t)head;
    uint8_t* rows = (uint8_t*)((q & 1) ? c.v : c.k) + (g * c.sh + lo * c.ss) * elem_bytes + u * 16;
    *reinterpret_cast<uint4*>(rows + to[j] * step) = load_once<uint4>(rows + from[j] * step);
  }
}

// ---- long -----------------------------------------------------------------------------------------------------------------------
// A workgroup's share: `share` consecutive slots, kShare or more; at most kMaxShares of them a sequence.
constexpr int kThreads = 256, kWaves = kThreads / 64, kShare = 1024, kMaxShares = 1024;
constexpr int kHistWords = 3 * kBins + 8;   // a sequence's digits; then: recent slots, digit 0, rank left, digits 0 and 1, rank left, key, rank left
enum { kRecents = 3 * kBins, kBin0, kLeft0, kPrefix, kLeft1 };

struct Share {
  int b, n, budget, lo, hi, blk, blocks;   // [lo, hi) of the n slots in use
  int64_t at, plane0;                      // of the workgroup's records in the plane; of the sequence's slots
  uint32_t* hist;
};
template <class TAB>
__device__ __forceinline__ Share my_share(const TAB& tab, const CacheView& c, const EvictWork& w) {
  Share s;
  int b = 0;
  while (b + 1 < tab.batch && (int)blockIdx.x >= tab.cu_new[b + 1]) ++b;   // (cu_new: workgroups)
  s.b = b;
  const int64_t cap = tab.cu[b + 1] - tab.cu[b];
  s.n = max(0, (int)min((int64_t)c.lens[b], cap));
  s.budget = tab.units[b];
  s.blk = (int)blockIdx.x - tab.cu_new[b];
  s.blocks = tab.cu_new[b + 1] - tab.cu_new[b];
  const int64_t share = max((int64_t)kShare, (cap + kMaxShares - 1) / kMaxShares);
  s.lo = (int)min((int64_t)s.n, s.blk * share);
  s.hi = (int)min((int64_t)s.n, s.lo + share);
  s.at = (int64_t)blockIdx.y * tab.cu_new[tab.batch] + blockIdx.x;
  s.plane0 = blockIdx.y * c.slots + tab.cu[b];
  s.hist = w.hist + ((int64_t)blockIdx.y * tab.batch + b) * kHistWords;
  return s;
}

template <class TAB>
__global__ __launch_bounds__(kThreads) void cache_evict_init_kernel(TAB tab, CacheView c, EvictWork w) {
  short_kernel_priority();
  __shared__ uint32_t sh[kWaves];
  const Share s = my_share(tab, c, w);
  if (s.blk == 0 && threadIdx.x == 0) {
    if (blockIdx.y == 0) w.lens_out[s.b] = min(s.n, s.budget);
    w.count[blockIdx.y * tab.batch + s.b] = 0;
  }
  if (s.n <= s.budget) return;
  for (int i = s.blk * kThreads + threadIdx.x; i < kHistWords; i += s.blocks * kThreads) s.hist[i] = 0;
  uint32_t top = 0;
  if (w.keep_tail > 0)
    for (int j = s.lo + threadIdx.x; j < s.hi; j += kThreads) top = max(top, (uint32_t)max(0, c.pos[s.plane0 + j]));
  top = waves_largest<kWaves>(wave_largest(top), sh);
  if (threadIdx.x == 0) w.tops[s.at] = (int32_t)top;
}

// positions above this are recent (all workgroups of a sequence agree: the largest of their shares' largest)
__device__ __forceinline__ int64_t recent_from(const Share& s, const EvictWork& w, uint32_t* sh) {
  uint32_t top = 0;
  for (int i = threadIdx.x; i < s.blocks; i += kThreads) top = max(top, (uint32_t)w.tops[s.at - s.blk + i]);
  return (int64_t)waves_largest<kWaves>(wave_largest(top), sh) - w.keep_tail;
}
// f(slot, key, recent) for a thread's slots of the share
template <class F>
__device__ __forceinline__ void each_slot(const Share& s, const CacheView& c, const EvictWork& w, int64_t recent, F f) {
  for (int j = s.lo + threadIdx.x; j < s.hi; j += kThreads)
    f(j, score_key(w.scores[s.plane0 + j]), w.keep_tail > 0 && (int64_t)c.pos[s.plane0 + j] > recent);
}
// the digit with the left-th key, from a merged histogram
__device__ __forceinline__ void find_digit(const uint32_t* merged, uint32_t* hist, uint32_t left, uint32_t* sh, uint32_t* res) {
  for (int i = threadIdx.x; i < kBins; i += kThreads) hist[i] = merged[i];
  __syncthreads();
  find_bin<kThreads>(hist, left, sh, res);
}

// DIGIT 0, 1, 2: histogram of a digit of the keys that agree with the digits found so far
template <class TAB, int DIGIT>
__global__ __launch_bounds__(kThreads) void cache_evict_digit_kernel(TAB tab, CacheView c, EvictWork w) {
  short_kernel_priority();
  __shared__ uint32_t hist[kBins], sh[3][kWaves], res[3];
  const Share s = my_share(tab, c, w);
  if (s.n <= s.budget) return;
  const int64_t recent = recent_from(s, w, sh[0]);
  uint32_t prefix = 0;
  if (DIGIT > 0) {
    const uint32_t recents = s.hist[kRecents];
    if (recents >= (uint32_t)s.budget) return;   // (the first of them stay)
    const uint32_t left = DIGIT == 1 ? (uint32_t)s.budget - recents : s.hist[kLeft0];
    find_digit(s.hist + (DIGIT - 1) * kBins, hist, left, sh[1], res);
    prefix = DIGIT == 1 ? res[0] : s.hist[kBin0] << 11 | res[0];
    if (s.blk == 0 && threadIdx.x == 0) {
      s.hist[DIGIT == 1 ? kBin0 : kPrefix] = prefix;
      s.hist[DIGIT == 1 ? kLeft0 : kLeft1] = res[1];
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < kBins; i += kThreads) hist[i] = 0;
  __syncthreads();
  uint32_t recents = 0;
  each_slot(s, c, w, recent, [&](int, uint32_t key, bool is_recent) {
    recents += is_recent;
    if (is_recent) return;
    if (DIGIT == 0) atomicAdd(&hist[key >> 21], 1u);
    if (DIGIT == 1 && key >> 21 == prefix) atomicAdd(&hist[key >> 10 & (kBins - 1)], 1u);
    if (DIGIT == 2 && key >> 10 == prefix) atomicAdd(&hist[key & 1023], 1u);
  });
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads)
    if (hist[i]) atomicAdd(&s.hist[DIGIT * kBins + i], hist[i]);
  if (DIGIT == 0) {
    recents = (uint32_t)__builtin_amdgcn_readlane((int)wave_sums(recents), 63);
    if ((threadIdx.x & 63) == 0 && recents) atomicAdd(&s.hist[kRecents], recents);
  }
}

// What decides a slot: it stays for sure, or if its rank among the equal ones is below need.
struct Verdict {
  bool crowd;
  uint32_t tau, need;
  int64_t recent;
  __device__ __forceinline__ bool sure(uint32_t key, bool is_recent) const { return !crowd && (is_recent || key > tau); }
  __device__ __forceinline__ bool tie(uint32_t key, bool is_recent) const { return crowd ? is_recent : !is_recent && key == tau; }
};
__device__ __forceinline__ Verdict verdict(const Share& s, const EvictWork& w, uint32_t* hist, uint32_t (*sh)[kWaves], uint32_t* res) {
  Verdict v;
  v.recent = recent_from(s, w, sh[0]);
  const uint32_t recents = s.hist[kRecents];
  v.crowd = recents >= (uint32_t)s.budget;
  v.tau = 0;
  v.need = (uint32_t)s.budget;
  if (!v.crowd) {   // (the same for the whole workgroup)
    find_digit(s.hist + 2 * kBins, hist, s.hist[kLeft1], sh[1], res);
    v.tau = s.hist[kPrefix] << 10 | res[0];
    v.need = res[1];
  }
  return v;
}

// a share's slots that stay for sure and equal ones, below the budget and from it on
template <class TAB>
__global__ __launch_bounds__(kThreads) void cache_evict_count_kernel(TAB tab, CacheView c, EvictWork w) {
  short_kernel_priority();
  __shared__ uint32_t hist[kBins], sh[6][kWaves], res[3];
  const Share s = my_share(tab, c, w);
  if (s.n <= s.budget) return;
  const Verdict v = verdict(s, w, hist, sh, res);
  uint32_t count[4] = {};
  each_slot(s, c, w, v.recent, [&](int j, uint32_t key, bool is_recent) {
    count[j < s.budget ? 0 : 1] += v.sure(key, is_recent);
    count[j < s.budget ? 2 : 3] += v.tie(key, is_recent);
  });
  uint32_t ignored;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t all = waves_sum<kWaves>((uint32_t)__builtin_amdgcn_readlane((int)wave_sums(count[i]), 63), sh[2 + i], &ignored);
    if (threadIdx.x == 0) w.counts[s.at * 4 + i] = all;
  }
}

template <class TAB>
__global__ __launch_bounds__(kThreads) void cache_evict_place_kernel(TAB tab, CacheView c, EvictWork w) {
  short_kernel_priority();
  __shared__ uint32_t hist[kBins], sh[8][kWaves], res[3];
  const Share s = my_share(tab, c, w);
  if (s.n <= s.budget) return;
  const Verdict v = verdict(s, w, hist, sh, res);
  // The shares before this one: four of kMaxShares records a thread, in order.  Equal ones that they keep follow from those before them;
  // then their holes (slots below the budget that do not stay) and moves.
  const int per = (s.blocks + kThreads - 1) / kThreads, i0 = min(s.blocks, (int)threadIdx.x * per), i1 = min(s.blocks, i0 + per);
  const int64_t cap = tab.cu[s.b + 1] - tab.cu[s.b], share = max((int64_t)kShare, (cap + kMaxShares - 1) / kMaxShares);
  const uint4* records = reinterpret_cast<const uint4*>(w.counts) + (s.at - s.blk);
  uint32_t ties = 0;
  for (int i = i0; i < i1; ++i) ties += records[i].z + records[i].w;
  const uint32_t scan = wave_sums(ties);
  uint32_t run;
  waves_sum<kWaves>((uint32_t)__builtin_amdgcn_readlane((int)scan, 63), sh[2], &run);
  run += scan - ties;   // equal ones before the thread's first share
  uint32_t mine = 0, holes = 0, moves = 0, all_moves = 0;
  for (int i = i0; i < i1; ++i) {
    const uint4 r = records[i];
    const uint32_t free_ = v.need > run ? v.need - run : 0, low = min(r.z, free_), high = min(r.w, free_ - low);
    const uint32_t below = (uint32_t)(max((int64_t)0, min((int64_t)s.budget, min((int64_t)s.n, (i + 1) * share)) - min((int64_t)s.budget, i * share)));
    if (i < s.blk) { mine += r.z + r.w; holes += below - r.x - low; moves += r.y + high; }
    all_moves += r.y + high;
    run += r.z + r.w;
  }
  uint32_t ignored;
  auto total = [&](uint32_t x, uint32_t* at) { return waves_sum<kWaves>((uint32_t)__builtin_amdgcn_readlane((int)wave_sums(x), 63), at, &ignored); };
  uint32_t tie_rank = total(mine, sh[3]), hole_at = total(holes, sh[4]), move_at = total(moves, sh[5]);
  all_moves = total(all_moves, sh[6]);
  if (s.blk == 0 && threadIdx.x == 0) w.count[blockIdx.y * tab.batch + s.b] = (int32_t)all_moves;
  for (int j0 = s.lo; j0 < s.hi; j0 += kThreads) {
    const int j = j0 + threadIdx.x;
    const bool in = j < s.hi;
    const uint32_t key = in ? score_key(w.scores[s.plane0 + j]) : 0u;
    const bool is_recent = in && w.keep_tail > 0 && (int64_t)c.pos[s.plane0 + j] > v.recent;
    const bool tie = in && v.tie(key, is_recent);
    __syncthreads();
    uint32_t before;
    const uint64_t tie_mask = __ballot(tie);
    const uint32_t all_ties = waves_sum<kWaves>(__popcll(tie_mask), sh[0], &before);
    const bool kept = in && (v.sure(key, is_recent) || (tie && tie_rank + before + lanes_before(tie_mask) < v.need));
    const bool hole = in && j < s.budget && !kept, move = in && j >= s.budget && kept;
    const uint64_t hole_mask = __ballot(hole), move_mask = __ballot(move);
    uint32_t holes_before, moves_before;
    const uint32_t all_holes = waves_sum<kWaves>(__popcll(hole_mask), sh[1], &holes_before);
    const uint32_t moved_here = waves_sum<kWaves>(__popcll(move_mask), sh[7], &moves_before);
    if (hole) w.holes[s.plane0 + hole_at + holes_before + lanes_before(hole_mask)] = j;
    if (move) w.moved[s.plane0 + move_at + moves_before + lanes_before(move_mask)] = j;
    tie_rank += all_ties;
    hole_at += all_holes;
    move_at += moved_here;
  }
}

constexpr int64_t kRowBlocks = 8192;   // workgroups that move rows, at most

// ---- rows -----------------------------------------------------------------------------------------------------------------------
// blockIdx.y: KV head and tensor, blockIdx.z: sequence; a thread per unit of a moved row at a time, and the first one of a key's row, of a plane's
// first head, also moves the slot's mass and position.  How many rows move is known on the device alone: workgroups for all
// that might would mostly find nothing (16 caches of 8 heads, 40 % of the possible rows move: 57.9 us, and 47.8 with the 8192 workgroups
// here, 52.6 with 2048), so a few go through them in turns.
template <class TAB, class V>
__global__ __launch_bounds__(256) void cache_evict_rows_kernel(TAB tab, CacheView c, EvictWork w, int elem_bytes, uint32_t units_per_row) {
  short_kernel_priority();
  const int b = blockIdx.z, g = blockIdx.y >> 1, plane = c.planes > 1 ? g : 0;
  const int64_t lo = tab.cu[b], plane0 = plane * c.slots + lo, step = c.ss * elem_bytes;
  const uint32_t units = (uint32_t)w.count[plane * tab.batch + b] * units_per_row;
  uint8_t* rows = (uint8_t*)((blockIdx.y & 1) ? c.v : c.k) + ((int64_t)g * c.sh + lo * c.ss) * elem_bytes;
  const bool about = (blockIdx.y & 1) == 0 && (c.planes > 1 || g == 0);
  for (uint32_t e = blockIdx.x * 256 + threadIdx.x; e < units; e += gridDim.x * 256) {
    const uint32_t j = e / units_per_row;
    const int64_t u = (e - j * units_per_row) * (int64_t)sizeof(V), to = w.holes[plane0 + j], from = w.moved[plane0 + j];
    *reinterpret_cast<V*>(rows + to * step + u) = load_once<V>(rows + from * step + u);
    if (about && u == 0) {
      if (c.mass) c.mass[plane0 + to] = c.mass[plane0 + from];
      if (c.pos) c.pos[plane0 + to] = c.pos[plane0 + from];
    }
  }
}

template <int THREADS, int PER, class TAB>
void launch_short(const TAB& tab, const CacheView& c, const EvictWork& w, int elem_bytes, bool fused, hipStream_t st) {
  const dim3 grid((unsigned)tab.batch, (unsigned)c.planes);
  if (fused) cache_evict_short_kernel<TAB, THREADS, PER, true><<<grid, THREADS, 0, st>>>(tab, c, w, elem_bytes);
  else cache_evict_short_kernel<TAB, THREADS, PER, false><<<grid, THREADS, 0, st>>>(tab, c, w, elem_bytes);
}

}  // namespace

int evict_shares(int64_t cap) {
  const int64_t share = std::max<int64_t>(kShare, ceil_div(cap, kMaxShares));
  return (int)std::max<int64_t>(1, ceil_div(cap, share));
}
size_t evict_hist_words() { return kHistWords; }

hipError_t launch_cache_evict(const CacheTable& t, const CacheView& c, const EvictWork& w, int elem_bytes, hipStream_t st) {
  int64_t most = 0, longest = 0;   // rows that may move, slots
  for (int b = 0; b < t.batch; ++b) {
    const int64_t over = t.cu[b + 1] - t.cu[b] - t.units[b];
    most = std::max(most, std::min<int64_t>(over, t.units[b]));
    longest = std::max(longest, t.cu[b + 1] - t.cu[b]);
  }
  const uintptr_t bits = (uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)((c.sh | c.ss | c.d) * elem_bytes);
  const int64_t heads = c.planes > 1 ? 1 : c.G;
  const bool fused = longest <= kEvictShort && bits % 16 == 0 && most <= kFusedRows && most * heads * 2 * c.d * elem_bytes <= kFusedBytes;
  CacheTable u = t;
  if (longest > kEvictShort) {
    u.cu_new[0] = 0;
    for (int b = 0; b < t.batch; ++b) u.cu_new[b + 1] = u.cu_new[b] + evict_shares(t.cu[b + 1] - t.cu[b]);
  }
  with_cache_table(u, [&](const auto& tab) {
    using TAB = std::decay_t<decltype(tab)>;
    if (longest <= 4096) launch_short<1024, 4>(tab, c, w, elem_bytes, fused, st);   // (2081 slots 6.4 us; 512 threads 6.8, 256 9.4)
    else if (longest <= 8192) launch_short<1024, 8>(tab, c, w, elem_bytes, fused, st);
    else if (longest <= 16384) launch_short<1024, 16>(tab, c, w, elem_bytes, fused, st);
    else if (longest <= kEvictShort) launch_short<1024, 32>(tab, c, w, elem_bytes, fused, st);
    else {
      const dim3 grid((unsigned)u.cu_new[t.batch], (unsigned)c.planes);
      cache_evict_init_kernel<TAB><<<grid, kThreads, 0, st>>>(tab, c, w);
      cache_evict_digit_kernel<TAB, 0><<<grid, kThreads, 0, st>>>(tab, c, w);
      cache_evict_digit_kernel<TAB, 1><<<grid, kThreads, 0, st>>>(tab, c, w);
      cache_evict_digit_kernel<TAB, 2><<<grid, kThreads, 0, st>>>(tab, c, w);
      cache_evict_count_kernel<TAB><<<grid, kThreads, 0, st>>>(tab, c, w);
      cache_evict_place_kernel<TAB><<<grid, kThreads, 0, st>>>(tab, c, w);
    }
    if (most <= 0 || fused) return;
    auto rows = [&](auto unit) {
      using V = decltype(unit);
      const uint32_t upr = (uint32_t)(c.d * elem_bytes / (int)sizeof(V));
      const int64_t all = ceil_div(most * upr, 256), some = std::max<int64_t>(kRowBlocks / (2 * (int64_t)c.G * t.batch), 1);
      cache_evict_rows_kernel<TAB, V><<<dim3((unsigned)std::min(all, some), 2 * (unsigned)c.G, (unsigned)t.batch), 256, 0, st>>>(tab, c, w, elem_bytes, upr);
    };
    if (bits % 16 == 0) rows(uint4{});
    else if (bits % 4 == 0) rows(uint32_t{});
    else rows(uint16_t{});
  });
  return hipGetLastError();
}

}  // namespace skv
