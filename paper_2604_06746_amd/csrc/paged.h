// Internal declarations of the operators on a cache held in 8 bits, in pages (paged_*.hip, paged_api.cpp).
#pragma once
#include "cache.h"
#include "rotary.h"

#include <cmath>

namespace skv {

// The cache as kernels see it.
struct PagedView {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int64_t sp, sh, st;       // strides in elements, which are bytes
  const int32_t* pages;
  int64_t pst;
  const int32_t* lens;
  float* mass;
  int32_t* missed;
  int G, d, shift, n_pages, max_pages, batch;   // shift: log2 of the page size
};

constexpr int kBlock = 16;        // slots that share a page whatever its size: what the attend kernels go by
constexpr float kTopCode = 448.f;
constexpr float kLeastScale = 0x1p-64f, kMostScale = 0x1p64f;

// Fresh tokens of the sequences, by value in the kernel arguments.
template <int N>
struct FreshTab {
  int32_t cu_new[N + 1];
  int32_t batch;
};
template <class F>
void with_fresh_table(const CacheTable& s, F f) {
  auto take = [&](auto t) {
    constexpr int n = sizeof(t.cu_new) / sizeof(int32_t);
    for (int i = 0; i < n; ++i) t.cu_new[i] = s.cu_new[i];
    t.batch = s.batch;
    f(t);
  };
  if (s.batch > 8) take(FreshTab<kMaxBatch>{}); else take(FreshTab<8>{});
}

struct PagedRows {
  const void *k, *v;
  int64_t sh, st;
  const int32_t* pos;       // or NULL: positions are the slots'
  RotaryView rotary;
  const void* q;            // or NULL
  int64_t qst, qsh;
  void* q_out;
  int H;
  int32_t* lens_out;
};
hipError_t launch_paged_append(const CacheTable& t, const PagedView& c, const PagedRows& w, bool bf16, hipStream_t st);

// Waves of a workgroup that takes a whole short sequence's slots, so that nothing has to be joined.
constexpr int kShortWaves = 8;
// An attend call is cut like one on a cache of slots (AttendPlan, AttendWork): x in AttendWork are here the weights of blocks of kBlock slots
// as their log2, head h, block i of sequence b at h xs + b blocks + i.  Weights in units of 2^u that are not small are kApart there, and the pair
// (u, log2 in those units) lies at twice that place behind all of them.
constexpr float kSmallUnit = 1024.f, kApart = INFINITY;
struct PagedUnit {
  float unit, weight;
};
struct PagedPlan : AttendPlan {
  int waves;   // of a workgroup: kAttendWaves, or kShortWaves (16 rows, nothing to join)
};
hipError_t launch_paged_attend(const CacheTable& t, const CacheView& v, const PagedView& c, const ScoreForm& f, const PagedPlan& p,
                               const AttendWork& w, bool bf16, hipStream_t st);
// a plan that gathers the weights: the chunks joined, and mass <- lambda mass + what the heads' blocks hold
hipError_t launch_paged_join(const CacheTable& t, const PagedView& c, const AttendWork& w, bool bf16, hipStream_t st);

#ifdef __HIPCC__
// The sequence of packed row r, which grows by little over the lanes: the count of those that end at or before the first lane's row, by a
// look of each lane at one end (one behind the other they cost 64 sequences 3 us), and on from there.
template <class TAB>
__device__ __forceinline__ int sequence_of(const TAB& t, int r) {
  const int lane = threadIdx.x & 63, first = __builtin_amdgcn_readfirstlane(r);
  int b = __popcll(__ballot(lane < t.batch && t.cu_new[min(lane, t.batch - 1) + 1] <= first));
  while (b + 1 < t.batch && r >= t.cu_new[b + 1]) ++b;
  return b;
}
// slots in use
__device__ __forceinline__ int paged_len(const PagedView& c, int b) {
  return (int)min((int64_t)max(c.lens[b], 0), (int64_t)c.max_pages << c.shift);
}
#endif

}  // namespace skv
