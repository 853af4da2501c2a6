// Internal declarations of the operators on a cache in use (cache_*.hip, cache_api.cpp).
#pragma once
#include "common.h"

namespace skv {

// Per-sequence table of a call on a cache, by value in the kernel arguments like SeqTab: in two sizes, for the same reason.
template <int N>
struct CacheTab {
  int64_t cu[N + 1];      // first slots (capacities)
  int32_t cu_new[N + 1];  // fresh tokens (append, attend, accept)
  int32_t units[N + 1];   // cumulative blocks of query rows (attend) or workgroups (weights), or the budgets (evict)
  int32_t reach[N + 1];   // attend: cumulative stretches of slots whose weights a workgroup gathers
  int32_t batch;
};
using CacheTable = CacheTab<kMaxBatch>;
using SmallCacheTable = CacheTab<8>;
template <class F>
void with_cache_table(const CacheTable& s, F f) {
  if (s.batch > 8) { f(s); return; }
  SmallCacheTable t;
  for (int i = 0; i <= 8; ++i) { t.cu[i] = s.cu[i]; t.cu_new[i] = s.cu_new[i]; t.units[i] = s.units[i]; t.reach[i] = s.reach[i]; }
  t.batch = s.batch;
  f(t);
}

// ... of which the copies need less than half.
template <int N>
struct RowTab {
  int64_t cu[N + 1];
  int32_t cu_new[N + 1];
  int32_t batch;
};
template <int N>
RowTab<N> row_table(const CacheTable& s) {
  RowTab<N> t;
  for (int i = 0; i <= N; ++i) { t.cu[i] = s.cu[i]; t.cu_new[i] = s.cu_new[i]; }
  t.batch = s.batch;
  return t;
}
template <class F>
void with_row_table(const CacheTable& s, F f) {
  if (s.batch > 8) f(row_table<kMaxBatch>(s)); else f(row_table<8>(s));
}

// The cache as kernels see it.
struct CacheView {
  void *k, *v;
  int64_t sh, ss;         // strides in elements
  int64_t slots;          // of the whole cache: the stride of the planes
  float* mass;
  int32_t* pos;
  const int32_t* lens;
  int32_t* missed;
  int G, d, planes;
};

// How scores are formed: c2 = scale log2(e); capped (Cap), and biased by distance (biased).
struct ScoreForm {
  float scale, c2, softcap, inv_cap;
  const float* slopes;
  const uint64_t* tree;
};

// What a call reads at least of the cache to read it past the caches (half of what the memory-side cache holds).
constexpr int64_t kStreamBytes = (int64_t)128 << 20;

// How an attend call is cut: a workgroup takes `rows` query rows of one KV head and a chunk of a sequence's slots; `units` of them per KV head are
// shared out by the lengths on the device (Cuts).
constexpr int kAttendWaves = 4;
constexpr int kScorePad = 32;   // words behind a sequence's scores: tiles are stored whole
struct AttendPlan {
  int mfma;               // 1: the bf16 matrix kernels (cache_attend_bf16.hip, 128 rows: cache_attend_rows.hip), 0: the fp32 one
  int rows;               // query rows of a workgroup
  int min_chunk;          // least slots of a chunk: a tile for every wave
  int gather;             // the weights are gathered: the first launch leaves the scores in the workspace
  int stream;             // 1: the cache is read past the caches (see cache_attend_bf16.hip)
  int join;               // a second launch joins the chunks (and gathers); else the first one writes out and lse
  int64_t units;          // workgroups of the first launch per KV head
  int64_t most_chunks;    // of a sequence when all are full
  size_t off_shares, off_ml, off_o, off_x, total_bytes;   // workspace: shares, (M, Z) and sums of the chunks, scores [H][slots]
};

struct AttendWork {
  const void* q;
  int64_t qst, qsh;
  void* out;
  float* lse;
  float *ml, *o, *x;      // partial results [workgroup][row of it], (M, Z) and sums of the padded head dim; x NULL: no weights
  int4* shares;           // [sequence] how the units were shared out: the first one, chunks, chunks with slots, slots in use
  int H, gs, min_chunk, units;
  uint32_t gs_recip;      // floor(2^32 / gs) + 1: divides a sequence's rows (below 2^18) exactly; 0: gs is 1
  float lambda;
  int64_t rows;           // new tokens x H
  int64_t xs;             // scores: head h, slot s of sequence b at h xs + cu[b] + kScorePad b + s
};

hipError_t launch_cache_append(const CacheTable& t, const CacheView& c, const void* k_new, const void* v_new, int64_t nsh,
                               int64_t nst, const int32_t* pos_new, const float* mass_new, int64_t nsp, int elem_bytes,
                               int32_t* lens_out, hipStream_t st);
hipError_t launch_cache_attend_f32(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p,
                                   const AttendWork& w, bool bf16, hipStream_t st);
// a plan with mfma set and 128 rows
hipError_t launch_cache_attend_rows(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p,
                                    const AttendWork& w, hipStream_t st);
// a plan with mfma set and 16 or 32
hipError_t launch_cache_attend_bf16(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p,
                                    const AttendWork& w, hipStream_t st);
hipError_t launch_cache_combine(const CacheTable& t, const CacheView& c, const AttendPlan& p, const AttendWork& w, bool bf16,
                                hipStream_t st);
hipError_t launch_cache_weights_f32(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendWork& w,
                                    const int32_t* path, const int32_t* n_accept, bool bf16, hipStream_t st);
// caches and queries that the bf16 matrix kernels take
hipError_t launch_cache_weights_bf16(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendWork& w,
                                     const int32_t* path, const int32_t* n_accept, hipStream_t st);
hipError_t launch_cache_accept(const CacheTable& t, const CacheView& c, const int32_t* path, const int32_t* n_accept,
                               int elem_bytes, int32_t* lens_out, hipStream_t st);
// Up to this capacity of the longest sequence a workgroup holds a sequence's keys in registers; beyond, the launches take turns at digits of
// them through records in the workspace: per plane and sequence evict_hist_words() words, per plane and share of a sequence's slots
// (evict_shares of its capacity) the largest position and four counts.
constexpr int64_t kEvictShort = 32768;
int evict_shares(int64_t cap);
size_t evict_hist_words();
struct EvictWork {
  const float* scores;
  int keep_tail;
  int32_t* lens_out;
  int32_t* count;         // [planes][batch] slots that move
  int32_t *holes, *moved; // [planes][slots of the cache]: where they go and come from, a sequence's from its first slot's place on
  uint32_t* hist;         // longer caches: [planes][batch][evict_hist_words()], ...
  int32_t* tops;          //                [planes][shares], ...
  uint32_t* counts;       //                [planes][shares][4]
};
hipError_t launch_cache_evict(const CacheTable& t, const CacheView& c, const EvictWork& w, int elem_bytes, hipStream_t st);

#ifdef __HIPCC__
// a sequence's slots in use, and its fresh tokens' first slot: negative where they are not there
struct Held {
  int n, base, fresh;
  int64_t lo;
};
template <class TAB>
__device__ __forceinline__ Held held(const TAB& t, const CacheView& c, int b) {
  Held h;
  h.lo = t.cu[b];
  const int32_t len = c.lens[b], missed = c.missed ? c.missed[b] : 0;
  h.n = max(0, (int)min((int64_t)len, t.cu[b + 1] - t.cu[b]));
  h.fresh = t.cu_new[b + 1] - t.cu_new[b];
  h.base = missed ? -1 : h.n - h.fresh;
  return h;
}

constexpr float kLog2e = 1.4426950408889634f;
// c tanh(y / c) of products s, y = scale s, in units of which the scores' own has `unit`, with errors of a few 2^-24 of the result: what is off by
// c's own roundings, as c - 2 c / (1 + e) is, shows in lse and in the weights of accepted drafts, which are fp32.
// u = y / c.  Near zero c u (1 + w P(w)), w = u^2, P of five terms that fit (tanh(u) / u - 1) / w up to u = 3/4 (1 + w P off by 3.3e-8 of itself).
// Beyond, c (1 - e) / (1 + e), e = exp(-2 |u|) < 0.23: what e is off by counts 2 e / (1 - e^2) < 0.48.
struct Cap {
  float in, in2, reach, top, c1, c2, c3, c4, c5;   // reach: the largest product near zero
  __device__ __forceinline__ Cap(const ScoreForm& f, float unit)
      : in(f.scale * f.inv_cap), in2(in * 2.885390082f), reach(0.75f / in), top(f.softcap * unit), c1(top * -0.33333068f),
        c2(top * 0.13326522f), c3(top * -0.05339028f), c4(top * 0.01966496f), c5(top * -0.00476953f) {}
  __device__ __forceinline__ float near_zero(float s) const {
    const float u = s * in, w = u * u;
    return u * fmaf(w, fmaf(w, fmaf(w, fmaf(w, fmaf(w, c5, c4), c3), c2), c1), top);
  }
  __device__ __forceinline__ float operator()(float s) const {
    const float e = __builtin_amdgcn_exp2f(-in2 * fabsf(s));
    const float far = copysignf(top * ((1.f - e) * __builtin_amdgcn_rcpf(1.f + e)), s);
    return fabsf(s) > reach ? far : near_zero(s);   // (NaN stays NaN)
  }
  // four at once: mostly all of a wave's are near zero, which spares them the exponential and the reciprocal (four trees of 64 drafts over 8K to
  // 16.5K slots, capped at 30: 114 us, sixteen at once 123, where rows with a few large scores hold up the others; without a cap 97)
  __device__ __forceinline__ void apply(float (&x)[4]) const {
    if (__any(fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3]))) > reach)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (*this)(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = near_zero(x[i]);
    }
  }
};
// products as scores in their own units, capped or not
__device__ __forceinline__ void scaled(const ScoreForm& f, const Cap& cap, float (&x)[4]) {
  if (f.softcap > 0.f) {
    cap.apply(x);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= f.scale;
  }
}
// a score biased by distance, in the log2 domain
__device__ __forceinline__ float biased(float y, float slope, int distance) { return fmaf(-slope, (float)distance, y) * kLog2e; }
// whether fresh token t (mask: its bits) sees slot s < n
__device__ __forceinline__ bool sees(uint64_t mask, int s, int base) { return s < base || ((mask >> (s - base)) & 1); }
__device__ __forceinline__ uint64_t row_mask(const ScoreForm& f, int64_t r, int t) {
  return f.tree ? f.tree[r] : (t >= 63 ? ~0ull : (2ull << t) - 1ull);
}

constexpr float kNothingSeen = -3.4028235e38f;   // the reference of a row that has seen nothing: no score that counts lies below

typedef __attribute__((ext_vector_type(4))) float floatx4;

// token of a sequence's row
__device__ __forceinline__ int token_of(const AttendWork& w, int row) { return w.gs_recip ? (int)__umulhi((uint32_t)row, w.gs_recip) : row; }

// What an attend kernel's workgroup leaves: the sums O (unnormalised), maxima M and normalisers Z of its chunk, log2 domain.
// Every wave holds 16 x RB rows over its own slots, in the layout of a 16x16 matrix result of V^T P^T: lane l has row l % 16 of
// each block and components 16 db + 4 (l / 16) .. +3; M is the same in a row's four lanes, Z each lane's own share.
// The waves' results are added up in wave order through LDS (buf: kFinishFloats), and written out by all threads: as the chunk's partial
// result, or, where a sequence has one chunk at most, as out and lse.
template <int DP, int RB>
constexpr int kFinishFloats = kAttendWaves * 16 * RB * (DP + 4 + 2);
template <class T> __device__ __forceinline__ void put_out(T* p, float x);
template <> __device__ __forceinline__ void put_out<float>(float* p, float x) { *p = x; }
template <> __device__ __forceinline__ void put_out<uint16_t>(uint16_t* p, float x) {
  const uint32_t u = __float_as_uint(x);   // round to nearest, ties to even; NaN stays NaN
  *p = x != x ? 0x7FC0 : (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}
// components c .. c + 3 of row r of a KV head's rows, as the chunk's partial result or, with one chunk, as out and lse
template <class T, int DP>
__device__ __forceinline__ void leave(const AttendWork& w, int d, int g, int r, int c, float top, float z, floatx4 o, int new0, int64_t part, int nc) {
  const int t = token_of(w, r);
  const int head = g * w.gs + (r - t * w.gs);
  const int64_t at = (int64_t)(new0 + t) * w.H + head;
  if (nc == 1 && !w.x) {
    const float inv = z != 0.f ? 1.f / z : 0.f;   // (NaN stays NaN)
    for (int i = 0; i < 4 && c + i < d; ++i) put_out<T>((T*)w.out + at * d + c + i, o[i] * inv);
    if (c == 0) w.lse[at] = z != 0.f ? (top + __builtin_amdgcn_logf(z)) * 0.6931471806f : -INFINITY;
  } else {
    *reinterpret_cast<floatx4*>(w.o + part * DP + c) = o;
    if (c == 0) { w.ml[part * 2] = top; w.ml[part * 2 + 1] = z; }
  }
}
template <class T, int DP, int RB>
__device__ __forceinline__ void finish_chunk(const floatx4 (&O)[DP / 16][RB], const float (&M)[RB], const float (&Zl)[RB],
                                             float* buf, const AttendWork& w, int d, int g, int row0, int rows, int new0, int nc) {
  constexpr int ROWS = 16 * RB, W = DP + 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q4 = lane >> 4;
  float* ml = buf + kAttendWaves * ROWS * W;   // [wave][row][2]
  float Z[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    Z[rb] = Zl[rb] + __shfl_xor(Zl[rb], 16);
    Z[rb] += __shfl_xor(Z[rb], 32);
  }
  __syncthreads();   // (buf lies where the waves kept their tiles)
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
    if (q4 == 0) {
      ml[(wave * ROWS + rb * 16 + l16) * 2] = M[rb];
      ml[(wave * ROWS + rb * 16 + l16) * 2 + 1] = Z[rb];
    }
  __syncthreads();
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = rb * 16 + l16;
    float top = ml[row * 2];
    for (int i = 1; i < kAttendWaves; ++i) top = fmaxf(top, ml[(i * ROWS + row) * 2]);
    const float f = __builtin_amdgcn_exp2f(M[rb] - top);
#pragma unroll
    for (int db = 0; db < DP / 16; ++db)
      *reinterpret_cast<floatx4*>(buf + (wave * ROWS + row) * W + db * 16 + 4 * q4) = O[db][rb] * f;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < ROWS * (DP / 4); e += 64 * kAttendWaves) {
    const int row = e / (DP / 4), c = e % (DP / 4) * 4;
    if (row0 + row >= rows || c >= d) continue;
    float top = ml[row * 2];
    for (int i = 1; i < kAttendWaves; ++i) top = fmaxf(top, ml[(i * ROWS + row) * 2]);
    float z = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < kAttendWaves; ++i) {
      z += ml[(i * ROWS + row) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(i * ROWS + row) * 2] - top);
      o += *reinterpret_cast<const floatx4*>(buf + (i * ROWS + row) * W + c);
    }
    leave<T, DP>(w, d, g, row0 + row, c, top, z, o, new0, (int64_t)blockIdx.x * ROWS + row, nc);
  }
}

// over the 64 lanes, by moves inside the rows of 16 and then between them (six vector instructions; shuffles take as many trips through the
// LDS crossbar): a lane's sum up to itself
__device__ __forceinline__ uint32_t sum_up(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);
  return x;
}
__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

// How the units of an attend call are shared out, sequence b in lane b: chunks of one length for all, so that workgroups end together however
// the lengths differ (a sequence of 16384 slots among 31 of 500, room for 16384 each: 28 us, by their room 86; 32 lengths spread evenly up to
// 16384: 171 and 182).  The length is the mean slots of a unit, made longer by a 16th until the chunks are no more than the units;
// the host sees to it that one chunk each is not.
struct Cuts {
  uint32_t n;        // slots in use, 0 where the fresh tokens are not among them for want of room
  uint32_t rcs, nc;  // blocks of query rows, chunks
  uint32_t end;      // units of the sequences up to this one
  int len;           // slots of a chunk, whole tiles
};
template <class TAB>
__device__ __forceinline__ Cuts cuts_of(const TAB& t, const CacheView& cache, const AttendWork& w) {
  const int lane = threadIdx.x & 63, b = min(lane, t.batch - 1);
  Cuts c;
  const int32_t len = cache.lens[b], missed = cache.missed ? cache.missed[b] : 0, fresh = t.cu_new[b + 1] - t.cu_new[b];
  const int64_t cap = t.cu[b + 1] - t.cu[b];
  c.n = missed ? 0u : (uint32_t)max(0, (int)min((int64_t)len, cap));
  c.rcs = lane < t.batch ? (uint32_t)(t.units[b + 1] - t.units[b]) : 0u;
  const uint32_t tiles = (int)c.n < fresh ? 0u : (c.n + 31u) / 32u, units = (uint32_t)w.units;
  const uint64_t mine = (uint64_t)tiles * c.rcs;   // (below 2^26 x 2^18; the sums of its halves stay below 2^32)
  const uint64_t total = ((uint64_t)from_lane(sum_up((uint32_t)(mine >> 24)), 63) << 24) + from_lane(sum_up((uint32_t)mine & 0xFFFFFFu), 63);
  uint32_t len32 = total >> 31 ? (uint32_t)((total + units - 1) / units) : ((uint32_t)total + units - 1) / units;
  len32 = max(len32, (uint32_t)w.min_chunk / 32u);
  for (;;) {
    c.nc = max(1u, (tiles + len32 - 1) / len32);
    c.end = sum_up(c.rcs * c.nc);
    if (from_lane(c.end, 63) <= units) break;
    len32 += (len32 + 15) / 16;
  }
  c.len = (int)min((uint64_t)len32 * 32, (uint64_t)0x7FFFFFFF);
  return c;
}

// workgroup -> (sequence, chunk, block of rows, KV head): the heads vary fastest, so that the workgroups which read the same
// slots for other rows are a multiple of the heads apart.  b < 0: a unit that nobody needs.
struct AttendPlace {
  int b, chunk, rc, g, nc;
  int s0, s1;   // the chunk's slots
  Held h;       // (n is 0 for a sequence that holds less than its fresh tokens)
};
template <class TAB>
__device__ __forceinline__ AttendPlace attend_place(const TAB& t, const CacheView& c, const AttendWork& w) {
  AttendPlace p;
  const Cuts k = cuts_of(t, c, w);
  const bool shifts = (c.G & (c.G - 1)) == 0;   // (a division costs some 40 instructions)
  const int u = shifts ? (int)(blockIdx.x >> __builtin_ctz(c.G)) : (int)(blockIdx.x / c.G);
  p.g = blockIdx.x - u * c.G;
  if (w.shares && blockIdx.x == 0 && (int)threadIdx.x < t.batch) {
    const int fresh = t.cu_new[threadIdx.x + 1] - t.cu_new[threadIdx.x];
    w.shares[threadIdx.x] = make_int4((int)(k.end - k.rcs * k.nc), (int)k.nc, (int)k.n < fresh || k.n == 0 ? 0 : (int)k.nc, (int)k.n);
  }
  p.b = __popcll(__ballot(k.end <= (uint32_t)u));
  if (p.b >= t.batch) { p.b = -1; return p; }
  const int rcs = (int)from_lane(k.rcs, p.b);
  p.nc = (int)from_lane(k.nc, p.b);
  const int at = u - ((int)from_lane(k.end, p.b) - rcs * p.nc);
  p.chunk = rcs == 1 ? at : at / rcs;
  p.rc = at - p.chunk * rcs;
  p.h.lo = t.cu[p.b];
  p.h.n = (int)from_lane(k.n, p.b);
  p.h.fresh = t.cu_new[p.b + 1] - t.cu_new[p.b];
  p.h.base = p.h.n - p.h.fresh;
  if (p.h.base < 0) p.h.n = 0;
  p.s0 = (int)min((int64_t)p.h.n, (int64_t)p.chunk * k.len);
  p.s1 = (int)min((int64_t)p.h.n, (int64_t)p.s0 + k.len);
  return p;
}
#endif

}  // namespace skv
