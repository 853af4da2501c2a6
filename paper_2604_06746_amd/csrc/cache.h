// Internal declarations of the operators on a cache in use (cache_*.hip, cache_api.cpp).
#pragma once
#include "common.h"

namespace skv {

// Per-sequence table of a call on a cache, by value in the kernel arguments like SeqTab: in two sizes, for the same reason.
template <int N>
struct CacheTab {
  int64_t cu[N + 1];      // first slots (capacities)
  int32_t cu_new[N + 1];  // fresh tokens (append, attend, accept)
  int32_t units[N + 1];   // cumulative workgroups (attend: x KV heads), or the budgets (evict)
  int32_t part[N + 1];    // attend: cumulative partial results (rows x chunks)
  int32_t reach[N + 1];   // ... and stretches of slots whose weights a workgroup gathers
  int32_t batch;
};
using CacheTable = CacheTab<kMaxBatch>;
using SmallCacheTable = CacheTab<8>;
template <class F>
void with_cache_table(const CacheTable& s, F f) {
  if (s.batch > 8) { f(s); return; }
  SmallCacheTable t;
  for (int i = 0; i <= 8; ++i) { t.cu[i] = s.cu[i]; t.cu_new[i] = s.cu_new[i]; t.units[i] = s.units[i]; t.part[i] = s.part[i]; t.reach[i] = s.reach[i]; }
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
  int G, d, planes;
};

// How scores are formed: c2 = scale log2(e); with a cap or slopes in full (MORE in the kernels).
struct ScoreForm {
  float scale, c2, softcap, inv_cap;
  const float* slopes;
  const uint64_t* tree;
};

// What a call reads at least of the cache to read it past the caches (half of what the memory-side cache holds).
constexpr int64_t kStreamBytes = (int64_t)128 << 20;

// How an attend call is cut: a workgroup takes 16 rb query rows of one KV head and one of nc chunks of the sequence's slots
// (nc: the table's units / row blocks).
constexpr int kAttendWaves = 4;
constexpr int kScorePad = 32;   // words behind a sequence's scores: tiles are stored whole
struct AttendPlan {
  int mfma;               // 1: the bf16 matrix kernel (cache_attend_bf16.hip), 0: the fp32 one (cache_attend_f32.hip)
  int rb;                 // 16-row blocks of a workgroup
  int min_chunk;          // least slots of a chunk: a tile for every wave
  int gather;             // the weights are gathered: the first launch leaves the scores in the workspace
  int stream;             // 1: the cache is read past the caches (see cache_attend_bf16.hip)
  int join;               // a second launch joins the chunks (and gathers); else the first one writes out and lse
  int64_t blocks;         // workgroups of the first launch
  int64_t most_chunks;    // of a sequence
  size_t off_ml, off_o, off_x, total_bytes;   // workspace: (M, Z) and sums of the chunks, scores [H][slots]
};

struct AttendWork {
  const void* q;
  int64_t qst, qsh;
  void* out;
  float* lse;
  float *ml, *o, *x;      // partial results as the table numbers them, [.][2] and [.][padded head dim]; x NULL: no weights
  int H, gs, min_chunk;
  uint32_t gs_recip;      // floor(2^32 / gs) + 1: divides a sequence's rows (below 2^18) exactly; 0: gs is 1
  float lambda;
  int64_t rows;           // new tokens x H
  int64_t xs;             // scores: head h, slot s of sequence b at h xs + cu[b] + kScorePad b + s
};

// Slots of a chunk when n of them are cut into at most nc: whole tiles for every wave.
__host__ __device__ inline int chunk_slots(int n, int nc, int min_chunk) {
  const int per = (n + nc - 1) / nc;
  return per <= min_chunk ? min_chunk : (per + 31) / 32 * 32;
}

hipError_t launch_cache_append(const CacheTable& t, const CacheView& c, const void* k_new, const void* v_new, int64_t nsh,
                               int64_t nst, const int32_t* pos_new, const float* mass_new, int64_t nsp, int elem_bytes,
                               int32_t* lens_out, hipStream_t st);
hipError_t launch_cache_attend_f32(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p,
                                   const AttendWork& w, bool bf16, hipStream_t st);
// a plan with mfma set
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
// a sequence's slots in use, and its fresh tokens' first slot; see: false where its rows see nothing
struct Held {
  int n, base, fresh;
  int64_t lo;
};
template <class TAB>
__device__ __forceinline__ Held held(const TAB& t, const int32_t* lens, int b) {
  Held h;
  h.lo = t.cu[b];
  h.n = max(0, (int)min((int64_t)lens[b], t.cu[b + 1] - t.cu[b]));
  h.fresh = t.cu_new[b + 1] - t.cu_new[b];
  h.base = h.n - h.fresh;
  return h;
}

// z of a score in full: capped, and biased by distance; in the log2 domain.
// tanh(y) = (1 - e) / (1 + e), e = exp(-2 |y|); below 1/4, where 1 - e cancels, its series (relative error of either < 4e-7).
__device__ __forceinline__ float tanh_of(float y) {
  const float a = fabsf(y), y2 = y * y;
  const float e = __builtin_amdgcn_exp2f(-2.885390082f * a);
  const float big = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), y);
  const float small = fmaf(y * y2, fmaf(y2, fmaf(y2, fmaf(y2, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), y);
  return a < 0.25f ? small : big;
}
__device__ __forceinline__ float full_score(const ScoreForm& f, float s, float slope, int distance) {
  float y = s * f.scale;
  if (f.softcap > 0.f) y = f.softcap * tanh_of(y * f.inv_cap);
  if (f.slopes) y = fmaf(-slope, (float)distance, y);
  return y * 1.4426950408889634f;
}
// whether fresh token t (mask: its bits) sees slot s < n
__device__ __forceinline__ bool sees(uint64_t mask, int s, int base) { return s < base || ((mask >> (s - base)) & 1); }
__device__ __forceinline__ uint64_t row_mask(const ScoreForm& f, int64_t r, int t) {
  return f.tree ? f.tree[r] : (t >= 63 ? ~0ull : (2ull << t) - 1ull);
}

constexpr float kNothingSeen = -1.0e30f;   // the reference of a row that has seen nothing

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
template <class T, int DP, int RB>
__device__ __forceinline__ void finish_chunk(const floatx4 (&O)[DP / 16][RB], const float (&M)[RB], const float (&Zl)[RB],
                                             float* buf, const AttendWork& w, int d, int g, int row0, int rows, int new0, int64_t part0, int nc,
                                             int chunk) {
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
    const int r = row0 + row, t = token_of(w, r);
    const int head = g * w.gs + (r - t * w.gs);
    const int64_t at = (int64_t)(new0 + t) * w.H + head;
    if (nc == 1 && !w.x) {
      const float inv = z > 0.f ? 1.f / z : 0.f;
      for (int i = 0; i < 4 && c + i < d; ++i) put_out<T>((T*)w.out + at * d + c + i, o[i] * inv);
      if (c == 0) w.lse[at] = z > 0.f ? (top + __builtin_amdgcn_logf(z)) * 0.6931471806f : -INFINITY;
    } else {
      const int64_t part = part0 + ((int64_t)t * w.H + head) * nc + chunk;
      *reinterpret_cast<floatx4*>(w.o + part * DP + c) = o;
      if (c == 0) { w.ml[part * 2] = top; w.ml[part * 2 + 1] = z; }
    }
  }
}

// workgroup -> (sequence, chunk, block of rows, KV head): the heads vary fastest, so that the workgroups which read the same
// slots for other rows are a multiple of the heads apart
struct AttendPlace {
  int b, chunk, rc, g, nc;
};
template <class TAB>
__device__ __forceinline__ AttendPlace attend_place(const TAB& t, int G, int gs, int rows_wg) {
  AttendPlace p;
  const bool shifts = (G & (G - 1)) == 0;   // (a division costs some 40 instructions)
  const int u = shifts ? (int)(blockIdx.x >> __builtin_ctz(G)) : (int)(blockIdx.x / G);
  p.g = blockIdx.x - u * G;
  int b = 0;
  while (b + 1 < t.batch && u >= t.units[b + 1]) ++b;
  const int rcs = ((t.cu_new[b + 1] - t.cu_new[b]) * gs + rows_wg - 1) / rows_wg;
  p.b = b;
  const int units = t.units[b + 1] - t.units[b], at = u - t.units[b];
  p.nc = rcs == 1 ? units : units / rcs;
  p.chunk = rcs == 1 ? at : at / rcs;
  p.rc = at - p.chunk * rcs;
  return p;
}
#endif

}  // namespace skv
