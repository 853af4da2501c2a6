// Attention of fresh tokens over a cache, and the accepted drafts' weights, in fp32 matrix instructions: fp32 caches, and bf16 ones
// (widened exactly) whose head dimension, alignment or strides the bf16 kernels do not take.
//
// x = z(scale q.k), a = softmax(x), out = a V, one pass over the cache: every wave keeps for its rows a running maximum M, Z = sum
// 2^(x-M) and O = sum 2^(x-M) v, and rescales Z and O when M grows.  S^T = K Q^T puts a row's scores of 16 slots into four lanes,
// four consecutive slots each, which is how the second product, O^T = V^T P^T, wants its right operand: P never leaves the lane.
// A wave works on its own tiles of 16 slots (LDS of its own, no barrier in the loop), the next tile's rows are loaded into registers
// meanwhile; the four waves of a workgroup take turns at a chunk's tiles and are joined at its end (finish_chunk).  M follows lazily, as in
// cache_attend_bf16.hip: the usual tile has no exchange between lanes and no rescaling.
//
// Single tokens are bound by reading the cache (8 x 32768 slots of 8 heads, 128 components: 338 us, 6.4 TB/s), trees by the waits between matrix
// and other instructions of two waves a SIMD (64 drafts over 8192 slots 129 us, 67 TFLOP/s of 154; 13 over four times 12.9K 228 us; in one run the first took
// 121 us, capped at 30 124).  On these two, lazy M gave 142 -> 136 and 247 -> 233, the priority the rest; two blocks of rows a workgroup 155 and 254 (registers), operands straight from memory
// 151 and 270.
#include "cache.h"

namespace skv {
namespace {

template <class T>
__device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen<float>(float x) { return x; }
template <> __device__ __forceinline__ float widen<uint16_t>(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// components c .. c+3 of a row; zeros from component d on.  VEC: the row is aligned to four elements and d a multiple of them
template <class T, bool VEC, bool NT = false>
__device__ __forceinline__ floatx4 load4(const T* row, int c, int d) {
  floatx4 r = {0.f, 0.f, 0.f, 0.f};
  if (VEC) {
    if (c < d) {
      typedef __attribute__((ext_vector_type(4))) T vec;
      const vec* at = reinterpret_cast<const vec*>(row + c);
      const vec x = NT ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = widen<T>(x[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < d) r[i] = widen<T>(row[c + i]);
  }
  return r;
}
// what a wave wrote to its part of the LDS is there for its own lanes (they run in step; this keeps the compiler from moving it)
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kTile = 16;
constexpr float kSlack = 8.f;   // how far above its reference a score may lie, log2

// S^T of a tile in LDS against 16 rows held as operands: lane l gets row l % 16, slots 4 (l / 16) .. +3.  Four sums that are added up at the
// end: a score of 45 is a dot product of 500, whose 128 terms added one behind the other are off by three times as much.
template <int DP>
__device__ __forceinline__ floatx4 tile_scores(const float* kt, const floatx4 (&qf)[DP / 16], int l16, int q4) {
  floatx4 acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const floatx4 kf = *reinterpret_cast<const floatx4*>(kt + l16 * (DP + 4) + s * 16 + 4 * q4);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j], qf[s][j], acc[j], 0, 0, 0);
  }
  return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

template <class TAB, class T, int DP, bool VEC, bool NT>
__global__ __launch_bounds__(64 * kAttendWaves) void cache_attend_f32_kernel(TAB tab, CacheView c, ScoreForm f, AttendWork w) {
  constexpr int W = DP + 4, UNITS = kTile * DP / 4 / 64;   // float4 units of a tile per lane
  constexpr int RING = kAttendWaves * 2 * kTile * W, FIN = kFinishFloats<DP, 1>;
  __shared__ __attribute__((aligned(16))) float lds[RING > FIN ? RING : FIN];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), l16 = lane & 15, q4 = lane >> 4;
  const AttendPlace p = attend_place(tab, c, w);
  if (p.b < 0) return;
  const Held& h = p.h;
  const int n = h.n, s0 = p.s0, s1 = p.s1;
  // the queries first: the length has no part in their addresses
  const int new0 = tab.cu_new[p.b], rows = h.fresh * w.gs, row0 = p.rc * 16;
  const int row = min(row0 + l16, rows - 1), t = token_of(w, row), head = p.g * w.gs + row - t * w.gs;
  const int64_t r = new0 + t;
  const T* qrow = (const T*)w.q + r * w.qst + (int64_t)head * w.qsh;
  floatx4 qf[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) qf[s] = load4<T, VEC>(qrow, s * 16 + 4 * q4, c.d);
  const uint64_t mask = row_mask(f, r, t);
  const bool more = f.softcap > 0.f || f.slopes;
  const Cap cap(f, 1.f);
  const float slope = f.slopes ? f.slopes[head] : 0.f;
  if (s0 >= s1 && (p.nc > 1 || w.x)) return;   // (the join reads no more chunks than have slots)
  const int32_t* pos = f.slopes ? c.pos + (c.planes > 1 ? p.g * c.slots : 0) + h.lo : nullptr;
  const T* kg = (const T*)c.k + (int64_t)p.g * c.sh + h.lo * c.ss;
  const T* vg = (const T*)c.v + (int64_t)p.g * c.sh + h.lo * c.ss;
  float* kt = lds + wave * 2 * kTile * W;
  float* vt = kt + kTile * W;

  floatx4 O[DP / 16][1];
  float M[1] = {kNothingSeen}, Z[1] = {0.f};
#pragma unroll
  for (int i = 0; i < DP / 16; ++i) O[i][0] = floatx4{0.f, 0.f, 0.f, 0.f};

  floatx4 kr[UNITS], vr[UNITS];
  int from[4] = {};   // positions of the lane's slots
  auto fetch = [&](int j0) __attribute__((always_inline)) {
    if (pos) {
#pragma unroll
      for (int i = 0; i < 4; ++i) from[i] = pos[min(j0 + 4 * q4 + i, n - 1)];
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int e = u * 64 + lane, s = min(j0 + e / (DP / 4), n - 1), col = e % (DP / 4) * 4;
      kr[u] = load4<T, VEC, NT>(kg + (int64_t)s * c.ss, col, c.d);
      vr[u] = load4<T, VEC, NT>(vg + (int64_t)s * c.ss, col, c.d);
    }
  };
  int j0 = s0 + wave * kTile;
  uint64_t odd = 0;
  if (j0 < s1) fetch(j0);
  const int at = pos && n > 0 ? pos[h.base + t] : 0;
  for (; j0 < s1; j0 += kAttendWaves * kTile) {
    wave_lds_fence();
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int e = u * 64 + lane, s = e / (DP / 4), col = e % (DP / 4) * 4;
      floatx4 v = vr[u];
      if (j0 + s >= h.base) {   // a fresh slot: what is not a number would reach rows that do not see it (0 x NaN)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!(fabsf(v[i]) < INFINITY)) {
            v[i] = 0.f;
            if (j0 + s < n) odd |= 1ull << (j0 + s - h.base);   // (rows that see it get NaN in the end)
          }
        }
      }
      *reinterpret_cast<floatx4*>(kt + s * W + col) = kr[u];
      *reinterpret_cast<floatx4*>(vt + s * W + col) = v;
    }
    wave_lds_fence();
    __builtin_amdgcn_s_setprio(0);
    const int far[4] = {at - from[0], at - from[1], at - from[2], at - from[3]};
    if (j0 + kAttendWaves * kTile < s1) fetch(j0 + kAttendWaves * kTile);
    // ahead of the other workgroup's waves until the tile is done, lest both be at the same instructions
    __builtin_amdgcn_s_setprio(1);
    const floatx4 acc = tile_scores<DP>(kt, qf, l16, q4);
    float x[4] = {acc[0], acc[1], acc[2], acc[3]};
    if (more) scaled(f, cap, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = j0 + 4 * q4 + i;
      const bool seen = s < s1 && sees(mask, min(s, n - 1), h.base);
      x[i] = more ? biased(x[i], slope, far[i]) : x[i] * f.c2;
      if (!seen) x[i] = -INFINITY;
      if (w.x && s < s1 && row0 + l16 < rows) w.x[head * w.xs + h.lo + kScorePad * p.b + s] = x[i];
    }
    float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    if (__any(top - M[0] > kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float Mn = fmaxf(M[0], top), shrink = __builtin_amdgcn_exp2f(M[0] - Mn);
      M[0] = Mn;
      Z[0] *= shrink;
#pragma unroll
      for (int db = 0; db < DP / 16; ++db) O[db][0] *= shrink;
    }
    float pr[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) pr[i] = __builtin_amdgcn_exp2f(x[i] - M[0]);
    Z[0] += (pr[0] + pr[1]) + (pr[2] + pr[3]);
#pragma unroll
    for (int db = 0; db < DP / 16; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        O[db][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(vt[(4 * q4 + i) * W + db * 16 + l16], pr[i], O[db][0], 0, 0, 0);
  }
  if (__any(odd != 0)) {
    for (int m = 1; m < 64; m <<= 1) odd |= (uint64_t)__shfl_xor((unsigned long long)odd, m);
#pragma unroll
    for (int db = 0; db < DP / 16; ++db) O[db][0] *= mask & odd ? NAN : 1.f;
  }
  finish_chunk<T, DP, 1>(O, M, Z, lds, w, c.d, p.g, row0, rows, new0, p.nc);
}

// Weights of the accepted drafts: a wave takes 16 slots of a plane, goes through the plane's KV heads and their accepted rows, and adds up
// each slot's weights in its lanes; no two waves share a slot, so the sums need no atomics and come in one order.
template <class TAB, class T, int DP, bool VEC>
__global__ __launch_bounds__(256) void cache_weights_f32_kernel(TAB tab, CacheView c, ScoreForm f, AttendWork w,
                                                                const int32_t* __restrict__ path, const int32_t* __restrict__ n_accept) {
  constexpr int W = DP + 4, UNITS = kTile * DP / 4 / 64;
  __shared__ __attribute__((aligned(16))) float lds[4 * kTile * W];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), l16 = lane & 15, q4 = lane >> 4;
  int b = 0;
  while (b + 1 < tab.batch && (int)blockIdx.x >= tab.units[b + 1]) ++b;
  const Held h = held(tab, c, b);
  const int j0 = (((int)blockIdx.x - tab.units[b]) * 4 + wave) * kTile;
  if (h.fresh == 0 || h.base < 0 || j0 >= h.n) return;
  const int n = h.n, new0 = tab.cu_new[b], plane = blockIdx.y;
  const int taken = n_accept ? max(0, min(n_accept[b], h.fresh)) : h.fresh, rows = taken * w.gs;
  const bool more = f.softcap > 0.f || f.slopes;
  const Cap cap(f, 1.f);
  const int32_t* pos = f.slopes ? c.pos + plane * c.slots + h.lo : nullptr;
  int from[4] = {};
  if (pos) {
#pragma unroll
    for (int i = 0; i < 4; ++i) from[i] = pos[min(j0 + 4 * q4 + i, n - 1)];
  }
  float* kt = lds + wave * kTile * W;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const int g0 = c.planes > 1 ? plane : 0, g1 = c.planes > 1 ? plane + 1 : c.G;
  for (int g = g0; g < g1 && rows > 0; ++g) {
    const T* kg = (const T*)c.k + (int64_t)g * c.sh + h.lo * c.ss;
    wave_lds_fence();
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int e = u * 64 + lane, s = min(j0 + e / (DP / 4), n - 1), col = e % (DP / 4) * 4;
      *reinterpret_cast<floatx4*>(kt + e / (DP / 4) * W + col) = load4<T, VEC>(kg + (int64_t)s * c.ss, col, c.d);
    }
    wave_lds_fence();
    for (int row0 = 0; row0 < rows; row0 += 16) {
      const int row = min(row0 + l16, rows - 1), i0 = token_of(w, row), head = g * w.gs + row - i0 * w.gs;
      const int t = path ? max(0, min(path[new0 + i0], h.fresh - 1)) : i0;
      const int64_t r = new0 + t;
      const T* qrow = (const T*)w.q + r * w.qst + (int64_t)head * w.qsh;
      floatx4 qf[DP / 16];
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) qf[s] = load4<T, VEC>(qrow, s * 16 + 4 * q4, c.d);
      const float lse2 = w.lse[r * w.H + head] * 1.4426950408889634f;
      const bool counts = row0 + l16 < rows && lse2 != -INFINITY;   // (one that is not a number counts)
      const uint64_t mask = row_mask(f, r, t);
      const float slope = f.slopes ? f.slopes[head] : 0.f;
      const int at = pos ? pos[h.base + t] : 0;
      const floatx4 acc = tile_scores<DP>(kt, qf, l16, q4);
      float y[4] = {acc[0], acc[1], acc[2], acc[3]};
      if (more) scaled(f, cap, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = more ? biased(y[i], slope, at - from[i]) : y[i] * f.c2;
        if (counts && sees(mask, min(j0 + 4 * q4 + i, n - 1), h.base)) sum[i] += __builtin_amdgcn_exp2f(x - lse2);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    for (int m = 1; m < 16; m <<= 1) sum[i] += __shfl_xor(sum[i], m);
    const int s = j0 + 4 * q4 + i;
    float* mass = c.mass + plane * c.slots + h.lo + s;
    if (l16 == 0 && s < n) *mass = fmaf(w.lambda, *mass, sum[i]);
  }
}

// 64, 128 or 256: what the kernels pad the head dimension to
template <class F>
void with_dim(int d, F f) {
  if (d <= 64) f(std::integral_constant<int, 64>{});
  else if (d <= 128) f(std::integral_constant<int, 128>{});
  else f(std::integral_constant<int, 256>{});
}
// whether rows are read four elements at a time
bool rows_of_four(const CacheView& c, const AttendWork& w, int esz) {
  const int64_t all = c.sh | c.ss | w.qst | w.qsh | c.d;
  return all % 4 == 0 && (((uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)w.q) & (uintptr_t)(4 * esz - 1)) == 0;
}
template <class T, class F>
hipError_t dispatch(const CacheTable& t, const CacheView& c, const AttendWork& w, F f) {
  with_cache_table(t, [&](const auto& tab) {
    with_dim(c.d, [&](auto dp) {
      if (rows_of_four(c, w, sizeof(T))) f(tab, dp, std::true_type{});
      else f(tab, dp, std::false_type{});
    });
  });
  return hipGetLastError();
}
template <class T>
hipError_t attend(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p, const AttendWork& w, hipStream_t st) {
  return dispatch<T>(t, c, w, [&](const auto& tab, auto dp, auto vec) {
    using TAB = std::decay_t<decltype(tab)>;
    constexpr int DP = decltype(dp)::value;
    constexpr bool VEC = decltype(vec)::value;
    const dim3 grid((unsigned)(p.units * c.G));
    if (VEC && p.stream) cache_attend_f32_kernel<TAB, T, DP, VEC, VEC><<<grid, 64 * kAttendWaves, 0, st>>>(tab, c, f, w);
    else cache_attend_f32_kernel<TAB, T, DP, VEC, false><<<grid, 64 * kAttendWaves, 0, st>>>(tab, c, f, w);
  });
}
template <class T>
hipError_t weights(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendWork& w, const int32_t* path,
                   const int32_t* n_accept, hipStream_t st) {
  CacheTable u = t;
  u.units[0] = 0;
  for (int b = 0; b < t.batch; ++b) u.units[b + 1] = u.units[b] + (int32_t)ceil_div(t.cu[b + 1] - t.cu[b], 4 * kTile);
  if (u.units[t.batch] == 0) return hipSuccess;
  return dispatch<T>(u, c, w, [&](const auto& tab, auto dp, auto vec) {
    cache_weights_f32_kernel<std::decay_t<decltype(tab)>, T, decltype(dp)::value, decltype(vec)::value>
        <<<dim3((unsigned)u.units[t.batch], (unsigned)c.planes), 256, 0, st>>>(tab, c, f, w, path, n_accept);
  });
}

}  // namespace

hipError_t launch_cache_attend_f32(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p,
                                   const AttendWork& w, bool bf16, hipStream_t st) {
  return bf16 ? attend<uint16_t>(t, c, f, p, w, st) : attend<float>(t, c, f, p, w, st);
}
hipError_t launch_cache_weights_f32(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendWork& w,
                                    const int32_t* path, const int32_t* n_accept, bool bf16, hipStream_t st) {
  return bf16 ? weights<uint16_t>(t, c, f, w, path, n_accept, st) : weights<float>(t, c, f, w, path, n_accept, st);
}

}  // namespace skv
