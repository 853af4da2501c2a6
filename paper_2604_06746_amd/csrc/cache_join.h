// What joins the chunks of an attend call's rows: cache_combine.hip (caches of slots), paged_join.hip (in pages).
// Chunk i of a row left (M_i, Z_i, O_i); with M = max M_i: Z = sum 2^(M_i - M) Z_i, out = sum 2^(M_i - M) O_i / Z, lse = ln 2 (M + log2 Z).
#pragma once
#include "cache.h"

#ifdef __HIPCC__
namespace skv {

typedef float __attribute__((ext_vector_type(2))) joined_t;   // (M, Z)

// over the 64 lanes, by moves inside the rows of 16 and then between them (six vector instructions; by shuffles six trips through the LDS
// crossbar, which made a plane of 32 heads' norms take 5 us)
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float x, float without) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(without), __float_as_int(x), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float last_lane(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)); }
__device__ __forceinline__ float wave_top(float x) {
  x = fmaxf(x, moved<0x111, 0xF>(x, -INFINITY));
  x = fmaxf(x, moved<0x112, 0xF>(x, -INFINITY));
  x = fmaxf(x, moved<0x114, 0xF>(x, -INFINITY));
  x = fmaxf(x, moved<0x118, 0xF>(x, -INFINITY));
  x = fmaxf(x, moved<0x142, 0xA>(x, -INFINITY));
  x = fmaxf(x, moved<0x143, 0xC>(x, -INFINITY));
  return last_lane(x);
}
__device__ __forceinline__ float wave_total(float x) {
  x += moved<0x111, 0xF>(x, 0.f);
  x += moved<0x112, 0xF>(x, 0.f);
  x += moved<0x114, 0xF>(x, 0.f);
  x += moved<0x118, 0xF>(x, 0.f);
  x += moved<0x142, 0xA>(x, 0.f);
  x += moved<0x143, 0xC>(x, 0.f);
  return last_lane(x);
}

constexpr int kAhead = 8;   // loads of a thread that are on their way at once

template <class T>
__device__ __forceinline__ void put_row(const AttendWork& w, int64_t at, int d, int col, floatx4 o, float top, float z) {
  const float inv = z != 0.f ? 1.f / z : 0.f;   // (NaN stays NaN)
  for (int e = 0; e < 4 && col + e < d; ++e) put_out<T>((T*)w.out + at * d + col + e, o[e] * inv);
  if (col == 0) w.lse[at] = z != 0.f ? (top + __builtin_amdgcn_logf(z)) * 0.6931471806f : -INFINITY;
}

// Some of a row's chunks, a lane group's four components of them.
struct Chunks {
  joined_t stat[kAhead];
  floatx4 sums[kAhead];
  __device__ __forceinline__ void load(const joined_t* ml, const float* po, int64_t step, int dp, int live, bool in, int i0, int stride) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k * stride;
      stat[k] = i < live ? ml[i * step] : joined_t{kNothingSeen, 0.f};
      sums[k] = in && i < live ? *reinterpret_cast<const floatx4*>(po + i * step * dp) : floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void add(float top, float& z, floatx4& o) const {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const float s = __builtin_amdgcn_exp2f(stat[k][0] - top);
      z = fmaf(s, stat[k][1], z);
      o += sums[k] * s;
    }
  }
};

// Row `at` by a workgroup of 256: lane groups of DP / 4 on shares of its chunks.  ml, po: the first chunk's, the next one's `step` further (po: the
// thread's components).  sh: 1024 words, zs: 4.
template <class T, int DP>
__device__ __forceinline__ void join_row(const AttendWork& w, int d, int64_t at, const joined_t* ml, const float* po, int64_t step, int live, float* sh, float* zs) {
  constexpr int LANES = DP / 4, PARTS = 256 / LANES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = threadIdx.x / LANES, col = threadIdx.x % LANES * 4;
  const bool in = col < d;
  Chunks c;
  c.load(ml, po, step, DP, live, in, part, PARTS);
  float top = kNothingSeen, z = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i = lane; i < live; i += 64) top = fmaxf(top, ml[i * step][0]);
  top = wave_top(top);
  c.add(top, z, o);
  for (int i = part + kAhead * PARTS; i < live; i += PARTS) {
    const joined_t m = ml[i * step];
    const float s = __builtin_amdgcn_exp2f(m[0] - top);
    z = fmaf(s, m[1], z);
    if (in) o += *reinterpret_cast<const floatx4*>(po + i * step * DP) * s;
  }
  // the shares: lanes of a wave that have the same components, then the waves
  for (int m = LANES; m < 64; m <<= 1) {
    z += __shfl_xor(z, m);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m);
  }
  if (lane < LANES) *reinterpret_cast<floatx4*>(sh + (wave * LANES + lane) * 4) = o;
  if (lane == 0) zs[wave] = z;
  __syncthreads();
  if ((int)threadIdx.x < LANES && in) {
    z = (zs[0] + zs[1]) + (zs[2] + zs[3]);
    o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) o += *reinterpret_cast<const floatx4*>(sh + (i * LANES + threadIdx.x) * 4);
    put_row<T>(w, at, d, col, o, top, z);
  }
}

// (M, Z) of a row's chunks from the lane's on, joined: a lane a chunk, for wave_top and wave_total of these.
__device__ __forceinline__ joined_t joined_stat(const joined_t* ml, int64_t step, int live, bool there) {
  const int lane = threadIdx.x & 63;
  joined_t a = there && lane < live ? ml[lane * step] : joined_t{kNothingSeen, 0.f};
  for (int k = lane + 64; there && k < live; k += 64) {
    const joined_t m = ml[k * step];
    const float top = fmaxf(a[0], m[0]);
    a = joined_t{top, a[1] * __builtin_amdgcn_exp2f(a[0] - top) + m[1] * __builtin_amdgcn_exp2f(m[0] - top)};
  }
  return a;
}

}  // namespace skv
#endif
