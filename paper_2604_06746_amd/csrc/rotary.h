// Rotary positions: the pairs of a row's components and their angles (rotate.hip, paged_append.hip).
#pragma once
#include "common.h"

#include <type_traits>

namespace skv {

struct RotaryView {
  const uint64_t* turns;
  int half;          // pairs; 0: nothing is turned
  int interleaved;
  float mag;
  float sign;        // -1: turned back
  int d;             // components of a row
};

// Rows are taken in units of eight components, four pairs each: pair p is (2p, 2p + 1), but (p, p + half) below `half` where halves are
// turned.  So from 2 half on both layouts copy the same way.
// VEC: bases and strides of whole 16 bytes and whole_units, so that a unit is one piece, or two of half the size.
constexpr int kUnit = 8;

hipError_t launch_rotate(const RotaryView& r, const void* x, int64_t xst, int64_t xsh, int64_t tokens, int heads, int d, bool bf16,
                         const int32_t* pos, void* out, int64_t ost, int64_t osh, hipStream_t st);
inline bool whole_units(const RotaryView& r) { return r.d % kUnit == 0 && (r.interleaved || r.half % 4 == 0); }

#ifdef __HIPCC__
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <class T> __device__ __forceinline__ T to_elem(float x);
template <> __device__ __forceinline__ float to_elem<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t to_elem<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

struct Unit {
  float a[4], b[4];
};
__device__ __forceinline__ bool unit_split(const RotaryView& r, int u) { return !r.interleaved && 4 * u < r.half; }

template <class T, bool VEC>
__device__ __forceinline__ Unit load_unit(const T* row, int u, const RotaryView& r) {
  Unit x;
  if (VEC) {
    typedef __attribute__((ext_vector_type(4))) T four;
    const bool split = unit_split(r, u);
    const four lo = *reinterpret_cast<const four*>(row + (split ? 4 * u : 8 * u));
    const four hi = *reinterpret_cast<const four*>(row + (split ? 4 * u + r.half : 8 * u + 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x.a[i] = as_float(split ? lo[i] : i < 2 ? lo[2 * i] : hi[2 * i - 4]);
      x.b[i] = as_float(split ? hi[i] : i < 2 ? lo[2 * i + 1] : hi[2 * i - 3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = 4 * u + i;
      const bool apart = !r.interleaved && p < r.half;
      const int first = apart ? p : 2 * p, second = apart ? p + r.half : 2 * p + 1;
      x.a[i] = first < r.d ? as_float(row[first]) : 0.f;
      x.b[i] = second < r.d ? as_float(row[second]) : 0.f;
    }
  }
  return x;
}
template <class T, bool VEC>
__device__ __forceinline__ void store_unit(T* row, int u, const RotaryView& r, const Unit& x) {
  if (VEC) {
    typedef __attribute__((ext_vector_type(4))) T four;
    const bool split = unit_split(r, u);
    four lo, hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = to_elem<T>(split ? x.a[i] : i & 1 ? x.b[i / 2] : x.a[i / 2]);
      hi[i] = to_elem<T>(split ? x.b[i] : i & 1 ? x.b[2 + i / 2] : x.a[2 + i / 2]);
    }
    *reinterpret_cast<four*>(row + (split ? 4 * u : 8 * u)) = lo;
    *reinterpret_cast<four*>(row + (split ? 4 * u + r.half : 8 * u + 4)) = hi;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = 4 * u + i;
      const bool apart = !r.interleaved && p < r.half;
      const int first = apart ? p : 2 * p, second = apart ? p + r.half : 2 * p + 1;
      if (first < r.d) row[first] = to_elem<T>(x.a[i]);
      if (second < r.d) row[second] = to_elem<T>(x.b[i]);
    }
  }
}

// Cosine and sine of a unit's four pairs at a position.  turns pos modulo 2^64 is the angle in 2^-64 turns; of its upper 32 bits the
// nearest quarter turn is taken off, and the rest, at most pi / 4 and off by 2^-32 of a turn, goes into the series of sine and cosine (whose
// first terms left out, x^11 / 11! and x^12 / 12!, are below 2e-9), so both are good to fp32's last bits at any position.
struct Spin {
  float c[4], s[4];
};
__device__ __forceinline__ void spin_one(uint64_t turns, int pos, float& c, float& s) {
  const uint32_t top = (uint32_t)((turns * (uint64_t)(int64_t)pos) >> 32);
  const uint32_t quarter = (top + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(top - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
  const float z = x * x;
  const float sn = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float u = quarter & 1 ? sn : cs, v = quarter & 1 ? cs : sn;
  c = (quarter + 1) & 2 ? -u : u;
  s = quarter & 2 ? -v : v;
}
__device__ __forceinline__ Spin spin_unit(const RotaryView& r, int u, int pos) {
  Spin w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = 4 * u + i;
    w.c[i] = 1.f;
    w.s[i] = 0.f;
    if (p < r.half) {
      spin_one(r.turns[p], pos, w.c[i], w.s[i]);
      w.c[i] *= r.mag;
      w.s[i] *= r.mag * r.sign;
    }
  }
  return w;
}
// (pairs from `half` on keep their bits)
__device__ __forceinline__ void turn(Unit& x, const Spin& w, int u, const RotaryView& r) {
  if (4 * u >= r.half) return;
  const int last = r.half - 4 * u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x.a[i], b = x.b[i];
    x.a[i] = i < last ? fmaf(a, w.c[i], -b * w.s[i]) : a;
    x.b[i] = i < last ? fmaf(b, w.c[i], a * w.s[i]) : b;
  }
}
#endif

}  // namespace skv
