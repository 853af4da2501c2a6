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

// Rows are taken in units of 2 P components, P pairs each: pair p is (2p, 2p + 1), but (p, p + half) below `half` where halves are turned.  So
// from 2 half on both layouts copy the same way.
// VEC: bases and strides of whole 16 bytes and whole_units, so that a unit is one piece, or two of half the size.
constexpr int kUnit = 8;   // components of a unit of four pairs

// From so many bytes in and out on rows go past the caches, what the memory-side cache keeps from one call to the next: keys of 131072 tokens
// (0.5 GB) 99 -> 92 us, queries of 4096 (67 MB) 13.0 -> 15.2.
constexpr int64_t kOnceBytes = (int64_t)256 << 20;

hipError_t launch_rotate(const RotaryView& r, const void* x, int64_t xst, int64_t xsh, int64_t tokens, int heads, int d, bool bf16,
                         const int32_t* pos, void* out, int64_t ost, int64_t osh, hipStream_t st);
inline bool whole_units(const RotaryView& r, int pairs = 4) { return r.d % (2 * pairs) == 0 && (r.interleaved || r.half % pairs == 0); }

#ifdef __HIPCC__
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <class T> __device__ __forceinline__ T to_elem(float x);
template <> __device__ __forceinline__ float to_elem<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t to_elem<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

template <int P>
struct Pairs {
  float a[P], b[P];
};
using Unit = Pairs<4>;
template <int P = 4>
__device__ __forceinline__ bool unit_split(const RotaryView& r, int u) { return !r.interleaved && P * u < r.half; }

template <class T, bool VEC, bool ONCE = false, int P = 4>
__device__ __forceinline__ Pairs<P> load_unit(const T* row, int u, const RotaryView& r) {
  Pairs<P> x;
  if (VEC) {
    typedef __attribute__((ext_vector_type(P))) T part;
    typedef __attribute__((ext_vector_type(2 * P))) T whole;
    auto get = [](auto* p) __attribute__((always_inline)) { return ONCE ? __builtin_nontemporal_load(p) : *p; };
    if (unit_split<P>(r, u)) {
      const part lo = get(reinterpret_cast<const part*>(row + P * u)), hi = get(reinterpret_cast<const part*>(row + P * u + r.half));
#pragma unroll
      for (int i = 0; i < P; ++i) { x.a[i] = as_float(lo[i]); x.b[i] = as_float(hi[i]); }
    } else {
      const whole v = get(reinterpret_cast<const whole*>(row + 2 * P * u));
#pragma unroll
      for (int i = 0; i < P; ++i) { x.a[i] = as_float(v[2 * i]); x.b[i] = as_float(v[2 * i + 1]); }
    }
  } else {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = P * u + i;
      const bool apart = !r.interleaved && p < r.half;
      const int first = apart ? p : 2 * p, second = apart ? p + r.half : 2 * p + 1;
      x.a[i] = first < r.d ? as_float(row[first]) : 0.f;
      x.b[i] = second < r.d ? as_float(row[second]) : 0.f;
    }
  }
  return x;
}
template <class T, bool VEC, bool ONCE = false, int P = 4>
__device__ __forceinline__ void store_unit(T* row, int u, const RotaryView& r, const Pairs<P>& x) {
  if (VEC) {
    typedef __attribute__((ext_vector_type(P))) T part;
    typedef __attribute__((ext_vector_type(2 * P))) T whole;
    auto put = [](auto* p, auto v) __attribute__((always_inline)) { if (ONCE) __builtin_nontemporal_store(v, p); else *p = v; };
    if (unit_split<P>(r, u)) {
      part lo, hi;
#pragma unroll
      for (int i = 0; i < P; ++i) { lo[i] = to_elem<T>(x.a[i]); hi[i] = to_elem<T>(x.b[i]); }
      put(reinterpret_cast<part*>(row + P * u), lo);
      put(reinterpret_cast<part*>(row + P * u + r.half), hi);
    } else {
      whole v;
#pragma unroll
      for (int i = 0; i < P; ++i) { v[2 * i] = to_elem<T>(x.a[i]); v[2 * i + 1] = to_elem<T>(x.b[i]); }
      put(reinterpret_cast<whole*>(row + 2 * P * u), v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = P * u + i;
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
template <int P>
struct Spins {
  float c[P], s[P];
};
using Spin = Spins<4>;
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
template <int P = 4>
__device__ __forceinline__ Spins<P> spin_unit(const RotaryView& r, int u, int pos) {
  Spins<P> w;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int p = P * u + i;
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
template <int P>
__device__ __forceinline__ void turn(Pairs<P>& x, const Spins<P>& w, int u, const RotaryView& r) {
  if (P * u >= r.half) return;
  const int last = r.half - P * u;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const float a = x.a[i], b = x.b[i];
    x.a[i] = i < last ? fmaf(a, w.c[i], -b * w.s[i]) : a;
    x.b[i] = i < last ? fmaf(b, w.c[i], a * w.s[i]) : b;
  }
}
// One unit of a token's heads h0 .. h1 - 1, AT of them on their way at a time.
template <class T, bool VEC, bool ONCE, int AT, int P>
__device__ __forceinline__ void turn_heads(const T* from, int64_t fsh, T* to, int64_t tsh, int h0, int h1, int u, const RotaryView& r, const Spins<P>& w) {
  int h = h0;
  for (; h + AT <= h1; h += AT) {
    Pairs<P> x[AT];
#pragma unroll
    for (int i = 0; i < AT; ++i) x[i] = load_unit<T, VEC, ONCE, P>(from + (h + i) * fsh, u, r);
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      turn(x[i], w, u, r);
      store_unit<T, VEC, ONCE, P>(to + (h + i) * tsh, u, r, x[i]);
    }
  }
  for (; h < h1; ++h) {
    Pairs<P> x = load_unit<T, VEC, ONCE, P>(from + h * fsh, u, r);
    turn(x, w, u, r);
    store_unit<T, VEC, ONCE, P>(to + h * tsh, u, r, x);
  }
}
#endif

}  // namespace skv
