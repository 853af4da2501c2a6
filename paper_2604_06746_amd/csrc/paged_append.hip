// Rows of keys and values into the pages of sequences, in 8 bits: rotated on the way, each page and KV head by a scale of its own.
//
// s(A) = the least power of two with A <= 448 s, code = value / s to the nearest.  A power of two costs an 8-bit float nothing, and when a
// page's scale grows, its earlier codes move by exponents: only those that become subnormal lose bits.
// A workgroup takes what comes into one page for one KV head's keys or values: the largest magnitude first, then the codes, so no two
// workgroups share a scale.  Queries that come with the rows are other workgroups of the same launch.
#include "paged.h"

#include <algorithm>

namespace skv {
namespace {

__device__ __forceinline__ bool storable(float x) { return fabsf(x) <= kTopCode * kMostScale; }   // (not NaN either)
// the least power of two s, of kLeastScale at least, with a <= 448 s: 448 is 1.75 2^8
__device__ __forceinline__ float scale_for(float a) {
  const uint32_t up = __float_as_uint(a) + 0x1FFFFFu;   // the exponent carries where the mantissa is beyond 1.75
  return fmaxf(__uint_as_float((up & 0x7F800000u) > (8u << 23) ? (up & 0x7F800000u) - (8u << 23) : 0u), kLeastScale);
}
__device__ __forceinline__ float inverse(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }   // of a power of two
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t* row, int u, const RotaryView& r, const Unit& x) {
  uint32_t a, b;
  if (unit_split(r, u) || !VEC) {
    a = four_codes(x.a[0], x.a[1], x.a[2], x.a[3]);
    b = four_codes(x.b[0], x.b[1], x.b[2], x.b[3]);
  } else {
    a = four_codes(x.a[0], x.b[0], x.a[1], x.b[1]);
    b = four_codes(x.a[2], x.b[2], x.a[3], x.b[3]);
  }
  if (VEC) {
    const bool split = unit_split(r, u);
    *reinterpret_cast<uint32_t*>(row + (split ? 4 * u : 8 * u)) = a;
    *reinterpret_cast<uint32_t*>(row + (split ? 4 * u + r.half : 8 * u + 4)) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = 4 * u + i;
      const bool apart = !r.interleaved && p < r.half;
      row[apart ? p : 2 * p] = (uint8_t)(a >> (8 * i));
      row[apart ? p + r.half : 2 * p + 1] = (uint8_t)(b >> (8 * i));
    }
  }
}

template <class TAB, class T, bool VEC>
__global__ __launch_bounds__(256) void paged_append_kernel(TAB tab, PagedView c, PagedRows w, int q_blocks, int touched) {
  const int upr = c.d / kUnit;
  if ((int)blockIdx.x < q_blocks) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = e / upr;
    const int u = (int)(e - row * upr), r = (int)(row / w.H), h = (int)(row - (int64_t)r * w.H);
    if (r >= tab.cu_new[tab.batch]) return;
    int b = 0;
    while (b + 1 < tab.batch && r >= tab.cu_new[b + 1]) ++b;
    const int pos = w.pos ? w.pos[r] : paged_len(c, b) + r - tab.cu_new[b];
    Unit x = load_unit<T, VEC>((const T*)w.q + r * w.qst + h * w.qsh, u, w.rotary);
    turn(x, spin_unit(w.rotary, u, pos), u, w.rotary);
    store_unit<T, VEC>((T*)w.q_out + row * c.d, u, w.rotary, x);
    return;
  }
  __shared__ float tops[4];
  int i = (int)blockIdx.x - q_blocks;
  const int which = i % (2 * c.G);
  i /= 2 * c.G;
  const int k = i % touched, b = i / touched, g = which >> 1;
  const bool values = which & 1;
  const int fresh = tab.cu_new[b + 1] - tab.cu_new[b], n = paged_len(c, b), lane = threadIdx.x & 63;
  const int first = n >> c.shift, last = (int)(((int64_t)n + fresh - 1) >> c.shift);
  // whether the rows fit, and all their pages are there: every workgroup of the sequence sees the same
  bool fits = (int64_t)n + fresh <= (int64_t)c.max_pages << c.shift;
  if (fits && fresh > 0)
    for (int j = first + lane; j <= last; j += 64) fits &= (uint32_t)c.pages[b * c.pst + j] < (uint32_t)c.n_pages;
  fits = __all(fits);
  if (k == 0 && which == 0 && threadIdx.x == 0) {
    w.lens_out[b] = fits ? n + fresh : n;
    if (!fits && c.missed) c.missed[b] = 1;
  }
  const int j = first + k;
  if (!fits || fresh == 0 || j > last) return;
  const int page0 = j << c.shift, ps = 1 << c.shift;
  const int old = max(0, n - page0), r0 = page0 + old - n, rows = min(page0 + ps, n + fresh) - max(page0, n);   // fresh rows r0 .. r0 + rows - 1
  const int64_t page = c.pages[b * c.pst + j];
  RotaryView r = w.rotary;
  if (values) { r.half = 0; r.interleaved = 1; }
  const T* src = (const T*)(values ? w.v : w.k) + g * w.sh + (int64_t)(tab.cu_new[b] + r0) * w.st;
  uint8_t* dst = (values ? c.v : c.k) + page * c.sp + g * c.sh;
  float* scale = (values ? c.v_scale : c.k_scale) + page * c.G + g;
  auto get = [&](int e, int& row, int& u) __attribute__((always_inline)) {
    row = e / upr;
    u = e - row * upr;
    Unit x = load_unit<T, VEC>(src + row * w.st, u, r);
    if (r.half) turn(x, spin_unit(r, u, w.pos ? w.pos[tab.cu_new[b] + r0 + row] : n + r0 + row), u, r);
    return x;
  };
  float top = 0.f;
  for (int e = threadIdx.x; e < rows * upr; e += 256) {
    int row, u;
    const Unit x = get(e, row, u);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      top = storable(x.a[m]) ? fmaxf(top, fabsf(x.a[m])) : top;
      top = storable(x.b[m]) ? fmaxf(top, fabsf(x.b[m])) : top;
    }
  }
  for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
  if (lane == 0) tops[threadIdx.x >> 6] = top;
  const float before = old > 0 ? *scale : 0.f;
  __syncthreads();
  const float come = scale_for(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
  const float now = fmaxf(come, before), inv = inverse(now);
  if (threadIdx.x == 0) *scale = now;
  if (old > 0 && now > before) {   // the earlier rows' codes in the new scale
    const float ratio = before * inv;
    for (int e = threadIdx.x; e < old * (c.d / 4); e += 256) {
      const int row = e / (c.d / 4);
      uint32_t* at = reinterpret_cast<uint32_t*>(dst + row * c.st + (e - row * (c.d / 4)) * 4);
      typedef __attribute__((ext_vector_type(2))) float floatx2;
      const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(*at, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(*at, true);
      *at = four_codes(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
    }
  }
  for (int e = threadIdx.x; e < rows * upr; e += 256) {
    int row, u;
    Unit x = get(e, row, u);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      x.a[m] = storable(x.a[m]) ? x.a[m] * inv : NAN;
      x.b[m] = storable(x.b[m]) ? x.b[m] * inv : NAN;
    }
    store_codes<VEC>(dst + (old + row) * c.st, u, r, x);
  }
}

}  // namespace

hipError_t launch_paged_append(const CacheTable& t, const PagedView& c, const PagedRows& w, bool bf16, hipStream_t st) {
  const int e = bf16 ? 2 : 4, upr = c.d / kUnit;
  const uintptr_t bits = (uintptr_t)w.k | (uintptr_t)w.v | (uintptr_t)((w.sh | w.st) * e) |
                         (w.q ? (uintptr_t)w.q | (uintptr_t)w.q_out | (uintptr_t)((w.qst | w.qsh) * e) : 0);
  const bool vec = bits % 16 == 0 && whole_units(w.rotary);
  int64_t most = 0;
  for (int b = 0; b < t.batch; ++b) most = std::max<int64_t>(most, t.cu_new[b + 1] - t.cu_new[b]);
  const int64_t ps = (int64_t)1 << c.shift, touched = std::max<int64_t>(1, most > 0 ? (most + ps - 2) / ps + 1 : 1);
  const int64_t q_blocks = w.q ? ceil_div((int64_t)t.cu_new[t.batch] * w.H * upr, 256) : 0;
  const int64_t blocks = q_blocks + (int64_t)t.batch * touched * 2 * c.G;
  with_fresh_table(t, [&](const auto& tab) {
    using TAB = std::decay_t<decltype(tab)>;
    auto go = [&](auto elem, auto v) {
      paged_append_kernel<TAB, decltype(elem), decltype(v)::value><<<(unsigned)blocks, 256, 0, st>>>(tab, c, w, (int)q_blocks, (int)touched);
    };
    if (bf16) vec ? go(uint16_t{}, std::true_type{}) : go(uint16_t{}, std::false_type{});
    else vec ? go(float{}, std::true_type{}) : go(float{}, std::false_type{});
  });
  return hipGetLastError();
}

}  // namespace skv
