// Rows of keys and values into the pages of sequences, in 8 bits: rotated on the way, each page and KV head by a scale of its own.
//
// s(A) = the least power of two with A <= 448 s, code = value / s to the nearest.  A power of two costs an 8-bit float nothing, and when a
// page's scale grows, its earlier codes move by exponents: only those that become subnormal lose bits.
// A workgroup takes what comes into one page for one KV head's keys or values: the largest magnitude first, then the codes, so no two
// workgroups share a scale.  Queries that come with the rows are other workgroups of the same launch.
// Prompts are bound by memory, three quarters of it the queries': eight of 5715 tokens (1.03 GB) 229 us.  Rows that are read again for the
// codes 391 us; kept in registers, with the queries' angles shared by heads, 257; wide pieces, past the caches 240; checks for values that cannot be
// stored out of the way 235; keys' angles for eight heads 229 (for none of them 253).  A token of each of 64 sequences 4.8 us: a chain of
// length, table and scale, beside which its row is on its way.
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
  if (VEC && unit_split(r, u)) {
    *reinterpret_cast<uint32_t*>(row + 4 * u) = a;
    *reinterpret_cast<uint32_t*>(row + 4 * u + r.half) = b;
  } else if (VEC) {
    *reinterpret_cast<uint64_t*>(row + 8 * u) = (uint64_t)b << 32 | a;
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

// Which workgroup takes what: `pages` of them what comes into the touched pages, the others queries.
struct AppendCut {
  int touched;         // most pages that a sequence's rows go to
  int pages;           // workgroups for them
  uint32_t upr_recip;  // ceil(2^20 / units of a row): divides what a workgroup counts (256 rows at most)
  int heads, groups;   // query heads that a thread takes, and how many such groups there are
  int once;            // 1: queries go past the caches
  int keys;            // KV heads whose keys a workgroup takes one behind the other, for the angles serve all of them
  uint32_t units;      // query units: tokens x groups x units of a row
};

// HOLD: units of a thread, kept in registers from the search for the largest magnitude on.  ONE: a single token at most, which goes to the
// page of slot lens[b], so that its row is on its way before the length is known.
// SHARE: the workgroup (of 256 threads at most) takes several heads' keys, the next one's on their way.
template <class TAB, class T, bool VEC, int HOLD, bool ONE, bool SHARE>
__global__ __launch_bounds__(SHARE ? 256 : 1024) void paged_append_kernel(TAB tab, PagedView c, PagedRows w, AppendCut cut) {
  short_kernel_priority();
  const int upr = c.d / kUnit, lane = threadIdx.x & 63;
  if ((int)blockIdx.x >= cut.pages) {   // queries: the angles of a token's unit serve several heads
    const uint32_t e = (blockIdx.x - (uint32_t)cut.pages) * blockDim.x + threadIdx.x;
    if (e >= cut.units) return;
    const uint32_t rest = e / (uint32_t)upr;
    const int u = (int)(e - rest * upr), r = (int)(rest / (uint32_t)cut.groups), h0 = (int)(rest - (uint32_t)r * cut.groups) * cut.heads;
    const int b = sequence_of(tab, r);
    const int pos = w.pos ? w.pos[r] : paged_len(c, b) + r - tab.cu_new[b];
    const Spin spin = spin_unit(w.rotary, u, pos);
    const T* from = (const T*)w.q + r * w.qst;
    T* to = (T*)w.q_out + (int64_t)r * w.H * c.d;
    if (cut.once) turn_heads<T, VEC, true, 4>(from, w.qsh, to, (int64_t)c.d, h0, min(w.H, h0 + cut.heads), u, w.rotary, spin);
    else turn_heads<T, VEC, false, 4>(from, w.qsh, to, (int64_t)c.d, h0, min(w.H, h0 + cut.heads), u, w.rotary, spin);
    return;
  }
  __shared__ float tops[2][16];
  const int key_groups = (c.G + cut.keys - 1) / cut.keys;
  int i = (int)blockIdx.x;
  const int which = i % (key_groups + c.G);
  i /= key_groups + c.G;
  const int k = ONE ? 0 : i % cut.touched, b = ONE ? i : i / cut.touched;
  const bool values = which >= key_groups;
  const int g0 = values ? which - key_groups : which * cut.keys, g1 = SHARE && !values ? min(c.G, g0 + cut.keys) : g0 + 1;
  const int fresh = tab.cu_new[b + 1] - tab.cu_new[b];
  RotaryView r = w.rotary;
  if (values) { r.half = 0; r.interleaved = 1; }
  const T* src = (const T*)(values ? w.v : w.k) + (int64_t)tab.cu_new[b] * w.st;
  int row[HOLD], unit[HOLD];
#pragma unroll
  for (int m = 0; m < HOLD; ++m) {
    const int e = (int)(threadIdx.x + m * blockDim.x);
    row[m] = (int)(((uint32_t)e * cut.upr_recip) >> 20);
    unit[m] = e - row[m] * upr;
  }
  auto exchanged = [&](float top, float* place) __attribute__((always_inline)) {   // the largest of all threads'
    for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    if (blockDim.x > 64) {
      if (lane == 0) place[threadIdx.x >> 6] = top;
      __syncthreads();
      for (int m = 0; m < (int)blockDim.x >> 6; ++m) top = fmaxf(top, place[m]);
    }
    return top;
  };
  Unit x[HOLD];
  auto load = [&](int g, int r0, int rows) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < HOLD; ++m) {
      x[m] = Unit{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      if (row[m] < rows) x[m] = load_unit<T, VEC>(src + g * w.sh + (int64_t)(r0 + row[m]) * w.st, unit[m], r);
    }
  };
  if (ONE) load(g0, 0, fresh);
  const int n = paged_len(c, b);
  const int first = n >> c.shift, last = (int)(((int64_t)n + fresh - 1) >> c.shift);
  // whether the rows fit, and all their pages are there: every workgroup of the sequence sees the same
  bool fits = (int64_t)n + fresh <= (int64_t)c.max_pages << c.shift;
  int page = -1;
  if (fits && fresh > 0) {
    for (int j = first + lane; j <= last; j += 64) {
      const int id = c.pages[b * c.pst + j];
      fits &= (uint32_t)id < (uint32_t)c.n_pages;
      if (j == first + k) page = id;
    }
  }
  fits = __all(fits);
  page = __builtin_amdgcn_readlane(page, k & 63);
  if (k == 0 && which == 0 && threadIdx.x == 0) {
    w.lens_out[b] = fits ? n + fresh : n;
    if (!fits && c.missed) c.missed[b] = 1;
  }
  const int j = first + k;
  if (!fits || fresh == 0 || j > last) return;
  const int page0 = j << c.shift, ps = 1 << c.shift;
  const int old = max(0, n - page0), r0 = page0 + old - n, rows = min(page0 + ps, n + fresh) - max(page0, n);   // fresh rows r0 .. r0 + rows - 1
  if (!ONE) load(g0, r0, rows);
  auto spin_of = [&](int m) __attribute__((always_inline)) { return spin_unit(r, unit[m], w.pos ? w.pos[tab.cu_new[b] + r0 + row[m]] : n + r0 + row[m]); };
  Spin spin[SHARE ? HOLD : 1];
  if (SHARE && r.half) {
#pragma unroll
    for (int m = 0; m < HOLD; ++m)
      if (row[m] < rows) spin[m] = spin_of(m);
  }
  for (int g = g0; g < g1; ++g) {
    uint8_t* dst = (values ? c.v : c.k) + page * c.sp + g * c.sh;
    float* scale = (values ? c.v_scale : c.k_scale) + (int64_t)page * c.G + g;
    const float before = old > 0 ? *scale : 0.f;
    float top = 0.f;
#pragma unroll
    for (int m = 0; m < HOLD; ++m) {
      if (r.half && row[m] < rows) turn(x[m], SHARE ? spin[SHARE ? m : 0] : spin_of(m), unit[m], r);
#pragma unroll
      for (int q = 0; q < 4; ++q) top = fmaxf(top, fmaxf(fabsf(x[m].a[q]), fabsf(x[m].b[q])));   // (NaN does not count)
    }
    top = exchanged(top, tops[(g - g0) & 1]);   // (two places in turns: a wave is at most one barrier ahead)
    // What cannot be stored is rare: the conversion makes NaN of NaN, and larger values are looked for only where there are some.
    const bool odd = !(top <= kTopCode * kMostScale);
    if (odd) {
      top = 0.f;
#pragma unroll
      for (int m = 0; m < HOLD; ++m)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          x[m].a[q] = storable(x[m].a[q]) ? x[m].a[q] : NAN;
          x[m].b[q] = storable(x[m].b[q]) ? x[m].b[q] : NAN;
          top = fmaxf(top, fmaxf(fabsf(x[m].a[q]), fabsf(x[m].b[q])));
        }
      __syncthreads();
      top = exchanged(top, tops[(g - g0) & 1]);
      __syncthreads();
    }
    const float come = scale_for(top), now = fmaxf(come, before), inv = 1.f / now;   // (exact: powers of two)
    if (old > 0 && now > before) {   // the earlier rows' codes in the new scale
      const float ratio = before * inv;
      for (int e = threadIdx.x; e < old * (c.d / 4); e += blockDim.x) {
        const int at_row = e / (c.d / 4);
        uint32_t* at = reinterpret_cast<uint32_t*>(dst + at_row * c.st + (e - at_row * (c.d / 4)) * 4);
        typedef __attribute__((ext_vector_type(2))) float floatx2;
        const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(*at, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(*at, true);
        *at = four_codes(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
      }
    }
    if (threadIdx.x == 0) *scale = now;   // (every thread has read it: the largest of all has been exchanged)
    Unit coded[SHARE ? HOLD : 1];
    auto code = [&](int m, Unit& to) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        to.a[q] = x[m].a[q] * inv;
        to.b[q] = x[m].b[q] * inv;
      }
    };
    if constexpr (SHARE) {   // (the next head's rows come while these are stored)
#pragma unroll
      for (int m = 0; m < HOLD; ++m) code(m, coded[m]);
      if (g + 1 < g1) load(g + 1, r0, rows);
    }
#pragma unroll
    for (int m = 0; m < HOLD; ++m) {
      if (!SHARE) code(m, coded[0]);
      if (row[m] < rows) store_codes<VEC>(dst + (old + row[m]) * c.st, unit[m], r, coded[SHARE ? m : 0]);
    }
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
  const int ps = 1 << c.shift;
  AppendCut cut;
  cut.touched = (int)(most > 0 ? (most + ps - 2) / ps + 1 : 1);
  // threads: four units each, from a wave to sixteen
  const int units = (int)std::min<int64_t>(std::max<int64_t>(1, most), ps) * upr;
  int threads = 64;
  while (threads < 1024 && threads * 4 < units) threads *= 2;
  // (one head a workgroup where there are few, or units fill its registers)
  cut.keys = 1;
  while (w.rotary.half && most > 1 && threads <= 256 && cut.keys < 8 && 2 * cut.keys <= c.G && (int64_t)t.batch * cut.touched * (c.G / (2 * cut.keys)) >= 512) cut.keys *= 2;
  cut.pages = t.batch * cut.touched * ((int)ceil_div(c.G, cut.keys) + c.G);
  cut.upr_recip = (uint32_t)(((1u << 20) + upr - 1) / upr);
  // query heads of a thread: as many as leave the chip filled
  const int64_t tokens = w.q ? t.cu_new[t.batch] : 0;
  cut.heads = w.q ? (int)std::min<int64_t>(w.H, std::max<int64_t>(1, tokens * upr * w.H / (1 << 18))) : 1;
  cut.groups = w.q ? (int)ceil_div(w.H, cut.heads) : 1;
  cut.once = 2 * tokens * w.H * c.d * e >= kOnceBytes;
  cut.units = (uint32_t)(tokens * cut.groups * upr);
  const int64_t blocks = cut.pages + ceil_div((int64_t)cut.units, threads);
  if (blocks * threads >> 32) {   // a launch takes fewer than 2^32 threads: the sequences one by one, which leaves out what is there for the longest one's pages
    if (t.batch == 1) return hipErrorInvalidConfiguration;
    for (int b = 0; b < t.batch; ++b) {
      const int64_t r = t.cu_new[b];
      CacheTable one = {};
      one.cu_new[1] = t.cu_new[b + 1] - t.cu_new[b];
      one.batch = 1;
      PagedView v = c;
      v.pages += b * c.pst;
      v.lens += b;
      v.missed = c.missed ? c.missed + b : nullptr;
      v.batch = 1;
      PagedRows x = w;
      x.k = (const uint8_t*)w.k + r * w.st * e;
      x.v = (const uint8_t*)w.v + r * w.st * e;
      x.pos = w.pos ? w.pos + r : nullptr;
      x.q = w.q && one.cu_new[1] > 0 ? (const uint8_t*)w.q + r * w.qst * e : nullptr;
      x.q_out = (uint8_t*)w.q_out + r * w.H * c.d * e;
      x.lens_out = w.lens_out + b;
      const hipError_t st1 = launch_paged_append(one, v, x, bf16, st);
      if (st1 != hipSuccess) return st1;
    }
    return hipSuccess;
  }
  with_fresh_table(t, [&](const auto& tab) {
    using TAB = std::decay_t<decltype(tab)>;
    auto go = [&](auto elem, auto v, auto hold, auto one, auto share) {
      paged_append_kernel<TAB, decltype(elem), decltype(v)::value, decltype(hold)::value, decltype(one)::value, decltype(share)::value>
          <<<(unsigned)blocks, threads, 0, st>>>(tab, c, w, cut);
    };
    auto by_size = [&](auto elem, auto v) {
      const std::integral_constant<int, 1> h1; const std::integral_constant<int, 4> h4; const std::integral_constant<int, 8> h8;
      const std::true_type yes; const std::false_type no;
      if (most <= 1) go(elem, v, h1, yes, no);
      else if (cut.keys > 1) go(elem, v, h4, no, yes);
      else if (units <= 4 * threads) go(elem, v, h4, no, no);
      else go(elem, v, h8, no, no);
    };
    if (bf16) vec ? by_size(uint16_t{}, std::true_type{}) : by_size(uint16_t{}, std::false_type{});
    else vec ? by_size(float{}, std::true_type{}) : by_size(float{}, std::false_type{});
  });
  return hipGetLastError();
}

}  // namespace skv
