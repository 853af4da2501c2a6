// Rows of a cache in use: new ones into the free slots, and the accepted drafts' rows to the front of the fresh ones.
// Copies: bound by memory, or for the few rows of a decoding step by one launch and its chain of loads (length, row, store).
#include "cache.h"

#include <algorithm>

namespace skv {
namespace {

// One thread per unit (16, 4 or 2 bytes) of a row, as in the row gather.  blockIdx.y: sequence, so that its offsets are scalars (picked from the
// table by each thread they cost a token of 64 sequences 2 us); its rows of all KV heads and both tensors lie one behind the other, so
// that a single token still fills workgroups.  The first unit of a key's row, of a plane's first head, also brings position and mass.
template <class TAB, class V, bool POW2>
__global__ __launch_bounds__(256) void cache_append_kernel(TAB tab, CacheView c, const uint8_t* __restrict__ k_new,
                                                           const uint8_t* __restrict__ v_new, int64_t nsh, int64_t nst, int elem_bytes,
                                                           uint32_t units_per_row, uint32_t upr_shift, const int32_t* __restrict__ pos_new,
                                                           const float* __restrict__ mass_new, int64_t nsp, int32_t* __restrict__ lens_out) {
  short_kernel_priority();
  const int b = blockIdx.y;
  const uint32_t fresh = (uint32_t)(tab.cu_new[b + 1] - tab.cu_new[b]);
  const int64_t lo = tab.cu[b], cap = tab.cu[b + 1] - lo, first = tab.cu_new[b];
  const uint32_t per = fresh * units_per_row, e = blockIdx.x * 256 + threadIdx.x;
  uint32_t plane = 0, t = 0, u = 0;   // (tensor, head) pair, token, unit
  bool mine = false;
  V x;
  if (fresh > 0) {
    plane = e / per;
    const uint32_t rest = e - plane * per;
    t = POW2 ? rest >> upr_shift : rest / units_per_row;
    u = rest - t * units_per_row;
    mine = plane < 2u * (uint32_t)c.G;
  }
  const bool second = plane >= (uint32_t)c.G;
  const int64_t g = second ? plane - c.G : plane;
  if (mine) x = load_once<V>((second ? v_new : k_new) + (g * nsh + (first + t) * nst) * elem_bytes + (int64_t)u * sizeof(V));
  const int n = max(0, (int)min((int64_t)c.lens[b], cap));   // (the row is on its way while the length is)
  const bool fits = n + (int64_t)fresh <= cap;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    lens_out[b] = fits ? n + (int)fresh : n;
    if (!fits && c.missed) c.missed[b] = 1;
  }
  if (!mine || !fits) return;
  const int64_t slot = lo + n + t;
  *reinterpret_cast<V*>((uint8_t*)(second ? c.v : c.k) + (g * c.sh + slot * c.ss) * elem_bytes + (int64_t)u * sizeof(V)) = x;
  if (u == 0 && plane < (uint32_t)c.planes) {
    if (pos_new) c.pos[plane * c.slots + slot] = pos_new[plane * nsp + first + t];
    if (c.mass) c.mass[plane * c.slots + slot] = mass_new ? mass_new[plane * nsp + first + t] : 0.f;
  }
}

// The accepted rows of one KV head and tensor (blockIdx.y, .z), or a plane's positions and masses (the last blockIdx.z), of sequence
// blockIdx.x: all of a block of columns is in registers before any of it is written, so paths may come in any order.
constexpr int kColumns = 64, kHold = STRUCTKV_MAX_DRAFTS * kColumns / 256;
template <class TAB, class V>
__global__ __launch_bounds__(256) void cache_accept_kernel(TAB tab, CacheView c, const int32_t* __restrict__ path,
                                                           const int32_t* __restrict__ n_accept, int elem_bytes, int units_per_row,
                                                           int32_t* __restrict__ lens_out) {
  short_kernel_priority();
  __shared__ int from[STRUCTKV_MAX_DRAFTS];
  const int b = blockIdx.x;
  const Held h = held(tab, c, b);
  const bool whole = h.base >= 0;
  const int taken = !whole ? 0 : n_accept ? max(0, min(n_accept[b], h.fresh)) : h.fresh;
  if (blockIdx.y == 0 && blockIdx.z == 2 && threadIdx.x == 0) lens_out[b] = whole ? h.base + taken : h.n;
  if (taken == 0 || !path) return;
  if ((int)threadIdx.x < taken) from[threadIdx.x] = max(0, min(path[tab.cu_new[b] + threadIdx.x], h.fresh - 1));
  __syncthreads();
  const int64_t g = blockIdx.y, first = h.lo + h.base;
  if (blockIdx.z == 2) {
    if (g >= c.planes) return;
    const int i = threadIdx.x;
    int32_t pos = 0;
    float mass = 0.f;
    const int64_t p = g * c.slots + first;
    if (i < taken) {
      if (c.pos) pos = c.pos[p + from[i]];
      if (c.mass) mass = c.mass[p + from[i]];
    }
    __syncthreads();
    if (i < taken) {
      if (c.pos) c.pos[p + i] = pos;
      if (c.mass) c.mass[p + i] = mass;
    }
    return;
  }
  uint8_t* rows = (uint8_t*)(blockIdx.z ? c.v : c.k) + (g * c.sh + first * c.ss) * elem_bytes;
  const int64_t step = c.ss * elem_bytes;
  for (int c0 = 0; c0 < units_per_row; c0 += kColumns) {
    const int cols = min(kColumns, units_per_row - c0), units = taken * cols;
    V x[kHold];
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int e = i * 256 + threadIdx.x, row = e / cols;
      if (e < units) x[i] = *reinterpret_cast<const V*>(rows + from[row] * step + (c0 + e - row * cols) * (int)sizeof(V));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int e = i * 256 + threadIdx.x, row = e / cols;
      if (e < units && from[row] != row) *reinterpret_cast<V*>(rows + row * step + (c0 + e - row * cols) * (int)sizeof(V)) = x[i];
    }
  }
}

// the widest unit that pointers, strides and rows allow
template <class F>
void with_unit(uintptr_t bits, F f) {
  if (bits % 16 == 0) f(uint4{});
  else if (bits % 4 == 0) f(uint32_t{});
  else f(uint16_t{});
}

}  // namespace

hipError_t launch_cache_append(const CacheTable& t, const CacheView& c, const void* k_new, const void* v_new, int64_t nsh,
                               int64_t nst, const int32_t* pos_new, const float* mass_new, int64_t nsp, int elem_bytes,
                               int32_t* lens_out, hipStream_t st) {
  int64_t most = 0;
  for (int b = 0; b < t.batch; ++b) most = std::max<int64_t>(most, t.cu_new[b + 1] - t.cu_new[b]);
  const uintptr_t bits = (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)c.k | (uintptr_t)c.v |
                         (uintptr_t)((nsh | nst | c.sh | c.ss | c.d) * elem_bytes);
  with_row_table(t, [&](const auto& tab) {
    with_unit(bits, [&](auto unit) {
      using V = decltype(unit);
      using TAB = std::decay_t<decltype(tab)>;
      const uint32_t upr = (uint32_t)(c.d * elem_bytes / (int)sizeof(V)), shift = (uint32_t)__builtin_ctz(upr);
      const dim3 grid((unsigned)std::max<int64_t>(1, ceil_div(most * 2 * c.G * upr, 256)), (unsigned)t.batch);
      const uint8_t *k8 = (const uint8_t*)k_new, *v8 = (const uint8_t*)v_new;
      if ((upr & (upr - 1)) == 0)
        cache_append_kernel<TAB, V, true><<<grid, 256, 0, st>>>(tab, c, k8, v8, nsh, nst, elem_bytes, upr, shift, pos_new, mass_new, nsp, lens_out);
      else
        cache_append_kernel<TAB, V, false><<<grid, 256, 0, st>>>(tab, c, k8, v8, nsh, nst, elem_bytes, upr, shift, pos_new, mass_new, nsp, lens_out);
    });
  });
  return hipGetLastError();
}

hipError_t launch_cache_accept(const CacheTable& t, const CacheView& c, const int32_t* path, const int32_t* n_accept,
                               int elem_bytes, int32_t* lens_out, hipStream_t st) {
  const uintptr_t bits = (uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)((c.sh | c.ss | c.d) * elem_bytes);
  with_row_table(t, [&](const auto& tab) {
    with_unit(bits, [&](auto unit) {
      using V = decltype(unit);
      cache_accept_kernel<std::decay_t<decltype(tab)>, V><<<dim3((unsigned)t.batch, (unsigned)c.G, 3), 256, 0, st>>>(
          tab, c, path, n_accept, elem_bytes, c.d * elem_bytes / (int)sizeof(V), lens_out);
    });
  });
  return hipGetLastError();
}

}  // namespace skv
