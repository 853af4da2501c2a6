// Rows of a cache in use: new ones into the free slots, and the accepted drafts' rows to the front of the fresh ones.
// Copies: bound by memory, or for the few rows of a decoding step by one launch and its chain of loads (length, row, store).
#include "cache.h"

namespace skv {
namespace {

// One thread per unit (16, 4 or 2 bytes) of a row, as in the row gather; the threads of a block of their own at the end take positions,
// masses and lengths.  blockIdx.y: KV head, blockIdx.z: tensor.
template <class TAB, class V>
__global__ __launch_bounds__(256) void cache_append_kernel(TAB tab, CacheView c, const uint8_t* __restrict__ k_new,
                                                           const uint8_t* __restrict__ v_new, int64_t nsh, int64_t nst, int elem_bytes,
                                                           uint32_t units_per_row, const int32_t* __restrict__ pos_new,
                                                           const float* __restrict__ mass_new, int64_t nsp, unsigned row_blocks,
                                                           int32_t* __restrict__ lens_out) {
  short_kernel_priority();
  const int64_t total = tab.cu_new[tab.batch];
  if (blockIdx.x < row_blocks) {
    const uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r = (int64_t)(e / units_per_row);
    if (r >= total) return;
    const uint32_t u = (uint32_t)(e - (uint64_t)r * units_per_row);
    int b = 0;
    for (int i = 1; i < tab.batch; ++i) b += r >= tab.cu_new[i];
    const int64_t g = blockIdx.y;
    const uint8_t* src = (blockIdx.z ? v_new : k_new) + (g * nsh + r * nst) * elem_bytes + (int64_t)u * sizeof(V);
    const V x = load_once<V>(src);   // (on its way while the length is)
    const Held h = held(tab, c.lens, b);
    if (h.lo + h.n + h.fresh > tab.cu[b + 1]) return;
    const int64_t slot = h.lo + h.n + (r - tab.cu_new[b]);
    *reinterpret_cast<V*>((uint8_t*)(blockIdx.z ? c.v : c.k) + (g * c.sh + slot * c.ss) * elem_bytes + (int64_t)u * sizeof(V)) = x;
    return;
  }
  if (blockIdx.y | blockIdx.z) return;
  const int64_t at = (int64_t)(blockIdx.x - row_blocks) * 256 + threadIdx.x;
  if (at < tab.batch) {
    const Held h = held(tab, c.lens, (int)at);
    lens_out[at] = h.lo + h.n + h.fresh > tab.cu[at + 1] ? h.n : h.n + h.fresh;
  }
  if (at >= total * c.planes) return;
  const int64_t p = at / total, r = at - p * total;
  int b = 0;
  for (int i = 1; i < tab.batch; ++i) b += r >= tab.cu_new[i];
  const Held h = held(tab, c.lens, b);
  if (h.lo + h.n + h.fresh > tab.cu[b + 1]) return;
  const int64_t slot = p * c.slots + h.lo + h.n + (r - tab.cu_new[b]);
  if (pos_new) c.pos[slot] = pos_new[p * nsp + r];
  if (c.mass) c.mass[slot] = mass_new ? mass_new[p * nsp + r] : 0.f;
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
  const Held h = held(tab, c.lens, b);
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
  const int64_t total = t.cu_new[t.batch];
  const uintptr_t bits = (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)c.k | (uintptr_t)c.v |
                         (uintptr_t)((nsh | nst | c.sh | c.ss | c.d) * elem_bytes);
  with_cache_table(t, [&](const auto& tab) {
    with_unit(bits, [&](auto unit) {
      using V = decltype(unit);
      const uint32_t upr = (uint32_t)(c.d * elem_bytes / (int)sizeof(V));
      const unsigned row_blocks = (unsigned)ceil_div(total * upr, 256);
      const unsigned rest = (unsigned)ceil_div(total * c.planes > t.batch ? total * c.planes : t.batch, 256);
      cache_append_kernel<std::decay_t<decltype(tab)>, V><<<dim3(row_blocks + rest, (unsigned)c.G, 2), 256, 0, st>>>(
          tab, c, (const uint8_t*)k_new, (const uint8_t*)v_new, nsh, nst, elem_bytes, upr, pos_new, mass_new, nsp, row_blocks, lens_out);
    });
  });
  return hipGetLastError();
}

hipError_t launch_cache_accept(const CacheTable& t, const CacheView& c, const int32_t* path, const int32_t* n_accept,
                               int elem_bytes, int32_t* lens_out, hipStream_t st) {
  const uintptr_t bits = (uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)((c.sh | c.ss | c.d) * elem_bytes);
  with_cache_table(t, [&](const auto& tab) {
    with_unit(bits, [&](auto unit) {
      using V = decltype(unit);
      cache_accept_kernel<std::decay_t<decltype(tab)>, V><<<dim3((unsigned)t.batch, (unsigned)c.G, 3), 256, 0, st>>>(
          tab, c, path, n_accept, elem_bytes, c.d * elem_bytes / (int)sizeof(V), lens_out);
    });
  });
  return hipGetLastError();
}

}  // namespace skv
