// What the bf16 matrix kernels on a cache share.
#pragma once
#include "cache.h"

namespace skv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float floatx2;
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef const __attribute__((address_space(1))) void* gbl_ptr_t;

// s_waitcnt with only the vector-memory counter constrained (gfx9 encoding: vmcnt in bits 3:0 and 15:14); no access moves across
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "the counter's range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
}
// ... with only the LDS counter constrained, to zero
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4) | (0 << 8));
  asm volatile("" ::: "memory");
}

// the workgroup's barrier, with loads to LDS left on their way; no access moves across
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A tile of V whose first slot is fresh slot `first` (or lies that far before them): what is not a number in fresh slots would reach rows
// that do not see them (0 x NaN), so there are zeros in its place; the fresh slots where there was some are returned, and rows that see one
// of those get NaN in the end.  By the lanes of a wave, PIECES of 64 units from `from` on.  The usual tile, which has none, costs a look.
template <int SEGS, int PIECES>
__device__ __forceinline__ uint64_t clear_odd_values(uint8_t* vt, int first, int fresh, int from) {
  typedef __attribute__((ext_vector_type(4))) uint32_t four;
  constexpr int ROWS = 64 / SEGS;
  const int lane = threadIdx.x & 63;
  uint32_t any = 0;
#pragma unroll
  for (int u = 0; u < PIECES; ++u) {
    const four v = *reinterpret_cast<const four*>(vt + ((from + u) * 64 + lane) * 16);
    uint32_t odd = 0;   // a half's exponent of ones carries into its sign's place
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= (v[e] & 0x7F807F80u) + 0x00800080u;
    any |= first + (from + u) * ROWS + lane / SEGS >= 0 ? odd & 0x80008000u : 0u;
  }
  if (!__any(any != 0)) return 0;
  uint64_t odd_slots = 0;
#pragma unroll 1
  for (int u = from; u < from + PIECES; ++u) {
    four* piece = reinterpret_cast<four*>(vt + (u * 64 + lane) * 16);
    four v = *piece;
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool low = (v[e] & 0x7F80u) == 0x7F80u, high = (v[e] & 0x7F800000u) == 0x7F800000u;
      odd |= low || high;
      v[e] &= (low ? 0xFFFF0000u : ~0u) & (high ? 0xFFFFu : ~0u);
    }
    odd &= first + u * ROWS + lane / SEGS >= 0;
    if (odd) *piece = v;
    const uint64_t lanes = __ballot(odd);
#pragma unroll 1
    for (int r = 0; r < ROWS; ++r) {
      const int s = first + u * ROWS + r;
      if (((lanes >> (r * SEGS)) & ((1ull << SEGS) - 1)) && s < fresh) odd_slots |= 1ull << s;
    }
  }
  wait_lds();
  return odd_slots;
}

// From references of this size on a scaled score and its row's reference, both rounded alike, are subtracted: an fma takes them apart by the
// reference's rounding, 2^-24 of it, which is then beyond what an exponent bears.
constexpr float kHuge = 16777216.f;

enum { kPlain = 0, kCapped = 1, kBiased = 2 };   // how scores are formed: scaled; capped; with a bias, and capped or not
template <class F>
void with_mode(const ScoreForm& f, F go) {
  if (f.slopes) go(std::integral_constant<int, kBiased>{});
  else if (f.softcap > 0.f) go(std::integral_constant<int, kCapped>{});
  else go(std::integral_constant<int, kPlain>{});
}

// A tile of 32 rows on its way to LDS, 16-byte pieces: piece (row, seg) at unit row * SEGS + (seg ^ swizzle(row)).  The swizzles let 16 lanes
// with a row each and one seg (K), and 32 lanes with 8-byte pieces of eight rows (V) use every bank once.
template <int SEGS> __device__ __forceinline__ constexpr int swizzle_k(int s) { return SEGS == 16 ? (s & 15) : ((s >> 1) & 7); }
template <int SEGS> __device__ __forceinline__ constexpr int swizzle_v(int s) { return SEGS == 16 ? (s & 7) << 1 : ((s >> 1) & 3) << 1; }

}  // namespace skv
