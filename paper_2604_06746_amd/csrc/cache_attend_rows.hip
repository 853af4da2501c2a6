// Attention of many fresh rows over a bf16 cache (trees of drafts): 128 query rows of a KV head a workgroup, 32 a wave.
//
// S^T = K Q^T and O^T = V^T P^T tile by tile of 32 slots, with 32x32x16 matrix instructions: a lane holds one row's scores of sixteen slots, so the
// softmax needs one exchange between lanes, and only where a score lies 2^8 above the row's reference.  The weights enter as hi + lo, two bf16
// numbers of 16 bits in all (one would be off by 2^-9 of each weight, as much as the result's own rounding).  The waves share the tiles: they are
// fetched once a workgroup, three ahead in a ring of four, with one meeting a tile.  A tile's scores are multiplied while the weights of
// the one before are formed, and its first half's values are while the second half's weights are: per tile 24 matrix instructions of
// 32 cycles and some 150 others of 4, which one wave alone would do in turns.
//
// Bound by the matrix units at the clock that they leave: four trees of 64 drafts over 8K to 16.5K slots (52 GFLOP; with the weights' second
// part 78), capped at 30, 97 us, 800 TFLOP/s of matrix instructions.  The cap's some 150 instructions a tile have no products above them: passes
// back to back, the join among them, take 114 us with it and 97 without.  Four waves with tiles of their own and 16x16x32 instructions took 106 to
// 113 us where this kernel took 92, with a cap of fewer bits.
#include "cache_bf16.h"

namespace skv {
namespace {

typedef __attribute__((ext_vector_type(16))) float floatx16;

// What the matrix instruction wants of V for D / 32 blocks of 32 components and two steps of 16 slots: ds_read_b64_tr_b16 reads, by 16 lanes,
// 8 bytes each, four rows of 16 numbers and hands lane i column i of them.  The wait is part of the statement: nothing uses or moves a register
// before it is there.
typedef __attribute__((ext_vector_type(2))) uint32_t pair;
__device__ __forceinline__ bf16x8 joined(pair a, pair b) {
  typedef __attribute__((ext_vector_type(4))) uint32_t four;
  return __builtin_bit_cast(bf16x8, four{a[0], a[1], b[0], b[1]});
}
#define SKV_COLUMNS(r0, r1, r2, r3, at) \
  "ds_read_b64_tr_b16 %" r0 ", %" at "\n\tds_read_b64_tr_b16 %" r1 ", %" at " offset:%[o1]\n\t" \
  "ds_read_b64_tr_b16 %" r2 ", %" at " offset:%[o2]\n\tds_read_b64_tr_b16 %" r3 ", %" at " offset:%[o3]\n\t"
__device__ __forceinline__ void read_columns(bf16x8 (&v)[2][4], uint32_t a) {
  pair r[16];
  asm volatile(SKV_COLUMNS("0", "1", "2", "3", "16") SKV_COLUMNS("4", "5", "6", "7", "17") SKV_COLUMNS("8", "9", "10", "11", "18")
               SKV_COLUMNS("12", "13", "14", "15", "19") "s_waitcnt lgkmcnt(0)"
               : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]),
                 "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
               : "v"(a), "v"(a ^ 64u), "v"(a ^ 128u), "v"(a ^ 192u), [o1] "n"(8 * 256), [o2] "n"(16 * 256), [o3] "n"(24 * 256)
               : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[0][i] = joined(r[4 * i], r[4 * i + 1]); v[1][i] = joined(r[4 * i + 2], r[4 * i + 3]); }
}
__device__ __forceinline__ void read_columns(bf16x8 (&v)[2][2], uint32_t a) {
  pair r[8];
  asm volatile(SKV_COLUMNS("0", "1", "2", "3", "8") SKV_COLUMNS("4", "5", "6", "7", "9") "s_waitcnt lgkmcnt(0)"
               : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
               : "v"(a), "v"(a ^ 64u), [o1] "n"(8 * 128), [o2] "n"(16 * 128), [o3] "n"(24 * 128)
               : "memory");
#pragma unroll
  for (int i = 0; i < 2; ++i) { v[0][i] = joined(r[4 * i], r[4 * i + 1]); v[1][i] = joined(r[4 * i + 2], r[4 * i + 3]); }
}

constexpr float kSlack = 8.f;   // how far above its reference a score may lie, log2
constexpr int kPlaces = 4;      // tiles of the ring
// V's swizzle: the 32 lanes that read at once have 64 bytes of four rows
template <int SEGS> __device__ __forceinline__ constexpr int swizzle_wide(int s) { return SEGS == 16 ? (s & 3) << 2 : ((s >> 1) & 1) << 2; }

template <class TAB, int D, int MODE>
__global__ __launch_bounds__(64 * kAttendWaves, 2) void cache_attend_rows_kernel(TAB tab, CacheView c, ScoreForm f, AttendWork w) {
  constexpr int RW = kAttendWaves, KS = D / 16, DB = D / 32, SEGS = D / 8, ROW = D + 4;
  constexpr int TILE = 32 * D * 2, NI = TILE / 1024 / RW;            // bytes of a tile of K or V, a wave's load instructions for it
  constexpr int POS = MODE == kBiased ? 256 : 0, NT = 2 * NI + (POS ? 1 : 0);
  constexpr int SLOT = 2 * TILE + POS, RING = kPlaces * SLOT, FIN = 32 * RW * ROW * 4;
  static_assert(TILE / 1024 % RW == 0, "a tile's loads split evenly over the waves");
  constexpr int ODD = RING > FIN ? RING : FIN;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[ODD + 8];
  const int lane = threadIdx.x & 63, l16 = lane & 15, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const AttendPlace p = attend_place(tab, c, w);
  if (p.b < 0) return;
  const Held& h = p.h;
  const int n = h.n, s0 = p.s0, s1 = p.s1;
  if (s0 >= s1 && p.nc > 1) return;   // (the join reads no more chunks than have slots)
  const int new0 = tab.cu_new[p.b], rows = h.fresh * w.gs, row0 = p.rc * 32 * RW + 32 * wave;
  const int row = min(row0 + l32, rows - 1), t = token_of(w, row), head = p.g * w.gs + row - t * w.gs;
  bf16x8 qf[KS];
  const uint16_t* qrow = (const uint16_t*)w.q + (int64_t)(new0 + t) * w.qst + (int64_t)head * w.qsh;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qrow + ks * 16 + 8 * half);
  const uint64_t mask = row_mask(f, new0 + t, t);
  const uint16_t* kg = (const uint16_t*)c.k + (int64_t)p.g * c.sh + h.lo * c.ss;
  const uint16_t* vg = (const uint16_t*)c.v + (int64_t)p.g * c.sh + h.lo * c.ss;
  const int32_t* pos = MODE == kBiased ? c.pos + (c.planes > 1 ? p.g * c.slots : 0) + h.lo : nullptr;
  const float slope = MODE == kBiased ? f.slopes[head] : 0.f;
  const int at = MODE == kBiased && n > 0 ? pos[h.base + t] : 0;
  uint32_t koff[NI], voff[NI];   // of the pieces this lane fetches, from the tile's first row
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int unit = (i * RW + wave) * 64 + lane, s = unit / SEGS;
    koff[i] = (uint32_t)(s * c.ss + ((unit % SEGS) ^ swizzle_k<SEGS>(s)) * 8) * 2u;
    voff[i] = (uint32_t)(s * c.ss + ((unit % SEGS) ^ swizzle_wide<SEGS>(s)) * 8) * 2u;
  }
  const int tiles = s1 > s0 ? (s1 - s0 + 31) / 32 : 0;
  auto fetch = [&](int i) __attribute__((always_inline)) {
    const int j0 = s0 + 32 * i;
    uint8_t* to = lds + (i & (kPlaces - 1)) * SLOT;
    const uint8_t* kb = (const uint8_t*)(kg + (int64_t)j0 * c.ss);
    const uint8_t* vb = (const uint8_t*)(vg + (int64_t)j0 * c.ss);
    if (j0 + 32 <= n) {
#pragma unroll
      for (int k = 0; k < NI; ++k) {
        __builtin_amdgcn_global_load_lds((gbl_ptr_t)(kb + koff[k]), (lds_ptr_t)(to + (k * RW + wave) * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((gbl_ptr_t)(vb + voff[k]), (lds_ptr_t)(to + TILE + (k * RW + wave) * 1024), 16, 0, 0);
      }
    } else {   // rows past the end re-read the last one (their scores are masked)
      const int last = n - 1 - j0;
#pragma unroll
      for (int k = 0; k < NI; ++k) {
        const int unit = (k * RW + wave) * 64 + lane, s = unit / SEGS;
        const uint32_t from = (uint32_t)(min(s, last) * c.ss);
        __builtin_amdgcn_global_load_lds((gbl_ptr_t)(kb + (from + ((unit % SEGS) ^ swizzle_k<SEGS>(s)) * 8) * 2u),
                                         (lds_ptr_t)(to + (k * RW + wave) * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((gbl_ptr_t)(vb + (from + ((unit % SEGS) ^ swizzle_wide<SEGS>(s)) * 8) * 2u),
                                         (lds_ptr_t)(to + TILE + (k * RW + wave) * 1024), 16, 0, 0);
      }
    }
    // (by every wave, the same to the same place, so that the waits know how many there are)
    if (POS) __builtin_amdgcn_global_load_lds((gbl_ptr_t)(pos + min(j0 + l32, n - 1)), (lds_ptr_t)(to + 2 * TILE), 4, 0, 0);
  };
  // (kept in registers from here on; nothing of it is on its way when the first tiles are requested)
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
#pragma unroll
  for (int i = 0; i < kPlaces - 1; ++i)
    if (i < tiles) fetch(i);

  auto highest = [](const floatx16& y) __attribute__((always_inline)) {
    float top = y[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, y[e]);
    return top;
  };
  floatx16 O[DB], x;
  float top = kNothingSeen;
  float M = kNothingSeen, Z = 0.f;
  bool huge = false;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) O[db][e] = 0.f;
  const int edge = min(s1, f.tree || h.fresh > 1 ? max(h.base, 0) : n);
  const Cap cap(f, MODE == kCapped ? kLog2e : 1.f);
  const int ka = l32 * SEGS, kx = swizzle_k<SEGS>(l32);
  const int vs = 4 * half + (l16 >> 2);
  const uint32_t va = (uint32_t)(uintptr_t)(lds_ptr_t)(lds + TILE) + (vs * SEGS + ((2 * ((lane >> 4) & 1) + ((l16 >> 1) & 1)) ^ swizzle_wide<SEGS>(vs))) * 16 + (l16 & 1) * 8;
  auto read_rows = [&](bf16x8 (&kf)[KS], int i) __attribute__((always_inline)) {
    const uint8_t* kt = lds + (i & (kPlaces - 1)) * SLOT;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[ks] = *reinterpret_cast<const bf16x8*>(kt + (ka + ((ks * 2 + half) ^ kx)) * 16);
  };
  auto products = [&](const bf16x8 (&kf)[KS]) __attribute__((always_inline)) {
    floatx16 y;
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], y, 0, 0, 0);
    return y;
  };
  unsigned long long* odd = reinterpret_cast<unsigned long long*>(lds + ODD);   // fresh slots whose values are not all numbers (beside
  // a second __shared__ variable the compiler waits for every load before it reads a tile: 92 -> 98 us)
  if (threadIdx.x == 0) *odd = 0;
  wait_lds();
  if (tiles > 0) {
    if (tiles > 2) wait_loads<2 * NT>();
    else if (tiles > 1) wait_loads<NT>();
    else wait_loads<0>();
    meet();
    bf16x8 kf[KS];
    read_rows(kf, 0);
    x = products(kf);
    if (MODE == kPlain) top = highest(x);
  }
  for (int i = 0; i < tiles; ++i) {
    const int j0 = s0 + 32 * i;
    // this wave's part of the next tile is there, then everyone's; the place of the tile before is free
    if (i + 2 < tiles) wait_loads<NT>();
    else wait_loads<0>();
    meet();
    if (i + kPlaces - 1 < tiles) fetch(i + kPlaces - 1);
    const bool ragged = j0 + 32 > edge;
    if (h.base >= 0 && j0 + 32 > h.base) {   // each wave a part of the tile
      constexpr int PART = 32 * SEGS / 64 / RW;
      const uint64_t some = clear_odd_values<SEGS, PART>(lds + (i & (kPlaces - 1)) * SLOT + TILE, j0 - h.base, h.fresh, wave * PART);
      if (some && lane == 0) atomicOr(odd, (unsigned long long)some);
      meet();
    }
    if (row0 >= rows) continue;   // (a wave without rows only fetches)
    if (MODE == kCapped) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float y[4] = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
        cap.apply(y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * q + e] = y[e];
      }
    } else if (MODE == kBiased) {
      typedef __attribute__((ext_vector_type(4))) int intx4;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const intx4 fr = *reinterpret_cast<const intx4*>(lds + (i & (kPlaces - 1)) * SLOT + 2 * TILE + (8 * q + 4 * half) * 4);
        float y[4] = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
        scaled(f, cap, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * q + e] = biased(y[e], slope, at - fr[e]);
      }
    }
    float c2 = MODE == kPlain ? f.c2 : 1.f;
    if (ragged) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int s = j0 + 8 * (e >> 2) + 4 * half + (e & 3);
        if (s >= s1 || !sees(mask, s, h.base)) x[e] = -INFINITY;
      }
    }
    if (MODE != kPlain || ragged) top = highest(x);
    if (__any(fmaf(top, c2, -M) > kSlack)) {
      top *= c2;
      top = fmaxf(top, __shfl_xor(top, 32));
      const float Mn = fmaxf(M, top), shrink = __builtin_amdgcn_exp2f(M - Mn);
      M = Mn;
      Z *= shrink;
#pragma unroll
      for (int db = 0; db < DB; ++db) O[db] *= shrink;
      if (MODE == kPlain) huge = __any(fabsf(M) >= kHuge && M > kNothingSeen);
    }
    if (MODE == kPlain && huge) {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] *= c2;
      c2 = 1.f;
    }
    // (ahead of the other workgroup's waves from here on: theirs are then elsewhere in their tiles; 99 -> 91 us)
    __builtin_amdgcn_s_setprio(1);
    bf16x8 kf[KS], vf[2][DB];
    read_rows(kf, i + 1);   // (behind the last tile whatever lies there: not used)
    read_columns(vf, va + (i & (kPlaces - 1)) * SLOT);
    // the next tile's scores under the first half's weights, the second half's weights under the first one's products: a matrix instruction
    // leaves room for about six others
    floatx16 next;
#pragma unroll
    for (int e = 0; e < 16; ++e) next[e] = 0.f;
    floatx2 pr;
    float z = 0.f;   // (a tile's by itself: a lane has half of its row's slots)
    bf16x8 hi[2], lo[2];
    auto weigh = [&](int s, int u) __attribute__((always_inline)) {   // part u of 8: numbers 2 (u / 2) and the one behind of half s
      const int e = u & ~1;
      if (u % 2 == 0) {
        pr = floatx2{__builtin_amdgcn_exp2f(fmaf(x[8 * s + e], c2, -M)), __builtin_amdgcn_exp2f(fmaf(x[8 * s + e + 1], c2, -M))};
      } else {
        z += pr[0] + pr[1];
        const bf16x2 up = __builtin_convertvector(pr, bf16x2);
        const floatx2 rest = {pr[0] - (float)up[0], pr[1] - (float)up[1]};
        const bf16x2 down = __builtin_convertvector(rest, bf16x2);
        hi[s][e] = up[0]; hi[s][e + 1] = up[1];
        lo[s][e] = down[0]; lo[s][e + 1] = down[1];
      }
    };
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      __builtin_amdgcn_sched_barrier(0);
      next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], qf[k], next, 0, 0, 0);
#pragma unroll
      for (int u = k * 8 / KS; u < (k + 1) * 8 / KS; ++u) weigh(0, u);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int k = 0; k < 2 * DB; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        O[k % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s][k % DB], k < DB ? hi[s] : lo[s], O[k % DB], 0, 0, 0);
        if (s == 0) {
#pragma unroll
          for (int u = k * 4 / DB; u < (k + 1) * 4 / DB; ++u) weigh(1, u);
        } else if (k == DB) {
          if (MODE == kPlain) top = highest(next);
          Z += z;
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
    x = next;
  }
  // through LDS, each wave by itself, to whole rows
  __syncthreads();
  if (mask & *odd) {
#pragma unroll
    for (int db = 0; db < DB; ++db) O[db] *= NAN;
  }
  float* buf = reinterpret_cast<float*>(lds) + wave * 32 * ROW;
  Z += __shfl_xor(Z, 32);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<floatx4*>(buf + l32 * ROW + 32 * db + 8 * q + 4 * half) = floatx4{O[db][4 * q], O[db][4 * q + 1], O[db][4 * q + 2], O[db][4 * q + 3]};
  wait_lds();
  for (int e = lane; e < 32 * (D / 4); e += 64) {
    const int r = e / (D / 4), at4 = e % (D / 4) * 4;
    const float m = __shfl(M, r), z = __shfl(Z, r);
    if (row0 + r >= rows) continue;
    leave<uint16_t, D>(w, D, p.g, row0 + r, at4, m, z, *reinterpret_cast<const floatx4*>(buf + r * ROW + at4), new0, (int64_t)blockIdx.x * 32 * RW + 32 * wave + r, p.nc);
  }
}

template <int D>
hipError_t attend(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p, const AttendWork& w, hipStream_t st) {
  with_cache_table(t, [&](const auto& tab) {
    with_mode(f, [&](auto mode) {
      cache_attend_rows_kernel<std::decay_t<decltype(tab)>, D, decltype(mode)::value><<<dim3((unsigned)(p.units * c.G)), 64 * kAttendWaves, 0, st>>>(tab, c, f, w);
    });
  });
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_attend_rows(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p,
                                    const AttendWork& w, hipStream_t st) {
  return c.d == 128 ? attend<128>(t, c, f, p, w, st) : attend<64>(t, c, f, p, w, st);
}

}  // namespace skv
