// Attention of fresh tokens over a bf16 cache of 64 or 128 components, in bf16 matrix instructions.
//
// The same split and the same sums as in cache_attend_f32.hip: S^T = K Q^T, so that a lane has one query row and, of a tile of 32 slots,
// eight of them (4 q .. 4 q + 3 and 16 more, q = lane / 16); O^T = V^T P^T takes them as they are when V's rows are handed to the matrix
// instruction in that order, which ds_read_b64_tr_b16 does: it gives a lane four consecutive slots' values of one component.
// P goes into the product as two bf16 numbers, p = hi + lo (16 bits of it): what a single one would lose, 2^-8 of every weight, is as much
// as the output's own rounding, and the matrix pipe has room while the cache is what binds.
//
// A single token's work is to read the cache: 512 bytes of K and V per slot and KV head against 16 matrix instructions per 32 of
// them.  Tiles go from memory to LDS without registers (global_load_lds), each wave has room for one tile of its own and no barrier: as
// soon as K's half has been used the next tile's K is requested into it, and likewise V, and the waves of a CU (eight at 128
// components) fill each other's waits with about 100 KB on their way.
// NT: tiles are fetched with the non-temporal policy, where no other workgroup reads them and the cache is larger than what the memory-side
// cache keeps from one step to the next: 4 GB 715 -> 623 us (6.9 TB/s), 216 MB 81 -> 72 us.  The stores of the scores (128 bytes a
// slot of 32 heads) are what gathering weights costs: 846 us with them and their reading, 696 where they stayed in a cache.
// Rows beyond 32 of a KV head are other workgroups', which read the tiles again, from the XCD's L2; beyond 64 cache_attend_rows.hip has them.
// The rows' references M follow lazily: they are raised only when a score lies more than 2^8 above one of them, so that the usual tile has
// no exchange between lanes and no rescaling.
#include "cache_bf16.h"

namespace skv {
namespace {

// What the matrix instruction wants of V for four blocks of 16 components: ds_read_b64_tr_b16 reads, by 16 lanes, 8 bytes each, four rows of
// 16 numbers and hands lane i column i of them.  The wait is part of the statement: nothing uses or moves a register before it is there.
template <int HALF>
__device__ __forceinline__ void read_columns(bf16x8 (&v)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
  typedef __attribute__((ext_vector_type(2))) uint32_t pair;
  pair r[8];
  asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
               "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
               "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
               "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
               : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(HALF)
               : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    typedef __attribute__((ext_vector_type(4))) uint32_t four;
    const four f = {r[2 * i][0], r[2 * i][1], r[2 * i + 1][0], r[2 * i + 1][1]};
    v[i] = __builtin_bit_cast(bf16x8, f);
  }
}
typedef floatx4 __attribute__((aligned(4))) floatx4_at_4;

constexpr float kSlack = 8.f;                    // how far above its reference a score may lie, log2

template <class TAB, int D, int RB, int MODE, bool SAVE, bool NT>
__global__ __launch_bounds__(64 * kAttendWaves, 2) void cache_attend_bf16_kernel(TAB tab, CacheView c, ScoreForm f, AttendWork w) {
  constexpr int KS = D / 32, DB = D / 16, SEGS = D / 8;   // steps of the first product, row blocks of the second, 16-byte pieces of a row
  constexpr int TILE = 32 * D * 2, NI = TILE / 1024;      // bytes of a tile of K or V, load instructions for it
  constexpr int POS = MODE == kBiased ? 256 : 0, NP = POS ? 1 : 0;   // its positions
  constexpr int SLOT = 2 * TILE + POS, RING = kAttendWaves * SLOT, FIN = kFinishFloats<D, RB> * 4;
  constexpr int NK = NI + NP;                             // load instructions of a tile's first half: K and positions
  constexpr int NS = SAVE ? 2 : 0;                        // stores of a tile's scores
  __shared__ __attribute__((aligned(1024))) uint8_t lds[RING > FIN ? RING : FIN];
  const int lane = threadIdx.x & 63, l16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const AttendPlace p = attend_place(tab, c, w);
  if (p.b < 0) return;
  const Held& h = p.h;
  const int n = h.n, s0 = p.s0, s1 = p.s1;
  // the queries first: the length has no part in their addresses
  const int new0 = tab.cu_new[p.b], rows = h.fresh * w.gs, row0 = p.rc * 16 * RB;
  bf16x8 qf[RB][KS];
  uint64_t mask[RB];
  float slope[RB];
  int at[RB];
  float* save = nullptr;   // where this lane's scores go
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = min(row0 + rb * 16 + l16, rows - 1), t = token_of(w, row), head = p.g * w.gs + row - t * w.gs;
    const int64_t r = new0 + t;
    const uint16_t* qrow = (const uint16_t*)w.q + r * w.qst + (int64_t)head * w.qsh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[rb][ks] = *reinterpret_cast<const bf16x8*>(qrow + ks * 32 + 8 * q4);
    mask[rb] = row_mask(f, r, t);
    slope[rb] = MODE == kBiased ? f.slopes[head] : 0.f;
    if (SAVE) save = w.x + head * w.xs + h.lo + kScorePad * p.b;
  }
  if (s0 >= s1 && (p.nc > 1 || w.x)) return;   // (the join reads no more chunks than have slots)

  const uint16_t* kg = (const uint16_t*)c.k + (int64_t)p.g * c.sh + h.lo * c.ss;
  const uint16_t* vg = (const uint16_t*)c.v + (int64_t)p.g * c.sh + h.lo * c.ss;
  const int32_t* pos = MODE == kBiased ? c.pos + (c.planes > 1 ? p.g * c.slots : 0) + h.lo : nullptr;
  uint8_t* kt = lds + wave * SLOT;
  uint8_t* vt = kt + TILE;
  auto swz_k = [](int s) { return swizzle_k<SEGS>(s); };
  auto swz_v = [](int s) { return swizzle_v<SEGS>(s); };
  uint32_t koff[NI], voff[NI];   // of the pieces this lane fetches, from the tile's first row
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int unit = i * 64 + lane, s = unit / SEGS;
    koff[i] = (uint32_t)(s * c.ss + ((unit % SEGS) ^ swz_k(s)) * 8) * 2u;
    voff[i] = (uint32_t)(s * c.ss + ((unit % SEGS) ^ swz_v(s)) * 8) * 2u;
  }
  // (rows past the end re-read the last one: their scores are masked)
  auto fetch = [&](const uint16_t* from, const uint32_t (&off)[NI], auto swz, int j0, uint8_t* to) __attribute__((always_inline)) {
    const uint8_t* base = (const uint8_t*)(from + (int64_t)j0 * c.ss);
    if (j0 + 32 <= n) {
#pragma unroll
      for (int i = 0; i < NI; ++i) __builtin_amdgcn_global_load_lds((gbl_ptr_t)(base + off[i]), (lds_ptr_t)(to + i * 1024), 16, 0, NT ? 2 : 0);
    } else {
      const int last = n - 1 - j0;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int unit = i * 64 + lane, s = unit / SEGS;
        __builtin_amdgcn_global_load_lds((gbl_ptr_t)(base + (uint32_t)(min(s, last) * c.ss + ((unit % SEGS) ^ swz(s)) * 8) * 2u),
                                         (lds_ptr_t)(to + i * 1024), 16, 0, NT ? 2 : 0);
      }
    }
  };
  auto fetch_k = [&](int j0) __attribute__((always_inline)) {
    fetch(kg, koff, swz_k, j0, kt);
    if (POS) __builtin_amdgcn_global_load_lds((gbl_ptr_t)(pos + min(j0 + (lane & 31), n - 1)), (lds_ptr_t)(kt + 2 * TILE), 4, 0, 0);
  };
  auto fetch_v = [&](int j0) __attribute__((always_inline)) { fetch(vg, voff, swz_v, j0, vt); };

  // this wave's tiles: wave, wave + 4, ...
  const int tiles = s1 > s0 ? (s1 - s0 + 31) / 32 : 0, mine = tiles > wave ? (tiles - wave + kAttendWaves - 1) / kAttendWaves : 0;
  if (mine > 0) { fetch_k(s0 + 32 * wave); fetch_v(s0 + 32 * wave); }

#pragma unroll
  for (int rb = 0; rb < RB; ++rb) at[rb] = MODE == kBiased && n > 0 ? pos[h.base + token_of(w, min(row0 + rb * 16 + l16, rows - 1))] : 0;
  // (kept in registers from here on; pinned once all of them are on their way)
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[rb][ks]));

  floatx4 O[DB][RB];
  float M[RB], Z[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    M[rb] = kNothingSeen; Z[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) O[db][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  // from here on rows differ in what they see: the first fresh slot, or the end
  const int edge = min(s1, f.tree || h.fresh > 1 ? max(h.base, 0) : n);
  const Cap cap(f, MODE == kCapped ? kLog2e : 1.f);
  uint64_t odd = 0;   // fresh slots whose values are not all numbers
  bool huge = false;

  for (int i = 0; i < mine; ++i) {
    const int j0 = s0 + 32 * (wave + kAttendWaves * i), next = j0 + 32 * kAttendWaves;
    // K (and the positions) are there; what followed them, the scores of the tile before and V, may be on its way
    if (i > 0) wait_loads<NS + NI>(); else wait_loads<NI>();
    floatx4 x[2][RB];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) x[kb][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int s = kb * 16 + l16;
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + (s * SEGS + ((ks * 4 + q4) ^ swz_k(s))) * 16);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) x[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rb][ks], x[kb][rb], 0, 0, 0);
      }
    // scores in the log2 domain, but for their scale where there is nothing else to them
    if (MODE == kCapped) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float y[4] = {x[kb][rb][0], x[kb][rb][1], x[kb][rb][2], x[kb][rb][3]};
          cap.apply(y);
          x[kb][rb] = floatx4{y[0], y[1], y[2], y[3]};
        }
    } else if (MODE == kBiased) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        typedef __attribute__((ext_vector_type(4))) int intx4;
        const intx4 fr = *reinterpret_cast<const intx4*>(kt + 2 * TILE + (kb * 16 + 4 * q4) * 4);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float y[4] = {x[kb][rb][0], x[kb][rb][1], x[kb][rb][2], x[kb][rb][3]};
          scaled(f, cap, y);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[kb][rb][e] = biased(y[e], slope[rb], at[rb] - fr[e]);
        }
      }
    }
    wait_lds();   // K has been read: its place is free
    if (i + 1 < mine) fetch_k(next);
    float c2 = MODE == kPlain ? f.c2 : 1.f;
    const bool ragged = j0 + 32 > edge;
    if (ragged) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int s = j0 + kb * 16 + 4 * q4 + e;
            if (s >= s1 || !sees(mask[rb], s, h.base)) x[kb][rb][e] = -INFINITY;
          }
    }
    bool high = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float a = fmaxf(fmaxf(x[0][rb][0], x[0][rb][1]), fmaxf(x[0][rb][2], x[0][rb][3]));
      const float b = fmaxf(fmaxf(x[1][rb][0], x[1][rb][1]), fmaxf(x[1][rb][2], x[1][rb][3]));
      high |= fmaf(fmaxf(a, b), c2, -M[rb]) > kSlack;
    }
    if (__any(high)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float a = fmaxf(fmaxf(x[0][rb][0], x[0][rb][1]), fmaxf(x[0][rb][2], x[0][rb][3]));
        const float b = fmaxf(fmaxf(x[1][rb][0], x[1][rb][1]), fmaxf(x[1][rb][2], x[1][rb][3]));
        float top = fmaxf(a, b) * c2;
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float Mn = fmaxf(M[rb], top), shrink = __builtin_amdgcn_exp2f(M[rb] - Mn);
        M[rb] = Mn;
        Z[rb] *= shrink;
#pragma unroll
        for (int db = 0; db < DB; ++db) O[db][rb] *= shrink;
        if (MODE == kPlain) huge |= __any(fabsf(M[rb]) >= kHuge && M[rb] > kNothingSeen);
      }
    }
    if (MODE == kPlain && huge) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) x[kb][rb] *= c2;
      c2 = 1.f;
    }
    if (SAVE) {
      // Two stores from every wave, whatever the tile holds, so that the waits know how many there are: some lane has a row, and slots
      // from the end on, up to a tile's, have room.
      static_assert(!SAVE || RB == 1, "the stores that the waits count");
      asm volatile("" ::: "memory");
      if (row0 + l16 < rows) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) *reinterpret_cast<floatx4_at_4*>(save + j0 + kb * 16 + 4 * q4) = x[kb][0] * c2;
      }
      asm volatile("" ::: "memory");
    }
    bf16x8 hi[RB], lo[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float z = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const floatx2 pr = {__builtin_amdgcn_exp2f(fmaf(x[kb][rb][e], c2, -M[rb])), __builtin_amdgcn_exp2f(fmaf(x[kb][rb][e + 1], c2, -M[rb]))};
          z += pr[0] + pr[1];
          const bf16x2 up = __builtin_convertvector(pr, bf16x2);
          const floatx2 rest = {pr[0] - (float)up[0], pr[1] - (float)up[1]};
          const bf16x2 down = __builtin_convertvector(rest, bf16x2);
          hi[rb][kb * 4 + e] = up[0]; hi[rb][kb * 4 + e + 1] = up[1];
          lo[rb][kb * 4 + e] = down[0]; lo[rb][kb * 4 + e + 1] = down[1];
        }
      Z[rb] += z;
    }
    if (i + 1 < mine) wait_loads<NS + NK>(); else wait_loads<NS>();
    if (h.base >= 0 && j0 + 32 > h.base) odd |= clear_odd_values<SEGS, NI>(vt, j0 - h.base, h.fresh, 0);
    // (the swizzle is a whole number of 32-byte pairs, so the block of components enters the address as an exclusive or)
    const int vs = 4 * q4 + (l16 >> 2);
    const uint32_t va = (uint32_t)(uintptr_t)(lds_ptr_t)vt + (vs * SEGS + (((l16 >> 1) & 1) ^ swz_v(vs))) * 16 + (l16 & 1) * 8;
#pragma unroll
    for (int d4 = 0; d4 < DB; d4 += 4) {
      bf16x8 vf[4];
      read_columns<16 * D * 2>(vf, va ^ (d4 << 5), va ^ ((d4 + 1) << 5), va ^ ((d4 + 2) << 5), va ^ ((d4 + 3) << 5));
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          O[d4 + j][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j], hi[rb], O[d4 + j][rb], 0, 0, 0);
          O[d4 + j][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j], lo[rb], O[d4 + j][rb], 0, 0, 0);
        }
    }
    if (i + 1 < mine) fetch_v(next);   // (read_columns has waited)
  }
  if (odd) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int db = 0; db < DB; ++db) O[db][rb] *= mask[rb] & odd ? NAN : 1.f;
  }
  finish_chunk<uint16_t, D, RB>(O, M, Z, reinterpret_cast<float*>(lds), w, D, p.g, row0, rows, new0, p.nc);
}

template <int D, int RB>
hipError_t attend(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p, const AttendWork& w, hipStream_t st) {
  with_cache_table(t, [&](const auto& tab) {
    using TAB = std::decay_t<decltype(tab)>;
    const dim3 grid((unsigned)(p.units * c.G)), block(64 * kAttendWaves);
    auto go = [&](auto mode, auto save) {
      constexpr int MODE = decltype(mode)::value;
      constexpr bool SAVE = decltype(save)::value;
      if (p.stream) cache_attend_bf16_kernel<TAB, D, RB, MODE, SAVE, true><<<grid, block, 0, st>>>(tab, c, f, w);
      else cache_attend_bf16_kernel<TAB, D, RB, MODE, SAVE, false><<<grid, block, 0, st>>>(tab, c, f, w);
    };
    auto by_mode = [&](auto save) { with_mode(f, [&](auto mode) { go(mode, save); }); };
    if constexpr (RB == 1) {
      if (w.x) { by_mode(std::true_type{}); return; }
    }
    by_mode(std::false_type{});
  });
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_attend_bf16(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendPlan& p,
                                    const AttendWork& w, hipStream_t st) {
  if (c.d == 128) return p.rows == 16 ? attend<128, 1>(t, c, f, p, w, st) : attend<128, 2>(t, c, f, p, w, st);
  return p.rows == 16 ? attend<64, 1>(t, c, f, p, w, st) : attend<64, 2>(t, c, f, p, w, st);
}

}  // namespace skv
