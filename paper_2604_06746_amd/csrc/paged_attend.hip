// Attention of fresh tokens over a cache held in 8 bits, in pages.
//
// The split and the sums of cache_attend_bf16.hip: S^T = K Q^T, so that a lane has one query row and four slots of each block of 16, and
// O^T = V^T P^T takes the weights as they lie.  What is stored in 8 bits is exact in 16: keys enter their product as bf16 (queries too, those
// in fp32 as three parts), values theirs as fp16, the weights in two parts that add up to 22 bits.  Where
// a sequence's bf16 rows are more than a workgroup's, the matrix instructions count, and weights have one part, 11 bits: 2^-12 of a weight beside the
// result's own rounding of 2^-9, which turns the last bit of one result in 25 (with two parts one in 500, but 512 tokens over 32768 slots 367 -> 424 us,
// 4096 tokens by themselves 244 -> 267; where a workgroup has all rows the second part costs 0 to 2 %).
// A block of 16 slots lies in one page, so its scales are the same for all lanes: a key's scale multiplies the block's scores; a value's is
// part of the weight, w = 2^(y + log2 s_v - M), with the row's reference M a whole number, so that nothing of it is rounded.
// Blocks come straight from memory to registers: a lane's 16 bytes of a key are operands as they lie, since the order of components in a
// product is free; of the values a lane reads 8 bytes of each of four rows and puts rows beside each other with byte permutes.
// The waves take shares of a chunk's blocks; a lane looks up one block's page, place and scales, and only blocks of pages that are there are
// in the list that a wave goes by, so dropped pages cost nothing.
//
// Single tokens are bound by reading the codes: eight caches of 64K to 128K slots (1.6 GB) 266 us, 6.1 TB/s, past the caches (ONCE; through them
// 281); with two pairs of blocks in turns, where one at a time took 300.  256 workgroups more or 512 are no faster (268, 270).  Chunks of a prompt are bound by
// the issue port, which two waves a SIMD keep busy for 64 % of the time: 512 tokens over 32768 slots 366 us, 750 TFLOP/s; of the 252 vector instructions that a
// tile of 32 rows and 32 slots takes, 80 decode and 32 are matrix instructions.  64 rows a wave (one wave a SIMD) 421 us.
// Usual scores and scales take that loop; what fp32's range or bits do not bear in it is found there and done over with care, in a loop behind it
// (inside the first one that code cost chains of eight over four caches of 16K slots 31 -> 42 us).
#include "paged.h"

namespace skv {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 halfx8;
typedef __attribute__((ext_vector_type(2))) _Float16 halfx2;
typedef __attribute__((ext_vector_type(2))) float floatx2;
typedef __attribute__((ext_vector_type(4))) uint32_t four;

// Weights are at most 2^kTop (65504 is fp16's last number); when one would be more, the reference is raised so that the largest is some 2^kFresh.
constexpr float kTop = 15.f, kFresh = 7.f;
// From references of this size on, whole numbers only just, the fma takes a product and its row's reference apart by the latter's rounding, in the end by
// more than an exponent bears.  The wave then takes its blocks once more (CARE), by scores rounded once and references in two parts: N, the highest score,
// and L, a small number that has the values' scales: w = 2^((y - N) + (log2 s_v - L)).
constexpr float kHuge = 8388608.f;
// A weight has its value's scale, and its share of the norm is taken without it again; beside values of 2^100 as much that is nothing for weights
// that count.  So a wave that meets scales on both sides of these takes its blocks with care too, the norm's shares by exponents of their own.  (Within them what is
// lost is below 2^-49 of the norm.)
constexpr float kTinyScale = 0x1p-20f, kLargeScale = 0x1p12f;

// ONCE: past the caches
template <int N, bool ONCE> __device__ __forceinline__ void load_bytes(uint32_t (&to)[N / 4], const uint8_t* p) {
  typedef __attribute__((ext_vector_type(N / 4))) uint32_t vec;
  const vec x = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const vec*>(p)) : *reinterpret_cast<const vec*>(p);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) to[i] = x[i];
}
// an offset that is widened where it is used, so that the load takes it beside a base in scalar registers (widened ahead of a loop it costs
// an addition of 64 bits a load, and registers whose reuse waits for loads)
__device__ __forceinline__ uint32_t in_place(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}
// over the four lanes that share a row
__device__ __forceinline__ float row_total(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float row_top(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, bool high) {
  return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, false));
}
__device__ __forceinline__ uint32_t half_pair(uint32_t codes, bool high) {
  return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.f, false));
}
__device__ __forceinline__ bf16x8 eight_keys(uint32_t a, uint32_t b) {
  const four r = {bf16_pair(a, false), bf16_pair(a, true), bf16_pair(b, false), bf16_pair(b, true)};
  return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ float lane_float(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }

// components c .. c+7 of a query row, as one bf16 part or as three that add up to it
template <class T, int QP>
__device__ __forceinline__ void load_query(bf16x8 (&q)[QP], const T* row, int c, int d, bool aligned) {
  typedef __attribute__((ext_vector_type(4))) T vec;
  T x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = 0;
  if (c < d) {
    if (aligned) {
      const vec lo = *reinterpret_cast<const vec*>(row + c), hi = *reinterpret_cast<const vec*>(row + c + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = lo[i]; x[4 + i] = hi[i]; }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = row[c + i];
    }
  }
  if constexpr (QP == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[0][i] = __builtin_bit_cast(__bf16, x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float rest = x[i];
#pragma unroll
      for (int part = 0; part < QP; ++part) {
        // (cut off: to the nearest, the largest numbers would become infinity)
        const uint32_t bits = __float_as_uint(rest) & 0xFFFF0000u;
        q[part][i] = __builtin_bit_cast(__bf16, (uint16_t)(bits >> 16));
        rest -= __uint_as_float(bits);
      }
    }
  }
}

// What the waves of a workgroup leave, added up in their order through LDS and written out by all threads (leave), 16 rows at a time.  A lane
// holds components 4 W q4 + W e + j of its rows in O[j][rb][e].  What a wave puts there has its weights' sum
// between 1/2 and 1, the power of two taken to M; with references in two parts (apart), relative to N.
template <int DP, int WAVES>
constexpr int kFinishBlocks = WAVES * 16 * (DP + 4 + 2);
template <class T, int DP, int RB, int WAVES>
__device__ __forceinline__ void finish_blocks(const floatx4 (&O)[DP / 16][RB], const float (&Ml)[RB], const float (&Zl)[RB], const float (*apart)[2], float* buf,
                                              const AttendWork& w, int d, int g, int row0, int rows, int new0, int nc) {
  constexpr int PITCH = DP + 4, W = DP / 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q4 = lane >> 4;
  float* ml = buf + WAVES * 16 * PITCH;   // [wave][row][2]
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (row0 + rb * 16 >= rows) break;
    float z = row_total(Zl[rb]), M = Ml[rb];
    int shift = M > kNothingSeen ? -__builtin_amdgcn_frexp_expf(z) : 0;   // (0 for 0 and NaN)
    if (apart) {
      M = apart[rb * 16 + l16][0];
      shift = (int)apart[rb * 16 + l16][1];
    } else {
      M -= (float)shift;
    }
    z = ldexpf(z, shift);
    if (rb > 0) __syncthreads();
    if (q4 == 0) {
      ml[(wave * 16 + l16) * 2] = M;
      ml[(wave * 16 + l16) * 2 + 1] = z;
    }
    __syncthreads();
    float top = ml[l16 * 2];
    for (int i = 1; i < WAVES; ++i) top = fmaxf(top, ml[(i * 16 + l16) * 2]);
    const float f = ldexpf(__builtin_amdgcn_exp2f(M - top), shift);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < W; j += 4)
        *reinterpret_cast<floatx4*>(buf + (wave * 16 + l16) * PITCH + W * (4 * q4 + e) + j) =
            floatx4{O[j][rb][e], O[j + 1][rb][e], O[j + 2][rb][e], O[j + 3][rb][e]} * f;
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * (DP / 4); e += 64 * WAVES) {
      const int row = e / (DP / 4), c = e % (DP / 4) * 4;
      if (row0 + rb * 16 + row >= rows || c >= d) continue;
      float best = ml[row * 2];
      for (int i = 1; i < WAVES; ++i) best = fmaxf(best, ml[(i * 16 + row) * 2]);
      float sum = 0.f;
      floatx4 o = {0.f, 0.f, 0.f, 0.f};
      for (int i = 0; i < WAVES; ++i) {
        sum += ml[(i * 16 + row) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(i * 16 + row) * 2] - best);
        o += *reinterpret_cast<const floatx4*>(buf + (i * 16 + row) * PITCH + c);
      }
      leave<T, DP>(w, d, g, row0 + rb * 16 + row, c, best, sum, o, new0, (int64_t)blockIdx.x * 16 * RB + rb * 16 + row, nc);
    }
  }
}

// Two blocks on their way, or at work: their codes, and what all lanes know of them.
template <int DP>
struct Pair {
  uint32_t k[2][DP / 64][4], v[2][4][DP / 64];
  float kf[2], lv[2], iv[2];   // of the scores; log2 of the values' scale, and its inverse
  int at[2];                   // their places in the batch of 64 that starts at block `base`
  int base;
  bool any, two;
};

// HELD: batches of 64 blocks whose weights stay in LDS until they go to memory, for 16 / HELD rows of a KV head at most; 0: nobody wants them.
template <class TAB, class T, int DP, int RB, bool CAPPED, int HELD, bool ONCE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, RB * DP > 256 ? 1 : 2) void paged_attend_kernel(TAB tab, CacheView view, PagedView c, ScoreForm f, AttendWork w, bool aligned) {
  constexpr bool F32 = std::is_same<T, float>::value;
  constexpr int QP = F32 ? 3 : 1, PP = F32 || ONCE ? 2 : 1, KP = DP / 64, W = DP / 16;
  constexpr bool AHEAD = DP <= 128 && (RB == 1 || !F32);   // (the others have no registers for it)
  constexpr bool TIGHT = F32 && DP > 128;   // places are worked out where they are used, which takes fewer registers
  constexpr bool SAVE = HELD > 0;
  constexpr int kBatch = 64, kPitch = HELD * kBatch + 1;
  static_assert(!SAVE || (16 / (SAVE ? HELD : 1)) * kPitch <= 16 * (DP + 4), "the blocks' weights lie where the waves' sums come later");
  __shared__ __attribute__((aligned(16))) float buf[kFinishBlocks<DP, WAVES>];
  __shared__ float parts[WAVES][16 * RB][2];   // (N, L) of the waves' rows, where huge
  const int lane = threadIdx.x & 63, l16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const AttendPlace p = attend_place(tab, view, w);
  if (p.b < 0) return;
  const Held& h = p.h;
  const int n = h.n, new0 = tab.cu_new[p.b], rows = h.fresh * w.gs, row0 = p.rc * 16 * RB;
  bf16x8 qf[RB][2 * KP][QP];
  int limit[RB];   // the first slot that the lane's row does not see
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = min(row0 + rb * 16 + l16, rows - 1), t = token_of(w, row), head = p.g * w.gs + row - t * w.gs;
    const T* q = (const T*)w.q + (int64_t)(new0 + t) * w.qst + (int64_t)head * w.qsh;
#pragma unroll
    for (int ks = 0; ks < 2 * KP; ++ks) load_query<T, QP>(qf[rb][ks], q, 64 * (ks / 2) + 16 * q4 + 8 * (ks & 1), c.d, aligned);
    limit[rb] = h.base + t + 1;
  }
  if (p.s0 >= p.s1 && (p.nc > 1 || w.x)) return;   // (the join reads no more chunks than have slots)
  const int edge = h.base + token_of(w, row0) + 1;   // from here on rows differ in what they see
  const int end = min(p.s1, h.base + token_of(w, min(row0 + 16 * RB - 1, rows - 1)) + 1);

  floatx4 O[W][RB];
  float M[RB], Z[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    M[rb] = kNothingSeen; Z[rb] = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) O[j][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const Cap cap(f, CAPPED ? kLog2e : 1.f);
  bool again = false;   // the blocks are to be taken with care
  bool tiny = false, large = false;
  bool huge = false;    // the references are in `parts`, and M is 0
  int odd = 0x7FFFFFFF;   // the first fresh slot behind the first one whose values are not all numbers

  const int lb = c.shift - 4, first = p.s0 / kBlock, last = end > p.s0 ? (end + kBlock - 1) / kBlock : first;
  const int share = ((last - first + 2 * WAVES - 1) / (2 * WAVES)) * 2;
  const int mine0 = first + wave * share, mine1 = min(last, mine0 + share);
  // A lane's block of the batch that is being fetched: place and scales
  float kf = 0.f, lv = 0.f, iv = 0.f;
  int64_t off = 0;
  uint64_t todo = 0;
  int next = mine0, base = mine0;
  // What a lane reads of a block.  In the place of components behind the last one it reads the first: queries have zeros there, and nobody
  // asks for those of the result.
  auto key_at = [&](int i, uint32_t part) __attribute__((always_inline)) { return (uint32_t)(l16 * c.st) + (64 * i + part < (uint32_t)c.d ? 64 * i + part : 0); };
  uint32_t k_at[KP], v_at[4];
#pragma unroll
  for (int i = 0; i < KP; ++i) k_at[i] = key_at(i, 16 * q4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v_at[i] = (uint32_t)((4 * q4 + i) * c.st) + (W * l16 < c.d ? W * l16 : 0);
  auto take_again = [&]() __attribute__((always_inline)) {   // (what the usual loop still does comes to nothing)
    again = true;
    todo = 0;
    next = mine1;
  };
  auto fetch = [&](Pair<DP>& x) __attribute__((always_inline)) {
    bool turned = false, live = false;   // to another batch; the lane's block is there
    float ks = 1.f, vs = 1.f;
    while (todo == 0 && next < mine1) {
      turned = true;
      base = next;
      next += kBatch;
      const int block = base + lane;
      const int page = block < mine1 ? c.pages[p.b * c.pst + (block >> lb)] : -1;
      live = (uint32_t)page < (uint32_t)c.n_pages;
      const int64_t at = (int64_t)(live ? page : 0) * c.G + p.g;
      ks = c.k_scale[at];
      vs = c.v_scale[at];
      off = (int64_t)page * c.sp + (int64_t)((block & ((1 << lb) - 1)) * kBlock) * c.st;
      todo = __ballot(live);
    }
    x.any = todo != 0;
    x.base = base;
    x.at[0] = x.any ? __builtin_ctzll(todo) : 0;
    todo &= todo - 1;
    x.two = todo != 0;
    x.at[1] = x.two ? __builtin_ctzll(todo) : x.at[0];
    todo &= todo - 1;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int at = x.at[kb];
      // The loads are made past the last block too, for the waits to count them: all lanes read the pool's first bytes, then.
      const bool there = kb ? x.two : x.any;
      const uint32_t lo = from_lane((uint32_t)off, at), hi = from_lane((uint32_t)((uint64_t)off >> 32), at), mask = there ? ~0u : 0u;
      const int64_t place = there ? (int64_t)((uint64_t)hi << 32 | lo) + p.g * c.sh : 0;
      const uint8_t *kp = c.k + place, *vp = c.v + place;
#pragma unroll
      for (int i = 0; i < KP; ++i) load_bytes<16, ONCE>(x.k[kb][i], kp + in_place((TIGHT ? key_at(i, in_place(16 * q4)) : k_at[i]) & mask));
#pragma unroll
      for (int i = 0; i < 4; ++i) load_bytes<W, ONCE>(x.v[kb][i], vp + in_place((TIGHT ? in_place(v_at[0]) + i * (uint32_t)c.st : v_at[i]) & mask));
    }
    if (turned) {   // (the scales come while the codes are on their way)
      kf = CAPPED ? ks : fmaxf(ks * f.c2, 0x1p-149f);   // (not 0, which makes NaN of what is masked)
      const float vc = fminf(fmaxf(vs, kLeastScale), kMostScale);
      lv = __builtin_amdgcn_logf(vc);
      iv = 1.f / vc;
      tiny |= __any(live && vc < kTinyScale);
      large |= __any(live && vc > kLargeScale);
      if (tiny && large && !again) take_again();
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      x.kf[kb] = lane_float(kf, x.at[kb]);
      x.lv[kb] = lane_float(lv, x.at[kb]);
      x.iv[kb] = lane_float(iv, x.at[kb]);
    }
  };
  // The blocks' weights, in LDS row by row, on their way to memory: a store among the loads holds up those behind it until it has reached
  // memory, so as many batches at once as there is room for (one at a time: a token over eight caches of 64K to 128K 288 us, four: 279).
  // They are held as the log2 of their sums; with CARE, since a large reference would take their bits, in units of it, and what leaves for rows whose
  // reference is no small number is kApart, the reference and they behind the others.  (So for all rows: 289 us.)
  const int some = min(16, rows - row0);
  float* held = buf + wave * (16 / (SAVE ? HELD : 1)) * kPitch;
  int held_base = mine0;
  auto put_held = [&](auto care) __attribute__((always_inline)) {
    float* to = w.x + (int64_t)(p.g * w.gs + row0) * w.xs + ((int64_t)p.b * c.max_pages << lb);
    const int until = min(mine1, held_base + HELD * kBatch);
    if constexpr (!decltype(care)::value) {
      for (int j = held_base + lane; j < until; j += kBatch)
        for (int r = 0; r < some; r += 4) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = held[(r + i) * kPitch + j - held_base];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (r + i < some) to[(r + i) * w.xs + j] = x[i];
        }
    } else {
      PagedUnit* pairs = reinterpret_cast<PagedUnit*>(w.x + w.H * w.xs) + (to - w.x);
      const float N = huge ? parts[wave][l16][0] : M[0], L = huge ? parts[wave][l16][1] : 0.f;
#pragma nounroll
      for (int r = 0; r < some; ++r) {
        const float n = lane_float(N, r), l = lane_float(L, r);
        const bool small = fabsf(n) < kSmallUnit;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
          const int j = held_base + i * kBatch + lane;
          if (j >= until) continue;
          const float x = held[r * kPitch + i * kBatch + lane] + l;
          to[r * w.xs + j] = small ? n + x : kApart;
          if (!small) pairs[r * w.xs + j] = PagedUnit{n, x};
        }
      }
    }
  };
  // ... in units of 2^-by (all that there is room for: what is not held yet may be anything)
  auto shift_held = [&](float by) __attribute__((always_inline)) {
#pragma nounroll
    for (int r = 0; r < some; ++r) {
      const float x = lane_float(by, r);
#pragma unroll
      for (int i = 0; i < HELD; ++i) held[r * kPitch + i * kBatch + lane] += x;
    }
  };
  // Where huge: scores made the exponents of their weights, (y - N) + (log2 s_v - L), the references first moved, by -step, where one would be too large.
  auto to_exponents = [&](floatx4 (&y)[2][RB], float (&f2)[2], float (&lv)[2], float (&step)[RB]) __attribute__((always_inline)) {
#pragma clang fp contract(off)   // (scores are rounded before anything is subtracted)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float N = parts[wave][rb * 16 + l16][0], L = parts[wave][rb * 16 + l16][1], top = -INFINITY, most = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        float best = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[kb][rb][e] = y[kb][rb][e] * f2[kb];
          best = fmaxf(best, y[kb][rb][e]);
        }
        top = fmaxf(top, best);
        most = fmaxf(most, (best - N) + (lv[kb] - L));
      }
      step[rb] = 0.f;
      if (__any(top - N > kTop || most > kTop)) {
        const float Nn = fmaxf(N, row_top(top));
        most = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) most = fmaxf(most, (y[kb][rb][e] - Nn) + lv[kb]);
        const float Ln = fmaxf(ceilf(L + (N - Nn)), ceilf(row_top(most)) - kFresh);   // (whole: a shift in the end)
        step[rb] = (N - Nn) + (L - Ln);
        parts[wave][rb * 16 + l16][0] = N = Nn;
        parts[wave][rb * 16 + l16][1] = L = Ln;
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[kb][rb][e] = (y[kb][rb][e] - N) + (lv[kb] - L);
    }
    f2[0] = f2[1] = 1.f;
    lv[0] = lv[1] = 0.f;
  };
  auto work = [&](Pair<DP>& x, auto care) __attribute__((always_inline)) {
    constexpr bool CARE = decltype(care)::value;
    const int s0[2] = {(x.base + x.at[0]) * kBlock, (x.base + x.at[1]) * kBlock};
    floatx4 y[2][RB];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) y[kb][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KP; ++i)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const bf16x8 k8 = eight_keys(x.k[kb][i][2 * half], x.k[kb][i][2 * half + 1]);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int part = QP - 1; part >= 0; --part)
              y[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, qf[rb][2 * i + half][part], y[kb][rb], 0, 0, 0);
        }
      if (CAPPED) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float z[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = y[kb][rb][e] * x.kf[kb];
          cap.apply(z);
          y[kb][rb] = floatx4{z[0], z[1], z[2], z[3]};
        }
      }
    }
    // (capped scores are in the log2 domain; the others are still to be multiplied)
    float f2[2] = {CAPPED ? 1.f : x.kf[0], CAPPED ? 1.f : x.kf[1]}, lv[2] = {x.lv[0], x.lv[1]};
    auto best = [&](int kb, int rb) __attribute__((always_inline)) {
      return fmaxf(fmaxf(y[kb][rb][0], y[kb][rb][1]), fmaxf(y[kb][rb][2], y[kb][rb][3]));
    };
    if (max(s0[0], s0[1]) + kBlock > edge || !x.two) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (s0[kb] + 4 * q4 + e >= limit[rb] || !(kb ? x.two : x.any)) y[kb][rb][e] = -INFINITY;
        // values of slots that are not in use count for nothing; what is not a number in fresh slots would reach rows that do not see them
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int s = s0[kb] + 4 * q4 + i;
#pragma unroll
          for (int j = 0; j < W / 4; ++j) {
            const uint32_t nan = ((x.v[kb][i][j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
            if (s >= n || !(kb ? x.two : x.any)) x.v[kb][i][j] = 0u;
            else if (s > h.base && nan) {
              odd = min(odd, s);
              x.v[kb][i][j] &= ~((nan >> 7) * 0xFFu);
            }
          }
        }
      }
    }
    bool high = CARE && huge;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        high |= fmaf(best(kb, rb), f2[kb], lv[kb] - M[rb]) > kTop;
    if (__any(high)) {
      float step[RB];   // of the references, downwards
      if (!CARE || !huge) {
        float Mn[RB];
        bool far = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const float top = row_top(fmaxf(fmaf(best(0, rb), f2[0], lv[0]), fmaf(best(1, rb), f2[1], lv[1])));
          Mn[rb] = fmaxf(M[rb], ceilf(top) - kFresh);
          far |= fabsf(Mn[rb]) >= (SAVE && !CARE ? kSmallUnit : kHuge) && Mn[rb] > kNothingSeen;
          step[rb] = M[rb] - Mn[rb];
        }
        far = __any(far);
        if (!CARE && far) take_again();
        if (CARE) huge = far;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          if (CARE && huge) {
            parts[wave][rb * 16 + l16][0] = M[rb];
            parts[wave][rb * 16 + l16][1] = 0.f;
          }
          M[rb] = CARE && huge ? 0.f : Mn[rb];
        }
      }
      if (CARE && huge) to_exponents(y, f2, lv, step);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float shrink = __builtin_amdgcn_exp2f(step[rb]), least = fmaxf(step[rb], -4096.f), whole = rintf(least);
        Z[rb] = ldexpf(CARE ? Z[rb] * __builtin_amdgcn_exp2f(least - whole) : Z[rb], (int)whole);   // (may be far above the weights, whose own shrinks to nothing)
#pragma unroll
        for (int j = 0; j < W; ++j) O[j][rb] *= shrink;
        if (SAVE && CARE) shift_held(step[rb]);
      }
    }
    if (SAVE && x.base - held_base >= HELD * kBatch) {
      put_held(care);
      held_base = x.base;
    }
    halfx8 weight[RB][PP];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float m = lv[kb] - M[rb];
        float z = 0.f;
        if (CARE) {
#pragma unroll
          for (int e = 0; e < 4; ++e) z += __builtin_amdgcn_exp2f(fmaf(y[kb][rb][e], f2[kb], m - x.lv[kb]));
        }
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const floatx2 pr = {__builtin_amdgcn_exp2f(fmaf(y[kb][rb][e], f2[kb], m)), __builtin_amdgcn_exp2f(fmaf(y[kb][rb][e + 1], f2[kb], m))};
          if (!CARE) z += pr[0] + pr[1];
          floatx2 rest = pr;
#pragma unroll
          for (int part = 0; part < PP; ++part) {
            const halfx2 r = __builtin_convertvector(rest, halfx2);
            weight[rb][part][kb * 4 + e] = r[0];
            weight[rb][part][kb * 4 + e + 1] = r[1];
            rest = floatx2{rest[0] - (float)r[0], rest[1] - (float)r[1]};
          }
        }
        Z[rb] = CARE ? Z[rb] + z : fmaf(z, x.iv[kb], Z[rb]);
        if (SAVE) {
          z = row_total(CARE ? z : z * x.iv[kb]);
          if (lane < some && (kb ? x.two : x.any)) held[l16 * kPitch + x.base - held_base + x.at[kb]] = __builtin_amdgcn_logf(z) + (CARE ? 0.f : M[0]);
        }
      }
#pragma unroll
    for (int j4 = 0; j4 < W / 4; ++j4) {
      four v[4];   // components 4 j4 .. +3 of the lane's: eight slots each
#pragma unroll
      for (int pair = 0; pair < 4; ++pair) {
        const uint32_t even = x.v[pair >> 1][2 * (pair & 1)][j4], uneven = x.v[pair >> 1][2 * (pair & 1) + 1][j4];
        const uint32_t lo = __builtin_amdgcn_perm(uneven, even, 0x05010400u), hi = __builtin_amdgcn_perm(uneven, even, 0x07030602u);
        v[0][pair] = half_pair(lo, false);
        v[1][pair] = half_pair(lo, true);
        v[2][pair] = half_pair(hi, false);
        v[3][pair] = half_pair(hi, true);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int part = PP - 1; part >= 0; --part)
            O[4 * j4 + j][rb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, v[j]), weight[rb][part], O[4 * j4 + j][rb], 0, 0, 0);
    }
  };
  // two pairs in turns: one at work while the other is on its way
  // (a pool without pages has no memory that the loads past the last block could read)
  const std::false_type usual;
  const std::true_type care;
  Pair<DP> a;
  a.any = false;
  if (c.n_pages > 0) fetch(a);
  if (a.any) {
    if constexpr (AHEAD) {
      Pair<DP> b;
      while (todo != 0 || next < mine1) {   // (one way out: a second one, between the halves, makes the waits for loads give up their counts)
        fetch(b);
        work(a, usual);
        fetch(a);
        if (b.any) work(b, usual);
      }
      if (a.any) work(a, usual);
    } else {
      do {
        work(a, usual);
        fetch(a);
      } while (a.any);
    }
    if (__builtin_expect(again, false)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        M[rb] = kNothingSeen; Z[rb] = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) O[j][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
      todo = 0;
      next = base = held_base = mine0;
      fetch(a);
      do {
        work(a, care);
        fetch(a);
      } while (a.any);
      if (SAVE) put_held(care);
    } else if (SAVE) {
      put_held(usual);
    }
  }
  // Fresh slots behind the first that all rows see were not looked at: a NaN among their values has left one in the sums, and then it is looked for.
  // (In each pair of blocks that holds some it would cost a sixth of a prompt's first chunk.)
  const int seen0 = max(h.base + 1, mine0 * kBlock), seen1 = min(edge, mine1 * kBlock);
  if (!SAVE && seen0 < seen1) {
    float sum = 0.f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int j = 0; j < W; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = fmaf(O[j][rb][e], 0.f, sum);
    if (__any(sum != sum))
      for (int block = seen0 / kBlock; block * kBlock < seen1; ++block) {
        const int page = c.pages[p.b * c.pst + (block >> lb)];
        if ((uint32_t)page >= (uint32_t)c.n_pages) continue;
        const uint8_t* vp = c.v + page * c.sp + p.g * c.sh + (int64_t)((block & ((1 << lb) - 1)) * kBlock) * c.st;
        for (int i = 0; i < 4; ++i) {
          uint32_t v[W / 4];
          load_bytes<W, false>(v, vp + (uint32_t)(v_at[0] + i * c.st));
          const int s = block * kBlock + 4 * q4 + i;
          for (int j = 0; j < W / 4; ++j)
            if ((((v[j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) && s >= seen0 && s < seen1) odd = min(odd, s);
        }
      }
  }
  if (__any(odd != 0x7FFFFFFF)) {
    for (int m = 32; m; m >>= 1) odd = min(odd, __shfl_xor(odd, m));
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int j = 0; j < W; ++j) O[j][rb] *= limit[rb] > odd ? NAN : 1.f;
  }
  finish_blocks<T, DP, RB, WAVES>(O, M, Z, huge ? parts[wave] : nullptr, buf, w, c.d, p.g, row0, rows, new0, p.nc);
}

}  // namespace

// Compiled in six parts, one object each with SKV_PAGED_PART = 0 .. 5 (in one they take minutes); part 0 also holds the dispatch.
template <class T, int DP>
hipError_t attend(const CacheTable& t, const CacheView& v, const PagedView& c, const ScoreForm& f, const PagedPlan& p, const AttendWork& w, hipStream_t st) {
  const bool aligned = (((uintptr_t)w.q | (uintptr_t)((w.qst | w.qsh) * (int64_t)sizeof(T))) & 15) == 0;
  with_cache_table(t, [&](const auto& tab) {
    using TAB = std::decay_t<decltype(tab)>;
    auto go = [&](auto rb, auto save, auto waves) {
      constexpr int RB = decltype(rb)::value, WAVES = decltype(waves)::value, HELD = decltype(save)::value;
      auto form = [&](auto capped, auto once) {
        paged_attend_kernel<TAB, T, DP, RB, decltype(capped)::value, HELD, decltype(once)::value, WAVES>
            <<<(unsigned)(p.units * c.G), 64 * WAVES, 0, st>>>(tab, v, c, f, w, aligned);
      };
      auto by_cap = [&](auto once) { f.softcap > 0.f ? form(std::true_type{}, once) : form(std::false_type{}, once); };
      p.stream ? by_cap(std::true_type{}) : by_cap(std::false_type{});
    };
    const std::integral_constant<int, kAttendWaves> four;
    const std::integral_constant<int, kShortWaves> more;
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 0> none;
    if (w.x && w.gs <= 4) go(one, four, four);
    else if (w.x) go(one, one, four);
    else if (p.rows == 16 && p.waves == kAttendWaves) go(one, none, four);
    else if (p.rows == 16) go(one, none, more);
    else if constexpr (DP <= 128 || sizeof(T) == 2) go(std::integral_constant<int, 2>{}, none, four);
  });
  return hipGetLastError();
}

#define SKV_PAGED_INST(T, DP) \
  template hipError_t attend<T, DP>(const CacheTable&, const CacheView&, const PagedView&, const ScoreForm&, const PagedPlan&, const AttendWork&, hipStream_t)
#if SKV_PAGED_PART == 0
SKV_PAGED_INST(uint16_t, 64);
extern SKV_PAGED_INST(uint16_t, 128);
extern SKV_PAGED_INST(uint16_t, 256);
extern SKV_PAGED_INST(float, 64);
extern SKV_PAGED_INST(float, 128);
extern SKV_PAGED_INST(float, 256);

template <class T>
hipError_t by_dim(const CacheTable& t, const CacheView& v, const PagedView& c, const ScoreForm& f, const PagedPlan& p, const AttendWork& w, hipStream_t st) {
  if (c.d <= 64) return attend<T, 64>(t, v, c, f, p, w, st);
  if (c.d <= 128) return attend<T, 128>(t, v, c, f, p, w, st);
  return attend<T, 256>(t, v, c, f, p, w, st);
}

hipError_t launch_paged_attend(const CacheTable& t, const CacheView& v, const PagedView& c, const ScoreForm& f, const PagedPlan& p,
                               const AttendWork& w, bool bf16, hipStream_t st) {
  return bf16 ? by_dim<uint16_t>(t, v, c, f, p, w, st) : by_dim<float>(t, v, c, f, p, w, st);
}
#elif SKV_PAGED_PART == 1
SKV_PAGED_INST(uint16_t, 128);
#elif SKV_PAGED_PART == 2
SKV_PAGED_INST(uint16_t, 256);
#elif SKV_PAGED_PART == 3
SKV_PAGED_INST(float, 64);
#elif SKV_PAGED_PART == 4
SKV_PAGED_INST(float, 128);
#else
SKV_PAGED_INST(float, 256);
#endif

}  // namespace skv
