// Attention of fresh tokens over a cache held in 8 bits, in pages.
//
// The split and the sums of cache_attend_bf16.hip: S^T = K Q^T, so that a lane has one query row and four slots of each block of 16, and
// O^T = V^T P^T takes the weights as they lie.  What is stored in 8 bits is exact in 16: keys enter their product as bf16 (queries too, those
// in fp32 as three parts), values theirs as fp16, where weights keep 11 bits (fp32 outputs: two parts, 22 bits).
// A block of 16 slots lies in one page, so its scales are the same for all lanes: a key's scale multiplies the block's scores; a value's is
// part of the weight, w = 2^(y + log2 s_v - M), with the row's reference M a whole number, so that nothing of it is rounded.
// Blocks come straight from memory to registers: a lane's 16 bytes of a key are operands as they lie, since the order of components in a
// product is free; of the values a lane reads 8 bytes of each of four rows and puts rows beside each other with byte permutes.
// The waves take shares of a chunk's blocks; a lane looks up one block's page, place and scales, and only blocks of pages that are there are
// in the list that a wave goes by, so dropped pages cost nothing.
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

template <int N> __device__ __forceinline__ void load_bytes(uint32_t (&to)[N / 4], const uint8_t* p) {
  typedef __attribute__((ext_vector_type(N / 4))) uint32_t vec;
  if constexpr (N == 4) {
    to[0] = *reinterpret_cast<const uint32_t*>(p);
  } else {
    const vec x = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) to[i] = x[i];
  }
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
        q[part][i] = (__bf16)rest;
        rest -= (float)q[part][i];
      }
    }
  }
}

// What the waves of a workgroup leave, added up in their order through LDS and written out by all threads (leave).  A lane holds components
// 4 W q4 + W e + j of its rows in O[j][rb][e].
template <class T, int DP, int RB>
__device__ __forceinline__ void finish_blocks(const floatx4 (&O)[DP / 16][RB], const float (&M)[RB], const float (&Zl)[RB], float* buf,
                                              const AttendWork& w, int d, int g, int row0, int rows, int new0, int nc) {
  constexpr int ROWS = 16 * RB, PITCH = DP + 4, W = DP / 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q4 = lane >> 4;
  float* ml = buf + kAttendWaves * ROWS * PITCH;   // [wave][row][2]
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float z = Zl[rb] + __shfl_xor(Zl[rb], 16);
    z += __shfl_xor(z, 32);
    if (q4 == 0) {
      ml[(wave * ROWS + rb * 16 + l16) * 2] = M[rb];
      ml[(wave * ROWS + rb * 16 + l16) * 2 + 1] = z;
    }
  }
  __syncthreads();
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = rb * 16 + l16;
    float top = ml[row * 2];
    for (int i = 1; i < kAttendWaves; ++i) top = fmaxf(top, ml[(i * ROWS + row) * 2]);
    const float f = __builtin_amdgcn_exp2f(M[rb] - top);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < W; j += 4)
        *reinterpret_cast<floatx4*>(buf + (wave * ROWS + row) * PITCH + W * (4 * q4 + e) + j) =
            floatx4{O[j][rb][e], O[j + 1][rb][e], O[j + 2][rb][e], O[j + 3][rb][e]} * f;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < ROWS * (DP / 4); e += 64 * kAttendWaves) {
    const int row = e / (DP / 4), c = e % (DP / 4) * 4;
    if (row0 + row >= rows || c >= d) continue;
    float top = ml[row * 2];
    for (int i = 1; i < kAttendWaves; ++i) top = fmaxf(top, ml[(i * ROWS + row) * 2]);
    float z = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < kAttendWaves; ++i) {
      z += ml[(i * ROWS + row) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(i * ROWS + row) * 2] - top);
      o += *reinterpret_cast<const floatx4*>(buf + (i * ROWS + row) * PITCH + c);
    }
    leave<T, DP>(w, d, g, row0 + row, c, top, z, o, new0, (int64_t)blockIdx.x * ROWS + row, nc);
  }
}

template <class TAB, class T, int DP, int RB, bool CAPPED, bool SAVE>
__global__ __launch_bounds__(64 * kAttendWaves, 2) void paged_attend_kernel(TAB tab, CacheView view, PagedView c, ScoreForm f, AttendWork w, bool aligned) {
  constexpr bool F32 = std::is_same<T, float>::value;
  constexpr int QP = F32 ? 3 : 1, PP = F32 ? 2 : 1, KP = DP / 64, W = DP / 16;
  __shared__ __attribute__((aligned(16))) float buf[kFinishFloats<DP, RB>];
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
  int odd = 0x7FFFFFFF;   // the first fresh slot behind the first one whose values are not all numbers

  const int lb = c.shift - 4, first = p.s0 / kBlock, last = end > p.s0 ? (end + kBlock - 1) / kBlock : first;
  const int share = ((last - first + 2 * kAttendWaves - 1) / (2 * kAttendWaves)) * 2;
  const int mine0 = first + wave * share, mine1 = min(last, mine0 + share);
  float* save = SAVE ? w.x + (int64_t)(p.g * w.gs + min(row0 + l16, rows - 1)) * w.xs + ((int64_t)p.b * c.max_pages << lb) : nullptr;
  for (int base = mine0; base < mine1; base += 64) {
    const int block = base + lane;
    const int page = block < mine1 ? c.pages[p.b * c.pst + (block >> lb)] : -1;
    const bool live = (uint32_t)page < (uint32_t)c.n_pages;
    const float ks = live ? c.k_scale[(int64_t)page * c.G + p.g] : 1.f, vs = live ? c.v_scale[(int64_t)page * c.G + p.g] : 1.f;
    const float kf = CAPPED ? ks : ks * f.c2;
    const float vc = fminf(fmaxf(vs, kLeastScale), kMostScale);
    const float lv = __builtin_amdgcn_logf(vc), iv = 1.f / vc;
    const int64_t off = (int64_t)page * c.sp + (int64_t)((block & ((1 << lb) - 1)) * kBlock) * c.st;
    uint64_t todo = __ballot(live);
    while (todo) {
      int at[2];
      at[0] = __builtin_ctzll(todo);
      todo &= todo - 1;
      const bool two = todo != 0;
      at[1] = two ? __builtin_ctzll(todo) : at[0];
      todo &= todo - 1;
      uint32_t kr[2][KP][4], vr[2][4][W / 4];
      float kb_f[2], lvb[2], ivb[2];
      int s0[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int64_t o = (int64_t)(((uint64_t)from_lane((uint32_t)((uint64_t)off >> 32), at[kb]) << 32) | from_lane((uint32_t)off, at[kb])) + p.g * c.sh;
        kb_f[kb] = lane_float(kf, at[kb]);
        lvb[kb] = lane_float(lv, at[kb]);
        ivb[kb] = lane_float(iv, at[kb]);
        s0[kb] = (base + at[kb]) * kBlock;
        const uint8_t *kp = c.k + o + l16 * c.st + 16 * q4, *vp = c.v + o + 4 * q4 * c.st + W * l16;
#pragma unroll
        for (int i = 0; i < KP; ++i) {
          if (64 * i + 16 * q4 < c.d) load_bytes<16>(kr[kb][i], kp + 64 * i);
          else kr[kb][i][0] = kr[kb][i][1] = kr[kb][i][2] = kr[kb][i][3] = 0u;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (W * l16 < c.d) load_bytes<W>(vr[kb][i], vp + i * c.st);
          else
#pragma unroll
            for (int j = 0; j < W / 4; ++j) vr[kb][i][j] = 0u;
        }
      }
      floatx4 x[2][RB];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) x[kb][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KP; ++i)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const bf16x8 k8 = eight_keys(kr[kb][i][2 * half], kr[kb][i][2 * half + 1]);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
              for (int part = QP - 1; part >= 0; --part)
                x[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, qf[rb][2 * i + half][part], x[kb][rb], 0, 0, 0);
          }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = x[kb][rb][e] * kb_f[kb];
          if (CAPPED) cap.apply(y);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[kb][rb][e] = y[e];
        }
      }
      if (max(s0[0], s0[1]) + kBlock > edge || !two) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (s0[kb] + 4 * q4 + e >= limit[rb] || (kb && !two)) x[kb][rb][e] = -INFINITY;
          // values of slots that are not in use count for nothing; what is not a number in fresh slots would reach rows that do not see them
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int s = s0[kb] + 4 * q4 + i;
#pragma unroll
            for (int j = 0; j < W / 4; ++j) {
              const uint32_t nan = ((vr[kb][i][j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
              if (s >= n) vr[kb][i][j] = 0u;
              else if (s > h.base && nan) {
                odd = min(odd, s);
                vr[kb][i][j] &= ~((nan >> 7) * 0xFFu);
              }
            }
          }
        }
      }
      bool high = false;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          high |= fmaxf(fmaxf(x[kb][rb][0], x[kb][rb][1]), fmaxf(x[kb][rb][2], x[kb][rb][3])) - (M[rb] - lvb[kb]) > kTop;
      if (__any(high)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float top = -INFINITY;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
            top = fmaxf(top, fmaxf(fmaxf(x[kb][rb][0], x[kb][rb][1]), fmaxf(x[kb][rb][2], x[kb][rb][3])) + lvb[kb]);
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float Mn = fmaxf(M[rb], ceilf(top) - kFresh), shrink = __builtin_amdgcn_exp2f(M[rb] - Mn);
          M[rb] = Mn;
          Z[rb] *= shrink;
#pragma unroll
          for (int j = 0; j < W; ++j) O[j][rb] *= shrink;
        }
      }
      halfx8 weight[RB][PP];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const float m = M[rb] - lvb[kb];
          float z = 0.f;
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const floatx2 pr = {__builtin_amdgcn_exp2f(x[kb][rb][e] - m), __builtin_amdgcn_exp2f(x[kb][rb][e + 1] - m)};
            z += pr[0] + pr[1];
            floatx2 rest = pr;
#pragma unroll
            for (int part = 0; part < PP; ++part) {
              const halfx2 r = __builtin_convertvector(rest, halfx2);
              weight[rb][part][kb * 4 + e] = r[0];
              weight[rb][part][kb * 4 + e + 1] = r[1];
              rest = floatx2{rest[0] - (float)r[0], rest[1] - (float)r[1]};
            }
          }
          Z[rb] = fmaf(z, ivb[kb], Z[rb]);
          if (SAVE) {
            z += __shfl_xor(z, 16);
            z += __shfl_xor(z, 32);
            if (q4 == 0 && row0 + l16 < rows && (kb == 0 || two)) save[base + at[kb]] = m + __builtin_amdgcn_logf(z);
          }
        }
#pragma unroll
      for (int j4 = 0; j4 < W / 4; ++j4) {
        four v[4];   // components 4 j4 .. +3 of the lane's: eight slots each
#pragma unroll
        for (int pair = 0; pair < 4; ++pair) {
          const uint32_t even = vr[pair >> 1][2 * (pair & 1)][j4], uneven = vr[pair >> 1][2 * (pair & 1) + 1][j4];
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
    }
  }
  if (__any(odd != 0x7FFFFFFF)) {
    for (int m = 32; m; m >>= 1) odd = min(odd, __shfl_xor(odd, m));
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int j = 0; j < W; ++j) O[j][rb] *= limit[rb] > odd ? NAN : 1.f;
  }
  finish_blocks<T, DP, RB>(O, M, Z, buf, w, c.d, p.g, row0, rows, new0, p.nc);
}

template <class T, int DP>
hipError_t attend(const CacheTable& t, const CacheView& v, const PagedView& c, const ScoreForm& f, const AttendPlan& p, const AttendWork& w, hipStream_t st) {
  const bool aligned = (((uintptr_t)w.q | (uintptr_t)((w.qst | w.qsh) * (int64_t)sizeof(T))) & 15) == 0;
  with_cache_table(t, [&](const auto& tab) {
    using TAB = std::decay_t<decltype(tab)>;
    const dim3 grid((unsigned)(p.units * c.G)), block(64 * kAttendWaves);
    auto go = [&](auto rb, auto save) {
      constexpr int RB = decltype(rb)::value;
      constexpr bool SAVE = decltype(save)::value;
      if (f.softcap > 0.f) paged_attend_kernel<TAB, T, DP, RB, true, SAVE><<<grid, block, 0, st>>>(tab, v, c, f, w, aligned);
      else paged_attend_kernel<TAB, T, DP, RB, false, SAVE><<<grid, block, 0, st>>>(tab, v, c, f, w, aligned);
    };
    if (w.x) go(std::integral_constant<int, 1>{}, std::true_type{});
    else if (p.rows == 16) go(std::integral_constant<int, 1>{}, std::false_type{});
    else go(std::integral_constant<int, 2>{}, std::false_type{});
  });
  return hipGetLastError();
}

template <class T>
hipError_t by_dim(const CacheTable& t, const CacheView& v, const PagedView& c, const ScoreForm& f, const AttendPlan& p, const AttendWork& w, hipStream_t st) {
  if (c.d <= 64) return attend<T, 64>(t, v, c, f, p, w, st);
  if (c.d <= 128) return attend<T, 128>(t, v, c, f, p, w, st);
  return attend<T, 256>(t, v, c, f, p, w, st);
}

}  // namespace

hipError_t launch_paged_attend(const CacheTable& t, const CacheView& v, const PagedView& c, const ScoreForm& f, const AttendPlan& p,
                               const AttendWork& w, bool bf16, hipStream_t st) {
  return bf16 ? by_dim<uint16_t>(t, v, c, f, p, w, st) : by_dim<float>(t, v, c, f, p, w, st);
}

}  // namespace skv
