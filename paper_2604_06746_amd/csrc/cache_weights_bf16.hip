// Weights of the accepted drafts over a bf16 cache of 64 or 128 components: mass[s] <- lambda mass[s] + sum over rows of 2^(x_s - lse).
//
// S = Q K^T in 16x16x32 matrix instructions: a lane has one slot and four rows of each block of 16, so a slot's sum over rows stays in the
// lane until its tile ends.  The rows are few (a path's tokens times the heads of a group) and are held as operands, 64 at a time;
// what binds is reading K once.  K's tiles go straight to LDS, two places a wave, one requested while the other is used.
// The four waves of a workgroup share a stretch of slots: by KV heads where one mass takes several (each wave's sums in LDS,
// added in wave order at the end), by tiles where there are fewer heads than waves.  No atomics: one order of sums.
#include "cache_bf16.h"

#include <algorithm>

namespace skv {
namespace {

constexpr int kRowBlocks = 4;   // 16-row blocks held at a time: a row a lane
constexpr int kRowBytes = 64 * (8 + 4 * 4);   // what a wave knows of them

template <class TAB, int D, int MODE, bool NT>
__global__ __launch_bounds__(256, 2) void cache_weights_bf16_kernel(TAB tab, CacheView c, ScoreForm f, AttendWork w,
                                                                    const int32_t* __restrict__ path,
                                                                    const int32_t* __restrict__ n_accept, int stretch, int head_waves) {
  constexpr int KS = D / 32, SEGS = D / 8, TILE = 32 * D * 2, NI = TILE / 1024;
  constexpr int POS = MODE == kBiased ? 256 : 0, NK = NI + (POS ? 1 : 0), SLOT = TILE + POS;
  typedef __attribute__((ext_vector_type(4))) int intx4;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];   // two places a wave, what it knows of its rows, [head_waves][stretch] sums
  const int lane = threadIdx.x & 63, l16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  int b = 0;
  while (b + 1 < tab.batch && (int)blockIdx.x >= tab.units[b + 1]) ++b;
  const Held h = held(tab, c, b);
  // the path, a token a lane, and its length are on their way while the sequence's is
  const int new0 = tab.cu_new[b], accepted = n_accept ? n_accept[b] : 0;
  const int step = path && lane < h.fresh ? max(0, min(path[new0 + lane], h.fresh - 1)) : lane;
  const int n = h.n, s0 = ((int)blockIdx.x - tab.units[b]) * stretch, s1 = min(n, s0 + stretch);
  if (h.fresh == 0 || h.base < 0 || s0 >= n) return;
  const int plane = blockIdx.y;
  const int taken = n_accept ? max(0, min(accepted, h.fresh)) : h.fresh, rows = taken * w.gs;
  uint8_t* ring = lds + wave * 2 * SLOT;
  uint8_t* about = lds + 4 * 2 * SLOT + wave * kRowBytes;
  uint64_t* row_sees = reinterpret_cast<uint64_t*>(about);
  float* row_norm = reinterpret_cast<float*>(about + 512);
  float* row_slope = row_norm + 64;
  int* row_at = reinterpret_cast<int*>(row_norm + 128);
  int* row_token = reinterpret_cast<int*>(row_norm + 192);
  const int32_t* pos = MODE == kBiased ? c.pos + (int64_t)plane * c.slots + h.lo : nullptr;
  // this wave's heads and tiles
  const int tile_waves = 4 / head_waves, hw = wave / tile_waves, tw = wave % tile_waves;
  float* all = reinterpret_cast<float*>(lds + 4 * (2 * SLOT + kRowBytes));
  float* sums = all + hw * stretch;
  for (int s = threadIdx.x; s < head_waves * stretch; s += 256) all[s] = 0.f;
  __syncthreads();
  const int g0 = c.planes > 1 ? plane : 0, g1 = c.planes > 1 ? plane + 1 : c.G;
  const int tiles = (s1 - s0 + 31) / 32, mine = tiles > tw ? (tiles - tw + tile_waves - 1) / tile_waves : 0;
  const Cap cap(f, MODE == kCapped ? kLog2e : 1.f);
  const int edge = f.tree || h.fresh > 1 ? h.base : n;   // from here on rows differ in what they see

  uint32_t off[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int unit = i * 64 + lane, s = unit / SEGS;
    off[i] = (uint32_t)(s * c.ss + ((unit % SEGS) ^ swizzle_k<SEGS>(s)) * 8) * 2u;
  }
  for (int g = g0 + hw; g < g1 && mine > 0; g += head_waves) {
    const uint16_t* kg = (const uint16_t*)c.k + (int64_t)g * c.sh + h.lo * c.ss;
    auto fetch = [&](int i) __attribute__((always_inline)) {
      const int j0 = s0 + 32 * (tw + tile_waves * i);
      uint8_t* to = ring + (i & 1) * SLOT;
      const uint8_t* base = (const uint8_t*)(kg + (int64_t)j0 * c.ss);
      if (j0 + 32 <= n) {
#pragma unroll
        for (int k = 0; k < NI; ++k) __builtin_amdgcn_global_load_lds((gbl_ptr_t)(base + off[k]), (lds_ptr_t)(to + k * 1024), 16, 0, NT ? 2 : 0);
      } else {   // rows past the end re-read the last one (their sums are not kept)
        const int last = n - 1 - j0;
#pragma unroll
        for (int k = 0; k < NI; ++k) {
          const int unit = k * 64 + lane, s = unit / SEGS;
          __builtin_amdgcn_global_load_lds((gbl_ptr_t)(base + (uint32_t)(min(s, last) * c.ss + ((unit % SEGS) ^ swizzle_k<SEGS>(s)) * 8) * 2u),
                                           (lds_ptr_t)(to + k * 1024), 16, 0, NT ? 2 : 0);
        }
      }
      if (POS) __builtin_amdgcn_global_load_lds((gbl_ptr_t)(pos + min(j0 + (lane & 31), n - 1)), (lds_ptr_t)(to + TILE), 4, 0, 0);
    };
    for (int row0 = 0; row0 < rows; row0 += 16 * kRowBlocks) {
      const int blocks = min(kRowBlocks, (rows - row0 + 15) / 16);
      fetch(0);
      if (mine > 1) fetch(1);
      // what the rows need to be known by, a lane a row (one without a norm has weights of zero, one whose norm is not a number has those), then the rows as operands
      {
        const int row = min(row0 + lane, rows - 1), i = token_of(w, row), head = g * w.gs + row - i * w.gs;
        const int t = __shfl(step, i);
        const float lse2 = w.lse[(int64_t)(new0 + t) * w.H + head] * 1.4426950408889634f;
        row_norm[lane] = row0 + lane < rows && lse2 != -INFINITY ? lse2 : INFINITY;
        if (MODE == kBiased) {
          row_slope[lane] = f.slopes[head];
          row_at[lane] = pos[h.base + t];
        }
        row_token[lane] = t;
        row_sees[lane] = row_mask(f, new0 + t, t);
      }
      wait_lds();
      bf16x8 qf[kRowBlocks][KS];
#pragma unroll
      for (int rb = 0; rb < kRowBlocks; ++rb) {
        const int row = min(row0 + rb * 16 + l16, rows - 1), i = token_of(w, row);
        const uint16_t* qrow = (const uint16_t*)w.q + (int64_t)(new0 + row_token[rb * 16 + l16]) * w.qst + (int64_t)(g * w.gs + row - i * w.gs) * w.qsh;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[rb][ks] = *reinterpret_cast<const bf16x8*>(qrow + ks * 32 + 8 * q4);
      }
#pragma unroll
      for (int rb = 0; rb < kRowBlocks; ++rb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[rb][ks]));
      for (int i = 0; i < mine; ++i) {
        const int j0 = s0 + 32 * (tw + tile_waves * i);
        if (i + 1 < mine) wait_loads<NK>(); else wait_loads<0>();
        const uint8_t* kt = ring + (i & 1) * SLOT;
        bf16x8 kf[2][KS];
        int from[2] = {0, 0};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const int s = kb * 16 + l16;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks)
            kf[kb][ks] = *reinterpret_cast<const bf16x8*>(kt + (s * SEGS + ((ks * 4 + q4) ^ swizzle_k<SEGS>(s))) * 16);
          if (POS) from[kb] = *reinterpret_cast<const int*>(kt + TILE + s * 4);
        }
        wait_lds();
        if (i + 2 < mine) fetch(i + 2);
        float sum[2] = {0.f, 0.f};
        const bool ragged = j0 + 32 > edge;
#pragma unroll
        for (int rb = 0; rb < kRowBlocks; ++rb) {
          if (rb >= blocks) break;
          const floatx4 norm = *reinterpret_cast<const floatx4*>(row_norm + rb * 16 + 4 * q4);
          floatx4 slope = {0.f, 0.f, 0.f, 0.f};
          intx4 at = {0, 0, 0, 0};
          if (MODE == kBiased) {
            slope = *reinterpret_cast<const floatx4*>(row_slope + rb * 16 + 4 * q4);
            at = *reinterpret_cast<const intx4*>(row_at + rb * 16 + 4 * q4);
          }
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[rb][ks], kf[kb][ks], x, 0, 0, 0);
            float y[4] = {x[0], x[1], x[2], x[3]};
            if (MODE == kCapped) cap.apply(y);
            else if (MODE == kBiased) scaled(f, cap, y);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float p;
              if (MODE == kPlain) p = __builtin_amdgcn_exp2f(fmaf(y[e], f.c2, -norm[e]));
              else if (MODE == kCapped) p = __builtin_amdgcn_exp2f(y[e] - norm[e]);
              else p = __builtin_amdgcn_exp2f(biased(y[e], slope[e], at[e] - from[kb]) - norm[e]);
              if (ragged) {   // (a slot that the row does not see may hold anything)
                const int s = j0 + kb * 16 + l16;
                if (s >= n || norm[e] == INFINITY || !sees(row_sees[rb * 16 + 4 * q4 + e], s, h.base)) p = 0.f;
              }
              sum[kb] += p;
            }
          }
        }
        // the four lanes of a slot, in any of them the same sum
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          sum[kb] += __shfl_xor(sum[kb], 16);
          sum[kb] += __shfl_xor(sum[kb], 32);
        }
        if (q4 < 2 && j0 + q4 * 16 + l16 < s1) sums[j0 - s0 + q4 * 16 + l16] += q4 ? sum[1] : sum[0];
      }
      wait_lds();
    }
  }
  __syncthreads();
  float* mass = c.mass + (int64_t)plane * c.slots + h.lo;
  for (int s = s0 + threadIdx.x; s < s1; s += 256) {
    const int i = s - s0;
    float sum = all[i];
    for (int h = 1; h < head_waves; ++h) sum += all[h * stretch + i];
    mass[s] = fmaf(w.lambda, mass[s], sum);
  }
}

template <int D>
hipError_t weights(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendWork& w, const int32_t* path,
                   const int32_t* n_accept, hipStream_t st) {
  // waves by heads: as many as there are heads for one mass
  const int heads = c.planes > 1 ? 1 : c.G, head_waves = heads >= 4 ? 4 : heads >= 2 ? 2 : 1;
  // slots of a workgroup: at least a tile for every wave; longer ones where that leaves 512 workgroups (twice the CUs), up to 512, or 1024 where the
  // waves share the tiles (eight caches of 8K to 16.5K slots, 8 planes: 46.4 -> 44.7 us; 1536 and 2048 slots 49)
  int64_t all = 0;
  for (int b = 0; b < t.batch; ++b) all += t.cu[b + 1] - t.cu[b];
  const int least = 32 * (4 / head_waves);
  const int64_t most = head_waves == 1 ? 1024 : 512;
  int stretch = (int)std::max<int64_t>(least, std::min<int64_t>(most, all * c.planes / 512 / 32 * 32));
  const bool stream = all * c.G * D * 2 >= kStreamBytes;
  CacheTable u = t;
  u.units[0] = 0;
  for (int b = 0; b < t.batch; ++b) u.units[b + 1] = u.units[b] + (int32_t)ceil_div(t.cu[b + 1] - t.cu[b], stretch);
  if (u.units[t.batch] == 0) return hipSuccess;
  with_cache_table(u, [&](const auto& tab) {
    with_mode(f, [&](auto mode) {
      constexpr int MODE = decltype(mode)::value;
      const size_t lds = 4 * (2 * (32 * D * 2 + (MODE == kBiased ? 256 : 0)) + kRowBytes) + sizeof(float) * head_waves * stretch;   // 80 KB at most
      using TAB = std::decay_t<decltype(tab)>;
      const dim3 grid((unsigned)u.units[t.batch], (unsigned)c.planes);
      if (stream) cache_weights_bf16_kernel<TAB, D, MODE, true><<<grid, 256, lds, st>>>(tab, c, f, w, path, n_accept, stretch, head_waves);
      else cache_weights_bf16_kernel<TAB, D, MODE, false><<<grid, 256, lds, st>>>(tab, c, f, w, path, n_accept, stretch, head_waves);
    });
  });
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_weights_bf16(const CacheTable& t, const CacheView& c, const ScoreForm& f, const AttendWork& w,
                                     const int32_t* path, const int32_t* n_accept, hipStream_t st) {
  return c.d == 128 ? weights<128>(t, c, f, w, path, n_accept, st) : weights<64>(t, c, f, w, path, n_accept, st);
}

}  // namespace skv
