// Rows of queries or keys turned by their positions, forwards or back.
// A pass over memory: x in, y out; the angles of a unit's pairs are formed once for the heads that a thread takes, and a unit is one piece of 16
// bytes (fp32: two pairs, bf16: four), or two pieces where halves are turned.  Keys of 131072 tokens (8 heads of 128, 0.54 GB) 92 us, 5.8 TB/s;
// fp32 rows of 8191 tokens (32 heads of 80, 20 turned) 38 us, 4.4 TB/s (in units of four pairs 46).
#include "rotary.h"

#include <algorithm>

namespace skv {
namespace {

// A thread of many heads has four on their way at once: queries of 32 heads, 45720 tokens, 158 -> 140 us (5.4 TB/s); of eight heads it costs
// (keys of 131072 tokens 92 -> 104 us), and in fp32 (8191 tokens of 32 heads of 80 components 38.2 -> 39.4).
constexpr int kManyHeads = 16;
constexpr int64_t kLaunchUnits = (int64_t)1 << 31;

// P: pairs of a unit.  ONCE: past the caches.  AT: heads that are on their way at once.
template <class T, bool VEC, bool ONCE, int P, int AT>
__global__ __launch_bounds__(256) void rotate_kernel(RotaryView r, const T* x, int64_t xst, int64_t xsh, uint32_t units, int heads, int upr, const int32_t* pos, T* out,
                                                     int64_t ost, int64_t osh, int per) {
  const uint32_t e = blockIdx.x * 256 + threadIdx.x;
  if (e >= units) return;
  const int64_t t = e / (uint32_t)upr;
  const int u = (int)(e - (uint32_t)t * upr), h0 = blockIdx.y * per, h1 = min(heads, h0 + per);
  const Spins<P> w = spin_unit<P>(r, u, pos[t]);
  turn_heads<T, VEC, ONCE, AT, P>(x + t * xst, xsh, out + t * ost, osh, h0, h1, u, r, w);
}

}  // namespace

hipError_t launch_rotate(const RotaryView& r, const void* x, int64_t xst, int64_t xsh, int64_t tokens, int heads, int d, bool bf16,
                         const int32_t* pos, void* out, int64_t ost, int64_t osh, hipStream_t st) {
  const int e = bf16 ? 2 : 4;
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)out | (uintptr_t)((xst | xsh | ost | osh) * e);
  auto go = [&](auto elem, auto v, auto once, auto pairs) {
    using T = decltype(elem);
    constexpr int P = decltype(pairs)::value;
    const int upr = (int)ceil_div(d, 2 * P);
    const int per = (int)std::min<int64_t>(heads, std::max<int64_t>(1, std::min(tokens * upr, kLaunchUnits) * heads / (1 << 18)));
    auto form = [&](auto at) {   // (a launch takes fewer than 2^32 threads)
      const int64_t most = kLaunchUnits / upr;
      for (int64_t t = 0; t < tokens; t += most) {
        const uint32_t units = (uint32_t)(std::min(most, tokens - t) * upr);
        rotate_kernel<T, decltype(v)::value, decltype(once)::value, P, decltype(at)::value>
            <<<dim3((unsigned)ceil_div((int64_t)units, 256), (unsigned)ceil_div(heads, per)), 256, 0, st>>>(r, (const T*)x + t * xst, xst, xsh, units, heads, upr, pos + t,
                                                                                                           (T*)out + t * ost, ost, osh, per);
      }
    };
    per >= kManyHeads && bf16 ? form(std::integral_constant<int, 4>{}) : form(std::integral_constant<int, 1>{});
  };
  const std::true_type yes; const std::false_type no;
  const std::integral_constant<int, 2> two; const std::integral_constant<int, 4> four;
  const bool once = kOnceBytes <= 2 * tokens * heads * d * e;
  auto by_once = [&](auto elem, auto pairs) { once ? go(elem, yes, yes, pairs) : go(elem, yes, no, pairs); };
  if (bf16) {
    if (bits % 16 || !whole_units(r)) go(uint16_t{}, no, no, four);
    else by_once(uint16_t{}, four);
  } else {
    if (bits % 16 || !whole_units(r)) go(float{}, no, no, four);
    else if (r.interleaved) by_once(float{}, two);
    else by_once(float{}, four);
  }
  return hipGetLastError();
}

}  // namespace skv
