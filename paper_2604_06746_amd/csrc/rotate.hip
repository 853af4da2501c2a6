// Rows of queries or keys turned by their positions, forwards or back.
// A pass over memory: x in, y out; the angles of a unit of eight components are formed once for the heads that a thread takes.
#include "rotary.h"

#include <algorithm>

namespace skv {
namespace {

template <class T, bool VEC>
__global__ __launch_bounds__(256) void rotate_kernel(RotaryView r, const T* x, int64_t xst, int64_t xsh, int64_t units, int heads, int upr, const int32_t* pos, T* out,
                                                     int64_t ost, int64_t osh, int per) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= units) return;
  const int64_t t = e / upr;
  const int u = (int)(e - t * upr), h0 = blockIdx.y * per, h1 = min(heads, h0 + per);
  const Spin w = spin_unit(r, u, pos[t]);
  const T* from = x + t * xst;
  T* to = out + t * ost;
  for (int h = h0; h < h1; ++h) {
    Unit v = load_unit<T, VEC>(from + h * xsh, u, r);
    turn(v, w, u, r);
    store_unit<T, VEC>(to + h * osh, u, r, v);
  }
}

}  // namespace

hipError_t launch_rotate(const RotaryView& r, const void* x, int64_t xst, int64_t xsh, int64_t tokens, int heads, int d, bool bf16,
                         const int32_t* pos, void* out, int64_t ost, int64_t osh, hipStream_t st) {
  const int e = bf16 ? 2 : 4, upr = (int)ceil_div(d, kUnit);
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)out | (uintptr_t)((xst | xsh | ost | osh) * e);
  const bool vec = bits % 16 == 0 && whole_units(r);
  const int64_t units = tokens * upr;
  const int per = (int)std::min<int64_t>(heads, std::max<int64_t>(1, units * heads / (1 << 18)));
  const dim3 grid((unsigned)ceil_div(units, 256), (unsigned)ceil_div(heads, per));
  auto go = [&](auto elem, auto v) {
    using T = decltype(elem);
    rotate_kernel<T, decltype(v)::value><<<grid, 256, 0, st>>>(r, (const T*)x, xst, xsh, units, heads, upr, pos, (T*)out, ost, osh, per);
  };
  if (bf16) vec ? go(uint16_t{}, std::true_type{}) : go(uint16_t{}, std::false_type{});
  else vec ? go(float{}, std::true_type{}) : go(float{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace skv
