// C-ABI entry points of rotary positions and of the cache held in 8 bits, in pages: argument checks, the cut of an attend call, workspace,
// launches.  As in api.cpp no device memory is allocated and nothing synchronises.
#include "paged.h"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace skv {
namespace {

constexpr int kMostHeads = 4096;
// scale log2(e) is multiplied by a page's scale (2^64 at most) before it meets a product
constexpr float kMostScoreScale = 0x1p62f;

int bytes_of(int dtype) { return dtype == STRUCTKV_DTYPE_BF16 ? 2 : 4; }

structkv_status check_dtype(int dtype) {
  if (dtype != STRUCTKV_DTYPE_F32 && dtype != STRUCTKV_DTYPE_BF16) return fail(STRUCTKV_ERR_UNSUPPORTED, "dtype %d is neither f32 (0) nor bf16 (1)", dtype);
  return STRUCTKV_OK;
}

structkv_status check_rotary(const structkv_rotary* r, int head_dim, bool inverse, RotaryView* v) {
  if (!r->turns || ((uintptr_t)r->turns & 7)) return fail(STRUCTKV_ERR_INVALID_ARG, "turns is NULL or not 8-byte aligned");
  if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_dim > head_dim)
    return fail(STRUCTKV_ERR_INVALID_ARG, "rot_dim must be even, 2 .. head_dim (%d), got %d", head_dim, r->rot_dim);
  if (r->interleaved != 0 && r->interleaved != 1) return fail(STRUCTKV_ERR_INVALID_ARG, "interleaved must be 0 or 1, got %d", r->interleaved);
  if (!std::isfinite(r->magnitude)) return fail(STRUCTKV_ERR_INVALID_ARG, "magnitude must be finite");
  *v = RotaryView{r->turns, r->rot_dim / 2, r->interleaved, r->magnitude, inverse ? -1.f : 1.f, head_dim};
  return STRUCTKV_OK;
}

// rows do not overlap: in the order of their strides, each lies behind all that the smaller ones reach
bool lie_apart(int64_t row, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2) {
  struct Dim { int64_t n, s; } dims[3] = {{n0, s0}, {n1, s1}, {n2, s2}};
  std::sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.s < b.s; });
  __int128 reach = row;
  for (const Dim& x : dims) {
    if (x.n <= 1) continue;
    if (x.s < reach) return false;
    reach += (__int128)x.s * (x.n - 1);
  }
  return true;
}

// t: capacities, in slots
structkv_status check_paged(const structkv_paged* c, CacheTable* t, PagedView* v) {
  if (!c) return fail(STRUCTKV_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_kv_heads < 1 || c->head_dim < 1) return fail(STRUCTKV_ERR_INVALID_ARG, "n_kv_heads and head_dim must be >= 1");
  if (c->n_kv_heads > kMostHeads) return fail(STRUCTKV_ERR_UNSUPPORTED, "n_kv_heads %d > %d", c->n_kv_heads, kMostHeads);
  if (c->head_dim > 256 || c->head_dim % 16) return fail(STRUCTKV_ERR_UNSUPPORTED, "head_dim must be a multiple of 16 up to 256, got %d", c->head_dim);
  const structkv_status st = check_dtype(c->dtype);
  if (st != STRUCTKV_OK) return st;
  int shift = 4;
  while (shift < 8 && (1 << shift) != c->page_size) ++shift;
  if ((1 << shift) != c->page_size) return fail(STRUCTKV_ERR_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256, got %d", c->page_size);
  if (c->n_pages < 0 || c->max_pages < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "n_pages or max_pages is negative");
  if ((int64_t)c->max_pages << shift >= ((int64_t)1 << 31) - 1024) return fail(STRUCTKV_ERR_UNSUPPORTED, "a capacity of 2^31 slots or more");
  if (c->batch < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "batch must be >= 0, got %d", c->batch);
  if (c->batch > kMaxBatch) return fail(STRUCTKV_ERR_UNSUPPORTED, "batch %d exceeds STRUCTKV_MAX_BATCH (%d)", c->batch, kMaxBatch);
  if (c->batch > 1 && c->pages_stride < c->max_pages) return fail(STRUCTKV_ERR_INVALID_ARG, "pages_stride (%lld) < max_pages", (long long)c->pages_stride);
  if (c->n_pages > 0) {
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return fail(STRUCTKV_ERR_INVALID_ARG, "k, v, k_scale or v_scale is NULL");
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return fail(STRUCTKV_ERR_INVALID_ARG, "k or v is not 16-byte aligned");
    if (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3) return fail(STRUCTKV_ERR_INVALID_ARG, "k_scale or v_scale is not 4-byte aligned");
    if ((c->stride_page | c->stride_head | c->stride_tok) % 16 || c->stride_page < 0 || c->stride_head < 0 || c->stride_tok < 0)
      return fail(STRUCTKV_ERR_INVALID_ARG, "strides must be multiples of 16, and not negative");
    if (c->stride_tok >= ((int64_t)1 << 26)) return fail(STRUCTKV_ERR_UNSUPPORTED, "stride_tok of 2^26 or more");
    if (!lie_apart(c->head_dim, c->n_pages, c->stride_page, c->n_kv_heads, c->stride_head, c->page_size, c->stride_tok))
      return fail(STRUCTKV_ERR_INVALID_ARG, "rows of the pool overlap");
  }
  if (c->batch > 0) {
    if (c->max_pages > 0 && (!c->pages || ((uintptr_t)c->pages & 3))) return fail(STRUCTKV_ERR_INVALID_ARG, "pages is NULL or not 4-byte aligned");
    if (!c->lens || ((uintptr_t)c->lens & 3)) return fail(STRUCTKV_ERR_INVALID_ARG, "lens is NULL or not 4-byte aligned");
  }
  if (((uintptr_t)c->mass | (uintptr_t)c->missed) & 3) return fail(STRUCTKV_ERR_INVALID_ARG, "mass or missed is not 4-byte aligned");
  memset(t, 0, sizeof(*t));
  t->batch = c->batch;
  for (int b = 0; b < c->batch; ++b) t->cu[b + 1] = (int64_t)(b + 1) * ((int64_t)c->max_pages << shift);
  *v = PagedView{(uint8_t*)c->k, (uint8_t*)c->v, c->k_scale, c->v_scale, c->stride_page, c->stride_head, c->stride_tok, c->pages,
                 c->pages_stride, c->lens, c->mass, c->missed, c->n_kv_heads, c->head_dim, shift, c->n_pages, c->max_pages, c->batch};
  return STRUCTKV_OK;
}

structkv_status check_fresh(const structkv_paged* c, const int64_t* cu_new, int64_t most, CacheTable* t) {
  if (!cu_new) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_new is NULL");
  if (cu_new[0] != 0) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_new[0] must be 0");
  for (int b = 0; b < c->batch; ++b) {
    const int64_t n = cu_new[b + 1] - cu_new[b];
    if (n < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_new decreases at %d", b);
    if (most && n > most)
      return fail(STRUCTKV_ERR_UNSUPPORTED, "sequence %d: %lld fresh tokens, at most STRUCTKV_MAX_CHUNK (%lld) are taken", b, (long long)n, (long long)most);
    if (cu_new[b + 1] >= ((int64_t)1 << 31)) return fail(STRUCTKV_ERR_UNSUPPORTED, "2^31 new tokens or more");
    t->cu_new[b + 1] = (int32_t)cu_new[b + 1];
  }
  return STRUCTKV_OK;
}

structkv_status check_query_heads(const structkv_paged* c, int32_t H) {
  if (H < 1 || H % c->n_kv_heads) return fail(STRUCTKV_ERR_INVALID_ARG, "n_kv_heads (%d) must divide n_q_heads (%d)", c->n_kv_heads, H);
  if (H > kMostHeads) return fail(STRUCTKV_ERR_UNSUPPORTED, "n_q_heads %d > %d", H, kMostHeads);
  return STRUCTKV_OK;
}

// Workgroups: two a CU, chunks of at least kLeast slots.  (Sixteen caches of 1K to 6.6K slots: 512 32.7 us, 768 33.0, 1024 35.2; four of 8K to 16.5K, 32 rows:
// 512 31 us, 1024 39.)
constexpr int64_t kUnits = 512, kLeast = 128;
// ... of 256 where a workgroup has 32 rows, whose partial results cost more to join: chains of 64 over 1000 slots 17.3 -> 14.2 us, of 13 over 4000
// 16.2 -> 13.7, of 13 over 1000 12.4 -> 13.4 (512: 14.4, 14.3 and 14.9).
constexpr int64_t kLeastRows = 256;
// Capacity from which on a block of rows is cut in two even where the blocks fill the chip.
constexpr int64_t kCut = 4096;
// ... while the rows, each of them a workgroup of 256 threads of the second launch, are no more than a launch takes.
constexpr int64_t kMostJoined = (int64_t)1 << 23;

// Capacity up to which a workgroup of kShortWaves takes all slots of a sequence where there would be chunks to join: a token over 256 slots 9.3 ->
// 6.5 us, over 512 9.3 -> 8.5, over 1031 9.7 -> 11.5.
constexpr int64_t kWhole = 512;

int64_t block_slots(const PagedView& v) { return ((int64_t)v.max_pages << v.shift) / kBlock; }

structkv_status plan_paged(const PagedView& v, int H, bool gather, bool bf16, CacheTable* t, PagedPlan* p) {
  const int64_t G = v.G, gs = H / v.G, cap = (int64_t)v.max_pages << v.shift;
  memset(p, 0, sizeof(*p));
  p->mfma = 1;
  p->gather = gather;
  int64_t most_rows = 0;
  for (int b = 0; b < v.batch; ++b) most_rows = std::max<int64_t>(most_rows, (int64_t)(t->cu_new[b + 1] - t->cu_new[b]) * gs);
  if (most_rows >= (1 << 18)) return fail(STRUCTKV_ERR_UNSUPPORTED, "%lld query rows of a KV head in one sequence, they must stay below 2^18", (long long)most_rows);
  p->rows = gather || most_rows <= 16 || (!bf16 && v.d > 128) ? 16 : 32;   // (32 rows of 256 components in fp32: no registers for it)
  const int64_t least = p->rows == 16 ? kLeast : kLeastRows;
  p->min_chunk = (int)least;
  // No other workgroup of the sequence reads the codes: past the caches (sixteen sequences of 32K slots 197 -> 181 us, 32 of 8K 107 -> 96; 64 of
  // 2K in turns with other calls 67 -> 61, the same ones again and again 43 -> 47).
  // Where sequences share a long prefix's pages, which only the table on the device knows, that costs what the caches would have kept (sixteen that
  // share 32K 105 -> 124, four that share 64K 60 -> 90, 32 that share 8K 61 -> 62), and they are still read faster than pages of their own.
  p->stream = most_rows <= p->rows;
  int64_t blocks = 0, chunks = 0;
  for (int b = 0; b < v.batch; ++b) {
    const int64_t rcs = ceil_div((int64_t)(t->cu_new[b + 1] - t->cu_new[b]) * gs, p->rows);
    blocks += rcs;
    chunks += rcs * std::max<int64_t>(1, ceil_div(cap, least));
    t->units[b + 1] = (int32_t)blocks;
  }
  const bool cut = p->rows == 16 && cap >= kCut && (int64_t)t->cu_new[v.batch] * H < kMostJoined;
  const bool whole = !gather && p->rows == 16 && cap <= kWhole && blocks < std::min(chunks, kUnits / G);
  p->waves = whole ? kShortWaves : kAttendWaves;
  p->units = whole ? blocks : std::max(blocks, std::min(chunks, std::max(kUnits / G, cut ? 2 * blocks : 0)));
  const int64_t gathers = gather ? v.batch * ceil_div(block_slots(v), 64) + (int64_t)t->cu_new[v.batch] * H : 0;
  p->join = gather || p->units > blocks;
  // (a launch takes fewer than 2^32 threads)
  if (p->units * G * 64 * p->waves >> 32 || gathers >> 31) return fail(STRUCTKV_ERR_UNSUPPORTED, "too many workgroups for one launch");
  const int64_t each = std::max<int64_t>(p->min_chunk, ceil_div(cap * blocks, std::max<int64_t>(1, p->units)));
  p->most_chunks = blocks > 0 ? ceil_div(cap, each) : 0;
  const int64_t part = p->join ? p->units * G * p->rows : 0;
  const int dp = v.d <= 64 ? 64 : v.d <= 128 ? 128 : 256;
  size_t off = 0;
  p->off_shares = off; off += p->join ? align_up(sizeof(int4) * (size_t)v.batch, 256) : 0;
  p->off_ml = off; off += align_up((size_t)part * 2 * sizeof(float), 256);
  p->off_o = off;  off += align_up((size_t)part * dp * sizeof(float), 256);
  p->off_x = off;  off += gather ? align_up((size_t)H * v.batch * block_slots(v) * 3 * sizeof(float), 256) : 0;
  p->total_bytes = off;
  return STRUCTKV_OK;
}

// ... at most, however new_tokens spread: the partial results are joined where there are kUnits of 32 rows, or twice as many blocks of 16
// as the rows make.
size_t most_paged_bytes(const PagedView& v, int H, int64_t new_tokens) {
  const int64_t gs = H / v.G, with_tokens = std::min<int64_t>(v.batch, new_tokens);
  const int dp = v.d <= 64 ? 64 : v.d <= 128 ? 128 : 256;
  const int64_t blocks16 = with_tokens * ceil_div(gs, 16) + new_tokens * gs / 16;
  const size_t part = (size_t)std::max<int64_t>(32 * kUnits, 2 * blocks16 * 16 * v.G);
  return align_up(sizeof(int4) * (size_t)v.batch, 256) + align_up(part * 2 * sizeof(float), 256) + align_up(part * dp * sizeof(float), 256) +
         (v.mass ? align_up((size_t)H * v.batch * block_slots(v) * 3 * sizeof(float), 256) : 0);
}

uint32_t gs_reciprocal(int gs) { return gs > 1 ? (uint32_t)(((uint64_t)1 << 32) / gs) + 1u : 0u; }

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" {

structkv_status structkv_rotary_turns(int32_t rot_dim, double base, int32_t scaling, double factor, double original, double low,
                                      double high, uint64_t* turns_out, float* magnitude_out) {
  clear_error();
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > 65536) return fail(STRUCTKV_ERR_INVALID_ARG, "rot_dim must be even, 2 .. 65536, got %d", rot_dim);
  if (!(base > 1.0) || !std::isfinite(base)) return fail(STRUCTKV_ERR_INVALID_ARG, "base must be finite and > 1");
  if (scaling < STRUCTKV_ROTARY_PLAIN || scaling > STRUCTKV_ROTARY_BANDS) return fail(STRUCTKV_ERR_INVALID_ARG, "scaling %d is none of the five", scaling);
  if (scaling != STRUCTKV_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return fail(STRUCTKV_ERR_INVALID_ARG, "factor must be finite and >= 1");
  if (scaling == STRUCTKV_ROTARY_NTK && rot_dim < 4) return fail(STRUCTKV_ERR_INVALID_ARG, "this scaling needs rot_dim >= 4");
  const bool bands = scaling == STRUCTKV_ROTARY_BANDS, yarn = scaling == STRUCTKV_ROTARY_YARN;
  if (bands || yarn) {
    if (!(original > 0.0) || !(low > 0.0) || !(high > 0.0) || !std::isfinite(original) || !std::isfinite(low) || !std::isfinite(high))
      return fail(STRUCTKV_ERR_INVALID_ARG, "original, low and high must be finite and > 0");
    if (bands ? !(low < high) : !(low > high)) return fail(STRUCTKV_ERR_INVALID_ARG, bands ? "low must be less than high" : "low must be more than high");
  }
  if (!turns_out || !magnitude_out) return fail(STRUCTKV_ERR_INVALID_ARG, "turns_out or magnitude_out is NULL");
  const long double two_pi = 6.283185307179586476925286766559005768L;
  if (scaling == STRUCTKV_ROTARY_NTK) base = (double)(base * powl(factor, (long double)rot_dim / (rot_dim - 2)));
  if (!std::isfinite(base)) return fail(STRUCTKV_ERR_INVALID_ARG, "the scaled base leaves the range of 64 bits");
  double lo = 0.0, hi = 0.0;
  if (yarn) {
    auto at = [&](double turns) { return rot_dim * std::log(original / (turns * 2.0 * M_PI)) / (2.0 * std::log(base)); };
    lo = std::max(0.0, std::floor(at(low)));
    hi = std::min(rot_dim - 1.0, std::ceil(at(high)));
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    long double f = powl((long double)base, -2.0L * i / rot_dim);
    if (scaling == STRUCTKV_ROTARY_LINEAR) f /= factor;
    if (yarn) {
      const long double ramp = std::min(1.0, std::max(0.0, (i - lo) / std::max(hi - lo, 1e-3)));
      f = f * (1.0L - ramp) + f / factor * ramp;
    }
    if (bands) {
      const long double smooth = std::min(1.0L, std::max(0.0L, (original * f / two_pi - low) / ((long double)high - low)));
      f = f * smooth + f / factor * (1.0L - smooth);
    }
    turns_out[i] = (uint64_t)(f / two_pi * 18446744073709551616.0L + 0.5L);   // (f is at most a radian)
  }
  *magnitude_out = yarn ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return STRUCTKV_OK;
}

structkv_status structkv_rotate(const structkv_rotary* rotary, const void* x, int64_t x_stride_tok, int64_t x_stride_head,
                                int64_t tokens, int32_t n_heads, int32_t head_dim, int32_t dtype, const int32_t* pos, int32_t inverse,
                                void* out, int64_t out_stride_tok, int64_t out_stride_head, void* stream) {
  clear_error();
  RotaryView r;
  if (!rotary) return fail(STRUCTKV_ERR_INVALID_ARG, "rotary is NULL");
  if (n_heads < 1 || head_dim < 1 || tokens < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "n_heads and head_dim must be >= 1, tokens >= 0");
  if (head_dim > 65536) return fail(STRUCTKV_ERR_UNSUPPORTED, "head_dim %d > 65536", head_dim);
  structkv_status st = check_dtype(dtype);
  if (st == STRUCTKV_OK) st = check_rotary(rotary, head_dim, inverse != 0, &r);
  if (st != STRUCTKV_OK) return st;
  if (inverse != 0 && inverse != 1) return fail(STRUCTKV_ERR_INVALID_ARG, "inverse must be 0 or 1, got %d", inverse);
  if (x_stride_tok < 0 || x_stride_head < 0 || out_stride_tok < 0 || out_stride_head < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "negative stride");
  if (tokens == 0) return STRUCTKV_OK;
  if (!x || !out || !pos) return fail(STRUCTKV_ERR_INVALID_ARG, "x, out or pos is NULL");
  const uintptr_t e = bytes_of(dtype);
  if (((uintptr_t)x | (uintptr_t)out) & (e - 1)) return fail(STRUCTKV_ERR_INVALID_ARG, "x or out is not aligned to its elements");
  if ((uintptr_t)pos & 3) return fail(STRUCTKV_ERR_INVALID_ARG, "pos is not 4-byte aligned");
  if (!lie_apart(head_dim, tokens, out_stride_tok, n_heads, out_stride_head, 1, 0)) return fail(STRUCTKV_ERR_INVALID_ARG, "rows of out overlap");
  if (x == out && ((x_stride_tok != out_stride_tok && tokens > 1) || (x_stride_head != out_stride_head && n_heads > 1)))
    return fail(STRUCTKV_ERR_INVALID_ARG, "out is x, but its strides are others");
  if (tokens >= ((int64_t)1 << 35) || n_heads > 65535) return fail(STRUCTKV_ERR_UNSUPPORTED, "2^35 rows or more, or more than 65535 heads");
  SKV_HIP_CHECK(launch_rotate(r, x, x_stride_tok, x_stride_head, tokens, n_heads, head_dim, dtype == STRUCTKV_DTYPE_BF16, pos, out,
                              out_stride_tok, out_stride_head, (hipStream_t)stream));
  return STRUCTKV_OK;
}

size_t structkv_paged_workspace_bytes(const structkv_paged* cache, int32_t n_q_heads, int64_t new_tokens) {
  CacheTable t;
  PagedView v;
  clear_error();
  if (check_paged(cache, &t, &v) != STRUCTKV_OK || check_query_heads(cache, n_q_heads) != STRUCTKV_OK) return 0;
  if (new_tokens < 0 || new_tokens > (int64_t)STRUCTKV_MAX_CHUNK * kMaxBatch) {
    fail(STRUCTKV_ERR_INVALID_ARG, "new_tokens (%lld) outside [0, STRUCTKV_MAX_CHUNK x STRUCTKV_MAX_BATCH]", (long long)new_tokens);
    return 0;
  }
  return std::max<size_t>(256, most_paged_bytes(v, n_q_heads, new_tokens));
}

structkv_status structkv_paged_append(const structkv_paged* cache, const void* k_new, const void* v_new, int64_t new_stride_head,
                                      int64_t new_stride_tok, const int64_t* cu_new, const structkv_rotary* rotary,
                                      const int32_t* pos_new, int32_t n_q_heads, const void* q, int64_t q_stride_tok,
                                      int64_t q_stride_head, void* q_out, int32_t* lens_out, void* stream) {
  clear_error();
  CacheTable t;
  PagedView v;
  structkv_status st = check_paged(cache, &t, &v);
  if (st == STRUCTKV_OK) st = check_fresh(cache, cu_new, 0, &t);
  RotaryView r = {nullptr, 0, 1, 1.f, 1.f, cache ? cache->head_dim : 0};
  if (st == STRUCTKV_OK && rotary) st = check_rotary(rotary, cache->head_dim, false, &r);
  if (st == STRUCTKV_OK && q) st = check_query_heads(cache, n_q_heads);
  if (st != STRUCTKV_OK) return st;
  if (q && !rotary) return fail(STRUCTKV_ERR_INVALID_ARG, "q is given to be rotated, but rotary is NULL");
  if (cache->batch == 0) return STRUCTKV_OK;
  if (!lens_out || ((uintptr_t)lens_out & 3)) return fail(STRUCTKV_ERR_INVALID_ARG, "lens_out is NULL or not 4-byte aligned");
  const uintptr_t a = (uintptr_t)cache->lens, z = (uintptr_t)lens_out, bytes = sizeof(int32_t) * (uintptr_t)cache->batch;
  if (a < z + bytes && z < a + bytes) return fail(STRUCTKV_ERR_INVALID_ARG, "lens_out must not be cache->lens: it is written while those are read");
  const int64_t total = t.cu_new[cache->batch], upr = cache->head_dim / kUnit;
  if (total > 0) {
    const uintptr_t e = bytes_of(cache->dtype);
    if (!k_new || !v_new) return fail(STRUCTKV_ERR_INVALID_ARG, "k_new or v_new is NULL");
    if (((uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)q | (uintptr_t)q_out) & (e - 1))
      return fail(STRUCTKV_ERR_INVALID_ARG, "k_new, v_new, q or q_out is not aligned to its elements");
    if (new_stride_head < 0 || new_stride_tok < 0 || q_stride_tok < 0 || q_stride_head < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "negative stride");
    if ((uintptr_t)pos_new & 3) return fail(STRUCTKV_ERR_INVALID_ARG, "pos_new is not 4-byte aligned");
    if (q && !q_out) return fail(STRUCTKV_ERR_INVALID_ARG, "q_out is NULL");
    int64_t most = 0;
    for (int b = 0; b < cache->batch; ++b) most = std::max<int64_t>(most, t.cu_new[b + 1] - t.cu_new[b]);
    const int64_t pages = (most + cache->page_size - 2) / cache->page_size + 1;
    // (numbers that fit what the launch counts them in, the queries' workgroups fewer than 2^24, unless a thread takes all heads of a token's unit)
    if ((q && total * upr >= ((int64_t)1 << 31) - ((int64_t)1 << 24)) ||
        ((int64_t)1 << 25) + (q ? total * upr / 64 : 0) + (int64_t)cache->batch * pages * 2 * cache->n_kv_heads >= ((int64_t)1 << 31))
      return fail(STRUCTKV_ERR_UNSUPPORTED, "too many rows for one launch");
  }
  const PagedRows w = {k_new, v_new, new_stride_head, new_stride_tok, pos_new, r, total > 0 ? q : nullptr, q_stride_tok, q_stride_head, q_out,
                       n_q_heads, lens_out};
  const hipError_t launched = launch_paged_append(t, v, w, cache->dtype == STRUCTKV_DTYPE_BF16, (hipStream_t)stream);
  if (launched == hipErrorInvalidConfiguration) return fail(STRUCTKV_ERR_UNSUPPORTED, "too many rows for one launch");
  SKV_HIP_CHECK(launched);
  return STRUCTKV_OK;
}

structkv_status structkv_paged_attend(const structkv_paged* cache, int32_t n_q_heads, float scale, float softcap, const void* q,
                                      int64_t q_stride_tok, int64_t q_stride_head, const int64_t* cu_new, float lambda, void* out,
                                      float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  CacheTable t;
  PagedView v;
  structkv_status st = check_paged(cache, &t, &v);
  if (st == STRUCTKV_OK) st = check_fresh(cache, cu_new, STRUCTKV_MAX_CHUNK, &t);
  if (st == STRUCTKV_OK) st = check_query_heads(cache, n_q_heads);
  if (st != STRUCTKV_OK) return st;
  if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(STRUCTKV_ERR_INVALID_ARG, "scale must be finite and >= 0 (0 = 1/sqrt(head_dim))");
  if (!(softcap >= 0.f) || !std::isfinite(softcap)) return fail(STRUCTKV_ERR_INVALID_ARG, "softcap must be finite and >= 0 (0 = none)");
  const float s = scale > 0.f ? scale : 1.0f / std::sqrt((float)cache->head_dim);
  if (softcap > 0.f && (!std::isfinite(1.f / softcap) || !std::isfinite(2.f * softcap) || !std::isfinite(s / softcap * 4.f) || !std::isnormal(s / softcap)))
    return fail(STRUCTKV_ERR_UNSUPPORTED, "softcap, 1 / softcap or scale / softcap leaves fp32's range");
  if (softcap == 0.f && !(s <= kMostScoreScale)) return fail(STRUCTKV_ERR_UNSUPPORTED, "a scale beyond 2^62 leaves fp32's range where a page's largest comes to it");
  if (!(lambda >= 0.f && lambda <= 1.f)) return fail(STRUCTKV_ERR_INVALID_ARG, "lambda must be in [0,1]");
  if (lambda > 0.f && !cache->mass) return fail(STRUCTKV_ERR_INVALID_ARG, "lambda > 0 needs the cache's mass");
  const uintptr_t e = bytes_of(cache->dtype);
  if ((uintptr_t)q & (e - 1)) return fail(STRUCTKV_ERR_INVALID_ARG, "q is not aligned to its elements");
  if (q_stride_tok < 0 || q_stride_head < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "negative stride of q");
  if (cache->batch == 0 || t.cu_new[cache->batch] == 0) return STRUCTKV_OK;
  if (!q || !out || !lse_out) return fail(STRUCTKV_ERR_INVALID_ARG, "q, out or lse_out is NULL");
  if (((uintptr_t)out & (e - 1)) || ((uintptr_t)lse_out & 3)) return fail(STRUCTKV_ERR_INVALID_ARG, "out or lse_out is not aligned to its elements");
  if (lambda > 0.f)
    for (int b = 0; b < cache->batch; ++b)
      if (t.cu_new[b + 1] - t.cu_new[b] > 1) return fail(STRUCTKV_ERR_INVALID_ARG, "sequence %d: lambda > 0 is for single tokens", b);
  PagedPlan p;
  st = plan_paged(v, n_q_heads, lambda > 0.f, cache->dtype == STRUCTKV_DTYPE_BF16, &t, &p);
  if (st != STRUCTKV_OK) return st;
  if (!workspace || ((uintptr_t)workspace & 255)) return fail(STRUCTKV_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
  if (workspace_bytes < p.total_bytes) return fail(STRUCTKV_ERR_WORKSPACE, "workspace has %zu bytes, this call needs %zu", workspace_bytes, p.total_bytes);
  uint8_t* w8 = (uint8_t*)workspace;
  const int gs = n_q_heads / cache->n_kv_heads;
  const ScoreForm f = {s, (float)((double)s * 1.4426950408889634), softcap, softcap > 0.f ? 1.f / softcap : 0.f, nullptr, nullptr};
  const CacheView view = {nullptr, nullptr, 0, 0, t.cu[cache->batch], nullptr, nullptr, cache->lens, cache->missed, cache->n_kv_heads, cache->head_dim, 1};
  const AttendWork w = {q, q_stride_tok, q_stride_head, out, lse_out, (float*)(w8 + p.off_ml), (float*)(w8 + p.off_o),
                        p.gather ? (float*)(w8 + p.off_x) : nullptr, p.join ? (int4*)(w8 + p.off_shares) : nullptr, n_q_heads, gs, p.min_chunk,
                        (int)p.units, gs_reciprocal(gs), lambda, (int64_t)t.cu_new[cache->batch] * n_q_heads, (int64_t)cache->batch * block_slots(v)};
  const bool bf16 = cache->dtype == STRUCTKV_DTYPE_BF16;
  SKV_HIP_CHECK(launch_paged_attend(t, view, v, f, p, w, bf16, (hipStream_t)stream));
  if (p.gather) SKV_HIP_CHECK(launch_paged_join(t, v, w, bf16, (hipStream_t)stream));
  else if (p.join) SKV_HIP_CHECK(launch_cache_combine(t, view, p, w, bf16, (hipStream_t)stream));
  return STRUCTKV_OK;
}

}  // extern "C"
