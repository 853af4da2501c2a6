// C-ABI entry points of the operators on a cache in use: argument checks, the cut of an attend call, workspace, launches.
// As in api.cpp no device memory is allocated and nothing synchronises.
#include "cache.h"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace skv {
namespace {

constexpr int kMaxHeads = 4096;

structkv_status check_cache(const structkv_cache* c, CacheTable* t, CacheView* v) {
  if (!c) return fail(STRUCTKV_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_kv_heads < 1 || c->head_dim < 1) return fail(STRUCTKV_ERR_INVALID_ARG, "n_kv_heads and head_dim must be >= 1");
  if (c->n_kv_heads > kMaxHeads) return fail(STRUCTKV_ERR_UNSUPPORTED, "n_kv_heads %d > %d", c->n_kv_heads, kMaxHeads);
  if (c->head_dim > 256) return fail(STRUCTKV_ERR_UNSUPPORTED, "head_dim %d > 256", c->head_dim);
  if (c->dtype != STRUCTKV_DTYPE_F32 && c->dtype != STRUCTKV_DTYPE_BF16)
    return fail(STRUCTKV_ERR_UNSUPPORTED, "dtype %d is neither f32 (0) nor bf16 (1)", c->dtype);
  if (c->planes != 1 && c->planes != c->n_kv_heads)
    return fail(STRUCTKV_ERR_INVALID_ARG, "planes must be 1 or n_kv_heads (%d), got %d", c->n_kv_heads, c->planes);
  if (c->batch < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "batch must be >= 0, got %d", c->batch);
  if (c->batch > kMaxBatch) return fail(STRUCTKV_ERR_UNSUPPORTED, "batch %d exceeds STRUCTKV_MAX_BATCH (%d)", c->batch, kMaxBatch);
  if (!c->cu_slots) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_slots is NULL");
  if (c->cu_slots[0] != 0) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_slots[0] must be 0");
  memset(t, 0, sizeof(*t));
  t->batch = c->batch;
  for (int b = 0; b < c->batch; ++b) {
    if (c->cu_slots[b + 1] < c->cu_slots[b]) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_slots decreases at %d", b);
    if (c->cu_slots[b + 1] - c->cu_slots[b] >= ((int64_t)1 << 31) - 1024)
      return fail(STRUCTKV_ERR_UNSUPPORTED, "sequence %d has a capacity of 2^31 slots or more", b);
    t->cu[b + 1] = c->cu_slots[b + 1];
  }
  const int64_t slots = t->cu[c->batch];
  if (slots > ((int64_t)1 << 40)) return fail(STRUCTKV_ERR_UNSUPPORTED, "more than 2^40 slots");
  if (c->stride_slot < c->head_dim) return fail(STRUCTKV_ERR_INVALID_ARG, "stride_slot (%lld) < head_dim", (long long)c->stride_slot);
  if (c->n_kv_heads > 1 && c->stride_head < c->head_dim)
    return fail(STRUCTKV_ERR_INVALID_ARG, "stride_head (%lld) < head_dim", (long long)c->stride_head);
  if (c->n_kv_heads > 1 && slots > 1 && c->stride_head < (slots - 1) * c->stride_slot + c->head_dim &&
      c->stride_slot < (c->n_kv_heads - 1) * c->stride_head + c->head_dim)
    return fail(STRUCTKV_ERR_INVALID_ARG, "rows of the cache overlap: neither the heads nor the slots lie apart");
  if (c->batch > 0 && (!c->lens || ((uintptr_t)c->lens & 3))) return fail(STRUCTKV_ERR_INVALID_ARG, "lens is NULL or not 4-byte aligned");
  if (slots > 0 && (!c->k || !c->v)) return fail(STRUCTKV_ERR_INVALID_ARG, "k or v is NULL");
  const uintptr_t esz = c->dtype == STRUCTKV_DTYPE_BF16 ? 2 : 4;
  if (((uintptr_t)c->k | (uintptr_t)c->v) & (esz - 1)) return fail(STRUCTKV_ERR_INVALID_ARG, "k or v is not aligned to its elements");
  if (((uintptr_t)c->mass | (uintptr_t)c->pos | (uintptr_t)c->missed) & 3)
    return fail(STRUCTKV_ERR_INVALID_ARG, "mass, pos or missed is not 4-byte aligned");
  *v = CacheView{c->k, c->v, c->n_kv_heads > 1 ? c->stride_head : 0, c->stride_slot, slots, c->mass, c->pos, c->lens, c->missed,
                 c->n_kv_heads, c->head_dim, c->planes};
  return STRUCTKV_OK;
}

int elem_bytes(const structkv_cache* c) { return c->dtype == STRUCTKV_DTYPE_BF16 ? 2 : 4; }

structkv_status check_new(const structkv_cache* c, const int64_t* cu_new, int64_t most, CacheTable* t) {
  if (!cu_new) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_new is NULL");
  if (cu_new[0] != 0) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_new[0] must be 0");
  for (int b = 0; b < c->batch; ++b) {
    const int64_t n = cu_new[b + 1] - cu_new[b];
    if (n < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "cu_new decreases at %d", b);
    if (most && n > most)
      return fail(STRUCTKV_ERR_UNSUPPORTED, "sequence %d: %lld fresh tokens, at most STRUCTKV_MAX_DRAFTS (%lld) are taken", b,
                  (long long)n, (long long)most);
    if (cu_new[b + 1] >= ((int64_t)1 << 31)) return fail(STRUCTKV_ERR_UNSUPPORTED, "2^31 new tokens or more");
    t->cu_new[b + 1] = (int32_t)cu_new[b + 1];
  }
  return STRUCTKV_OK;
}

structkv_status check_lens_out(const structkv_cache* c, const int32_t* lens_out) {
  if (!lens_out || ((uintptr_t)lens_out & 3)) return fail(STRUCTKV_ERR_INVALID_ARG, "lens_out is NULL or not 4-byte aligned");
  const uintptr_t a = (uintptr_t)c->lens, b = (uintptr_t)lens_out, n = sizeof(int32_t) * (uintptr_t)c->batch;
  if (a < b + n && b < a + n) return fail(STRUCTKV_ERR_INVALID_ARG, "lens_out must not be cache->lens: it is written while those are read");
  return STRUCTKV_OK;
}

structkv_status check_heads(const structkv_cache* c, int32_t H) {
  if (H < 1 || H % c->n_kv_heads)
    return fail(STRUCTKV_ERR_INVALID_ARG, "n_kv_heads (%d) must divide n_q_heads (%d)", c->n_kv_heads, H);
  if (H > kMaxHeads) return fail(STRUCTKV_ERR_UNSUPPORTED, "n_q_heads %d > %d", H, kMaxHeads);
  return STRUCTKV_OK;
}

// what attend and accept share: heads, form of the scores, queries
structkv_status check_scores(const structkv_cache* c, int32_t H, float scale, float softcap, const float* slopes, const void* q,
                             int64_t qst, int64_t qsh, const uint64_t* tree, float lambda, ScoreForm* f) {
  structkv_status st = check_heads(c, H);
  if (st != STRUCTKV_OK) return st;
  if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(STRUCTKV_ERR_INVALID_ARG, "scale must be finite and >= 0 (0 = 1/sqrt(head_dim))");
  if (!(softcap >= 0.f) || !std::isfinite(softcap)) return fail(STRUCTKV_ERR_INVALID_ARG, "softcap must be finite and >= 0 (0 = none)");
  const float s = scale > 0.f ? scale : 1.0f / std::sqrt((float)c->head_dim);
  // what the kernels work with (Cap): each by itself, since a product of a tiny and a huge one is no help to a score of zero
  if (softcap > 0.f && (!std::isfinite(1.f / softcap) || !std::isfinite(2.f * softcap) || !std::isfinite(s / softcap * 4.f) || !std::isnormal(s / softcap)))
    return fail(STRUCTKV_ERR_UNSUPPORTED, "softcap, 1 / softcap or scale / softcap leaves fp32's range");
  if (!(lambda >= 0.f && lambda <= 1.f)) return fail(STRUCTKV_ERR_INVALID_ARG, "lambda must be in [0,1]");
  if (lambda > 0.f && !c->mass) return fail(STRUCTKV_ERR_INVALID_ARG, "lambda > 0 needs the cache's mass");
  if (slopes && !c->pos) return fail(STRUCTKV_ERR_INVALID_ARG, "slopes need the cache's pos");
  if (((uintptr_t)slopes & 3) || ((uintptr_t)tree & 7)) return fail(STRUCTKV_ERR_INVALID_ARG, "slopes or tree_mask is misaligned");
  if ((uintptr_t)q & (uintptr_t)(elem_bytes(c) - 1)) return fail(STRUCTKV_ERR_INVALID_ARG, "q is not aligned to its elements");
  if (qst < 0 || qsh < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "negative stride of q");
  *f = ScoreForm{s, (float)((double)s * 1.4426950408889634), softcap, softcap > 0.f ? 1.f / softcap : 0.f, slopes, tree};
  return STRUCTKV_OK;
}

uint32_t reciprocal(int gs) { return gs > 1 ? (uint32_t)(((uint64_t)1 << 32) / gs) + 1u : 0u; }
int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

size_t score_bytes(int H, int64_t slots, int batch) { return align_up((size_t)H * (size_t)(slots + kScorePad * batch) * sizeof(float), 256); }

// what the bf16 matrix kernels take: whole 16-byte pieces, and a tile's rows within 32 bits
bool mfma_fits(const structkv_cache* c, const void* q, int64_t qst, int64_t qsh) {
  const int64_t strides = (c->n_kv_heads > 1 ? c->stride_head : 0) | c->stride_slot | qst | qsh;
  return c->dtype == STRUCTKV_DTYPE_BF16 && (c->head_dim == 64 || c->head_dim == 128) && strides % 8 == 0 &&
         (((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)q) & 15) == 0 && c->stride_slot < ((int64_t)1 << 25);
}

// Workgroups: two a CU (more or fewer, 256 to 4096, were slower), at least kLeastChunk slots each.
constexpr int64_t kAttendBlocks = 512, kLeastChunk = 128;
// Mean slots of a block of rows from which on it is cut in two even where the blocks fill the chip (plan_attend).
constexpr int64_t kCutSlots = 4096, kCutSlotsGathered = 1024;

structkv_status plan_attend(const structkv_cache* c, int H, bool gather, bool mfma, CacheTable* t, AttendPlan* p) {
  const int gs = H / c->n_kv_heads;
  memset(p, 0, sizeof(*p));
  p->mfma = mfma;
  p->gather = gather;
  int64_t most_rows = 0;
  for (int b = 0; b < c->batch; ++b) most_rows = std::max<int64_t>(most_rows, (int64_t)(t->cu_new[b + 1] - t->cu_new[b]) * gs);
  // 128 rows (32 a wave, the tiles shared) where there are more than two blocks of 32 and where enough chunks of them fill the chip: four trees
  // of 64 drafts over 16512 slots 118 us with, 131 without (one call behind the other); of 16 drafts (64 rows) 68 and 60, one of 64 over 2000
  // slots 25 and 20.  One tree makes the whole batch take them: beside 31 single tokens of 8K slots each one of 20 drafts 222 and 255, beside 15
  // one of 64 118 and 123, but beside 63 545 and 407 (a token's workgroup has one wave of four at work).
  int64_t wide_units = 0;
  for (int b = 0; b < c->batch; ++b)
    wide_units += ceil_div((int64_t)(t->cu_new[b + 1] - t->cu_new[b]) * gs, 128) * ceil_div(t->cu[b + 1] - t->cu[b], kLeastChunk);
  const bool wide = most_rows > 64 && wide_units >= kAttendBlocks / c->n_kv_heads;
  p->rows = !mfma || gather || most_rows <= 16 ? 16 : wide ? 128 : 32;
  p->min_chunk = kAttendWaves * (mfma ? 32 : 16);
  const int rows_wg = p->rows;
  p->stream = most_rows <= rows_wg && t->cu[c->batch] * c->n_kv_heads * c->head_dim * 2 * elem_bytes(c) >= kStreamBytes;
  // units: what fills the chip twice over the KV heads, no chunk below kLeastChunk slots in full sequences, a chunk at least of each
  int64_t blocks = 0, chunks = 0, stretches = 0;   // (of 64 slots, the fewest whose weights a workgroup of the join gathers)
  double work = 0;   // slots that the units of a KV head read in all
  for (int b = 0; b < c->batch; ++b) {
    const int64_t rcs = ceil_div((int64_t)(t->cu_new[b + 1] - t->cu_new[b]) * gs, rows_wg), cap = t->cu[b + 1] - t->cu[b];
    blocks += rcs;
    chunks += rcs * std::max<int64_t>(1, ceil_div(cap, kLeastChunk));
    work += (double)rcs * (double)cap;
    stretches += gather ? ceil_div(cap, 64) * c->planes : 0;
    t->units[b + 1] = (int32_t)blocks;
  }
  // Two a block of rows at least, so that long sequences of large batches are cut too, where that pays for the launch that joins them: 64
  // sequences of 8192 slots 309 us without, 320 with, one of 8192 among 63 of 400 88 and 34; with gathered weights, where the join is there
  // anyway, 64 of 2112 slots 113 and 114, one among short ones 41 and 25, but 64 of 300 27 and 31.
  const bool cut = rows_wg == 16 && work >= (double)(gather ? kCutSlotsGathered : kCutSlots) * (double)blocks;
  p->units = std::max(blocks, std::min(chunks, std::max(kAttendBlocks / c->n_kv_heads, cut ? 2 * blocks : 0)));
  if (p->units * c->n_kv_heads >= ((int64_t)1 << 31) || stretches >= ((int64_t)1 << 30))
    return fail(STRUCTKV_ERR_UNSUPPORTED, "too many workgroups for one launch");
  p->join = gather || p->units > blocks;
  const int64_t each = std::max<int64_t>(p->min_chunk, (int64_t)std::ceil(work / (double)std::max<int64_t>(1, p->units)));
  for (int b = 0; b < c->batch; ++b)
    if (t->cu_new[b + 1] > t->cu_new[b]) p->most_chunks = std::max(p->most_chunks, ceil_div(t->cu[b + 1] - t->cu[b], each));
  const int64_t part = p->units * c->n_kv_heads * rows_wg;
  const size_t parts = p->join ? (size_t)part : 0;
  size_t off = 0;
  p->off_shares = off; off += p->join ? align_up(sizeof(int4) * (size_t)c->batch, 256) : 0;
  p->off_ml = off; off += align_up(parts * 2 * sizeof(float), 256);
  p->off_o = off;  off += align_up(parts * padded_dim(c->head_dim) * sizeof(float), 256);
  p->off_x = off;  off += gather ? score_bytes(H, t->cu[c->batch], c->batch) : 0;
  p->total_bytes = off;
  return STRUCTKV_OK;
}

// ... at most, however new_tokens spread over the sequences.  Of plan_attend's units per KV head those that are joined are kAttendBlocks in all, or
// blocks of 16 rows: twice those where sequences are long enough to be cut, once where single tokens gather their weights.  A sequence's T gs rows
// are at most (T gs + 15) / 16 such blocks.
size_t most_attend_bytes(const structkv_cache* c, int H, int64_t new_tokens, int64_t slots) {
  const int64_t gs = H / c->n_kv_heads, G = c->n_kv_heads, with_tokens = std::min<int64_t>(c->batch, new_tokens);
  int64_t longest = 0;
  for (int b = 0; b < c->batch; ++b) longest = std::max(longest, c->cu_slots[b + 1] - c->cu_slots[b]);
  const bool wide = c->dtype == STRUCTKV_DTYPE_BF16 && (c->head_dim == 64 || c->head_dim == 128);
  const int64_t rows = std::min<int64_t>(new_tokens, STRUCTKV_MAX_DRAFTS) * gs, rows_wg = !wide || rows <= 16 ? 16 : rows <= 64 ? 32 : 128;
  const int64_t any = longest >= kCutSlots ? 2 * ((new_tokens * gs + 15 * with_tokens) / 16) : 0;
  const int64_t single = c->mass ? (longest >= kCutSlotsGathered ? 2 : 1) * with_tokens * ceil_div(gs, 16) : 0;
  const size_t parts = (size_t)std::max(rows_wg * kAttendBlocks, 16 * G * std::max(any, single));
  return align_up(sizeof(int4) * (size_t)c->batch, 256) + align_up(parts * 2 * sizeof(float), 256) + align_up(parts * padded_dim(c->head_dim) * sizeof(float), 256) +
         (c->mass ? score_bytes(H, slots, c->batch) : 0);
}

struct EvictSpace {
  size_t off_count, off_holes, off_moved, off_hist, off_tops, off_counts, total_bytes;
};
EvictSpace evict_space(const structkv_cache* c) {
  EvictSpace e;
  size_t off = 0, shares = 0;
  const size_t P = (size_t)c->planes, slots = (size_t)c->cu_slots[c->batch];
  int64_t longest = 0;
  for (int b = 0; b < c->batch; ++b) {
    const int64_t cap = c->cu_slots[b + 1] - c->cu_slots[b];
    longest = std::max(longest, cap);
    shares += (size_t)evict_shares(cap);
  }
  auto take = [&](size_t words) { const size_t at = off; off += align_up(words * 4, 256); return at; };
  e.off_count = take(P * c->batch);
  e.off_holes = take(P * slots);
  e.off_moved = take(P * slots);
  const bool digits = longest > kEvictShort;
  e.off_hist = take(digits ? P * c->batch * evict_hist_words() : 0);
  e.off_tops = take(digits ? P * shares : 0);
  e.off_counts = take(digits ? P * shares * 4 : 0);
  e.total_bytes = off;
  return e;
}

structkv_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!ws || ((uintptr_t)ws & 255)) return fail(STRUCTKV_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
  if (bytes < need) return fail(STRUCTKV_ERR_WORKSPACE, "workspace has %zu bytes, this call needs %zu", bytes, need);
  return STRUCTKV_OK;
}

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" {

size_t structkv_cache_workspace_bytes(const structkv_cache* cache, int32_t n_q_heads, int64_t new_tokens) {
  CacheTable t;
  CacheView v;
  clear_error();
  if (check_cache(cache, &t, &v) != STRUCTKV_OK || check_heads(cache, n_q_heads) != STRUCTKV_OK) return 0;
  if (new_tokens < 0 || new_tokens > (int64_t)STRUCTKV_MAX_DRAFTS * kMaxBatch) {
    fail(STRUCTKV_ERR_INVALID_ARG, "new_tokens (%lld) outside [0, STRUCTKV_MAX_DRAFTS x STRUCTKV_MAX_BATCH]", (long long)new_tokens);
    return 0;
  }
  return std::max<size_t>(256, std::max(most_attend_bytes(cache, n_q_heads, new_tokens, v.slots), evict_space(cache).total_bytes));
}

structkv_status structkv_cache_append(const structkv_cache* cache, const void* k_new, const void* v_new,
                                      int64_t new_stride_head, int64_t new_stride_tok, const int64_t* cu_new,
                                      const int32_t* pos_new, const float* mass_new, int64_t new_stride_plane,
                                      int32_t* lens_out, void* stream) {
  clear_error();
  CacheTable t;
  CacheView v;
  structkv_status st = check_cache(cache, &t, &v);
  if (st == STRUCTKV_OK) st = check_new(cache, cu_new, 0, &t);
  if (st != STRUCTKV_OK || cache->batch == 0) return st;
  st = check_lens_out(cache, lens_out);
  if (st != STRUCTKV_OK) return st;
  const int64_t total = t.cu_new[cache->batch];
  const int e = elem_bytes(cache);
  if (total > 0) {
    if (!k_new || !v_new) return fail(STRUCTKV_ERR_INVALID_ARG, "k_new or v_new is NULL");
    if (((uintptr_t)k_new | (uintptr_t)v_new) & (uintptr_t)(e - 1))
      return fail(STRUCTKV_ERR_INVALID_ARG, "k_new or v_new is not aligned to its elements");
    if (new_stride_head < 0 || new_stride_tok < 0 || new_stride_plane < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "negative stride");
    if ((pos_new == nullptr) != (cache->pos == nullptr))
      return fail(STRUCTKV_ERR_INVALID_ARG, "pos_new must be given where the cache keeps positions, and only there");
    if (mass_new && !cache->mass) return fail(STRUCTKV_ERR_INVALID_ARG, "mass_new given, but the cache keeps no mass");
    if (((uintptr_t)pos_new | (uintptr_t)mass_new) & 3) return fail(STRUCTKV_ERR_INVALID_ARG, "pos_new or mass_new is not 4-byte aligned");
    for (int b = 0; b < cache->batch; ++b)
      if ((int64_t)(t.cu_new[b + 1] - t.cu_new[b]) * cache->n_kv_heads * cache->head_dim * (int64_t)e >= ((int64_t)1 << 32) - 4096)
        return fail(STRUCTKV_ERR_UNSUPPORTED, "sequence %d: too many rows for one launch (rows*n_kv_heads*head_dim*element bytes must stay below 2^32)", b);
  }
  SKV_HIP_CHECK(launch_cache_append(t, v, k_new, v_new, new_stride_head, new_stride_tok, pos_new, mass_new, new_stride_plane, e,
                                    lens_out, (hipStream_t)stream));
  return STRUCTKV_OK;
}

structkv_status structkv_cache_attend(const structkv_cache* cache, int32_t n_q_heads, float scale, float softcap,
                                      const float* slopes, const void* q, int64_t q_stride_tok, int64_t q_stride_head,
                                      const int64_t* cu_new, const uint64_t* tree_mask, float lambda, void* out,
                                      float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  CacheTable t;
  CacheView v;
  ScoreForm f;
  structkv_status st = check_cache(cache, &t, &v);
  if (st == STRUCTKV_OK) st = check_new(cache, cu_new, STRUCTKV_MAX_DRAFTS, &t);
  if (st == STRUCTKV_OK) st = check_scores(cache, n_q_heads, scale, softcap, slopes, q, q_stride_tok, q_stride_head, tree_mask, lambda, &f);
  if (st != STRUCTKV_OK || cache->batch == 0 || t.cu_new[cache->batch] == 0) return st;
  if (!q || !out || !lse_out) return fail(STRUCTKV_ERR_INVALID_ARG, "q, out or lse_out is NULL");
  if (((uintptr_t)out & (uintptr_t)(elem_bytes(cache) - 1)) || ((uintptr_t)lse_out & 3))
    return fail(STRUCTKV_ERR_INVALID_ARG, "out or lse_out is not aligned to its elements");
  if (lambda > 0.f)
    for (int b = 0; b < cache->batch; ++b)
      if (t.cu_new[b + 1] - t.cu_new[b] > 1)
        return fail(STRUCTKV_ERR_INVALID_ARG, "sequence %d: lambda > 0 is for single tokens; drafts gather their weights in structkv_cache_accept", b);
  AttendPlan p;
  const bool bf16 = cache->dtype == STRUCTKV_DTYPE_BF16;
  st = plan_attend(cache, n_q_heads, lambda > 0.f, mfma_fits(cache, q, q_stride_tok, q_stride_head), &t, &p);
  if (st == STRUCTKV_OK) st = check_workspace(workspace, workspace_bytes, p.total_bytes);
  if (st != STRUCTKV_OK) return st;
  uint8_t* w8 = (uint8_t*)workspace;
  const int gs = n_q_heads / cache->n_kv_heads;
  const AttendWork w = {q, q_stride_tok, q_stride_head, out, lse_out, (float*)(w8 + p.off_ml), (float*)(w8 + p.off_o),
                        p.gather ? (float*)(w8 + p.off_x) : nullptr, p.join ? (int4*)(w8 + p.off_shares) : nullptr, n_q_heads, gs, p.min_chunk, (int)p.units, reciprocal(gs), lambda,
                        (int64_t)t.cu_new[cache->batch] * n_q_heads, v.slots + kScorePad * cache->batch};
  if (p.mfma && p.rows == 128) SKV_HIP_CHECK(launch_cache_attend_rows(t, v, f, p, w, (hipStream_t)stream));
  else if (p.mfma) SKV_HIP_CHECK(launch_cache_attend_bf16(t, v, f, p, w, (hipStream_t)stream));
  else SKV_HIP_CHECK(launch_cache_attend_f32(t, v, f, p, w, bf16, (hipStream_t)stream));
  if (p.join) SKV_HIP_CHECK(launch_cache_combine(t, v, p, w, bf16, (hipStream_t)stream));
  return STRUCTKV_OK;
}

structkv_status structkv_cache_accept(const structkv_cache* cache, int32_t n_q_heads, float scale, float softcap,
                                      const float* slopes, const void* q, int64_t q_stride_tok, int64_t q_stride_head,
                                      const float* lse, const int64_t* cu_new, const uint64_t* tree_mask,
                                      const int32_t* path, const int32_t* n_accept, float lambda, int32_t* lens_out,
                                      void* stream) {
  clear_error();
  CacheTable t;
  CacheView v;
  ScoreForm f;
  structkv_status st = check_cache(cache, &t, &v);
  if (st == STRUCTKV_OK) st = check_new(cache, cu_new, STRUCTKV_MAX_DRAFTS, &t);
  if (st == STRUCTKV_OK) st = check_scores(cache, n_q_heads, scale, softcap, slopes, q, q_stride_tok, q_stride_head, tree_mask, lambda, &f);
  if (st != STRUCTKV_OK || cache->batch == 0) return st;
  st = check_lens_out(cache, lens_out);
  if (st != STRUCTKV_OK) return st;
  if (((uintptr_t)lse | (uintptr_t)path | (uintptr_t)n_accept) & 3) return fail(STRUCTKV_ERR_INVALID_ARG, "lse, path or n_accept is not 4-byte aligned");
  const bool weigh = lambda > 0.f && t.cu_new[cache->batch] > 0;
  if (weigh && (!q || !lse)) return fail(STRUCTKV_ERR_INVALID_ARG, "lambda > 0 needs q and lse");
  if (weigh) {
    const AttendWork w = {q, q_stride_tok, q_stride_head, nullptr, const_cast<float*>(lse), nullptr, nullptr, nullptr, nullptr, n_q_heads,
                          n_q_heads / cache->n_kv_heads, 0, 0, reciprocal(n_q_heads / cache->n_kv_heads), lambda, 0, 0};
    if (mfma_fits(cache, q, q_stride_tok, q_stride_head)) SKV_HIP_CHECK(launch_cache_weights_bf16(t, v, f, w, path, n_accept, (hipStream_t)stream));
    else SKV_HIP_CHECK(launch_cache_weights_f32(t, v, f, w, path, n_accept, cache->dtype == STRUCTKV_DTYPE_BF16, (hipStream_t)stream));
  }
  SKV_HIP_CHECK(launch_cache_accept(t, v, path, n_accept, elem_bytes(cache), lens_out, (hipStream_t)stream));
  return STRUCTKV_OK;
}

structkv_status structkv_cache_evict(const structkv_cache* cache, const float* scores, const int64_t* budget,
                                     int32_t keep_tail, int32_t* lens_out, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  clear_error();
  CacheTable t;
  CacheView v;
  structkv_status st = check_cache(cache, &t, &v);
  if (st != STRUCTKV_OK || cache->batch == 0) return st;
  st = check_lens_out(cache, lens_out);
  if (st != STRUCTKV_OK) return st;
  if (!budget) return fail(STRUCTKV_ERR_INVALID_ARG, "budget is NULL");
  if (keep_tail < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "keep_tail < 0");
  if (keep_tail > 0 && !cache->pos) return fail(STRUCTKV_ERR_INVALID_ARG, "keep_tail > 0 needs the cache's pos");
  if (!scores) scores = cache->mass;
  if (v.slots > 0 && (!scores || ((uintptr_t)scores & 3)))
    return fail(STRUCTKV_ERR_INVALID_ARG, "scores is NULL (and the cache keeps no mass) or not 4-byte aligned");
  const int64_t units = (int64_t)cache->head_dim * elem_bytes(cache) / 2;
  for (int b = 0; b < cache->batch; ++b) {
    if (budget[b] < 0) return fail(STRUCTKV_ERR_INVALID_ARG, "budget[%d] < 0", b);
    const int64_t cap = t.cu[b + 1] - t.cu[b];
    t.units[b] = (int32_t)std::min(budget[b], cap);
    if (std::min(cap - t.units[b], (int64_t)t.units[b]) * units >= ((int64_t)1 << 31) - 4096)
      return fail(STRUCTKV_ERR_UNSUPPORTED, "too many rows may move for one launch (rows*head_dim*element bytes/2 must stay below 2^31)");
  }
  const EvictSpace e = evict_space(cache);
  st = check_workspace(workspace, workspace_bytes, e.total_bytes);
  if (st != STRUCTKV_OK) return st;
  uint8_t* w8 = (uint8_t*)workspace;
  const EvictWork w = {scores, keep_tail, lens_out, (int32_t*)(w8 + e.off_count), (int32_t*)(w8 + e.off_holes), (int32_t*)(w8 + e.off_moved),
                       (uint32_t*)(w8 + e.off_hist), (int32_t*)(w8 + e.off_tops), (uint32_t*)(w8 + e.off_counts)};
  SKV_HIP_CHECK(launch_cache_evict(t, v, w, elem_bytes(cache), (hipStream_t)stream));
  return STRUCTKV_OK;
}

}  // extern "C"
