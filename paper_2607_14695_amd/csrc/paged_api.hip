// C ABI of the backbone operators (declared in include/reflex.h): checks of
// the host-visible arguments, then one or two launches on the caller's stream.
// What lies in device memory (row offsets, lengths, page table) is checked by
// the kernels, entry by entry, where they use it.
#include <float.h>
#include <math.h>
#include <string.h>

#include "paged.h"

using namespace reflex;

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 27;
// sequences times K/V heads where a workgroup, or several, have one of each
constexpr int64_t kMaxLists = int64_t(1) << 18;

#define RFX_CHECK(expr)              \
  do {                               \
    const int rc_ = (expr);          \
    if (rc_ != REFLEX_OK) return rc_; \
  } while (0)

int check_dtype(int32_t dtype) {
  return dtype == REFLEX_DTYPE_F32 || dtype == REFLEX_DTYPE_BF16 ? REFLEX_OK : REFLEX_EINVAL;
}

int check_rows(const reflex_rows* r, int64_t n_rows, int32_t dtype) {
  if (!r) return REFLEX_EINVAL;
  if (n_rows == 0) return REFLEX_OK;
  const int64_t unit = dtype == REFLEX_DTYPE_BF16 ? 8 : 4;  // elements in 16 bytes
  if (!r->data || ((uintptr_t)r->data & 15) || r->row_stride % unit || r->head_stride % unit) return REFLEX_EINVAL;
  return REFLEX_OK;
}

int check_plan(const reflex_rotary* p) {
  if (!p || p->head_dim < 16 || p->head_dim > 2 * REFLEX_MAX_PAIRS || p->head_dim % 16) return REFLEX_EINVAL;
  if (p->n_axes < 1 || p->n_axes > REFLEX_MAX_AXES) return REFLEX_EINVAL;
  for (int i = 0; i < p->head_dim / 2; ++i)
    if (p->axis[i] >= p->n_axes) return REFLEX_EINVAL;
  return REFLEX_OK;
}

int check_cache(const reflex_paged_cache* c) {
  if (!c || !c->k || !c->v || ((uintptr_t)c->k & 15) || ((uintptr_t)c->v & 15)) return REFLEX_EINVAL;
  if (c->store < REFLEX_STORE_F32 || c->store > REFLEX_STORE_INT8) return REFLEX_EINVAL;
  if (c->store >= REFLEX_STORE_FP8 &&
      (!c->k_scale || !c->v_scale || ((uintptr_t)c->k_scale & 3) || ((uintptr_t)c->v_scale & 3)))
    return REFLEX_EINVAL;
  if (c->page_size < 1 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return REFLEX_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return REFLEX_EINVAL;
  if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535) return REFLEX_EINVAL;
  if ((double)c->n_pages * c->n_kv_heads * c->page_size >= 2147483648.0) return REFLEX_EINVAL;
  return REFLEX_OK;
}

int check_batch(const reflex_paged_batch* b, const reflex_paged_cache* c, int64_t n_rows) {
  if (!b || b->n_seqs < 0 || b->max_pages < 0 || b->max_length < 0) return REFLEX_EINVAL;
  if (n_rows < 0 || n_rows > kMaxRows) return REFLEX_EINVAL;
  if ((int64_t)b->max_pages * c->page_size > (int64_t(1) << 30)) return REFLEX_EINVAL;
  if (n_rows == 0) return REFLEX_OK;
  if (!b->cu_rows || (b->n_seqs > 0 && !b->lengths) || (b->n_seqs > 0 && b->max_pages > 0 && !b->page_table))
    return REFLEX_EINVAL;
  return REFLEX_OK;
}

int check_store(const reflex_paged_cache* c, int32_t dtype) {
  if (c->store == REFLEX_STORE_F32 && dtype != REFLEX_DTYPE_F32) return REFLEX_EDTYPE;
  if (c->store == REFLEX_STORE_BF16 && dtype != REFLEX_DTYPE_BF16) return REFLEX_EDTYPE;
  return REFLEX_OK;
}

Rows rows_of(const reflex_rows* r) { return Rows{reinterpret_cast<const char*>(r->data), r->row_stride, r->head_stride}; }

Pages pages_of(const reflex_paged_cache* c) {
  Pages p;
  p.k = reinterpret_cast<char*>(c->k);
  p.v = reinterpret_cast<char*>(c->v);
  p.k_scale = c->k_scale;
  p.v_scale = c->v_scale;
  p.n_pages = c->n_pages;
  p.shift = __builtin_ctz((unsigned)c->page_size);
  p.n_kv = c->n_kv_heads;
  p.dh = c->head_dim;
  return p;
}

Seqs seqs_of(const reflex_paged_batch* b) {
  return Seqs{b->cu_rows, b->lengths, b->page_table, b->n_seqs, b->max_pages};
}

int elem_bytes(const reflex_paged_cache* c) {
  return c->store == REFLEX_STORE_F32 ? 4 : c->store == REFLEX_STORE_BF16 ? 2 : 1;
}

// the length that the longest sequence is expected to have
int64_t expected_keys(const reflex_paged_cache* c, const reflex_paged_batch* b) {
  const int64_t cap = (int64_t)b->max_pages * c->page_size;
  return b->max_length > 0 && b->max_length < cap ? b->max_length : cap;
}

int check_lists(const reflex_paged_cache* c, const reflex_paged_batch* b) {
  return (int64_t)b->n_seqs * c->n_kv_heads <= kMaxLists ? REFLEX_OK : REFLEX_EINVAL;
}

int check_words(int32_t words) { return words >= 1 && words <= kMaxTreeWords ? REFLEX_OK : REFLEX_EINVAL; }

// In weighed attention the rows' maxima and sums lie behind the splits' partial
// results, and the scores behind these.
size_t whole_256(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

int check_attention(const reflex_rows* q, const reflex_rows* out, int64_t n_rows, int32_t dtype, float scale,
                    int32_t window, const void* workspace, size_t workspace_bytes, size_t need) {
  RFX_CHECK(check_rows(q, n_rows, dtype));
  RFX_CHECK(check_rows(out, n_rows, dtype));
  const double s2 = fabs((double)scale) * 1.4426950408889634;
  if (!(s2 <= (double)FLT_MAX) || window < 0) return REFLEX_EINVAL;
  if (need && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) return REFLEX_EINVAL;
  return REFLEX_OK;
}

void fill_attention(PagedAttnArgs& a, const reflex_paged_cache* cache, const reflex_paged_batch* batch,
                    const reflex_rows* q, const reflex_rows* out, int64_t n_rows, int32_t n_q_heads, int32_t dtype,
                    float scale, int32_t causal, int32_t window, int nsplit, void* workspace) {
  a.c = pages_of(cache);
  a.q = seqs_of(batch);
  a.x = rows_of(q);
  a.o = rows_of(out);
  a.n_rows = n_rows;
  a.n_q = n_q_heads;
  a.group = n_q_heads / cache->n_kv_heads;
  const double s2 = fabs((double)scale) * 1.4426950408889634, tiny = 0x1p-126;
  // (scaled up by 2^64 and then cut off at 2^-126 a score of 2^128 is 2^-62: 0)
  a.scale2 = (float)(s2 < tiny ? fmax(s2 * 0x1p64, tiny) : s2);
  a.factor = (scale < 0.f ? -1.f : 1.f) * (s2 < tiny ? 0x1p-64f : 1.f);
  a.causal = causal != 0;
  a.window = window;
  a.nsplit = nsplit;
  const size_t rows = (size_t)n_rows * n_q_heads * nsplit;
  a.part_o = reinterpret_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(reinterpret_cast<char*>(workspace) + rows * cache->head_dim * sizeof(float));
  a.tree = nullptr;
  a.tree_words = 0;
  a.units = 0;
  a.tile_rows = 0;
  a.stats = nullptr;
  a.scores = nullptr;
  a.score_pitch = 0;
  a.row_splits = 1;
  a.merge_with_sums = false;
}

int done(hipError_t e) { return e == hipSuccess ? REFLEX_OK : hip_fail(e); }

int accept_rows(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const int32_t* path, int32_t max_path,
                const int32_t* counts, float* weights, int32_t* lengths, void* stream) {
  RFX_CHECK(check_cache(cache));
  RFX_CHECK(check_batch(batch, cache, 1));
  RFX_CHECK(check_lists(cache, batch));
  if (max_path < 0) return REFLEX_EINVAL;
  if (batch->n_seqs == 0) return REFLEX_OK;
  if ((max_path > 0 && !path) || !counts || !lengths) return REFLEX_EINVAL;
  const PagedAcceptArgs a{pages_of(cache), seqs_of(batch), path, counts, max_path, weights, lengths};
  return done(launch_paged_accept(a, elem_bytes(cache), cache->store >= REFLEX_STORE_FP8, reinterpret_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int reflex_rotary_init(reflex_rotary* plan, int32_t head_dim, int32_t n_axes, const int32_t* sections, double theta,
                       int32_t ladder) {
  if (!plan || !sections || head_dim < 16 || head_dim > 2 * REFLEX_MAX_PAIRS || head_dim % 16) return REFLEX_EINVAL;
  if (n_axes < 1 || n_axes > REFLEX_MAX_AXES || !(theta > 0.0) || !isfinite(theta)) return REFLEX_EINVAL;
  if (ladder != REFLEX_LADDER_SHARED && ladder != REFLEX_LADDER_PER_AXIS) return REFLEX_EINVAL;
  const int half = head_dim / 2;
  int left = half;
  for (int a = 0; a < n_axes; ++a) {
    if (sections[a] < 0 || sections[a] > left) return REFLEX_EINVAL;
    left -= sections[a];
  }
  if (left != 0) return REFLEX_EINVAL;
  memset(plan, 0, sizeof(*plan));
  plan->head_dim = head_dim;
  plan->n_axes = n_axes;
  const double two_pi = 6.283185307179586476925;
  int i = 0;
  for (int a = 0; a < n_axes; ++a)
    for (int j = 0; j < sections[a]; ++j, ++i) {
      const double e = ladder == REFLEX_LADDER_SHARED ? (double)i / half : (double)j / sections[a];
      plan->axis[i] = (uint8_t)a;
      plan->turns[i] = pow(theta, -e) / two_pi;
    }
  return REFLEX_OK;
}

int reflex_rotary_apply(const reflex_rotary* plan, const int64_t* positions, int64_t pos_stride, const reflex_rows* x,
                        const reflex_rows* y, int64_t n_rows, int32_t n_heads, int32_t dtype, int32_t inverse,
                        void* stream) {
  RFX_CHECK(check_plan(plan));
  RFX_CHECK(check_dtype(dtype));
  if (n_rows < 0 || n_rows > kMaxRows || n_heads < 1 || n_heads > 65535) return REFLEX_EINVAL;
  RFX_CHECK(check_rows(x, n_rows, dtype));
  RFX_CHECK(check_rows(y, n_rows, dtype));
  if (n_rows == 0) return REFLEX_OK;
  if (!positions) return REFLEX_EINVAL;
  RotaryArgs a;
  a.pos = positions;
  a.ps = pos_stride;
  a.x = rows_of(x);
  a.y = rows_of(y);
  a.n_rows = n_rows;
  a.n_heads = n_heads;
  a.heads_per = n_heads;
  a.inverse = inverse != 0;
  a.plan = *plan;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(dtype == REFLEX_DTYPE_BF16 ? launch_rotary<bf16_t>(a, s) : launch_rotary<float>(a, s));
}

int reflex_paged_write(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const reflex_rows* k,
                       const reflex_rows* v, int64_t n_rows, int32_t dtype, const reflex_rotary* rotary,
                       const int64_t* positions, int64_t pos_stride, void* stream) {
  RFX_CHECK(check_cache(cache));
  RFX_CHECK(check_dtype(dtype));
  RFX_CHECK(check_batch(batch, cache, n_rows));
  RFX_CHECK(check_rows(k, n_rows, dtype));
  RFX_CHECK(check_rows(v, n_rows, dtype));
  if (rotary) {
    RFX_CHECK(check_plan(rotary));
    if (rotary->head_dim != cache->head_dim) return REFLEX_EINVAL;
  } else if (positions) {
    return REFLEX_EINVAL;
  }
  RFX_CHECK(check_store(cache, dtype));
  if (n_rows == 0 || batch->n_seqs == 0) return REFLEX_OK;
  PagedWriteArgs a;
  a.c = pages_of(cache);
  a.q = seqs_of(batch);
  a.k = rows_of(k);
  a.v = rows_of(v);
  a.n_rows = n_rows;
  a.heads_per = cache->n_kv_heads;
  a.rotate = rotary != nullptr;
  a.pos = positions;
  a.ps = pos_stride;
  if (rotary)
    a.plan = *rotary;
  else
    memset(&a.plan, 0, sizeof(a.plan));
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(dtype == REFLEX_DTYPE_BF16 ? launch_paged_write<bf16_t>(a, cache->store, s)
                                         : launch_paged_write<float>(a, cache->store, s));
}

int reflex_paged_read(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const reflex_rows* k,
                      const reflex_rows* v, int64_t n_rows, int32_t dtype, void* stream) {
  RFX_CHECK(check_cache(cache));
  RFX_CHECK(check_dtype(dtype));
  RFX_CHECK(check_batch(batch, cache, n_rows));
  RFX_CHECK(check_rows(k, n_rows, dtype));
  RFX_CHECK(check_rows(v, n_rows, dtype));
  RFX_CHECK(check_store(cache, dtype));
  if (n_rows == 0 || batch->n_seqs == 0) return REFLEX_OK;
  PagedReadArgs a;
  a.c = pages_of(cache);
  a.q = seqs_of(batch);
  a.k = rows_of(k);
  a.v = rows_of(v);
  a.n_rows = n_rows;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(dtype == REFLEX_DTYPE_BF16 ? launch_paged_read<bf16_t>(a, cache->store, s)
                                         : launch_paged_read<float>(a, cache->store, s));
}

int reflex_paged_attention_workspace(const reflex_paged_cache* cache, const reflex_paged_batch* batch, int64_t n_rows,
                                     int32_t n_q_heads, int32_t dtype, size_t* bytes) {
  if (!bytes) return REFLEX_EINVAL;
  RFX_CHECK(check_cache(cache));
  RFX_CHECK(check_dtype(dtype));
  RFX_CHECK(check_batch(batch, cache, n_rows));
  RFX_CHECK(check_store(cache, dtype));
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads || n_rows * (int64_t)n_q_heads > (int64_t(1) << 23))
    return REFLEX_EINVAL;
  *bytes = n_rows == 0 || batch->n_seqs == 0 ? 0 : paged_attention_plan(*cache, *batch, n_rows, n_q_heads, dtype, 0).bytes;
  return REFLEX_OK;
}

int reflex_paged_attention(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const reflex_rows* q,
                           const reflex_rows* out, int64_t n_rows, int32_t n_q_heads, int32_t dtype, float scale,
                           int32_t causal, int32_t window, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  RFX_CHECK(reflex_paged_attention_workspace(cache, batch, n_rows, n_q_heads, dtype, &need));
  PagedAttnArgs a;
  RFX_CHECK(check_attention(q, out, n_rows, dtype, scale, window, workspace, workspace_bytes, need));
  if (n_rows == 0 || batch->n_seqs == 0) return REFLEX_OK;
  fill_attention(a, cache, batch, q, out, n_rows, n_q_heads, dtype, scale, causal, window,
                 paged_attention_plan(*cache, *batch, n_rows, n_q_heads, dtype, window).nsplit, workspace);
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(dtype == REFLEX_DTYPE_BF16 ? launch_paged_attention<bf16_t>(a, cache->store, s)
                                         : launch_paged_attention<float>(a, cache->store, s));
}

int reflex_paged_tree(const reflex_paged_batch* batch, const int32_t* parents, int64_t n_rows, uint64_t* mask,
                      int32_t mask_words, int64_t* positions, void* stream) {
  if (!batch || batch->n_seqs < 0 || batch->n_seqs > kMaxLists || n_rows < 0 || n_rows > kMaxRows) return REFLEX_EINVAL;
  RFX_CHECK(check_words(mask_words));
  if (n_rows == 0 || batch->n_seqs == 0) return REFLEX_OK;
  if (!batch->cu_rows || !batch->lengths || !parents || !mask || ((uintptr_t)mask & 7) || ((uintptr_t)positions & 7))
    return REFLEX_EINVAL;
  const PagedTreeArgs a{seqs_of(batch), parents, n_rows, mask_words, mask, positions};
  return done(launch_paged_tree(a, reinterpret_cast<hipStream_t>(stream)));
}

int reflex_paged_tree_attention_workspace(const reflex_paged_cache* cache, const reflex_paged_batch* batch,
                                          int64_t n_rows, int32_t n_q_heads, int32_t dtype, size_t* bytes) {
  RFX_CHECK(reflex_paged_attention_workspace(cache, batch, n_rows, n_q_heads, dtype, bytes));
  if (n_rows > 0 && batch->n_seqs > 0) *bytes = paged_tree_plan(*cache, *batch, n_rows, n_q_heads, dtype).bytes;
  return REFLEX_OK;
}

int reflex_paged_tree_attention(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const reflex_rows* q,
                                const reflex_rows* out, int64_t n_rows, int32_t n_q_heads, int32_t dtype, float scale,
                                const uint64_t* mask, int32_t mask_words, void* workspace, size_t workspace_bytes,
                                void* stream) {
  size_t need = 0;
  RFX_CHECK(reflex_paged_tree_attention_workspace(cache, batch, n_rows, n_q_heads, dtype, &need));
  RFX_CHECK(check_words(mask_words));
  PagedAttnArgs a;
  RFX_CHECK(check_attention(q, out, n_rows, dtype, scale, 0, workspace, workspace_bytes, need));
  if (n_rows == 0 || batch->n_seqs == 0) return REFLEX_OK;
  if (!mask || ((uintptr_t)mask & 7)) return REFLEX_EINVAL;
  const PagedTreePlan p = paged_tree_plan(*cache, *batch, n_rows, n_q_heads, dtype);
  fill_attention(a, cache, batch, q, out, n_rows, n_q_heads, dtype, scale, 0, 0, p.nsplit, workspace);
  a.tree = mask;
  a.tree_words = mask_words;
  a.units = p.units;
  a.tile_rows = p.tile_rows;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(dtype == REFLEX_DTYPE_BF16 ? launch_paged_tree_attention<bf16_t>(a, cache->store, s)
                                         : launch_paged_tree_attention<float>(a, cache->store, s));
}

int reflex_paged_accept(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const int32_t* path,
                        int32_t max_path, const int32_t* counts, int32_t* lengths, void* stream) {
  return accept_rows(cache, batch, path, max_path, counts, nullptr, lengths, stream);
}

int reflex_paged_weighed_accept(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const int32_t* path,
                                int32_t max_path, const int32_t* counts, float* weights, int32_t* lengths, void* stream) {
  if (batch && batch->n_seqs != 0 && (!weights || ((uintptr_t)weights & 3))) return REFLEX_EINVAL;
  return accept_rows(cache, batch, path, max_path, counts, weights, lengths, stream);
}

int reflex_paged_weighed_attention_workspace(const reflex_paged_cache* cache, const reflex_paged_batch* batch,
                                             int64_t n_rows, int32_t n_q_heads, int32_t dtype, size_t* bytes) {
  RFX_CHECK(reflex_paged_attention_workspace(cache, batch, n_rows, n_q_heads, dtype, bytes));
  RFX_CHECK(check_lists(cache, batch));
  if (n_rows > 0 && batch->n_seqs > 0) {
    const size_t rows = (size_t)n_rows * n_q_heads;
    *bytes = whole_256(whole_256(*bytes) + rows * sizeof(float2)) +
             paged_weigh_plan(*cache, *batch, n_rows, n_q_heads, dtype).bytes;
  }
  return REFLEX_OK;
}

int reflex_paged_weighed_attention(const reflex_paged_cache* cache, const reflex_paged_batch* batch,
                                   const reflex_rows* q, const reflex_rows* out, int64_t n_rows, int32_t n_q_heads,
                                   int32_t dtype, float scale, int32_t causal, int32_t window, float* weights,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0, part = 0;
  RFX_CHECK(reflex_paged_weighed_attention_workspace(cache, batch, n_rows, n_q_heads, dtype, &need));
  RFX_CHECK(reflex_paged_attention_workspace(cache, batch, n_rows, n_q_heads, dtype, &part));
  PagedAttnArgs a;
  RFX_CHECK(check_attention(q, out, n_rows, dtype, scale, window, workspace, workspace_bytes, need));
  if (n_rows == 0 || batch->n_seqs == 0) return REFLEX_OK;
  if (!weights || ((uintptr_t)weights & 3)) return REFLEX_EINVAL;
  fill_attention(a, cache, batch, q, out, n_rows, n_q_heads, dtype, scale, causal, window,
                 paged_attention_plan(*cache, *batch, n_rows, n_q_heads, dtype, window).nsplit, workspace);
  char* const stats = reinterpret_cast<char*>(workspace) + whole_256(part);
  a.stats = reinterpret_cast<float2*>(stats);
  const PagedWeighPlan p = paged_weigh_plan(*cache, *batch, n_rows, n_q_heads, dtype);
  a.row_splits = p.row_splits;
  a.merge_with_sums = p.row_splits == 0 && a.nsplit > 1 && p.few;
  a.score_pitch = p.pitch;
  if (p.bytes) a.scores = reinterpret_cast<float*>(stats + whole_256((size_t)n_rows * n_q_heads * sizeof(float2)));
  const int64_t keys = expected_keys(cache, batch);
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(dtype == REFLEX_DTYPE_BF16 ? launch_paged_weighed_attention<bf16_t>(a, cache->store, weights, keys, p.few, s)
                                         : launch_paged_weighed_attention<float>(a, cache->store, weights, keys, p.few, s));
}

int reflex_paged_evict_workspace(const reflex_paged_cache* cache, const reflex_paged_batch* batch, int32_t keep,
                                 size_t* bytes) {
  if (!bytes) return REFLEX_EINVAL;
  RFX_CHECK(check_cache(cache));
  RFX_CHECK(check_batch(batch, cache, 1));
  RFX_CHECK(check_lists(cache, batch));
  if (keep < 1 || keep > (1 << 30)) return REFLEX_EINVAL;
  *bytes = (size_t)batch->n_seqs * cache->n_kv_heads * (sizeof(int2) + (size_t)keep * sizeof(int32_t));
  return REFLEX_OK;
}

int reflex_paged_evict(const reflex_paged_cache* cache, const reflex_paged_batch* batch, float* weights, int32_t keep,
                       int32_t sinks, int32_t recent, int32_t* kept, int32_t* lengths, void* workspace,
                       size_t workspace_bytes, void* stream) {
  size_t need = 0;
  RFX_CHECK(reflex_paged_evict_workspace(cache, batch, keep, &need));
  if (sinks < 0 || recent < 0 || (int64_t)sinks + recent > keep) return REFLEX_EINVAL;
  if (batch->n_seqs == 0) return REFLEX_OK;
  if (!weights || ((uintptr_t)weights & 3) || !lengths) return REFLEX_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return REFLEX_EINVAL;
  int2* const cut = reinterpret_cast<int2*>(workspace);
  const PagedEvictArgs a{pages_of(cache), seqs_of(batch), weights, keep,    sinks, recent,
                         kept,            lengths,        reinterpret_cast<int32_t*>(cut + batch->n_seqs * cache->n_kv_heads),
                         cut};
  return done(launch_paged_evict(a, elem_bytes(cache), cache->store >= REFLEX_STORE_FP8, expected_keys(cache, batch),
                                 reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
