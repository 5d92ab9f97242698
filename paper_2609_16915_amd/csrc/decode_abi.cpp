// C ABI of decoding in the clear (the 8-bit cache, attention over it, drafted tokens):
// validation on the host, then the launch functions of decode.hpp.
#include <hip/hip_runtime.h>

#include <cmath>
#include <utility>

#include "clear_checks.hpp"
#include "decode.hpp"
#include "internal.hpp"

using namespace rosetta;

namespace {

// Sizes past these would leave the kernels' index types.
constexpr size_t MAX_ROWS = (size_t)1 << 30, MAX_HEADS = (size_t)1 << 15, MAX_BATCH = 65535;
constexpr size_t MAX_TABLE = (size_t)1 << 30, MAX_DIM = 256;  // (positions; a page's, too)
constexpr size_t MAX_PLACE = (size_t)1 << 26;  // 16 places stay within 31-bit offsets
constexpr size_t MAX_VOCAB = (size_t)1 << 30, MAX_WORDS = (size_t)1 << 20;

// [n0][n1][dim] of distinct elements, strides s0 and s1, as rows of an Array: false where
// the strides let elements meet.
bool as_rows(Array &r, const char *name, const void *p, size_t n0, size_t s0, size_t n1, size_t s1,
             size_t dim, size_t elem, bool out) {
  if (n0 > 1 && n1 > 1 && s0 < s1) {
    std::swap(n0, n1);
    std::swap(s0, s1);
  }
  if (n1 <= 1) s1 = dim;
  if (s1 < dim || s1 > MAX_STRIDE) return false;
  const size_t len = n1 ? (n1 - 1) * s1 + dim : 0;
  if (n0 <= 1) s0 = len;
  if (s0 < len || (n0 > 1 && s0 > MAX_STRIDE)) return false;
  r = Array{name, p, n0, len, s0, elem, out, {Runs{n1, dim, s1}}};
  return true;
}

rosetta_status check_heads(Array &r, const char *name, const void *p, size_t rows, size_t row,
                           size_t heads, size_t head, size_t dim, int dtype, bool out) {
  if (!as_rows(r, name, p, rows, row, heads, head, dim, type_bytes(dtype), out))
    return fail(ROSETTA_ERR_PARAMS, "%s: strides of %zu and %zu elements for %zu x %zu x %zu", name,
                row, head, rows, heads, dim);
  return ROSETTA_OK;
}

// What a cache and the rows of a call come to: the kernels' forms, and the arrays.
struct Given {
  Cache c;
  Packed r;
  Array k, v, ks, vs, table, starts, lens;
};

rosetta_status check_given(const rosetta_kv_cache *c, const rosetta_kv_rows *r, bool out, Given &g) {
  if (!c) return fail(ROSETTA_ERR_NULL, "cache is NULL");
  if (!r) return fail(ROSETTA_ERR_NULL, "rows is NULL");
  if (c->kv_heads < 1 || c->pages < 1) return fail(ROSETTA_ERR_PARAMS, "a cache of nothing");
  if (c->dim < 16 || c->dim % 16 || c->dim > MAX_DIM)
    return fail(ROSETTA_ERR_UNSUPPORTED, "heads of %zu: multiples of 16 up to %zu", c->dim, MAX_DIM);
  if (c->page < 16 || (c->page & (c->page - 1)) || c->page > MAX_TABLE)
    return fail(ROSETTA_ERR_UNSUPPORTED, "pages of %zu: powers of two from 16 on", c->page);
  if (c->kv_heads > MAX_HEADS || c->pages >= (size_t)1 << 31)
    return fail(ROSETTA_ERR_UNSUPPORTED, "a cache of %zu pages and %zu heads", c->pages, c->kv_heads);
  if (r->batch > MAX_BATCH || r->rows >= MAX_ROWS || r->table_len > MAX_TABLE)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%zu rows of %zu sequences, %zu pages each", r->rows,
                r->batch, r->table_len);
  if (r->table_len < 1) return fail(ROSETTA_ERR_PARAMS, "a table of no pages");
  if (r->table_len * c->page > MAX_TABLE)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%zu pages of %zu positions each", r->table_len, c->page);
  Array inner;
  if (c->place_stride % 16 || c->head_stride % 16 || c->page_stride % 16 ||
      c->place_stride > MAX_PLACE ||
      !as_rows(inner, "cache", c->k, c->page, c->place_stride, c->kv_heads, c->head_stride, c->dim, 1,
               out))
    return fail(ROSETTA_ERR_PARAMS, "cache: strides of %zu, %zu and %zu elements", c->page_stride,
                c->head_stride, c->place_stride);
  const size_t extent = (inner.rows - 1) * inner.stride + inner.len;
  const size_t page_stride = c->pages > 1 ? c->page_stride : extent;
  if (page_stride < extent || c->page_stride > MAX_STRIDE)
    return fail(ROSETTA_ERR_PARAMS, "cache: pages of %zu elements %zu apart", extent, c->page_stride);
  Array scales;
  if (!as_rows(scales, "cache", c->k_scale, c->pages, c->scale_page_stride, c->kv_heads,
               c->scale_head_stride, c->page, 4, out))
    return fail(ROSETTA_ERR_PARAMS, "cache: scale strides of %zu and %zu", c->scale_page_stride,
                c->scale_head_stride);
  g.k = Array{"cache k", c->k, c->pages, extent, page_stride, 1, out,
              {Runs{inner.rows, inner.len, inner.stride}, inner.inner[0]}};
  g.v = g.k;
  g.v.name = "cache v";
  g.v.p = c->v;
  g.ks = scales;
  g.ks.name = "cache k_scale";
  g.vs = scales;
  g.vs.name = "cache v_scale";
  g.vs.p = c->v_scale;
  if (r->batch > 1 && (r->table_stride < r->table_len || r->table_stride > MAX_STRIDE))
    return fail(ROSETTA_ERR_PARAMS, "table: a stride of %zu entries for rows of %zu", r->table_stride,
                r->table_len);
  g.table = Array{"table", r->table, r->batch, r->table_len,
                  r->batch > 1 ? r->table_stride : r->table_len, 4, false};
  g.starts = Array{"starts", r->starts, 1, r->batch + 1, r->batch + 1, 4, false};
  g.lens = Array{"lens", r->lens, 1, r->batch, r->batch, 4, false};
  int log = 4;
  while ((size_t)1 << log < c->page) ++log;
  g.c = Cache{c->k, c->v, c->k_scale, c->v_scale, c->pages, c->kv_heads, c->dim, log,
              c->page_stride, c->head_stride, c->place_stride, c->scale_page_stride,
              c->scale_head_stride};
  g.r = Packed{r->table, r->table_stride, r->table_len, r->starts, r->lens, r->batch, r->rows};
  return ROSETTA_OK;
}

// Once there is something to do: what the kernels will read is there.
rosetta_status need_given(const Given &g) {
  for (const Array *a : {&g.k, &g.v, &g.ks, &g.vs, &g.table, &g.starts, &g.lens})
    if (!a->p) return fail(ROSETTA_ERR_NULL, "%s is NULL", a->name);
  for (const Array *a : {&g.k, &g.v})
    if ((uintptr_t)a->p % 16)
      return fail(ROSETTA_ERR_PARAMS, "%s does not start on 16 bytes", a->name);
  return ROSETTA_OK;
}

}  // namespace

extern "C" {

rosetta_status rosetta_kv_write(const void *k, size_t k_row_stride, size_t k_head_stride,
                                const void *v, size_t v_row_stride, size_t v_head_stride, int dtype,
                                const rosetta_kv_cache *cache, const rosetta_kv_rows *rows,
                                void *stream) {
  if (!is_type(dtype)) return fail(ROSETTA_ERR_PARAMS, "type %d", dtype);
  Given g;
  TRY(check_given(cache, rows, true, g));
  Array ak, av;
  TRY(check_heads(ak, "k", k, rows->rows, k_row_stride, cache->kv_heads, k_head_stride, cache->dim,
                  dtype, false));
  TRY(check_heads(av, "v", v, rows->rows, v_row_stride, cache->kv_heads, v_head_stride, cache->dim,
                  dtype, false));
  if (rows->rows == 0 || rows->batch == 0) return done(hipSuccess, "");
  NEED(k);
  NEED(v);
  TRY(need_given(g));
  TRY(check_arrays({ak, av, g.table, g.starts, g.lens, g.k, g.v, g.ks, g.vs}));
  return done(launch_kv_write({k, k_row_stride, k_head_stride}, {v, v_row_stride, v_head_stride},
                              dtype, g.c, g.r, (hipStream_t)stream), "rosetta_kv_write");
}

rosetta_status rosetta_kv_read(const rosetta_kv_cache *cache, const rosetta_kv_rows *rows, int dtype,
                               void *k, size_t k_row_stride, size_t k_head_stride, void *v,
                               size_t v_row_stride, size_t v_head_stride, void *stream) {
  if (!is_type(dtype)) return fail(ROSETTA_ERR_PARAMS, "type %d", dtype);
  Given g;
  TRY(check_given(cache, rows, false, g));
  Array ak, av;
  TRY(check_heads(ak, "k", k, rows->rows, k_row_stride, cache->kv_heads, k_head_stride, cache->dim,
                  dtype, true));
  TRY(check_heads(av, "v", v, rows->rows, v_row_stride, cache->kv_heads, v_head_stride, cache->dim,
                  dtype, true));
  if (rows->rows == 0 || rows->batch == 0) return done(hipSuccess, "");
  NEED(k);
  NEED(v);
  TRY(need_given(g));
  TRY(check_arrays({ak, av, g.table, g.starts, g.lens, g.k, g.v, g.ks, g.vs}));
  return done(launch_kv_read(g.c, g.r, dtype, {k, k_row_stride, k_head_stride},
                             {v, v_row_stride, v_head_stride}, (hipStream_t)stream),
              "rosetta_kv_read");
}

rosetta_status rosetta_kv_keep(const rosetta_kv_cache *cache, const rosetta_kv_rows *rows,
                               const int32_t *path, const int32_t *count, int32_t *lens_out,
                               void *stream) {
  Given g;
  TRY(check_given(cache, rows, true, g));
  if (rows->batch == 0) return done(hipSuccess, "");
  if (rows->rows) NEED(path);
  NEED(count);
  NEED(lens_out);
  TRY(need_given(g));
  const Array ap{"path", path, 1, rows->rows, rows->rows, 4, false};
  const Array ac{"count", count, 1, rows->batch, rows->batch, 4, false};
  const Array al{"lens_out", lens_out, 1, rows->batch, rows->batch, 4, true};
  TRY(check_arrays({ap, ac, g.table, g.starts, g.lens, g.k, g.v, g.ks, g.vs, al}));
  return done(launch_kv_keep(g.c, g.r, path, count, lens_out, (hipStream_t)stream),
              "rosetta_kv_keep");
}

rosetta_status rosetta_tree_masks(const int32_t *parents, const int32_t *starts, size_t batch,
                                  size_t rows, size_t words, uint64_t *masks, void *stream) {
  if (batch > MAX_BATCH || rows >= MAX_ROWS || words > MAX_WORDS || rows * words >= (size_t)1 << 32)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%zu rows of %zu sequences, %zu words each", rows, batch,
                words);
  if (words < 1) return fail(ROSETTA_ERR_PARAMS, "masks of no words");
  if (rows == 0 || batch == 0) return done(hipSuccess, "");
  NEED(parents);
  NEED(starts);
  NEED(masks);
  const Array ap{"parents", parents, 1, rows, rows, 4, false};
  const Array as{"starts", starts, 1, batch + 1, batch + 1, 4, false};
  const Array am{"masks", masks, 1, rows * words, rows * words, 8, true};
  TRY(check_arrays({ap, as, am}));
  return done(launch_tree_masks(parents, starts, batch, rows, words, masks, (hipStream_t)stream),
              "rosetta_tree_masks");
}

size_t rosetta_kv_attention_workspace_bytes(size_t heads, size_t kv_heads, size_t dim, size_t batch,
                                            size_t rows, size_t max_rows, size_t positions) {
  if (!rows || !batch || !max_rows || !kv_heads || heads % kv_heads || !dim) return 0;
  return kv_attention_workspace(heads, kv_heads, dim, batch, rows, max_rows, positions);
}

rosetta_status rosetta_kv_attention(const void *q, size_t q_row_stride, size_t q_head_stride,
                                    int dtype, size_t heads, const rosetta_kv_cache *cache,
                                    const rosetta_kv_rows *rows, size_t max_rows,
                                    const uint64_t *masks, size_t words, float scale, void *out,
                                    size_t out_row_stride, size_t out_head_stride, float *lse,
                                    void *workspace, size_t workspace_bytes, void *stream) {
  if (!is_type(dtype)) return fail(ROSETTA_ERR_PARAMS, "type %d", dtype);
  if (dtype == ROSETTA_F32)
    return fail(ROSETTA_ERR_UNSUPPORTED, "32-bit queries: pass bf16 or f16");
  if (!(scale >= 0.f) || !std::isfinite(scale))
    return fail(ROSETTA_ERR_PARAMS, "scale must be finite and >= 0");
  Given g;
  TRY(check_given(cache, rows, false, g));
  if (heads < 1 || heads % cache->kv_heads)
    return fail(ROSETTA_ERR_PARAMS, "%zu heads over %zu of the cache", heads, cache->kv_heads);
  if (heads > MAX_HEADS || max_rows >= MAX_ROWS || rows->rows * heads >= (size_t)1 << 31 ||
      max_rows * (heads / cache->kv_heads) >= MAX_ROWS)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%zu rows of %zu heads", rows->rows, heads);
  if (masks && (words > MAX_WORDS || words * 64 < max_rows))
    return fail(ROSETTA_ERR_PARAMS, "masks of %zu words for %zu rows", words, max_rows);
  Array aq, ao;
  TRY(check_heads(aq, "q", q, rows->rows, q_row_stride, heads, q_head_stride, cache->dim, dtype,
                  false));
  TRY(check_heads(ao, "out", out, rows->rows, out_row_stride, heads, out_head_stride, cache->dim,
                  dtype, true));
  if (rows->rows == 0 || rows->batch == 0 || max_rows == 0) return done(hipSuccess, "");
  NEED(q);
  NEED(out);
  TRY(need_given(g));
  const size_t need = rosetta_kv_attention_workspace_bytes(
      heads, cache->kv_heads, cache->dim, rows->batch, rows->rows, max_rows,
      rows->table_len * cache->page);
  if (workspace_bytes < need)
    return fail(ROSETTA_ERR_SIZE, "workspace holds %zu bytes, the call needs %zu", workspace_bytes,
                need);
  if (need) NEED(workspace);
  const Array am{"masks", masks, 1, rows->rows * words, rows->rows * words, 8, false};
  const Array al{"lse", lse, 1, rows->rows * heads, rows->rows * heads, 4, true};
  const Array ws{"workspace", need ? workspace : nullptr, 1, need / 16, need / 16, 16, true};
  TRY(check_arrays({aq, g.table, g.starts, g.lens, g.k, g.v, g.ks, g.vs, am, ao, al, ws}));
  AttendArgs a{};
  a.q = {q, q_row_stride, q_head_stride};
  a.dtype = dtype;
  a.cache = g.c;
  a.packed = g.r;
  a.heads = heads;
  a.max_rows = max_rows;
  a.masks = masks;
  a.words = words;
  a.scale = scale;
  a.out = {out, out_row_stride, out_head_stride};
  a.lse = lse;
  a.workspace = need ? workspace : nullptr;
  return done(launch_kv_attention(a, (hipStream_t)stream), "rosetta_kv_attention");
}

size_t rosetta_verify_drafts_workspace_bytes(size_t batch, size_t vocab) {
  return batch && vocab ? verify_drafts_workspace(batch, vocab) : 0;
}

rosetta_status rosetta_verify_drafts(const void *p, size_t p_stride, const void *q, size_t q_stride,
                                     int dtype, const int64_t *drafts, const int32_t *parents,
                                     const float *u, const int32_t *starts, size_t batch,
                                     size_t rows, size_t vocab, int64_t *tokens, int32_t *path,
                                     int32_t *count, void *workspace, size_t workspace_bytes,
                                     void *stream) {
  if (!is_type(dtype)) return fail(ROSETTA_ERR_PARAMS, "type %d", dtype);
  if (vocab < 1) return fail(ROSETTA_ERR_PARAMS, "a vocabulary of none");
  if (vocab > MAX_VOCAB || batch > MAX_BATCH || rows >= MAX_ROWS)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%zu rows of %zu sequences over a vocabulary of %zu", rows,
                batch, vocab);
  const size_t b = type_bytes(dtype);
  const Array ap{"p", p, rows, vocab, p_stride, b, false}, aq{"q", q, rows, vocab, q_stride, b, false};
  TRY(check_strides({ap, aq}));
  if (batch == 0) return done(hipSuccess, "");
  if (rows) {
    NEED(p);
    NEED(q);
    NEED(drafts);
    NEED(u);
    NEED(tokens);
    NEED(path);
  }
  NEED(starts);
  NEED(count);
  const size_t need = rosetta_verify_drafts_workspace_bytes(batch, vocab);
  if (workspace_bytes < need)
    return fail(ROSETTA_ERR_SIZE, "workspace holds %zu bytes, the call needs %zu", workspace_bytes,
                need);
  if (need) NEED(workspace);
  const Array ad{"drafts", drafts, 1, rows, rows, 8, false};
  const Array ar{"parents", parents, 1, rows, rows, 4, false};
  const Array au{"u", u, 1, rows, rows, 4, false};
  const Array as{"starts", starts, 1, batch + 1, batch + 1, 4, false};
  const Array at{"tokens", tokens, 1, rows, rows, 8, true}, ah{"path", path, 1, rows, rows, 4, true};
  const Array ac{"count", count, 1, batch, batch, 4, true};
  const Array ws{"workspace", need ? workspace : nullptr, 1, need / 8, need / 8, 8, true};
  TRY(check_arrays({ap, aq, ad, ar, au, as, at, ah, ac, ws}));
  return done(launch_verify_drafts({p, q, p_stride, q_stride, dtype, drafts, parents, u, starts,
                                    batch, rows, vocab, tokens, path, count, workspace},
                                   (hipStream_t)stream), "rosetta_verify_drafts");
}

}  // extern "C"
