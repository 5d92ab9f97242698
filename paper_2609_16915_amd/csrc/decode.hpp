// Decoding in the clear: what decode_abi.cpp and its kernels (kv_cache.hip,
// kv_attention.hip, verify_drafts.hip) share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "clear.hpp"
#include "internal.hpp"

namespace rosetta {

// Rows of heads of `dim` elements each, by strides in elements.
struct HeadRows {
  const void *p;
  size_t row, head;
};

// Where a sequence's rows and positions are: rows [first, first + n), the last of
// them at position base + n - 1.  Whatever starts and lens hold, the rows are among
// the call's.
struct Span {
  int first, n;
  int64_t base;
};
__host__ __device__ inline Span span_of(int64_t start, int64_t end, int64_t length, size_t rows) {
  const int64_t all = (int64_t)rows;
  const int64_t first = start < 0 ? 0 : start > all ? all : start;
  const int64_t last = end < first ? first : end > all ? all : end;
  const int n = (int)(last - first);
  return {(int)first, n, length - n};
}
__host__ __device__ inline Span span_of(const int *starts, const int *lens, size_t b, size_t rows) {
  return span_of(starts[b], starts[b + 1], lens ? lens[b] : 0, rows);
}

// Where position t of a sequence lies in the cache: its page, or -1 where there is
// none (t outside the table, or an entry that names no page).
__host__ __device__ inline int64_t page_of(const int *table, size_t table_len, int page_log,
                                           size_t pages, int64_t t) {
  if (t < 0 || (size_t)(t >> page_log) >= table_len) return -1;
  const int64_t pg = table[t >> page_log];
  return pg >= 0 && (size_t)pg < pages ? pg : -1;
}

// The cache as the kernels see it (rosetta_kv_cache, its page a power of two).
struct Cache {
  int8_t *k, *v;
  float *k_scale, *v_scale;
  size_t pages, kv_heads, dim;
  int page_log;
  size_t page_stride, head_stride, place_stride, scale_page_stride, scale_head_stride;
};
// The rows of a call (rosetta_kv_rows).
struct Packed {
  const int *table;
  size_t table_stride, table_len;
  const int *starts, *lens;
  size_t batch, rows;
};

hipError_t launch_kv_write(const HeadRows &k, const HeadRows &v, int dtype, const Cache &c,
                           const Packed &r, hipStream_t st);
hipError_t launch_kv_read(const Cache &c, const Packed &r, int dtype, const HeadRows &k,
                          const HeadRows &v, hipStream_t st);
hipError_t launch_kv_keep(const Cache &c, const Packed &r, const int *path, const int *count,
                          int *lens_out, hipStream_t st);
hipError_t launch_tree_masks(const int *parents, const int *starts, size_t batch, size_t rows,
                             size_t words, uint64_t *masks, hipStream_t st);

struct AttendArgs {
  HeadRows q;
  int dtype;
  Cache cache;
  Packed packed;
  size_t heads, max_rows;
  const uint64_t *masks;
  size_t words;
  float scale;
  HeadRows out;
  float *lse;
  void *workspace;
};
size_t kv_attention_workspace(size_t heads, size_t kv_heads, size_t dim, size_t batch, size_t rows,
                              size_t max_rows, size_t positions);
hipError_t launch_kv_attention(const AttendArgs &a, hipStream_t st);

struct VerifyArgs {
  const void *p, *q;
  size_t p_stride, q_stride;
  int dtype;
  const int64_t *drafts;
  const int *parents;
  const float *u;
  const int *starts;
  size_t batch, rows, vocab;
  int64_t *tokens;
  int *path, *count;
  void *workspace;
};
size_t verify_drafts_workspace(size_t batch, size_t vocab);
hipError_t launch_verify_drafts(const VerifyArgs &a, hipStream_t st);

}  // namespace rosetta
