// C ABI of the clear side (8-bit layers and the vocabulary loss): validation
// on the host, then one launch function of clear.hpp per call.
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "clear.hpp"
#include "internal.hpp"

using namespace rosetta;

namespace {

// Sizes past these would leave the kernels' index types.  (What a grid does not hold, the
// launch functions tell before they enqueue anything: hipErrorInvalidConfiguration.)
constexpr size_t MAX_DIM = (size_t)1 << 24, MAX_LOSS_DIM = (size_t)1 << 20;
constexpr size_t MAX_ROWS = (size_t)1 << 31;
constexpr size_t MAX_STRIDE = (size_t)1 << 32;
constexpr size_t MAX_K = 131071;  // 128 * 128 * k < 2^31

rosetta_status fail(rosetta_status st, const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return st;
}

rosetta_status done(hipError_t e, const char *what) {
  if (e == hipSuccess) {
    set_last_error("");
    return ROSETTA_OK;
  }
  (void)hipGetLastError();
  if (e == hipErrorOutOfMemory)
    return fail(ROSETTA_ERR_NOMEM, "%s: %s", what, hipGetErrorString(e));
  if (e == hipErrorInvalidConfiguration)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%s: sizes that one launch does not hold", what);
  return fail(ROSETTA_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

bool is_type(int t) { return t == ROSETTA_F32 || t == ROSETTA_BF16 || t == ROSETTA_F16; }

// A named device array: rows of `len` elements of `elem` bytes, `stride` apart.
struct Array {
  const char *name;
  const void *p;
  size_t rows, len, stride, elem;
  bool out;
  // (past 64 bits where a caller's sizes are: 2^31 rows 2^32 elements apart)
  unsigned __int128 bytes() const {
    return rows && len ? ((unsigned __int128)(rows - 1) * stride + len) * elem : 0;
  }
};

// Whether two arrays share memory: by the whole ranges, or, rows as far apart in both
// (columns of one buffer), by where the second's rows lie between the first's.
bool overlap(const Array &a, const Array &b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  if (!(x < y + b.bytes() && y < x + a.bytes())) return false;
  const size_t pitch = a.stride * a.elem;
  if (a.rows < 2 || b.rows < 2 || pitch != b.stride * b.elem) return true;
  const size_t at = y >= x ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;
  return at < a.len * a.elem || at + b.len * b.elem > pitch;
}

rosetta_status check_strides(std::initializer_list<Array> as) {
  for (const Array &a : as)
    if (a.p && (a.stride < a.len || a.stride > MAX_STRIDE))
      return fail(ROSETTA_ERR_PARAMS, "%s: a stride of %zu elements for rows of %zu", a.name,
                  a.stride, a.len);
  return ROSETTA_OK;
}

// Alignment to the element, and outputs apart from everything else; an output
// and an input named in `same` may be one array.
rosetta_status check_arrays(std::initializer_list<Array> as, const char *out = nullptr,
                            std::initializer_list<const char *> same = {}) {
  for (const Array &a : as)
    if (a.p && (uintptr_t)a.p % a.elem)
      return fail(ROSETTA_ERR_PARAMS, "%s is not aligned to its elements", a.name);
  for (const Array *a = as.begin(); a != as.end(); ++a)
    for (const Array *b = a + 1; b != as.end(); ++b) {
      if (!a->p || !b->p || (!a->out && !b->out)) continue;
      if (!overlap(*a, *b)) continue;
      bool fine = false;
      for (const char *s : same)
        fine |= a->name == s && b->name == out && a->p == b->p && a->stride == b->stride;
      if (!fine) return fail(ROSETTA_ERR_ALIAS, "%s overlaps %s", b->name, a->name);
    }
  return ROSETTA_OK;
}

rosetta_status check_sizes(size_t rows, size_t dim) {
  if (dim < 1) return fail(ROSETTA_ERR_PARAMS, "rows of no elements");
  if (dim > MAX_DIM || rows >= MAX_ROWS)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%zu rows of %zu elements", rows, dim);
  return ROSETTA_OK;
}

// hipMemset would not do: a caller may capture this in a graph
__global__ void k_zero(char *p, size_t row, size_t stride, size_t rows) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < row * rows;
       i += (size_t)gridDim.x * 256)
    p[i / row * stride + i % row] = 0;
}

hipError_t zero_rows(void *p, size_t row, size_t stride, size_t rows, hipStream_t st) {
  size_t g = (row * rows + 255) / 256;
  g = g > 65536 ? 65536 : g;
  if (!g) return hipSuccess;
  hipLaunchKernelGGL(k_zero, dim3((unsigned)g), dim3(256), 0, st, (char *)p, row, stride, rows);
  return hipGetLastError();
}

#define TRY(x)                        \
  do {                                \
    const rosetta_status st_ = (x);   \
    if (st_ != ROSETTA_OK) return st_; \
  } while (0)
#define NEED(p)                                                          \
  do {                                                                   \
    if (!(p)) return fail(ROSETTA_ERR_NULL, #p " is NULL");              \
  } while (0)

}  // namespace

extern "C" {

rosetta_status rosetta_rms_norm(const void *x, size_t x_stride, const void *residual,
                                size_t residual_stride, const void *weight, int weight_dtype,
                                int dtype, size_t rows, size_t dim, float eps, void *h,
                                size_t h_stride, void *y, size_t y_stride, int8_t *q,
                                size_t q_stride, float *scale, float *inv_rms, void *stream) {
  if (!is_type(dtype) || (weight && weight_dtype != dtype && weight_dtype != ROSETTA_F32))
    return fail(ROSETTA_ERR_PARAMS, "types %d and %d (weight)", dtype, weight_dtype);
  if (!(eps >= 0.f)) return fail(ROSETTA_ERR_PARAMS, "eps must be >= 0");
  TRY(check_sizes(rows, dim));
  const size_t b = type_bytes(dtype);
  const Array ax{"x", x, rows, dim, x_stride, b, false};
  const Array ar{"residual", residual, rows, dim, residual_stride, b, false};
  const Array aw{"weight", weight, 1, dim, dim, weight ? type_bytes(weight_dtype) : 1, false};
  const Array ah{"h", h, rows, dim, h_stride, b, true}, ay{"y", y, rows, dim, y_stride, b, true};
  const Array aq{"q", q, rows, dim, q_stride, 1, true};
  const Array as{"scale", scale, 1, rows, rows, 4, true};
  const Array ai{"inv_rms", inv_rms, 1, rows, rows, 4, true};
  TRY(check_strides({ax, ar, ah, ay, aq}));
  if (rows == 0) return done(hipSuccess, "");
  NEED(x);
  if (!q != !scale) return fail(ROSETTA_ERR_NULL, "q and scale go together");
  TRY(check_arrays({ax, ar, aw, ah, ay, aq, as, ai}, ah.name, {ax.name, ar.name}));
  NormArgs a{};
  a.x = {x, x_stride};
  a.residual = {residual, residual_stride};
  a.weight = weight;
  a.weight_dtype = weight_dtype;
  a.dtype = dtype;
  a.rows = rows;
  a.dim = dim;
  a.eps = eps;
  a.h = {h, h_stride};
  a.y = {y, y_stride};
  a.q = {q, q_stride};
  a.scale = scale;
  a.inv_rms = inv_rms;
  return done(launch_rms_norm(a, (hipStream_t)stream), "rosetta_rms_norm");
}

size_t rosetta_rms_norm_backward_workspace_bytes(size_t rows, size_t dim) {
  return norm_back_groups(rows) * dim * sizeof(float);
}

rosetta_status rosetta_rms_norm_backward(const void *gy, size_t gy_stride, const void *gh,
                                         size_t gh_stride, const void *h, size_t h_stride,
                                         const void *weight, int weight_dtype,
                                         const float *inv_rms, int dtype, size_t rows, size_t dim,
                                         void *gx, size_t gx_stride, float *gweight,
                                         void *workspace, size_t workspace_bytes, void *stream) {
  if (!is_type(dtype) || (weight && weight_dtype != dtype && weight_dtype != ROSETTA_F32))
    return fail(ROSETTA_ERR_PARAMS, "types %d and %d (weight)", dtype, weight_dtype);
  TRY(check_sizes(rows, dim));
  const size_t b = type_bytes(dtype);
  const Array ay{"gy", gy, rows, dim, gy_stride, b, false};
  const Array ag{"gh", gh, rows, dim, gh_stride, b, false};
  const Array ah{"h", h, rows, dim, h_stride, b, false};
  const Array aw{"weight", weight, 1, dim, dim, weight ? type_bytes(weight_dtype) : 1, false};
  const Array ai{"inv_rms", inv_rms, 1, rows, rows, 4, false};
  const Array ax{"gx", gx, rows, dim, gx_stride, b, true};
  const Array agw{"gweight", gweight, 1, dim, dim, 4, true};
  const size_t need = rosetta_rms_norm_backward_workspace_bytes(rows, dim);
  const Array ws{"workspace", gweight ? workspace : nullptr, 1, need / 4, need / 4, 4, true};
  TRY(check_strides({ay, ag, ah, ax}));
  if (rows == 0)
    return done(gweight ? zero_rows(gweight, dim * 4, dim * 4, 1, (hipStream_t)stream)
                        : hipSuccess, "rosetta_rms_norm_backward");
  NEED(gy);
  NEED(h);
  NEED(inv_rms);
  NEED(gx);
  if (gweight) {
    if (workspace_bytes < need)
      return fail(ROSETTA_ERR_SIZE, "workspace holds %zu bytes, the call needs %zu",
                  workspace_bytes, need);
    NEED(workspace);
  }
  TRY(check_arrays({ay, ag, ah, aw, ai, ax, agw, ws}, ax.name, {ay.name, ag.name}));
  NormBackArgs a{};
  a.gy = {gy, gy_stride};
  a.gh = {gh, gh_stride};
  a.h = {h, h_stride};
  a.weight = weight;
  a.weight_dtype = weight_dtype;
  a.dtype = dtype;
  a.inv_rms = inv_rms;
  a.rows = rows;
  a.dim = dim;
  a.gx = {gx, gx_stride};
  a.gweight = gweight;
  a.partial = gweight ? (float *)workspace : nullptr;
  return done(launch_rms_norm_backward(a, (hipStream_t)stream), "rosetta_rms_norm_backward");
}

rosetta_status rosetta_quantize_rows(const void *x, size_t x_stride, int dtype, size_t rows,
                                     size_t dim, int8_t *q, size_t q_stride, float *scale,
                                     void *stream) {
  if (!is_type(dtype)) return fail(ROSETTA_ERR_PARAMS, "type %d", dtype);
  TRY(check_sizes(rows, dim));
  const Array ax{"x", x, rows, dim, x_stride, type_bytes(dtype), false};
  const Array aq{"q", q, rows, dim, q_stride, 1, true};
  const Array as{"scale", scale, 1, rows, rows, 4, true};
  TRY(check_strides({ax, aq}));
  if (rows == 0) return done(hipSuccess, "");
  NEED(x);
  NEED(q);
  NEED(scale);
  TRY(check_arrays({ax, aq, as}));
  NormArgs a{};
  a.x = {x, x_stride};
  a.dtype = dtype;
  a.rows = rows;
  a.dim = dim;
  a.q = {q, q_stride};
  a.scale = scale;
  return done(launch_quantize_rows(a, (hipStream_t)stream), "rosetta_quantize_rows");
}

rosetta_status rosetta_dequantize_rows(const int8_t *q, size_t q_stride, const float *scale,
                                       int dtype, size_t rows, size_t dim, void *out,
                                       size_t out_stride, void *stream) {
  if (!is_type(dtype)) return fail(ROSETTA_ERR_PARAMS, "type %d", dtype);
  TRY(check_sizes(rows, dim));
  const Array aq{"q", q, rows, dim, q_stride, 1, false};
  const Array as{"scale", scale, 1, rows, rows, 4, false};
  const Array ao{"out", out, rows, dim, out_stride, type_bytes(dtype), true};
  TRY(check_strides({aq, ao}));
  if (rows == 0) return done(hipSuccess, "");
  NEED(q);
  NEED(scale);
  NEED(out);
  TRY(check_arrays({aq, as, ao}));
  return done(launch_dequantize_rows(q, q_stride, scale, dtype, rows, dim, {out, out_stride},
                                     (hipStream_t)stream), "rosetta_dequantize_rows");
}

size_t rosetta_q8_matmul_workspace_bytes(size_t m, size_t n, size_t k) {
  return m && n ? q8_matmul_workspace(m, n, k) : 0;
}

rosetta_status rosetta_q8_matmul(const int8_t *a, size_t a_stride, const float *a_scale,
                                 const int8_t *b, size_t b_stride, const float *b_scale,
                                 const float *bias, void *out, size_t out_stride, int out_dtype,
                                 size_t m, size_t n, size_t k, void *workspace,
                                 size_t workspace_bytes, void *stream) {
  if (!is_type(out_dtype)) return fail(ROSETTA_ERR_PARAMS, "type %d", out_dtype);
  if (n < 1) return fail(ROSETTA_ERR_PARAMS, "rows of no elements");
  if (k > MAX_K)
    return fail(ROSETTA_ERR_UNSUPPORTED, "k = %zu: sums of more than %zu products may leave 32 bits",
                k, MAX_K);
  if (m >= MAX_ROWS || n >= MAX_ROWS || ((m + 15) / 16) * ((n + 15) / 16) >= MAX_ROWS)
    return fail(ROSETTA_ERR_UNSUPPORTED, "an output of %zu x %zu", m, n);
  const Array aa{"a", a, m, k, a_stride, 1, false}, ab{"b", b, n, k, b_stride, 1, false};
  const Array as{"a_scale", a_scale, 1, m, m, 4, false}, bs{"b_scale", b_scale, 1, n, n, 4, false};
  const Array bi{"bias", bias, 1, n, n, 4, false};
  const Array ao{"out", out, m, n, out_stride, type_bytes(out_dtype), true};
  TRY(check_strides({aa, ab, ao}));
  if (m == 0) return done(hipSuccess, "");
  if (k > 0) {
    NEED(a);
    NEED(b);
  }
  NEED(a_scale);
  NEED(b_scale);
  NEED(out);
  const size_t need = workspace ? rosetta_q8_matmul_workspace_bytes(m, n, k) : 0;
  if (workspace && workspace_bytes < need)
    return fail(ROSETTA_ERR_SIZE, "workspace holds %zu bytes, the call needs %zu", workspace_bytes,
                need);
  const Array ws{"workspace", need ? workspace : nullptr, 1, need / 16, need / 16, 16, true};
  TRY(check_arrays({aa, ab, as, bs, bi, ao, ws}));
  const Q8Args q{a, b, a_stride, b_stride, a_scale, b_scale, bias, out, out_stride, out_dtype,
                 m, n, k, need ? (int *)workspace : nullptr};
  return done(launch_q8_matmul(q, (hipStream_t)stream), "rosetta_q8_matmul");
}

static rosetta_status check_loss(int dtype, size_t rows, size_t dim, size_t vocab) {
  if (!is_type(dtype)) return fail(ROSETTA_ERR_PARAMS, "type %d", dtype);
  if (dtype == ROSETTA_F32)
    return fail(ROSETTA_ERR_UNSUPPORTED, "32-bit hidden states: pass bf16 or f16");
  TRY(check_sizes(rows, dim));
  if (vocab < 1) return fail(ROSETTA_ERR_PARAMS, "a vocabulary of none");
  if (dim > MAX_LOSS_DIM || vocab >= MAX_ROWS || ((rows + 15) / 16) * ((vocab + 15) / 16) >= MAX_ROWS)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%zu rows of %zu over a vocabulary of %zu", rows, dim,
                vocab);
  return ROSETTA_OK;
}

size_t rosetta_cross_entropy_workspace_bytes(size_t rows, size_t dim, size_t vocab) {
  return rows && dim && vocab ? cross_entropy_workspace(rows, dim, vocab) : 0;
}

rosetta_status rosetta_cross_entropy(const void *h, size_t h_stride, const void *w,
                                     size_t w_stride, int dtype, const int64_t *targets,
                                     int64_t ignore_index, size_t rows, size_t dim, size_t vocab,
                                     float *loss, float *lse, void *workspace,
                                     size_t workspace_bytes, void *stream) {
  TRY(check_loss(dtype, rows, dim, vocab));
  const size_t need = rosetta_cross_entropy_workspace_bytes(rows, dim, vocab);
  const Array ah{"h", h, rows, dim, h_stride, 2, false}, aw{"w", w, vocab, dim, w_stride, 2, false};
  const Array at{"targets", targets, 1, rows, rows, 8, false};
  const Array al{"loss", loss, 1, rows, rows, 4, true}, ae{"lse", lse, 1, rows, rows, 4, true};
  const Array ws{"workspace", workspace, 1, need / 16, need / 16, 16, true};
  TRY(check_strides({ah, aw}));
  if (rows == 0) return done(hipSuccess, "");
  NEED(h);
  NEED(w);
  NEED(targets);
  NEED(loss);
  NEED(lse);
  if (workspace_bytes < need)
    return fail(ROSETTA_ERR_SIZE, "workspace holds %zu bytes, the call needs %zu", workspace_bytes,
                need);
  NEED(workspace);
  TRY(check_arrays({ah, aw, at, al, ae, ws}));
  LossArgs a{};
  a.h = h;
  a.w = w;
  a.h_stride = h_stride;
  a.w_stride = w_stride;
  a.dtype = dtype;
  a.targets = targets;
  a.ignore_index = ignore_index;
  a.rows = rows;
  a.dim = dim;
  a.vocab = vocab;
  a.loss = loss;
  a.lse = lse;
  a.workspace = workspace;
  return done(launch_cross_entropy(a, (hipStream_t)stream), "rosetta_cross_entropy");
}

size_t rosetta_cross_entropy_backward_workspace_bytes(size_t rows, size_t dim, size_t vocab) {
  return rows && dim && vocab ? cross_entropy_backward_workspace(rows, dim, vocab) : 0;
}

rosetta_status rosetta_cross_entropy_backward(const void *h, size_t h_stride, const void *w,
                                              size_t w_stride, int dtype, const int64_t *targets,
                                              int64_t ignore_index, const float *lse,
                                              const float *gloss, size_t rows, size_t dim,
                                              size_t vocab, void *gh, size_t gh_stride, void *gw,
                                              size_t gw_stride, void *workspace,
                                              size_t workspace_bytes, void *stream) {
  TRY(check_loss(dtype, rows, dim, vocab));
  const size_t need = rosetta_cross_entropy_backward_workspace_bytes(rows, dim, vocab);
  const Array ah{"h", h, rows, dim, h_stride, 2, false}, aw{"w", w, vocab, dim, w_stride, 2, false};
  const Array at{"targets", targets, 1, rows, rows, 8, false};
  const Array ae{"lse", lse, 1, rows, rows, 4, false}, ag{"gloss", gloss, 1, rows, rows, 4, false};
  const Array agh{"gh", gh, rows, dim, gh_stride, 2, true};
  const Array agw{"gw", gw, vocab, dim, gw_stride, 2, true};
  const Array ws{"workspace", workspace, 1, need / 16, need / 16, 16, true};
  TRY(check_strides({ah, aw, agh, agw}));
  if (rows == 0)
    return done(gw ? zero_rows(gw, dim * 2, gw_stride * 2, vocab, (hipStream_t)stream) : hipSuccess,
                "rosetta_cross_entropy_backward");
  NEED(h);
  NEED(w);
  NEED(targets);
  NEED(lse);
  NEED(gloss);
  if (workspace_bytes < need)
    return fail(ROSETTA_ERR_SIZE, "workspace holds %zu bytes, the call needs %zu", workspace_bytes,
                need);
  NEED(workspace);
  TRY(check_arrays({ah, aw, at, ae, ag, agh, agw, ws}));
  LossArgs a{};
  a.h = h;
  a.w = w;
  a.h_stride = h_stride;
  a.w_stride = w_stride;
  a.dtype = dtype;
  a.targets = targets;
  a.ignore_index = ignore_index;
  a.rows = rows;
  a.dim = dim;
  a.vocab = vocab;
  a.lse = const_cast<float *>(lse);
  a.gloss = gloss;
  a.gh = gh;
  a.gw = gw;
  a.gh_stride = gh_stride;
  a.gw_stride = gw_stride;
  a.workspace = workspace;
  return done(launch_cross_entropy_backward(a, (hipStream_t)stream),
              "rosetta_cross_entropy_backward");
}

}  // extern "C"
