// The clear side (8-bit layers and the vocabulary loss): what clear_abi.cpp
// and its kernels (clear_norm.hip, q8_matmul.hip, cross_entropy.hip) share.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "internal.hpp"

namespace rosetta {

// Allow a kernel more than the default 64 KiB of dynamic LDS.
template <typename K>
inline hipError_t allow_lds(K kernel, size_t bytes) {
  if (bytes <= 65536) return hipSuccess;
  return hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                             (int)bytes);
}

// Whether one launch takes so many workgroups: it counts threads in 32 bits.
inline bool grid_fits(size_t blocks, size_t threads) { return blocks * threads < (size_t)1 << 32; }

using bf16 = __bf16;
using f16 = _Float16;

inline size_t type_bytes(int dtype) { return dtype == ROSETTA_F32 ? 4 : 2; }

// Rows of `dim` elements at `p`, `stride` elements apart.
struct Rows {
  void *p;
  size_t stride;
};
struct CRows {
  const void *p;
  size_t stride;
};

struct NormArgs {
  CRows x, residual;
  const void *weight;
  int weight_dtype, dtype;
  size_t rows, dim;
  float eps;
  Rows h, y, q;
  float *scale, *inv_rms;
};
hipError_t launch_rms_norm(const NormArgs &a, hipStream_t st);
// scale and q of x itself
hipError_t launch_quantize_rows(const NormArgs &a, hipStream_t st);
hipError_t launch_dequantize_rows(const int8_t *q, size_t q_stride, const float *scale, int dtype,
                                  size_t rows, size_t dim, Rows out, hipStream_t st);

struct NormBackArgs {
  CRows gy, gh, h;
  const void *weight;
  int weight_dtype, dtype;
  const float *inv_rms;
  size_t rows, dim;
  Rows gx;
  float *gweight;
  float *partial;  // [norm_back_groups(rows)][dim]
};
size_t norm_back_groups(size_t rows);
hipError_t launch_rms_norm_backward(const NormBackArgs &a, hipStream_t st);

struct Q8Args {
  const int8_t *a, *b;
  size_t a_stride, b_stride;
  const float *a_scale, *b_scale, *bias;
  void *out;
  size_t out_stride;
  int out_dtype;
  size_t m, n, k;
  int *workspace;  // q8_matmul_workspace bytes, or null
};
size_t q8_matmul_workspace(size_t m, size_t n, size_t k);
hipError_t launch_q8_matmul(const Q8Args &a, hipStream_t st);

struct LossArgs {
  const void *h, *w;
  size_t h_stride, w_stride;
  int dtype;
  const int64_t *targets;
  int64_t ignore_index;
  size_t rows, dim, vocab;
  float *loss, *lse;           // forward: out; backward: lse read
  const float *gloss;          // backward
  void *gh, *gw;               // backward, either may be null
  size_t gh_stride, gw_stride;
  void *workspace;
};
size_t cross_entropy_workspace(size_t rows, size_t dim, size_t vocab);
size_t cross_entropy_backward_workspace(size_t rows, size_t dim, size_t vocab);
hipError_t launch_cross_entropy(const LossArgs &a, hipStream_t st);
hipError_t launch_cross_entropy_backward(const LossArgs &a, hipStream_t st);

}  // namespace rosetta
