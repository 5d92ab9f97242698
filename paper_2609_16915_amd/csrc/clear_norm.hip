// Root-mean-square norm with the residual's addition and an 8-bit output,
// its gradient, and rows to 8 bits and back.
//
// All of it is bound by memory: one pass, every element read once and every
// result written once, a row held in registers between its reduction and its
// use.  One reduction serves both the norm and the 8-bit scale, since
//   y / scale = h w inv_rms / (max|h w| inv_rms / 127) = h w * (127 / max|h w|):
// the sum of h^2 and the maximum of |h w| are taken together, and q needs
// neither inv_rms nor a second pass.
#include "clear.hpp"

namespace rosetta {

namespace {

constexpr int VEC = 8;  // elements of a thread's load: 16 bytes of bf16 or f16

template <class T>
__device__ inline float to_f(T v) { return (float)v; }
template <class T>
__device__ inline T from_f(float v) { return (T)v; }  // to nearest, ties to even

// Eight consecutive elements.  The address may be any multiple of the
// element's size: the copy compiles to the widest loads, which the hardware
// takes unaligned.
template <class T>
struct __attribute__((packed, aligned(1))) Pack {
  T v[VEC];
};

template <class T>
__device__ inline void load8(const T *p, size_t left, float (&f)[VEC]) {
  if (left >= VEC) {
    Pack<T> v;
    __builtin_memcpy(&v, p, sizeof v);
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = to_f(v.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = (size_t)i < left ? to_f(p[i]) : 0.f;
  }
}

template <class T>
__device__ inline void store8(T *p, size_t left, const float (&f)[VEC]) {
  if (left >= VEC) {
    Pack<T> v;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v.v[i] = from_f<T>(f[i]);
    __builtin_memcpy(p, &v, sizeof v);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if ((size_t)i < left) p[i] = from_f<T>(f[i]);
  }
}

__device__ inline void store8_q(int8_t *p, size_t left, const float (&f)[VEC]) {
  int8_t b[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i)
    b[i] = (int8_t)(int)fminf(fmaxf(rintf(f[i]), -127.f), 127.f);
  if (left >= VEC) {
    __builtin_memcpy(p, b, VEC);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if ((size_t)i < left) p[i] = b[i];
  }
}

// Sum of a and maximum of b over the `TPR` threads of a row; every thread of
// the row gets both.  TPR is a wave or a whole workgroup of more.
template <int TPR>
__device__ inline void row_reduce(float &a, float &b, float *lds) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    a += __shfl_xor(a, m);
    b = fmaxf(b, __shfl_xor(b, m));
  }
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    const int wave = threadIdx.x / 64;
    __syncthreads();  // (the words may still be read for the row before)
    if (threadIdx.x % 64 == 0) {
      lds[2 * wave] = a;
      lds[2 * wave + 1] = b;
    }
    __syncthreads();
    a = lds[0];
    b = lds[1];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      a += lds[2 * w];
      b = fmaxf(b, lds[2 * w + 1]);
    }
  }
}

// 127 / max for the scaling to 8 bits, as two factors so that neither
// overflows where the maximum is tiny.
__device__ inline void q_factors(float top, float &f0, float &f1) {
  f0 = top < 0x1p-100f ? 0x1p100f : 1.f;
  f1 = top > 0.f ? 127.f / (top * f0) : 0.f;
}

// One row per TPR threads, NV vectors of a thread in registers; NV = 0: rows
// of any length, read again where they are used.  NORM false: x alone to
// 8 bits.
template <class T, class W, int TPR, int NV, bool NORM>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) k_rms_norm(NormArgs a) {
  constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;
  __shared__ float lds[2 * 16];
  const size_t row = (size_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  if (row >= a.rows) return;  // (whole waves: a row of fewer threads is one wave)
  const int t = threadIdx.x % TPR;
  const size_t dim = a.dim;
  const T *x = (const T *)a.x.p + row * a.x.stride;
  const T *r = a.residual.p ? (const T *)a.residual.p + row * a.residual.stride : nullptr;
  const W *w = (const W *)a.weight;
  T *ho = a.h.p ? (T *)a.h.p + row * a.h.stride : nullptr;
  T *yo = a.y.p ? (T *)a.y.p + row * a.y.stride : nullptr;
  int8_t *qo = a.q.p ? (int8_t *)a.q.p + row * a.q.stride : nullptr;

  float sum = 0.f, top = 0.f;
  // h and h w of the vector at column c
  auto get = [&](size_t c, float (&h)[VEC], float (&hw)[VEC]) {
    load8(x + c, dim - c, h);
    if (NORM && r) {
      float s[VEC];
      load8(r + c, dim - c, s);
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[i] += s[i];
    }
    if (NORM && w) {
      float s[VEC];
      load8(w + c, dim - c, s);
#pragma unroll
      for (int i = 0; i < VEC; ++i) hw[i] = h[i] * s[i];
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) hw[i] = h[i];
    }
  };
  auto count = [&](const float (&h)[VEC], const float (&hw)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      // (a NaN reaches the sum, and the scale through it)
      sum = NORM ? fmaf(h[i], h[i], sum) : sum + h[i] * 0.f;
      top = fmaxf(top, fabsf(hw[i]));
    }
  };
  float f0, f1, inv = 1.f;
  auto finish = [&]() {
    row_reduce<TPR>(sum, top, lds);
    if (NORM) inv = 1.f / sqrtf(sum / (float)dim + a.eps);
    q_factors(top, f0, f1);
    if (t == 0) {
      if (a.scale) a.scale[row] = NORM ? top * inv / 127.f : top / 127.f + sum;
      if (NORM && a.inv_rms) a.inv_rms[row] = inv;
    }
  };
  auto put = [&](size_t c, const float (&hw)[VEC]) {
    float o[VEC];
    if (yo) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = hw[i] * inv;
      store8(yo + c, dim - c, o);
    }
    if (qo) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = hw[i] * f0 * f1;
      store8_q(qo + c, dim - c, o);
    }
  };

  if constexpr (NV > 0) {
    float hw[NV][VEC];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const size_t c = ((size_t)v * TPR + t) * VEC;
      if (c < dim) {
        float h[VEC];
        get(c, h, hw[v]);
        if (ho) store8(ho + c, dim - c, h);
        count(h, hw[v]);
      }
    }
    finish();
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const size_t c = ((size_t)v * TPR + t) * VEC;
      if (c < dim) put(c, hw[v]);
    }
  } else {
    float h[VEC], hw[VEC];
    for (size_t c = (size_t)t * VEC; c < dim; c += (size_t)TPR * VEC) {
      get(c, h, hw);
      count(h, hw);
    }
    finish();
    // h is written last, column by column as it is read: it may be x or residual
    for (size_t c = (size_t)t * VEC; c < dim; c += (size_t)TPR * VEC) {
      get(c, h, hw);
      if (ho) store8(ho + c, dim - c, h);
      put(c, hw);
    }
  }
}

template <class T, class W, bool NORM>
hipError_t norm_by_size(const NormArgs &a, hipStream_t st) {
  auto go = [&](auto kernel, int tpr) {
    const int per = tpr < 256 ? 256 / tpr : 1;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.rows + per - 1) / per)),
                       dim3(tpr < 256 ? 256 : tpr), 0, st, a);
    return hipGetLastError();
  };
  const size_t d = a.dim;
  if (d <= 64 * VEC) return go(k_rms_norm<T, W, 64, 1, NORM>, 64);
  if (d <= 256 * VEC) return go(k_rms_norm<T, W, 256, 1, NORM>, 256);
  if (d <= 256 * VEC * 2) return go(k_rms_norm<T, W, 256, 2, NORM>, 256);
  if (d <= 256 * VEC * 4) return go(k_rms_norm<T, W, 256, 4, NORM>, 256);
  if (d <= 1024 * VEC * 2) return go(k_rms_norm<T, W, 1024, 2, NORM>, 1024);
  return go(k_rms_norm<T, W, 1024, 0, NORM>, 1024);
}

template <class T>
__global__ void __launch_bounds__(256)
k_dequantize_rows(const int8_t *__restrict__ q, size_t q_stride, const float *__restrict__ scale,
                  size_t dim, T *__restrict__ out, size_t out_stride, size_t rows) {
  // a wave's 64 vectors run along a row; blockIdx.y counts pieces of rows
  const size_t c = ((size_t)blockIdx.x * 64 + threadIdx.x % 64) * VEC;
  if (c >= dim) return;
  for (size_t row = (size_t)blockIdx.y * 4 + threadIdx.x / 64; row < rows;
       row += (size_t)gridDim.y * 4) {
    const float s = scale[row];
    float f[VEC];
    load8(q + row * q_stride + c, dim - c, f);
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] *= s;
    store8(out + row * out_stride + c, dim - c, f);
  }
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs &a, hipStream_t st) {
  const bool wf = a.weight && a.weight_dtype == ROSETTA_F32;
  switch (a.dtype) {
    case ROSETTA_F32: return norm_by_size<float, float, true>(a, st);
    case ROSETTA_BF16:
      return wf ? norm_by_size<bf16, float, true>(a, st) : norm_by_size<bf16, bf16, true>(a, st);
    default:
      return wf ? norm_by_size<f16, float, true>(a, st) : norm_by_size<f16, f16, true>(a, st);
  }
}

hipError_t launch_quantize_rows(const NormArgs &a, hipStream_t st) {
  switch (a.dtype) {
    case ROSETTA_F32: return norm_by_size<float, float, false>(a, st);
    case ROSETTA_BF16: return norm_by_size<bf16, bf16, false>(a, st);
    default: return norm_by_size<f16, f16, false>(a, st);
  }
}

hipError_t launch_dequantize_rows(const int8_t *q, size_t q_stride, const float *scale, int dtype,
                                  size_t rows, size_t dim, Rows out, hipStream_t st) {
  const size_t gx = (dim + 64 * VEC - 1) / (64 * VEC);
  size_t gy = (rows + 3) / 4;
  gy = gy > 32768 ? 32768 : gy;
  auto go = [&](auto *o) {
    using T = std::remove_pointer_t<decltype(o)>;
    hipLaunchKernelGGL(k_dequantize_rows<T>, dim3((unsigned)gx, (unsigned)gy), dim3(256), 0, st, q,
                       q_stride, scale, dim, o, out.stride, rows);
    return hipGetLastError();
  };
  switch (dtype) {
    case ROSETTA_F32: return go((float *)out.p);
    case ROSETTA_BF16: return go((bf16 *)out.p);
    default: return go((f16 *)out.p);
  }
}

// ---------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------

namespace {

constexpr size_t BACK_GROUPS = 512;  // two workgroups of rows per CU

// A workgroup takes rows blockIdx.x, + gridDim.x, ..; each thread keeps the sums
// over rows of its columns' gy h inv_rms and writes them to the workgroup's
// row of `partial`, which k_sum_partial adds up in order.  NV = 0: rows of any
// length; the sums are then kept in `partial` itself.
template <class T, class W, int TPR, int NV>
__global__ void __launch_bounds__(TPR) k_rms_norm_backward(NormBackArgs a) {
  __shared__ float lds[2 * 16];
  const int t = threadIdx.x;
  const size_t dim = a.dim;
  const W *w = (const W *)a.weight;
  float *part = a.partial ? a.partial + (size_t)blockIdx.x * dim : nullptr;
  constexpr int NS = NV > 0 ? NV : 1;
  float sums[NS][VEC];
#pragma unroll
  for (int v = 0; v < NS; ++v)
#pragma unroll
    for (int i = 0; i < VEC; ++i) sums[v][i] = 0.f;

  for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *gy = (const T *)a.gy.p + row * a.gy.stride;
    const T *gh = a.gh.p ? (const T *)a.gh.p + row * a.gh.stride : nullptr;
    const T *h = (const T *)a.h.p + row * a.h.stride;
    T *gx = (T *)a.gx.p + row * a.gx.stride;
    const float inv = a.inv_rms[row];
    float dot = 0.f, none = 0.f;
    // h and gy w of the vector at column c, and the terms of gweight
    auto get = [&](size_t c, float (&hv)[VEC], float (&g)[VEC], float (&s)[VEC], bool add) {
      load8(gy + c, dim - c, g);
      load8(h + c, dim - c, hv);
      if (add) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[i] = fmaf(g[i] * inv, hv[i], s[i]);
      }
      if (w) {
        float u[VEC];
        load8(w + c, dim - c, u);
#pragma unroll
        for (int i = 0; i < VEC; ++i) g[i] *= u[i];
      }
    };
    auto put = [&](size_t c, const float (&hv)[VEC], const float (&g)[VEC], float k) {
      float o[VEC];
      if (gh) {
        load8(gh + c, dim - c, o);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) o[i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] += g[i] * inv - hv[i] * k;
      store8(gx + c, dim - c, o);
    };
    if constexpr (NV > 0) {
      float hv[NV][VEC], g[NV][VEC];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) {
          get(c, hv[v], g[v], sums[v], true);
#pragma unroll
          for (int i = 0; i < VEC; ++i) dot = fmaf(g[v][i], hv[v][i], dot);
        }
      }
      row_reduce<TPR>(dot, none, lds);
      const float k = dot * inv * inv * inv / (float)dim;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) put(c, hv[v], g[v], k);
      }
    } else {
      float hv[VEC], g[VEC], s[VEC];
      for (size_t c = (size_t)t * VEC; c < dim; c += (size_t)TPR * VEC) {
        if (part && row != blockIdx.x) {
          load8(part + c, dim - c, s);
        } else {
#pragma unroll
          for (int i = 0; i < VEC; ++i) s[i] = 0.f;
        }
        get(c, hv, g, s, true);
        if (part) store8(part + c, dim - c, s);
#pragma unroll
        for (int i = 0; i < VEC; ++i) dot = fmaf(g[i], hv[i], dot);
      }
      row_reduce<TPR>(dot, none, lds);
      const float k = dot * inv * inv * inv / (float)dim;
      for (size_t c = (size_t)t * VEC; c < dim; c += (size_t)TPR * VEC) {
        get(c, hv, g, s, false);
        put(c, hv, g, k);
      }
    }
  }
  if constexpr (NV > 0) {
    if (part) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) store8(part + c, dim - c, sums[v]);
      }
    }
  }
}

// gweight[c] = sum of partial[g][c] over the groups: 64 columns of a workgroup,
// each of its 16 waves a sixteenth of the groups, joined in order.
__global__ void __launch_bounds__(1024)
k_sum_partial(const float *__restrict__ partial, size_t groups, size_t dim,
              float *__restrict__ out) {
  __shared__ float lds[16][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const size_t c = (size_t)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < dim)
    for (size_t g = wave; g < groups; g += 16) s += partial[g * dim + c];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < dim) {
    for (int w = 1; w < 16; ++w) s += lds[w][lane];
    out[c] = s;
  }
}

template <class T, class W>
hipError_t back_by_size(const NormBackArgs &a, hipStream_t st) {
  const size_t groups = norm_back_groups(a.rows);
  auto go = [&](auto kernel, int tpr) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(tpr), 0, st, a);
    return hipGetLastError();
  };
  const size_t d = a.dim;
  hipError_t e;
  if (d <= 64 * VEC) e = go(k_rms_norm_backward<T, W, 64, 1>, 64);
  else if (d <= 256 * VEC) e = go(k_rms_norm_backward<T, W, 256, 1>, 256);
  else if (d <= 256 * VEC * 2) e = go(k_rms_norm_backward<T, W, 256, 2>, 256);
  else if (d <= 512 * VEC * 2) e = go(k_rms_norm_backward<T, W, 512, 2>, 512);
  else if (d <= 1024 * VEC * 2) e = go(k_rms_norm_backward<T, W, 1024, 2>, 1024);
  else e = go(k_rms_norm_backward<T, W, 1024, 0>, 1024);
  if (e != hipSuccess || !a.gweight) return e;
  hipLaunchKernelGGL(k_sum_partial, dim3((unsigned)((d + 63) / 64)), dim3(1024), 0, st, a.partial,
                     groups, d, a.gweight);
  return hipGetLastError();
}

}  // namespace

size_t norm_back_groups(size_t rows) { return rows < BACK_GROUPS ? rows : BACK_GROUPS; }

hipError_t launch_rms_norm_backward(const NormBackArgs &a, hipStream_t st) {
  const bool wf = a.weight && a.weight_dtype == ROSETTA_F32;
  switch (a.dtype) {
    case ROSETTA_F32: return back_by_size<float, float>(a, st);
    case ROSETTA_BF16:
      return wf ? back_by_size<bf16, float>(a, st) : back_by_size<bf16, bf16>(a, st);
    default: return wf ? back_by_size<f16, float>(a, st) : back_by_size<f16, f16>(a, st);
  }
}

}  // namespace rosetta
