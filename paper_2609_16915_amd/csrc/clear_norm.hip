// Root-mean-square norm with the residual's addition and an 8-bit output,
// its gradient, and rows to 8 bits and back.
//
// All of it is bound by memory: one pass, every element read once and every
// result written once, a row held in registers between its reduction and its
// use.  One reduction serves both the norm and the 8-bit scale, since
//   y / scale = h w inv_rms / (max|h w| inv_rms / 127) = h w * (127 / max|h w|):
// the sum of h^2 and the maximum of |h w| are taken together, and q needs
// neither inv_rms nor a second pass.  Sums, the norm and scales are 32-bit floats;
// what is stored in fewer bits is rounded once, from them.
#include <algorithm>
#include <type_traits>

#include "clear.hpp"

namespace rosetta {

namespace {

constexpr int VEC = 8;  // elements of a thread's load: 16 bytes of bf16 or f16

template <class T>
__device__ inline float to_f(T v) { return (float)v; }
template <class T>
__device__ inline T from_f(float v) { return (T)v; }  // to nearest, ties to even

// Eight consecutive elements.  What is written goes past the caches (16384 x 4096
// to 8 bits and back to values: 115.9 us for 130.5).  The address may be any multiple of the
// element's size: the copy compiles to the widest loads, which the hardware
// takes unaligned.
template <class T>
struct __attribute__((packed, aligned(1))) Pack {
  T v[VEC];
};

// (How many elements are left of the row: all eight, known where the row is a
// whole number of vectors.)
struct Whole {
  __device__ constexpr operator size_t() const { return VEC; }
};

template <class T, class L>
__device__ inline void load8(const T *p, L left, float (&f)[VEC]) {
  if ((size_t)left >= VEC) {
    Pack<T> v;
    __builtin_memcpy(&v, p, sizeof v);
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = to_f(v.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = (size_t)i < (size_t)left ? to_f(p[i]) : 0.f;
  }
}

// The same as it lies, widened where it is used: a row's loads wait in few
// registers.
template <class T>
struct Raw {
  static constexpr int WORDS = sizeof(T) * VEC / 4;
  int w[WORDS];
  __device__ float operator[](int i) const {
    if constexpr (std::is_same_v<T, float>) {
      return __builtin_bit_cast(float, w[i]);
    } else if constexpr (std::is_same_v<T, bf16>) {
      return __builtin_bit_cast(float, i % 2 ? w[i / 2] & (int)0xffff0000 : w[i / 2] << 16);
    } else {
      using v2h = __attribute__((ext_vector_type(2))) _Float16;
      return (float)__builtin_bit_cast(v2h, w[i / 2])[i % 2];
    }
  }
};

// Asked for in one load, also where the row ends inside the vector: the row's last
// eight are then read, and settle() moves them down once they are there (a branch
// around each load would wait for the one before).  `dim`: the row's length.
template <class T, class L>
__device__ inline void load8_raw(const T *p, L left, size_t dim, Raw<T> &v) {
  if constexpr (std::is_same_v<L, Whole>) {
    __builtin_memcpy(&v, p, sizeof v);
  } else if (dim >= VEC) {
    __builtin_memcpy(&v, p - (left < VEC ? VEC - left : 0), sizeof v);
  } else {
    T e[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) e[i] = (size_t)i < (size_t)left ? p[i] : (T)0.f;
    __builtin_memcpy(&v, e, sizeof v);
  }
}
template <class T, class L>
__device__ inline void settle(L left, size_t dim, Raw<T> &v) {
  if constexpr (!std::is_same_v<L, Whole>) {
    if (left < VEC && dim >= VEC) {
      const int by = (int)(VEC - left);  // elements, zeros from above
      constexpr int W = Raw<T>::WORDS;
#pragma unroll
      for (int n = 4; n >= 1; n /= 2) {
        if (!(by & n)) continue;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          if (sizeof(T) == 2 && n == 1)
            v.w[i] = (int)((unsigned)v.w[i] >> 16) | (i + 1 < W ? v.w[i + 1] << 16 : 0);
          else
            v.w[i] = i + n * W / VEC < W ? v.w[i + n * W / VEC] : 0;
        }
      }
    }
  }
}

template <class T, class L>
__device__ inline void store8(T *p, L left, const float (&f)[VEC]) {
  if ((size_t)left >= VEC) {
    Pack<T> v;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v.v[i] = from_f<T>(f[i]);
    using v4u = __attribute__((ext_vector_type(4), aligned(2))) int;
#pragma unroll
    for (int i = 0; i < (int)(sizeof v / 16); ++i) {
      v4u w;
      __builtin_memcpy(&w, (const char *)&v + 16 * i, 16);
      __builtin_nontemporal_store(w, (v4u *)p + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if ((size_t)i < (size_t)left) p[i] = from_f<T>(f[i]);
  }
}

template <class L>
__device__ inline void store8_q(int8_t *p, L left, const float (&f)[VEC]) {
  int8_t b[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i)
    b[i] = (int8_t)(int)fminf(fmaxf(rintf(f[i]), -127.f), 127.f);
  if ((size_t)left >= VEC) {
    using v2u = __attribute__((ext_vector_type(2), aligned(1))) int;
    v2u w;
    __builtin_memcpy(&w, b, VEC);
    __builtin_nontemporal_store(w, (v2u *)p);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if ((size_t)i < (size_t)left) p[i] = b[i];
  }
}

// The larger of two, or NaN if either is (fmaxf gives the other one): one instruction.
__device__ inline float max_or_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Sum of a and maximum of b (NaN if any is) over the `TPR` threads of a row; every thread
// of the row gets both.  TPR is a power of two up to a wave, or a whole workgroup of
// more.
template <int TPR>
__device__ inline void row_reduce(float &a, float &b, float *lds) {
#pragma unroll
  for (int m = TPR < 64 ? TPR / 2 : 32; m >= 1; m >>= 1) {
    a += __shfl_xor(a, m);
    b = max_or_nan(b, __shfl_xor(b, m));
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
      b = max_or_nan(b, lds[2 * w + 1]);
    }
  }
}

// 127 / max for the scaling to 8 bits, as two factors so that neither
// overflows where the maximum is tiny.
__device__ inline void q_factors(float top, float &f0, float &f1) {
  f0 = top < 0x1p-100f ? 0x1p100f : 1.f;
  f1 = top > 0.f ? 127.f / (top * f0) : 0.f;
}

// TPR threads to a row and NV vectors of a thread in registers, rows one after
// the other with the next one's loads under way; NV = 0: rows of any length, read
// again where they are used.  NORM false: x alone to 8 bits.
//
// Bound by memory: 7 bytes an element in bf16 with residual, h and q.  16384 x 4096
// takes 88 us, 5.3 TB/s (a row per block without the next one's loads: 126 us).
template <class T, class W, int TPR, int NV, bool NORM, bool WHOLE>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) k_rms_norm(NormArgs a) {
  constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;
  __shared__ float lds[2 * 16];
  const size_t first = (size_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  const size_t step = (size_t)gridDim.x * ROWS;
  const int t = threadIdx.x % TPR;
  const size_t dim = a.dim;
  auto left = [&](size_t c) {
    if constexpr (WHOLE) return Whole{};
    else return dim - c;
  };
  const W *w = (const W *)a.weight;

  float sum, top, f0, f1, inv = 1.f;
  auto count = [&](const float (&h)[VEC], const float (&hw)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      // (a NaN of h or of the weight reaches the maximum, and the scale through it; an
      // infinity to 8 bits without the norm the sum, so that its scale is NaN)
      sum = NORM ? fmaf(h[i], h[i], sum) : sum + h[i] * 0.f;
      top = max_or_nan(top, fabsf(hw[i]));
    }
  };
  auto finish = [&](size_t row) {
    row_reduce<TPR>(sum, top, lds);
    if (NORM) inv = 1.f / sqrtf(sum / (float)dim + a.eps);
    q_factors(top, f0, f1);
    if (t == 0) {
      // (sum - sum: nothing, or NaN where the squares overflowed, inv then being 0)
      if (a.scale) a.scale[row] = NORM ? top * inv / 127.f + (sum - sum) : top / 127.f + sum;
      if (NORM && a.inv_rms) a.inv_rms[row] = inv;
    }
  };
  auto put = [&](size_t row, size_t c, const float (&hw)[VEC]) {
    float o[VEC];
    if (a.y.p) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = hw[i] * inv;
      store8((T *)a.y.p + row * a.y.stride + c, left(c), o);
    }
    if (a.q.p) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = hw[i] * f0 * f1;
      store8_q((int8_t *)a.q.p + row * a.q.stride + c, left(c), o);
    }
  };

  if constexpr (NV > 0) {
    Raw<T> xr[NV], rr[NV];
    Raw<W> wr[NV];
    auto ask = [&](size_t row) {
      const T *x = (const T *)a.x.p + row * a.x.stride;
      const T *r = (const T *)a.residual.p + row * a.residual.stride;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) {
          load8_raw(x + c, left(c), dim, xr[v]);
          if (NORM && a.residual.p) load8_raw(r + c, left(c), dim, rr[v]);
        }
      }
    };
    if (first < a.rows) ask(first);
    if (NORM && w) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) load8_raw(w + c, left(c), dim, wr[v]), settle(left(c), dim, wr[v]);
      }
    }
    for (size_t row = first; row < a.rows; row += step) {
      T *ho = (T *)a.h.p + row * a.h.stride;
      float hw[NV][VEC];
      sum = top = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) {
          float h[VEC];
          settle(left(c), dim, xr[v]);
          if (NORM && a.residual.p) settle(left(c), dim, rr[v]);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            h[i] = xr[v][i];
            if (NORM && a.residual.p) h[i] += rr[v][i];
            hw[v][i] = NORM && w ? h[i] * wr[v][i] : h[i];
          }
          if (a.h.p) store8(ho + c, left(c), h);
          count(h, hw[v]);
        }
      }
      if (row + step < a.rows) ask(row + step);
      finish(row);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) put(row, c, hw[v]);
      }
    }
  } else {
    for (size_t row = first; row < a.rows; row += step) {
      const T *x = (const T *)a.x.p + row * a.x.stride;
      const T *r = a.residual.p ? (const T *)a.residual.p + row * a.residual.stride : nullptr;
      T *ho = a.h.p ? (T *)a.h.p + row * a.h.stride : nullptr;
      float h[VEC], hw[VEC];
      // h and h w of the vector at column c
      auto get = [&](size_t c) {
        load8(x + c, left(c), h);
        if (NORM && r) {
          float s[VEC];
          load8(r + c, left(c), s);
#pragma unroll
          for (int i = 0; i < VEC; ++i) h[i] += s[i];
        }
        float s[VEC];
        if (NORM && w) load8(w + c, left(c), s);
#pragma unroll
        for (int i = 0; i < VEC; ++i) hw[i] = NORM && w ? h[i] * s[i] : h[i];
      };
      sum = top = 0.f;
      for (size_t c = (size_t)t * VEC; c < dim; c += (size_t)TPR * VEC) {
        get(c);
        count(h, hw);
      }
      finish(row);
      // h is written last, column by column as it is read: it may be x or residual
      for (size_t c = (size_t)t * VEC; c < dim; c += (size_t)TPR * VEC) {
        get(c);
        if (ho) store8(ho + c, left(c), h);
        put(row, c, hw);
      }
    }
  }
}

template <class T, class W, bool NORM, bool WHOLE>
hipError_t norm_by_size(const NormArgs &a, hipStream_t st) {
  auto go = [&](auto kernel, int tpr) {
    const int per = tpr < 256 ? 256 / tpr : 1;
    // four waves a SIMD: with their next rows under way they have enough to wait for
    const size_t most = 1024 / (tpr < 256 ? 256 : tpr) * (size_t)std::max(1, device_cus());
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(most, (a.rows + per - 1) / per)),
                       dim3(tpr < 256 ? 256 : tpr), 0, st, a);
    return hipGetLastError();
  };
  const size_t d = a.dim;
  if (d <= 64 * VEC) return go(k_rms_norm<T, W, 64, 1, NORM, WHOLE>, 64);
  // (32768 x 1024 to 8 bits and back: 55 us for 72 with 256 threads to a row)
  if (d <= 64 * VEC * 2) return go(k_rms_norm<T, W, 64, 2, NORM, WHOLE>, 64);
  if (d <= 256 * VEC) return go(k_rms_norm<T, W, 256, 1, NORM, WHOLE>, 256);
  if (d <= 256 * VEC * 2) return go(k_rms_norm<T, W, 256, 2, NORM, WHOLE>, 256);
  if (d <= 256 * VEC * 4) return go(k_rms_norm<T, W, 256, 4, NORM, WHOLE>, 256);
  if (d <= 1024 * VEC * 2) return go(k_rms_norm<T, W, 1024, 2, NORM, WHOLE>, 1024);
  return go(k_rms_norm<T, W, 1024, 0, NORM, WHOLE>, 1024);
}

template <class T, class W, bool NORM>
hipError_t norm_by_length(const NormArgs &a, hipStream_t st) {
  return a.dim % VEC ? norm_by_size<T, W, NORM, false>(a, st) : norm_by_size<T, W, NORM, true>(a, st);
}

// Bound by memory: 3 bytes an element to bf16; 16384 x 4096 takes 35 us.
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
    case ROSETTA_F32: return norm_by_length<float, float, true>(a, st);
    case ROSETTA_BF16:
      return wf ? norm_by_length<bf16, float, true>(a, st) : norm_by_length<bf16, bf16, true>(a, st);
    default:
      return wf ? norm_by_length<f16, float, true>(a, st) : norm_by_length<f16, f16, true>(a, st);
  }
}

hipError_t launch_quantize_rows(const NormArgs &a, hipStream_t st) {
  switch (a.dtype) {
    case ROSETTA_F32: return norm_by_length<float, float, false>(a, st);
    case ROSETTA_BF16: return norm_by_length<bf16, bf16, false>(a, st);
    default: return norm_by_length<f16, f16, false>(a, st);
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

constexpr size_t BACK_GROUPS = 512;  // two workgroups of rows per CU (three: 56.4 us for 53.8)

// With y = h inv w, inv = (mean h^2 + eps)^(-1/2):
//   gx = gh + inv gy w - h inv^3 mean(gy w h),  gweight = sum over rows of gy h inv.
//
// A workgroup takes rows in turn, one at a time or, up to a wave's to each, as many
// as its 256 threads hold; each thread keeps the sums
// over rows of its columns' gy h inv_rms and writes them to the workgroup's
// row of `partial`, which k_sum_partial adds up in order.  NV = 0: rows of any
// length; the sums are then kept in `partial` itself.
//
// Bound by memory: 8 bytes an element in bf16.  8192 x 4096 takes 53 us with the
// sums, 5.0 TB/s (without the next row's loads under way 113 us: eight waves a CU
// wait for a row, reduce it and write it, in turn).
template <class T, class W, int TPR, int NV, bool WHOLE>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) k_rms_norm_backward(NormBackArgs a) {
  constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;
  __shared__ float lds[ROWS > 1 ? 256 * NV * VEC : 2 * 16];
  const size_t first = (size_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  const size_t step = (size_t)gridDim.x * ROWS;
  const int t = threadIdx.x % TPR;
  const size_t dim = a.dim;
  auto left = [&](size_t c) {
    if constexpr (WHOLE) return Whole{};
    else return dim - c;
  };
  const W *w = (const W *)a.weight;
  float *part = a.partial ? a.partial + (size_t)blockIdx.x * dim : nullptr;
  constexpr int NS = NV > 0 ? NV : 1;
  float sums[NS][VEC];
#pragma unroll
  for (int v = 0; v < NS; ++v)
#pragma unroll
    for (int i = 0; i < VEC; ++i) sums[v][i] = 0.f;

  float none = 0.f;
  if constexpr (NV > 0) {
    Raw<T> yr[NV], hr[NV], gr[NV];
    Raw<W> wr[NV];
    float inv_next = 0.f;
    auto ask = [&](size_t row) {
      const T *gy = (const T *)a.gy.p + row * a.gy.stride;
      const T *h = (const T *)a.h.p + row * a.h.stride;
      inv_next = a.inv_rms[row];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) {
          load8_raw(gy + c, left(c), dim, yr[v]);
          load8_raw(h + c, left(c), dim, hr[v]);
        }
      }
    };
    // (gh is used last, so it is asked for once the row before is written and stays as
    // it lies: widened ahead with the others, rows of four vectors a thread take more
    // registers still, 1258 x 16320 in 32 bits 148 us for 106.  Those of 32 bits, and
    // ragged ones of 16, do not fit as it is: 36 to 208 bytes of a thread's values go
    // through scratch memory, 3.1 TB/s at that size.)
    auto ask_gh = [&](size_t row) {
      const T *gh = (const T *)a.gh.p + row * a.gh.stride;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) load8_raw(gh + c, left(c), dim, gr[v]);
      }
    };
    if (first < a.rows) ask(first);
    if (first < a.rows && a.gh.p) ask_gh(first);
    if (w) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) load8_raw(w + c, left(c), dim, wr[v]), settle(left(c), dim, wr[v]);
      }
    }
    for (size_t row = first; row < a.rows; row += step) {
      T *gx = (T *)a.gx.p + row * a.gx.stride;
      const float inv = inv_next;
      float hv[NV][VEC], g[NV][VEC], dot = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) {
          settle(left(c), dim, yr[v]);
          settle(left(c), dim, hr[v]);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            hv[v][i] = hr[v][i];
            g[v][i] = yr[v][i];
            sums[v][i] = fmaf(g[v][i] * inv, hv[v][i], sums[v][i]);
            if (w) g[v][i] *= wr[v][i];
            dot = fmaf(g[v][i], hv[v][i], dot);
          }
        }
      }
      if (row + step < a.rows) ask(row + step);
      row_reduce<TPR>(dot, none, lds);
      const float k = dot * inv * inv * inv / (float)dim;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) {
          float o[VEC];
          if (a.gh.p) settle(left(c), dim, gr[v]);
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            o[i] = (a.gh.p ? gr[v][i] : 0.f) + (g[v][i] * inv - hv[v][i] * k);
          store8(gx + c, left(c), o);
        }
      }
      if (a.gh.p && row + step < a.rows) ask_gh(row + step);
    }
  } else {
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
      const T *gy = (const T *)a.gy.p + row * a.gy.stride;
      const T *gh = a.gh.p ? (const T *)a.gh.p + row * a.gh.stride : nullptr;
      const T *h = (const T *)a.h.p + row * a.h.stride;
      T *gx = (T *)a.gx.p + row * a.gx.stride;
      const float inv = a.inv_rms[row];
      float hv[VEC], g[VEC], s[VEC], dot = 0.f;
      // h and gy w of the vector at column c, and the terms of gweight
      auto get = [&](size_t c, bool add) {
        load8(gy + c, left(c), g);
        load8(h + c, left(c), hv);
        if (add) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) s[i] = fmaf(g[i] * inv, hv[i], s[i]);
        }
        if (w) {
          float u[VEC];
          load8(w + c, left(c), u);
#pragma unroll
          for (int i = 0; i < VEC; ++i) g[i] *= u[i];
        }
      };
      for (size_t c = (size_t)t * VEC; c < dim; c += (size_t)TPR * VEC) {
        if (part && row != blockIdx.x) {
          load8(part + c, left(c), s);
        } else {
#pragma unroll
          for (int i = 0; i < VEC; ++i) s[i] = 0.f;
        }
        get(c, true);
        if (part) store8(part + c, left(c), s);
#pragma unroll
        for (int i = 0; i < VEC; ++i) dot = fmaf(g[i], hv[i], dot);
      }
      row_reduce<TPR>(dot, none, lds);
      const float k = dot * inv * inv * inv / (float)dim;
      for (size_t c = (size_t)t * VEC; c < dim; c += (size_t)TPR * VEC) {
        get(c, false);
        float o[VEC];
        if (gh) load8(gh + c, left(c), o);
#pragma unroll
        for (int i = 0; i < VEC; ++i) o[i] = (gh ? o[i] : 0.f) + g[i] * inv - hv[i] * k;
        store8(gx + c, left(c), o);
      }
    }
  }
  if constexpr (ROWS > 1) {
    if (part) {
      // the sums of the rows side by side, in order
      constexpr int COLUMNS = TPR * NV * VEC;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          lds[threadIdx.x / TPR * COLUMNS + (v * TPR + t) * VEC + i] = sums[v][i];
      __syncthreads();
      for (int c = threadIdx.x; c < COLUMNS && c < (int)dim; c += 256) {
        float s = lds[c];
#pragma unroll
        for (int i = 1; i < ROWS; ++i) s += lds[i * COLUMNS + c];
        part[c] = s;
      }
    }
  } else if constexpr (NV > 0) {
    if (part) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const size_t c = ((size_t)v * TPR + t) * VEC;
        if (c < dim) store8(part + c, left(c), sums[v]);
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
  if (c < dim) {
#pragma unroll 8
    for (size_t g = wave; g < groups; g += 16) s += partial[g * dim + c];
  }
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < dim) {
    for (int w = 1; w < 16; ++w) s += lds[w][lane];
    out[c] = s;
  }
}

template <class T, class W, bool WHOLE>
hipError_t back_by_size(const NormBackArgs &args, hipStream_t st) {
  NormBackArgs a = args;
  size_t groups = 1;
  auto go = [&](auto kernel, int tpr) {
    // Four rows to a group at least once there is one to a CU: the joining reads as
    // much as a row per group.  One group alone writes the sums themselves (up to
    // four rows: one after the other they cost less than the joining's launch).
    const size_t side = std::max(1, 256 / tpr), turns = (a.rows + side - 1) / side;
    const size_t quarter = side > 1 ? turns : (turns + 3) / 4;
    groups = a.rows <= 4 ? 1 : std::max(quarter, std::min(turns, (size_t)std::max(1, device_cus())));
    groups = std::min(norm_back_groups(a.rows), groups);
    if (groups == 1) a.partial = a.gweight;
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(tpr < 256 ? 256 : tpr), 0, st, a);
    return hipGetLastError();
  };
  const size_t d = a.dim;
  hipError_t e;
  // (24414 rows of 64: 15 us with the joining, the host's share, for 37 with a wave to
  // each and one to a workgroup; 32768 of 1024: 44 for 68 with 256 threads to each)
  if (d <= 8 * VEC) e = go(k_rms_norm_backward<T, W, 8, 1, WHOLE>, 8);
  else if (d <= 16 * VEC) e = go(k_rms_norm_backward<T, W, 16, 1, WHOLE>, 16);
  else if (d <= 32 * VEC) e = go(k_rms_norm_backward<T, W, 32, 1, WHOLE>, 32);
  else if (d <= 64 * VEC) e = go(k_rms_norm_backward<T, W, 64, 1, WHOLE>, 64);
  else if (d <= 64 * VEC * 2) e = go(k_rms_norm_backward<T, W, 64, 2, WHOLE>, 64);
  else if (d <= 256 * VEC) e = go(k_rms_norm_backward<T, W, 256, 1, WHOLE>, 256);
  else if (d <= 256 * VEC * 2) e = go(k_rms_norm_backward<T, W, 256, 2, WHOLE>, 256);
  else if (d <= 512 * VEC * 2) e = go(k_rms_norm_backward<T, W, 512, 2, WHOLE>, 512);
  else if (d <= 512 * VEC * 4) e = go(k_rms_norm_backward<T, W, 512, 4, WHOLE>, 512);
  else e = go(k_rms_norm_backward<T, W, 1024, 0, WHOLE>, 1024);
  if (e != hipSuccess || !a.gweight || groups == 1) return e;
  hipLaunchKernelGGL(k_sum_partial, dim3((unsigned)((d + 63) / 64)), dim3(1024), 0, st, a.partial,
                     groups, d, a.gweight);
  return hipGetLastError();
}

template <class T, class W>
hipError_t back_by_length(const NormBackArgs &a, hipStream_t st) {
  return a.dim % VEC ? back_by_size<T, W, false>(a, st) : back_by_size<T, W, true>(a, st);
}

}  // namespace

size_t norm_back_groups(size_t rows) { return rows < BACK_GROUPS ? rows : BACK_GROUPS; }

hipError_t launch_rms_norm_backward(const NormBackArgs &a, hipStream_t st) {
  const bool wf = a.weight && a.weight_dtype == ROSETTA_F32;
  switch (a.dtype) {
    case ROSETTA_F32: return back_by_length<float, float>(a, st);
    case ROSETTA_BF16:
      return wf ? back_by_length<bf16, float>(a, st) : back_by_length<bf16, bf16>(a, st);
    default: return wf ? back_by_length<f16, float>(a, st) : back_by_length<f16, f16>(a, st);
  }
}

}  // namespace rosetta
