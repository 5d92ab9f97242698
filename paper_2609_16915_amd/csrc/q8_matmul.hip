// 8-bit matrix product with a scale per token and per channel.
//
// X are the channels (b, contiguous in the output's rows), Y the tokens (a).
#include "mma_tile.hpp"

namespace rosetta {

namespace {

template <class O, bool ALIGNED, int BX, int BY, int WX, int WY>
__global__ void __launch_bounds__(64 * WX *WY) k_q8_tile(Q8Args a) {
  using Tl = Tile<int8_t, BX, BY, WX, WY>;
  extern __shared__ char lds[];
  const unsigned gx = (unsigned)((a.n + BX - 1) / BX), gy = (unsigned)((a.m + BY - 1) / BY);
  unsigned tx, ty;
  band_tile(xcd_block(blockIdx.x, gridDim.x), gx, gy, tx, ty);
  const Operand X{(const char *)a.b, (int64_t)a.b_stride, (int64_t)a.n, (int64_t)a.k};
  const Operand Y{(const char *)a.a, (int64_t)a.a_stride, (int64_t)a.m, (int64_t)a.k};
  v4i acc[Tl::TX][Tl::TY] = {};
  Tl::template run<ALIGNED>(X, Y, (int64_t)tx * BX, (int64_t)ty * BY, 0, (int64_t)a.k, lds, acc);

  const int64_t x0 = (int64_t)tx * BX + Tl::x_at();
  float bs[Tl::TX][4], bias[Tl::TX][4];
#pragma unroll
  for (int i = 0; i < Tl::TX; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t x = x0 + 4 * i + r;
      bs[i][r] = x < (int64_t)a.n ? a.b_scale[x] : 0.f;
      bias[i][r] = a.bias && x < (int64_t)a.n ? a.bias[x] : 0.f;
    }
#pragma unroll
  for (int j = 0; j < Tl::TY; ++j) {
    const int64_t y = (int64_t)ty * BY + Tl::y_at() + 16 * j;
    if (y >= (int64_t)a.m) continue;
    const float as = a.a_scale[y];
    O *out = (O *)a.out + y * (int64_t)a.out_stride;
    float f[4 * Tl::TX];
#pragma unroll
    for (int i = 0; i < Tl::TX; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        f[4 * i + r] = (float)acc[i][j][r] * as * bs[i][r] + bias[i][r];
    if (x0 < (int64_t)a.n) store_run(out + x0, (int64_t)a.n - x0, f);
  }
}

template <class O, int NX, int NY>
__global__ void __launch_bounds__(1024) k_q8_thin(Q8Args a) {
  using Th = Thin<int8_t, NX, NY>;
  extern __shared__ char lds[];
  const Operand X{(const char *)a.b, (int64_t)a.b_stride, (int64_t)a.n, (int64_t)a.k};
  const Operand Y{(const char *)a.a, (int64_t)a.a_stride, (int64_t)a.m, (int64_t)a.k};
  const int64_t x0 = (int64_t)xcd_block(blockIdx.x, gridDim.x) * 16 * NX;
  const v4i s = Th::run(X, Y, x0, lds);
  const int t = threadIdx.x;
  const int64_t x = x0 + 16 * (t / 64 % NX) + 4 * (t % 64 / 16), y = 16 * (t / 64 / NX) + t % 16;
  if (t >= Th::SUMS || y >= (int64_t)a.m || x >= (int64_t)a.n) return;
  const float as = a.a_scale[y];
  float f[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t c = x + r < (int64_t)a.n ? x + r : (int64_t)a.n - 1;
    f[r] = (float)s[r] * as * a.b_scale[c] + (a.bias ? a.bias[c] : 0.f);
  }
  store_run((O *)a.out + y * (int64_t)a.out_stride + x, (int64_t)a.n - x, f);
}

template <class O, bool ALIGNED, int BX, int BY, int WX, int WY>
hipError_t tile(const Q8Args &a, hipStream_t st) {
  using Tl = Tile<int8_t, BX, BY, WX, WY>;
  auto k = k_q8_tile<O, ALIGNED, BX, BY, WX, WY>;
  const hipError_t e = allow_lds(k, Tl::LDS);
  if (e != hipSuccess) return e;
  const size_t blocks = (a.n + BX - 1) / BX * ((a.m + BY - 1) / BY);
  hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(Tl::THREADS), Tl::LDS, st, a);
  return hipGetLastError();
}

template <class O, int NX, int NY>
hipError_t thin(const Q8Args &a, hipStream_t st) {
  using Th = Thin<int8_t, NX, NY>;
  hipLaunchKernelGGL((k_q8_thin<O, NX, NY>), dim3((unsigned)((a.n + 16 * NX - 1) / (16 * NX))),
                     dim3(Th::THREADS), Th::LDS, st, a);
  return hipGetLastError();
}

template <class O, bool ALIGNED>
hipError_t by_size(const Q8Args &a, hipStream_t st) {
  const size_t cus = (size_t)device_cus();
  auto blocks = [&](size_t x, size_t y) { return (a.n + x - 1) / x * ((a.m + y - 1) / y); };
  // Few tokens: bound by the channels' bytes, so every CU needs channels to read,
  // and the more each block has the less often the tokens are read.
  if (a.m <= 16)
    return blocks(64, 16) >= cus   ? thin<O, 4, 1>(a, st)
           : blocks(32, 16) >= cus ? thin<O, 2, 1>(a, st)
                                   : thin<O, 1, 1>(a, st);
  if (a.m <= 32) return blocks(32, 32) >= cus ? thin<O, 2, 2>(a, st) : thin<O, 1, 2>(a, st);
  if (a.m <= 64) return thin<O, 1, 4>(a, st);
  if (blocks(256, 256) >= cus) return tile<O, ALIGNED, 256, 256, 4, 2>(a, st);
  return tile<O, ALIGNED, 128, 128, 2, 2>(a, st);
}

template <class O>
hipError_t by_alignment(const Q8Args &a, hipStream_t st) {
  const Operand X{(const char *)a.b, (int64_t)a.b_stride, (int64_t)a.n, (int64_t)a.k};
  const Operand Y{(const char *)a.a, (int64_t)a.a_stride, (int64_t)a.m, (int64_t)a.k};
  return rows_aligned(X) && rows_aligned(Y) ? by_size<O, true>(a, st) : by_size<O, false>(a, st);
}

}  // namespace

hipError_t launch_q8_matmul(const Q8Args &a, hipStream_t st) {
  switch (a.out_dtype) {
    case ROSETTA_F32: return by_alignment<float>(a, st);
    case ROSETTA_BF16: return by_alignment<bf16>(a, st);
    default: return by_alignment<f16>(a, st);
  }
}

}  // namespace rosetta
