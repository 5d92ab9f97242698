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

template <class O, bool ALIGNED>
hipError_t by_size(const Q8Args &a, hipStream_t st) {
  constexpr int BX = 128, BY = 128;
  using Tl = Tile<int8_t, BX, BY, 2, 2>;
  const size_t blocks = (a.n + BX - 1) / BX * ((a.m + BY - 1) / BY);
  hipLaunchKernelGGL((k_q8_tile<O, ALIGNED, BX, BY, 2, 2>), dim3((unsigned)blocks),
                     dim3(Tl::THREADS), Tl::LDS, st, a);
  return hipGetLastError();
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
