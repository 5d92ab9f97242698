// 8-bit matrix product with a scale per token and per channel.
//
// X are the channels (b, contiguous in the output's rows), Y the tokens (a).  The
// sums are exact in 32-bit integers, so they may be split at will: where there
// are few outputs for the length of their sums, blocks take parts of the sums,
// which k_q8_join adds up.
#include <algorithm>

#include "mma_tile.hpp"

namespace rosetta {

namespace {

// Four neighbouring outputs from their sums.
template <class O>
__device__ inline void put4(const Q8Args &a, int64_t y, int64_t x, v4i s) {
  const float as = a.a_scale[y];
  float f[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t c = x + r < (int64_t)a.n ? x + r : (int64_t)a.n - 1;
    f[r] = (float)s[r] * as * a.b_scale[c] + (a.bias ? a.bias[c] : 0.f);
  }
  store_run((O *)a.out + y * (int64_t)a.out_stride + x, (int64_t)a.n - x, f);
}

// Part `split` of the sums, rows of n rounded up to 4.
__device__ inline int *part_at(const Q8Args &a, int64_t ld, unsigned split, int64_t y, int64_t x) {
  return a.workspace + ((int64_t)split * (int64_t)a.m + y) * ld + x;
}

template <class O, int BX, int BY, int STAGES>
using Q8Tile = Tile<int8_t, BX, BY, 4, 2, STAGES, false, false, sizeof(O) == 2>;

// `run`: bytes of the rows per split, all of them in one.  8192 x 14336 x 4096 takes
// 386 us (2.49 POP/s; 235 MB of outputs leave at the ends of seven rounds of tiles).
// Outputs past the caches: 380 us there and 686 for 706 over 8192 bytes, but 236 for
// 190 over 16384 x 16384 x 128 and 61 for 58 over 4096 x 4096 x 4096; so through them.
template <class O, bool ALIGNED, int BX, int BY, int STAGES>
__global__ void __launch_bounds__(512) k_q8_tile(Q8Args a, int splits, int run) {
  using Tl = Q8Tile<O, BX, BY, STAGES>;
  // a lane's x: RUNS of RUN, 16 apart
  constexpr int RUN = sizeof(O) == 2 ? 4 * Tl::TX : 4, RUNS = 4 * Tl::TX / RUN;
  extern __shared__ char lds[];
  const unsigned gx = (unsigned)((a.n + BX - 1) / BX), gy = (unsigned)((a.m + BY - 1) / BY);
  const unsigned b = xcd_block(blockIdx.x, gridDim.x), split = b / (gx * gy);
  unsigned tx, ty;
  band_tile(b % (gx * gy), gx, gy, tx, ty);
  const int64_t k0 = (int64_t)split * run, k1 = k0 + run < (int64_t)a.k ? k0 + run : (int64_t)a.k;
  v4i acc[Tl::TX][Tl::TY];
  Tl::template run<ALIGNED>({{(const char *)a.b, (int64_t)a.b_stride, (int64_t)a.n, (int64_t)a.k},
                             {(const char *)a.a, (int64_t)a.a_stride, (int64_t)a.m, (int64_t)a.k},
                             (int64_t)tx * BX, (int64_t)ty * BY, k0, k1},
                            lds, acc);
  const int64_t x0 = (int64_t)tx * BX + Tl::x_at(), y0 = (int64_t)ty * BY + Tl::y_at();
  if (splits > 1) {
    const int64_t ld = ((int64_t)a.n + 3) / 4 * 4;
#pragma unroll
    for (int j = 0; j < Tl::TY; ++j) {
      if (y0 + 16 * j >= (int64_t)a.m) continue;
#pragma unroll
      for (int i = 0; i < Tl::TX; ++i)
        if (const int64_t x = x0 + (RUNS == 1 ? 4 : 16) * i; x < ld)
          *(v4i *)part_at(a, ld, split, y0 + 16 * j, x) = acc[i][j];
    }
    return;
  }
  const int64_t left = (int64_t)a.n - x0;
  if (left <= 0) return;
  // (all that is read, before anything is written: in between, every row would
  // wait for its own scale)
  float bs[RUNS][RUN], bias[RUNS][RUN] = {}, as[Tl::TY];
#pragma unroll
  for (int c = 0; c < RUNS; ++c) {
    load_run(a.b_scale + x0 + 16 * c, left - 16 * c, bs[c]);
    if (a.bias) load_run(a.bias + x0 + 16 * c, left - 16 * c, bias[c]);
  }
#pragma unroll
  for (int j = 0; j < Tl::TY; ++j) as[j] = y0 + 16 * j < (int64_t)a.m ? a.a_scale[y0 + 16 * j] : 0.f;
#pragma unroll
  for (int j = 0; j < Tl::TY; ++j) {
    const int64_t y = y0 + 16 * j;
    if (y >= (int64_t)a.m) continue;
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      float f[RUN];
#pragma unroll
      for (int i = 0; i < RUN; ++i)
        f[i] = (float)acc[c + i / 4][j][i % 4] * as[j] * bs[c][i] + bias[c][i];
      store_run((O *)a.out + y * (int64_t)a.out_stride + x0 + 16 * c, left - 16 * c, f);
    }
  }
}

// 33 tokens, 4096 x 14336: 13 us and 3 for joining its four parts; one token, 14336 x
// 4096: 12 us, 4.9 TB/s.
template <class O, int NX, int NY, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) k_q8_thin(Q8Args a, int splits, int run) {
  using Th = Thin<int8_t, NX, NY, WAVES>;
  extern __shared__ char lds[];
  const Operand X{(const char *)a.b, (int64_t)a.b_stride, (int64_t)a.n, (int64_t)a.k};
  const Operand Y{(const char *)a.a, (int64_t)a.a_stride, (int64_t)a.m, (int64_t)a.k};
  const unsigned b = xcd_block(blockIdx.x, gridDim.x), split = b % splits;
  const int64_t x0 = (int64_t)(b / splits) * 16 * NX, ld = ((int64_t)a.n + 3) / 4 * 4;
  const int k0 = (int)split * run, k1 = k0 + run < (int)a.k ? k0 + run : (int)a.k;
  Th::run(X, Y, x0, k0, k1, lds);
  for (int t = threadIdx.x; t < Th::SUMS; t += Th::THREADS) {
    const int64_t x = x0 + 16 * (t / 64 % NX) + 4 * (t % 64 / 16), y = 16 * (t / 64 / NX) + t % 16;
    if (y >= (int64_t)a.m || x >= (int64_t)a.n) continue;
    const v4i s = Th::sum(t, lds);
    if (splits > 1) *(v4i *)part_at(a, ld, split, y, x) = s;
    else put4<O>(a, y, x, s);
  }
}

// The parts added up, in order, and scaled.  Bound by memory and its launch.
template <class O>
__global__ void __launch_bounds__(256) k_q8_join(Q8Args a, int splits) {
  const int64_t ld = ((int64_t)a.n + 3) / 4 * 4, of = ld / 4 * (int64_t)a.m;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= of) return;
  const int64_t y = i / (ld / 4), x = i % (ld / 4) * 4;
  v4i s = *(const v4i *)part_at(a, ld, 0, y, x);
  for (int q = 1; q < splits; ++q) s += *(const v4i *)part_at(a, ld, q, y, x);
  put4<O>(a, y, x, s);
}

// How a product is cut up.  DEEP: small tiles with a CU each, whose steps are loaded
// four ahead (1024 x 4096 x 4096: 21 us for 25; where two tiles share a CU they cover
// for each other, 2200 TOP/s with two stages and 1908 with four).
enum class Cut { THIN, SMALL, DEEP, LARGE };
struct Plan {
  Cut cut;
  int nx, ny;  // THIN
  int splits, run;
};

size_t tiles(size_t a, size_t b) { return (a + b - 1) / b; }

Plan plan(size_t m, size_t n, size_t k) {
  const size_t cus = std::max(1, device_cus()), steps = tiles(k, STEP);
  Plan p{Cut::THIN, 1, 1, 1, 0};
  size_t parts = 1;
  // Few tokens: bound by the channels' bytes, so every CU needs channels to read,
  // and the more a block has the less often the tokens are read.  (Rows of less
  // than half a step for each of a block's waves leave most of them idle: tiles.)
  const bool thin = k >= 8 * STEP;
  if (thin && m <= 16) {
    p.nx = tiles(n, 64) >= cus ? 4 : tiles(n, 32) >= cus ? 2 : 1;
  } else if (thin && m <= 64) {
    // 64 channels a block; where those are too few for the chip, parts of their
    // sums, one round of blocks and 16 steps each at least (33 tokens, 4096 x 14336:
    // four parts 16.9 us, eight in two rounds 19.9; 16 channels in one part 24.5)
    p.nx = 4;
    p.ny = (int)tiles(m, 16);
    parts = std::max((size_t)1, std::min(cus / tiles(n, 64), steps / 16));
  } else {
    // Large tiles do a product at half the cost of small ones but come one to a
    // CU, small ones two: the smaller of the two times, in steps of a large one.
    const size_t nl = tiles(n, 256) * tiles(m, 256), ns = tiles(n, 128) * tiles(m, 128);
    const double large = (double)tiles(nl, cus) * (steps + 3);
    const double small = (ns <= cus ? 0.42 : 0.63 * ((double)ns / (2 * cus) + 0.5)) * (steps + 3);
    p.cut = large <= small ? Cut::LARGE : Cut::SMALL;
    // Too few small tiles for the chip: parts of their sums, as many as pay.  In us:
    // a step 0.55 while tiles have a CU each, 0.5 for each that shares one; the
    // joining 6 and what it writes and reads at 4 TB/s (1024 tokens, 4096 x 4096: one
    // part 24.3, two 34.4; 128 tokens, 4096 x 14336: 14 parts 24.9, one 71).
    if (p.cut == Cut::SMALL) {
      double best = 1e30;
      bool alone = false;
      for (size_t q = 1; q <= std::max((size_t)1, std::min(2 * cus / ns, steps / 8)); ++q) {
        const double each = ns * q <= cus ? 0.55 : 0.5 * (double)(ns * q) / (double)cus;
        const double t = (double)tiles(steps, q) * each +
                         (q > 1 ? 6 + (double)q * (double)m * (double)n * 8 / 4e6 : 0);
        if (t < best) best = t, parts = q, alone = ns * q <= cus;
      }
      if (alone) p.cut = Cut::DEEP;
    }
  }
  p.run = (int)(tiles(steps, parts) * STEP);
  p.splits = k ? (int)tiles(k, (size_t)p.run) : 1;
  return p;
}

template <class O, bool ALIGNED, int BX, int BY, int STAGES>
hipError_t tile(const Q8Args &a, const Plan &p, hipStream_t st) {
  using Tl = Q8Tile<O, BX, BY, STAGES>;
  auto k = k_q8_tile<O, ALIGNED, BX, BY, STAGES>;
  const size_t blocks = tiles(a.n, BX) * tiles(a.m, BY) * p.splits;
  if (!grid_fits(blocks, Tl::THREADS)) return hipErrorInvalidConfiguration;
  const hipError_t e = allow_lds(k, Tl::LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(Tl::THREADS), Tl::LDS, st, a, p.splits, p.run);
  return hipGetLastError();
}

template <class O, int NX, int NY, int WAVES>
hipError_t thin(const Q8Args &a, const Plan &p, hipStream_t st) {
  using Th = Thin<int8_t, NX, NY, WAVES>;
  auto k = k_q8_thin<O, NX, NY, WAVES>;
  const size_t blocks = tiles(a.n, 16 * NX) * p.splits;
  if (!grid_fits(blocks, Th::THREADS)) return hipErrorInvalidConfiguration;
  const hipError_t e = allow_lds(k, Th::LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(Th::THREADS), Th::LDS, st, a, p.splits, p.run);
  return hipGetLastError();
}

template <class O>
hipError_t launch(const Q8Args &a, hipStream_t st) {
  Plan p = plan(a.m, a.n, a.k);
  if (!a.workspace) {
    p.splits = 1;
    p.run = (int)a.k;
  }
  const Operand X{(const char *)a.b, (int64_t)a.b_stride, (int64_t)a.n, (int64_t)a.k};
  const Operand Y{(const char *)a.a, (int64_t)a.a_stride, (int64_t)a.m, (int64_t)a.k};
  const bool al = rows_aligned(X) && rows_aligned(Y);
  const size_t quads = tiles(a.n, 4) * a.m;
  if (p.splits > 1 && !grid_fits(tiles(quads, 256), 256)) return hipErrorInvalidConfiguration;
  hipError_t e = hipSuccess;
  switch (p.cut) {
    case Cut::THIN:
      switch (p.ny * 8 + p.nx) {
        case 9: e = thin<O, 1, 1, 16>(a, p, st); break;
        case 10: e = thin<O, 2, 1, 16>(a, p, st); break;
        case 12: e = thin<O, 4, 1, 16>(a, p, st); break;
        case 20: e = thin<O, 4, 2, 8>(a, p, st); break;
        case 28: e = thin<O, 4, 3, 8>(a, p, st); break;
        default: e = thin<O, 4, 4, 8>(a, p, st); break;
      }
      break;
    case Cut::SMALL:
      e = al ? tile<O, true, 128, 128, 2>(a, p, st) : tile<O, false, 128, 128, 2>(a, p, st);
      break;
    case Cut::DEEP:
      e = al ? tile<O, true, 128, 128, 4>(a, p, st) : tile<O, false, 128, 128, 2>(a, p, st);
      break;
    case Cut::LARGE:
      e = al ? tile<O, true, 256, 256, 2>(a, p, st) : tile<O, false, 256, 256, 2>(a, p, st);
      break;
  }
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(k_q8_join<O>, dim3((unsigned)tiles(quads, 256)), dim3(256), 0, st, a,
                     p.splits);
  return hipGetLastError();
}

}  // namespace

size_t q8_matmul_workspace(size_t m, size_t n, size_t k) {
  const Plan p = plan(m, n, k);
  return p.splits == 1 ? 0 : (size_t)p.splits * m * tiles(n, 4) * 4 * sizeof(int);
}

hipError_t launch_q8_matmul(const Q8Args &a, hipStream_t st) {
  switch (a.out_dtype) {
    case ROSETTA_F32: return launch<float>(a, st);
    case ROSETTA_BF16: return launch<bf16>(a, st);
    default: return launch<f16>(a, st);
  }
}

}  // namespace rosetta
