// Softmax cross entropy over a vocabulary from hidden states and head weights,
// and its gradients.  The logits live in registers only.
//
// Forward: tiles of logits (X: rows of w, Y: rows of h), each reduced to a
// maximum and a sum of exponentials per row and tile, joined afterwards: lse = log
// sum exp l, loss = lse - l[target].
// Backward, a piece of the vocabulary at a time: the tiles again, turned into
// gl = g (exp(l - lse) - one-hot) and stored for the piece, then gh += gl w and
// gw = gl^T h.  gl and w are read as they lie, turned on the way from LDS; h, small,
// is turned once.
//
// Products of 16-bit numbers summed in 32 bits; statistics in 32 bits.  gl alone is
// rounded to 16 bits between two steps, which keeps its products on the matrix
// pipes at full rate and costs at most half a unit in its last place.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mma_tile.hpp"

namespace rosetta {

namespace {

// Tiles of many rows, and of few rows or short ones; the latter's steps loaded four
// ahead where there is one to a CU at most.
template <int BX_, int BY_, int WX_, int WY_, int STAGES_>
struct Shape {
  static constexpr int BX = BX_, BY = BY_, WX = WX_, WY = WY_, THREADS = 64 * WX * WY;
  static constexpr int STAGES = STAGES_;
};
using Large = Shape<256, 256, 4, 2, 2>;
using Small = Shape<128, 128, 4, 2, 2>;
using Deep = Shape<128, 128, 4, 2, 4>;
template <class T, class S, bool YA = false>
using TileOf = Tile<T, S::BX, S::BY, S::WX, S::WY, S::STAGES, false, YA>;

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float GL_UP = 0x1p14f;  // largest |gl| as it is held
// Powers of two by which a row of gl that weighs little is held larger than the others.
template <class T>
constexpr int ROW_UP = std::is_same_v<T, f16> ? 24 : 0;
// Rows of h that are turned together: the pitch of what they give stays within a
// tile's offsets.
constexpr size_t H_ROWS = (size_t)1 << 20;
static_assert((int64_t)(H_ROWS * 2) <= MAX_LD && H_ROWS % 64 == 0, "");

size_t up(size_t a, size_t b) { return (a + b - 1) / b * b; }
size_t tiles(size_t a, size_t b) { return (a + b - 1) / b; }
// Small tiles that have a CU each.
size_t few_tiles() { return (size_t)std::max(1, device_cus()); }

struct Stat {
  float top, sum;
};

// What is taken off the logits before their exponentials: the maximum, or nothing where
// that is an infinity (the sum is then 0 or infinite, as it should be).
__device__ inline float level(float top) { return fabsf(top) == INFINITY ? 0.f : top; }

// (a, b) as one: sums of exponentials above the larger maximum
__device__ inline Stat join(Stat a, Stat b) {
  const float top = fmaxf(a.top, b.top);
  if (fabsf(top) == INFINITY) return {top, a.sum + b.sum};
  return {top, a.sum * __expf(a.top - top) + b.sum * __expf(b.top - top)};
}

__device__ inline bool counts(int64_t target, int64_t ignore, size_t vocab) {
  return target != ignore && target >= 0 && target < (int64_t)vocab;
}

// Row `row`, or the last where there is none: what is read for it is not used.
__device__ inline int64_t row_in(const LossArgs &a, int64_t row) {
  return row < (int64_t)a.rows ? row : (int64_t)a.rows - 1;
}

template <class T>
__device__ inline Operand w_rows(const LossArgs &a) {
  return {(const char *)a.w, (int64_t)(a.w_stride * sizeof(T)), (int64_t)a.vocab,
          (int64_t)(a.dim * sizeof(T))};
}
template <class T>
__device__ inline Operand h_rows(const LossArgs &a) {
  return {(const char *)a.h, (int64_t)(a.h_stride * sizeof(T)), (int64_t)a.rows,
          (int64_t)(a.dim * sizeof(T))};
}

// part[tile of x][row], and the logit of each row's target.  Bound by the matrix
// pipes under the power limit: 4096 rows of 4096 over 128000 in 3.07-3.16 ms from card
// to card, 1.36-1.40 PFLOP/s.
template <class T, class S, bool ALIGNED>
__global__ void __launch_bounds__(S::THREADS)
k_loss_tile(LossArgs a, Stat *__restrict__ part, float *__restrict__ at_target) {
  using Tl = TileOf<T, S>;
  constexpr int BX = S::BX, BY = S::BY, RUN = 4 * Tl::TX;
  extern __shared__ char lds[];
  const unsigned gx = (unsigned)((a.vocab + BX - 1) / BX), gy = (unsigned)((a.rows + BY - 1) / BY);
  unsigned tx, ty;
  band_tile(xcd_block(blockIdx.x, gridDim.x), gx, gy, tx, ty);
  int64_t target[Tl::TY];
  auto ask = [&] {
#pragma unroll
    for (int j = 0; j < Tl::TY; ++j)
      target[j] = a.targets[row_in(a, (int64_t)ty * BY + Tl::y_at() + 16 * j)];
  };
  if constexpr (Tl::ROOM) ask();
  v4f acc[Tl::TX][Tl::TY];
  Tl::template run<ALIGNED>({w_rows<T>(a), h_rows<T>(a), (int64_t)tx * BX, (int64_t)ty * BY, 0,
                             (int64_t)(a.dim * sizeof(T))},
                            lds, acc);
  const int64_t x0 = (int64_t)tx * BX + Tl::x_at();
  Stat *joint = (Stat *)lds;  // [S::WX][BY]
  if (x0 + RUN > (int64_t)a.vocab) {
#pragma unroll
    for (int i = 0; i < RUN; ++i)
      if (x0 + i >= (int64_t)a.vocab) {
#pragma unroll
        for (int j = 0; j < Tl::TY; ++j) acc[i / 4][j][i % 4] = -INFINITY;
      }
  }
  if constexpr (!Tl::ROOM) ask();
#pragma unroll
  for (int j = 0; j < Tl::TY; ++j) {
    const int y = Tl::y_at() + 16 * j;
    const int64_t row = (int64_t)ty * BY + y;
    const int64_t at = target[j] < 0 ? -1 : target[j] - x0;
    if (at >= 0 && at < RUN && x0 + at < (int64_t)a.vocab && row < (int64_t)a.rows) {
#pragma unroll
      for (int i = 0; i < RUN; ++i)
        if (at == i) at_target[row] = acc[i / 4][j][i % 4];
    }
    Stat s{-INFINITY, 0.f};
#pragma unroll
    for (int i = 0; i < RUN; ++i) s.top = fmaxf(s.top, acc[i / 4][j][i % 4]);
    const float low = level(s.top) * LOG2E;
#pragma unroll
    for (int i = 0; i < RUN; ++i)
      s.sum += __builtin_amdgcn_exp2f(fmaf(acc[i / 4][j][i % 4], LOG2E, -low));
#pragma unroll
    for (int m = 16; m <= 32; m <<= 1)
      s = join(s, Stat{__shfl_xor(s.top, m), __shfl_xor(s.sum, m)});
    if (threadIdx.x % 64 < 16) joint[(threadIdx.x / 64 % S::WX) * BY + y] = s;
  }
  __syncthreads();
  for (int y = threadIdx.x; y < BY; y += Tl::THREADS) {
    const int64_t row = (int64_t)ty * BY + y;
    if (row >= (int64_t)a.rows) break;
    Stat s = joint[y];
    for (int w = 1; w < S::WX; ++w) s = join(s, joint[w * BY + y]);
    part[(size_t)tx * a.rows + row] = s;
  }
}

// The same for at most 16 NY rows.  Bound by w's bytes: 8 rows of 4096 over 128000 in
// 180 us, 5.8 TB/s.
template <class T, int NX, int NY>
__global__ void __launch_bounds__(1024)
k_loss_thin(LossArgs a, Stat *__restrict__ part, float *__restrict__ at_target) {
  using Th = Thin<T, NX, NY, 16>;
  extern __shared__ char lds[];
  const int64_t bytes = (int64_t)a.dim * sizeof(T);
  const Operand X{(const char *)a.w, (int64_t)(a.w_stride * sizeof(T)), (int64_t)a.vocab, bytes};
  const Operand Y{(const char *)a.h, (int64_t)(a.h_stride * sizeof(T)), (int64_t)a.rows, bytes};
  const size_t tx = xcd_block(blockIdx.x, gridDim.x);
  const int64_t x0 = (int64_t)tx * 16 * NX;
  const int t = threadIdx.x;
  Th::run(X, Y, x0, 0, bytes, lds);
  v4f l = {0, 0, 0, 0};
  if (t < Th::SUMS) l = Th::sum(t, lds);
  const int64_t x = x0 + 16 * (t / 64 % NX) + 4 * (t % 64 / 16), row = 16 * (t / 64 / NX) + t % 16;
  Stat s{-INFINITY, 0.f};
  if (t < Th::SUMS && row < (int64_t)a.rows) {
    const int64_t target = a.targets[row];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (x + r >= (int64_t)a.vocab) l[r] = -INFINITY;
      if (x + r == target) at_target[row] = l[r];
      s.top = fmaxf(s.top, l[r]);
    }
    const float low = level(s.top);
#pragma unroll
    for (int r = 0; r < 4; ++r) s.sum += __expf(l[r] - low);
  }
#pragma unroll
  for (int m = 16; m <= 32; m <<= 1) s = join(s, Stat{__shfl_xor(s.top, m), __shfl_xor(s.sum, m)});
  Stat *joint = (Stat *)lds;  // [NX][16 NY]
  __syncthreads();            // (the waves' sums have been read)
  if (t < Th::SUMS && t % 64 < 16) joint[t / 64 % NX * 16 * NY + row] = s;
  __syncthreads();
  if (t < 16 * NY && t < (int64_t)a.rows) {
    s = joint[t];
    for (int i = 1; i < NX; ++i) s = join(s, joint[i * 16 * NY + t]);
    part[tx * a.rows + t] = s;
  }
}

// The tiles' parts joined, R rows to a block of 1024 threads.
template <int R>
__global__ void __launch_bounds__(1024)
k_loss_join(LossArgs a, const Stat *__restrict__ part, size_t nt,
            const float *__restrict__ at_target) {
  constexpr int P = 1024 / R, AHEAD = 8;
  __shared__ Stat lds[P][R];
  const int r = threadIdx.x % R, p = threadIdx.x / R;
  const size_t row = (size_t)blockIdx.x * R + r;
  Stat s{-INFINITY, 0.f};
  if (row < a.rows) {
    for (size_t t = p; t < nt; t += P * AHEAD) {
      Stat f[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        f[i] = t + i * P < nt ? part[(t + i * P) * a.rows + row] : Stat{-INFINITY, 0.f};
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) s = join(s, f[i]);
    }
  }
  lds[p][r] = s;
#pragma unroll
  for (int h = P / 2; h >= 1; h /= 2) {
    __syncthreads();
    if (p < h) lds[p][r] = s = join(s, lds[p + h][r]);
  }
  if (p == 0 && row < a.rows) {
    const float lse = s.top + logf(s.sum);
    a.lse[row] = lse;
    const int64_t target = a.targets[row];
    a.loss[row] = target == a.ignore_index ? 0.f
                  : counts(target, a.ignore_index, a.vocab) ? lse - at_target[row]
                                                           : NAN;
  }
}

// Factors of the rows of gl, coef[row], and what their products are multiplied
// by in the end, coef[rows] and coef[rows + 2 + row]; coef[rows + 1]: whether any of
// the latter is not 1.  gl is held in 16 bits as multiples of max |gloss| /
// GL_UP: the term -1 of a target is then exact in either type where all rows
// weigh the same (rounding gloss itself put one error on all of them: gradients
// off by 0.0026 of their norm, 0.0017 so), and f16 has room for probabilities
// down to 2^-28.  The largest of those that are finite: one that is not would be
// everybody's factor, and stays its own row's this way.  In f16 a row that weighs less
// than half of the largest is held up to 2^24 times larger for gh (at 2^-24 of the largest
// its probabilities below 2^-15 would be lost otherwise), and brought to the common factor
// for gw, which sums over the rows: half a step is 2^-39 of the largest factor there.
template <class T>
__device__ inline void loss_coef(const LossArgs &a, float *coef, float *lds) {
  const int threads = blockDim.x;
  constexpr int AHEAD = 8;
  // rows first, + threads, .. : gloss of those that count, else 0
  auto read = [&](size_t first, float (&g)[AHEAD]) {
    int64_t target[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const size_t t = first + (size_t)i * threads, in = t < a.rows ? t : a.rows - 1;
      target[i] = t < a.rows ? a.targets[in] : -1;
      g[i] = a.gloss[in];
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (!counts(target[i], a.ignore_index, a.vocab)) g[i] = 0.f;
  };
  float top = 0.f, g[AHEAD];
  for (size_t t = threadIdx.x; t < a.rows; t += (size_t)threads * AHEAD) {
    read(t, g);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (fabsf(g[i]) < INFINITY) top = fmaxf(top, fabsf(g[i]));
  }
  for (int m = 32; m >= 1; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = top;
  __syncthreads();
  for (int w = 0; w < threads / 64; ++w) top = fmaxf(top, lds[w]);
  const bool some = top > 0.f;
  bool unlike = false;
  for (size_t t = threadIdx.x; t < a.rows; t += (size_t)threads * AHEAD) {
    if (a.rows > (size_t)threads * AHEAD) read(t, g);  // (else they are still there)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const size_t row = t + (size_t)i * threads;
      if (row >= a.rows) continue;
      float c = some ? g[i] / top * GL_UP : g[i];
      if constexpr (ROW_UP<T> > 0) {
        int up = 0;
        if (some && c != 0.f && fabsf(c) < GL_UP) {
          (void)frexpf(c / GL_UP, &up);  // (its exponent, at most 0)
          up = up < -ROW_UP<T> ? ROW_UP<T> : -up;
        }
        c = ldexpf(c, up);
        coef[a.rows + 2 + row] = ldexpf(1.f, -up);
        unlike |= up != 0;
      }
      coef[row] = c;
    }
  }
  unlike = __syncthreads_or(unlike);
  if (threadIdx.x == 0) {
    coef[a.rows] = some ? top / GL_UP : 1.f;
    coef[a.rows + 1] = unlike ? 1.f : 0.f;
  }
}

// gl [rows][vp] of the vocabulary rows [v0, v0 + here), `w`, and of h, `here` rounded up to whole
// tiles, zeros beyond the vocabulary.  As k_loss_tile, and gl's bytes at the tiles'
// ends: 4096 x 4096 over 128000 in 3.3-3.4 ms.
template <class T, class S>
__global__ void __launch_bounds__(S::THREADS)
k_loss_grad_tile(LossArgs a, Operand w, Operand h, size_t v0, size_t here, size_t vp,
                 const float *__restrict__ coef, T *__restrict__ gl) {
  using Tl = TileOf<T, S>;
  constexpr int BX = S::BX, BY = S::BY, RUN = 4 * Tl::TX;
  extern __shared__ char lds[];
  const unsigned gx = (unsigned)((here + BX - 1) / BX), gy = (unsigned)((a.rows + BY - 1) / BY);
  unsigned tx, ty;
  band_tile(xcd_block(blockIdx.x, gridDim.x), gx, gy, tx, ty);
  // what the epilogue reads, all before it writes anything
  float coefs[Tl::TY], lses[Tl::TY];
  int64_t target[Tl::TY];
  auto ask = [&] {
#pragma unroll
    for (int j = 0; j < Tl::TY; ++j) {
      const int64_t row = row_in(a, (int64_t)ty * BY + Tl::y_at() + 16 * j);
      coefs[j] = coef[row];
      lses[j] = a.lse[row];
      target[j] = a.targets[row];
    }
  };
  if constexpr (Tl::ROOM) ask();
  v4f acc[Tl::TX][Tl::TY];
  Tl::template run<true>({w, h, (int64_t)tx * BX, (int64_t)ty * BY, 0, w.bytes}, lds, acc);
  const int64_t x0 = (int64_t)tx * BX + Tl::x_at();
  const int64_t left = (int64_t)a.vocab - (int64_t)v0 - x0;  // words of the run that exist
  if constexpr (!Tl::ROOM) ask();
#pragma unroll
  for (int j = 0; j < Tl::TY; ++j) {
    const int64_t row = (int64_t)ty * BY + Tl::y_at() + 16 * j;
    if (row >= (int64_t)a.rows) continue;
    const float c = coefs[j], lse = lses[j] * LOG2E;
    const int64_t at = target[j] < 0 ? -1 : target[j] - (int64_t)v0 - x0;
    float f[RUN];
    // (c = 0: a row that takes no part, whatever its logits are)
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      const float e = __builtin_amdgcn_exp2f(fmaf(acc[i / 4][j][i % 4], LOG2E, -lse));
      f[i] = c == 0.f ? 0.f : e * c;
    }
    if (at >= 0 && at < RUN) {
#pragma unroll
      for (int i = 0; i < RUN; ++i)
        if (at == i) f[i] -= c;
    }
    if (left < RUN) {
#pragma unroll
      for (int i = 0; i < RUN; ++i)
        if (i >= left) f[i] = 0.f;
    }
    store_run(gl + row * (int64_t)vp + x0, RUN, f);
  }
}

// Tile (bx, by) of out [cols][ld] = in [rows][cols] the other way round, zeros in
// columns [rows, ld) and for rows that are not `wanted`; ld a multiple of 8; 256
// threads.
template <class T, class Wanted>
__device__ inline void transpose(const T *in, size_t in_stride, size_t rows, size_t cols, T *out,
                                 size_t ld, size_t bx, size_t by, T (*lds)[72], Wanted wanted) {
  const size_t r0 = bx * 64, c0 = by * 64;
  const int l = threadIdx.x % 8 * 8;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = threadIdx.x / 8 + 32 * h;
    T v[8] = {};
    if (r0 + i < rows && wanted(r0 + i)) {
      const T *src = in + (r0 + i) * in_stride + c0 + l;
      if (c0 + l + 8 <= cols) {
        __builtin_memcpy(v, src, sizeof v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c0 + l + e < cols) v[e] = src[e];
      }
    }
    *(v4i *)&lds[i][l] = *(const v4i *)v;
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = threadIdx.x / 8 + 32 * h;
    T v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = lds[l + e][i];
    if (c0 + i < cols && r0 + l < ld) *(v4i *)(out + (c0 + i) * ld + r0 + l) = *(const v4i *)v;
  }
}

// Rows that lie so that tiles can take them: `ld` apart, a multiple of 8 and the
// next to their length, zeros at their ends.  Bound by memory.
template <class T>
__global__ void __launch_bounds__(256)
k_loss_pack(const T *__restrict__ in, size_t in_stride, size_t rows, size_t dim,
            T *__restrict__ out, size_t ld) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, row = i / (ld / 8), c = i % (ld / 8) * 8;
  if (row >= rows) return;
  *(v4i *)(out + row * ld + c) = load_frag((const char *)(in + row * in_stride), c * sizeof(T),
                                           dim * sizeof(T));
}

// What comes before the pieces: the factors (block 0), and h_t in tiles (the
// others; none where gw is not wanted), [dim][ld_t] for every H_ROWS rows.
template <class T>
__global__ void __launch_bounds__(256)
k_loss_begin(LossArgs a, float *__restrict__ coef, T *__restrict__ h_t, size_t ld_t) {
  __shared__ T lds[64][72];
  if (blockIdx.x == 0) {
    loss_coef<T>(a, coef, (float *)lds);
    return;
  }
  const size_t across = (a.rows + 63) / 64, b = blockIdx.x - 1;
  const size_t r0 = b % across * 64 / H_ROWS * H_ROWS;
  // (a row that takes no part, whatever it holds, is zeros: NaN times 0 is NaN)
  transpose((const T *)a.h + r0 * a.h_stride, a.h_stride, a.rows - r0, a.dim, h_t + r0 * a.dim, ld_t,
            b % across - r0 / 64, b / across, lds,
            [&](size_t row) { return counts(a.targets[r0 + row], a.ignore_index, a.vocab); });
}

// part[split][row][d] (+)= gl [rows][vp] times the piece's `here` rows of w: split s
// takes an equal run of them, perhaps none of the last.  4096 x 4096 over 128000 in
// 2.96-3.03 ms, 1.42-1.45 PFLOP/s (with w turned first 3.1 and 0.4 for turning it).
template <class T, class S>
__global__ void __launch_bounds__(S::THREADS)
k_loss_gh_tile(size_t rows, size_t dim, size_t vp, const T *__restrict__ gl, Operand w,
               float *__restrict__ part, size_t run, int add) {
  using Tl = Tile<T, S::BX, S::BY, S::WX, S::WY, 2, true>;
  constexpr int BX = S::BX, BY = S::BY;
  extern __shared__ char lds[];
  const unsigned gx = (unsigned)((dim + BX - 1) / BX), gy = (unsigned)((rows + BY - 1) / BY);
  const unsigned b = xcd_block(blockIdx.x, gridDim.x), split = b / (gx * gy);
  unsigned tx, ty;
  band_tile(b % (gx * gy), gx, gy, tx, ty);
  const int64_t ld = (int64_t)vp * sizeof(T), bytes = w.rows * (int64_t)sizeof(T);
  const int64_t k0 = (int64_t)(split * run * sizeof(T)), k1 = k0 + (int64_t)(run * sizeof(T));
  v4f acc[Tl::TX][Tl::TY];
  Tl::template run<true>({w, {(const char *)gl, ld, (int64_t)rows, bytes}, (int64_t)tx * BX,
                          (int64_t)ty * BY, k0, k1 < bytes ? k1 : bytes},
                         lds, acc);
  const int64_t x0 = (int64_t)tx * BX + Tl::x_at();
#pragma unroll
  for (int j = 0; j < Tl::TY; ++j) {
    const int64_t row = (int64_t)ty * BY + Tl::y_at() + 16 * j;
    if (row >= (int64_t)rows) continue;
#pragma unroll
    for (int i = 0; i < Tl::TX; ++i) {
      const int64_t x = x0 + 16 * i, left = (int64_t)dim - x;
      if (left <= 0) continue;
      float *out = part + ((size_t)split * rows + row) * dim + x;
      float f[4] = {};
      if (add) load_run(out, left, f);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] += acc[i][j][e];
      store_run(out, left, f);
    }
  }
}

// gl, `width` columns of it, to the rows' common factor; by all blocks of 256 threads.
// Where they have it already, the usual case, nothing but a word is read.
template <class T>
__device__ inline void common_factor(const float *coef, size_t rows, size_t width, size_t vp, T *gl) {
  if (coef[rows + 1] == 0.f) return;
  const size_t each = width / 8;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < rows * each;
       i += (size_t)gridDim.x * 256) {
    const size_t row = i / each;
    const float down = coef[rows + 2 + row];
    if (down == 1.f) continue;
    T v[8], *at = gl + row * vp + i % each * 8;
    *(v4i *)v = *(const v4i *)at;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)((float)v[e] * down);
    *(v4i *)at = *(const v4i *)v;
  }
}

template <class T>
__global__ void __launch_bounds__(256)
k_loss_common(const float *__restrict__ coef, size_t rows, size_t width, size_t vp,
              T *__restrict__ gl) {
  common_factor(coef, rows, width, vp, gl);
}

// The parts added up, four columns to each of 256 / P threads, P threads a run of the
// parts each.  (42 rows of 256, 180 parts: 4 us with 16, 27 with one.)  With `gl`, the
// last piece of it also goes to the common factor: a launch of its own would take 4 us.
template <class T, int P>
__global__ void __launch_bounds__(256)
k_loss_gh_join(const float *__restrict__ part, int splits, size_t rows, size_t dim,
               const float *__restrict__ coef, T *__restrict__ out, size_t out_stride,
               T *__restrict__ gl, size_t width, size_t vp) {
  constexpr int Q = 256 / P;
  if constexpr (ROW_UP<T> > 0) {
    if (gl) common_factor(coef, rows, width, vp, gl);
  }
  __shared__ float lds[P > 1 ? P : 1][Q][4];
  const size_t quads = (dim + 3) / 4, i = (size_t)blockIdx.x * Q + threadIdx.x % Q;
  const int p = threadIdx.x / Q, each = (splits + P - 1) / P;
  const size_t row = i / quads, c = i % quads * 4;
  const int64_t left = (int64_t)(dim - c);
  const bool in = i < quads * rows;
  float s[4] = {};
  if (in) {
    const int end = (p + 1) * each < splits ? (p + 1) * each : splits;
#pragma unroll 4
    for (int q = p * each; q < end; ++q) {
      float f[4];
      load_run(part + ((size_t)q * rows + row) * dim + c, left, f);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += f[e];
    }
  }
  if constexpr (P > 1) {
    __builtin_memcpy(lds[p][threadIdx.x % Q], s, sizeof s);
    __syncthreads();
    if (p > 0) return;
#pragma unroll
    for (int q = 1; q < P; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += lds[q][threadIdx.x % Q][e];
  }
  if (!in) return;
  const float back = coef[rows];
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] *= back;
  if constexpr (ROW_UP<T> > 0) {
    const float down = coef[rows + 2 + row];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] *= down;
  }
  store_run(out + row * out_stride + c, left, s);
}

// gw rows [v0, v0 + here) = gl [rows][vp] the other way, times h_t [dim][ld_t] of every
// H_ROWS rows.  4096 x 4096 over 128000 in 3.2-3.3 ms with gw's 1 GB, 1.30-1.34 PFLOP/s.
template <class T, class S, bool PAST>
__global__ void __launch_bounds__(S::THREADS)
k_loss_gw_tile(LossArgs a, size_t v0, size_t here, size_t vp, size_t ld_t,
               const float *__restrict__ coef, const T *__restrict__ gl,
               const T *__restrict__ h_t) {
  using Tl = TileOf<T, S, true>;
  constexpr int BX = S::BX, BY = S::BY, RUN = 4 * Tl::TX;
  extern __shared__ char lds[];
  const unsigned gx = (unsigned)((a.dim + BX - 1) / BX), gy = (unsigned)((here + BY - 1) / BY);
  unsigned tx, ty;
  band_tile(xcd_block(blockIdx.x, gridDim.x), gx, gy, tx, ty);
  const int64_t ld_h = (int64_t)(ld_t * sizeof(T)), ld_g = (int64_t)(vp * sizeof(T));
  const float back = coef[a.rows];
  v4f acc[Tl::TX][Tl::TY];
  Tl::clear(acc);
  for (size_t r0 = 0; r0 < a.rows; r0 += H_ROWS) {
    const size_t rows = a.rows - r0 < H_ROWS ? a.rows - r0 : H_ROWS;
    Tl::template add<true>({{(const char *)(h_t + r0 * a.dim), ld_h, (int64_t)a.dim, ld_h},
                            {(const char *)(gl + r0 * vp), ld_g, (int64_t)rows, ld_g},
                            (int64_t)tx * BX, (int64_t)ty * BY, 0, (int64_t)(rows * sizeof(T))},
                           lds, acc);
  }
  const int64_t x0 = (int64_t)tx * BX + Tl::x_at(), left = (int64_t)a.dim - x0;
  if (left <= 0) return;
#pragma unroll
  for (int j = 0; j < Tl::TY; ++j) {
    const int64_t v = (int64_t)v0 + (int64_t)ty * BY + Tl::y_at() + 16 * j;
    if (v >= (int64_t)a.vocab) continue;
    float f[RUN];
#pragma unroll
    for (int i = 0; i < RUN; ++i) f[i] = acc[i / 4][j][i % 4] * back;
    store_run<PAST>((T *)a.gw + v * (int64_t)a.gw_stride + x0, left, f);
  }
}

// Whether Thin takes the logits, bound by w's bytes like any other way, and w's rows
// in its blocks.  Short rows (less than half a step for each of a block's waves) would
// leave most of its waves idle; past 16 rows it pays where w is too few tiles for the
// chip (32 rows of 4096 over 8000: 19 us for 51; over 128000: 273 for 221).
bool thin(size_t rows, size_t dim, size_t vocab) {
  return 2 * dim >= 8 * STEP && (rows <= 16 || (rows <= 32 && tiles(vocab, 128) <= few_tiles()));
}
constexpr size_t thin_x(size_t rows) { return rows <= 16 ? 64 : 32; }
// Whether large tiles take the logits: one a CU at half the cost, small ones two,
// whose ends overlap; in steps of a large tile (777 rows of 768 over 50257: 421 us
// in all with small ones, 454 with large; 4096 of 4096 over 128000: 62 and 44 ms
// by this count).
bool large(size_t rows, size_t dim, size_t vocab) {
  const double steps = (double)tiles(2 * dim, STEP);
  const double l = (double)tiles(tiles(rows, 256) * tiles(vocab, 256), 256) * (steps + 4);
  const double s = 0.66 * ((double)(tiles(rows, 128) * tiles(vocab, 128)) / 512 + 0.5) * (steps + 2);
  return l <= s;
}
size_t forward_x(size_t rows, size_t dim, size_t vocab) {
  return thin(rows, dim, vocab) ? thin_x(rows) : large(rows, dim, vocab) ? Large::BX : Small::BX;
}

// Pieces of the vocabulary and what the workspace holds.
struct Plan {
  size_t vp, pieces, ld_t, splits, run;
  size_t ld, coef, gl, w, h, h_t, part, bytes;
};

template <class S>
Plan plan(size_t rows, size_t dim, size_t vocab) {
  constexpr size_t BX = S::BX, BY = S::BY;
  constexpr size_t BUDGET = (size_t)1 << 30;
  Plan p{};
  p.ld_t = up(std::min(rows, H_ROWS), 64);
  p.ld = up(dim, 8);
  const size_t column = 2 * (rows + p.ld);
  size_t vp = BUDGET / column / BX * BX;
  // (at most 2^20: a tile's rows of gl within 32-bit offsets of its first)
  vp = vp < BX ? BX : vp > ((size_t)1 << 20) ? (size_t)1 << 20 : vp;
  p.pieces = tiles(up(vocab, BX), vp);
  p.vp = up(tiles(vocab, p.pieces), BX);
  p.pieces = tiles(vocab, p.vp);
  // enough blocks for gh: its tiles are few, its sums long
  const size_t t = tiles(dim, BX) * tiles(rows, BY);
  size_t s = (BX == 256 ? 256 : 512) / t;
  const size_t most = p.vp / 512;
  s = s > most ? most : s;
  p.splits = s < 1 ? 1 : s;
  p.run = up(tiles(p.vp, p.splits), 64);
  p.splits = tiles(p.vp, p.run);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up(bytes, 256);
    return here;
  };
  p.coef = take((2 * rows + 2) * 4);
  p.gl = take(rows * p.vp * 2);
  p.w = take(p.ld * p.vp * 2);
  p.h = take(p.ld * rows * 2);
  p.h_t = take(tiles(rows, H_ROWS) * dim * p.ld_t * 2);
  p.part = take(p.splits * rows * dim * 4);
  p.bytes = at;
  return p;
}

bool aligned(const LossArgs &a) {
  const Operand X{(const char *)a.w, (int64_t)(a.w_stride * 2), (int64_t)a.vocab,
                  (int64_t)(a.dim * 2)};
  const Operand Y{(const char *)a.h, (int64_t)(a.h_stride * 2), (int64_t)a.rows,
                  (int64_t)(a.dim * 2)};
  return rows_aligned(X) && rows_aligned(Y);
}

// Launch of `kernel` with its LDS allowed, `e` the status so far; `dry`: only whether the
// grid holds it.
#define LAUNCH(KERNEL, BLOCKS, THREADS, LDS, ...)                                               \
  do {                                                                                          \
    const size_t blocks_ = BLOCKS;                                                              \
    if (e == hipSuccess && !grid_fits(blocks_, THREADS)) e = hipErrorInvalidConfiguration;      \
    if (e == hipSuccess && !dry) e = allow_lds(KERNEL, LDS);                                     \
    if (e == hipSuccess && !dry) {                                                              \
      hipLaunchKernelGGL(KERNEL, dim3((unsigned)blocks_), dim3(THREADS), LDS, st, __VA_ARGS__);  \
      e = hipGetLastError();                                                                    \
    }                                                                                           \
  } while (0)

template <class T>
hipError_t forward(const LossArgs &a, hipStream_t st, bool dry) {
  const size_t nx = tiles(a.vocab, forward_x(a.rows, a.dim, a.vocab));
  Stat *part = (Stat *)a.workspace;
  float *at_target = (float *)(part + nx * a.rows);
  hipError_t e = hipSuccess;
  auto tile = [&](auto shape) {
    using S = decltype(shape);
    auto k = aligned(a) ? k_loss_tile<T, S, true> : k_loss_tile<T, S, false>;
    LAUNCH(k, nx * tiles(a.rows, S::BY), S::THREADS, (TileOf<T, S>::LDS), a, part, at_target);
  };
  const bool few = thin(a.rows, a.dim, a.vocab);
  if (few && a.rows <= 16)
    LAUNCH((k_loss_thin<T, 4, 1>), nx, 1024, (Thin<T, 4, 1, 16>::LDS), a, part, at_target);
  else if (few)
    LAUNCH((k_loss_thin<T, 2, 2>), nx, 1024, (Thin<T, 2, 2, 16>::LDS), a, part, at_target);
  else if (large(a.rows, a.dim, a.vocab)) tile(Large{});
  else if (aligned(a) && nx * tiles(a.rows, Deep::BY) <= few_tiles()) tile(Deep{});
  else tile(Small{});
  // (few rows: more threads to each)
  if (a.rows <= 64) LAUNCH(k_loss_join<2>, tiles(a.rows, 2), 1024, 0, a, part, nx, at_target);
  else LAUNCH(k_loss_join<16>, tiles(a.rows, 16), 1024, 0, a, part, nx, at_target);
  return e;
}

template <class T, class S>
hipError_t backward(const LossArgs &a, hipStream_t st, bool dry) {
  constexpr size_t BX = S::BX, BY = S::BY;
  using Tl = TileOf<T, S>;
  const Plan p = plan<S>(a.rows, a.dim, a.vocab);
  char *ws = (char *)a.workspace;
  float *coef = (float *)(ws + p.coef), *part = (float *)(ws + p.part);
  T *gl = (T *)(ws + p.gl), *w_p = (T *)(ws + p.w), *h_p = (T *)(ws + p.h), *h_t = (T *)(ws + p.h_t);
  const bool al = aligned(a);
  hipError_t e = hipSuccess;
  LAUNCH(k_loss_begin<T>, 1 + (a.gw ? tiles(a.rows, 64) * tiles(a.dim, 64) : 0), 256, 0, a, coef, h_t,
         p.ld_t);
  // rows of h or of a piece of w as the tiles take them
  auto rows_of = [&](const void *at, size_t stride, size_t rows, T *packed) {
    const int64_t bytes = (int64_t)(p.ld * sizeof(T));
    if (al) return Operand{(const char *)at, (int64_t)(stride * sizeof(T)), (int64_t)rows, bytes};
    LAUNCH(k_loss_pack<T>, tiles(rows * (p.ld / 8), 256), 256, 0, (const T *)at, stride, rows, a.dim,
           packed, p.ld);
    return Operand{(const char *)packed, bytes, (int64_t)rows, bytes};
  };
  const Operand h = rows_of(a.h, a.h_stride, a.rows, h_p);
  for (size_t i = 0; i < p.pieces && e == hipSuccess; ++i) {
    const size_t v0 = i * p.vp, here = a.vocab - v0 < p.vp ? a.vocab - v0 : p.vp;
    const Operand w = rows_of((const T *)a.w + v0 * a.w_stride, a.w_stride, here, w_p);
    const size_t many = tiles(here, BX) * tiles(a.rows, BY);
    if (BX == Deep::BX && many <= few_tiles())
      LAUNCH((k_loss_grad_tile<T, Deep>), many, S::THREADS, (TileOf<T, Deep>::LDS), a, w, h, v0, here,
             p.vp, coef, gl);
    else
      LAUNCH((k_loss_grad_tile<T, S>), many, S::THREADS, Tl::LDS, a, w, h, v0, here, p.vp, coef, gl);
    if (a.gh)
      LAUNCH((k_loss_gh_tile<T, S>), p.splits * tiles(a.dim, BX) * tiles(a.rows, BY), S::THREADS,
             Tl::LDS, a.rows, a.dim, p.vp, gl, w, part, p.run, i > 0);
    const size_t width = up(here, BX);
    if (a.gh && i + 1 == p.pieces) {
      // (many parts of few outputs: sixteen threads to each)
      const size_t quads = tiles(a.dim, 4) * a.rows;
      const bool few = p.splits >= 32 && quads < ((size_t)1 << 16);
      auto k = few ? k_loss_gh_join<T, 16> : k_loss_gh_join<T, 1>;
      LAUNCH(k, tiles(quads, few ? 16 : 256), 256, 0, part, (int)p.splits, a.rows, a.dim, coef,
             (T *)a.gh, a.gh_stride, a.gw ? gl : nullptr, width, p.vp);
    } else if constexpr (ROW_UP<T> > 0) {
      if (a.gw)
        LAUNCH(k_loss_common<T>, std::min((size_t)1024, tiles(a.rows * width, 8 * 256)), 256, 0, coef,
               a.rows, width, p.vp, gl);
    }
    if (a.gw) {
      const size_t many = tiles(a.dim, BX) * tiles(here, BY);
      auto gw = [&](auto shape) {
        using G = decltype(shape);
        auto k = past_caches((const T *)a.gw, a.gw_stride) ? k_loss_gw_tile<T, G, true>
                                                           : k_loss_gw_tile<T, G, false>;
        LAUNCH(k, many, G::THREADS, (TileOf<T, G, true>::LDS), a, v0, here, p.vp, p.ld_t, coef, gl,
               h_t);
      };
      if (BX == Deep::BX && many <= few_tiles()) gw(Deep{});
      else gw(S{});
    }
  }
  return e;
}

// All launches of a call, or none: every grid is looked at first, where the sizes are such
// that one may be too large (the joining of the parts has 64 threads to a row, others less
// than two to an element).
hipError_t checked(hipError_t (*call)(const LossArgs &, hipStream_t, bool), const LossArgs &a,
                   hipStream_t st) {
  const size_t most = (size_t)1 << 31;
  if (a.rows * a.dim >= most || a.rows * a.vocab >= most || std::max(a.rows, a.vocab) >= most / 64) {
    const hipError_t e = call(a, st, true);
    if (e != hipSuccess) return e;
  }
  return call(a, st, false);
}

}  // namespace

size_t cross_entropy_workspace(size_t rows, size_t dim, size_t vocab) {
  return up(tiles(vocab, forward_x(rows, dim, vocab)) * rows * sizeof(Stat) + rows * 4, 16);
}
size_t cross_entropy_backward_workspace(size_t rows, size_t dim, size_t vocab) {
  return (large(rows, dim, vocab) ? plan<Large>(rows, dim, vocab) : plan<Small>(rows, dim, vocab)).bytes;
}

hipError_t launch_cross_entropy(const LossArgs &a, hipStream_t st) {
  auto k = a.dtype == ROSETTA_BF16 ? forward<bf16> : forward<f16>;
  return checked(k, a, st);
}
hipError_t launch_cross_entropy_backward(const LossArgs &a, hipStream_t st) {
  if (large(a.rows, a.dim, a.vocab))
    return checked(a.dtype == ROSETTA_BF16 ? backward<bf16, Large> : backward<f16, Large>, a, st);
  return checked(a.dtype == ROSETTA_BF16 ? backward<bf16, Small> : backward<f16, Small>, a, st);
}

}  // namespace rosetta
