// Tiles of products of two matrices with contiguous rows, X [nx][k] and
// Y [ny][k], on the matrix cores: acc[x][y] = sum_k X[x][k] Y[y][k], for 8-bit
// integers (32-bit integer sums) and bf16 or f16 (32-bit float sums).
//
// All three take 16 bytes of a row per lane and instruction, so the code counts
// in bytes: a row's step is 128 bytes, two instructions deep.  x is the axis
// that is contiguous in the caller's output; a lane holds runs of it.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "clear.hpp"

namespace rosetta {

using v4i = __attribute__((ext_vector_type(4))) int;
using v4f = __attribute__((ext_vector_type(4))) float;
using v8bf = __attribute__((ext_vector_type(8))) __bf16;
using v8h = __attribute__((ext_vector_type(8))) _Float16;

constexpr int STEP = 128;  // bytes of a row per step
constexpr int FRAG = 16;   // bytes of a row per lane and instruction

// acc (16 x 16, lane l: y = l % 16, x = 4 (l / 16) + 0..3) += product of a
// fragment of X (lane l: row l % 16, bytes 16 (l / 16) .. + 16 of 64) and one
// of Y (the same).
template <class T>
struct Mma;
template <>
struct Mma<int8_t> {
  using Acc = v4i;
  __device__ static Acc mac(v4i x, v4i y, Acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, c, 0, 0, 0);
  }
};
template <>
struct Mma<bf16> {
  using Acc = v4f;
  __device__ static Acc mac(v4i x, v4i y, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, x),
                                                   __builtin_bit_cast(v8bf, y), c, 0, 0, 0);
  }
};
template <>
struct Mma<f16> {
  using Acc = v4f;
  __device__ static Acc mac(v4i x, v4i y, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x),
                                                  __builtin_bit_cast(v8h, y), c, 0, 0, 0);
  }
};

// A matrix operand: `rows` rows of `bytes` bytes, `ld` bytes apart.  The rows a
// tile has beyond `rows` read the last one instead; what they give is never
// written.
struct Operand {
  const char *p;
  int64_t ld;
  int64_t rows;
  int64_t bytes;
};

// Whether rows can be brought in by 16 bytes at a time straight to LDS.
inline bool rows_aligned(const Operand &o) {
  return (uintptr_t)o.p % FRAG == 0 && o.ld % FRAG == 0 && o.bytes % FRAG == 0;
}

// Block b of `blocks`, numbered so that each of the eight XCDs (blocks are
// dealt to them in turn) gets a run of consecutive ones: neighbours share rows
// in that XCD's L2.
__device__ inline unsigned xcd_block(unsigned b, unsigned blocks) {
  const unsigned x = b % 8, at = b / 8, each = blocks / 8, more = blocks % 8;
  return x * each + (x < more ? x : more) + at;
}

// Tile (tx, ty) of a grid of gx x gy of them: runs of `BAND` tiles of y, so that
// a run of blocks is about square.
__device__ inline void band_tile(unsigned b, unsigned gx, unsigned gy, unsigned &tx,
                                 unsigned &ty) {
  constexpr unsigned BAND = 8;
  const unsigned per = BAND * gx, band = b / per, in = b % per;
  const unsigned left = gy - band * BAND, high = left < BAND ? left : BAND;
  ty = band * BAND + in % high;
  tx = in / high;
}

// 16 bytes of a row at any byte address, zeros from byte `end` on.
__device__ inline v4i load_frag(const char *row, int64_t at, int64_t end) {
  v4i v = {0, 0, 0, 0};
  if (at + FRAG <= end) {
    __builtin_memcpy(&v, row + at, FRAG);
  } else if (at < end) {
    uint8_t b[FRAG];
#pragma unroll
    for (int i = 0; i < FRAG; ++i) b[i] = at + i < end ? (uint8_t)row[at + i] : 0;
    __builtin_memcpy(&v, b, FRAG);
  }
  return v;
}

// A workgroup's BX x BY tile, WX x WY waves of (BX / WX) x (BY / WY) each.
//
// A stage of LDS holds 128 bytes of each of the tile's rows.  Chunk c (16
// bytes) of a row lies at place c ^ key, key = (m >> 1) & 7 for the row's index
// m in its fragment, which spreads the 16 rows of a fragment over all banks.
// Row 4 g + r of fragment i of a wave's X is its row g * 4 TX + 4 i + r, so that
// a lane's accumulators are runs of 4 TX consecutive x.
template <class T, int BX, int BY, int WX, int WY>
struct Tile {
  static constexpr int WAVES = WX * WY, THREADS = 64 * WAVES;
  static constexpr int TX = BX / WX / 16, TY = BY / WY / 16;
  static constexpr int STAGE = (BX + BY) * STEP;
  static constexpr int LDS = 2 * STAGE;
  static constexpr int LOADS = (BX + BY) / 8 / WAVES;  // of 8 rows, per wave and stage
  static_assert((BX + BY) / 8 % WAVES == 0 && BX / 8 % WAVES == 0, "loads divide evenly");
  using Acc = typename Mma<T>::Acc;

  __device__ static int key_x(int row) {
    const int m = (row / (4 * TX) & 3) * 4 + (row & 3);
    return (m >> 1) & 7;
  }
  __device__ static int key_y(int row) { return (row >> 1) & 7; }

  // acc += X rows [x0, x0 + BX) times Y rows [y0, y0 + BY) over bytes
  // [k0, k1) of the rows (k0 a multiple of 16).
  template <bool ALIGNED>
  __device__ static void run(const Operand &X, const Operand &Y, int64_t x0, int64_t y0,
                             int64_t k0, int64_t k1, char *lds, Acc (&acc)[TX][TY]) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int wx = wave % WX, wy = wave / WX;
    // this lane's source of each load: row 8 q + lane / 8, chunk (lane % 8) ^ key
    const char *src[LOADS];
    int chunk[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = (i * WAVES + wave) * 8 + lane / 8;
      const bool isx = i < BX / 8 / WAVES;
      const int r = isx ? row : row - BX;
      const Operand &o = isx ? X : Y;
      int64_t at = (isx ? x0 : y0) + r;
      at = at < o.rows ? at : o.rows - 1;
      chunk[i] = ((lane % 8) ^ (isx ? key_x(r) : key_y(r))) * FRAG;
      src[i] = o.p + at * o.ld;
    }
    auto load = [&](int64_t k, char *stage) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const v4i v = load_frag(src[i], k + chunk[i], k1);
        *(v4i *)(stage + (i * WAVES + wave) * 1024 + lane * FRAG) = v;
      }
    };
    // this lane's place in fragment 0 of its wave's X and Y
    const int m = lane % 16, g = lane / 16;
    const int key = (m >> 1) & 7;
    const int atx = (wx * (BX / WX) + (m / 4) * 4 * TX + m % 4) * STEP;
    const int aty = (BX + wy * (BY / WY) + m) * STEP;
    auto compute = [&](const char *stage) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int c = ((s * 4 + g) ^ key) * FRAG;
        v4i x[TX], y[TY];
#pragma unroll
        for (int i = 0; i < TX; ++i) x[i] = *(const v4i *)(stage + atx + i * 4 * STEP + c);
#pragma unroll
        for (int j = 0; j < TY; ++j) y[j] = *(const v4i *)(stage + aty + j * 16 * STEP + c);
#pragma unroll
        for (int j = 0; j < TY; ++j)
#pragma unroll
          for (int i = 0; i < TX; ++i) acc[i][j] = Mma<T>::mac(x[i], y[j], acc[i][j]);
      }
    };
    int b = 0;
    if (k0 < k1) load(k0, lds);
    for (int64_t k = k0; k < k1; k += STEP, b ^= 1) {
      __syncthreads();
      if (k + STEP < k1) load(k + STEP, lds + (b ^ 1) * STAGE);
      compute(lds + b * STAGE);
    }
    __syncthreads();
  }

  // x and y (within the tile) of acc[i][j][r] of this lane: x_at() + 4 i + r and
  // y_at() + 16 j
  __device__ static int x_at() {
    return (threadIdx.x / 64) % WX * (BX / WX) + (threadIdx.x % 64) / 16 * 4 * TX;
  }
  __device__ static int y_at() {
    return (threadIdx.x / 64) / WX * (BY / WY) + threadIdx.x % 16;
  }
};

// n consecutive values at p, of which the first `left` are written.
template <class T, int N>
__device__ inline void store_run(T *p, int64_t left, const float (&f)[N]) {
  T v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (T)f[i];
  if (left >= N) {
    __builtin_memcpy(p, v, sizeof v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) p[i] = v[i];
  }
}

}  // namespace rosetta
