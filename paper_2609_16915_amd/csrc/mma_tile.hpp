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

// The furthest that rows brought in straight to LDS may be apart: a tile's 256 then
// lie, with their 2^30 bytes at most, within 31-bit offsets of its first.
constexpr int64_t MAX_LD = (int64_t)1 << 22;

// Whether rows can be brought in by 16 bytes at a time straight to LDS.
inline bool rows_aligned(const Operand &o) {
  return (uintptr_t)o.p % FRAG == 0 && o.ld % FRAG == 0 && o.bytes % FRAG == 0 && o.ld <= MAX_LD &&
         o.bytes <= (int64_t)1 << 30;
}

// Memory at `base`, for buffer loads (raw, 32-bit offsets).
__device__ inline v4i buffer_at(const char *base) {
  const uint64_t b = (uint64_t)base;
  return v4i{__builtin_amdgcn_readfirstlane((int)b),
             __builtin_amdgcn_readfirstlane((int)(b >> 32) & 0xffff), -1, 0x00027000};
}

// The same, `ahead` bytes on.
__device__ inline v4i buffer_on(v4i buf, int64_t ahead) {
  const uint64_t b = ((uint64_t)(uint32_t)buf.x | (uint64_t)(uint32_t)buf.y << 32) + ahead;
  return v4i{(int)b, (int)(b >> 32), buf.z, buf.w};
}

// 16 bytes per lane from buf + at + k to LDS address `lds` + 16 lane.  Nothing
// waits for it but barrier_loaded().
__device__ inline void load_to_lds(v4i buf, int at, int k, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(
                   __builtin_amdgcn_readfirstlane(lds)),
               "v"(at), "s"(buf), "s"(k)
               : "memory", "m0");
}

// All but N of this wave's LDS loads have landed and its LDS reads are done; then
// all waves'.
template <int N = 0>
__device__ inline void barrier_loaded() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
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
// Bound by the matrix pipes under the card's power limit: 256 x 256 with eight
// waves keeps them busy 65 % (8 bits) to 75 % (16 bits) of the time at 1.7-1.8 GHz,
// 2.6 POP/s and 1.41 PFLOP/s over 14336 x 8192 x 4096 bytes.  Measured on the way
// there (8 bits, TOP/s): all of a stage's reads before its products 2061, the other
// half's reads and the loads spread between products 2582; waves 2 x 4 instead of 4 x
// 2 2207, four waves of 128 x 128 1665; stages of 64 bytes in a ring of four 2400; 32 x
// 32 products 2339.  In 128 x 128 tiles 2200, 64 KB of LDS, two to a CU.
//
// A stage of LDS holds 128 bytes of each of the tile's rows.  Chunk c (16
// bytes) of a row lies at place c ^ key, key = (m >> 1) & 7 for the row's index
// m in its fragment, which spreads the 16 rows of a fragment over all banks.
// Row 4 g + r of fragment i of a wave's X is its row g * 4 TX + 4 i + r, so that
// a lane's accumulators are runs of 4 TX consecutive x.
//
// XA, YA (16-bit types, ALIGNED only): X or Y lies the other way, k rows of columns
// (bytes: the columns'; x0 or y0 a column; k1 is then exact, and the other
// operand's rows go on to whole 16 bytes with zeros).  Its stage holds 64 such rows
// of BX or BY columns; chunk c (32 bytes, a fragment's 16 columns) of row k lies at
// place c ^ key, key = (k & 3) | (k >> 1 & 4), and a fragment's lanes read it turned
// by 4 x 4 (ds_read_b64_tr_b16: lane l of 16 gives the address of row l / 4, columns
// 4 (l % 4) .. + 4, and gets column l of the four rows).  With XA a lane's
// accumulators are runs of 4 x only.
//
// RUNS false: row m of fragment i of a wave's X is its row 16 i + m, and a lane's
// accumulators are runs of 4 x, four lanes' next to each other: 32-bit outputs then
// leave 64 bytes together (4096 x 4096 x 4096 bytes to f32: 62 us for 73 with each
// lane's 16 bytes alone in their 64; in 16 bits a lane's runs are 32 bytes, and lanes
// that trade halves for 64 gained nothing).
template <class T, int BX, int BY, int WX, int WY, int STAGES = 2, bool XA = false, bool YA = false,
          bool RUNS = !XA>
struct Tile {
  static constexpr int WAVES = WX * WY, THREADS = 64 * WAVES;
  static constexpr int TX = BX / WX / 16, TY = BY / WY / 16;
  static constexpr int STAGE = (BX + BY) * STEP;
  static constexpr int LDS = STAGES * STAGE;  // what the stages take
  static constexpr int LOADS = (BX + BY) / 8 / WAVES;  // of 8 rows, per wave and stage
  static_assert((BX + BY) / 8 % WAVES == 0 && BX / 8 % WAVES == 0, "loads divide evenly");
  // whether registers are left for what an epilogue reads to be asked for before the
  // products
  static constexpr bool ROOM = TX * TY <= 8;
  using Acc = typename Mma<T>::Acc;

  __device__ static int key_x(int row) {
    const int m = RUNS ? (row / (4 * TX) & 3) * 4 + (row & 3) : row;
    return (m >> 1) & 7;
  }
  __device__ static int key_y(int row) { return (row >> 1) & 7; }
  __device__ static int key_k(int row) { return (row & 3) | (row >> 1 & 4); }

  // A tile: rows [x0, x0 + BX) of X and [y0, y0 + BY) of Y over bytes [k0, k1)
  // of the rows (k0 a multiple of 16; ALIGNED: k1 too).  x0 < X.rows and y0 <
  // Y.rows: a tile has a row at least, or its loads would leave the matrix.  ALIGNED:
  // ld at most MAX_LD.
  struct Place {
    Operand X, Y;
    int64_t x0, y0, k0, k1;
  };

  __device__ static void clear(Acc (&acc)[TX][TY]) {
#pragma unroll
    for (int i = 0; i < TX; ++i)
#pragma unroll
      for (int j = 0; j < TY; ++j) acc[i][j] = Acc{0, 0, 0, 0};
  }

  // The tile's sums, and their addition to what is there.
  template <bool ALIGNED>
  __device__ static void run(const Place &p, char *lds, Acc (&acc)[TX][TY]) {
    clear(acc);
    add<ALIGNED>(p, lds, acc);
  }

  // The stages are free when it returns.  (Blocks that go through
  // several tiles, the next one's first loads under the present one's epilogue,
  // gained 2 % with the barest epilogue and lost 1-8 % with the real ones, whose
  // values then no longer fit the registers.)
  template <bool ALIGNED>
  __device__ static void add(const Place &p, char *lds, Acc (&acc)[TX][TY]) {
    const int lane = threadIdx.x % 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wx = wave % WX, wy = wave / WX;
    constexpr int LX = BX / 8 / WAVES;  // loads of X, the rest are of Y
    // this lane's place in fragment 0 of its wave's X and Y
    const int m = lane % 16, g = lane / 16;
    const int key = (m >> 1) & 7;
    const int atx = (wx * (BX / WX) + (RUNS ? (m / 4) * 4 * TX + m % 4 : m)) * STEP;
    const int aty = (BX + wy * (BY / WY) + m) * STEP;
    if (p.k0 >= p.k1) return;
    static_assert(!(XA || YA) || (sizeof(T) == 2 && ALIGNED), "");
    // Fragment f of this wave's part, across: rows of `width` bytes at `at`, their
    // chunks from `first` on.
    auto read_across = [&](const char *at, int width, int first, int s, int f) {
      using v4s = __attribute__((ext_vector_type(4))) short;
      using lds_v4s = __attribute__((address_space(3))) v4s;
      const int row = 8 * g + m / 4;  // of half 0; the half and the 4 x 16 block keep its key
      at += row * width + ((first + f) ^ key_k(row)) * 32 + m % 4 * 8 + s * 32 * width;
      struct {
        v4s h[2];
      } v;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        v.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(at + h * 4 * width));
      return __builtin_bit_cast(v4i, v);
    };
    auto read_x = [&](const char *stage, int s, int i) {
      if constexpr (XA) return read_across(stage, 2 * BX, wx * TX, s, i);
      else return *(const v4i *)(stage + atx + i * (RUNS ? 4 : 16) * STEP + ((s * 4 + g) ^ key) * FRAG);
    };
    auto read_y = [&](const char *stage, int s, int j) {
      if constexpr (YA) return read_across(stage + BX * STEP, 2 * BY, wy * TY, s, j);
      else return *(const v4i *)(stage + aty + j * 16 * STEP + ((s * 4 + g) ^ key) * FRAG);
    };
    // Half s of a stage to registers; of a step's last bytes only `left` count.
    auto read = [&](const char *stage, int s, v4i(&x)[TX], v4i(&y)[TY], int left, auto tail) {
#pragma unroll
      for (int i = 0; i < TX; ++i) x[i] = read_x(stage, s, i);
#pragma unroll
      for (int j = 0; j < TY; ++j) y[j] = read_y(stage, s, j);
      if (tail.value && (s * 4 + g) * FRAG >= left) {
#pragma unroll
        for (int i = 0; i < TX; ++i) x[i] = v4i{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < TY; ++j) y[j] = v4i{0, 0, 0, 0};
      }
    };
    auto multiply = [&](const v4i(&x)[TX], const v4i(&y)[TY]) {
#pragma unroll
      for (int j = 0; j < TY; ++j)
#pragma unroll
        for (int i = 0; i < TX; ++i) acc[i][j] = Mma<T>::mac(x[i], y[j], acc[i][j]);
    };
    // Half s of a stage to (x, y) while (px, py) are multiplied, a few reads and
    // loads at a time between products.
    auto half = [&](const char *stage, int s, v4i(&x)[TX], v4i(&y)[TY], const v4i(&px)[TX],
                    const v4i(&py)[TY], auto load) {
      constexpr int READS = TX + TY;
#pragma unroll
      for (int j = 0; j < TY; ++j) {
#pragma unroll
        for (int i = j * LOADS / TY; i < (j + 1) * LOADS / TY; ++i) load(i);
#pragma unroll
        for (int i = j * READS / TY; i < (j + 1) * READS / TY; ++i) {
          if (i < TX) x[i] = read_x(stage, s, i);
          else y[i - TX] = read_y(stage, s, i - TX);
        }
#pragma unroll
        for (int i = 0; i < TX; ++i) acc[i][j] = Mma<T>::mac(px[i], py[j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    v4i x0f[TX], y0f[TY], x1f[TX], y1f[TY];
    constexpr std::false_type whole{};
    // Row of the tile and byte of the step of this lane's load i: row 8 q + lane / 8
    // of X or Y, chunk (lane % 8) ^ key.
    auto row_of = [&](int i) { return (i * WAVES + wave) * 8 + lane / 8 - (i < LX ? 0 : BX); };
    auto chunk_of = [&](int i) {
      const int r = row_of(i);
      return ((lane % 8) ^ (i < LX ? key_x(r) : key_y(r))) * FRAG;
    };
    // rows past the last are the last again
    auto row_in = [&](int i) {
      const int64_t left = (i < LX ? p.X.rows - p.x0 : p.Y.rows - p.y0) - 1;
      const int r = row_of(i);
      return r < left ? r : (int)left;
    };
    if constexpr (ALIGNED) {
      const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
      const v4i bx = buffer_at(p.X.p + p.x0 * (XA ? (int64_t)sizeof(T) : p.X.ld));
      const v4i by = buffer_at(p.Y.p + p.y0 * (YA ? (int64_t)sizeof(T) : p.Y.ld));
      int at[LOADS], k = (int)p.k0;
      const int end = (int)p.k1, left = (end - k - 1) % STEP + 1;
      auto is_across = [](int i) { return i < LX ? XA : YA; };
      // Across: row of the step and byte of the row of this lane's load i; columns
      // past the last are the first again.
      auto across_piece = [&](int i) { return ((i - (i < LX ? 0 : LX)) * WAVES + wave) * 64 + lane; };
      auto across_row = [&](int i) { return across_piece(i) / ((i < LX ? BX : BY) / 8); };
      auto across_byte = [&](int i) {
        const int piece = across_piece(i) % ((i < LX ? BX : BY) / 8);
        const int byte = ((piece / 2) ^ key_k(across_row(i))) * 32 + piece % 2 * FRAG;
        const int64_t first = (i < LX ? p.x0 : p.y0) * (int64_t)sizeof(T);
        return first + byte + FRAG <= (i < LX ? p.X.bytes : p.Y.bytes) ? byte : 0;
      };
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int ld = (int)(i < LX ? p.X.ld : p.Y.ld);
        at[i] = is_across(i) ? across_row(i) * ld + across_byte(i) : row_in(i) * ld + chunk_of(i);
      }
      auto load_one = [&](int i, int at, int k, int stage) {
        const unsigned to = base + stage + (i * WAVES + wave) * 1024;
        const v4i buf = i < LX ? bx : by;
        if (is_across(i))
          load_to_lds(buffer_on(buf, k / (int)sizeof(T) * (i < LX ? p.X.ld : p.Y.ld)), at, 0, to);
        else load_to_lds(buf, at, k, to);
      };
      // the last step may be part of one: chunks (across: rows) beyond it read its
      // first again, and read() takes them as zeros
      auto load_any = [&](int k, int stage) {
        if (k + STEP <= end) {
#pragma unroll
          for (int i = 0; i < LOADS; ++i) load_one(i, at[i], k, stage);
        } else if (k < end) {
#pragma unroll
          for (int i = 0; i < LOADS; ++i) {
            if (is_across(i))
              load_one(i, across_row(i) * (int)sizeof(T) < left ? at[i] : across_byte(i), k, stage);
            else load_one(i, at[i] - (chunk_of(i) < left ? 0 : chunk_of(i)), k, stage);
          }
        }
      };
#pragma unroll
      for (int i = 0; i < STAGES; ++i) load_any(k + i * STEP, i * STAGE);
      int b = 0;
      auto next = [](int b) { return b + STAGE == LDS ? 0 : b + STAGE; };
      barrier_loaded();
      // Both halves of a step in registers, one ahead: the second half's reads go
      // with the first's products, then, the next step's loads having landed, the
      // next first half's with the second's.
      if (k + STEP <= end) read(lds, 0, x0f, y0f, STEP, whole);
      for (; k + (STAGES + 1) * STEP <= end; k += STEP, b = next(b)) {
        half(lds + b, 1, x1f, y1f, x0f, y0f, [](int) {});
        barrier_loaded<(STAGES - 2) * LOADS>();
        half(lds + next(b), 0, x0f, y0f, x1f, y1f, [&](int i) {
          load_one(i, at[i], k + STAGES * STEP, b);
        });
      }
      // at most STAGES more whole steps and a part of one
      for (; k + STEP <= end; k += STEP, b = next(b)) {
        read(lds + b, 1, x1f, y1f, STEP, whole);
        multiply(x0f, y0f);
        barrier_loaded();
        load_any(k + STAGES * STEP, b);
        if (k + 2 * STEP <= end) read(lds + next(b), 0, x0f, y0f, STEP, whole);
        multiply(x1f, y1f);
      }
      if (k < end) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          read(lds + b, s, x0f, y0f, left, std::true_type{});
          multiply(x0f, y0f);
        }
      }
    } else {
      v4i ahead[LOADS];
      auto fetch = [&](int64_t k) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const char *src =
              i < LX ? p.X.p + (p.x0 + row_in(i)) * p.X.ld : p.Y.p + (p.y0 + row_in(i)) * p.Y.ld;
          if (k + STEP <= p.k1) __builtin_memcpy(&ahead[i], src + k + chunk_of(i), FRAG);
          else ahead[i] = load_frag(src, k + chunk_of(i), p.k1);
        }
      };
      int b = 0;
      fetch(p.k0);
      for (int64_t k = p.k0; k < p.k1; k += STEP, b = STAGE - b) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          *(v4i *)(lds + b + (i * WAVES + wave) * 1024 + lane * FRAG) = ahead[i];
        __syncthreads();
        if (k + STEP < p.k1) fetch(k + STEP);
        read(lds + b, 0, x0f, y0f, STEP, whole);
        multiply(x0f, y0f);
        read(lds + b, 1, x0f, y0f, STEP, whole);
        multiply(x0f, y0f);
      }
    }
    __syncthreads();
  }

  // x and y (within the tile) of acc[i][j][r] of this lane: x_at() + 4 i + r (RUNS
  // false: + 16 i + r) and y_at() + 16 j
  __device__ static int x_at() {
    return (threadIdx.x / 64) % WX * (BX / WX) + (threadIdx.x % 64) / 16 * (RUNS ? 4 * TX : 4);
  }
  __device__ static int y_at() {
    return (threadIdx.x / 64) / WX * (BY / WY) + threadIdx.x % 16;
  }
};

// A few rows of Y (16 NY at most): a workgroup takes 16 NX rows of X, its waves
// the steps of the rows in turn, straight from memory to registers (the rows of
// X are read once, those of Y come from the L2), two steps ahead of the products.
// The waves' sums are then added up, in order, in LDS.
//
// Bound by memory: 14336 rows of 4096 bytes in 12 us, 128000 of 8192 in 180 us (5.8
// TB/s).  The loads of X past the caches: 14.4 and 200 us, since a row's 128 bytes
// come in two halves.
template <class T, int NX, int NY, int WAVES_>
struct Thin {
  static constexpr int WAVES = WAVES_, THREADS = 64 * WAVES;
  static constexpr int LDS = WAVES * NX * NY * 1024;
  static constexpr int SUMS = NX * NY * 64;  // quadruples of sums
  using Acc = typename Mma<T>::Acc;

  // Quadruple t of the sums, once run() is done: x = x0 + 16 (t / 64 % NX) + 4 (t %
  // 64 / 16) + 0..3, y = 16 (t / 64 / NX) + t % 16.
  __device__ static Acc sum(int t, const char *lds) {
    Acc s = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += ((const Acc *)lds)[w * SUMS + t];
    return s;
  }

  // Over bytes [k0, k1) of the rows, k0 a multiple of STEP.
  __device__ static void run(const Operand &X, const Operand &Y, int64_t x0, int k0, int k1,
                             char *lds) {
    const int lane = threadIdx.x % 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int m = lane % 16, g = lane / 16;
    const char *xs[NX], *ys[NY];
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int64_t r = x0 + 16 * i + m;
      xs[i] = X.p + (r < X.rows ? r : X.rows - 1) * X.ld + g * FRAG;
    }
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      const int64_t r = 16 * j + m;
      ys[j] = Y.p + (r < Y.rows ? r : Y.rows - 1) * Y.ld + g * FRAG;
    }
    struct Step {
      v4i x[NX][2], y[NY][2];
    };
    auto load = [&](Step &f, int k) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < NX; ++i) __builtin_memcpy(&f.x[i][h], xs[i] + k + h * 64, FRAG);
#pragma unroll
        for (int j = 0; j < NY; ++j) __builtin_memcpy(&f.y[j][h], ys[j] + k + h * 64, FRAG);
      }
    };
    Acc acc[NX][NY];
#pragma unroll
    for (int i = 0; i < NX; ++i)
#pragma unroll
      for (int j = 0; j < NY; ++j) acc[i][j] = Acc{0, 0, 0, 0};
    auto multiply = [&](const Step &f) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < NX; ++i)
#pragma unroll
          for (int j = 0; j < NY; ++j) acc[i][j] = Mma<T>::mac(f.x[i][h], f.y[j][h], acc[i][j]);
    };
    constexpr int TURN = WAVES * STEP;
    const int whole = k0 + (k1 - k0) / STEP * STEP;
    Step a, b;
    int k = k0 + wave * STEP;
    if (k < whole) load(a, k);
    if (k + TURN < whole) load(b, k + TURN);
    for (; k + TURN < whole; k += 2 * TURN) {
      multiply(a);
      if (k + 2 * TURN < whole) load(a, k + 2 * TURN);
      multiply(b);
      if (k + 3 * TURN < whole) load(b, k + 3 * TURN);
    }
    if (k < whole) multiply(a);
    // what is left of a step, by the wave whose turn it is
    if (whole < k1 && (whole - k0) / STEP % WAVES == wave) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < NX; ++i)
          a.x[i][h] = load_frag(xs[i] - g * FRAG, whole + h * 64 + g * FRAG, k1);
#pragma unroll
        for (int j = 0; j < NY; ++j)
          a.y[j][h] = load_frag(ys[j] - g * FRAG, whole + h * 64 + g * FRAG, k1);
      }
      multiply(a);
    }
    Acc *sums = (Acc *)lds;
#pragma unroll
    for (int j = 0; j < NY; ++j)
#pragma unroll
      for (int i = 0; i < NX; ++i) sums[(wave * NX * NY + j * NX + i) * 64 + lane] = acc[i][j];
    __syncthreads();
  }
};

// N consecutive values at p, of which the first `left` are there (zeros after).
template <int N>
__device__ inline void load_run(const float *p, int64_t left, float (&f)[N]) {
  if (left >= N) {
    __builtin_memcpy(f, p, sizeof f);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = i < left ? p[i] : 0.f;
  }
}

// Whether rows that nobody reads here again may go past the caches: where they begin
// and end with whole pieces of 64 bytes, or what is written of a piece goes out alone
// (40000 rows of 3520 in 16 bits: 176 us past the caches, 198 through them; of 3511
// 453 and 356).
template <class T>
inline bool past_caches(const T *p, size_t stride) {
  return (((uintptr_t)p | stride * sizeof(T)) & 63) == 0;
}

// N consecutive values at p, of which the first `left` are written; PAST: past the
// caches.  (A branch at run time would leave both ways through them: the compiler
// takes the two stores for one.)
template <bool PAST = false, class T, int N>
__device__ inline void store_run(T *p, int64_t left, const float (&f)[N]) {
  T v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (T)f[i];
  if (left >= N) {
    // (16 bytes at a time, at any address)
    using v4u = __attribute__((ext_vector_type(4), aligned(2))) int;
    static_assert(sizeof v % 16 == 0 || N == 4);
    if constexpr (sizeof v % 16) {
      __builtin_memcpy(p, v, sizeof v);
    } else {
#pragma unroll
      for (int i = 0; i < (int)(sizeof v / 16); ++i) {
        v4u w;
        __builtin_memcpy(&w, (const char *)v + 16 * i, 16);
        if constexpr (PAST) __builtin_nontemporal_store(w, (v4u *)p + i);
        else ((v4u *)p)[i] = w;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) p[i] = v[i];
  }
}

}  // namespace rosetta
