// Attention over the 8-bit cache: one token, a prompt, or a tree of drafted tokens.
//
//   out = sum_t softmax_t(scale <q, k_t>) v_t,   k_t = k_scale[t] K[t], v_t alike,
// over the positions that a row sees, in one pass: the running maximum, the sum and
// the products with the values go along, and parts of a long sequence are joined at
// the end.
//
// The rows of a sequence that share a head of the cache (positions times the heads of
// its group) are the columns of the products: S^T = K Q^T, O^T = V^T P^T, both on
// v_mfma_f32_16x16x32_f16.  A lane then holds four positions' scores of one row, which
// are just what it feeds to the second product, and a run of dim / 4 of that row's
// outputs: neither goes through LDS.  (The order of the second product's terms is
// free: a lane's eight are positions 4 g .. + 3 of two tiles of sixteen.)
//
// 8 bits become f16 on the way, exactly: 0x6400 | (b + 128) is 1024 + b + 128.  Values
// are turned (eight positions of one column for the eight columns of one position) by
// the byte permutations that widen them.  A row of q is held in f16 on a power of two
// that brings its largest value to 2^13: bf16 has fewer bits than f16, so only what is
// below 2^-27 of the largest loses any.  The weights of the second product, exp(s - m)
// v_scale, are rounded to f16 (2^-12 of themselves, beside outputs of 2^-9 in bf16);
// their reference takes in the largest v_scale met, so that they are at most 2^15.
// The sum of the weights is that of the unrounded exponentials.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "decode.hpp"
#include "mma_tile.hpp"

namespace rosetta {

namespace {

using v2h = __attribute__((ext_vector_type(2))) _Float16;
using v2i = __attribute__((ext_vector_type(2))) int;
using u32 = uint32_t;

constexpr float NONE = -__builtin_inff();

// ---- 8 bits to f16 ----

// Pairs (x, y) of bytes, biased by 128, under exponents that make them 1024 + x, + y.
__device__ inline u32 from_1152(u32 w) {
  v2h h = __builtin_bit_cast(v2h, w);
  h += v2h{(_Float16)-1152.f, (_Float16)-1152.f};
  return __builtin_bit_cast(u32, h);
}

// Four bytes of a word as four halves.
__device__ inline v2i widen(u32 w) {
  w ^= 0x80808080u;
  return v2i{(int)from_1152(__builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)),
             (int)from_1152(__builtin_amdgcn_perm(0x64646464u, w, 0x04030402u))};
}

// Byte i of a and of b as two halves.
template <int I>
__device__ inline u32 widen_two(u32 a, u32 b) {
  return from_1152(__builtin_amdgcn_perm(b, a, 0x0c000c00u | (4 + I) << 16 | I) ^ 0x64806480u);
}

__device__ inline v4f mac(v4i x, v4i y, v4f c) { return Mma<f16>::mac(x, y, c); }

// Sum and maximum over the four lanes of a row (l, l ^ 16, l ^ 32, l ^ 48).  A swap of a
// value with its copy leaves either half's values in both, one half's in each: two
// instructions, where a shuffle goes by way of LDS.  (In assembly: the compiler's builtin
// gives its first result twice.)
template <class F>
__device__ inline float across(float a, F f) {
  float b = a;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  a = f(a, b);
  b = a;
  asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  return f(a, b);
}
__device__ inline float row_max(float a) {
  return across(a, [](float x, float y) { return fmaxf(x, y); });
}
__device__ inline float row_sum(float a) {
  return across(a, [](float x, float y) { return x + y; });
}

// What a launch works on.
struct Work {
  AttendArgs a;
  int group, parts;  // heads to a head of the cache, parts of a sequence
  int row_blocks;    // workgroups to the rows of a sequence and head
  float *sums;       // parts > 1: [rows][heads][parts][DIM], (reference, sum) [..][parts]
  float2 *ends;
};

// One sequence and head of the cache, as its workgroups see it.
struct Seq {
  Span sp;
  int64_t length;  // positions that are in the table
  const int *table;
  const int8_t *k, *v;  // of the head
  const float *ks, *vs;
};
__device__ inline Seq seq_of(const AttendArgs &a, int b, int head) {
  Seq s;
  const Packed &r = a.packed;
  s.sp = span_of(r.starts, r.lens, b, r.rows);
  s.sp.n = s.sp.n < (int)a.max_rows ? s.sp.n : (int)a.max_rows;
  const int64_t capacity = (int64_t)r.table_len << a.cache.page_log;
  const int64_t length = r.lens[b];
  s.length = length < 0 ? 0 : length > capacity ? capacity : length;
  s.table = r.table + b * r.table_stride;
  s.k = a.cache.k + head * a.cache.head_stride;
  s.v = a.cache.v + head * a.cache.head_stride;
  s.ks = a.cache.k_scale + head * a.cache.scale_head_stride;
  s.vs = a.cache.v_scale + head * a.cache.scale_head_stride;
  return s;
}

// Sixteen positions from t on (a multiple of 16), which lie in one page.
struct Sixteen {
  const int8_t *k, *v;
  const float *ks, *vs;
  bool there;  // (where not, page 0 is read and not used)
};
__device__ inline Sixteen sixteen_at(const Seq &s, const AttendArgs &a, int64_t t) {
  const Cache &c = a.cache;
  int64_t pg = page_of(s.table, a.packed.table_len, c.page_log, c.pages, t);
  Sixteen x;
  x.there = pg >= 0;
  pg = pg < 0 ? 0 : pg;
  const int64_t place = t & (((int64_t)1 << c.page_log) - 1);
  const int64_t at = pg * c.page_stride + place * c.place_stride;
  const int64_t sat = pg * c.scale_page_stride + place;
  x.k = s.k + at;
  x.v = s.v + at;
  x.ks = s.ks + sat;
  x.vs = s.vs + sat;
  return x;
}

// A row of a workgroup: its query, and where it reads and writes.  rows past the last
// have at < 0.
struct Row {
  int i, head;  // place among the sequence's rows, head of q
  int64_t at;   // row of the call
};
__device__ inline Row row_of(const Seq &s, int r, int group, int kv_head) {
  Row x;
  x.i = r / group;
  x.head = kv_head * group + r % group;
  x.at = x.i < s.sp.n ? s.sp.first + x.i : -1;
  return x;
}

// D: the row length that the tiles take, at least dim (a multiple of 16).  NY: groups of
// 16 rows.
template <int D, int NY>
struct Rows16 {
  static constexpr int KS = D / 32;  // products of 32 over a row
  static constexpr int NX = D / 16;  // groups of 16 outputs
  v4i q[NY][KS];
  float factor[NY];   // of a score, in powers of two
  float top[NY];      // the largest score before the factor
  float big[NY];      // the largest v_scale
  float ref[NY], sum[NY];
  v4f o[NX][NY];

  // q's values k .. + 7 of a lane come from its row's first(ks) on.  `at` gives the Row
  // of group j.
  template <class T, class At, class First>
  __device__ void load(const AttendArgs &a, At at, First first) {
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      const Row r = at(j);
      float f[KS][8];
      float m = 0.f, odd = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int d = first(ks);
        struct __attribute__((packed, aligned(1))) {
          T v[8];
        } x;
        if (r.at >= 0 && d < (int)a.cache.dim) {
          __builtin_memcpy(&x, (const T *)a.q.p + r.at * a.q.row + r.head * a.q.head + d, sizeof x);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) x.v[i] = (T)0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f[ks][i] = (float)x.v[i];
          m = fmaxf(m, fabsf(f[ks][i]));
          odd += f[ks][i] * 0.f;
        }
      }
      m = row_max(m);
      odd = row_sum(odd);  // NaN where the row holds NaN or an infinity
      const int up = m > 0.f ? 13 - __builtin_amdgcn_frexp_expf(m) : 0;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        _Float16 h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = (_Float16)ldexpf(f[ks][i], up);
        __builtin_memcpy(&q[j][ks], h, 16);
      }
      factor[j] = ldexpf(a.scale * 1.44269504088896340736f, -up) + odd;
      top[j] = NONE;
      big[j] = 0.f;
      ref[j] = 0.f;
      sum[j] = 0.f;
#pragma unroll
      for (int i = 0; i < NX; ++i) o[i][j] = v4f{0, 0, 0, 0};
    }
  }

  // Scores s[x][j] (tile x of TILES, four positions of row j) to weights, two tiles to a
  // fragment.  ks, vs: the scales of the lane's positions.  seen(x, r, j), where MASKED:
  // whether row j sees position r of tile x.
  template <bool MASKED, int TILES, class Seen>
  __device__ void weigh(const v4f (&s)[TILES][NY], const v4f (&ks)[TILES], const v4f (&vs)[TILES],
                        Seen seen, v4i (&w)[TILES / 2][NY]) {
    float largest = 0.f;
    if constexpr (!MASKED) {
#pragma unroll
      for (int x = 0; x < TILES; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (vs[x][r] < __builtin_inff()) largest = fmaxf(largest, vs[x][r]);
      largest = row_max(largest);
    }
    bool grows = false;
    float before[NY];
    u32 seen_by[NY];
    float z[NY][TILES][4];
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      float m = NONE;
      seen_by[j] = 0;
#pragma unroll
      for (int x = 0; x < TILES; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = s[x][j][r] * ks[x][r];
          if constexpr (MASKED) {
            const bool there = seen(x, r, j);
            seen_by[j] |= (u32)there << (4 * x + r);
            v = there ? v : NONE;
            if (there && vs[x][r] < __builtin_inff()) largest = fmaxf(largest, vs[x][r]);
          }
          z[j][x][r] = v;
          m = fmaxf(m, v);
        }
      m = row_max(m);
      if constexpr (MASKED) largest = row_max(largest);
      before[j] = ref[j];
      const bool none = top[j] == NONE;
      grows |= m > top[j] || largest > big[j];
      top[j] = fmaxf(top[j], m);
      big[j] = fmaxf(big[j], largest);
      int e = __builtin_amdgcn_frexp_expf(big[j]);
      e = e < -80 ? -80 : e > 100 ? 100 : e;
      ref[j] = top[j] == NONE ? 0.f : fmaf(top[j], factor[j], (float)(e - 15));
      if (none) before[j] = NONE;
      if constexpr (MASKED) largest = 0.f;
    }
    if (__any(grows)) {
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        const float by = before[j] == NONE ? 0.f : __builtin_amdgcn_exp2f(before[j] - ref[j]);
        sum[j] *= by;
#pragma unroll
        for (int i = 0; i < NX; ++i) o[i][j] *= by;
      }
    }
#pragma unroll
    for (int j = 0; j < NY; ++j) {
#pragma unroll
      for (int x = 0; x < TILES; ++x) {
        _Float16 h[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p = __builtin_amdgcn_exp2f(fmaf(z[j][x][r], factor[j], -ref[j]));
          float y = p * vs[x][r];
          if constexpr (MASKED) {
            const bool there = seen_by[j] >> (4 * x + r) & 1;
            p = there ? p : 0.f;
            y = there ? y : 0.f;
          }
          sum[j] += p;
          h[r] = (_Float16)y;
        }
        __builtin_memcpy((char *)&w[x / 2][j] + 8 * (x % 2), h, 8);
      }
    }
  }

  // The end of group j: a part's sums, or the row itself.  A lane's outputs are DIM / 4
  // in a row from DIM / 4 g on.
  __device__ void store(const Work &w, const Row &r, int j, int part) const {
    const AttendArgs &a = w.a;
    const float total = row_sum(sum[j]);
    if (r.at < 0) return;
    const bool none = top[j] == NONE && total == 0.f;  // (NaN scores leave no largest)
    const int g = threadIdx.x % 64 / 16;
    constexpr int RUN = D / 4;
    const int d0 = g * RUN;
    const size_t row = r.at * a.heads + r.head;
    if (w.parts > 1) {
      const size_t at = row * w.parts + part;
      if (g == 0) w.ends[at] = float2{none ? NONE : ref[j], total};
      if (none) return;
      float *to = w.sums + at * D + d0;
#pragma unroll
      for (int c = 0; c < RUN / 4; ++c) {
        v4f v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = value(j, 4 * c + e);
        *(v4f *)(to + 4 * c) = v;
      }
      return;
    }
    const float inv = none ? 0.f : 1.f / total;
    if (a.lse && g == 0)
      a.lse[row] = none ? NONE : (ref[j] + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
#pragma unroll
    for (int c = 0; c < RUN; c += 8) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = c + e < RUN ? value(j, c + e) * inv : 0.f;
      put8(a, r, d0 + c, f, RUN - c);
    }
  }
  // Output d0 + n of the lane's run: o[i][j][r] is d = D / 4 g + D / 16 r + i.
  __device__ float value(int j, int n) const { return o[n % NX][j][n / NX]; }

  __device__ static void put8(const AttendArgs &a, const Row &r, int d, const float (&f)[8], int n) {
    char *to = (char *)a.out.p + 2 * (r.at * a.out.row + r.head * a.out.head + d);
    if (d >= (int)a.cache.dim) return;
    if (a.dtype == ROSETTA_BF16) put<bf16>(to, f, n);
    else put<f16>(to, f, n);
  }
  template <class T>
  __device__ static void put(char *to, const float (&f)[8], int n) {
    T h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (T)f[i];
    if (n >= 8) __builtin_memcpy(to, h, 16);
    else __builtin_memcpy(to, h, 8);
  }
};

// Whether a row at place i sees position t, base = its sequence's first row's; masks: of
// the row, or null.
__device__ inline bool sees(const Seq &s, const AttendArgs &a, const uint64_t *mask, int i,
                            int64_t t) {
  const int64_t j = t - s.sp.base;
  if (t >= s.length) return false;
  if (j < 0) return true;
  if (!a.masks) return j <= i;
  return j < s.sp.n && j < (int64_t)a.words * 64 && mask && (mask[j >> 6] >> (j & 63) & 1);
}

// [from, to) of part `part` of `length` positions, multiples of `unit` but for the end.
__device__ inline void part_of(int64_t length, int parts, int part, int unit, int64_t &from,
                               int64_t &to) {
  const int64_t units = (length + unit - 1) / unit;
  from = units * part / parts * unit;
  to = units * (part + 1) / parts * unit;
  to = to < length ? to : length;
}

// ---- few rows: the cache goes by once, straight to registers ----
template <int D, int NY>
__global__ void __launch_bounds__(256) k_attend_few(Work w) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const AttendArgs &a = w.a;
  const int lane = threadIdx.x % 64, m = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int kv_heads = (int)a.cache.kv_heads;
  unsigned id = blockIdx.x;
  const int head = id % kv_heads;
  id /= kv_heads;
  const int b = id % (unsigned)a.packed.batch;
  id /= (unsigned)a.packed.batch;
  const int part = id % (unsigned)w.parts, block = id / (unsigned)w.parts;
  const Seq s = seq_of(a, b, head);
  const int r0 = block * 16 * NY;
  if (r0 >= s.sp.n * w.group) return;
  auto row = [&](int j) { return row_of(s, r0 + 16 * j + m, w.group, head); };

  // product ks of 32 takes bytes 16 g + 8 (ks % 2) .. + 8 of chunk ks / 2 of 64
  Rows16<D, NY> x;
  auto first = [&](int ks) { return 64 * (ks / 2) + 16 * g + 8 * (ks % 2); };
  if (a.dtype == ROSETTA_BF16) x.template load<bf16>(a, row, first);
  else x.template load<f16>(a, row, first);

  // positions that some row sees, and that every row sees
  const int last = std::min((r0 + 16 * NY - 1) / w.group, s.sp.n - 1);
  int64_t end = a.masks ? s.length : std::min(s.length, s.sp.base + last + 1);
  const int64_t all = std::min(s.length, s.sp.base + (a.masks ? 0 : r0 / w.group + 1));
  int64_t from, to;
  part_of(end < 0 ? 0 : end, w.parts, part, 32, from, to);

  constexpr int NS = D / 64, VB = D / 16;  // K: 16 bytes of NS chunks, V: VB bytes of a row
  using vb = std::conditional_t<VB == 4, int, std::conditional_t<VB == 8, v2i, v4i>>;
  struct Step {
    v4i k[2][NS];
    vb v[2][4];
    v4f ks[2], vs[2];
    bool there;
  };
  const int dim = (int)a.cache.dim, stride = (int)a.cache.place_stride;
  int kat[NS], vat;
#pragma unroll
  for (int c = 0; c < NS; ++c) kat[c] = m * stride + (64 * c + 16 * g < dim ? 64 * c + 16 * g : 0);
  vat = 4 * g * stride + (VB * m < dim ? VB * m : 0);
  auto load = [&](Step &f, int64_t t) {
    f.there = true;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Sixteen at = sixteen_at(s, a, t + 16 * h);
      f.there = f.there && at.there;
#pragma unroll
      for (int c = 0; c < NS; ++c) f.k[h][c] = *(const v4i *)(at.k + kat[c]);
#pragma unroll
      for (int r = 0; r < 4; ++r) f.v[h][r] = *(const vb *)(at.v + vat + r * stride);
      __builtin_memcpy(&f.ks[h], at.ks + 4 * g, 16);
      __builtin_memcpy(&f.vs[h], at.vs + 4 * g, 16);
    }
  };
  auto use = [&](const Step &f, int64_t t) {
    v4f sc[2][NY];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < NY; ++j) sc[h][j] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < NS; ++c) {
        const v2i a0 = widen(f.k[h][c].x), a1 = widen(f.k[h][c].y);
        const v2i b0 = widen(f.k[h][c].z), b1 = widen(f.k[h][c].w);
        const v4i ka = {a0.x, a0.y, a1.x, a1.y}, kb = {b0.x, b0.y, b1.x, b1.y};
#pragma unroll
        for (int j = 0; j < NY; ++j) {
          sc[h][j] = mac(ka, x.q[j][2 * c], sc[h][j]);
          sc[h][j] = mac(kb, x.q[j][2 * c + 1], sc[h][j]);
        }
      }
    v4i p[1][NY];
    if (t + 32 <= all && f.there) {
      x.template weigh<false>(sc, f.ks, f.vs, [](int, int, int) { return true; }, p);
    } else {
      const bool there[2] = {sixteen_at(s, a, t).there, sixteen_at(s, a, t + 16).there};
      const uint64_t *mask[NY];
      int at[NY];
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        const Row r = row(j);
        at[j] = r.i;
        mask[j] = a.masks && r.at >= 0 ? a.masks + r.at * a.words : nullptr;
      }
      x.template weigh<true>(sc, f.ks, f.vs, [&](int h, int r, int j) {
        return there[h] && sees(s, a, mask[j], at[j], t + 16 * h + 4 * g + r);
      }, p);
    }
    auto bytes = [&](int h, int r, int word) {
      if constexpr (VB == 4) return (u32)f.v[h][r];
      else return (u32)f.v[h][r][word];
    };
#pragma unroll
    for (int word = 0; word < VB / 4; ++word) {
      auto turn = [&](auto byte) {
        constexpr int I = decltype(byte)::value;
        const v4i v = {(int)widen_two<I>(bytes(0, 0, word), bytes(0, 1, word)),
                       (int)widen_two<I>(bytes(0, 2, word), bytes(0, 3, word)),
                       (int)widen_two<I>(bytes(1, 0, word), bytes(1, 1, word)),
                       (int)widen_two<I>(bytes(1, 2, word), bytes(1, 3, word))};
#pragma unroll
        for (int j = 0; j < NY; ++j) x.o[4 * word + I][j] = mac(v, p[0][j], x.o[4 * word + I][j]);
      };
      turn(std::integral_constant<int, 0>{});
      turn(std::integral_constant<int, 1>{});
      turn(std::integral_constant<int, 2>{});
      turn(std::integral_constant<int, 3>{});
    }
  };
  // the waves take steps of 32 positions in turn, the next one's loads under way
  constexpr int TURN = 4 * 32;
  Step f, n;
  int64_t t = from + 32 * wave;
  if (t < to) load(f, t);
  for (; t < to; t += 2 * TURN) {
    if (t + TURN < to) load(n, t + TURN);
    use(f, t);
    if (t + TURN >= to) break;
    if (t + 2 * TURN < to) load(f, t + 2 * TURN);
    use(n, t + TURN);
  }

  // The waves' sums together, in order: waves 2 and 3 to 0 and 1, 1 to 0.
  constexpr int EACH = 64 * (4 * Rows16<D, NY>::NX * NY + 3 * NY);
  float *mine = (float *)lds;
#pragma unroll
  for (int half = 2; half >= 1; half /= 2) {
    if (wave >= half && wave < 2 * half) {
      float *to = mine + (wave - half) * EACH + lane;
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        to[(3 * j) * 64] = x.top[j];
        to[(3 * j + 1) * 64] = x.ref[j];
        to[(3 * j + 2) * 64] = x.sum[j];
      }
      v4f *of = (v4f *)(mine + (wave - half) * EACH + 3 * NY * 64) + lane;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int j = 0; j < NY; ++j) of[(i * NY + j) * 64] = x.o[i][j];
    }
    __syncthreads();
    if (wave < half) {
      const float *of = mine + wave * EACH + lane;
      const v4f *o = (const v4f *)(mine + wave * EACH + 3 * NY * 64) + lane;
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        const float top = of[(3 * j) * 64], ref = of[(3 * j + 1) * 64];
        const bool here = x.top[j] != NONE, there = top != NONE;
        const float both = !here ? ref : !there ? x.ref[j] : fmaxf(ref, x.ref[j]);
        const float fa = here ? __builtin_amdgcn_exp2f(x.ref[j] - both) : 0.f;
        const float fb = there ? __builtin_amdgcn_exp2f(ref - both) : 0.f;
        x.ref[j] = both;
        x.top[j] = fmaxf(x.top[j], top);
        x.sum[j] = x.sum[j] * fa + of[(3 * j + 2) * 64] * fb;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) x.o[i][j] = x.o[i][j] * fa + o[(i * NY + j) * 64] * fb;
      }
    }
    __syncthreads();
  }
  if (wave == 0) {
#pragma unroll
    for (int j = 0; j < NY; ++j) x.store(w, row(j), j, part);
  }
}

// ---- parts of a sequence joined: one thread to four outputs of a row ----
template <int D>
__global__ void __launch_bounds__(256) k_attend_join(Work w) {
  const AttendArgs &a = w.a;
  constexpr int LANES = D / 4, ROWS = 256 / LANES;
  const Span sp = span_of(a.packed.starts, a.packed.lens, blockIdx.y, a.packed.rows);
  const int n = sp.n < (int)a.max_rows ? sp.n : (int)a.max_rows;
  const int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (r >= n * (int64_t)a.heads) return;
  const int lane = threadIdx.x % LANES;
  const size_t row = sp.first * a.heads + r;
  const float2 *ends = w.ends + row * w.parts;
  const v4f *sums = (const v4f *)(w.sums + row * w.parts * D) + lane;
  float ref = NONE;
  bool any = false;
  for (int p = 0; p < w.parts; ++p) {
    any |= ends[p].x != NONE;
    ref = fmaxf(ref, ends[p].x);
  }
  float total = 0.f;
  v4f o = {0, 0, 0, 0};
  for (int p = 0; p < w.parts; ++p) {
    const float2 e = ends[p];
    if (e.x == NONE) continue;
    const float f = __builtin_amdgcn_exp2f(e.x - ref);
    total += e.y * f;
    o += sums[(size_t)p * LANES] * f;
  }
  const float inv = any ? 1.f / total : 0.f;
  if (a.lse && lane == 0) a.lse[row] = any ? (ref + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : NONE;
  if (lane * 4 >= (int)a.cache.dim) return;
  Row at;
  at.at = sp.first + (int)(r / (int64_t)a.heads);
  at.head = (int)(r % (int64_t)a.heads);
  const float f[8] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  Rows16<D, 1>::put8(a, at, lane * 4, f, 4);
}

}  // namespace

namespace {

struct Plan {
  int d, ny, parts, row_blocks;
};

Plan plan_of(size_t heads, size_t kv_heads, size_t dim, size_t batch, size_t max_rows,
             size_t positions) {
  Plan p;
  p.d = dim <= 64 ? 64 : dim <= 128 ? 128 : 256;
  const size_t group = heads / kv_heads, rows = max_rows * group;
  p.ny = rows <= 16 || p.d == 256 ? 1 : 2;  // (two groups of 256 do not fit the registers)
  p.row_blocks = (int)((rows + 16 * p.ny - 1) / (16 * p.ny));
  const size_t blocks = batch * kv_heads * p.row_blocks;
  size_t parts = blocks ? (1024 + blocks - 1) / blocks : 1;
  parts = std::min(parts, (positions + 127) / 128);
  p.parts = (int)std::max<size_t>(1, std::min<size_t>(parts, 128));
  return p;
}

template <class F>
hipError_t by_dim(int d, F f) {
  if (d == 64) return f(std::integral_constant<int, 64>{});
  if (d == 128) return f(std::integral_constant<int, 128>{});
  return f(std::integral_constant<int, 256>{});
}

}  // namespace

size_t kv_attention_workspace(size_t heads, size_t kv_heads, size_t dim, size_t batch, size_t rows,
                              size_t max_rows, size_t positions) {
  const Plan p = plan_of(heads, kv_heads, dim, batch, max_rows, positions);
  return p.parts > 1 ? rows * heads * p.parts * (p.d * sizeof(float) + sizeof(float2)) : 0;
}

hipError_t launch_kv_attention(const AttendArgs &a, hipStream_t st) {
  const size_t positions = a.packed.table_len << a.cache.page_log;
  const Plan p = plan_of(a.heads, a.cache.kv_heads, a.cache.dim, a.packed.batch, a.max_rows, positions);
  Work w{a, (int)(a.heads / a.cache.kv_heads), p.parts, p.row_blocks, nullptr, nullptr};
  if (p.parts > 1) {
    w.sums = (float *)a.workspace;
    w.ends = (float2 *)(w.sums + a.packed.rows * a.heads * p.parts * p.d);
  }
  const size_t blocks = a.packed.batch * a.cache.kv_heads * p.parts * p.row_blocks;
  const size_t joins = (a.max_rows * a.heads * p.d / 4 + 255) / 256;
  if (!grid_fits(blocks, 256) || (p.parts > 1 && (a.packed.batch > 65535 || !grid_fits(joins * a.packed.batch, 256))))
    return hipErrorInvalidConfiguration;
  return by_dim(p.d, [&](auto d) {
    constexpr int D = decltype(d)::value;
    hipError_t e = hipSuccess;
    auto few = [&](auto ny) {
      constexpr int NY = decltype(ny)::value;
      constexpr size_t LDS = 2 * 64 * (4 * (D / 16) * NY + 3 * NY) * sizeof(float);
      e = allow_lds(k_attend_few<D, NY>, LDS);
      if (e != hipSuccess) return;
      hipLaunchKernelGGL((k_attend_few<D, NY>), dim3((unsigned)blocks), dim3(256), LDS, st, w);
      e = hipGetLastError();
    };
    if (p.ny == 1) few(std::integral_constant<int, 1>{});
    else if constexpr (D < 256) few(std::integral_constant<int, 2>{});
    if (e != hipSuccess || p.parts == 1) return e;
    hipLaunchKernelGGL(k_attend_join<D>, dim3((unsigned)joins, (unsigned)a.packed.batch), dim3(256), 0,
                       st, w);
    return hipGetLastError();
  });
}

}  // namespace rosetta
