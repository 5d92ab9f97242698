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
// v_scale, are rounded to f16 (by 2^-11 of themselves at most; a bf16 output by 2^-8);
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

// What a score is multiplied with, at least: not 0, since what is not seen has a score of
// -infinity, and so little that no other score, 2^128 at most, comes to anything by it.
constexpr float LEAST = 0x1p-149f;

// (by value: std::min's references kept its operands in scratch memory, and with them
// all that follows from them in vector registers)
__device__ inline int least(int a, int b) { return a < b ? a : b; }

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
// The larger ones, NaN passed over (fmaxf would quiet each operand first).
__device__ inline float max2(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ inline u32 max3(u32 a, u32 b, u32 c) {
  u32 r;
  asm("v_max3_u32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ inline u32 bits_of(float a) { return __builtin_bit_cast(u32, a); }
__device__ inline float row_max(float a) {
  return across(a, [](float x, float y) { return max2(x, y); });
}
__device__ inline float row_sum(float a) {
  return across(a, [](float x, float y) { return x + y; });
}
// ---- scales of any size ----
//
// The first pass over the cache takes for granted, but looks, what holds for scales as caches
// have them:
//  - no key's scale is FAR.  Products <q, K> go up to 2^28 (q to 2^13, K to 2^7, 256 of them),
//    and times 2^100 past what 32 bits hold.
//  - no value's is.  A row's exponentials are at most 2^15 over the largest scale of its values,
//    and too many would be below what 32 bits hold for their sum.
//  - the largest of the values' scales is not alone.  A row's reference is that of its largest
//    score and of its largest scale, which need not be one position's: where the largest scale
//    weighs little, all weights are small beside it.  f16 holds them, from 2^15 on, in steps of
//    2^-24, so that n of them are off by n 2^-25 together; where the row's largest output is LOST
//    times n or more, that is 2^-11 of it at most.  It is PLENTY, too, or more, so that the largest
//    weight is 2^-2 at least and those beside it have their bits.
//  - they do not grow by APART from one step to the next: what was added up would be 0 beside
//    them.
// Where one does not hold, the pass is made again, with keys' scales 2^-28 as large (and 2^28
// times as much to each score) if some are FAR, with values' so if some of them are, and a row's
// reference that of its largest product of exponential and scale, which takes twice as long together.  To look costs a prompt of 8192
// 688 us -> 697, one of 4096 with heads of 64 125 -> 130, of 256 328 -> 343, trees of 25 30.5
// -> 31.6, 64 tokens 134.2 -> 134.7.
constexpr float FAR = 0x1p100f, NEARER = 0x1p-28f;
constexpr int AGAIN = 1, FAR_KEYS = 2, FAR_VALUES = 4;  // what a pass asks for
constexpr float LOST = 0x1p-7f, PLENTY = 32;  // (2^-25, values up to 2^7, 2^11; 2^-2 2^7)
constexpr float APART = 0x1p60f;
__device__ inline bool is_apart(float before, float now) {
  return now > before * APART && before > 0.f;
}

// The scales of a position: where one of them is no number, or infinite, or it is not there,
// the score is none, and the value counts as 0, so that rows that do not see it are not touched.
__device__ inline void settle(float &k, float &v, bool there) {
  const bool fine = there && fabsf(v) < __builtin_inff() && fabsf(k) < __builtin_inff();
  k = fine ? k : __builtin_nanf("");
  v = fine ? v : 0.f;
}

// The value N lanes on, in a ring of sixteen.
template <int N>
__device__ inline float turned(float a) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, a), 0x120 + N,
                                                            0xf, 0xf, false));
}

// 2^x as two factors, the second 1 but where one number would not hold it: references lie as far
// apart as the values' scales.
struct Power {
  float a, b;
};
__device__ inline Power power(float x) {
  const float near = fmaxf(x, -100.f);
  return {__builtin_amdgcn_exp2f(near), __builtin_amdgcn_exp2f(x - near)};
}

// A sum and outputs 2^x times as large.
__device__ inline void bring(float &sum, v4f &o, float x) {
  if (x < -100.f) {
    x += 100.f;
    sum *= 0x1p-100f;
    o *= 0x1p-100f;
  }
  const float by = __builtin_amdgcn_exp2f(x);
  sum *= by;
  o *= by;
}

// What a launch works on.
struct Work {
  AttendArgs a;
  int group, parts;  // heads to a head of the cache, parts of a sequence
  int row_blocks;    // workgroups to the rows of a sequence and head
  int joiners;       // groups of threads to the parts of a row
  float *sums;       // parts > 1: [rows][heads][parts][DIM], (reference, sum) [..][parts]
  float2 *ends;
};

// The launch's arguments where they lie, for a function that is called: an address that the
// compiler knows to be the same in all lanes.
__device__ inline const Work *alike(const Work *w) {
  const uint64_t p = (uintptr_t)w;
  const u32 lo = __builtin_amdgcn_readfirstlane((u32)p);
  const u32 hi = __builtin_amdgcn_readfirstlane((u32)(p >> 32));
  return (const Work *)(const __attribute__((address_space(4))) Work *)(((uint64_t)hi << 32) | lo);
}

// A word that a whole wave reads, through the scalar cache: what a launch only reads, at
// an address that all lanes share.
__device__ inline int shared_word(const int *p) {
  return *(const __attribute__((address_space(4))) int *)(uintptr_t)p;
}

// One sequence and head of the cache, as its workgroups see it.  Positions are 32-bit, as
// lens is (a sequence without any has base = -n).
struct Seq {
  int first, n, base;
  int length;  // positions that are in the table
  const int *table;
  const int8_t *k, *v;  // of the head
  const float *ks, *vs;
};
__device__ inline Seq seq_of(const AttendArgs &a, int b, int head) {
  Seq s;
  const Packed &r = a.packed;
  const int lens = shared_word(r.lens + b);
  const Span sp = span_of(shared_word(r.starts + b), shared_word(r.starts + b + 1), lens, r.rows);
  s.first = sp.first;
  s.n = sp.n < (int)a.max_rows ? sp.n : (int)a.max_rows;
  s.base = lens > 0 ? lens - sp.n : -sp.n;
  const int64_t capacity = (int64_t)r.table_len << a.cache.page_log;
  s.length = lens < 0 ? 0 : lens > capacity ? (int)capacity : lens;
  s.table = r.table + b * r.table_stride;
  s.k = a.cache.k + head * a.cache.head_stride;
  s.v = a.cache.v + head * a.cache.head_stride;
  s.ks = a.cache.k_scale + head * a.cache.scale_head_stride;
  s.vs = a.cache.v_scale + head * a.cache.scale_head_stride;
  return s;
}

// The page of positions t .. + 15 (t a multiple of 16, so that they lie in one), or what
// names none.  Asked for ahead of what is read there.
__device__ inline int entry_at(const Seq &s, const AttendArgs &a, int t) {
  const u32 at = (u32)t >> a.cache.page_log;
  return at < a.packed.table_len ? shared_word(s.table + at) : -1;
}

// Those positions, of the entry's page.
struct Sixteen {
  const int8_t *k, *v;
  const float *ks, *vs;
};
__device__ inline bool is_page(const AttendArgs &a, int entry) {
  return (size_t)(u32)entry < a.cache.pages && entry >= 0;
}
__device__ inline Sixteen sixteen_at(const Seq &s, const AttendArgs &a, int entry, int t) {
  const Cache &c = a.cache;
  const size_t pg = is_page(a, entry) ? entry : 0;  // (where none, page 0 is read and not used)
  const size_t place = t & ((1 << c.page_log) - 1);
  const size_t at = pg * c.page_stride + place * c.place_stride;
  const size_t sat = pg * c.scale_page_stride + place;
  return {s.k + at, s.v + at, s.ks + sat, s.vs + sat};
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
  x.at = x.i < s.n ? s.first + x.i : -1;
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
  float big[NY];      // the largest v_scale, whatever its sign
  float ref[NY], sum[NY];
  v4f o[NX][NY];

  // q's values k .. + 7 of a lane come from its row's first(ks) on.  `at` gives the Row
  // of group j, of which row `some` of the call is one for sure.  All of it is asked for
  // before any is used (under conditions of their own the loads went one after the other).
  template <class T, class At, class First>
  __device__ void load(const AttendArgs &a, int some, At at, First first) {
    v4i raw[NY][KS];
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      const Row r = at(j);
      const T *from = (const T *)a.q.p + (r.at >= 0 ? r.at : some) * a.q.row + r.head * a.q.head;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int d = first(ks);
        __builtin_memcpy(&raw[j][ks], from + (d < (int)a.cache.dim ? d : 0), 16);
      }
    }
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      const bool mine = at(j).at >= 0;
      float f[KS][8];
      float m = 0.f, odd = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bool in = mine && first(ks) < (int)a.cache.dim;
        T x[8];
        __builtin_memcpy(x, &raw[j][ks], 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f[ks][i] = in ? (float)x[i] : 0.f;
          m = fmaxf(m, fabsf(f[ks][i]));
          odd += f[ks][i] * 0.f;
        }
      }
      m = row_max(m);
      odd = row_sum(odd);  // NaN where the row holds NaN or an infinity
      // (no more than 2^120, which brings bf16's smallest to f16's normal numbers, and keeps
      // the factor one)
      const int up = m > 0.f ? least(13 - __builtin_amdgcn_frexp_expf(m), 120) : 0;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        _Float16 h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = (_Float16)ldexpf(f[ks][i], up);
        __builtin_memcpy(&q[j][ks], h, 16);
      }
      factor[j] = fmaxf(ldexpf(a.scale * 1.44269504088896340736f, -up), LEAST) + odd;
    }
    clear();
  }
  __device__ void clear() {
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      top[j] = NONE;
      big[j] = 0.f;
      ref[j] = 0.f;
      sum[j] = 0.f;
#pragma unroll
      for (int i = 0; i < NX; ++i) o[i][j] = v4f{0, 0, 0, 0};
    }
  }
  // What the scales that the rows saw, over n positions, ask for.
  __device__ int asks(bool far_keys, bool apart, int n) const {
    // (a few outputs of a row say it as a rule)
    bool again = some_lost<1>(n), far = false;
    if (__any(again)) again = some_lost<NX>(n);
#pragma unroll
    for (int j = 0; j < NY; ++j) far |= big[j] >= FAR;
    return (far_keys ? FAR_KEYS : 0) | (__any(far) ? FAR_VALUES : 0) |
           (__any(again || apart) ? AGAIN : 0);
  }
  template <int X>
  __device__ bool some_lost(int n) const {
    const float enough = fmaxf((float)n * LOST, PLENTY);
    bool lost = false;
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      float l = 0.f;
#pragma unroll
      for (int i = 0; i < X; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) l = max2(l, fabsf(o[i][j][r]));
      lost |= row_max(l) < enough && big[j] > 0.f && sum[j] > 0.f;
    }
    return lost;
  }
  // Scores as they are, of keys' scales NEARER times as large.
  __device__ void nearer_keys() {
#pragma unroll
    for (int j = 0; j < NY; ++j)
      factor[j] = factor[j] > LEAST ? factor[j] * (1 / NEARER) : factor[j];
  }
  // Sums that are as much smaller as the outputs of values' scales NEARER times as large.
  __device__ void nearer_values() {
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      ref[j] += 28;
      sum[j] *= NEARER;
    }
  }

  // Scores s[x][j] (tile x of TILES, four positions of row j): times their keys' scales,
  // and the largest so far.
  template <int TILES>
  __device__ static void scaled(v4f (&s)[TILES][NY], int x, const v4f &ks, float (&m)[NY]) {
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      s[x][j] *= ks;
      m[j] = max3(m[j], s[x][j][0], s[x][j][1]);
      m[j] = max3(m[j], s[x][j][2], s[x][j][3]);
    }
  }

  // The references for the scores s, m their largest: what was added up so far goes over to
  // them.  vs(x): the values' scales of the lane's positions, most() the largest of all.
  // bits(j), where `masked` (the same in all lanes): bit 16 x + r says whether row j sees
  // position r of tile x; what it does not see becomes -infinity.
  template <int TILES, class Vs, class Most, class Bits>
  __device__ void refer(v4f (&s)[TILES][NY], float (&m)[NY], Vs vs, Most most, bool masked,
                        Bits bits, int *apart) {
    float largest[NY];
    if (masked) {
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        const uint64_t seen = bits(j);
        float l = 0.f;
        m[j] = NONE;
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
          const u32 b = (u32)(seen >> (16 * x)) & 0xf;
          const v4f v = vs(x);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bool there = b & (1u << r);
            s[x][j][r] = there ? s[x][j][r] : NONE;
            l = max2(l, there ? fabsf(v[r]) : 0.f);
            m[j] = max2(m[j], s[x][j][r]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        largest[j] = row_max(l);
      }
    } else {
      const float l = most();
#pragma unroll
      for (int j = 0; j < NY; ++j) largest[j] = l;
    }
    bool grows = false;
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      m[j] = row_max(m[j]);
      grows |= m[j] > top[j] || largest[j] > big[j];
    }
    if (__any(grows)) {
      bool far_apart = false;
#pragma unroll
      for (int j = 0; j < NY; ++j) far_apart |= is_apart(big[j], largest[j]);
      if (__any(far_apart)) *apart = 1;
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        const float before = ref[j];
        const bool none = top[j] == NONE;
        top[j] = max2(top[j], m[j]);
        big[j] = max2(big[j], largest[j]);
        int e = __builtin_amdgcn_frexp_expf(big[j]);
        e = e < -80 ? -80 : e > 100 ? 100 : e;
        ref[j] = top[j] == NONE ? 0.f : fmaf(top[j], factor[j], (float)(e - 15));
        const float by = none ? 0.f : __builtin_amdgcn_exp2f(before - ref[j]);
        sum[j] *= by;
#pragma unroll
        for (int i = 0; i < NX; ++i) o[i][j] *= by;
      }
    }
  }

  // The same in the other pass: the reference is that of the largest product, and such that no
  // exponential is past 2^95.
  template <int TILES, class Vs, class Bits>
  __device__ void refer_odd(v4f (&s)[TILES][NY], Vs vs, bool masked, Bits bits) {
#pragma unroll
    for (int j = 0; j < NY; ++j) {
      const uint64_t seen = masked ? bits(j) : ~(uint64_t)0;
      float m = NONE, lift = NONE;
#pragma unroll
      for (int x = 0; x < TILES; ++x) {
        const u32 b = (u32)(seen >> (16 * x)) & 0xf;
        const v4f v = vs(x);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[x][j][r] = b & (1u << r) ? s[x][j][r] : NONE;
          m = max2(m, s[x][j][r]);
          lift = max2(lift, fmaf(s[x][j][r], factor[j], __builtin_amdgcn_logf(fabsf(v[r]))));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      m = row_max(m);
      lift = row_max(lift) - 15;
      const float before = ref[j];
      const bool none = top[j] == NONE;
      top[j] = max2(top[j], m);
      ref[j] = max3(fmaf(top[j], factor[j], -95.f), lift, none ? NONE : before);
      if (top[j] == NONE) ref[j] = 0.f;
      const Power by = power(none ? 0.f : before - ref[j]);
      sum[j] = sum[j] * by.a * by.b;
#pragma unroll
      for (int i = 0; i < NX; ++i) o[i][j] = o[i][j] * by.a * by.b;
    }
  }

  // The weights of row j in a tile, to half `half` of a fragment.
  __device__ void weigh(const v4f &s, const v4f &vs, int j, int half, v4i &w) {
    _Float16 h[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[r], factor[j], -ref[j]));
      sum[j] += p;
      h[r] = (_Float16)(p * vs[r]);
    }
    __builtin_memcpy((char *)&w + 8 * half, h, 8);
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
      // (a reference that is no number would be passed over in the join: the sum says it)
      if (g == 0) w.ends[at] = float2{none ? NONE : ref[j] == ref[j] ? ref[j] : 0.f, total};
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

// The first n of 64 bits.
__device__ inline uint64_t below(int64_t n) {
  return n <= 0 ? 0 : n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1;
}

// Which of the 64 positions from t on the row at place i sees (mask: its words, where the
// call has masks and the row is one).
__device__ inline uint64_t seen_from(const Seq &s, const AttendArgs &a, const uint64_t *mask, int i,
                                     int t) {
  const uint64_t there = below(s.length - t);
  const int j = t - s.base;  // of bit 0
  if (!a.masks) return there & below((int64_t)i + 1 - j);
  uint64_t m = 0;
  if (mask && j > -64 && j < s.n) {
    if (j < 0) {
      m = mask[0] << -j;
    } else {
      const size_t word = j >> 6;
      const int by = j & 63;
      if (word < a.words) m = mask[word] >> by;
      if (by && word + 1 < a.words) m |= mask[word + 1] << (64 - by);
    }
    m &= below(s.n - j);
  }
  return there & (below(-(int64_t)j) | m);
}

// [from, to) of part `part` of `length` positions, multiples of `unit` but for the end.
__device__ inline void part_of(int length, int parts, int part, int unit, int &from, int &to) {
  const int64_t units = ((int64_t)length + unit - 1) / unit;
  from = (int)(units * part / parts * unit);
  const int64_t end = units * (part + 1) / parts * unit;
  to = end < length ? (int)end : length;
}

// ---- few rows: the cache goes by once, straight to registers ----
//
// The waves take steps of 32 positions in turn.  A step's keys make room for the next
// one's as soon as the scores are there, its values after the second product: no
// register waits twice, and the other waves' work covers the rest of the way.
//
// ODD: the other pass, `given` what the first one asked for.  That returns what it asks for, the same in all
// threads; if it does, nothing is stored.
template <int D, int NY, bool ODD>
__device__ __forceinline__ int attend_few(const Work &w, char *lds, int given) {
  const AttendArgs &a = w.a;
  const int lane = threadIdx.x % 64, m = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int kv_heads = (int)a.cache.kv_heads;
  // Several groups of rows read the same part of the cache: one right after the other, so
  // that they find it in the caches (trees of 25 in seven groups 28 us, 35 with the
  // sequences in between; 32 all on one XCD, which then gets the long sequences).  With one
  // group the sequences go by in turn (64 of 2048 to 8192 positions 133 us, 141 with their
  // parts next to each other).
  unsigned id = blockIdx.x;
  const unsigned batch = (unsigned)a.packed.batch, parts = (unsigned)w.parts;
  const int head = id % kv_heads;
  id /= kv_heads;
  const int block = id % (unsigned)w.row_blocks;
  id /= (unsigned)w.row_blocks;
  const int b = w.row_blocks > 1 ? id / parts : id % batch;
  const int part = w.row_blocks > 1 ? id % parts : id / batch;
  const Seq s = seq_of(a, b, head);
  const int r0 = block * 16 * NY;
  if (r0 >= s.n * w.group) return 0;
  auto row = [&](int j) { return row_of(s, r0 + 16 * j + m, w.group, head); };

  // positions that some row sees, and that every row sees
  const int last = least((r0 + 16 * NY - 1) / w.group, s.n - 1);
  const int end = a.masks ? s.length : least(s.length, s.base + last + 1);
  const int all = least(s.length, s.base + (a.masks ? 0 : r0 / w.group + 1));
  int from, to;
  part_of(end < 0 ? 0 : end, w.parts, part, 32, from, to);

  constexpr int NS = D / 64, VB = D / 16;  // K: 16 bytes of NS chunks, V: VB bytes of a row
  using vb = std::conditional_t<VB == 4, int, std::conditional_t<VB == 8, v2i, v4i>>;
  v4i fk[2][NS];
  vb fv[2][4];
  v4f fks[2], fvs[2];
  const u32 dim = (u32)a.cache.dim, stride = (u32)a.cache.place_stride;
  u32 kat[NS];
#pragma unroll
  for (int c = 0; c < NS; ++c) kat[c] = m * stride + (64 * c + 16 * g < dim ? 64 * c + 16 * g : 0);
  const u32 vat = 4 * g * stride + (VB * m < dim ? VB * m : 0);
  auto load_keys = [&](const Sixteen (&at)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int c = 0; c < NS; ++c) fk[h][c] = *(const v4i *)(at[h].k + kat[c]);
    }
  };
  auto load_values = [&](const Sixteen (&at)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int r = 0; r < 4; ++r) fv[h][r] = *(const vb *)(at[h].v + vat + r * stride);
    }
  };
  auto load_scales = [&](const Sixteen (&at)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      __builtin_memcpy(&fks[h], at[h].ks + 4 * g, 16);
      __builtin_memcpy(&fvs[h], at[h].vs + 4 * g, 16);
    }
  };
  constexpr int TURN = 4 * 32;
  // product ks of 32 takes bytes 16 g + 8 (ks % 2) .. + 8 of chunk ks / 2 of 64
  Rows16<D, NY> x;
  auto first = [&](int ks) { return 64 * (ks / 2) + 16 * g + 8 * (ks % 2); };
  // behind the waves' sums: whether a wave met a key's scale that is FAR, values' that are APART
  // (four words each), and what all of it comes to
  constexpr int EACH = 64 * (4 * Rows16<D, NY>::NX * NY + 4 * NY);
  int *asked = (int *)lds + 2 * EACH;
  asked[4 + wave] = 0;
  bool far_keys = false;  // (this wave's, the same in all lanes)
  // The scales of a step settled: the largest of the values', and whether one of the keys' is FAR.
  auto settle_step = [&](const int (&entries)[2], int t, float &most) {
    const int room = s.length - t - 4 * g;
    bool far = false;
    most = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool page = is_page(a, entries[h]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float k = fks[h][r], v = fvs[h][r];
        settle(k, v, page && 16 * h + r < room);
        fks[h][r] = k;
        fvs[h][r] = v;
        most = max2(most, fabsf(v));
        far |= fabsf(k) >= FAR;
      }
    }
    return __any(far);
  };
  int t = from + 32 * wave;
  // table entries: of this step, and of the next
  int now[2], next[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    now[h] = t < to ? entry_at(s, a, t + 16 * h) : -1;
    next[h] = t + TURN < to ? entry_at(s, a, t + TURN + 16 * h) : -1;
  }
  if (t < to) {
    const Sixteen at[2] = {sixteen_at(s, a, now[0], t), sixteen_at(s, a, now[1], t + 16)};
    load_keys(at);
    load_scales(at);
    load_values(at);
  }

  if (a.dtype == ROSETTA_BF16) x.template load<bf16>(a, s.first, row, first);
  else x.template load<f16>(a, s.first, row, first);
  if (given & FAR_KEYS) x.nearer_keys();

  for (; t < to; t += TURN) {
    const bool more = t + TURN < to;
    const Sixteen ahead[2] = {sixteen_at(s, a, next[0], t + TURN),
                              sixteen_at(s, a, next[1], t + TURN + 16)};
    int later[2] = {-1, -1};
    if (t + 2 * TURN < to) {
#pragma unroll
      for (int h = 0; h < 2; ++h) later[h] = entry_at(s, a, t + 2 * TURN + 16 * h);
    }
    v4f sc[2][NY];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < NY; ++j) sc[h][j] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < NS; ++c) {
        const v2i a0 = widen(fk[h][c].x), a1 = widen(fk[h][c].y);
        const v2i b0 = widen(fk[h][c].z), b1 = widen(fk[h][c].w);
        const v4i ka = {a0.x, a0.y, a1.x, a1.y}, kb = {b0.x, b0.y, b1.x, b1.y};
#pragma unroll
        for (int j = 0; j < NY; ++j) {
          sc[h][j] = mac(ka, x.q[j][2 * c], sc[h][j]);
          sc[h][j] = mac(kb, x.q[j][2 * c + 1], sc[h][j]);
        }
      }
    if (more) load_keys(ahead);
    // The largest of the scales, as bits: of numbers that are positive and finite, of
    // which all are as a rule.
    u32 tops[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        tops[0] = max3(tops[0], bits_of(fks[h][r]), bits_of(fks[h][r + 1]));
        tops[1] = max3(tops[1], bits_of(fvs[h][r]), bits_of(fvs[h][r + 1]));
      }
    float most = __builtin_bit_cast(float, tops[1]);
    if (ODD || __any(tops[0] >= bits_of(FAR) || tops[1] >= bits_of(FAR))) {
      const bool now_far = settle_step(now, t, most);
      if constexpr (ODD) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          fks[h] *= given & FAR_KEYS ? NEARER : 1.f;
          fvs[h] *= given & FAR_VALUES ? NEARER : 1.f;
        }
      } else {
        far_keys |= now_far;
      }
    }
    v4i p[1][NY];
    const bool there[2] = {is_page(a, now[0]), is_page(a, now[1])};
    const uint64_t in = (there[0] ? 0xffffu : 0u) | (there[1] ? 0xffff0000u : 0u);
    float largest[NY];
#pragma unroll
    for (int j = 0; j < NY; ++j) largest[j] = NONE;
#pragma unroll
    for (int h = 0; h < 2; ++h) x.template scaled<2>(sc, h, fks[h], largest);
    const bool masked = !(t + 32 <= all && there[0] && there[1]);
    auto vs = [&](int h) { return fvs[h]; };
    auto bits = [&](int j) {
      const Row r = row(j);
      const uint64_t *mask = a.masks && r.at >= 0 ? a.masks + r.at * a.words : nullptr;
      return (seen_from(s, a, mask, r.i, t) & in) >> (4 * g);
    };
    if constexpr (ODD) x.template refer_odd<2>(sc, vs, masked, bits);
    else
      x.template refer<2>(
          sc, largest, vs, [&] { return row_max(most); }, masked, bits, asked + 4 + wave);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < NY; ++j) x.weigh(sc[h][j], fvs[h], j, h, p[0][j]);
    if (more) load_scales(ahead);
    auto bytes = [&](int h, int r, int word) {
      if constexpr (VB == 4) return (u32)fv[h][r];
      else return (u32)fv[h][r][word];
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
    if (more) load_values(ahead);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      now[h] = next[h];
      next[h] = later[h];
    }
  }
  if (given & FAR_VALUES) x.nearer_values();

  // The waves' sums together, in order: waves 2 and 3 to 0 and 1, 1 to 0.
  float *mine = (float *)lds;
  if (!ODD) asked[wave] = far_keys;
#pragma unroll
  for (int half = 2; half >= 1; half /= 2) {
    if (wave >= half && wave < 2 * half) {
      float *to = mine + (wave - half) * EACH + lane;
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        to[(4 * j) * 64] = x.top[j];
        to[(4 * j + 1) * 64] = x.ref[j];
        to[(4 * j + 2) * 64] = x.sum[j];
        to[(4 * j + 3) * 64] = x.big[j];
      }
      v4f *of = (v4f *)(mine + (wave - half) * EACH + 4 * NY * 64) + lane;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int j = 0; j < NY; ++j) of[(i * NY + j) * 64] = x.o[i][j];
    }
    __syncthreads();
    if (wave < half) {
      const float *of = mine + wave * EACH + lane;
      const v4f *o = (const v4f *)(mine + wave * EACH + 4 * NY * 64) + lane;
      bool apart = false;
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        const float top = of[(4 * j) * 64], ref = of[(4 * j + 1) * 64], big = of[(4 * j + 3) * 64];
        const bool here = x.top[j] != NONE, there = top != NONE;
        const float both = !here ? ref : !there ? x.ref[j] : fmaxf(ref, x.ref[j]);
        const float da = here ? x.ref[j] - both : NONE, db = there ? ref - both : NONE;
        x.ref[j] = both;
        x.top[j] = fmaxf(x.top[j], top);
        if constexpr (ODD) {
          const Power fa = power(da), fb = power(db);
          x.sum[j] = x.sum[j] * fa.a * fa.b + of[(4 * j + 2) * 64] * fb.a * fb.b;
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
            x.o[i][j] = x.o[i][j] * fa.a * fa.b + o[(i * NY + j) * 64] * fb.a * fb.b;
        } else {
          const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
          x.sum[j] = x.sum[j] * fa + of[(4 * j + 2) * 64] * fb;
#pragma unroll
          for (int i = 0; i < D / 16; ++i) x.o[i][j] = x.o[i][j] * fa + o[(i * NY + j) * 64] * fb;
          apart |= is_apart(x.big[j], big) || is_apart(big, x.big[j]);
          x.big[j] = fmaxf(x.big[j], big);
        }
      }
      if (!ODD && __any(apart)) asked[4 + wave] = 1;
    }
    __syncthreads();
  }
  int again = 0;
  if (wave == 0) {
    if constexpr (!ODD) {
      const v4i keys = *(const v4i *)asked, values = *(const v4i *)(asked + 4);
      again = x.asks(keys[0] | keys[1] | keys[2] | keys[3],
                     values[0] | values[1] | values[2] | values[3], to - from);
      asked[8] = again;
    }
    if (!again) {
#pragma unroll
      for (int j = 0; j < NY; ++j) x.store(w, row(j), j, part);
    }
  }
  if constexpr (!ODD) {
    __syncthreads();
    again = __builtin_amdgcn_readfirstlane(asked[8]);
  }
  return again;
}

// (A function of its own: beside the first pass its registers cost that 10 %, on heads of 64.
// The scratch memory that the compiler reports is where it saves the kernel's registers.)
template <int D, int NY>
__device__ __attribute__((noinline)) void
attend_few_odd(const Work *w, __attribute__((address_space(3))) char *lds, int given) {
  attend_few<D, NY, true>(*alike(w), (char *)lds, given);
}

// (waves to a SIMD as the first pass has them by itself: the function would take more registers)
template <int D, int NY>
__global__ void __launch_bounds__(256, (D == 64 ? 3 : D == 128 ? 2 : 1) + (D <= 128 && NY == 1))
    k_attend_few(Work w) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int again = attend_few<D, NY, false>(w, lds, 0);
  if (again)
    attend_few_odd<D, NY>((const Work *)(const void *)__builtin_amdgcn_kernarg_segment_ptr(),
                          (__attribute__((address_space(3))) char *)lds, again);
}

// MACS matrix instructions with VALUS vector instructions spread between them.
template <int MACS, int VALUS>
__device__ inline void interleave() {
#pragma unroll
  for (int i = 0; i < MACS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, (VALUS + MACS - 1) / MACS, 0);
  }
}

// ---- many rows: tiles of the cache widened once, in LDS, for all of a workgroup's rows ----
//
// A tile is 64 positions.  Each of the four waves brings in sixteen of them and writes
// them to LDS as the fragments that the products take, so that every read there is 16
// bytes a lane, in lane order.  One tile is used while the next is written and the one
// after is on its way.
template <int D, int NY>
struct Many {
  static constexpr int KS = D / 32, NX = D / 16, NS = D / 64, VB = D / 16;
  static constexpr int TILE = 64;
  static constexpr int KEYS = 4 * KS * 1024, VALUES = 2 * NX * 1024;
  static constexpr int STAGE = KEYS + VALUES + 2 * TILE * 4 + 32;  // and scales, what is there, largest
  static constexpr int LDS = 2 * STAGE;  // (and 32 bytes for what the waves ask for)
  static constexpr int ROWS = 4 * 16 * NY;
};

// (ODD and what it returns as for attend_few)
template <int D, int NY, bool ODD>
__device__ __forceinline__ int attend_many(const Work &w, char *lds, int given) {
  using M = Many<D, NY>;
  const AttendArgs &a = w.a;
  const int lane = threadIdx.x % 64, m = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int kv_heads = (int)a.cache.kv_heads;
  // Heads in turn: with eight of them, or a divisor, an XCD has the same ones throughout, and
  // some of every sequence; the blocks with most to see first.  (Runs of blocks to an XCD
  // give it whole sequences, the long or the short ones: four of 512 to 2048 positions 134
  // us in turn, 210 so; one of 4096 with two heads of 256, 329 and 541.)
  unsigned rest = blockIdx.x;
  const int head = rest % kv_heads;
  rest /= kv_heads;
  const int block = w.row_blocks - 1 - rest % (unsigned)w.row_blocks;
  rest /= (unsigned)w.row_blocks;
  const int part = rest % (unsigned)w.parts, b = rest / (unsigned)w.parts;
  const Seq s = seq_of(a, b, head);
  const int r0 = block * M::ROWS;
  if (r0 >= s.n * w.group) return 0;
  const int rw = r0 + 16 * NY * wave;
  auto row = [&](int j) { return row_of(s, rw + 16 * j + m, w.group, head); };

  Rows16<D, NY> x;
  auto first = [&](int ks) { return 32 * ks + 8 * g; };
  if (a.dtype == ROSETTA_BF16) x.template load<bf16>(a, s.first, row, first);
  else x.template load<f16>(a, s.first, row, first);
  if (given & FAR_KEYS) x.nearer_keys();
  uint64_t far_keys = 0;  // lanes that met some

  // what some row of the workgroup sees, of this wave sees, and all of this wave's see
  const int n1 = s.n - 1;
  const int last = least((r0 + M::ROWS - 1) / w.group, n1);
  const int mine_last = least((rw + 16 * NY - 1) / w.group, n1);
  const int end = a.masks ? s.length : least(s.length, s.base + last + 1);
  int some = a.masks ? s.length : least(s.length, s.base + mine_last + 1);
  const int all = least(s.length, s.base + (a.masks ? 0 : rw / w.group + 1));
  if (rw >= s.n * w.group) some = 0;
  int from, to;
  part_of(end < 0 ? 0 : end, w.parts, part, M::TILE, from, to);

  using vb = std::conditional_t<M::VB == 4, int, std::conditional_t<M::VB == 8, v2i, v4i>>;
  struct Sub {
    v4i k[M::NS];
    vb v[4];
    float ks, vs;
    bool there;
    int room;  // positions that are there, from its first on
  } sub;
  const u32 dim = (u32)a.cache.dim, stride = (u32)a.cache.place_stride;
  u32 kat[M::NS];
#pragma unroll
  for (int c = 0; c < M::NS; ++c)
    kat[c] = m * stride + (64 * c + 16 * g < dim ? 64 * c + 16 * g : 0);
  const u32 vat = 4 * g * stride + (M::VB * m < dim ? M::VB * m : 0);
  // (the table's entry for the tile after the one to be loaded is asked for with it)
  int entry = from < to ? entry_at(s, a, from + 16 * wave) : -1;
  auto load = [&](int t) {
    const Sixteen at = sixteen_at(s, a, entry, t + 16 * wave);
    sub.there = is_page(a, entry);
    sub.room = sub.there ? s.length - (t + 16 * wave) : 0;
    entry = t + M::TILE < to ? entry_at(s, a, t + M::TILE + 16 * wave) : -1;
#pragma unroll
    for (int c = 0; c < M::NS; ++c) sub.k[c] = *(const v4i *)(at.k + kat[c]);
#pragma unroll
    for (int r = 0; r < 4; ++r) sub.v[r] = *(const vb *)(at.v + vat + r * stride);
    sub.ks = at.ks[m];
    sub.vs = at.vs[m];
  };
  // in PIECES: what a piece does runs beside products
  constexpr int PIECES = M::NX / 4;
  auto write_piece = [&](char *stage, int piece) {
#pragma unroll
    for (int c = piece * M::NS / PIECES; c < (piece + 1) * M::NS / PIECES; ++c) {
      char *to = stage + (((wave * M::KS + 2 * c + g / 2) * 64 + g % 2 * 32 + m) * 16);
      const v2i a0 = widen(sub.k[c].x), a1 = widen(sub.k[c].y);
      const v2i b0 = widen(sub.k[c].z), b1 = widen(sub.k[c].w);
      *(v4i *)to = v4i{a0.x, a0.y, a1.x, a1.y};
      *(v4i *)(to + 256) = v4i{b0.x, b0.y, b1.x, b1.y};
    }
    auto word = [&](int r, int i) {
      if constexpr (M::VB == 4) return (u32)sub.v[r];
      else return (u32)sub.v[r][i];
    };
    char *to = stage + M::KEYS + wave / 2 * M::NX * 1024 + lane * 16 + wave % 2 * 8;
    auto turn = [&](auto byte) {
      constexpr int I = decltype(byte)::value;
      *(v2i *)(to + (4 * piece + I) * 1024) =
          v2i{(int)widen_two<I>(word(0, piece), word(1, piece)),
              (int)widen_two<I>(word(2, piece), word(3, piece))};
    };
    turn(std::integral_constant<int, 0>{});
    turn(std::integral_constant<int, 1>{});
    turn(std::integral_constant<int, 2>{});
    turn(std::integral_constant<int, 3>{});
    if (piece) return;
    float *scales = (float *)(stage + M::KEYS + M::VALUES);
    settle(sub.ks, sub.vs, m < sub.room);
    if constexpr (ODD) {
      sub.ks *= given & FAR_KEYS ? NEARER : 1.f;
      sub.vs *= given & FAR_VALUES ? NEARER : 1.f;
    } else {
      far_keys |= __ballot(fabsf(sub.ks) >= FAR);
    }
    // the largest v_scale of the sixteen
    float most = fabsf(sub.vs);
    most = max2(most, turned<8>(most));
    most = max2(most, turned<4>(most));
    most = max2(most, turned<2>(most));
    most = max2(most, turned<1>(most));
    // (the lanes of a place write the same)
    scales[16 * wave + m] = sub.ks;
    scales[M::TILE + 16 * wave + m] = sub.vs;
    ((int *)(scales + 2 * M::TILE))[wave] = sub.there;
    scales[2 * M::TILE + 4 + wave] = most;
  };
  int *asked = (int *)(lds + M::LDS);  // what the waves ask for; whether values' scales are APART
  asked[4 + wave] = 0;
  auto write = [&](char *stage) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) write_piece(stage, i);
  };
  auto use = [&](const char *stage, int t, char *next) {
    const v4i *keys = (const v4i *)stage + lane;
    const v4i *values = (const v4i *)(stage + M::KEYS) + lane;
    const float *scales = (const float *)(stage + M::KEYS + M::VALUES);
    auto ks = [&](int h) { return *(const v4f *)(scales + 16 * h + 4 * g); };
    auto vs = [&](int h) { return *(const v4f *)(scales + M::TILE + 16 * h + 4 * g); };
    v4f sc[4][NY];
    float largest[NY];
#pragma unroll
    for (int j = 0; j < NY; ++j) largest[j] = NONE;
    // The next fragments are on their way while the present ones are multiplied (and no
    // more: all of them at once do not fit the registers), and what the scores go through
    // is spread between the products that follow, here and below: a wave's vector and
    // matrix instructions then run side by side.  The wave at its products goes first
    // where two want to issue (16384 rows of 128 over 4096 positions: 204 us -> 198).
    v4i kf[2][M::KS];
    if constexpr (D < 256) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int c = 0; c < M::KS; ++c) kf[0][c] = keys[c * 64];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
#pragma unroll
      for (int j = 0; j < NY; ++j) sc[h][j] = v4f{0, 0, 0, 0};
      if (h < 3) {
#pragma unroll
        for (int c = 0; c < M::KS; ++c) kf[(h + 1) % 2][c] = keys[((h + 1) * M::KS + c) * 64];
      }
#pragma unroll
      for (int c = 0; c < M::KS; ++c)
#pragma unroll
        for (int j = 0; j < NY; ++j) sc[h][j] = mac(kf[h % 2][c], x.q[j][c], sc[h][j]);
      if (h > 0) {
        x.template scaled<4>(sc, h - 1, ks(h - 1), largest);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (D < 256) __builtin_amdgcn_s_setprio(0);
    x.template scaled<4>(sc, 3, ks(3), largest);
    const int *there = (const int *)(scales + 2 * M::TILE);
    const int here = __builtin_amdgcn_readfirstlane(there[0] & there[1] & there[2] & there[3]);
    const bool masked = !(t + M::TILE <= all && here);
    auto bits = [&](int j) {
      uint64_t in = 0;
#pragma unroll
      for (int h = 0; h < 4; ++h) in |= (uint64_t)(there[h] ? 0xffff : 0) << (16 * h);
      const Row r = row(j);
      const uint64_t *mask = a.masks && r.at >= 0 ? a.masks + r.at * a.words : nullptr;
      return (seen_from(s, a, mask, r.i, t) & in) >> (4 * g);
    };
    if constexpr (ODD) {
      x.template refer_odd<4>(sc, vs, masked, bits);
    } else {
      x.template refer<4>(
          sc, largest, vs,
          [&] {
            const v4f most = *(const v4f *)(scales + 2 * M::TILE + 4);
            return max3(max2(most[0], most[1]), most[2], most[3]);
          },
          masked, bits, asked + 4 + wave);
    }
    v4i p[2][NY];
    constexpr int G = 4, EACH = M::NX / G;  // groups of products with the values, per half
    v4i vf[2][G];
#pragma unroll
    for (int i = 0; i < G; ++i) vf[0][i] = values[i * 64];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < NY; ++j) x.weigh(sc[h][j], vs(h), j, h, p[0][j]);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (D < 256) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int n = 0; n < 2 * EACH; ++n) {
      if (n + 1 < 2 * EACH) {
#pragma unroll
        for (int i = 0; i < G; ++i) vf[(n + 1) % 2][i] = values[((n + 1) * G + i) * 64];
      }
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const int at = (n * G + i) % M::NX, u = n * G / M::NX;
#pragma unroll
        for (int j = 0; j < NY; ++j) x.o[at][j] = mac(vf[n % 2][i], p[u][j], x.o[at][j]);
      }
      // beside the first half's products the second half's weights, a share to a group
      // (beside the second half's, the next tile)
      if (n < EACH) {
#pragma unroll
        for (int k = n * 2 * NY / EACH; k < (n + 1) * 2 * NY / EACH; ++k)
          x.weigh(sc[2 + k / NY][k % NY], vs(2 + k / NY), k % NY, k / NY, p[1][k % NY]);
        interleave<G * NY, 2 * NY / EACH * 18>();
      } else {  // (behind the last tile what was there before, which nobody reads)
        write_piece(next, n - EACH);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (D < 256) __builtin_amdgcn_s_setprio(0);
  };
  if (from < to) {
    load(from);
    write(lds);
    if (from + M::TILE < to) load(from + M::TILE);
  }
  int at = 0;
  int t = from;
  for (; t < least(some, to); t += M::TILE, at ^= 1) {
    __syncthreads();  // this tile is written, and the one before it no longer read
    use(lds + at * M::STAGE, t, lds + (at ^ 1) * M::STAGE);
    if (t + 2 * M::TILE < to) load(t + 2 * M::TILE);
  }
  for (; t < to; t += M::TILE, at ^= 1) {  // (what only other waves see)
    __syncthreads();
    if (t + M::TILE < to) write(lds + (at ^ 1) * M::STAGE);
    if (t + 2 * M::TILE < to) load(t + 2 * M::TILE);
  }
  if constexpr (ODD) {
    if (given & FAR_VALUES) x.nearer_values();
  } else {
    // (what one wave asks for, all do: they write each other's tiles)
    asked[wave] = x.asks(far_keys, asked[4 + wave], to - from);
    __syncthreads();
    const v4i all = *(const v4i *)asked;
    const int again = __builtin_amdgcn_readfirstlane(all[0] | all[1] | all[2] | all[3]);
    if (again) return again;
  }
#pragma unroll
  for (int j = 0; j < NY; ++j) x.store(w, row(j), j, part);
  return 0;
}

template <int D, int NY>
__device__ __attribute__((noinline)) void
attend_many_odd(const Work *w, __attribute__((address_space(3))) char *lds, int given) {
  attend_many<D, NY, true>(*alike(w), (char *)lds, given);
}

template <int D, int NY>
__global__ void __launch_bounds__(256, D == 256 ? 1 : D == 128 ? 2 : 3) k_attend_many(Work w) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int again = attend_many<D, NY, false>(w, lds, 0);
  if (again)
    attend_many_odd<D, NY>((const Work *)(const void *)__builtin_amdgcn_kernarg_segment_ptr(),
                           (__attribute__((address_space(3))) char *)lds, again);
}

// ---- parts of a sequence joined ----
//
// D / 4 threads of four outputs to a row, and `w.joiners` such groups, a power of two, to
// its parts: bound by latency, so that a thread's parts are read ahead of each other.
// 128 parts of 32 rows: 86 us with one group.
template <int D>
__global__ void __launch_bounds__(256) k_attend_join(Work w) {
  const AttendArgs &a = w.a;
  constexpr int LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ v4f sums[GROUPS][LANES];
  __shared__ float2 ends[GROUPS];
  const Seq s = seq_of(a, blockIdx.y, 0);
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int sub = group % w.joiners;
  const int64_t r = (int64_t)blockIdx.x * (GROUPS / w.joiners) + group / w.joiners;
  const bool mine = r < s.n * (int64_t)a.heads;
  const size_t row = s.first * a.heads + r;
  const float2 *from = w.ends + row * w.parts;
  const v4f *parts = (const v4f *)(w.sums + row * w.parts * D) + lane;
  // the parts sub, sub + joiners, ...
  constexpr int AHEAD = 4;
  float ref = NONE, total = 0.f;
  v4f o = {0, 0, 0, 0};
  for (int p0 = sub; mine && p0 < w.parts; p0 += AHEAD * w.joiners) {
    float2 e[AHEAD];
    v4f v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int p = least(p0 + i * w.joiners, w.parts - 1);
      e[i] = from[p];
      v[i] = parts[(size_t)p * LANES];
    }
    const float before = ref;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (p0 + i * w.joiners >= w.parts) e[i].x = NONE;
      ref = fmaxf(ref, e[i].x);
    }
    if (ref == NONE) continue;
    bring(total, o, before - ref);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (e[i].x == NONE) continue;  // (its outputs were not written)
      bring(e[i].y, v[i], e[i].x - ref);
      total += e[i].y;
      o += v[i];
    }
  }
  sums[group][lane] = o;
  if (lane == 0) ends[group] = float2{ref, total};
  __syncthreads();
  if (sub || !mine) return;
  float all = NONE;
  for (int i = 0; i < w.joiners; ++i) all = fmaxf(all, ends[group + i].x);
  const bool none = all == NONE;
  total = 0.f;
  o = v4f{0, 0, 0, 0};
  for (int i = 0; i < w.joiners && !none; ++i) {
    float sum = ends[group + i].y;
    v4f part = sums[group + i][lane];
    bring(sum, part, ends[group + i].x - all);
    total += sum;
    o += part;
  }
  const float inv = none ? 0.f : 1.f / total;
  if (a.lse && lane == 0)
    a.lse[row] = none ? NONE : (all + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
  if (lane * 4 >= (int)a.cache.dim) return;
  Row at;
  at.at = s.first + (int)(r / (int64_t)a.heads);
  at.head = (int)(r % (int64_t)a.heads);
  const float f[8] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  Rows16<D, 1>::put8(a, at, lane * 4, f, 4);
}

}  // namespace

namespace {

struct Plan {
  int d, ny, parts, row_blocks;
  bool many;
};

Plan plan_of(size_t heads, size_t kv_heads, size_t dim, size_t batch, size_t max_rows,
             size_t positions) {
  Plan p;
  p.d = dim <= 64 ? 64 : dim <= 128 ? 128 : 256;
  const size_t group = heads / kv_heads, rows = max_rows * group;
  // Tiles widened once for all rows against ones that each wave widens for itself, without
  // a barrier and in smaller pieces (microseconds, the first against the second):
  // rows of 256 58 : 93 (512 rows over 4096 positions, four sequences); of 128 17 : 26
  // (four of 1024 over 256), 213 : 323 (16384 over 4096), 31 : 26 (four of 64 over 4096);
  // of 64 141 : 202 (32768 over 4096), 42 : 43 (two of 8192 over 1024, 512 workgroups of
  // the first), 110 : 93 (12 heads of 4096 over 4096, 384 of them).
  const size_t large = batch * kv_heads * ((rows + 127) / 128);
  p.many = p.d == 256 ? rows > 32 : rows > 128 && (p.d == 128 || large >= 512);
  // (two groups of 256 do not fit the registers beside what is on its way)
  p.ny = p.d == 256 || rows <= 16 ? 1 : 2;
  const size_t each = 16 * p.ny * (p.many ? 4 : 1);
  p.row_blocks = (int)((rows + each - 1) / each);
  // Parts until the CUs have the workgroups that they hold of the tiles' kernel, long ones,
  // or two of the other: sums that are joined cost their way to memory and back (four
  // sequences of 1024 rows over 256 positions: 34 us in two parts, 17 in one; 1024 rows
  // over 4096: 48 us in eight, 54 in four).  One group of rows is cut in two at least, so
  // that long sequences end sooner (64 of 2048 to 8192 positions: 147 us in one, 133 in two).
  const size_t blocks = batch * kv_heads * p.row_blocks;
  const size_t wanted = p.d == 256 ? 256 : 512;
  const size_t least_part = !p.many ? 128 : p.d == 256 ? 256 : 512;
  size_t parts = (wanted + blocks - 1) / blocks;
  if (!p.many && p.row_blocks == 1 && blocks < 1024) parts = std::max<size_t>(parts, 2);
  parts = std::min(parts, (positions + least_part - 1) / least_part);
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
  const Plan p = plan_of(heads, kv_heads, dim, batch, std::min(max_rows, rows), positions);
  return p.parts > 1 ? rows * heads * p.parts * (p.d * sizeof(float) + sizeof(float2)) : 0;
}

hipError_t launch_kv_attention(const AttendArgs &given, hipStream_t st) {
  AttendArgs a = given;
  a.max_rows = std::min(a.max_rows, a.packed.rows);
  const size_t positions = a.packed.table_len << a.cache.page_log;
  const Plan p = plan_of(a.heads, a.cache.kv_heads, a.cache.dim, a.packed.batch, a.max_rows, positions);
  Work w{a, (int)(a.heads / a.cache.kv_heads), p.parts, p.row_blocks, 1, nullptr, nullptr};
  if (p.parts > 1) {
    w.sums = (float *)a.workspace;
    w.ends = (float2 *)(w.sums + a.packed.rows * a.heads * p.parts * p.d);
  }
  const size_t blocks = a.packed.batch * a.cache.kv_heads * p.parts * p.row_blocks;
  // (a few parts to a group of threads)
  const int groups = 1024 / p.d;
  while (w.joiners < groups && w.joiners * 4 < p.parts) w.joiners *= 2;
  const size_t each = groups / w.joiners, joins = (a.max_rows * a.heads + each - 1) / each;
  if (!grid_fits(blocks, 256) || (p.parts > 1 && (a.packed.batch > 65535 || !grid_fits(joins * a.packed.batch, 256))))
    return hipErrorInvalidConfiguration;
  return by_dim(p.d, [&](auto d) {
    constexpr int D = decltype(d)::value;
    hipError_t e = hipSuccess;
    auto few = [&](auto ny) {
      constexpr int NY = decltype(ny)::value;
      constexpr size_t LDS = 2 * 64 * (4 * (D / 16) * NY + 4 * NY) * sizeof(float) + 48;
      e = allow_lds(k_attend_few<D, NY>, LDS);
      if (e != hipSuccess) return;
      hipLaunchKernelGGL((k_attend_few<D, NY>), dim3((unsigned)blocks), dim3(256), LDS, st, w);
      e = hipGetLastError();
    };
    if (p.many) {
      constexpr int NY = D == 256 ? 1 : 2;
      using M = Many<D, NY>;
      e = allow_lds(k_attend_many<D, NY>, M::LDS + 32);
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL((k_attend_many<D, NY>), dim3((unsigned)blocks), dim3(256), M::LDS + 32, st, w);
      e = hipGetLastError();
    } else if (p.ny == 1) few(std::integral_constant<int, 1>{});
    else if constexpr (D < 256) few(std::integral_constant<int, 2>{});
    if (e != hipSuccess || p.parts == 1) return e;
    hipLaunchKernelGGL(k_attend_join<D>, dim3((unsigned)joins, (unsigned)a.packed.batch), dim3(256), 0,
                       st, w);
    return hipGetLastError();
  });
}

}  // namespace rosetta
