// The 8-bit cache of keys and values: rows written to it with a scale per head, read
// back, and, of a tree of drafted tokens, the accepted ones moved together; and the
// bit masks that say which drafted tokens a drafted token follows.
//
// All of it is bound by memory (long prompts) or by the latency of a few dependent
// loads (single tokens): starts -> sequence -> table -> place.
#include <type_traits>

#include "decode.hpp"

namespace rosetta {

namespace {

constexpr int SEARCH = 1024;  // starts held in LDS

// The sequence of a row: the last b with starts[b] <= row.  (A search in LDS where
// the starts fit: six dependent loads from memory would be 3 us.)
struct Search {
  const int *starts;
  int batch;
  bool held;
  const int *lds;
  // (all threads of the workgroup)
  __device__ Search(const int *starts, size_t batch, int *lds)
      : starts(starts), batch((int)batch), held(batch < SEARCH), lds(lds) {
    if (held) {
      for (int i = threadIdx.x; i <= this->batch; i += blockDim.x) lds[i] = starts[i];
      __syncthreads();
    }
  }
  __device__ int at(int i) const { return held ? lds[i] : starts[i]; }
  __device__ int of(int row) const {
    int lo = 0, hi = batch;  // starts[lo] <= row < starts[hi], where there is such
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (at(mid) <= row) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

// Page and place of a row's position, page -1 where it has none, -2 where the row is of
// no sequence.
struct Place {
  int64_t page;
  int at;
};

// Those of a workgroup's rows, [lo, hi] of the call's: looked up once where they are of one
// sequence.
struct Places {
  const Cache &c;
  const Packed &r;
  Search search;
  int b0, b1;
  Span one;
  __device__ Places(const Cache &c, const Packed &r, size_t lo, size_t hi, int *lds)
      : c(c), r(r), search(r.starts, r.batch, lds) {
    b0 = __builtin_amdgcn_readfirstlane(search.of((int)lo));
    b1 = __builtin_amdgcn_readfirstlane(search.of((int)(hi < r.rows ? hi : r.rows - 1)));
    one = span_of(r.starts, r.lens, b0, r.rows);
  }
  __device__ Place of(size_t row) const {
    if (row >= r.rows) return {-2, 0};
    if (b0 == b1) return at(b0, one, (int)row);
    const int b = search.of((int)row);
    return at(b, span_of(r.starts, r.lens, b, r.rows), (int)row);
  }
  __device__ Place at(int b, const Span &sp, int row) const {
    if (row < sp.first || row >= sp.first + sp.n) return {-2, 0};
    const int64_t t = sp.base + (row - sp.first);
    return {page_of(r.table + b * r.table_stride, r.table_len, c.page_log, c.pages, t),
            (int)t & ((1 << c.page_log) - 1)};
  }
};

template <class T>
__device__ inline void load8(const T *p, float (&f)[8]) {
  struct __attribute__((packed, aligned(1))) {
    T v[8];
  } v;
  __builtin_memcpy(&v, p, sizeof v);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)v.v[i];
}

template <class T>
__device__ inline void store8(T *p, const float (&f)[8]) {
  struct __attribute__((packed, aligned(1))) {
    T v[8];
  } v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v.v[i] = (T)f[i];
  __builtin_memcpy(p, &v, sizeof v);
}

// A workgroup takes UNITS times 256 / LANES consecutive rows of one head's keys or values,
// LANES threads of eight elements to a row: what it writes to a page, scales among it,
// lies together.
template <int LANES>
struct Item {
  static constexpr int ROWS = 256 / LANES;
  size_t first, row;  // of the workgroup, and this thread's in the first unit
  int head, lane;
  bool values, mine;
  template <int UNITS>
  __device__ Item(const Cache &c, std::integral_constant<int, UNITS>) {
    // (heads first: neighbours read the same rows)
    const unsigned all = 2 * (unsigned)c.kv_heads, which = blockIdx.x % all;
    first = (size_t)(blockIdx.x / all) * (UNITS * ROWS);
    row = first + threadIdx.x / LANES;
    lane = threadIdx.x % LANES;
    head = which % (unsigned)c.kv_heads;
    values = which >= (unsigned)c.kv_heads;
    mine = (size_t)lane * 8 < c.dim;
  }
};

// scale = max / 127, q = x / scale to nearest, ties to even, both divisions rounded as
// 32-bit floats are: half the maximum is such a tie, and a product with 1 / scale would
// put it on either side.  The quotient comes from the reciprocal and one correction by
// the remainder (three operations for the eleven of a division).
//
// 32768 rows of 8 heads of 128 in bf16, keys and values: 57 us (3.5 TB/s) with four units, each
// asked for before the first is used, and their places looked up together (78 with one).
template <class T, int LANES, int UNITS>
__global__ void __launch_bounds__(256) k_kv_write(HeadRows k, HeadRows v, Cache c, Packed r) {
  __shared__ int lds[SEARCH];
  const Item<LANES> it(c, std::integral_constant<int, UNITS>{});
  constexpr int ROWS = Item<LANES>::ROWS;
  const HeadRows &from = it.values ? v : k;
  float x[UNITS][8] = {};
#pragma unroll
  for (int n = 0; n < UNITS; ++n) {
    const size_t row = it.row + n * ROWS;
    if (it.mine && row < r.rows)
      load8((const T *)from.p + row * from.row + it.head * from.head + it.lane * 8, x[n]);
  }
  const Places places(c, r, it.first, it.first + UNITS * ROWS - 1, lds);
#pragma unroll
  for (int n = 0; n < UNITS; ++n) {
    const Place at = places.of(it.row + n * ROWS);
    float top = 0.f;  // (NaN or infinite with any that is)
#pragma unroll
    for (int i = 0; i < 8; ++i) top = __builtin_elementwise_maximum(top, fabsf(x[n][i]));
#pragma unroll
    for (int m = LANES / 2; m >= 1; m >>= 1)
      top = __builtin_elementwise_maximum(top, __shfl_xor(top, m));
    const float scale = top / 127.f;
    const float inv = 1.f / scale;
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s[i] = x[n][i] * inv;
      s[i] = fmaf(fmaf(-s[i], scale, x[n][i]), inv, s[i]);
    }
    if (__any(!(top >= 0x1p-60f))) {  // (remainders would lose bits, or no number)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        s[i] = top >= 0x1p-60f ? s[i] : scale > 0.f ? x[n][i] / scale : 0.f;
    }
    if (at.page < 0) continue;
    struct __attribute__((aligned(8))) {
      int8_t v[8];
    } q;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      q.v[i] = (int8_t)(int)fminf(fmaxf(rintf(s[i]), -127.f), 127.f);
    int8_t *to = (it.values ? c.v : c.k) + at.page * c.page_stride + it.head * c.head_stride +
                 at.at * c.place_stride;
    if (it.mine) __builtin_memcpy(__builtin_assume_aligned(to + it.lane * 8, 8), &q, 8);
    if (it.lane == 0)
      (it.values ? c.v_scale : c.k_scale)[at.page * c.scale_page_stride +
                                          it.head * c.scale_head_stride + at.at] = scale;
  }
}

template <class T, int LANES, int UNITS>
__global__ void __launch_bounds__(256) k_kv_read(HeadRows k, HeadRows v, Cache c, Packed r) {
  __shared__ int lds[SEARCH];
  const Item<LANES> it(c, std::integral_constant<int, UNITS>{});
  constexpr int ROWS = Item<LANES>::ROWS;
  const Places places(c, r, it.first, it.first + UNITS * ROWS - 1, lds);
  if (!it.mine) return;
  Place at[UNITS];
  uint64_t q[UNITS];
  float scale[UNITS];
#pragma unroll
  for (int n = 0; n < UNITS; ++n) at[n] = places.of(it.row + n * ROWS);
#pragma unroll
  for (int n = 0; n < UNITS; ++n) {
    // (where there is none, the first page's is read and not used)
    const size_t pg = at[n].page < 0 ? 0 : at[n].page;
    q[n] = *(const uint64_t *)((it.values ? c.v : c.k) + pg * c.page_stride +
                               it.head * c.head_stride + at[n].at * c.place_stride + it.lane * 8);
    scale[n] = (it.values ? c.v_scale : c.k_scale)[pg * c.scale_page_stride +
                                                   it.head * c.scale_head_stride + at[n].at];
  }
  const HeadRows &to = it.values ? v : k;
#pragma unroll
  for (int n = 0; n < UNITS; ++n) {
    if (at[n].page == -2) continue;  // a row of no sequence
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      f[i] = at[n].page < 0 ? 0.f : (float)(int8_t)(q[n] >> (8 * i)) * scale[n];
    store8((T *)to.p + (it.row + n * ROWS) * to.row + it.head * to.head + it.lane * 8, f);
  }
}

// One workgroup moves the rows of one sequence and head, keys or values, as many at a
// time as it has threads for: all are read before any is written, and since path[i] >=
// i what is written lies before all that is still to be read.
template <int LANES>
__global__ void __launch_bounds__(256) k_kv_keep(Cache c, Packed r, const int *path,
                                                 const int *count, int *lens_out) {
  const size_t b = blockIdx.x;
  const int head = blockIdx.y % c.kv_heads;
  const bool values = blockIdx.y >= c.kv_heads;
  const Span sp = span_of(r.starts, r.lens, b, r.rows);
  const int kept = min(max(count[b], 0), sp.n);
  if (blockIdx.y == 0 && threadIdx.x == 0) lens_out[b] = (int)(sp.base + kept);
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  int8_t *base = (values ? c.v : c.k) + head * c.head_stride;
  float *scales = (values ? c.v_scale : c.k_scale) + head * c.scale_head_stride;
  const int *table = r.table + b * r.table_stride;
  const int mask = (1 << c.page_log) - 1;
  for (int i0 = 0; i0 < kept; i0 += 256 / LANES) {
    const int i = i0 + group;
    const int from = i < kept ? path[sp.first + i] : -1;
    const int64_t ts = sp.base + from, td = sp.base + i;
    const bool moves = from > i && from < sp.n;
    const int64_t ps = moves ? page_of(table, r.table_len, c.page_log, c.pages, ts) : -1;
    const int64_t pd = moves ? page_of(table, r.table_len, c.page_log, c.pages, td) : -1;
    const bool both = ps >= 0 && pd >= 0;
    uint64_t q = 0;
    float s = 0.f;
    const bool mine = (size_t)lane * 8 < c.dim;
    if (both) {
      if (mine)
        q = *(const uint64_t *)(base + ps * c.page_stride + (ts & mask) * c.place_stride + lane * 8);
      s = scales[ps * c.scale_page_stride + (ts & mask)];
    }
    __syncthreads();
    if (both) {
      if (mine)
        *(uint64_t *)(base + pd * c.page_stride + (td & mask) * c.place_stride + lane * 8) = q;
      if (lane == 0) scales[pd * c.scale_page_stride + (td & mask)] = s;
    }
    __syncthreads();
  }
}

// One thread a node: up through the parents, which lie before their children, so that
// its words are done one after the other, the last first.
__global__ void __launch_bounds__(256) k_tree_masks(const int *parents, const int *starts,
                                                    size_t batch, size_t rows, int words,
                                                    uint64_t *masks) {
  __shared__ int lds[SEARCH];
  const Search search(starts, batch, lds);
  const size_t row = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (row >= rows) return;
  const Span sp = span_of(starts, nullptr, search.of((int)row), rows);
  const int place = (int)row - sp.first;
  int i = place < sp.n ? place : -1;  // (no sequence's: below 0 already, or behind its rows)
  for (int word = words - 1; word >= 0; --word) {
    uint64_t m = 0;
    while (i >= 64 * word) {
      if (i < 64 * word + 64) m |= (uint64_t)1 << (i - 64 * word);
      const int up = parents[sp.first + i];
      i = up < i ? up : -1;
    }
    masks[row * words + word] = m;
  }
}

template <class F>
hipError_t by_lanes(size_t dim, F f) {
  if (dim <= 16) return f(std::integral_constant<int, 2>{});
  if (dim <= 64) return f(std::integral_constant<int, 8>{});
  if (dim <= 128) return f(std::integral_constant<int, 16>{});
  return f(std::integral_constant<int, 32>{});
}

template <class F>
hipError_t by_type(int dtype, F f) {
  if (dtype == ROSETTA_F32) return f(0.f);
  if (dtype == ROSETTA_BF16) return f((bf16)0.f);
  return f((f16)0.f);
}

hipError_t grid_of(size_t x, size_t y, dim3 &grid) {
  if (!grid_fits(x * y, 256) || y > 65535) return hipErrorInvalidConfiguration;
  grid = dim3((unsigned)x, (unsigned)y);
  return hipSuccess;
}

}  // namespace

// Four units to a workgroup where that leaves it enough of them.
template <class F>
hipError_t by_units(size_t rows, size_t rows_each, size_t heads, F f) {
  if ((rows + rows_each - 1) / rows_each * heads >= 4096) return f(std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, 1>{});
}

hipError_t launch_kv_write(const HeadRows &k, const HeadRows &v, int dtype, const Cache &c,
                           const Packed &r, hipStream_t st) {
  return by_type(dtype, [&](auto type) {
    return by_lanes(c.dim, [&](auto lanes) {
      constexpr int LANES = decltype(lanes)::value, ROWS = 256 / LANES;
      return by_units(r.rows, ROWS, 2 * c.kv_heads, [&](auto units) {
        constexpr int UNITS = decltype(units)::value;
        dim3 grid;
        const hipError_t e = grid_of((r.rows + UNITS * ROWS - 1) / (UNITS * ROWS) * 2 * c.kv_heads, 1, grid);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((k_kv_write<decltype(type), LANES, UNITS>), grid, dim3(256), 0, st, k, v,
                           c, r);
        return hipGetLastError();
      });
    });
  });
}

hipError_t launch_kv_read(const Cache &c, const Packed &r, int dtype, const HeadRows &k,
                          const HeadRows &v, hipStream_t st) {
  return by_type(dtype, [&](auto type) {
    return by_lanes(c.dim, [&](auto lanes) {
      constexpr int LANES = decltype(lanes)::value, ROWS = 256 / LANES;
      return by_units(r.rows, ROWS, 2 * c.kv_heads, [&](auto units) {
        constexpr int UNITS = decltype(units)::value;
        dim3 grid;
        const hipError_t e = grid_of((r.rows + UNITS * ROWS - 1) / (UNITS * ROWS) * 2 * c.kv_heads, 1, grid);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((k_kv_read<decltype(type), LANES, UNITS>), grid, dim3(256), 0, st, k, v, c,
                           r);
        return hipGetLastError();
      });
    });
  });
}

hipError_t launch_kv_keep(const Cache &c, const Packed &r, const int *path, const int *count,
                          int *lens_out, hipStream_t st) {
  return by_lanes(c.dim, [&](auto lanes) {
    dim3 grid;
    const hipError_t e = grid_of(r.batch, 2 * c.kv_heads, grid);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_kv_keep<lanes.value>, grid, dim3(256), 0, st, c, r, path, count, lens_out);
    return hipGetLastError();
  });
}

hipError_t launch_tree_masks(const int *parents, const int *starts, size_t batch, size_t rows,
                             size_t words, uint64_t *masks, hipStream_t st) {
  dim3 grid;
  const hipError_t e = grid_of((rows + 255) / 256, 1, grid);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_tree_masks, grid, dim3(256), 0, st, parents, starts, batch, rows,
                     (int)words, masks);
  return hipGetLastError();
}

}  // namespace rosetta
