// Drafted tokens verified against the target's probabilities, from given random
// numbers: which of a tree's (or a chain's) tokens are accepted, and the token that
// follows them.
//
// The walk starts at node 0.  At a node, with p the target's distribution there and q
// the drafter's, from which the node's children were drawn, the children are tried in
// turn; what is left of p after k of them were rejected is, up to a factor,
//   r_k = (p - c_k q)+,  z_k its sum,  c_0 = 0, z_0 = 1,  c_(k+1) = c_k + z_k:
// taking q off r_k / z_k is taking z_k q off r_k.  A child with token x and random
// number u is accepted where u q(x) <= r_k(x) / z_k, strictly: u z_k q(x) < p(x) - c_k
// q(x).  Where no child is, the last token is drawn from r_k.  So a rejection costs one
// pass over two rows, and nothing but c is kept of it.  r_0 is p itself: the drafter has
// no distribution at a leaf, so that q is not read where c is 0.
//
// All in 64 bits: a draw lies next to one of the vocabulary's borders, and in 32 bits
// one draw in a hundred or so would depend on the order of the sum.
//
// Bound by latency: the passes depend on each other, and each is a launch (its sum is
// needed whole before the walk goes on).  A few launches of many workgroups, which
// walk again from the sums so far, then one workgroup a sequence for what is left.
#include <algorithm>

#include "decode.hpp"

namespace rosetta {

namespace {

constexpr int PIECES = 64;   // of a row, at most: a lane each
constexpr int PIECE = 2048;  // values of a piece, at least
constexpr int NODES = 1024;  // of a sequence that take part
constexpr int TEAM = 1024;   // threads of the last kernel
constexpr int ROUNDS = 3;    // launches of many workgroups before it, at most

struct Job {
  VerifyArgs a;
  int pieces, rounds;
  size_t piece;   // values of a piece
  double *sums;   // [rounds][batch][pieces]
};

// Sum over a wave, the same bits in every lane, in an order that its size decides.
__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m);
  return x;
}

// (p - c q)+, and p+ without q.  (NaN: nothing)
__device__ inline double above_0(double r) { return r > 0 ? r : 0; }
template <class T>
__device__ inline double left_at(const T *p, const T *q, double c, size_t v) {
  double r = (double)(float)p[v];
  if (c != 0) r -= c * (double)(float)q[v];
  return above_0(r);
}

// A wave's walk through one sequence's tree.  Lanes hold 64 nodes at a time.
template <class T>
struct Walk {
  const VerifyArgs &a;
  Span sp;
  int n, at, node = 0, count = 1, held = -1;
  double c = 0, z = 1;
  bool rejected = false;
  int parent;
  int64_t token;
  double p, q, u;

  __device__ Walk(const VerifyArgs &a, int b)
      : a(a), sp(span_of(a.starts, nullptr, b, a.rows)), n(sp.n < NODES ? sp.n : NODES), at(1) {}

  __device__ void hold(int block) {
    held = block;
    const int i = block * 64 + threadIdx.x % 64;
    parent = -1;
    token = -1;
    p = q = u = 0;
    if (i >= n) return;
    const int up = a.parents ? a.parents[sp.first + i] : i - 1;
    token = a.drafts[sp.first + i];
    if (up < 0 || up >= i || token < 0 || (size_t)token >= a.vocab) return;
    parent = up;
    p = (double)(float)((const T *)a.p)[(size_t)(sp.first + up) * a.p_stride + token];
    q = (double)(float)((const T *)a.q)[(size_t)(sp.first + up) * a.q_stride + token];
    u = a.u[sp.first + i];
  }

  // Goes on until a child is rejected (true: (node, c) is what the sum z is wanted of)
  // or the walk ends (false).
  template <class Accept>
  __device__ bool go(Accept accept) {
    while (at < n) {
      if (at / 64 != held) hold(at / 64);
      const int lane = threadIdx.x % 64;
      uint64_t children = __ballot(parent == node && held * 64 + lane >= at);
      if (!children) {
        at = (held + 1) * 64;
        continue;
      }
      const int i = __builtin_ctzll(children);
      at = held * 64 + i + 1;
      const double px = __shfl(p, i), qx = __shfl(q, i), ux = __shfl(u, i);
      if (ux * z * qx < px - c * qx) {
        node = at - 1;
        accept(count++, node, __shfl(token, i));
        c = 0;
        z = 1;
        rejected = false;
      } else {
        c += z;
        rejected = true;
        return true;
      }
    }
    return false;
  }
};

// This thread's share, of `threads`, of the sum over values [lo, hi) of a row, N groups of
// four of either row asked for at a time.  Q: whether q is taken off.
template <int N, bool Q, class T>
__device__ double share_of(const T *p, const T *q, double c, size_t lo, size_t hi, int thread,
                           int threads) {
  struct __attribute__((packed, aligned(1))) Four {
    T v[4];
  };
  double s[2] = {0, 0};
  const int fours = (int)((hi - lo) / 4);
  for (int i0 = thread; i0 < fours; i0 += N * threads) {
    Four x[N], y[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = i0 + n * threads < fours ? i0 + n * threads : i0;
      __builtin_memcpy(&x[n], p + lo + 4 * (size_t)i, sizeof x[n]);
      if constexpr (Q) __builtin_memcpy(&y[n], q + lo + 4 * (size_t)i, sizeof y[n]);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (i0 + n * threads >= fours) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        double r = (double)(float)x[n].v[i];
        if constexpr (Q) r -= c * (double)(float)y[n].v[i];
        s[n % 2] += above_0(r);
      }
    }
  }
  for (size_t v = lo + 4 * (size_t)fours + thread; v < hi; v += threads)
    s[0] += left_at(p, q, Q ? c : 0., v);
  return s[0] + s[1];
}
// (c is the same in all of them)
template <int N, class T>
__device__ double share(const T *p, const T *q, double c, size_t lo, size_t hi, int thread,
                        int threads) {
  return c != 0 ? share_of<N, true>(p, q, c, lo, hi, thread, threads)
                : share_of<N, false>(p, q, c, lo, hi, thread, threads);
}

// One round: every workgroup walks as far as the sums so far go and makes its piece of
// the next one.
template <class T>
__global__ void __launch_bounds__(256) k_verify_round(Job j, int round) {
  __shared__ double shared[4];
  __shared__ int node;
  __shared__ double at;
  const VerifyArgs &a = j.a;
  const int b = blockIdx.y, piece = blockIdx.x, lane = threadIdx.x % 64;
  if (threadIdx.x < 64) {
    double sums[ROUNDS];  // of the rounds before (what a walk does not ask for is not read)
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
      sums[i] = i < round && lane < j.pieces ? j.sums[((size_t)i * a.batch + b) * j.pieces + lane] : 0.;
    Walk<T> w(a, b);
    bool more = w.n > 0 && w.go([](int, int, int64_t) {});
    int k = 0;
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      if (!more || i >= round) continue;
      k = i + 1;
      w.z = wave_sum(sums[i]);
      more = w.go([](int, int, int64_t) {});
    }
    if (lane == 0) {
      // a walk that has ended wants the whole of p, unless a rejection left something
      const bool ended = !more && w.rejected && w.z > 0;
      node = w.n <= 0 || k < round || ended ? -1 : w.sp.first + w.node;
      at = more ? w.c : 0.;
    }
  }
  __syncthreads();
  if (node < 0) return;
  const size_t lo = piece * j.piece, hi = lo + j.piece < a.vocab ? lo + j.piece : a.vocab;
  double s = share<2>((const T *)a.p + (size_t)node * a.p_stride,
                   (const T *)a.q + (size_t)node * a.q_stride, at, lo, hi, threadIdx.x, 256);
  s = wave_sum(s);
  if (lane == 0) shared[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    j.sums[((size_t)round * a.batch + b) * j.pieces + piece] =
        shared[0] + shared[1] + (shared[2] + shared[3]);
}

// The rest of the walk, and the draw.
template <class T>
__global__ void __launch_bounds__(TEAM) k_verify_end(Job j) {
  constexpr int WAVES = TEAM / 64;
  __shared__ double pieces[PIECES], before[TEAM / 64];
  __shared__ double at, aim, base;
  __shared__ int node, state, chosen, found, last;  // state: 0 sums wanted, 1 draw
  const VerifyArgs &a = j.a;
  const int b = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  Walk<T> w(a, b);
  const int first = w.sp.first;
  auto none = [&](int64_t lo, int64_t hi) {
    for (int64_t i = lo + threadIdx.x; i < hi; i += TEAM) a.path[i] = -1, a.tokens[i] = -1;
  };
  // (rows of no sequence; one that has none of its own may be the first or the last)
  if (b == 0) none(0, first);
  if ((size_t)b + 1 == a.batch) none(first + w.sp.n, a.rows);
  if (w.n <= 0) {
    if (threadIdx.x == 0) a.count[b] = 0;
    return;
  }
  auto accept = [&](int k, int i, int64_t token) {
    if (lane == 0) {
      a.path[first + k] = i;
      a.tokens[first + k - 1] = token;
    }
  };
  int k = 0;
  bool more = false, whole = false;  // whole: the sum wanted is of p itself
  for (bool start = true;; start = false) {
    if (wave == 0) {
      bool wanted;
      if (start) {
        more = w.go(accept);
        wanted = true;
        whole = !w.rejected;
      } else {
        double z = wave_sum(lane < j.pieces ? pieces[lane] : 0.);
        wanted = false;
        if (more) {
          w.z = z;
          more = w.go(accept);
          // done where it ended by a rejection, whose sum is there
          if (more || !w.rejected) wanted = true;
          whole = !w.rejected;
        }
        if (!wanted && !whole && !(w.z > 0)) wanted = whole = true;  // nothing left: from p
        z = whole ? z : w.z;
        if (lane == 0) aim = z;
      }
      if (lane == 0) {
        node = first + w.node;
        at = whole ? 0. : w.c;
        state = !wanted;
      }
    }
    __syncthreads();
    if (state) break;
    const T *p = (const T *)a.p + (size_t)node * a.p_stride;
    const T *q = (const T *)a.q + (size_t)node * a.q_stride;
    if (k < j.rounds) {
      if (threadIdx.x < j.pieces)
        pieces[threadIdx.x] = j.sums[((size_t)k * a.batch + b) * j.pieces + threadIdx.x];
    } else {
      for (int i = wave; i < j.pieces; i += WAVES) {
        const size_t lo = i * j.piece, hi = lo + j.piece < a.vocab ? lo + j.piece : a.vocab;
        const double s = wave_sum(share<8>(p, q, at, lo, hi, lane, 64));
        if (lane == 0) pieces[i] = s;
      }
    }
    ++k;
    __syncthreads();
  }
  // The first value whose running sum is past u times the whole: its piece, its thread,
  // itself.  Where rounding (or u >= 1) leaves none, the last that has any weight.
  if (threadIdx.x == 0) {
    const double goal = (double)a.u[first] * aim;
    double sum = 0;
    int in = -1, any = -1;
    double from = 0;
    for (int i = 0; i < j.pieces && in < 0; ++i) {
      if (pieces[i] > 0) any = i, from = sum;
      if (sum + pieces[i] > goal) in = i;
      else sum += pieces[i];
    }
    chosen = in >= 0 ? in : any;
    base = in >= 0 ? sum : from;
    aim = goal;
    found = 0x7fffffff;
    last = -1;
  }
  __syncthreads();
  int64_t drawn = -1;
  if (chosen >= 0) {
    const T *p = (const T *)a.p + (size_t)node * a.p_stride;
    const T *q = (const T *)a.q + (size_t)node * a.q_stride;
    const size_t lo = chosen * j.piece, hi = lo + j.piece < a.vocab ? lo + j.piece : a.vocab;
    const size_t each = (hi - lo + TEAM - 1) / TEAM;
    const size_t v0 = std::min(lo + threadIdx.x * each, hi), v1 = std::min(v0 + each, hi);
    double mine = 0;
    for (size_t v = v0; v < v1; ++v)
      mine += left_at(p, q, at, v);
    double upto = mine;  // inclusive over the wave, then with the waves before
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const double x = __shfl_up(upto, m);
      if (lane >= m) upto += x;
    }
    if (lane == 63) before[wave] = upto;
    __syncthreads();
    double from = base;
    for (int i = 0; i < wave; ++i) from += before[i];
    const double left = __shfl_up(upto, 1);
    const double excl = lane ? from + left : from, incl = from + upto;
    auto some = [&](double run) {  // the first value past the aim, or the last with weight
      int v_last = -1;
      for (size_t v = v0; v < v1; ++v) {
        const double r = left_at(p, q, at, v);
        if (!(r > 0)) continue;
        v_last = (int)v;
        run += r;
        if (run > aim) break;
      }
      return v_last;
    };
    // (of each wave the first thread with any weight that gets past the aim: sums in another
    // order may pass it at a word without weight, by their last bit)
    const uint64_t past = __ballot(mine > 0 && incl > aim);
    if (past && lane == __builtin_ctzll(past)) atomicMin(&found, some(excl));
    __syncthreads();
    if (found == 0x7fffffff) {  // (the same in every thread)
      const int v = mine > 0 ? some(-__builtin_inf()) : -1;
      if (v >= 0) atomicMax(&last, v);
    }
    __syncthreads();
    drawn = found != 0x7fffffff ? found : last;
  }
  // (wave 0 has the walk)
  __shared__ int kept;
  if (threadIdx.x == 0) {
    kept = w.count;
    a.count[b] = w.count;
    a.path[first] = 0;
    a.tokens[first + w.count - 1] = drawn;
  }
  __syncthreads();
  none(first + kept, first + w.sp.n);
}

int pieces_of(size_t vocab) {
  return (int)std::min<size_t>(PIECES, (vocab + PIECE - 1) / PIECE);
}
// Launches before the last: none where a row is but a few pieces; one for chains, which
// want one sum; for trees as many as the slowest sequence is likely to want (16 trees of 32
// over 128000 words: 51 us with one, 45 with two, 39 with three, 40 with four; one tree 20,
// 20, 22 and 25).
int rounds_of(bool tree, size_t batch, size_t vocab) {
  return pieces_of(vocab) < 4 ? 0 : !tree ? 1 : batch < 8 ? 2 : ROUNDS;
}

}  // namespace

size_t verify_drafts_workspace(size_t batch, size_t vocab) {
  return rounds_of(true, batch, vocab) * batch * pieces_of(vocab) * sizeof(double);
}

hipError_t launch_verify_drafts(const VerifyArgs &a, hipStream_t st) {
  Job j{a, pieces_of(a.vocab), rounds_of(a.parents != nullptr, a.batch, a.vocab), 0, (double *)a.workspace};
  j.piece = ((a.vocab + j.pieces - 1) / j.pieces + 3) / 4 * 4;
  j.pieces = (int)((a.vocab + j.piece - 1) / j.piece);
  if (a.batch > 65535 || !grid_fits(a.batch, TEAM)) return hipErrorInvalidConfiguration;
  auto run = [&](auto type) {
    using T = decltype(type);
    for (int r = 0; r < j.rounds; ++r)
      hipLaunchKernelGGL(k_verify_round<T>, dim3((unsigned)j.pieces, (unsigned)a.batch), dim3(256), 0,
                         st, j, r);
    hipLaunchKernelGGL(k_verify_end<T>, dim3((unsigned)a.batch), dim3(TEAM), 0, st, j);
    return hipGetLastError();
  };
  if (a.dtype == ROSETTA_F32) return run(0.f);
  if (a.dtype == ROSETTA_BF16) return run((bf16)0.f);
  return run((f16)0.f);
}

}  // namespace rosetta
