// Scores of rows of logits: log probability of a token, entropy, likeliest tokens; and the logits' gradient.
//
// With m the largest logit x of a row, z = scale (x - m), S = sum exp z and T = sum z exp z:
//   log p = z - log S,   entropy = log S - T / S,   dx = scale (g (1 - p) or -g p  -  h p (log p + entropy)).
// m, S and T come from one pass: what a thread has summed is rescaled where it meets a larger logit.  z is formed from the difference,
// so that neither a mask of the type's lowest value nor scale overflows it.  All is bound by the memory.
#include <algorithm>
#include <type_traits>

#include "tt_emb_internal.h"

namespace ttemb {

constexpr float kLn2 = 0.693147180559945f, kLog2e = 1.44269504088896f;
constexpr float kNothing = -1000.f;           // 2 to its power is 0
constexpr float kLowest = -3.402823466e38f;   // start of a maximum: a row of -infinity alone keeps it, and has S = 0

__device__ __forceinline__ float pow2(float z) { return __builtin_amdgcn_exp2f(z); }

struct Sums {
  float most, sum, tilt;  // largest logit m; sum of 2^y and of y 2^y with y = (x - m) c, c = scale / log 2
};

// Rescales to another maximum, which is no smaller.
template <bool ENT>
__device__ __forceinline__ void rescale(Sums& s, float most, float c) {
  const float y = fmaxf((s.most - most) * c, kNothing), f = pow2(y);
  if constexpr (ENT) s.tilt = f * fmaf(y, s.sum, s.tilt);
  s.sum *= f;
  s.most = most;
}

template <bool ENT, int N>
__device__ __forceinline__ void add_values(Sums& s, const float (&x)[N], float most_x, float c) {
  if (most_x > s.most) rescale<ENT>(s, most_x, c);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float y = (x[i] - s.most) * c;
    const float e = pow2(y);
    if constexpr (ENT) s.tilt = fmaf(e, fmaxf(y, kNothing), s.tilt);  // no 0 * infinity; where y is NaN, so is e
    s.sum += e;
  }
}

// Over groups of L lanes, the same in every lane of a group.
template <bool ENT, int L>
__device__ __forceinline__ void join_lanes(Sums& s, float c) {
  float most = s.most;
#pragma unroll
  for (int d = L / 2; d > 0; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
  rescale<ENT>(s, most, c);
#pragma unroll
  for (int d = L / 2; d > 0; d /= 2) {
    s.sum += __shfl_xor(s.sum, d);
    if constexpr (ENT) s.tilt += __shfl_xor(s.tilt, d);
  }
}

// Over a block, the same in every thread.  `part`: a place for each wavefront; free again after the caller's next barrier.
template <bool ENT, int NT>
__device__ __forceinline__ void join_block(Sums& s, float c, Sums* part) {
  join_lanes<ENT, kWave>(s, c);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = s;
  __syncthreads();
  constexpr int W = NT / kWave;
  s = part[threadIdx.x % W];
  join_lanes<ENT, W>(s, c);
}

// ---- order of logits: larger first, then the lower index; NaN before all

typedef unsigned long long Key;  // 0: nothing
__device__ __forceinline__ Key key_of(float x, int v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);  // -0 becomes +0
  const uint32_t o = x != x ? 0xffffffffu : (b >> 31 ? ~b : b | 0x80000000u);
  return (Key)o << 32 | (uint32_t)~v;
}
__device__ __forceinline__ float key_value(Key k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __builtin_bit_cast(float, o >> 31 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_index(Key k) { return (int)~(uint32_t)k; }

__device__ __forceinline__ Key read_lane(Key k, int lane) {
  return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}
__device__ __forceinline__ Key max_key(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key min_key(Key a, Key b) { return a > b ? b : a; }

// A bitonic sequence of a wavefront's keys into falling order.
__device__ __forceinline__ Key merged(Key k) {
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) {
    const Key o = __shfl_xor(k, d);
    k = lane & d ? min_key(k, o) : max_key(k, o);
  }
  return k;
}
__device__ __forceinline__ Key sorted(Key k) {
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int run = 2; run < kWave; run *= 2)
#pragma unroll
    for (int d = run / 2; d > 0; d /= 2) {
      const Key o = __shfl_xor(k, d);
      k = ((lane & d) != 0) == ((lane & run) == 0) ? min_key(k, o) : max_key(k, o);
    }
  return merged(k);
}
// The larger half of two falling lists, falling.
__device__ __forceinline__ Key joined(Key a, Key b) {
  return merged(max_key(a, __shfl(b, kWave - 1 - (int)(threadIdx.x % kWave))));
}

// The largest 64 keys that a wavefront has met, one a lane, falling; what does not exceed the one in lane top - 1 is not
// put in.
struct TopList {
  Key list, least;
  float least_value;
  int top;
  __device__ __forceinline__ explicit TopList(int n) : list(0), least(0), least_value(-INFINITY), top(n) {}
  __device__ __forceinline__ void settle() {
    least = read_lane(list, top - 1);
    least_value = least ? key_value(least) : -INFINITY;
  }
  // One key a lane (0: none).  Few are put in one by one, many sorted and joined.
  __device__ __forceinline__ void put(Key k) {
    uint64_t mask = __ballot(k > least);
    if (__popcll(mask) > 10) {
      list = joined(list, sorted(k > least ? k : 0));
      settle();
      return;
    }
    while (mask) {
      const Key n = read_lane(k, __ffsll((unsigned long long)mask) - 1);
      Key before = __shfl_up(list, 1);
      if (threadIdx.x % kWave == 0) before = ~(Key)0;
      list = list > n ? list : before > n ? n : before;
      settle();
      mask &= mask - 1;
      mask &= __ballot(k > least);
    }
  }
};

// The lists of W wavefronts joined into the first's.  `lists`: 64 places for each; free again after the next barrier.
template <int W>
__device__ __forceinline__ void join_lists(Key& list, Key* lists) {
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  lists[w * kWave + lane] = list;
#pragma unroll
  for (int half = W / 2; half > 0; half /= 2) {
    __syncthreads();
    if (w < half) {
      list = joined(list, lists[(w + half) * kWave + lane]);
      lists[w * kWave + lane] = list;
    }
  }
}

// ---- what is read and written

__device__ __forceinline__ float log_sum(const Sums& s) { return s.sum == 0.f ? -INFINITY : logf(s.sum); }

// One lane of the row's writes the numbers; the first `top` lanes of a wavefront write the list.
__device__ __forceinline__ void put_numbers(const TokenOut& o, const TokenRows& t, int64_t row, const Sums& s,
                                            int64_t token, float x) {
  const float logs = log_sum(s);
  const bool empty = s.sum == 0.f;
  if (o.logprob) o.logprob[row] = empty ? -INFINITY : (x - s.most) * t.scale - logs;
  if (o.entropy) {
    const float h = logs - s.tilt / s.sum * kLn2;
    o.entropy[row] = empty || h < 0.f ? 0.f : h;
  }
  if (o.state) {
    o.state[row] = s.most;
    o.state[t.rows + row] = logs;
  }
}
__device__ __forceinline__ void put_none(const TokenOut& o, const TokenRows& t, int64_t row) {
  if (o.logprob) o.logprob[row] = 0.f;
  if (o.entropy) o.entropy[row] = 0.f;
  if (o.state) o.state[row] = o.state[t.rows + row] = 0.f;
}
__device__ __forceinline__ void put_top(const TokenOut& o, const TokenRows& t, int64_t row, const Sums& s, Key k,
                                        int place) {
  if (place >= o.top) return;
  const bool none = k == 0, empty = s.sum == 0.f;
  o.top_ids[row * o.top + place] = none ? -1 : key_index(k);
  o.top_logprob[row * o.top + place] = none || empty ? -INFINITY : (key_value(k) - s.most) * t.scale - log_sum(s);
}

// A row's gradient: factor of p, of p log p, and what the token's place gets besides.
struct RowGradient {
  float most, logs2, a, b, token_part;
  int64_t token;  // -1: no place
  bool zero;      // nothing is read
};
__device__ __forceinline__ RowGradient loss_gradient(const TokenRows& t, const Sums& s, float w, int64_t token) {
  return {s.most, log2f(s.sum), t.scale * w, 0.f, -t.scale * w, token, s.sum == 0.f};
}
template <bool ENT>
__device__ __forceinline__ float gradient_of(const RowGradient& g, float x, int v, float c) {
  const float y = fmaf(x - g.most, c, -g.logs2), p = pow2(y);
  float d;
  if constexpr (ENT) d = p * fmaf(g.b, fmaxf(y, kNothing), g.a);
  else d = p * g.a;
  return v == g.token ? d + g.token_part : d;
}

// ---- narrow rows: L lanes hold one, N pieces each

template <class T, int L, int N>
struct NarrowRow {
  static constexpr int P = 16 / sizeof(T);
  float x[N * P];
  int first[N];  // the columns of the pieces; pieces at the end of a row start early, and hold their neighbour's too
  int own[N];    // from here on the columns are the piece's own
  __device__ __forceinline__ void load(const T* row, int cols, int lane) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
      own[q] = (q * L + lane) * P;
      first[q] = cols >= P ? min(own[q], cols - P) : 0;
      float v[P];
      if (own[q] >= cols) {
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = -INFINITY;
      } else if (cols >= P) {
        load_piece<P, T>(row + first[q], v);
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = i < cols ? (float)row[i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < P; ++i) x[q * P + i] = v[i];
    }
  }
  __device__ __forceinline__ bool mine(int q, int i, int cols) const {
    return first[q] + i >= own[q] && first[q] + i < cols;
  }
  template <bool ENT>
  __device__ __forceinline__ Sums sums(int cols, float c) const {
    float v[N * P], most = kLowest;
#pragma unroll
    for (int q = 0; q < N; ++q)
#pragma unroll
      for (int i = 0; i < P; ++i) {
        v[q * P + i] = mine(q, i, cols) ? x[q * P + i] : -INFINITY;
        most = fmaxf(most, v[q * P + i]);
      }
    Sums s{most, 0.f, 0.f};
    add_values<ENT>(s, v, most, c);
    join_lanes<ENT, L>(s, c);
    return s;
  }
};

constexpr int kNarrowThreads = 256;
template <class T, int L, int N>
__global__ __launch_bounds__(kNarrowThreads) void k_token_narrow(TokenRows t, TokenOut o) {
  constexpr int P = 16 / sizeof(T);
  const int lane = threadIdx.x % L;
  const T* x = (const T*)t.logits;
  for (int64_t row = (int64_t)blockIdx.x * (kNarrowThreads / L) + threadIdx.x / L; row < t.rows;
       row += (int64_t)gridDim.x * (kNarrowThreads / L)) {
    const int64_t token = t.tokens ? t.tokens[row] : 0;
    if ((uint64_t)token >= (uint64_t)t.cols) {
      if (lane == 0) put_none(o, t, row);
      if (o.top_ids)
        for (int k = lane; k < o.top; k += L) put_top(o, t, row, Sums{0.f, 0.f, 0.f}, 0, k);
      continue;
    }
    NarrowRow<T, L, N> r;
    r.load(x + row * t.ld, t.cols, lane);
    const float at = (float)x[row * t.ld + token];
    const Sums s = o.entropy ? r.template sums<true>(t.cols, t.c) : r.template sums<false>(t.cols, t.c);
    if (lane == 0) put_numbers(o, t, row, s, token, at);
    if (!o.top_ids) continue;
    Key last = ~(Key)0;
    for (int k = 0; k < o.top; ++k) {  // the largest that is smaller than the one before
      Key best = 0;
      if (last != 0) {
#pragma unroll
        for (int q = 0; q < N; ++q)
#pragma unroll
          for (int i = 0; i < P; ++i) {
            const Key n = key_of(r.x[q * P + i], r.first[q] + i);
            if (r.mine(q, i, t.cols) && n < last) best = max_key(best, n);
          }
#pragma unroll
        for (int d = L / 2; d > 0; d /= 2) best = max_key(best, __shfl_xor(best, d));
      }
      if (lane == k % L) put_top(o, t, row, s, best, k);
      last = best;
    }
  }
}

template <class T, class TO, int L, int N>
__global__ __launch_bounds__(kNarrowThreads) void k_token_loss_narrow(TokenRows t, const float* __restrict__ weights,
                                                                      float weight, float* __restrict__ logprob, TO* dx,
                                                                      int64_t ld_dx) {
  constexpr int P = 16 / sizeof(T);
  const int lane = threadIdx.x % L;
  const T* x = (const T*)t.logits;
  for (int64_t row = (int64_t)blockIdx.x * (kNarrowThreads / L) + threadIdx.x / L; row < t.rows;
       row += (int64_t)gridDim.x * (kNarrowThreads / L)) {
    const int64_t token = t.tokens[row];
    const bool counts = (uint64_t)token < (uint64_t)t.cols;
    NarrowRow<T, L, N> r;
    Sums s{0.f, 0.f, 0.f};
    RowGradient g{};
    if (counts) {
      r.load(x + row * t.ld, t.cols, lane);
      const float at = (float)x[row * t.ld + token];
      s = r.template sums<false>(t.cols, t.c);
      g = loss_gradient(t, s, weights ? weight * weights[row] : weight, token);
      if (lane == 0) logprob[row] = s.sum == 0.f ? -INFINITY : (at - s.most) * t.scale - log_sum(s);
    } else {
      g.zero = true;
      if (lane == 0) logprob[row] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int own = (q * L + lane) * P, first = t.cols >= P ? min(own, t.cols - P) : 0;
      if (own >= t.cols) continue;
      float v[P];
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = g.zero ? 0.f : gradient_of<false>(g, r.x[q * P + i], first + i, t.c);
      TO* to = dx + row * ld_dx + first;
      if (t.cols >= P) store_piece<P, TO>(to, v);
      else
#pragma unroll
        for (int i = 0; i < P; ++i)
          if (i < t.cols) to[i] = (TO)v[i];
    }
  }
}

// ---- wide rows: a block has one, or a part of one

// Four pieces of a row at a time by every thread of a block, then what is left of the columns [from, to): f(values,
// columns of their pieces, how many of them there are a piece).
template <int NT, class T, class F, class G>
__device__ __forceinline__ void sweep(const T* __restrict__ row, int from, int to, F&& four, G&& one) {
  constexpr int P = 16 / sizeof(T), U = 4;
  const int pieces = (to - from) / P;
  int k = threadIdx.x;
  for (; k - (int)threadIdx.x + U * NT <= pieces; k += U * NT) {  // the same for all
    typename Piece<T, P>::V v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *(const typename Piece<T, P>::V*)(row + from + (k + u * NT) * P);
    float x[U * P];
    int first[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      first[u] = from + (k + u * NT) * P;
#pragma unroll
      for (int i = 0; i < P; ++i) x[u * P + i] = (float)v[u][i];
    }
    four(x, first);
  }
  for (; k - (int)threadIdx.x < pieces; k += NT) {
    float x[P];
    const int first = from + min(k, pieces - 1) * P;
    load_piece<P, T>(row + first, x);
    if (k >= pieces) {
#pragma unroll
      for (int i = 0; i < P; ++i) x[i] = -INFINITY;
    }
    one(x, first, k < pieces);
  }
  const int rest = from + pieces * P + (int)threadIdx.x;
  if ((to - from) % P) {
    float x[1] = {rest < to ? (float)row[rest] : -INFINITY};
    one(x, rest, rest < to);
  }
}

template <int N>
__device__ __forceinline__ float largest(const float (&x)[N]) {
  float most = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) most = fmaxf(most, x[i]);
  return most;
}

template <bool ENT, bool TOP, int NT, class T>
__device__ __forceinline__ Sums row_sums(const T* __restrict__ row, int from, int to, float c, TopList& top) {
  Sums s{kLowest, 0.f, 0.f};
  sweep<NT>(
      row, from, to,
      [&](const auto& x, const auto& first) {
        constexpr int N = sizeof(x) / sizeof(float), U = sizeof(first) / sizeof(int), P = N / U;
        const float most = largest(x);
        add_values<ENT>(s, x, most, c);
        if constexpr (TOP) {
          if (!__any(!(most < top.least_value) || s.sum != s.sum)) return;
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (__any(!(x[i] < top.least_value))) top.put(key_of(x[i], first[i / P] + i % P));
        }
      },
      [&](const auto& x, int first, bool there) {
        constexpr int N = sizeof(x) / sizeof(float);
        add_values<ENT>(s, x, largest(x), c);
        if constexpr (TOP) {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (__any(there && !(x[i] < top.least_value))) top.put(there ? key_of(x[i], first + i) : 0);
        }
      });
  return s;
}

// Scores of a row by a block, or (splits > 1) the sums and the list of `per` columns of it.
template <class T, int NT, bool ENT, bool TOP>
__global__ __launch_bounds__(NT) void k_token_wide(TokenRows t, TokenOut o, int splits, int per, TokenParts parts) {
  __shared__ Sums part[NT / kWave];
  __shared__ Key lists[TOP ? NT : 1];
  const T* x = (const T*)t.logits;
  const int64_t work = t.rows * splits;
  for (int64_t b = blockIdx.x; b < work; b += gridDim.x) {
    const int64_t row = splits > 1 ? b / splits : b;
    const int split = splits > 1 ? (int)(b - row * splits) : 0;
    const int64_t token = t.tokens ? t.tokens[row] : 0;
    if ((uint64_t)token >= (uint64_t)t.cols) {
      if (splits == 1) {
        if (threadIdx.x == 0) put_none(o, t, row);
        if (TOP && threadIdx.x < kWave) put_top(o, t, row, Sums{0.f, 0.f, 0.f}, 0, threadIdx.x);
      }
      continue;
    }
    const float at = (float)x[row * t.ld + token];
    TopList top(TOP ? o.top : 1);
    const int from = split * per;
    Sums s = row_sums<ENT, TOP, NT>(x + row * t.ld, from, min(t.cols, from + per), t.c, top);
    join_block<ENT, NT>(s, t.c, part);
    if constexpr (TOP) join_lists<NT / kWave>(top.list, lists);
    if (splits > 1) {
      if (threadIdx.x == 0) parts.sums[b] = f4{s.most, s.sum, s.tilt, 0.f};
      if (TOP && threadIdx.x < kWave) parts.lists[b * kWave + threadIdx.x] = top.list;
    } else {
      if (threadIdx.x == 0) put_numbers(o, t, row, s, token, at);
      if (TOP && threadIdx.x < kWave) put_top(o, t, row, s, top.list, threadIdx.x);
    }
    __syncthreads();
  }
}

// The parts of a row joined by a block.
constexpr int kJoinThreads = 256;
template <class T, bool TOP>
__global__ __launch_bounds__(kJoinThreads) void k_token_join(TokenRows t, TokenOut o, int splits, TokenParts parts) {
  __shared__ Key lists[TOP ? kJoinThreads : 1];
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  const int64_t row = blockIdx.x;
  const int64_t token = t.tokens ? t.tokens[row] : 0;
  const bool counts = (uint64_t)token < (uint64_t)t.cols;
  if (!counts) {
    if (threadIdx.x == 0) put_none(o, t, row);
    if (TOP && w == 0) put_top(o, t, row, Sums{0.f, 0.f, 0.f}, 0, lane);
    return;
  }
  const float at = (float)((const T*)t.logits)[row * t.ld + token];
  Sums s{kLowest, 0.f, 0.f};
  if (lane < splits) {
    const f4 p = parts.sums[row * splits + lane];
    s = Sums{p.x, p.y, p.z};
  }
  join_lanes<true, kWave>(s, t.c);
  if (threadIdx.x == 0) put_numbers(o, t, row, s, token, at);
  if constexpr (TOP) {
    Key list = 0;
    for (int k = w; k < splits; k += kJoinThreads / kWave)
      list = joined(list, parts.lists[(row * splits + k) * kWave + lane]);
    join_lists<kJoinThreads / kWave>(list, lists);
    if (w == 0) put_top(o, t, row, s, list, lane);
  }
}

// ---- gradient

// Columns [from, to) of a row's gradient by a block.  Elements are read and written by the same thread: dx may be x.
template <bool ENT, int NT, class T, class TO>
__device__ __forceinline__ void put_gradient(const RowGradient& g, const T* x, TO* dx, int from, int to, float c,
                                             int thread) {
  constexpr int P = 16 / (sizeof(T) > sizeof(TO) ? sizeof(T) : sizeof(TO));
  const int pieces = (to - from) / P;
  for (int k = thread; k < pieces; k += NT) {
    const int first = from + k * P;
    float v[P];
    if (g.zero) {
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = 0.f;
    } else {
      load_piece<P, T>(x + first, v);
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = gradient_of<ENT>(g, v[i], first + i, c);
    }
    store_piece<P, TO, true>(dx + first, v);
  }
  const int rest = from + pieces * P + thread;
  if (rest < to) dx[rest] = (TO)(g.zero ? 0.f : gradient_of<ENT>(g, (float)x[rest], rest, c));
}

struct Upstream {
  const float *state, *entropy, *d_logprob, *d_entropy;
};

constexpr int kGradThreads = 256;
template <class T, class TO, bool ENT, int NT>
__global__ __launch_bounds__(kGradThreads) void k_token_grad(TokenRows t, Upstream u, TO* dx, int64_t ld_dx,
                                                             int splits, int per) {
  constexpr int kSide = kGradThreads / NT;  // rows beside each other in a block
  const int64_t work = t.rows * splits;
  for (int64_t b = (int64_t)blockIdx.x * kSide + threadIdx.x / NT; b < work; b += (int64_t)gridDim.x * kSide) {
    const int64_t row = splits > 1 ? b / splits : b;
    const int from = splits > 1 ? (int)(b - row * splits) * per : 0;
    const int64_t token = t.tokens ? t.tokens[row] : 0;
    RowGradient g{};
    g.zero = (uint64_t)token >= (uint64_t)t.cols;
    if (!g.zero) {
      const float logs = u.state[t.rows + row];
      const float d = u.d_logprob ? u.d_logprob[row] : 0.f, h = ENT ? u.d_entropy[row] : 0.f;
      g = RowGradient{u.state[row], logs * kLog2e, -t.scale * (ENT ? fmaf(h, u.entropy[row], d) : d), -t.scale * h * kLn2,
                      t.scale * d, t.tokens ? token : -1, logs == -INFINITY};
    }
    put_gradient<ENT, NT, T, TO>(g, (const T*)t.logits + row * t.ld, dx + row * ld_dx, from,
                                 min(t.cols, from + per), t.c, threadIdx.x % NT);
  }
}

// Log probability and gradient of a row by a block, which reads it a second time from the caches.
template <class T, class TO, int NT>
__global__ __launch_bounds__(NT) void k_token_loss(TokenRows t, const float* __restrict__ weights, float weight,
                                                   float* __restrict__ logprob, TO* dx, int64_t ld_dx) {
  __shared__ Sums part[NT / kWave];
  for (int64_t row = blockIdx.x; row < t.rows; row += gridDim.x) {
    const int64_t token = t.tokens[row];
    const T* x = (const T*)t.logits + row * t.ld;
    RowGradient g{};
    g.zero = (uint64_t)token >= (uint64_t)t.cols;
    if (g.zero) {
      if (threadIdx.x == 0) logprob[row] = 0.f;
    } else {
      const float at = (float)x[token];
      TopList none(1);
      Sums s = row_sums<false, false, NT>(x, 0, t.cols, t.c, none);
      join_block<false, NT>(s, t.c, part);  // its barrier also stands between all reads of x[token] and the first write
      g = loss_gradient(t, s, weights ? weight * weights[row] : weight, token);
      if (threadIdx.x == 0) logprob[row] = s.sum == 0.f ? -INFINITY : (at - s.most) * t.scale - log_sum(s);
    }
    put_gradient<false, NT, T, TO>(g, x, dx + row * ld_dx, 0, t.cols, t.c, threadIdx.x);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------
// host-side launchers

constexpr int64_t kMostBlocks = 1 << 20;
static int grid_of(int64_t blocks) { return (int)std::min(blocks, kMostBlocks); }

// Lanes and pieces of narrow rows: f(L, N) as constants; false: wider ones.
template <class T, class F>
static bool with_narrow(int cols, bool few, F&& f) {
  constexpr int P = 16 / sizeof(T);
  if (cols <= 4 * P) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
  else if (cols <= 16 * P) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
  else if (cols <= 64 * P) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else if (!few && cols <= 256 * P) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
  else return false;
  return true;
}

// How many blocks take a row of few rows, and how many columns each.
static int splits_of(int64_t rows, int cols, int* per) {
  int64_t n = std::min<int64_t>(kTokenParts / std::max<int64_t>(rows, 1), kWave);
  n = std::max<int64_t>(1, std::min<int64_t>(n, cols / 4096));
  *per = (int)((cols + n - 1) / n + 7) / 8 * 8;
  return (cols + *per - 1) / *per;
}

template <class T, int NT, bool ENT>
static void launch_wide(const TokenRows& t, const TokenOut& o, int splits, int per, const TokenParts& parts, hipStream_t st) {
  const int blocks = grid_of(t.rows * splits);
  if (o.top_ids) k_token_wide<T, NT, ENT, true><<<blocks, NT, 0, st>>>(t, o, splits, per, parts);
  else k_token_wide<T, NT, ENT, false><<<blocks, NT, 0, st>>>(t, o, splits, per, parts);
}

void launch_token_scores(const TokenRows& t, int type, const TokenOut& o, const TokenParts& parts, hipStream_t st) {
  with_type(type, [&](auto ti) {
    typedef decltype(ti) T;
    const bool narrow = with_narrow<T>(t.cols, o.top_ids != nullptr, [&](auto l, auto n) {
      constexpr int L = decltype(l)::value, N = decltype(n)::value, kSide = kNarrowThreads / L;
      k_token_narrow<T, L, N><<<grid_of((t.rows + kSide - 1) / kSide), kNarrowThreads, 0, st>>>(t, o);
    });
    if (narrow) return;
    int per;
    const int splits = splits_of(t.rows, t.cols, &per);
    constexpr int NT = 512;
    if (o.entropy) launch_wide<T, NT, true>(t, o, splits, per, parts, st);
    else launch_wide<T, NT, false>(t, o, splits, per, parts, st);
    if (splits == 1) return;
    if (o.top_ids) k_token_join<T, true><<<(int)t.rows, kJoinThreads, 0, st>>>(t, o, splits, parts);
    else k_token_join<T, false><<<(int)t.rows, kJoinThreads, 0, st>>>(t, o, splits, parts);
  });
}

template <class T, class TO>
static void launch_grad(const TokenRows& t, const Upstream& u, TO* dx, int64_t ld_dx, hipStream_t st) {
  auto go = [&](auto ent, auto nt, int splits, int per) {
    constexpr bool ENT = decltype(ent)::value;
    constexpr int NT = decltype(nt)::value, kSide = kGradThreads / NT;
    k_token_grad<T, TO, ENT, NT>
        <<<grid_of((t.rows * splits + kSide - 1) / kSide), kGradThreads, 0, st>>>(t, u, dx, ld_dx, splits, per);
  };
  auto sized = [&](auto ent) {
    if (t.cols <= 64) return go(ent, std::integral_constant<int, 16>{}, 1, t.cols);
    if (t.cols <= 1024) return go(ent, std::integral_constant<int, 64>{}, 1, t.cols);
    const int per = 16384;
    go(ent, std::integral_constant<int, kGradThreads>{}, (t.cols + per - 1) / per, per);
  };
  if (u.d_entropy) sized(std::true_type{});
  else sized(std::false_type{});
}

void launch_token_grad(const TokenRows& t, int type, const float* state, const float* entropy, const float* d_logprob,
                       const float* d_entropy, const tt_emb_matrix& dx, hipStream_t st) {
  const Upstream u{state, entropy, d_logprob, d_entropy};
  with_type(type, [&](auto ti) {
    with_type(dx.type, [&](auto to) { launch_grad<decltype(ti), decltype(to)>(t, u, (decltype(to)*)dx.data, dx.ld, st); });
  });
}

void launch_token_loss(const TokenRows& t, int type, const float* weights, float weight, float* logprob,
                       const tt_emb_matrix& dx, hipStream_t st) {
  with_type(type, [&](auto ti) {
    with_type(dx.type, [&](auto tout) {
      typedef decltype(ti) T;
      typedef decltype(tout) TO;
      TO* to = (TO*)dx.data;
      const bool narrow = with_narrow<T>(t.cols, false, [&](auto l, auto n) {
        constexpr int L = decltype(l)::value, N = decltype(n)::value, kSide = kNarrowThreads / L;
        k_token_loss_narrow<T, TO, L, N><<<grid_of((t.rows + kSide - 1) / kSide), kNarrowThreads, 0, st>>>(
            t, weights, weight, logprob, to, dx.ld);
      });
      if (!narrow) k_token_loss<T, TO, 1024><<<grid_of(t.rows), 1024, 0, st>>>(t, weights, weight, logprob, to, dx.ld);
    });
  });
}

}  // namespace ttemb
