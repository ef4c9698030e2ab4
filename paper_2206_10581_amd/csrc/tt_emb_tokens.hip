// Scores of rows of logits: log probability of a token, entropy, likeliest tokens; and the logits' gradient.
//
// With m the largest logit x of a row, z = scale (x - m), S = sum exp z and T = sum z exp z:
//   log p = z - log S,   entropy = log S - T / S,   dx = scale (g (1 - p) or -g p  -  h p (log p + entropy)).
// m, S and T come from one pass: what a thread has summed is rescaled where it meets a larger logit.  z is formed from the difference,
// so that neither a mask of the type's lowest value nor scale overflows it.  With entropy a logit of wide bf16 rows takes 11.6 vector
// instructions (counted, 2744 rows of 32,000): such rows are bound by the memory, narrow ones by what a row costs besides.
//
// Rows of up to 16 lanes' four pieces (256 fp32, 512 16-bit logits) are held by 4 or 16 lanes of a wavefront; wider ones are taken by
// a block of 64 to 1024 threads, or, of few rows, by several blocks whose sums a second launch joins.  Measured (one MI355X, us a
// call among others): 200,000 rows of 47 fp32 with entropy and three alternatives 18.4, 743 vector instructions for 16 rows; 48 of
// 128,000 bf16 with entropy and twenty 20.9, bound by its latencies; the loss of 4096 x 128,000 bf16 443 (2.1 GB read and written,
// 4.7 TB/s; a copy's rate 5.15), of 200,000 x 47 fp32 17.8 (4.3 TB/s).
#include <limits.h>

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

// Of every 2 D lanes (D = 16 or 32) what the lower and the upper half hold, in both.
struct Halves {
  uint32_t lower, upper;
};
template <int D>
__device__ __forceinline__ Halves halves(uint32_t v) {
  if constexpr (D == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return {r[0], r[1]};
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return {r[0], r[1]};
  }
}
// What the lane at distance D (a power of two) holds, where groups of D lanes hold the same: f(own, other) in every lane.
template <int D, class F>
__device__ __forceinline__ float joined_lanes(float v, F&& f) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  if constexpr (D >= 16) {
    const Halves r = halves<D>(b);
    return f(__builtin_bit_cast(float, r.lower), __builtin_bit_cast(float, r.upper));
  } else {  // neighbour, neighbouring pair, mirrored eight, mirrored sixteen
    constexpr int kMove = D == 1 ? 0xB1 : D == 2 ? 0x4E : D == 4 ? 0x141 : 0x140;
    return f(v, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp((int)b, kMove, 0xf, 0xf, true)));
  }
}
template <int L, class F>
__device__ __forceinline__ float over_lanes(float v, F&& f) {
  if constexpr (L > 1) v = joined_lanes<1>(v, f);
  if constexpr (L > 2) v = joined_lanes<2>(v, f);
  if constexpr (L > 4) v = joined_lanes<4>(v, f);
  if constexpr (L > 8) v = joined_lanes<8>(v, f);
  if constexpr (L > 16) v = joined_lanes<16>(v, f);
  if constexpr (L > 32) v = joined_lanes<32>(v, f);
  return v;
}
template <int L, class F>
__device__ __forceinline__ uint32_t lanes_of(uint32_t v, F&& f) {
  return __builtin_bit_cast(uint32_t, over_lanes<L>(__builtin_bit_cast(float, v), [&](float a, float b) {
                              return __builtin_bit_cast(float, f(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)));
                            }));
}
template <int L>
__device__ __forceinline__ float lanes_max(float v) {
  return over_lanes<L>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  return over_lanes<L>(v, [](float a, float b) { return a + b; });
}

// Over groups of L lanes, the same in every lane of a group.
template <bool ENT, int L>
__device__ __forceinline__ void join_lanes(Sums& s, float c) {
  rescale<ENT>(s, lanes_max<L>(s.most), c);
  s.sum = lanes_sum<L>(s.sum);
  if constexpr (ENT) s.tilt = lanes_sum<L>(s.tilt);
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

// What lane ^ D holds.
template <int D>
__device__ __forceinline__ uint32_t across(uint32_t v) {
  if constexpr (D >= 16) {
    const Halves r = halves<D>(v);
    return threadIdx.x & D ? r.lower : r.upper;
  } else if constexpr (D == 4) {  // mirrored eight, then mirrored four
    const int m = __builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true);
    return (uint32_t)__builtin_amdgcn_mov_dpp(m, 0x1B, 0xf, 0xf, true);
  } else {
    constexpr int kMove = D == 1 ? 0xB1 : D == 2 ? 0x4E : 0x128;  // the last: eight on, of sixteen
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kMove, 0xf, 0xf, true);
  }
}
template <int D>
__device__ __forceinline__ Key across(Key k) {
  return (Key)across<D>((uint32_t)(k >> 32)) << 32 | across<D>((uint32_t)k);
}
// One step of a sorting network: pairs at distance D, the larger first in groups of RUN lanes and last in every other.
template <int D, int RUN>
__device__ __forceinline__ Key ordered(Key k) {
  const bool upper = threadIdx.x & D, falling = RUN >= kWave || (threadIdx.x & RUN) == 0;
  const Key o = across<D>(k);
  return (k > o) == (upper != falling) ? k : o;
}
template <int RUN>
__device__ __forceinline__ Key merged(Key k) {
  if constexpr (RUN > 32) k = ordered<32, RUN>(k);
  if constexpr (RUN > 16) k = ordered<16, RUN>(k);
  if constexpr (RUN > 8) k = ordered<8, RUN>(k);
  if constexpr (RUN > 4) k = ordered<4, RUN>(k);
  if constexpr (RUN > 2) k = ordered<2, RUN>(k);
  return ordered<1, RUN>(k);
}
__device__ __forceinline__ Key sorted(Key k) {
  return merged<64>(merged<32>(merged<16>(merged<8>(merged<4>(merged<2>(k))))));
}
__device__ __forceinline__ uint32_t mirrored(uint32_t v) {  // lane 63 - l
  return across<32>(across<16>((uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true)));
}
// The larger half of two falling lists, falling.
__device__ __forceinline__ Key joined(Key a, Key b) {
  return merged<64>(max_key(a, (Key)mirrored((uint32_t)(b >> 32)) << 32 | mirrored((uint32_t)b)));
}

__device__ __forceinline__ uint32_t lane_place(uint64_t mask) {  // how many lanes of the mask lie below this one
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// x[i] for an i of each lane's own.
template <int N>
__device__ __forceinline__ float picked(const float (&x)[N], int i) {
  if constexpr (N == 1) {
    return x[0];
  } else {
    float half[(N + 1) / 2];
#pragma unroll
    for (int k = 0; k < (N + 1) / 2; ++k) {
      const float even = x[2 * k], odd = x[2 * k + 1 < N ? 2 * k + 1 : 2 * k];
      half[k] = i & 1 ? odd : even;
    }
    return picked<(N + 1) / 2>(half, i >> 1);
  }
}

// Keys in LDS, one behind the other, of which a wavefront makes a falling list of 64.
__device__ __forceinline__ Key listed(const Key* keys, int n) {
  const int lane = threadIdx.x % kWave;
  Key list = 0;
  for (int k = 0; k < n; k += kWave) {
    const Key next = sorted(k + lane < n ? keys[k + lane] : 0);
    list = k == 0 ? next : joined(list, next);
  }
  return list;
}

// The largest `top` keys of a row, by the wavefronts of a block.  Each has a list of those that it met, one a lane, falling (what
// follows the first `top` may be anything smaller); values that may belong to it wait in its share of `room` until there are 64,
// which are sorted and joined at once.  What is smaller than `least` is not looked at: at least `top` values of the block's first
// step, or of a step of the wavefront, or of its list are larger.
constexpr int kWaiting = 2 * kWave;
template <int NT>
struct TopRoom {
  static constexpr int W = NT / kWave;
  Key waiting[W][kWaiting], together[W * kWaiting], least[W];
  uint32_t most[NT];
  int count[W];
};
template <int NT>
struct TopList {
  static constexpr int W = NT / kWave;
  Key list, least;
  float least_value;
  int top, waiting;
  bool started;
  TopRoom<NT>* room;
  Key* buffer;
  __device__ __forceinline__ TopList(int n, TopRoom<NT>* r)
      : list(0), least(0), least_value(-INFINITY), top(n), waiting(0), started(false), room(r),
        buffer(r->waiting[threadIdx.x / kWave]) {}
  __device__ __forceinline__ void raise(Key k) {
    if (k > least) {
      least = k;
      least_value = key_value(k);
    }
  }
  // The places of N * 64 values of which at least `top` are not smaller: from the highest bit, as far as bf16 has them.
  template <int N>
  __device__ __forceinline__ void raise_to_top_of(const uint32_t (&o)[N]) {
    uint32_t t = 0;
#pragma unroll
    for (int b = 31; b >= 16; --b) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) n += __popcll(__ballot(o[i] >= (t | 1u << b)));
      if (n >= top) t |= 1u << b;
    }
    raise((Key)t << 32);
  }
  __device__ __forceinline__ void join_waiting() {
    wave_sync();
    list = joined(list, listed(buffer, waiting));
    waiting = 0;
    raise(read_lane(list, top - 1));
  }
  __device__ __forceinline__ void wait(Key k, bool in) {
    const uint64_t mask = __ballot(in);
    if (in) buffer[waiting + lane_place(mask)] = k;
    waiting += __popcll(mask);
  }
  // N values a lane, their largest, whether there is any and is(i) each, and index(i) of each.  The same steps for all threads
  // of a block.
  template <int N, class B, class I>
  __device__ __forceinline__ void offer(const float (&x)[N], float most, bool nan, bool there, B&& is, I&& index) {
    if (!started) {
      room->most[threadIdx.x] = there ? (uint32_t)(key_of(nan ? NAN : most, 0) >> 32) : 0;
      __syncthreads();
      uint32_t o[W];
#pragma unroll
      for (int w = 0; w < W; ++w) o[w] = room->most[w * kWave + threadIdx.x % kWave];
      raise_to_top_of(o);
      started = true;
    } else {
      if (!__any(!(most < least_value) || nan)) return;
      const uint32_t o[1] = {there ? (uint32_t)(key_of(nan ? NAN : most, 0) >> 32) : 0};
      raise_to_top_of(o);
    }
    uint32_t may = 0;  // which values may belong to the list
#pragma unroll
    for (int i = 0; i < N; ++i) may |= is(i) && !(x[i] < least_value) ? 1u << i : 0;
    while (__any(may != 0)) {
      const int i = __ffs(may) - 1;
      const Key k = may ? key_of(picked<N>(x, i), index(i)) : 0;
      wait(k, k >= least && k != 0);
      may &= may - 1;
      if (waiting >= kWave) join_waiting();
    }
  }
  // The block's list, in its first wavefront.
  __device__ __forceinline__ Key finish() {
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    if (lane == 0) room->least[w] = least;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < W; ++k) raise(room->least[k]);
    wait(list, lane < top && list >= least && list != 0);  // fewer than 64 wait
    wave_sync();
    Key keep[kWaiting / kWave];
    uint64_t mask[kWaiting / kWave];
    int n = 0;
#pragma unroll
    for (int k = 0; k < kWaiting / kWave; ++k) {
      keep[k] = k * kWave + lane < waiting ? buffer[k * kWave + lane] : 0;
      mask[k] = __ballot(keep[k] >= least && keep[k] != 0);
      n += __popcll(mask[k]);
    }
    if (lane == 0) room->count[w] = n;
    __syncthreads();
    int from = 0, all = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      from += k < w ? room->count[k] : 0;
      all += room->count[k];
    }
#pragma unroll
    for (int k = 0; k < kWaiting / kWave; ++k) {
      if (mask[k] >> lane & 1) room->together[from + lane_place(mask[k])] = keep[k];
      from += __popcll(mask[k]);
    }
    __syncthreads();
    return w == 0 ? listed(room->together, all) : 0;
  }
};
struct NoList {};  // in its place where none is wanted

// ---- what is read and written

// S is 1 at least (the largest logit's own term), or 0: the row is empty.
__device__ __forceinline__ float log_sum(const Sums& s) { return __builtin_amdgcn_logf(s.sum) * kLn2; }

// One lane of the row's writes the numbers, as many lanes as the list is long write that.
__device__ __forceinline__ void put_numbers(const TokenOut& o, const TokenRows& t, int64_t row, const Sums& s, float x) {
  const float logs = log_sum(s);
  const bool empty = s.sum == 0.f;
  if (o.logprob) o.logprob[row] = empty ? -INFINITY : (x - s.most) * t.scale - logs;
  if (o.entropy) {
    const float h = logs - s.tilt * __builtin_amdgcn_rcpf(s.sum) * kLn2;
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
  return {s.most, __builtin_amdgcn_logf(s.sum), t.scale * w, 0.f, -t.scale * w, token, s.sum == 0.f};
}
template <bool ENT, int N>
__device__ __forceinline__ void gradient_of(const RowGradient& g, float (&x)[N], int first, float c) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = fmaf(x[i] - g.most, c, -g.logs2), p = pow2(y);
    if constexpr (ENT) x[i] = p * fmaf(g.b, fmaxf(y, kNothing), g.a);
    else x[i] = p * g.a;
  }
  if ((uint64_t)(g.token - first) < (uint64_t)N) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = first + i == g.token ? x[i] + g.token_part : x[i];
  }
}

// ---- narrow rows: L lanes hold one, N pieces each
//
// Few lanes with many pieces each, as what a row costs in reductions, addresses and outputs is then shared by more rows of a
// wavefront: 200,000 rows of 47 fp32 with a list of three 20 us by 4 lanes of four pieces, 28 by 16 of one.

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
    float v[N][P], most = kLowest;
#pragma unroll
    for (int q = 0; q < N; ++q)
      if ((q + 1) * L * P <= cols) {  // whole pieces in all lanes
#pragma unroll
        for (int i = 0; i < P; ++i) most = fmaxf(most, v[q][i] = x[q * P + i]);
      } else if (q * L * P < cols) {
#pragma unroll
        for (int i = 0; i < P; ++i) most = fmaxf(most, v[q][i] = mine(q, i, cols) ? x[q * P + i] : -INFINITY);
      }
    Sums s{most, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < N; ++q)
      if (q * L * P < cols) add_values<ENT>(s, v[q], most, c);
    join_lanes<ENT, L>(s, c);
    return s;
  }
};

constexpr int kNarrowThreads = 256;
template <int N>
constexpr int kNarrowRows = N > 2 ? 1 : 4 / N;  // that a group of lanes has under way

// Narrow rows with their tokens: f(row, its token, the token's logit, the row's logits).  Rows that are left out are not read.
template <class T, int L, int N, class F>
__device__ __forceinline__ void narrow_rows(const TokenRows& t, F&& f) {
  constexpr int R = kNarrowRows<N>, kSide = kNarrowThreads / L;
  const int lane = threadIdx.x % L;
  for (int64_t row0 = (int64_t)blockIdx.x * kSide * R + threadIdx.x / L; row0 < t.rows; row0 += (int64_t)gridDim.x * kSide * R) {
    int64_t token[R];
    float at[R];
    NarrowRow<T, L, N> r[R];
#pragma unroll
    for (int j = 0; j < R; ++j) token[j] = t.tokens ? t.tokens[min(row0 + j * kSide, t.rows - 1)] : 0;
#pragma unroll
    for (int j = 0; j < R; ++j)
      if ((uint64_t)token[j] < (uint64_t)t.cols) {
        const T* row = (const T*)t.logits + min(row0 + j * kSide, t.rows - 1) * t.ld;
        r[j].load(row, t.cols, lane);
        at[j] = (float)row[token[j]];
      }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (row0 + j * kSide < t.rows) f(row0 + j * kSide, token[j], at[j], r[j]);
  }
}

template <class T, int L, int N>
__global__ __launch_bounds__(kNarrowThreads) void k_token_narrow(TokenRows t, TokenOut o) {
  constexpr int P = 16 / sizeof(T);
  const int lane = threadIdx.x % L;
  narrow_rows<T, L, N>(t, [&](int64_t row, int64_t token, float at, const NarrowRow<T, L, N>& r) {
    if ((uint64_t)token >= (uint64_t)t.cols) {
      if (lane == 0) put_none(o, t, row);
      if (o.top_ids)
        for (int k = lane; k < o.top; k += L) put_top(o, t, row, Sums{0.f, 0.f, 0.f}, 0, k);
      return;
    }
    const Sums s = o.entropy ? r.template sums<true>(t.cols, t.c) : r.template sums<false>(t.cols, t.c);
    if (lane == 0) put_numbers(o, t, row, s, at);
    if (!o.top_ids) return;
    // the largest that is left, `top` times: what is taken becomes 0
    uint32_t left[N * P];
#pragma unroll
    for (int q = 0; q < N; ++q)
#pragma unroll
      for (int i = 0; i < P; ++i)
        left[q * P + i] = r.mine(q, i, t.cols) ? (uint32_t)(key_of(r.x[q * P + i], 0) >> 32) : 0;
    Key mine = 0;  // place k's, in lane k % L
    for (int k = 0; k < o.top; ++k) {
      uint32_t best = 0;
#pragma unroll
      for (int i = 0; i < N * P; ++i) best = max(best, left[i]);
      const uint32_t most = lanes_of<L>(best, [](uint32_t a, uint32_t b) { return max(a, b); });
      uint32_t place = INT_MAX;
#pragma unroll
      for (int q = N - 1; q >= 0; --q)
#pragma unroll
        for (int i = P - 1; i >= 0; --i) place = left[q * P + i] == most ? (uint32_t)(r.first[q] + i) : place;
      place = lanes_of<L>(place, [](uint32_t a, uint32_t b) { return min(a, b); });
#pragma unroll
      for (int q = 0; q < N; ++q)
#pragma unroll
        for (int i = 0; i < P; ++i) left[q * P + i] = r.first[q] + i == (int)place ? 0 : left[q * P + i];
      if (lane == k % L) mine = most == 0 ? 0 : (Key)most << 32 | ~place;
      if (k % L == L - 1 || k == o.top - 1) put_top(o, t, row, s, mine, lane <= k % L ? k / L * L + lane : o.top);
    }
  });
}

template <class T, class TO, int L, int N>
__global__ __launch_bounds__(kNarrowThreads) void k_token_loss_narrow(TokenRows t, const float* __restrict__ weights,
                                                                      float weight, float* __restrict__ logprob, TO* dx,
                                                                      int64_t ld_dx) {
  constexpr int P = 16 / sizeof(T);
  const int lane = threadIdx.x % L;
  narrow_rows<T, L, N>(t, [&](int64_t row, int64_t token, float at, const NarrowRow<T, L, N>& r) {
    RowGradient g{};
    if ((uint64_t)token < (uint64_t)t.cols) {
        const Sums s = r.template sums<false>(t.cols, t.c);
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
      for (int i = 0; i < P; ++i) v[i] = r.x[q * P + i];
      if (!g.zero) gradient_of<false>(g, v, first, t.c);
      else
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = 0.f;
      TO* to = dx + row * ld_dx + first;
      if (t.cols >= P) store_piece<P, TO>(to, v);
      else
#pragma unroll
        for (int i = 0; i < P; ++i)
          if (i < t.cols) to[i] = (TO)v[i];
    }
  });
}

// ---- wide rows: a block has one, or a part of one

// Four pieces of a row at a time by every thread of a block: f(values, first columns of the pieces, how many values of each
// are not the piece's own, whether there are such).  The last piece of the columns [from, to) starts early where it is cut off;
// places without a piece hold -infinity.  The row has a piece's width at least.
template <int U, int NT, class T, class F>
__device__ __forceinline__ void last_step(const T* __restrict__ row, int from, int to, int k, F&& f) {
  constexpr int P = 16 / sizeof(T);
  int first[U], skip[U];
  typename Piece<T, P>::V v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int own = from + (k + u * NT) * P;
    first[u] = min(own, to - P);
    skip[u] = min(own - first[u], P);
    v[u] = *(const typename Piece<T, P>::V*)(row + first[u]);
  }
  float x[U * P];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < P; ++i) x[u * P + i] = i >= skip[u] ? (float)v[u][i] : -INFINITY;
  f(x, first, skip, std::true_type{});
}
template <int NT, class T, class F>
__device__ __forceinline__ void sweep(const T* __restrict__ row, int from, int to, F&& f) {
  constexpr int P = 16 / sizeof(T), U = 4;
  const int whole = (to - from) / P, pieces = (to - from + P - 1) / P;
  int k0 = 0;
  for (; k0 + U * NT <= whole; k0 += U * NT) {
    const int k = k0 + (int)threadIdx.x;
    typename Piece<T, P>::V v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *(const typename Piece<T, P>::V*)(row + from + (k + u * NT) * P);
    float x[U * P];
    int first[U];
    const int skip[U] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      first[u] = from + (k + u * NT) * P;
#pragma unroll
      for (int i = 0; i < P; ++i) x[u * P + i] = (float)v[u][i];
    }
    f(x, first, skip, std::false_type{});
  }
  const int k = k0 + (int)threadIdx.x, left = pieces - k0;
  if (left > 3 * NT) last_step<4, NT>(row, from, to, k, f);
  else if (left > 2 * NT) last_step<3, NT>(row, from, to, k, f);
  else if (left > NT) last_step<2, NT>(row, from, to, k, f);
  else if (left > 0) last_step<1, NT>(row, from, to, k, f);
}

template <int N>
__device__ __forceinline__ float largest(const float (&x)[N]) {
  float most = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) most = fmaxf(most, x[i]);
  return most;
}

template <int N>
__device__ __forceinline__ bool any_nan(const float (&x)[N]) {
  bool is = false;
#pragma unroll
  for (int i = 0; i < N; ++i) is |= x[i] != x[i];
  return is;
}

template <bool ENT, int NT, class T, class LIST>
__device__ __forceinline__ Sums row_sums(const T* __restrict__ row, int from, int to, float c, LIST& top) {
  Sums s{kLowest, 0.f, 0.f};
  sweep<NT>(row, from, to, [&](const auto& x, const auto& first, const auto& skip, auto edge) {
    constexpr int N = sizeof(x) / sizeof(float), P = N / (sizeof(first) / sizeof(int));
    constexpr bool kEdge = decltype(edge)::value;
    const float most = largest(x);
    add_values<ENT>(s, x, most, c);
    if constexpr (!std::is_same_v<LIST, NoList>) {  // a sum with NaN stays one: the largest does not tell of it
      const bool nan = __any(s.sum != s.sum) && any_nan(x);
      top.offer(x, most, nan, !kEdge || skip[0] < P, [&](int i) { return !kEdge || i % P >= skip[i / P]; },
                [&](int i) { return min(first[0] + i / P * NT * P, to - P) + i % P; });
    }
  });
  return s;
}

// Scores of a row by a block, or (splits > 1) the sums and the list of `per` columns of it.  What a list costs is not its values
// but finding them: a bound from the largest value of every thread leaves some 21 of 8192, which one wavefront sorts (48 rows of
// 128,000 bf16 with 20 places 14.7 us; with insertions into lists of all wavefronts 42, with sorts of all slots that hold one 26).
template <class T, int NT, bool ENT, bool TOP>
__global__ __launch_bounds__(NT) void k_token_wide(TokenRows t, TokenOut o, int splits, int per, TokenParts parts) {
  __shared__ Sums part[NT / kWave];
  __shared__ std::conditional_t<TOP, TopRoom<NT>, NoList> room;
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
    const int from = split * per;
    Sums s;
    Key list = 0;
    if constexpr (TOP) {
      TopList<NT> top(o.top, &room);
      s = row_sums<ENT, NT>(x + row * t.ld, from, min(t.cols, from + per), t.c, top);
      list = top.finish();
    } else {
      NoList none;
      s = row_sums<ENT, NT>(x + row * t.ld, from, min(t.cols, from + per), t.c, none);
    }
    join_block<ENT, NT>(s, t.c, part);
    if (splits > 1) {
      if (threadIdx.x == 0) parts.sums[b] = f4{s.most, s.sum, s.tilt, 0.f};
      if (TOP && threadIdx.x < kWave) parts.lists[b * kWave + threadIdx.x] = list;
    } else {
      if (threadIdx.x == 0) put_numbers(o, t, row, s, at);
      if (TOP && threadIdx.x < kWave) put_top(o, t, row, s, list, threadIdx.x);
    }
    __syncthreads();
  }
}

// The parts of a row joined by a block.  Of the lists the keys that are no smaller than the last one of some list; a wavefront
// has those of splits w, w + 16, ...
template <class T, bool TOP>
__global__ __launch_bounds__(TOP ? 1024 : kWave) void k_token_join(TokenRows t, TokenOut o, int splits, TokenParts parts) {
  constexpr int W = TOP ? 16 : 1, M = kWave / W;
  __shared__ Key keys[TOP ? kWave * kWave : 1];
  __shared__ int counts[W];
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  const int64_t row = blockIdx.x;
  const int64_t token = t.tokens ? t.tokens[row] : 0;
  const f4 p = parts.sums[row * splits + min(lane, splits - 1)];
  Key mine[M], least = 0;
  if constexpr (TOP) {
    const Key* lists = parts.lists + row * splits * kWave;
#pragma unroll
    for (int k = 0; k < M; ++k) mine[k] = lists[min(k * W + w, splits - 1) * kWave + lane];
    least = lists[min(lane, splits - 1) * kWave + o.top - 1];
  }
  if ((uint64_t)token >= (uint64_t)t.cols) {
    if (threadIdx.x == 0) put_none(o, t, row);
    if (TOP && w == 0) put_top(o, t, row, Sums{0.f, 0.f, 0.f}, 0, lane);
    return;
  }
  const float at = (float)((const T*)t.logits)[row * t.ld + token];
  Sums s{kLowest, 0.f, 0.f};
  if (lane < splits) s = Sums{p.x, p.y, p.z};
  join_lanes<true, kWave>(s, t.c);
  if (threadIdx.x == 0) put_numbers(o, t, row, s, at);
  if constexpr (TOP) {
    least = max_key(least, across<1>(least));
    least = max_key(least, across<2>(least));
    least = max_key(least, across<4>(least));
    least = max_key(least, across<8>(least));
    least = max_key(least, across<16>(least));
    least = max_key(least, across<32>(least));
    uint64_t mask[M];
    int n = 0;
#pragma unroll
    for (int k = 0; k < M; ++k) {
      mask[k] = __ballot(k * W + w < splits && lane < o.top && mine[k] >= least && mine[k] != 0);
      n += __popcll(mask[k]);
    }
    if (lane == 0) counts[w] = n;
    __syncthreads();
    const int before = counts[lane % W];
    int from = 0, all = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const int c = __builtin_amdgcn_readlane(before, k);
      from += k < w ? c : 0;
      all += c;
    }
#pragma unroll
    for (int k = 0; k < M; ++k) {
      if (mask[k] >> lane & 1) keys[from + lane_place(mask[k])] = mine[k];
      from += __popcll(mask[k]);
    }
    __syncthreads();
    if (w == 0) put_top(o, t, row, s, listed(keys, all), lane);
  }
}

// ---- gradient

// Columns [from, to) of a row's gradient by a block.  Elements are read and written by the same thread: dx may be x.  Written past
// the caches: the loss of 4096 x 128,000 bf16 443 us, through them 471.
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
      gradient_of<ENT>(g, v, first, c);
    }
    store_piece<P, TO, true>(dx + first, v);
  }
  const int rest = from + pieces * P + thread;
  if (rest < to) {
    float v[1] = {g.zero ? 0.f : (float)x[rest]};
    if (!g.zero) gradient_of<ENT>(g, v, rest, c);
    dx[rest] = (TO)v[0];
  }
}

struct Upstream {
  const float *state, *entropy, *d_logprob, *d_entropy;
};

// The last rows first: what the scores read last may still be in the last-level cache (4096 rows of 32,000 bf16, a third of them
// left out, scores and gradient 110.9 us, from the first on 112.0).
constexpr int kGradThreads = 256;
template <class T, class TO, bool ENT, int NT>
__global__ __launch_bounds__(kGradThreads) void k_token_grad(TokenRows t, Upstream u, TO* dx, int64_t ld_dx,
                                                             int splits, int per) {
  constexpr int kSide = kGradThreads / NT;  // rows beside each other in a block
  const int64_t work = t.rows * splits;
  for (int64_t b = (int64_t)blockIdx.x * kSide + threadIdx.x / NT; b < work; b += (int64_t)gridDim.x * kSide) {
    const int64_t back = splits > 1 ? b / splits : b, row = t.rows - 1 - back;
    const int from = splits > 1 ? (int)(b - back * splits) * per : 0;
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

// Log probability and gradient of a row by a block, which reads it a second time from the caches: bound by the memory, that reads
// and writes every logit once.  A row of 256 KB is far from fitting a compute unit's LDS; in registers, all of a compute unit's would
// hold one, and loading and storing would take turns.
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
      NoList none;
      Sums s = row_sums<false, NT>(x, 0, t.cols, t.c, none);
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
static bool with_narrow(int cols, F&& f) {
  constexpr int P = 16 / sizeof(T);
  if (cols <= 4 * P) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
  else if (cols <= 8 * P) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
  else if (cols <= 16 * P) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
  else if (cols <= 64 * P) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
  else return false;
  return true;
}

// How many blocks take a row of few rows, and how many columns each.  Rows of up to two steps of a block are not shared: the second
// launch costs more than it saves.  1 and 64 rows of 128,000 bf16 5.3 and 7.8 us shared by blocks of 512 threads, 10.4 and 12.2
// by one of 1024 each; of 32,000 5.4 and 6.0, against 4.3 and 4.9; no difference from 129 rows of 128,000 on.
static int splits_of(int64_t rows, int cols, int step, int* per) {
  int64_t n = std::min<int64_t>(kTokenParts / std::max<int64_t>(rows, 1), kWave);
  n = std::max<int64_t>(1, std::min<int64_t>(n, (cols + step / 2) / step));
  if (n <= 2) n = 1;
  *per = (int)((cols + n - 1) / n + 7) / 8 * 8;
  return (cols + *per - 1) / *per;
}

template <class T, int NT, bool TOP>
static void launch_wide(const TokenRows& t, const TokenOut& o, const TokenParts& parts, hipStream_t st) {
  int per;
  const int splits = splits_of(t.rows, t.cols, NT * 64 / (int)sizeof(T), &per), blocks = grid_of(t.rows * splits);
  if (o.entropy) k_token_wide<T, NT, true, TOP><<<blocks, NT, 0, st>>>(t, o, splits, per, parts);
  else k_token_wide<T, NT, false, TOP><<<blocks, NT, 0, st>>>(t, o, splits, per, parts);
  if (splits > 1) k_token_join<T, TOP><<<(int)t.rows, TOP ? 1024 : kWave, 0, st>>>(t, o, splits, parts);
}

void launch_token_scores(const TokenRows& t, int type, const TokenOut& o, const TokenParts& parts, hipStream_t st) {
  with_type(type, [&](auto ti) {
    typedef decltype(ti) T;
    // A long list of few rows is quicker made by blocks: a narrow row's takes 0.6 us for each place, whatever the rows, a block's
    // 3.5 ns for each row and 8 us.  20 rows of 100 bf16 with 16 and 64 places 13.7 and 39.6 us narrow, 7.8 and 8.6 by blocks; 100,000
    // rows 46 and 131 against 350 and more.
    const bool by_blocks = o.top_ids != nullptr && t.rows <= 160 * (o.top - 8) && t.cols * sizeof(T) >= 16;
    const bool narrow = !by_blocks && with_narrow<T>(t.cols, [&](auto l, auto n) {
      constexpr int L = decltype(l)::value, N = decltype(n)::value, kSide = kNarrowThreads / L * kNarrowRows<N>;
      k_token_narrow<T, L, N><<<grid_of((t.rows + kSide - 1) / kSide), kNarrowThreads, 0, st>>>(t, o);
    });
    if (narrow) return;
    // Threads of a block by the pieces of a row, of which a thread has four under way.  60M logits in all, us by 64 / 128 / 256 / 512
    // threads: rows of 704 bf16 (88 pieces) 44 / 62 / 115, 1160 fp32 (290) 42 / 49 / 73, 3500 bf16 (438) 26 / 29 / 36, 5000 bf16
    // (625) - / 27 / 33 / 50, 16,000 (2000) - / - / 28 / 27; 4096 rows of 32,000 - / - / 38 / 33.
    // Lists: 20,000 rows of 2500 with 20 places 43 / 66 / 116, 3000 of 8000 21 / 21 / 25; 500 of 32,000 with 8 31 / 23 / 15.
    const int64_t pieces = t.cols * (int64_t)sizeof(T) / 16;
    if (o.top_ids) {
      if (pieces <= 1024 && t.rows > 512) launch_wide<T, 64, true>(t, o, parts, st);
      else launch_wide<T, 256, true>(t, o, parts, st);
    } else if (pieces <= 512) {
      launch_wide<T, 64, false>(t, o, parts, st);
    } else if (pieces <= 1024) {
      launch_wide<T, 128, false>(t, o, parts, st);
    } else if (pieces <= 2048) {
      launch_wide<T, 256, false>(t, o, parts, st);
    } else {
      launch_wide<T, 512, false>(t, o, parts, st);
    }
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
    // Pieces of a row by its lanes: 150,000 rows of 1037 bf16 135 us by 64 lanes, 231 by 256; 30,000 of 4000 90 and 81, 20,000
    // of 2999 fp32 112 and 85.
    constexpr int P = 16 / (sizeof(T) > sizeof(TO) ? sizeof(T) : sizeof(TO));
    if (t.cols <= 16 * P) return go(ent, std::integral_constant<int, 16>{}, 1, t.cols);
    if (t.cols <= 260 * P) return go(ent, std::integral_constant<int, 64>{}, 1, t.cols);
    int per = 32768;  // columns of a block: as many as leave enough blocks
    while (per > 8192 && t.rows * ((t.cols + per - 1) / per) < 2048) per /= 2;
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
      const bool narrow = with_narrow<T>(t.cols, [&](auto l, auto n) {
        constexpr int L = decltype(l)::value, N = decltype(n)::value, kSide = kNarrowThreads / L * kNarrowRows<N>;
        k_token_loss_narrow<T, TO, L, N><<<grid_of((t.rows + kSide - 1) / kSide), kNarrowThreads, 0, st>>>(
            t, weights, weight, logprob, to, dx.ld);
      });
      if (narrow) return;
      // 60M logits in all, us by 64 / 128 / 256 / 512 / 1024 threads: rows of 704 bf16 (88 pieces) 61 / 88 / 137, 3500 (438) 58 / 49 /
      // 52, 5000 (625) - / - / 50 / 65 / 99, 16,000 (2000) - / - / 57 / 49 / 54, 32,000 (4000) - / - / 60 / 57 / 52; 4096 rows of
      // 128,000 - / - / 605 / 486 / 442: of more rows at once the caches hold less until they are read again.
      const int64_t pieces = t.cols * (int64_t)sizeof(T) / 16;
      auto go = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        k_token_loss<T, TO, NT><<<grid_of(t.rows), NT, 0, st>>>(t, weights, weight, logprob, to, dx.ld);
      };
      if (pieces <= 256) go(std::integral_constant<int, 64>{});
      else if (pieces <= 512) go(std::integral_constant<int, 128>{});
      else if (pieces <= 1024) go(std::integral_constant<int, 256>{});
      else if (pieces <= 2048) go(std::integral_constant<int, 512>{});
      else go(std::integral_constant<int, 1024>{});
    });
  });
}

}  // namespace ttemb
