// Position bias of attention: a table [buckets, heads] looked up by the distance of a key from a query, alone or added to
// scores, and its gradient, sums of the scores' gradients over all places of a bucket.
//
// A distance is j - i + o with one o for a sequence, so a head's bias has one value for every diagonal.  Bound by the memory.
// Measured (one MI355X, us a call among others): 16 x 4096 x 4096 bf16 written 86.5 (6.2 TB/s; a fill of that size into three
// buffers in turn 78), 7 x 12 x 509 x 1021 fp32 added 68.6 (5.1 TB/s read and written), 64 x 16 x 1 x 4097 bf16 8.8 (the call);
// sums of 8 x 16 x 2048 x 2048 bf16 206 (5.2 TB/s), of 3 x 12 x 129 x 515 fp32 18.8 (three launches).
#include <algorithm>
#include <type_traits>

#include "tt_emb_internal.h"

namespace ttemb {

__device__ __forceinline__ int64_t offset_of(const tt_emb_distances& d, int b) {
  constexpr int64_t kMost = int64_t(1) << 40;
  int64_t o = d.offset;
  if (d.offsets) {
    const int64_t p = d.offsets[b];
    if (__builtin_add_overflow(o, p, &o)) o = p < 0 ? -kMost : kMost;
  }
  return min(max(o, -kMost), kMost);
}
__device__ __forceinline__ int cut(int64_t distance, int span) {
  return (int)min(max(distance, -(int64_t)span), (int64_t)span);
}
__device__ __forceinline__ float any_value(const tt_emb_matrix& m, int64_t at) {
  if (m.type == TT_EMB_BF16) return (float)((const __bf16*)m.data)[at];
  if (m.type == TT_EMB_FP16) return (float)((const _Float16*)m.data)[at];
  return ((const float*)m.data)[at];
}

// a / b for a >= 0, b > 0: in 64 bits a division takes a microsecond
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (uint64_t)(a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// ---- bias

// The bias of distances in one head.
struct Values {
  tt_emb_matrix table;
  const int32_t* bucket_of;
  int span, h;
  float fill;
  __device__ __forceinline__ int bucket(int64_t distance) const { return bucket_of[cut(distance, span) + span]; }
  __device__ __forceinline__ float of(int u) const {
    return (uint32_t)u < (uint32_t)table.rows ? any_value(table, u * table.ld + h) : fill;
  }
  // Of N distances, `step` apart, all buckets before all values.
  template <int N>
  __device__ __forceinline__ void get(int64_t first, int step, float (&v)[N]) const {
    int u[N];
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = bucket(first + i * step);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = of(u[i]);
  }
};
__device__ __forceinline__ float added(float x, float bias) { return isinf(bias) ? bias : x + bias; }

constexpr int kBiasThreads = 256, kBiasAhead = 4;  // rows of a tile that a thread has under way
template <class TI, class TO, bool ADD>
constexpr int kBiasPiece = 16 / (ADD && sizeof(TI) > sizeof(TO) ? sizeof(TI) : sizeof(TO));

// Few queries: a block takes a row, a thread looks up its pieces' values; those beyond the span have one for all.  64 x 16 x 1 x
// 4097 bf16 7.7 us, with tiles 15.
constexpr int kFewQueries = 4;
template <class TI, class TO, bool ADD>
__global__ __launch_bounds__(kBiasThreads) void k_bias_few(tt_emb_matrix table, tt_emb_distances dist, float fill,
                                                           tt_emb_pairs in, tt_emb_pairs out, int64_t count) {
  constexpr int P = kBiasPiece<TI, TO, ADD>;
  for (int64_t row = blockIdx.x; row < count; row += gridDim.x) {
    const int64_t plane = quotient(row, out.queries);
    const int i = (int)(row - plane * out.queries), b = (int)quotient(plane, out.heads), h = (int)(plane - (int64_t)b * out.heads);
    const int64_t first = offset_of(dist, b) - i;  // distance of the first key
    const Values values{table, dist.bucket_of, dist.span, h, fill};
    const float low = values.of(values.bucket(-dist.span)), high = values.of(values.bucket(dist.span));
    const TI* from = (const TI*)in.data + (ADD ? b * in.batch_ld + h * in.head_ld + i * in.query_ld : 0);
    TO* to = (TO*)out.data + b * out.batch_ld + h * out.head_ld + i * out.query_ld;
    const int keys = (int)out.keys;
    for (int c = (int)threadIdx.x * P; c < keys; c += kBiasThreads * P) {
      if (c + P > keys) {  // cut off
        for (int j = c; j < keys; ++j) {
          float y = values.of(values.bucket(first + j));
          if constexpr (ADD) y = added((float)from[j], y);
          to[j] = (TO)y;
        }
        continue;
      }
      float x[P], y[P];
      if constexpr (ADD) load_piece<P, TI>(from + c, x);
      const bool before = first + c + P - 1 <= -dist.span, behind = first + c >= dist.span;
      if (before || behind) {
#pragma unroll
        for (int k = 0; k < P; ++k) y[k] = before ? low : high;
      } else {
        values.get(first + c, 1, y);
      }
      if constexpr (ADD) {
#pragma unroll
        for (int k = 0; k < P; ++k) y[k] = added(x[k], y[k]);
      }
      store_piece<P, TO, ADD>(to + c, y);
    }
  }
}

struct BiasTiles {
  int rows, cols;  // of a tile
  int down, across;
  int64_t count;
  int line;        // places of a line: rows + cols and some more, a multiple of 8
  bool in_place;
};

// A block takes a tile of one head, whose pieces its threads take in turn, row by row.  Its diagonals' values come first, four
// copies of the line, each a place further, so that any row finds its values in 16-byte words of one of them; a tile beyond the
// span has one value.  EVEN: all rows of all tiles are of whole pieces, and a block's threads take whole rows at once.  Where a
// thread takes two words of them, those of even and odd number lie apart, so that the threads of a wavefront read side by side.  A
// row's last piece starts early where it is cut off, and holds some of its neighbour's places.
template <class TI, class TO, bool ADD, bool EVEN>
__global__ __launch_bounds__(kBiasThreads) void k_bias_tiles(tt_emb_matrix table, tt_emb_distances dist, float fill,
                                                             tt_emb_pairs in, tt_emb_pairs out, BiasTiles tl) {
  extern __shared__ __attribute__((aligned(16))) float lines[];
  constexpr int P = kBiasPiece<TI, TO, ADD>, R = kBiasAhead, kAhead = 4;
  typedef typename Piece<TI, P>::V V;
  auto word = [&](int copy, int w) {  // where the word's four values are
    return copy * tl.line + (P == 8 ? (w & 1) * (tl.line / 2) + w / 2 * 4 : w * 4);
  };
  for (int64_t tile = blockIdx.x; tile < tl.count; tile += gridDim.x) {
    const int64_t strip = quotient(tile, tl.across), plane = quotient(strip, tl.down);
    const int j0 = (int)(tile - strip * tl.across) * tl.cols, i0 = (int)(strip - plane * tl.down) * tl.rows;
    const int b = (int)quotient(plane, out.heads), h = (int)(plane - (int64_t)b * out.heads);
    const int rows = (int)min((int64_t)tl.rows, out.queries - i0), cols = (int)min((int64_t)tl.cols, out.keys - j0);
    const int64_t first = offset_of(dist, b) + j0 - i0 - (rows - 1);  // distance of the first diagonal
    const Values values{table, dist.bucket_of, dist.span, h, fill};
    const TI* from = (const TI*)in.data + (ADD ? b * in.batch_ld + h * in.head_ld + i0 * in.query_ld + j0 : 0);
    TO* to = (TO*)out.data + b * out.batch_ld + h * out.head_ld + i0 * out.query_ld + j0;
    const uint32_t pieces = (uint32_t)(cols + P - 1) / P, down = kBiasThreads / pieces, right = kBiasThreads - down * pieces;
    int row = (int)(threadIdx.x / pieces), piece = (int)(threadIdx.x - row * pieces);
    struct Place {
      int r, c, own;  // row, first column, and the first that is the piece's own
    };
    auto take = [&](Place(&p)[R]) {  // the thread's next pieces
#pragma unroll
      for (int k = 0; k < R; ++k) {
        p[k] = Place{row, EVEN ? piece * P : max(min(piece * P, cols - P), 0), piece * P};
        row += (int)down;
        if constexpr (!EVEN) {
          piece += (int)right;
          row += piece >= (int)pieces;
          piece -= piece >= (int)pieces ? (int)pieces : 0;
        }
      }
    };
    const bool wide = EVEN || cols >= P;
    auto load = [&](const Place(&p)[R], V(&v)[R]) {
      if constexpr (ADD)
        if (wide) {
#pragma unroll
          for (int k = 0; k < R; ++k)
            if (p[k].r < rows) v[k] = *(const V*)(from + p[k].r * in.query_ld + p[k].c);
        }
    };
    Place p[R], after[R];
    V v[R], next[R];
    take(p);
    load(p, v);
    const bool one = first >= dist.span || first + rows + cols - 2 <= -dist.span;
    float all = 0.f;
    if (one) {
      all = values.of(values.bucket(first));
    } else {
      for (int x0 = threadIdx.x; x0 < rows + cols - 1; x0 += kAhead * kBiasThreads) {
        float w[kAhead];
        values.get(first + x0, kBiasThreads, w);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int x = x0 + k * kBiasThreads;
          if (x >= rows + cols - 1) continue;
#pragma unroll
          for (int s = 0; s < 4; ++s)
            if (x >= s) lines[word(s, (x - s) / 4) + (x - s) % 4] = w[k];
        }
      }
      __syncthreads();
    }
    while (p[0].r < rows) {
      take(after);
      load(after, next);
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (p[k].r >= rows) continue;
        const int a = p[k].c - p[k].r + rows - 1;  // the piece's first diagonal
        TO* at = to + p[k].r * out.query_ld + p[k].c;
        if (!wide) {  // a row shorter than a piece
#pragma unroll
          for (int i = 0; i < P; ++i) {
            if (i >= cols) continue;
            float y = one ? all : lines[word(0, (a + i) / 4) + (a + i) % 4];
            if constexpr (ADD) y = added((float)from[p[k].r * in.query_ld + i], y);
            at[i] = (TO)y;
          }
          continue;
        }
        float y[P];
        if (one) {
#pragma unroll
          for (int i = 0; i < P; ++i) y[i] = all;
        } else {
#pragma unroll
          for (int i = 0; i < P; i += 4) {
            const f4 w = *(const f4*)&lines[word(a % 4, a / 4 + i / 4)];
#pragma unroll
            for (int n = 0; n < 4; ++n) y[i + n] = w[n];
          }
        }
        if constexpr (ADD) {
#pragma unroll
          for (int i = 0; i < P; ++i) y[i] = added((float)v[k][i], y[i]);
          if (tl.in_place && p[k].own != p[k].c) {  // what it read of its neighbour's may have the bias already
#pragma unroll
            for (int i = 0; i < P; ++i)
              if (p[k].c + i >= p[k].own) at[i] = (TO)y[i];
            continue;
          }
        }
        store_piece<P, TO, true>(at, y);
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        p[k] = after[k];
        if constexpr (ADD) v[k] = next[k];
      }
    }
    if (!one) __syncthreads();
  }
}

// ---- sums of buckets

// The diagonals d = j - i of rows [i0, i1) that are told apart: [first, last], where first stands for all before it, too, and
// last for all behind.
struct Span {
  int first, last;
};
__device__ __forceinline__ Span span_of(int i0, int i1, int keys, int64_t offset, int span) {
  const int64_t low = 1 - i1, high = keys - 1 - i0;
  return {(int)min(max(-(int64_t)span - offset, low), high), (int)max(min((int64_t)span - offset, high), low)};
}

constexpr int kSumThreads = 256, kSumWaves = kSumThreads / kWave;
constexpr int kSumAhead = 4;  // rows that a wavefront has under way

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) v += __shfl_xor(v, d);
  return v;
}

// What a part sums: rows [i0, i1) of sequences [b0, b1) in head h.
struct PartPlace {
  int h, b0, b1, i0, i1;
  __device__ __forceinline__ PartPlace(const SumPlan& p, const tt_emb_pairs& g, int64_t part) {
    const int64_t plane = quotient(part, p.chunks);
    const int chunk = (int)(part - plane * p.chunks);
    h = (int)quotient(plane, p.groups);
    b0 = (int)(plane - (int64_t)h * p.groups) * p.group;
    b1 = min(b0 + p.group, g.batch);
    i0 = chunk * p.rows;
    i1 = (int)min((int64_t)i0 + p.rows, g.queries);
  }
};

// The sums of all before and behind, of a block's wavefronts, to the ends of its part.
__device__ __forceinline__ void put_ends(float before, float behind, const Span& d, float* __restrict__ out) {
  __shared__ float ends[kSumWaves][2];
  before = wave_sum(before);
  behind = wave_sum(behind);
  if (threadIdx.x % kWave == 0) {
    ends[threadIdx.x / kWave][0] = before;
    ends[threadIdx.x / kWave][1] = behind;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float a = 0.f, z = 0.f;
    for (int k = 0; k < kSumWaves; ++k) {
      a += ends[k][0];
      z += ends[k][1];
    }
    if (d.first == d.last) {
      out[0] = a + z;
    } else {
      out[0] = a;
      out[d.last - d.first] = z;
    }
  }
  __syncthreads();
}

// Short rows: a thread has a diagonal, which holds no more values than a row.  Bound by the requests to the caches, each of
// which brings 64 rows' lines: up to 64 keys, and to 512 where a part has few rows.  Against bands, us: 34 x 9 x 3022 x 40 bf16 66 / 165,
// x 66 184 / 182 (503 rows a part), 16 x 9 x 3022 x 128 134 / 104 (216), x 1022 x 100 fp32 33 / 41 (73), 8 x 16 x 1000 x 256 bf16
// 38 / 45 (63), x 200 x 500 19 / 23 (25).
constexpr int kShortKeys = 64, kShortRow = 512, kShortRows = 128;
template <class T>
__global__ __launch_bounds__(kSumThreads) void k_bias_sums_short(tt_emb_pairs g, tt_emb_distances dist, SumPlan p,
                                                                 float* __restrict__ parts, PartReach* __restrict__ reach) {
  constexpr int kAhead = 4;
  for (int64_t part = blockIdx.x; part < p.parts; part += gridDim.x) {
    const PartPlace t(p, g, part);
    const int keys = (int)g.keys;
    const int64_t offset = offset_of(dist, t.b0);
    const Span d = span_of(t.i0, t.i1, keys, offset, dist.span);
    float* out = parts + part * p.width;
    if (threadIdx.x == 0) reach[part] = PartReach{cut(d.first + offset, dist.span), cut(d.last + offset, dist.span)};
    float before = 0.f, behind = 0.f;
    for (int x = 1 - t.i1 + (int)threadIdx.x; x < keys - t.i0; x += kSumThreads) {
      const int from = max(t.i0, -x), to = min(t.i1, keys - x);
      float sum = 0.f;
      for (int b = t.b0; b < t.b1; ++b) {
        const T* at = (const T*)g.data + b * g.batch_ld + t.h * g.head_ld + x;
        for (int i = from; i < to; i += kAhead) {
          float v[kAhead];
#pragma unroll
          for (int n = 0; n < kAhead; ++n) v[n] = (float)at[min(i + n, to - 1) * (g.query_ld + 1)];
#pragma unroll
          for (int n = 0; n < kAhead; ++n) sum += i + n < to ? v[n] : 0.f;
        }
      }
      if (x <= d.first) before += sum;
      else if (x >= d.last) behind += sum;
      else out[x - d.first] = sum;
    }
    put_ends(before, behind, d, out);
  }
}

// Where a gradient's memory starts and ends: pieces may reach over a row's ends, but not over these.
template <class T>
struct Extent {
  const T *low, *high;
  __device__ __forceinline__ explicit Extent(const tt_emb_pairs& g) : low((const T*)g.data) {
    high = low + (g.batch - 1) * g.batch_ld + (g.heads - 1) * g.head_ld + (g.queries - 1) * g.query_ld + g.keys;
  }
};

// Groups [from, to) of 64 pieces in R rows, `p` in this lane's of the first.
template <int R, class T>
__device__ __forceinline__ float groups_sum(const T* p, int64_t ld, int from, int to) {
  constexpr int P = 16 / sizeof(T), U = 2;
  typedef typename Piece<T, P>::V V;
  float sum = 0.f;
  auto some = [&](auto count, int q) {
    constexpr int N = decltype(count)::value;
    V v[N][R];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int n = 0; n < N; ++n) v[n][r] = *(const V*)(p + r * ld + (q + n) * kWave * P);
    float s[N * R];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        s[n * R + r] = (float)v[n][r][0];
#pragma unroll
        for (int k = 1; k < P; ++k) s[n * R + r] += (float)v[n][r][k];
      }
#pragma unroll
    for (int n = 1; n < N * R; ++n) s[0] += s[n];
    sum += s[0];
  };
  for (; from + U <= to; from += U) some(std::integral_constant<int, U>{}, from);
  for (; from < to; ++from) some(std::integral_constant<int, 1>{}, from);
  return sum;
}

// A block sums the diagonals of some rows of one head and of p.group sequences, a lane B of them at a time: its accumulators
// stay, the row's place moves by a value from one row to the next, so that loads need not be aligned, and nothing is exchanged
// between lanes.  All before the first and behind the last diagonal are summed apart, row by row.  Bound by the memory where most
// places are: 8 x 16 x 2048 x 2048 bf16 with 255 diagonals apart 194 us (5.5 TB/s).  A call, with the joins: 203, with the band in a
// pass of its own 226, with a choice for every place 355.
template <class T, int B>
__global__ __launch_bounds__(kSumThreads) void k_bias_sums(tt_emb_pairs g, tt_emb_distances dist, int buckets, SumPlan p,
                                                           float* __restrict__ parts, PartReach* __restrict__ reach) {
  typedef typename Piece<T, 16 / sizeof(T)>::V VF;
  typedef typename Piece<T, B>::V VB;
  constexpr int P = 16 / sizeof(T), R = kSumAhead;
  __shared__ float sums[kSumWaves][kWave * B];
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const Extent<T> all(g);
  for (int64_t part = blockIdx.x; part < p.parts; part += gridDim.x) {
    const PartPlace t(p, g, part);
    const int h = t.h, b0 = t.b0, b1 = t.b1, i0 = t.i0, i1 = t.i1;
    const int keys = (int)g.keys;
    const int64_t offset = offset_of(dist, b0);
    const Span d = span_of(i0, i1, keys, offset, dist.span);
    float* out = parts + part * p.width;
    auto wanted = [&](int diagonal) {
      return (uint32_t)dist.bucket_of[cut(diagonal + offset, dist.span) + dist.span] < (uint32_t)buckets;
    };
    const bool low = wanted(d.first), high = wanted(d.last);
    float before = 0.f, behind = 0.f;
    if (threadIdx.x == 0) reach[part] = PartReach{cut(d.first + offset, dist.span), cut(d.last + offset, dist.span)};
    // what lies between: R rows of the band of 64 B diagonals from x0 on
    const int start = d.first + 1, end = d.last;
    float acc[B] = {};
    auto add_rows = [&](const T* rows, int i, int x0) {
      const int x = x0 + lane * B, to = (int)min((int64_t)i1, (int64_t)keys - x0);  // this lane's first diagonal
      if (i >= to || i + R + x0 + kWave * B <= 0) return;  // the band lies outside of these rows
      const T* at = rows + i * g.query_ld + (i + x);  // a row on is a column on
      VB v[R];
      if (i + x0 >= 0 && i + R - 1 + x0 + kWave * B <= keys && i + R <= to) {  // within all rows, for all lanes
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = *(const VB*)(at + r * (g.query_ld + 1));
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int k = 0; k < B; ++k) acc[k] += (float)v[r][k];
        return;
      }
      const T* first = rows + i * g.query_ld + (i + x0);
      // whether pieces that reach over the rows' ends stay within the memory, for all lanes
      const bool safe = first >= all.low && first + (R - 1) * (g.query_ld + 1) + kWave * B <= all.high;
      bool cut_off = false;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int j = i + r + x;
        const T* q = at + r * (g.query_ld + 1);
        const bool some = i + r < to && j + B > 0 && j < keys, whole = some && (safe || (q >= all.low && q + B <= all.high));
        v[r] = VB{};
        if (whole) v[r] = *(const VB*)q;
        cut_off = cut_off || (some && !whole);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int j = i + r + x;
#pragma unroll
        for (int k = 0; k < B; ++k) acc[k] += (uint32_t)(j + k) < (uint32_t)keys ? (float)v[r][k] : 0.f;
      }
      if (__any(cut_off)) {  // at the memory's ends: singly
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int j = i + r + x;
          const T* q = at + r * (g.query_ld + 1);
          if (i + r >= to || (q >= all.low && q + B <= all.high)) continue;
#pragma unroll
          for (int k = 0; k < B; ++k)
            if ((uint32_t)(j + k) < (uint32_t)keys) acc[k] += (float)q[k];
        }
      }
    };
    const bool one_band = end > start && end - start <= kWave * B;  // taken beside the rest, whose rows are in the caches then
    // Columns [0, i + until) of row i are before, [i + since, keys) behind.  R rows at a time: groups of 64 pieces that are so
    // in all of them are only added up; of the others the wanted places are, and those with none are left out.
    const int until = d.first + 1, since = max(d.last, d.first + 1), whole = keys / (kWave * P);
    for (int b = b0; b < b1; ++b) {
      const T* rows = (const T*)g.data + b * g.batch_ld + h * g.head_ld;
      for (int i = i0 + w * R; i < i1; i += kSumWaves * R) {
        const T* at = rows + i * g.query_ld + lane * P;
        const bool full = i + R <= i1;
        const int g0 = full && low ? min(max(i + until, 0) / (kWave * P), whole) : 0;
        const int g1 = full && high ? max(min((max(i + R - 1 + since, 0) + kWave * P - 1) / (kWave * P), whole), g0) : whole;
        before += groups_sum<R>(at, g.query_ld, 0, g0);
        behind += groups_sum<R>(at, g.query_ld, g1, whole);
        for (int q = g0 < g1 ? g0 : whole; q * kWave * P < keys; q = q + 1 == g1 ? whole : q + 1) {
          const int c0 = q * kWave * P, c = c0 + lane * P, edge = keys - c;
          // places [0, u) of row i are before, u + 1 of the next one's
          const int u = low ? i + until - c0 : -R, s = high ? i + since - c0 : kWave * P + R;
          if (u + R - 1 <= 0 && s >= min(kWave * P, keys - c0)) continue;
          VF v[R];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const T* p = at + r * g.query_ld + c0;
            v[r] = VF{};
            if (i + r >= i1 || edge <= 0) continue;
            if (q < whole || p + P <= all.high) {
              v[r] = *(const VF*)p;
            } else {
#pragma unroll
              for (int k = 0; k < P; ++k)
                if (k < edge) v[r][k] = p[k];
            }
          }
          if (q >= whole) {  // the row's end: what lies behind it counts as 0
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int k = 0; k < P; ++k) v[r][k] = k < edge ? v[r][k] : (T)0.f;
          }
          const int lu = u - lane * P, ls = s - lane * P;
          if (u + R - 1 > 0) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int k = 0; k < P; ++k) before += k - r < lu ? (float)v[r][k] : 0.f;
          }
          if (s < kWave * P) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int k = 0; k < P; ++k) behind += k - r >= ls ? (float)v[r][k] : 0.f;
          }
        }
        if (one_band) add_rows(rows, i, start);
      }
    }
    put_ends(before, behind, d, out);
    for (int x0 = start; x0 < end; x0 += kWave * B) {
      if (!one_band) {
#pragma unroll
        for (int k = 0; k < B; ++k) acc[k] = 0.f;
        for (int b = b0; b < b1; ++b) {
          const T* rows = (const T*)g.data + b * g.batch_ld + h * g.head_ld;
          // rows that meet the band at all
          const int from = max(i0, -(x0 + kWave * B - 1)), to = (int)min((int64_t)i1, (int64_t)keys - x0);
          for (int i = from + w * R; i < to; i += kSumWaves * R) add_rows(rows, i, x0);
        }
      }
#pragma unroll
      for (int k = 0; k < B; ++k) sums[w][lane * B + k] = acc[k];
      __syncthreads();
      for (int k = threadIdx.x; k < kWave * B && x0 + k < end; k += kSumThreads) {
        float s = 0.f;
#pragma unroll
        for (int n = 0; n < kSumWaves; ++n) s += sums[n][k];
        out[x0 + k - d.first] = s;
      }
      __syncthreads();
    }
  }
}

// total[head][distance - low]: all parts of a head and distance, in fp64, of `count` distances from `low` on.  A block has 64 of
// them, a wavefront some of the parts; those that a part tells apart, or stands for, are one behind the other in it.
// reached: which blocks' distances any part has, for any head.
constexpr int kJoinAhead = 8;
template <int W>
__global__ __launch_bounds__(W * kWave) void k_bias_join(int heads, int low, int count, SumPlan p,
                                                         const float* __restrict__ parts, const PartReach* __restrict__ reach,
                                                         double* __restrict__ total, int* __restrict__ reached) {
  __shared__ double sums[W][kWave];
  __shared__ int any[W];
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int per_head = p.groups * p.chunks, tiles = (count + kWave - 1) / kWave;
  for (int64_t tile = blockIdx.x; tile < (int64_t)tiles * heads; tile += gridDim.x) {
    const int h = (int)quotient(tile, tiles), t = (int)(tile - (int64_t)h * tiles), r = t * kWave + lane, distance = low + r;
    double sum = 0.0;
    bool has = false;
    for (int k0 = w; k0 < per_head; k0 += W * kJoinAhead) {
      PartReach a[kJoinAhead];
      float v[kJoinAhead];
#pragma unroll
      for (int n = 0; n < kJoinAhead; ++n) a[n] = reach[(int64_t)h * per_head + min(k0 + n * W, per_head - 1)];
#pragma unroll
      for (int n = 0; n < kJoinAhead; ++n) {
        const int k = k0 + n * W;
        v[n] = 0.f;
        if (k < per_head && r < count && distance >= a[n].first && distance <= a[n].last) {
          v[n] = parts[((int64_t)h * per_head + k) * p.width + (distance - a[n].first)];
          has = true;
        }
      }
#pragma unroll
      for (int n = 0; n < kJoinAhead; ++n) sum += (double)v[n];
    }
    sums[w][lane] = sum;
    const int some = __any(has);
    if (lane == 0) any[w] = some;
    __syncthreads();
    if (w == 0) {
      sum = 0.0;
      int all = 0;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        sum += sums[k][lane];
        all |= any[k];
      }
      if (all && r < count) total[(int64_t)h * count + r] = sum;
      if (h == 0 && lane == 0) reached[t] = all;
    }
    __syncthreads();
  }
}

// A sum in fp64 as a value of a table, rounded once: on the way to 16 bits fp32 holds it cut off towards zero, its last bit set
// where something was cut off, so that no such value lies halfway between two of 16 bits.
template <class T>
__device__ __forceinline__ T rounded_once(double x) {
  float f = (float)x;
  if constexpr (sizeof(T) < sizeof(float)) {
    const double back = (double)f;
    if (back != x && x == x) {
      const uint32_t b = __builtin_bit_cast(uint32_t, f);
      f = __builtin_bit_cast(float, (fabs(back) > fabs(x) ? b - 1 : b) | 1u);
    }
  }
  return (T)f;
}

// A block adds up the distances of one bucket in all heads: W * 64 * U at a time, first which they are, in order, then their
// totals, of few by a thread for each head, of more by a wavefront.  Every bucket looks at all distances, and one block has all
// of the bucket that holds what is far: with long spans and offsets the joins and this kernel are most of a call (10 x 30 x 11 x 1211
// fp16 with a span of 17,004: sums 13 us, joins 32, 16 buckets 21), and 65,537 buckets of a distance each take 2.8 ms.
constexpr int kFewDistances = 16;
template <class TO, int W, int U>
__global__ __launch_bounds__(W * kWave) void k_bias_buckets(int heads, const int32_t* __restrict__ bucket_of, int count,
                                                            const double* __restrict__ total, const int* __restrict__ reached,
                                                            TO* __restrict__ out, int64_t ld, int buckets, bool add) {
  constexpr int kThreads = W * kWave, kAhead = 4;
  __shared__ int found[U * kThreads], counts[kWave];
  __shared__ double sums[kThreads];  // of heads h0, h0 + 1, ...
  static_assert(U * W <= kWave, "a count for each lane");
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  for (int64_t at_u = blockIdx.x; at_u < buckets; at_u += gridDim.x) {  // in 64 bits: the step may lead beyond 2^31
    const int u = (int)at_u;
    for (int h0 = 0; h0 < heads; h0 += kThreads) {
      sums[threadIdx.x] = 0.0;
      for (int r0 = 0; r0 < count; r0 += U * kThreads) {
        uint64_t mask[U];
#pragma unroll
        for (int n = 0; n < U; ++n) {
          const int r = r0 + n * kThreads + (int)threadIdx.x, at = min(r, count - 1);
          mask[n] = __ballot((int)(bucket_of[at] == u) & (int)(reached[at / kWave] != 0) & (int)(r < count));
          if (lane == 0) counts[n * W + w] = __popcll(mask[n]);
        }
        __syncthreads();
        const int mine = lane < U * W ? counts[lane] : 0;
        int all = mine;  // of this place and all before it
#pragma unroll
        for (int k = 1; k < kWave; k *= 2) {
          const int before = __shfl_up(all, k);
          all += lane >= k ? before : 0;
        }
#pragma unroll
        for (int n = 0; n < U; ++n) {
          const int from = __builtin_amdgcn_readlane(all - mine, n * W + w);
          if (mask[n] >> lane & 1)
            found[from + __popcll(mask[n] & ((uint64_t(1) << lane) - 1))] = r0 + n * kThreads + (int)threadIdx.x;
        }
        const int n = __builtin_amdgcn_readlane(all, kWave - 1);
        __syncthreads();
        if (n <= kFewDistances) {
          const int h = h0 + (int)threadIdx.x;
          double sum = 0.0;
          if (h < heads)
            for (int m = 0; m < n; ++m) sum += total[(int64_t)h * count + found[m]];
          sums[threadIdx.x] += sum;
        } else {
          for (int h = h0 + w; h < min(heads, h0 + kThreads); h += W) {
            double sum = 0.0;
            for (int m = lane; m < n; m += kAhead * kWave) {
              double v[kAhead];
#pragma unroll
              for (int k = 0; k < kAhead; ++k) v[k] = total[(int64_t)h * count + found[min(m + k * kWave, n - 1)]];
#pragma unroll
              for (int k = 0; k < kAhead; ++k) sum += m + k * kWave < n ? v[k] : 0.0;
            }
#pragma unroll
            for (int k = kWave / 2; k > 0; k /= 2) sum += __shfl_xor(sum, k);
            if (lane == 0) sums[h - h0] += sum;
          }
        }
        __syncthreads();
      }
      const int h = h0 + (int)threadIdx.x;
      if (h < heads) {
        TO* to = out + u * ld + h;
        *to = rounded_once<TO>(add ? (double)(float)*to + sums[threadIdx.x] : sums[threadIdx.x]);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// host-side launchers

constexpr int64_t kMostBlocks = 1 << 20;

template <class TI, class TO, bool ADD>
static void launch_bias_of(const tt_emb_matrix& table, const tt_emb_distances& dist, float fill, const tt_emb_pairs& in,
                           const tt_emb_pairs& out, hipStream_t st) {
  constexpr int P = kBiasPiece<TI, TO, ADD>;
  const int64_t planes = (int64_t)out.batch * out.heads;
  if (out.queries <= kFewQueries) {
    const int64_t rows = planes * out.queries;
    k_bias_few<TI, TO, ADD><<<(int)std::min(rows, kMostBlocks), kBiasThreads, 0, st>>>(table, dist, fill, in, out, rows);
    return;
  }
  BiasTiles tl;
  // Pieces of a tile's rows: a tile of as many places has fewer diagonals where its sides are alike, and more tiles lie beyond the
  // span.  us by 64 / 128 / 256: 16 x 4096 x 4096 bf16 86 / 95 / 93, with a span over all of it 83 / 92 / 132, added 181 / 182 / 194,
  // 16 x 2048 x 4096 fp32 84 / 88 / 95; but of rows that are no whole tiles, 16 x 2000 x 4000 bf16 65 / 64 / 96, x 4001 87 / 64 /
  // 98, fp32 154 / 126 / 98, added 229 / 218 / 212.
  const int wide = (out.keys % (kWave * P) == 0 ? 1 : P == 8 ? 2 : 4) * kWave * P;
  tl.across = (int)((out.keys + wide - 1) / wide);
  tl.cols = (int)(((out.keys + tl.across - 1) / tl.across + P - 1) / P * P);  // about the same width for all
  tl.rows = (int)std::min<int64_t>(out.queries, std::min(1024, 8 * kBiasThreads * P / tl.cols));
  // Small tiles, of a batch of pieces for each thread: 7 x 12 x 509 x 1021 fp32, added, by 4 rows 72 us, by 8 77, by 16 89; 16 x 4096
  // x 4096 bf16 by tiles of 2048 columns and 8 rows 92, 32 rows 101, 4 rows 149.
  while (tl.rows * tl.cols > kBiasAhead * kBiasThreads * P &&
         planes * tl.across * ((out.queries + tl.rows - 1) / tl.rows) < 16384)
    tl.rows = (tl.rows + 1) / 2;
  tl.down = (int)((out.queries + tl.rows - 1) / tl.rows);
  tl.count = planes * tl.down * tl.across;
  tl.line = (tl.rows + tl.cols + 15) / 8 * 8;
  tl.in_place = ADD && in.data == out.data;
  const int blocks = (int)std::min(tl.count, kMostBlocks), lds = 4 * tl.line * (int)sizeof(float);
  // Whole pieces: written alone 101 to 91 us at 16 x 4096 x 4096 bf16 by tiles of 2048 columns, but added 203 to 233.
  if constexpr (!ADD)
    if (out.keys % tl.cols == 0 && kBiasThreads * P % tl.cols == 0) {
      k_bias_tiles<TI, TO, ADD, true><<<blocks, kBiasThreads, lds, st>>>(table, dist, fill, in, out, tl);
      return;
    }
  k_bias_tiles<TI, TO, ADD, false><<<blocks, kBiasThreads, lds, st>>>(table, dist, fill, in, out, tl);
}

void launch_bias(const tt_emb_matrix& table, const tt_emb_distances& dist, float fill, const tt_emb_pairs* in,
                 const tt_emb_pairs& out, hipStream_t st) {
  with_type(out.type, [&](auto to) {
    typedef decltype(to) TO;
    if (in == nullptr) launch_bias_of<TO, TO, false>(table, dist, fill, out, out, st);
    else with_type(in->type, [&](auto ti) { launch_bias_of<decltype(ti), TO, true>(table, dist, fill, *in, out, st); });
  });
}

SumPlan sum_plan(const tt_emb_pairs& g, int span, bool offsets) {
  SumPlan p{};
  const int64_t batch = g.batch, heads = g.heads;
  if (batch == 0 || heads == 0 || g.queries == 0 || g.keys == 0) return p;
  // parts of a head: enough blocks, of 16 rows at least
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(kSumParts / heads, batch * ((g.queries + 15) / 16)));
  p.group = offsets ? 1 : (int)((batch + want - 1) / want);
  p.groups = (int)((batch + p.group - 1) / p.group);
  const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(want / p.groups, (g.queries + 15) / 16));
  p.rows = (int)((g.queries + chunks - 1) / chunks);
  p.chunks = (int)((g.queries + p.rows - 1) / p.rows);
  p.width = std::min<int64_t>(p.rows + g.keys - 1, 2 * (int64_t)span + 1);
  p.parts = heads * p.groups * p.chunks;
  return p;
}

// Distances [low, low + count) that may occur: with one offset for all sequences no others have to be joined.
static void distances_of(const tt_emb_pairs& g, const tt_emb_distances& dist, int* low, int* count) {
  int64_t from = -(int64_t)dist.span, to = dist.span;
  if (dist.offsets == nullptr) {
    const int64_t far = int64_t(1) << 40, o = std::min(std::max(dist.offset, -far), far);
    from = std::min(std::max(o + 1 - g.queries, from), to);
    to = std::max(std::min(o + g.keys - 1, to), from);
  }
  *low = (int)from;
  *count = (int)(to - from) + 1;
}

void launch_bias_sums(const tt_emb_pairs& g, const tt_emb_distances& dist, const tt_emb_matrix& out, bool add,
                      const SumPlan& p, const SumWork& ws, hipStream_t st) {
  int low = 0, count = 0;
  if (p.parts > 0) {
    with_type(g.type, [&](auto t) {
      typedef decltype(t) T;
      const int blocks = (int)std::min(p.parts, kMostBlocks);
      if (g.keys <= kShortKeys || (g.keys <= kShortRow && p.rows <= kShortRows))
        k_bias_sums_short<T><<<blocks, kSumThreads, 0, st>>>(g, dist, p, ws.parts, ws.reach);
      else if (p.width - 2 <= kWave * 4)
        k_bias_sums<T, 4><<<blocks, kSumThreads, 0, st>>>(g, dist, (int)out.rows, p, ws.parts, ws.reach);
      else
        k_bias_sums<T, 8><<<blocks, kSumThreads, 0, st>>>(g, dist, (int)out.rows, p, ws.parts, ws.reach);
    });
    distances_of(g, dist, &low, &count);
    const int blocks = (int)std::min<int64_t>((int64_t)(count + kWave - 1) / kWave * g.heads, kMostBlocks);
    // Wavefronts of a block by the blocks, us by 4 / 16: 8 x 16 x 2048 x 2048 with 255 distances (64 blocks) 8.2 / 5.4, 2 x 8 x 512 x
    // 512 with 255 4.4 / 4.8; with 4095 distances (1024 blocks) 10.5 / 15.8, 1 x 32 x 4096 x 4096 with 8191 (4096) 17 / 49.
    if (blocks >= 1024)
      k_bias_join<4><<<blocks, 4 * kWave, 0, st>>>(g.heads, low, count, p, ws.parts, ws.reach, ws.total, ws.reached);
    else
      k_bias_join<16><<<blocks, 16 * kWave, 0, st>>>(g.heads, low, count, p, ws.parts, ws.reach, ws.total, ws.reached);
  }
  with_type(out.type, [&](auto t) {
    typedef decltype(t) TO;
    auto go = [&](auto waves, auto ahead) {
      constexpr int W = decltype(waves)::value, U = decltype(ahead)::value;
      k_bias_buckets<TO, W, U><<<(int)std::min(out.rows, kMostBlocks), W * kWave, 0, st>>>(
          g.heads, dist.bucket_of + dist.span + low, count, ws.total, ws.reached, (TO*)out.data, out.ld, (int)out.rows, add);
    };
    // Wavefronts of a bucket and distances ahead of each, us by 4 and 4 / 4 and 16 / 16 and 4: 255 distances in 32 buckets 5.8 / 8.0 /
    // 6.0, 1023 in 200 5.9 / 7.7 / 5.3, in 300 5.3 / 7.2 / 6.2, 643 in 1001 4.1 / 6.4 / 8.2; 4095 in 32 12.9 / 11.9 / 5.6, 8191 in 64
    // 24 / 22 / 9, in 600 18 / 16 / 14, in 8000 57 / 54 / 77.
    if (count <= 1024 && out.rows >= 256) go(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
    else if (out.rows >= 1024) go(std::integral_constant<int, 4>{}, std::integral_constant<int, 16>{});
    else go(std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
  });
}

}  // namespace ttemb
