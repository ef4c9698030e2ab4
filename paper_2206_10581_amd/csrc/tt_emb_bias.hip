// Position bias of attention: a table [buckets, heads] looked up by the distance of a key from a query, alone or added to
// scores, and its gradient, sums of the scores' gradients over all places of a bucket.
//
// A distance is j - i + o with one o for a sequence, so a head's bias has one value for every diagonal.
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

// ---- bias of tiles

constexpr int kBiasThreads = 256, kBiasCols = 1024, kBiasRows = 64;
constexpr int kBiasLine = kBiasCols + kBiasRows + 8;  // diagonals of a tile, and some more
struct BiasTiles {
  int rows, cols;  // of a tile; rows + cols below kBiasLine - 7
  int down, across;
  int64_t count;
  int lanes;       // log2 of the threads side by side
};

// A block takes a tile of one head.  Its diagonals' values come first, four copies of the line, each a place further, so
// that any row finds its values in 16-byte words of one of them.
template <class TI, class TO, bool ADD>
__global__ __launch_bounds__(kBiasThreads) void k_bias_tiles(tt_emb_matrix table, tt_emb_distances dist, float fill,
                                                             tt_emb_pairs in, tt_emb_pairs out, BiasTiles tl) {
  __shared__ __attribute__((aligned(16))) float line[4][kBiasLine];
  constexpr int P = 16 / (ADD && sizeof(TI) > sizeof(TO) ? sizeof(TI) : sizeof(TO));
  const int side = threadIdx.x & ((1 << tl.lanes) - 1), up = threadIdx.x >> tl.lanes, step = kBiasThreads >> tl.lanes;
  for (int64_t tile = blockIdx.x; tile < tl.count; tile += gridDim.x) {
    const int64_t plane = tile / ((int64_t)tl.down * tl.across);
    const int64_t place = tile - plane * tl.down * tl.across;
    const int b = (int)(plane / out.heads), h = (int)(plane - (int64_t)b * out.heads);
    const int i0 = (int)(place / tl.across) * tl.rows, j0 = (int)(place % tl.across) * tl.cols;
    const int rows = (int)min((int64_t)tl.rows, out.queries - i0), cols = (int)min((int64_t)tl.cols, out.keys - j0);
    const int64_t first = offset_of(dist, b) + j0 - i0 - (rows - 1);  // distance of the first diagonal
    for (int x = threadIdx.x; x < rows + cols - 1; x += kBiasThreads) {
      const int u = dist.bucket_of[cut(first + x, dist.span) + dist.span];
      const float v = (uint32_t)u < (uint32_t)table.rows ? any_value(table, u * table.ld + h) : fill;
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (x >= s) line[s][x - s] = v;
    }
    __syncthreads();
    const TI* from = (const TI*)in.data + (ADD ? b * in.batch_ld + h * in.head_ld + i0 * in.query_ld + j0 : 0);
    TO* to = (TO*)out.data + b * out.batch_ld + h * out.head_ld + i0 * out.query_ld + j0;
    for (int r = up; r < rows; r += step)
      for (int c = side * P; c < cols; c += P << tl.lanes) {
        const int a = c - r + rows - 1, s = a & 3;
        float v[P];
        if (c + P <= cols) {
#pragma unroll
          for (int i = 0; i < P; i += 4) {
            const f4 w = *(const f4*)&line[s][a - s + i];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i + k] = w[k];
          }
          if constexpr (ADD) {
            float x[P];
            load_piece<P, TI>(from + r * in.query_ld + c, x);
#pragma unroll
            for (int i = 0; i < P; ++i) v[i] = isinf(v[i]) ? v[i] : x[i] + v[i];
          }
          store_piece<P, TO, true>(to + r * out.query_ld + c, v);
        } else {
          for (int i = 0; c + i < cols; ++i) {
            float y = line[0][a + i];
            if constexpr (ADD) y = isinf(y) ? y : (float)from[r * in.query_ld + c + i] + y;
            to[r * out.query_ld + c + i] = (TO)y;
          }
        }
      }
    __syncthreads();
  }
}

// ---- sums of buckets

// The diagonals d = j - i of a sequence that are told apart: [first, last], where first stands for all before it, too, and
// last for all behind.
struct Span {
  int first, last;
};
__device__ __forceinline__ Span span_of(const tt_emb_pairs& g, int64_t offset, int span) {
  const int64_t low = 1 - g.queries, high = g.keys - 1;
  return {(int)min(max(-(int64_t)span - offset, low), high), (int)max(min((int64_t)span - offset, high), low)};
}

constexpr int kSumThreads = 256, kSumWaves = kSumThreads / kWave, kSumAhead = 4;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) v += __shfl_xor(v, d);
  return v;
}

// A block sums the diagonals of some rows of one head and of p.group sequences, a lane B of them at a time: its accumulators
// stay, the row's place moves by a value from one row to the next.  All before the first and behind the last
// diagonal are summed apart, row by row.  Fp32 sums of at most a few hundred values.
template <class T, int B>
__global__ __launch_bounds__(kSumThreads) void k_bias_sums(tt_emb_pairs g, tt_emb_distances dist, int buckets, SumPlan p,
                                                           float* __restrict__ parts) {
  constexpr int P = 16 / sizeof(T), R = kSumAhead;
  __shared__ float sums[kSumWaves][kWave * B];
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  for (int64_t part = blockIdx.x; part < p.parts; part += gridDim.x) {
    const int64_t plane = part / p.chunks;
    const int chunk = (int)(part - plane * p.chunks);
    const int h = (int)(plane / p.groups), b0 = (int)(plane - (int64_t)h * p.groups) * p.group;
    const int b1 = min(b0 + p.group, g.batch), i0 = chunk * p.rows, i1 = (int)min((int64_t)i0 + p.rows, g.queries);
    const int keys = (int)g.keys;
    const int64_t offset = offset_of(dist, b0);
    const Span d = span_of(g, offset, dist.span);
    float* out = parts + part * p.width;
    auto wanted = [&](int diagonal) {
      return (uint32_t)dist.bucket_of[cut(diagonal + offset, dist.span) + dist.span] < (uint32_t)buckets;
    };
    const bool low = wanted(d.first), high = wanted(d.last);
    float before = 0.f, behind = 0.f;
    for (int b = b0; b < b1; ++b) {
      const T* rows = (const T*)g.data + b * g.batch_ld + h * g.head_ld;
      for (int i = i0 + w * R; i < i1; i += kSumWaves * R) {
        // columns [0, until) of a row are before, [since, keys) behind
        int until[R], since[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const bool there = i + r < i1;
          until[r] = there && low ? min(max(i + r + d.first + 1, 0), keys) : 0;
          since[r] = there && high ? min(max(i + r + max(d.last, d.first + 1), 0), keys) : keys;
        }
        for (int c = lane * P; c < keys; c += kWave * P) {
          typename Piece<T, P>::V v[R];
          const bool whole = c + P <= keys;
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (whole && (c < until[r] || c + P > since[r]))
              v[r] = *(const typename Piece<T, P>::V*)(rows + (i + r) * g.query_ld + c);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (!(c < until[r] || c + P > since[r])) continue;
            float a = 0.f, z = 0.f;
            if (whole) {
#pragma unroll
              for (int k = 0; k < P; ++k) {
                a += c + k < until[r] ? (float)v[r][k] : 0.f;
                z += c + k >= since[r] ? (float)v[r][k] : 0.f;
              }
            } else {
              for (int k = 0; c + k < keys; ++k) {
                const float x = (float)rows[(i + r) * g.query_ld + c + k];
                a += c + k < until[r] ? x : 0.f;
                z += c + k >= since[r] ? x : 0.f;
              }
            }
            before += a;
            behind += z;
          }
        }
      }
    }
    before = wave_sum(before);
    behind = wave_sum(behind);
    if (lane == 0) {
      sums[w][0] = before;
      sums[w][1] = behind;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      float a = 0.f, z = 0.f;
      for (int k = 0; k < kSumWaves; ++k) {
        a += sums[k][0];
        z += sums[k][1];
      }
      if (d.first == d.last) {
        out[0] = a + z;
      } else {
        out[0] = a;
        out[d.last - d.first] = z;
      }
    }
    __syncthreads();
    for (int x0 = d.first + 1; x0 < d.last; x0 += kWave * B) {
      const int x = x0 + lane * B;  // this lane's first diagonal
      float acc[B] = {};
      for (int b = b0; b < b1; ++b) {
        const T* rows = (const T*)g.data + b * g.batch_ld + h * g.head_ld;
        // rows that meet the band at all
        const int from = max(i0, -(x0 + kWave * B - 1)), to = (int)min((int64_t)i1, (int64_t)keys - x0);
        for (int i = from + w * R; i < to; i += kSumWaves * R) {
          typename Piece<T, B>::V v[R];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const int j = i + r + x;
            if (i + r < to && j >= 0 && j + B <= keys && x + B <= d.last)
              v[r] = *(const typename Piece<T, B>::V*)(rows + (i + r) * g.query_ld + j);
          }
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const int j = i + r + x;
            if (i + r >= to) continue;
            if (j >= 0 && j + B <= keys && x + B <= d.last) {
#pragma unroll
              for (int k = 0; k < B; ++k) acc[k] += (float)v[r][k];
            } else {
#pragma unroll
              for (int k = 0; k < B; ++k)
                if (j + k >= 0 && j + k < keys && x + k < d.last) acc[k] += (float)rows[(i + r) * g.query_ld + j + k];
            }
          }
        }
      }
#pragma unroll
      for (int k = 0; k < B; ++k) sums[w][lane * B + k] = acc[k];
      __syncthreads();
      for (int k = threadIdx.x; k < kWave * B && x0 + k < d.last; k += kSumThreads) {
        float s = 0.f;
        for (int n = 0; n < kSumWaves; ++n) s += sums[n][k];
        out[x0 + k - d.first] = s;
      }
      __syncthreads();
    }
  }
}

// A block adds up all parts of one bucket and head.
template <class TO>
__global__ __launch_bounds__(kSumThreads) void k_bias_buckets(tt_emb_pairs g, tt_emb_distances dist, SumPlan p,
                                                              const float* __restrict__ parts, TO* __restrict__ out,
                                                              int64_t ld, int buckets, bool add) {
  __shared__ int found[kSumThreads], counts[kSumWaves];
  __shared__ double sums[kSumWaves];
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave, distances = 2 * dist.span + 1;
  const int per_head = p.groups * p.chunks;
  for (int64_t place = blockIdx.x; place < (int64_t)buckets * g.heads; place += gridDim.x) {
    const int u = (int)(place / g.heads), h = (int)(place - (int64_t)u * g.heads);
    double sum = 0.0;
    for (int r0 = 0; r0 < distances && per_head > 0; r0 += kSumThreads) {
      const int r = r0 + (int)threadIdx.x;
      const uint64_t mask = __ballot(r < distances && dist.bucket_of[min(r, distances - 1)] == u);
      if (lane == 0) counts[w] = __popcll(mask);
      __syncthreads();
      int before = 0, n = 0;
      for (int k = 0; k < kSumWaves; ++k) {
        before += k < w ? counts[k] : 0;
        n += counts[k];
      }
      if (mask >> lane & 1) found[before + __popcll(mask & ((uint64_t(1) << lane) - 1))] = r - dist.span;
      __syncthreads();
      if (n > 0) {
        int lanes = 0;
        while ((1 << lanes) < n) ++lanes;
        const int m = threadIdx.x & ((1 << lanes) - 1);
        if (m < n)
          for (int k = threadIdx.x >> lanes; k < per_head; k += kSumThreads >> lanes) {
            const int64_t offset = offset_of(dist, k / p.chunks * p.group);
            const Span d = span_of(g, offset, dist.span);
            // the diagonal of this distance, if it is told apart or is an end
            int64_t diagonal = found[m] - offset;
            if (found[m] == -dist.span && d.first + offset <= -dist.span) diagonal = d.first;
            else if (found[m] == dist.span && d.last + offset >= dist.span) diagonal = d.last;
            if (diagonal >= d.first && diagonal <= d.last)
              sum += (double)parts[((int64_t)h * per_head + k) * p.width + (diagonal - d.first)];
          }
      }
      __syncthreads();
    }
#pragma unroll
    for (int k = kWave / 2; k > 0; k /= 2) sum += __shfl_xor(sum, k);
    if (lane == 0) sums[w] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      sum = 0.0;
      for (int k = 0; k < kSumWaves; ++k) sum += sums[k];
      TO* to = out + u * ld + h;
      *to = (TO)(float)(add ? (double)(float)*to + sum : sum);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------
// host-side launchers

constexpr int64_t kMostBlocks = 1 << 20;

void launch_bias(const tt_emb_matrix& table, const tt_emb_distances& dist, float fill, const tt_emb_pairs* in,
                 const tt_emb_pairs& out, hipStream_t st) {
  BiasTiles tl;
  const int size = type_size(std::min(out.type, in ? in->type : out.type)), P = 16 / size;
  tl.cols = (int)std::min<int64_t>((out.keys + P - 1) / P * P, kBiasCols);
  tl.across = (int)((out.keys + tl.cols - 1) / tl.cols);
  const int64_t planes = (int64_t)out.batch * out.heads;
  tl.rows = (int)std::min<int64_t>(std::min<int64_t>(out.queries, kBiasLine - 8 - tl.cols), 65536 / tl.cols);
  // enough tiles for all compute units
  while (tl.rows > 8 && planes * tl.across * ((out.queries + tl.rows - 1) / tl.rows) < 2048) tl.rows /= 2;
  tl.down = (int)((out.queries + tl.rows - 1) / tl.rows);
  tl.count = planes * tl.down * tl.across;
  tl.lanes = 0;
  while ((1 << tl.lanes) < kBiasThreads && (P << tl.lanes) < tl.cols) ++tl.lanes;
  const int blocks = (int)std::min(tl.count, kMostBlocks);
  with_type(out.type, [&](auto to) {
    typedef decltype(to) TO;
    if (in == nullptr) {
      k_bias_tiles<TO, TO, false><<<blocks, kBiasThreads, 0, st>>>(table, dist, fill, out, out, tl);
      return;
    }
    with_type(in->type, [&](auto ti) {
      k_bias_tiles<decltype(ti), TO, true><<<blocks, kBiasThreads, 0, st>>>(table, dist, fill, *in, out, tl);
    });
  });
}

SumPlan sum_plan(const tt_emb_pairs& g, int span, bool offsets) {
  SumPlan p{};
  const int64_t batch = g.batch, heads = g.heads;
  if (batch == 0 || heads == 0 || g.queries == 0 || g.keys == 0) return p;
  p.width = std::min<int64_t>(g.queries + g.keys - 1, 2 * (int64_t)span + 1);
  // parts of a head: enough blocks, each with 16 times the values that it leaves
  const int64_t places = batch * g.queries * g.keys;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(kSumParts / heads, places / (16 * p.width)));
  p.group = offsets ? 1 : (int)((batch + want - 1) / want);
  p.groups = (int)((batch + p.group - 1) / p.group);
  const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(want / p.groups, (g.queries + 15) / 16));
  p.rows = (int)((g.queries + chunks - 1) / chunks);
  p.chunks = (int)((g.queries + p.rows - 1) / p.rows);
  p.parts = heads * p.groups * p.chunks;
  return p;
}

void launch_bias_sums(const tt_emb_pairs& g, const tt_emb_distances& dist, const tt_emb_matrix& out, bool add,
                      float* parts, hipStream_t st) {
  const SumPlan p = sum_plan(g, dist.span, dist.offsets != nullptr);
  if (p.parts > 0)
    with_type(g.type, [&](auto t) {
      typedef decltype(t) T;
      const int blocks = (int)std::min(p.parts, kMostBlocks);
      if (p.width - 2 <= kWave * 4)
        k_bias_sums<T, 4><<<blocks, kSumThreads, 0, st>>>(g, dist, (int)out.rows, p, parts);
      else
        k_bias_sums<T, 8><<<blocks, kSumThreads, 0, st>>>(g, dist, (int)out.rows, p, parts);
    });
  const int64_t places = out.rows * out.cols;
  with_type(out.type, [&](auto t) {
    typedef decltype(t) TO;
    k_bias_buckets<TO><<<(int)std::min(places, kMostBlocks), kSumThreads, 0, st>>>(g, dist, p, parts, (TO*)out.data, out.ld,
                                                                                 (int)out.rows, add);
  });
}

}  // namespace ttemb
