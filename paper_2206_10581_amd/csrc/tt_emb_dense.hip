// Plain embedding tables beside the tensor-train one: rows by id times a scale, and the table's gradient as
// sums over the positions of each id, found by a stable sort of the ids.  fp32, bf16 and fp16; products and sums
// in fp32, rounded once where a value is stored.
#include <type_traits>

#include "tt_emb_internal.h"

namespace ttemb {

constexpr int kDenseThreads = 256;
constexpr int kRowsAhead = 2;  // rows of a lookup that a thread has under way

// Values that a thread takes at once: 16 bytes of the type that is read.  VEC = 1: rows shorter than that.
// Rows start wherever their strides put them, so these vectors are aligned like single values.
template <class T, int VEC>
struct Piece {
  typedef T V __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
};
template <class T>
struct Piece<T, 1> {
  typedef T V;
};

template <int VEC, class T>
__device__ __forceinline__ void values_of(const typename Piece<T, VEC>::V& v, float (&x)[VEC]) {
  if constexpr (VEC == 1) {
    x[0] = (float)v;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = (float)v[i];
  }
}

template <int VEC, class T>
__device__ __forceinline__ void load_piece(const T* p, float (&x)[VEC]) {
  values_of<VEC, T>(*(const typename Piece<T, VEC>::V*)p, x);
}

template <int VEC, class T, bool PAST = false>
__device__ __forceinline__ void store_piece(T* p, const float (&x)[VEC]) {
  typename Piece<T, VEC>::V v;
  if constexpr (VEC == 1) {
    v = (T)x[0];
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = (T)x[i];
  }
  if constexpr (PAST) __builtin_nontemporal_store(v, (typename Piece<T, VEC>::V*)p);
  else *(typename Piece<T, VEC>::V*)p = v;
}

// How a block's threads are dealt: 2^lanes of them side by side along a row, blockIdx.y over what is left of it.
struct Lanes {
  int lanes;   // log2
  int pieces;  // of a row
};

// The last piece of a row that is no multiple of VEC starts early and holds some values of its neighbour again.
template <int VEC>
__device__ __forceinline__ int piece_start(int c, int cols) {
  return min(c * VEC, cols - VEC);
}

// out[b] = scale * W[ids[b]], zeros for ids outside the table.  A thread has two rows under way, first their ids.  Bound by
// the memory: rows are read through the caches, since ids repeat, and written past them.  16,384 rows of 4096 bf16
// (191 MB) 33 us, 200,000 of 100 fp32 (111 MB) 23; through the caches 44 and 38, one row at a time 52 and 42.
template <class TI, class TO, int VEC>
__global__ __launch_bounds__(kDenseThreads) void k_dense_rows(const TI* __restrict__ table, int64_t ld, int64_t rows,
                                                              const int64_t* __restrict__ ids, int B, float scale,
                                                              TO* __restrict__ out, int64_t ld_out, int cols, Lanes ln) {
  typedef typename Piece<TI, VEC>::V VI;
  constexpr int R = kRowsAhead;
  const int c = (blockIdx.y << ln.lanes) + (threadIdx.x & ((1 << ln.lanes) - 1));
  if (c >= ln.pieces) return;
  const int col = piece_start<VEC>(c, cols), side = kDenseThreads >> ln.lanes;
  for (int64_t b0 = (int64_t)blockIdx.x * side * R + (threadIdx.x >> ln.lanes); b0 < B;
       b0 += (int64_t)gridDim.x * side * R) {
    int64_t id[R];
    VI v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) id[r] = ids[min(b0 + r * side, (int64_t)B - 1)];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool inside = (uint64_t)id[r] < (uint64_t)rows;
      v[r] = VI{};
      if (inside) v[r] = *(const VI*)(table + id[r] * ld + col);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool inside = (uint64_t)id[r] < (uint64_t)rows;
      float x[VEC];
      values_of<VEC, TI>(v[r], x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] = inside ? x[i] * scale : 0.f;
      if (b0 + r * side < B) store_piece<VEC, TO, true>(out + (b0 + r * side) * ld_out + col, x);
    }
  }
}

// A gradient without positions
__global__ __launch_bounds__(kFillThreads) void k_fill(FillShare fill) {
  fill_share(fill, (int)blockIdx.x, (int)gridDim.x);
}

// How tile t of the sorted slots takes part in the runs that cross its borders.  A run that starts in a tile is
// summed by it alone if it ends in the next tile at the latest.  A longer one is cut at the borders of the tiles:
// the first tile's part goes to `tail`, every other's to `head`, and k_dense_join adds them up.
struct TileRuns {
  int s0, s1;        // slots of the tile
  int limit;         // end of the slots that the tile adds up, beyond s1 where its last run goes on
  uint32_t first, last;  // ids of its first and last slot
  bool began;        // the first slot's run began in an earlier tile
  bool head;         // and is a long one: the tile leaves its part
  bool tail;         // the last run begins here and is a long one
  __device__ __forceinline__ TileRuns(const uint32_t* __restrict__ key, int t, int tile, int B, uint32_t none) {
    s0 = t * tile;
    s1 = min(s0 + tile, B);
    first = key[s0];
    last = key[s1 - 1];
    const uint32_t prev = key[max(s0 - 1, 0)], prev2 = key[max(s0 - tile - 1, 0)];
    const uint32_t next = key[min(s1, B - 1)], after = key[min(s1 + tile, B - 1)];
    began = t >= 1 && prev == first;
    head = began && first < none && ((t >= 2 && prev2 == first) || (s1 < B && next == first));
    const bool goes_on = last < none && s1 < B && next == last && !(began && first == last);
    tail = goes_on && s1 + tile < B && after == last;
    limit = goes_on && !tail ? min(s1 + tile, B) : s1;
  }
};

template <class TO, int VEC, bool ADD>
__device__ __forceinline__ void put_sum(TO* __restrict__ row, int col, int c, float scale, const float (&sum)[VEC],
                                        const typename Piece<TO, VEC>::V& old) {
  float x[VEC];
  if constexpr (!ADD) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = scale * sum[i];
    store_piece<VEC, TO, true>(row + col, x);
  } else if (col == c * VEC) {
    values_of<VEC, TO>(old, x);
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = fmaf(scale, sum[i], x[i]);
    store_piece<VEC, TO, true>(row + col, x);
  } else {  // values that the neighbour has too are its own to add
    for (int i = c * VEC - col; i < VEC; ++i) {
      float s = 0.f;  // sum[i], with constant indexes
#pragma unroll
      for (int k = 0; k < VEC; ++k) s = k == i ? sum[k] : s;
      row[col + i] = (TO)fmaf(scale, s, (float)row[col + i]);
    }
  }
}

// Sums of the gradient rows of every id whose run of sorted slots a tile owns.  WAVE: a wavefront takes (a part of) one
// tile, so that keys and positions are scalars and their branches are its own; else 2^lanes threads do.
// Eight slots at a time: their keys and positions, then all rows (slots that are not the tile's read a row again that
// it reads anyway), and with ADD the table rows of those that end a run, then the sums in order.  Gradient rows pass
// the caches by, which hold what was just cleared: 16,384 rows of 4096 bf16 72 -> 45 us, 200,000 of 128 fp32 58 -> 40.
template <class TI, class TO, int VEC, bool ADD, bool WAVE>
__global__ __launch_bounds__(kDenseThreads) void k_dense_sum(const uint32_t* __restrict__ key,
                                                             const uint32_t* __restrict__ pos, int B, int tile,
                                                             uint32_t none, const TI* __restrict__ grad,
                                                             int64_t ld_grad, int cols, Lanes ln, float scale,
                                                             TO* __restrict__ out, int64_t ld,
                                                             float* __restrict__ head, float* __restrict__ tail,
                                                             int stride, uint32_t* __restrict__ starts) {
  typedef typename Piece<TI, VEC>::V VI;
  typedef typename Piece<TO, VEC>::V VO;
  constexpr int kAhead = kDenseAhead;
  const int c = (blockIdx.y << ln.lanes) + (threadIdx.x & ((1 << ln.lanes) - 1));
  if (c >= ln.pieces) return;
  const int col = piece_start<VEC>(c, cols), step = gridDim.x * (kDenseThreads >> ln.lanes);
  const int tiles = (B + tile - 1) / tile;
  int t = blockIdx.x * (kDenseThreads >> ln.lanes) + (threadIdx.x >> ln.lanes);
  if constexpr (WAVE) t = __builtin_amdgcn_readfirstlane(t);
  for (; t < tiles; t += step) {
    const TileRuns r(key, t, tile, B, none);
    if (c == 0) starts[t] = r.tail ? r.last : none;
    if (r.first >= none) continue;  // positions without an id are last
    const uint32_t any = pos[r.s0];
    float acc[VEC] = {};
    for (int s = r.s0; s < r.limit; s += kAhead) {
      uint32_t k[kAhead + 1], p[kAhead];
#pragma unroll
      for (int i = 0; i <= kAhead; ++i) k[i] = key[s + i];  // there are some entries behind the last
#pragma unroll
      for (int i = 0; i < kAhead; ++i) p[i] = pos[s + i];
      bool mine[kAhead + 1], ends[kAhead];
#pragma unroll
      for (int i = 0; i <= kAhead; ++i)
        mine[i] = s + i < r.limit && k[i] < none && (s + i < r.s1 || k[i] == r.last) &&
                  !(r.began && !r.head && k[i] == r.first);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ends[i] = mine[i] && !(mine[i + 1] && k[i + 1] == k[i]);
      VI x[kAhead];
      VO old[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        x[i] = __builtin_nontemporal_load((const VI*)(grad + (int64_t)(mine[i] ? p[i] : any) * ld_grad + col));
      if constexpr (ADD) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          if (ends[i]) old[i] = *(const VO*)(out + (int64_t)k[i] * ld + col);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (!mine[i]) continue;
        float v[VEC];
        values_of<VEC, TI>(x[i], v);
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[j] += v[j];
        if (!ends[i]) continue;
        if (r.began && k[i] == r.first) store_piece<VEC>(head + (size_t)t * stride + col, acc);
        else if (r.tail && k[i] == r.last) store_piece<VEC>(tail + (size_t)t * stride + col, acc);
        else put_sum<TO, VEC, ADD>(out + (int64_t)k[i] * ld, col, c, scale, acc, old[i]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
      }
    }
  }
}

// Long runs: the parts that their tiles left are added in a fixed order.  A block looks at 64 tiles and takes 128
// columns; a lane has four of them, and the halves (of narrower rows smaller parts) of a wavefront take a run's parts in
// turn.  A wavefront takes a run of its own, but all of them the one run of a block that has more than 64 parts.  65,536
// ids, half of them the same, rows of 1024 bf16: 88 us with four wavefronts on every run and its end looked for from 64
// tiles to the next 64, 25 so.  64 columns a block take 17 there, but 15 instead of 9 at 16,384 rows of 4096.
constexpr int kJoinThreads = 1024, kJoinWaves = kJoinThreads / kWave, kJoinTiles = kWave, kJoinCols = 128;
constexpr int kJoinLanes = kJoinCols / 4;  // at most
constexpr int kJoinAhead = 8;  // parts under way at once
template <class TO, bool ADD>
__global__ __launch_bounds__(kJoinThreads) void k_dense_join(const uint32_t* __restrict__ key, int B, int tile,
                                                             uint32_t none, int cols, float scale,
                                                             TO* __restrict__ out, int64_t ld,
                                                             const float* __restrict__ head,
                                                             const float* __restrict__ tail, int stride,
                                                             const uint32_t* __restrict__ start_ids, int lanes) {
  __shared__ f4 part[kJoinWaves][kJoinLanes];
  const int tiles = (B + tile - 1) / tile, lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  const int groups = kWave / lanes, group = lane / lanes, col = blockIdx.y * kJoinCols + lane % lanes * 4;
  // parts number p, p + step, ... of the run that starts in tile t, the first in `tail`, added over a wavefront
  auto sum_of = [&](int t, int parts, int p, int step) {
    f4 sum = {0.f, 0.f, 0.f, 0.f};
    for (; p < parts && col < cols; p += kJoinAhead * step) {
      f4 v[kJoinAhead];
#pragma unroll
      for (int i = 0; i < kJoinAhead; ++i) {
        const int q = min(p + i * step, parts - 1);
        v[i] = *(const f4*)((q == 0 ? tail : head) + (size_t)(t + q) * stride + col);
      }
#pragma unroll
      for (int i = 0; i < kJoinAhead; ++i)
        if (p + i * step < parts) sum += v[i];
    }
    for (int d = lanes; d < kWave; d *= 2)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], d);
    return sum;
  };
  auto put = [&](uint32_t id, const f4& sum) {
    TO* row = out + (int64_t)id * ld + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane < lanes && col + i < cols) row[i] = (TO)(ADD ? fmaf(scale, sum[i], (float)row[i]) : scale * sum[i]);
  };
  for (int t0 = blockIdx.x * kJoinTiles; t0 < tiles; t0 += gridDim.x * kJoinTiles) {
    const uint32_t start_id = start_ids[min(t0 + lane, tiles - 1)];
    unsigned long long starts = __ballot(t0 + lane < tiles && start_id < none);  // the same in every wavefront
    for (int n = 0; starts != 0; ++n) {
      const int t = t0 + __ffsll((long long)starts) - 1;
      starts &= starts - 1;
      if (starts != 0 && n % kJoinWaves != w) continue;
      const uint32_t id = (uint32_t)__builtin_amdgcn_readlane((int)start_id, t - t0);
      // The run holds the first slots of tiles t+1 and t+2; up to which: a look at the next 64 tiles, then at 64
      // places over what is left, and so on between two of these.
      int end = t + 3, hi = tiles;
      for (int step = 1;;) {
        const int at = end + lane * step;
        const unsigned long long others = __ballot(at >= hi || key[(int64_t)min(at, tiles - 1) * tile] != id);
        const int k = others != 0 ? __ffsll((long long)others) - 1 : kWave;  // tile end + (k-1) * step is its own
        if (step == 1 && k < kWave) {
          end += k;
          break;
        }
        if (k < kWave) hi = min(hi, end + k * step);
        if (k > 0) end += (k - 1) * step + 1;
        if (end >= hi) break;
        step = (hi - end + kWave - 1) / kWave;
      }
      if (end - t <= kWave) {  // every run but the last of the 64 tiles is such a one
        if (n % kJoinWaves == w) put(id, sum_of(t, end - t, group, groups));
        continue;
      }
      const f4 sum = sum_of(t, end - t, w * groups + group, kJoinWaves * groups);
      if (lane < lanes) part[w][lane] = sum;
      __syncthreads();
      if (w == 0) {
        f4 all = part[0][lane % lanes];
        for (int k = 1; k < kJoinWaves; ++k) all += part[k][lane % lanes];
        put(id, all);
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Few positions: one launch, without a sort.  A block has a position and 64 pieces of its row: it looks for the position's
// id among all of them, leaves if an earlier position has it, and adds up the rows of those that do, eight under way
// at once, four wavefronts taking eights in turn where there are more than eight.  Blocks in front of these clear the
// rows whose ids no position has, which they mark in LDS.

constexpr int kFewThreads = kDenseThreads, kFewWaves = kFewThreads / kWave, kFewLooks = kFewMost / kFewThreads;
static_assert(kFewThreads == kFillThreads, "all threads of a block clear");

// Clears the rows of the job that are not marked, as block number b of n (fill_share has the other case).
__device__ __forceinline__ void fill_unmarked(const FillJob& j, const uint32_t* marks, int b, int n) {
  const f4 zero = {0.f, 0.f, 0.f, 0.f};
  const int tid = threadIdx.x, width = j.width;
  auto marked = [&](int row) { return (marks[row >> 5] >> (row & 31)) & 1u; };
  if (j.pitch != width && j.rows > 1) {
    typedef f4 f4_any __attribute__((aligned(2)));
    const int pieces = (width + 15) / 16;
    int lanes = 0;
    while ((1 << lanes) < pieces && (1 << lanes) < kFillThreads) ++lanes;
    const int per = kFillThreads >> lanes;
    for (int64_t r = b * per + (tid >> lanes); r < j.rows; r += n * per) {
      if (marked((int)r)) continue;
      char* row = j.data + r * j.pitch;
      for (int c = tid & ((1 << lanes) - 1); c < pieces; c += 1 << lanes) {
        if (width >= 16) *(f4_any*)(row + min(c * 16, width - 16)) = zero;
        else
          for (int i = 0; i < width / 2; ++i) ((uint16_t*)row)[i] = 0;
      }
    }
    return;
  }
  // `count` two-byte units from byte `at` on, which lies in `row`, `in` bytes behind its start
  auto units = [&](int64_t at, int row, int in, int count) {
    for (int i = 0; i < count; ++i, in += 2) {
      for (; in >= width; in -= width) ++row;
      if (!marked(row)) *(uint16_t*)(j.data + at + 2 * i) = 0;
    }
  };
  // Four 16-byte words of a thread at once, 256 words apart: the place in the table of each follows from the one in front
  // by additions, and their looks at the marks wait together.
  constexpr int kWords = 4;
  const int last = (int)j.rows - 1;
  const int64_t bytes = j.rows * width, lead = min(bytes, (int64_t)(-(uintptr_t)j.data & 15u));
  const int64_t words = (bytes - lead) / 16, step = (int64_t)n * kWords * kFillThreads;
  int64_t i = (int64_t)b * kWords * kFillThreads + tid;
  int row = (int)((lead + i * 16) / width), in = (int)((lead + i * 16) % width);
  const int step_rows = (int)(step * 16 / width), step_in = (int)(step * 16 % width);
  const int side_rows = kFillThreads * 16 / width, side_in = kFillThreads * 16 % width;
  auto move = [&](int& r, int& e, int rows, int bytes_in) {
    r += rows;
    e += bytes_in;
    if (e >= width) {
      e -= width;
      ++r;
    }
  };
  for (; i < words; i += step) {
    int rows[kWords], ins[kWords];
    uint32_t any[kWords];
    rows[0] = row;
    ins[0] = in;
#pragma unroll
    for (int k = 1; k < kWords; ++k) {
      rows[k] = rows[k - 1];
      ins[k] = ins[k - 1];
      move(rows[k], ins[k], side_rows, side_in);
    }
#pragma unroll
    for (int k = 0; k < kWords; ++k) {  // words behind the end look at the last row
      any[k] = marked(min(rows[k], last));
      int r = rows[k];
      for (int e = ins[k] + 14; e >= width; e -= width) any[k] |= marked(min(++r, last));
    }
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      const int64_t at = i + k * kFillThreads;
      if (at >= words) break;
      if (!any[k]) *(f4*)(j.data + lead + at * 16) = zero;
      else units(lead + at * 16, rows[k], ins[k], 8);
    }
    move(row, in, step_rows, step_in);
  }
  if (b == 0 && tid == 0) {
    units(0, 0, 0, (int)(lead / 2));
    const int64_t at = lead + words * 16;
    if (at < bytes) units(at, (int)(at / width), (int)(at % width), (int)((bytes - at) / 2));
  }
}

template <class TI, class TO, int VEC, bool ADD>
__global__ __launch_bounds__(kFewThreads) void k_dense_few(TableSource src, int B, uint32_t none,
                                                           const TI* __restrict__ grad, int64_t ld_grad, int cols,
                                                           int pieces, float scale, TO* __restrict__ out, int64_t ld,
                                                           int clear, FillJob job) {
  typedef typename Piece<TI, VEC>::V VI;
  extern __shared__ uint32_t marks[];
  __shared__ float part[kFewWaves - 1][VEC][kWave];
  __shared__ int counts[kFewWaves];
  __shared__ uint16_t list[kFewMost];
  const int tid = threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave);
  if ((int)blockIdx.x < clear) {
    for (int i = tid; i < (int)(none + 31) / 32; i += kFewThreads) marks[i] = 0u;
    __syncthreads();
    for (int i = tid; i < B; i += kFewThreads) {
      const uint32_t id = key_of_id(src, i, none);
      if (id < none) atomicOr(&marks[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    fill_unmarked(job, marks, (int)blockIdx.x, clear);
    return;
  }
  const int slices = (pieces + kWave - 1) / kWave;
  const int at = (int)blockIdx.x - clear, b = at / slices, c = (at - b * slices) * kWave + lane;
  const uint32_t id = key_of_id(src, b, none);
  if (id >= none) return;
  // the positions that have this id, in order: every wavefront looks through its part of them all
  const int part_ids = (B + kFewWaves - 1) / kFewWaves, i0 = w * part_ids, i1 = min(i0 + part_ids, B);
  unsigned long long same[kFewLooks];
  int mine = 0;
#pragma unroll
  for (int m = 0; m < kFewLooks; ++m) {
    const int i = i0 + m * kWave + lane;
    same[m] = __ballot(i < i1 && key_of_id(src, min(i, B - 1), none) == id);
    mine += __popcll(same[m]);
  }
  if (lane == 0) counts[w] = mine;
  __syncthreads();
  int count = 0, before = 0;
#pragma unroll
  for (int v = 0; v < kFewWaves; ++v) {
    before += v < w ? counts[v] : 0;
    count += counts[v];
  }
#pragma unroll
  for (int m = 0; m < kFewLooks; ++m) {
    if ((same[m] >> lane) & 1ull) list[before + __popcll(same[m] & ((1ull << lane) - 1ull))] = (uint16_t)(i0 + m * kWave + lane);
    before += __popcll(same[m]);
  }
  __syncthreads();
  if (list[0] != b) return;  // an earlier position has it
  const int waves = min((count + kDenseAhead - 1) / kDenseAhead, kFewWaves);  // that have rows to add
  const int col = piece_start<VEC>(min(c, pieces - 1), cols);
  float acc[VEC] = {};
  for (int s = w * kDenseAhead; s < count && w < waves; s += 2 * waves * kDenseAhead) {
    const int s2 = s + waves * kDenseAhead;  // the next eight of this wavefront are asked for with these
    VI x[2][kDenseAhead];
    auto ask = [&](VI(&v)[kDenseAhead], int from) {
#pragma unroll
      for (int i = 0; i < kDenseAhead; ++i)
        v[i] = __builtin_nontemporal_load((const VI*)(grad + (int64_t)list[min(from + i, count - 1)] * ld_grad + col));
    };
    auto add = [&](const VI(&v)[kDenseAhead], int from) {
      float eight[VEC] = {};  // summed by themselves: no value goes through more than 8 + 32 + 4 additions
#pragma unroll
      for (int i = 0; i < kDenseAhead; ++i) {
        if (from + i >= count) continue;
        float f[VEC];
        values_of<VEC, TI>(v[i], f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) eight[j] += f[j];
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] += eight[j];
    };
    ask(x[0], s);
    if (s2 < count) ask(x[1], s2);
    add(x[0], s);
    if (s2 < count) add(x[1], s2);
  }
  if (waves > 1) {
    if (w > 0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) part[w - 1][j][lane] = acc[j];
    }
    __syncthreads();
    if (w == 0)
      for (int k = 0; k < waves - 1; ++k)
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[j] += part[k][j][lane];
  }
  if (w != 0 || c >= pieces) return;
  typename Piece<TO, VEC>::V old{};
  TO* row = out + (int64_t)id * ld;
  if constexpr (ADD) old = *(const typename Piece<TO, VEC>::V*)(row + col);
  put_sum<TO, VEC, ADD>(row, col, c, scale, acc, old);
}

// ---------------------------------------------------------------------------------------------
// host-side launchers

template <class F>
static void with_type(int type, F&& f) {
  switch (type) {
    case TT_EMB_BF16: f(__bf16{}); break;
    case TT_EMB_FP16: f(_Float16{}); break;
    default: f(float{}); break;
  }
}

// f gets the number of values of a piece: 16 bytes of a type, or one where the rows are shorter
template <class T, class F>
static void with_piece(int cols, F&& f) {
  constexpr int kVec = 16 / (int)sizeof(T);
  if (cols >= kVec) f(std::integral_constant<int, kVec>{});
  else f(std::integral_constant<int, 1>{});
}

// The same where a wavefront takes a row: the fewest values a thread that let it hold the row, and 16 bytes where none
// does.  Narrower pieces keep all lanes at work and fewer sums in registers.
template <class T, class F>
static void with_wave_piece(int cols, F&& f) {
  constexpr int kVec = 16 / (int)sizeof(T);
  if (cols <= kWave) f(std::integral_constant<int, 1>{});
  else if (cols <= 2 * kWave) f(std::integral_constant<int, 2>{});
  else if (kVec == 4 || cols <= 4 * kWave) f(std::integral_constant<int, 4>{});
  else f(std::integral_constant<int, kVec>{});
}

static Lanes lanes_of(int cols, int vec) {
  Lanes ln{0, (cols + vec - 1) / vec};
  while ((1 << ln.lanes) < ln.pieces && (1 << ln.lanes) < kDenseThreads) ++ln.lanes;
  return ln;
}

// Blocks for `rows` rows (or tiles) dealt like this; kernels stride over what a grid of 2^22 blocks leaves.
static dim3 grid_of(int64_t rows, const Lanes& ln) {
  const int64_t per = kDenseThreads >> ln.lanes, y = ((ln.pieces - 1) >> ln.lanes) + 1;
  const int64_t x = std::min<int64_t>((rows + per - 1) / per, (int64_t)(1 << 22) / y);
  return dim3((unsigned)x, (unsigned)y);
}

void launch_dense_rows(const tt_emb_matrix& table, const int64_t* ids, int B, float scale, const tt_emb_matrix& out,
                       hipStream_t st) {
  with_type(table.type, [&](auto ti) {
    with_type(out.type, [&](auto to) {
      using TI = decltype(ti);
      using TO = decltype(to);
      with_piece<std::conditional_t<sizeof(TI) == 4, TI, TO>>(table.cols, [&](auto vec) {
        const Lanes ln = lanes_of(table.cols, vec());
        k_dense_rows<TI, TO, vec()><<<grid_of((B + kRowsAhead - 1) / kRowsAhead, ln), kDenseThreads, 0, st>>>(
            (const TI*)table.data, table.ld, table.rows, ids, B, scale, (TO*)out.data, out.ld, table.cols, ln);
      });
    });
  });
}

bool dense_few(int B, const FillJob& job) {
  return B <= kFewMost && (job.width == 0 || (job.rows <= kFewRows && job.rows * job.width <= kFewBytes));
}

void launch_dense_few(const TableSource& src, int B, const tt_emb_matrix& grad, float scale, const tt_emb_matrix& out,
                      const FillJob& job, hipStream_t st) {
  const uint32_t none = (uint32_t)out.rows;
  const bool add = job.width == 0;
  with_type(grad.type, [&](auto ti) {
    with_type(out.type, [&](auto to) {
      using TI = decltype(ti);
      using TO = decltype(to);
      with_piece<TI>(grad.cols, [&](auto vec) {
        const int pieces = (grad.cols + vec() - 1) / vec(), slices = (pieces + kWave - 1) / kWave;
        const int clear = add ? 0 : kFewClear, lds = add ? 0 : (int)((out.rows + 31) / 32 * 4);
        auto launch = [&](auto kernel) {
          kernel<<<clear + B * slices, kFewThreads, lds, st>>>(src, B, none, (const TI*)grad.data, grad.ld, grad.cols,
                                                                 pieces, scale, (TO*)out.data, out.ld, clear, job);
        };
        if (add) launch(k_dense_few<TI, TO, vec(), true>);
        else launch(k_dense_few<TI, TO, vec(), false>);
      });
    });
  });
}

void launch_fill(const FillJob& job, hipStream_t st) {
  k_fill<<<kFillBlocks, kFillThreads, 0, st>>>(FillShare{job, 0, 1, 1});
}

// Sorted slots of a tile: few where few wavefronts are at work (a wavefront takes a row's 64 pieces), more where more
// parts of long runs cost as much as they bring.  Sums in us with tiles of 8 / 16 / 32: 129 rows of 512 bf16 5.4 / 7.9 /
// 13.9, 5003 of 1001 fp16 7.2 / 10.2 / 17.4, 50,000 of 24 fp32 8.3 / 13.1 / 19.8, 8192 of 2048 bf16 18.4 / 17.2 / 20.5,
// 16,384 of 4096 bf16 45.8 / 43.1 / 45.4, 200,000 of 128 fp32 33.6 / 35.0 / 39.7.  Sums and joins together with 8 / 16:
// 20,000 rows of 512 bf16 16.7 / 19.2, 65,536 of 256 23.1 / 21.4, 100,000 of 128 26.0 / 24.2.
// Rows of fewer than 64 values: few are summed by a wavefront each all the same, many by groups of lanes.  All kernels of
// a call in us, wavefronts / groups: 4295 ids, 8 bf16 values 15.2 / 18.6, 24 15.4 / 16.7, 56 16.7 / 18.5; 20,001 ids, 8
// values 34.5 / 36.3, 56 35.3 / 37.2; 50,000, 24 fp32 values 43.0 / 38.1; 145,827, 8 bf16 values 56.5 / 57.5, 24 55.5 / 48.9,
// 56 58.3 / 55.5.
constexpr int kNarrowIds = 1 << 15;
constexpr int64_t kTileFewPieces = (int64_t)64 << 16;
constexpr int kTileFewIds = 1 << 16;
int dense_tile(int B, int cols, int type) {
  const int piece = type == TT_EMB_FP32 ? 4 : 8;
  const bool few = (int64_t)B * ((cols + piece - 1) / piece) <= kTileFewPieces && B < kTileFewIds;
  return few ? kDenseTileLeast : 2 * kDenseTileLeast;
}
// Most tiles of any batch of up to max_batch rows.
int64_t dense_tiles_most(int cols, int64_t max_batch) {
  const int64_t few = std::min<int64_t>({max_batch, kTileFewIds - 1, kTileFewPieces / ((cols + 7) / 8)});
  return std::max((few + kDenseTileLeast - 1) / kDenseTileLeast,
                  (max_batch + 2 * kDenseTileLeast - 1) / (2 * kDenseTileLeast));
}

void launch_dense_sum(const DenseWork& ws, int sorted, int B, const tt_emb_matrix& grad, float scale,
                      const tt_emb_matrix& out, bool add, hipStream_t st) {
  const uint32_t none = (uint32_t)out.rows;
  const int tile = dense_tile(B, grad.cols, grad.type);
  const int64_t tiles = (B + tile - 1) / tile;
  with_type(grad.type, [&](auto ti) {
    with_type(out.type, [&](auto to) {
      using TI = decltype(ti);
      using TO = decltype(to);
      auto launch = [&](auto kernel, const Lanes& ln) {
        kernel<<<grid_of(tiles, ln), kDenseThreads, 0, st>>>(ws.sort.key[sorted], ws.sort.val[sorted], B, tile, none,
                                                             (const TI*)grad.data, grad.ld, grad.cols, ln, scale,
                                                             (TO*)out.data, out.ld, ws.head, ws.tail, ws.stride,
                                                             ws.starts);
      };
      auto sums = [&](auto vec, auto wave) {
        Lanes ln = lanes_of(grad.cols, vec());
        if (wave()) ln.lanes = std::max(ln.lanes, 6);
        if (add) launch(k_dense_sum<TI, TO, vec(), true, wave()>, ln);
        else launch(k_dense_sum<TI, TO, vec(), false, wave()>, ln);
      };
      if (grad.cols >= kWave || B <= kNarrowIds)
        with_wave_piece<TI>(grad.cols, [&](auto vec) { sums(vec, std::true_type{}); });
      else
        with_piece<TI>(grad.cols, [&](auto vec) { sums(vec, std::false_type{}); });
    });
  });
}

void launch_dense_join(const DenseWork& ws, int sorted, int B, int tile, float scale, const tt_emb_matrix& out, bool add,
                       hipStream_t st) {
  const uint32_t none = (uint32_t)out.rows;
  const int tiles = (B + tile - 1) / tile;
  int lanes = 1;
  while (lanes < kJoinLanes && lanes * 4 < out.cols) lanes *= 2;
  with_type(out.type, [&](auto to) {
    using TO = decltype(to);
    const dim3 grid((unsigned)std::min((tiles + kJoinTiles - 1) / kJoinTiles, 1 << 11),
                    (unsigned)(out.cols + kJoinCols - 1) / kJoinCols);
    auto launch = [&](auto kernel) {
      kernel<<<grid, kJoinThreads, 0, st>>>(ws.sort.key[sorted], B, tile, none, out.cols, scale, (TO*)out.data, out.ld,
                                            ws.head, ws.tail, ws.stride, ws.starts, lanes);
    };
    if (add) launch(k_dense_join<TO, true>);
    else launch(k_dense_join<TO, false>);
  });
}

}  // namespace ttemb
