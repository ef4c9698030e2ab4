// The 2-norm over all values of many tensors, and the tensors scaled to a largest norm.  Squares and their sums are
// held in 64 bits: no square overflows or vanishes that its value did not, and the order of the sums does not show
// in the rounded result.
//
// Both kernels are bound by the memory.  All blocks sweep over the tensors together, a unit each at a time, the second
// kernel from the end, where what the first one read last may still be in the last-level cache (300M values from bf16
// into fp32 432 us from the start, 386 from the end).
// Measured: norm of 300M fp32 values 199 us (6.0 TB/s), of 300M bf16 107 (5.6); scaled into fp32 382 (4.7 TB/s read and
// written, a copy's rate).
#include "tt_emb_internal.h"

namespace ttemb {

constexpr int kClipThreads = 256;
constexpr int kClipUnit = 4096;  // values that a block takes at once
// Most units that one block does alone, in one launch instead of two.  us a call, and alone, one block / many: norm of
// 16,000 values in 4 tensors 6.4 / 10.0 and 16.5 / 18.9, of 60,000 in 7 (18 units) 6.5 / 10.0 and 19.2 / 19.2, of 100,000 in
// 12 (30 units) 8.9 / 10.1 and 21.4 / 19.0; clipping 1000 values 6.8 / 10.7, 16,000 (7 units) 7.0 / 10.7, 60,000 12.5 / 10.8.
constexpr int kFewNorm = 24, kFewClip = 10;

// P values side by side, aligned like one
template <class T, int P>
struct Some {
  typedef T V __attribute__((ext_vector_type(P), aligned(sizeof(T))));
};

__host__ __device__ __forceinline__ int64_t units_of(int64_t count) { return (count + kClipUnit - 1) / kClipUnit; }

// This thread's share of the first min(left, kClipUnit) values at p, P at a time, all loads first: whole pieces go to
// whole(place, piece), the values of a piece that is cut off to single(place, value).
template <int P, class T, class W, class S>
__device__ __forceinline__ void unit_values(const T* p, int64_t left, W&& whole, S&& single) {
  typedef typename Some<T, P>::V V;
  constexpr int kStep = kClipThreads * P, kDeep = kClipUnit / kStep;
  const int at = threadIdx.x % kClipThreads * P;
  V v[kDeep];
  if (left >= kClipUnit) {
#pragma unroll
    for (int k = 0; k < kDeep; ++k) v[k] = *(const V*)(p + at + k * kStep);
#pragma unroll
    for (int k = 0; k < kDeep; ++k) whole(at + k * kStep, v[k]);
    return;
  }
  const int n = (int)left;
#pragma unroll
  for (int k = 0; k < kDeep; ++k)
    if (at + k * kStep + P <= n) v[k] = *(const V*)(p + at + k * kStep);
#pragma unroll
  for (int k = 0; k < kDeep; ++k)
    if (at + k * kStep + P <= n) whole(at + k * kStep, v[k]);
  const int cut = n / P * P;
  if (cut % kStep == at && cut < n)
    for (int i = cut; i < n; ++i) single(i, p[i]);
}

// Tensors of a launch: in its arguments, or in memory if they do not fit.
struct FewItems {
  ClipList list;
  __device__ __forceinline__ const ClipItem& operator[](int a) const { return list.item[a]; }
};
struct ManyItems {
  const ClipItem* __restrict__ item;
  __device__ __forceinline__ const ClipItem& operator[](int a) const { return item[a]; }
};

// The last of the tensors lo .. hi-1 that starts at or before unit u, which tensor lo does.
__device__ __forceinline__ int item_of(const FewItems& items, int lo, int hi, int64_t u) {
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    const bool before = items[mid].first <= u;
    lo = before ? mid : lo;
    hi = before ? hi : mid;
  }
  return lo;
}
// In memory: a wavefront looks at 64 places at once.
__device__ __forceinline__ int item_of(const ManyItems& items, int lo, int hi, int64_t u) {
  const int lane = threadIdx.x % kWave;
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
    const int k = __popcll(__ballot(at < hi && items[min(at, hi - 1)].first <= u)) - 1;
    lo += k * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// From one unit of a block to its next: a few tensors on (or back), or a search over what is left.  300M values in 300
// tensors 499 to 509 us with 8 to 16 steps, 537 with 3; 11M values in 290 tensors 31 to 36, 87 with steps alone.
constexpr int kItemSteps = 12;
template <class ITEMS>
__device__ __forceinline__ int next_item(const ITEMS& items, int a, int n, int64_t u) {
  for (int i = 0; i < kItemSteps; ++i, ++a)
    if (a + 1 >= n || items[a + 1].first > u) return a;
  return item_of(items, a, n, u);
}
template <class ITEMS>
__device__ __forceinline__ int earlier_item(const ITEMS& items, int a, int64_t u) {
  for (int i = 0; i < kItemSteps; ++i, --a)
    if (items[a].first <= u) return a;
  return item_of(items, 0, a + 1, u);
}

template <class T>
__device__ __forceinline__ double squares(const T* p, int64_t left) {
  constexpr int P = 16 / sizeof(T);
  double sum = 0.0;
  auto add = [&](T x) { sum = fma((double)(float)x, (double)(float)x, sum); };
  unit_values<P>(
      p, left,
      [&](int, const typename Some<T, P>::V& v) {
#pragma unroll
        for (int i = 0; i < P; ++i) add(v[i]);
      },
      [&](int, T x) { add(x); });
  return sum;
}

// Sum over the block's threads, in every thread.
template <int NT>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[NT / kWave];
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) v += __shfl_xor(v, d);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) s += part[w];
  return s;
}

// Squares of unit u, which lies in tensor a.
template <class ITEMS>
__device__ __forceinline__ double unit_squares(const ITEMS& items, int a, int64_t u) {
  const int64_t from = (u - items[a].first) * kClipUnit, left = items[a].count - from;
  const void* in = items[a].in;
  const int type = items[a].type;
  if (type == TT_EMB_BF16) return squares((const __bf16*)in + from, left);
  if (type == TT_EMB_FP16) return squares((const _Float16*)in + from, left);
  return squares((const float*)in + from, left);
}

template <class ITEMS>
__global__ __launch_bounds__(kClipThreads) void k_norm_parts(ITEMS items, int n, int64_t units,
                                                             double* __restrict__ parts) {
  double sum = 0.0;
  int64_t u = blockIdx.x;
  for (int a = item_of(items, 0, n, u); u < units; u += gridDim.x) {
    a = next_item(items, a, n, u);
    sum += unit_squares(items, a, u);
  }
  sum = block_sum<kClipThreads>(sum);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

// The norm of `n` parts, the same in every thread of every block.
template <int NT>
__device__ __forceinline__ double total_norm(const double* __restrict__ parts, int n, float scale) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += NT) sum += parts[i];
  return fabs((double)scale) * sqrt(block_sum<NT>(sum));
}

constexpr int kNormThreads = 1024;
__global__ __launch_bounds__(kNormThreads) void k_norm_total(const double* __restrict__ parts, int n, float scale,
                                                             float* __restrict__ norm) {
  const double all = total_norm<kNormThreads>(parts, n, scale);
  if (threadIdx.x == 0) *norm = (float)all;
}

// The product is formed in 64 bits: a factor for a norm beyond 1e38 is too small for a normal fp32 number.  Pieces of 16
// bytes of the wider type: what a wavefront stores at once lies together, and goes past the caches.  (With 32 bytes a
// thread 300M values from bf16 into fp32 took 635 us instead of 382, and 545 through the caches.)
template <class TI, class TO>
__device__ __forceinline__ void scaled(const TI* in, TO* out, int64_t left, double f) {
  constexpr int P = 16 / (sizeof(TI) > sizeof(TO) ? sizeof(TI) : sizeof(TO));
  typedef typename Some<TO, P>::V VO;
  unit_values<P>(
      in, left,
      [&](int at, const typename Some<TI, P>::V& v) {
        VO y;
#pragma unroll
        for (int i = 0; i < P; ++i) y[i] = (TO)(float)((double)(float)v[i] * f);
        __builtin_nontemporal_store(y, (VO*)(out + at));
      },
      [&](int at, TI x) { out[at] = (TO)(float)((double)(float)x * f); });
}

template <class TI>
__device__ __forceinline__ void scaled_to(const TI* in, void* out, int out_type, int64_t from, int64_t left, double f) {
  if (out_type == TT_EMB_BF16) scaled(in + from, (__bf16*)out + from, left, f);
  else if (out_type == TT_EMB_FP16) scaled(in + from, (_Float16*)out + from, left, f);
  else scaled(in + from, (float*)out + from, left, f);
}

template <class ITEMS>
__device__ __forceinline__ void scale_unit(const ITEMS& items, int a, int64_t u, double f) {
  const int64_t from = (u - items[a].first) * kClipUnit, left = items[a].count - from;
  const void* in = items[a].in;
  void* out = items[a].out;
  const int type = items[a].type, out_type = items[a].out_type;
  if (type == TT_EMB_BF16) scaled_to((const __bf16*)in, out, out_type, from, left, f);
  else if (type == TT_EMB_FP16) scaled_to((const _Float16*)in, out, out_type, from, left, f);
  else scaled_to((const float*)in, out, out_type, from, left, f);
}

__device__ __forceinline__ double clip_factor(double norm, float scale, float max_norm, float eps) {
  const double n = norm + (double)eps, most = (double)max_norm;
  return (double)scale * (n <= most ? 1.0 : most / n);  // 0 / 0 and inf / inf are within the limit; NaN stays
}

// Every block adds up the parts of the norm, which costs it less than a launch in between.
template <class ITEMS>
__global__ __launch_bounds__(kClipThreads) void k_clip(ITEMS items, int n, int64_t units,
                                                       bool in_place, const double* __restrict__ parts, int n_parts,
                                                       float scale, float max_norm, float eps,
                                                       float* __restrict__ norm) {
  const double all = total_norm<kClipThreads>(parts, n_parts, scale);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)all;
  const double f = clip_factor(all, scale, max_norm, eps);
  int64_t u = units - 1 - blockIdx.x;
  if (u < 0 || (in_place && f == 1.0)) return;  // nothing changes
  for (int a = item_of(items, 0, n, u); u >= 0; u -= gridDim.x) {
    a = earlier_item(items, a, u);
    scale_unit(items, a, u, f);
  }
}

// Few values: one block does all of it, four units at a time.
template <bool CLIP>
__global__ __launch_bounds__(kNormThreads) void k_norm_few(FewItems items, int n, int units, bool in_place, float scale,
                                                           float max_norm, float eps, float* __restrict__ norm) {
  const int u0 = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kClipThreads);  // a wavefront has one
  double sum = 0.0;
  for (int u = u0, a = 0; u < units; u += kNormThreads / kClipThreads) {
    while (a + 1 < n && items[a + 1].first <= u) ++a;
    sum += unit_squares(items, a, u);
  }
  const double all = fabs((double)scale) * sqrt(block_sum<kNormThreads>(sum));
  if (threadIdx.x == 0) *norm = (float)all;
  if constexpr (CLIP) {
    const double f = clip_factor(all, scale, max_norm, eps);
    if (in_place && f == 1.0) return;  // nothing changes
    for (int u = u0, a = 0; u < units; u += kNormThreads / kClipThreads) {
      while (a + 1 < n && items[a + 1].first <= u) ++a;
      scale_unit(items, a, u, f);
    }
  }
}

// Writes the tensors of a list to memory, with the unit that each starts at; `first`: that of the first one.
constexpr int kPutThreads = 192;
static_assert(kPutItems <= kPutThreads, "a thread has one tensor");
__global__ __launch_bounds__(kPutThreads) void k_put_items(PutList list, int n, int64_t first,
                                                           ClipItem* __restrict__ to) {
  __shared__ int64_t ends[kPutThreads / kWave];
  const int i = threadIdx.x, lane = i % kWave, w = i / kWave;
  const PutItem p = list.item[min(i, n - 1)];
  const int64_t count = p.count_types & ((int64_t(1) << kPutTypeBit) - 1), units = i < n ? units_of(count) : 0;
  int64_t end = units;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int64_t before = __shfl_up(end, d);
    end += lane >= d ? before : 0;
  }
  if (lane == kWave - 1) ends[w] = end;
  __syncthreads();
  for (int k = 0; k < w; ++k) end += ends[k];
  const int types = (int)(p.count_types >> kPutTypeBit);
  if (i < n) to[i] = ClipItem{p.in, p.out, count, first + end - units, types & 3, types >> 2};
}

int64_t clip_units(int64_t count) { return units_of(count); }

void launch_put_items(const PutList& list, int n, int64_t first, ClipItem* to, hipStream_t st) {
  k_put_items<<<1, kPutThreads, 0, st>>>(list, n, first, to);
}

template <class F>
static void with_items(const ClipTensors& t, F&& f) {
  if (t.many != nullptr) f(ManyItems{t.many});
  else f(FewItems{*t.few});
}

static int launch_norm_parts(const ClipTensors& t, double* parts, hipStream_t st) {  // returns how many it leaves
  const int blocks = (int)std::min<int64_t>(t.units, kClipBlocks);
  with_items(t, [&](auto items) { k_norm_parts<<<blocks, kClipThreads, 0, st>>>(items, t.n, t.units, parts); });
  return blocks;
}

void launch_norm(const ClipTensors& t, double* parts, float scale, float* norm, hipStream_t st) {
  if (t.many == nullptr && t.units <= kFewNorm) {
    k_norm_few<false><<<1, kNormThreads, 0, st>>>(FewItems{*t.few}, t.n, (int)t.units, true, scale, 0.f, 0.f, norm);
    return;
  }
  const int n = launch_norm_parts(t, parts, st);
  k_norm_total<<<1, kNormThreads, 0, st>>>(parts, n, scale, norm);
}

void launch_clip(const ClipTensors& t, double* parts, float scale, float max_norm, float eps, float* norm,
                 hipStream_t st) {
  if (t.many == nullptr && t.units <= kFewClip) {
    k_norm_few<true><<<1, kNormThreads, 0, st>>>(FewItems{*t.few}, t.n, (int)t.units, t.in_place, scale, max_norm, eps,
                                                 norm);
    return;
  }
  const int n = launch_norm_parts(t, parts, st);
  with_items(t, [&](auto items) {
    k_clip<<<n, kClipThreads, 0, st>>>(items, t.n, t.units, t.in_place, parts, n, scale, max_norm, eps, norm);
  });
}

}  // namespace ttemb
