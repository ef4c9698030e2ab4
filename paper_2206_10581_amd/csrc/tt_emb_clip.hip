// The 2-norm over all values of many tensors, and the tensors scaled to a largest norm.  Squares and their sums are
// held in 64 bits: no square overflows or vanishes that its value did not, and the order of the sums does not show
// in the rounded result.
#include "tt_emb_internal.h"

namespace ttemb {

constexpr int kClipThreads = 256;
constexpr int kClipPiece = 8;                           // values a thread takes at once
constexpr int kClipUnit = kClipThreads * kClipPiece;    // values a block takes at once

template <class T>
__device__ __forceinline__ void load8(const T* p, float (&x)[kClipPiece]) {
  typedef T V __attribute__((ext_vector_type(kClipPiece), aligned(sizeof(T))));
  const V v = *(const V*)p;
#pragma unroll
  for (int i = 0; i < kClipPiece; ++i) x[i] = (float)v[i];
}

template <class T>
__device__ __forceinline__ void store8(T* p, const float (&x)[kClipPiece]) {
  typedef T V __attribute__((ext_vector_type(kClipPiece), aligned(sizeof(T))));
  V v;
#pragma unroll
  for (int i = 0; i < kClipPiece; ++i) v[i] = (T)x[i];
  *(V*)p = v;
}

__host__ __device__ __forceinline__ int64_t units_of(int64_t count) { return (count + kClipUnit - 1) / kClipUnit; }

// f(first value of this thread, how many it has) for a thread's share of units [u, end) of a tensor of n values
template <class F>
__device__ __forceinline__ void pieces_of(int64_t u, int64_t end, int64_t n, F&& f) {
  for (; u < end; ++u) {
    const int64_t at = u * kClipUnit + threadIdx.x * kClipPiece;
    if (at < n) f(at, (int)min((int64_t)kClipPiece, n - at));
  }
}

// The last tensor of the list that starts at or before unit `at`.
__device__ __forceinline__ int item_of(const ClipList& list, int64_t at) {
  int a = 0, b = list.n - 1;
  while (a < b) {
    const int mid = (a + b + 1) / 2;
    const bool before = list.item[mid].first <= at;
    a = before ? mid : a;
    b = before ? b : mid - 1;
  }
  return a;
}

__device__ __forceinline__ int64_t share(int64_t units, int64_t part, int64_t parts) { return units * part / parts; }

template <class T>
__device__ __forceinline__ double squares(const T* p, int64_t u, int64_t end, int64_t n) {
  double sum = 0.0;
  pieces_of(u, end, n, [&](int64_t at, int left) {
    if (left == kClipPiece) {
      float x[kClipPiece];
      load8(p + at, x);
#pragma unroll
      for (int i = 0; i < kClipPiece; ++i) sum = fma((double)x[i], (double)x[i], sum);
    } else {
      for (int i = 0; i < left; ++i) sum = fma((double)(float)p[at + i], (double)(float)p[at + i], sum);
    }
  });
  return sum;
}

// Sum over the block's threads, in thread 0.
template <int NT>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[NT / kWave];
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) v += __shfl_xor(v, d);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  double s = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < NT / kWave; ++w) s += part[w];
  return s;
}

// Block b takes the b-th of as many equal shares of the list's units as there are blocks.
__global__ __launch_bounds__(kClipThreads) void k_norm_parts(ClipList list, double* __restrict__ parts) {
  double sum = 0.0;
  int64_t u = share(list.units, blockIdx.x, gridDim.x);
  const int64_t hi = share(list.units, blockIdx.x + 1, gridDim.x);
  for (int a = item_of(list, u); u < hi; ++a) {
    const int64_t first = list.item[a].first, n = list.item[a].count, end = min(hi, first + units_of(n));
    const void* in = list.item[a].in;
    const int type = list.item[a].type;
    if (type == TT_EMB_BF16) sum += squares((const __bf16*)in, u - first, end - first, n);
    else if (type == TT_EMB_FP16) sum += squares((const _Float16*)in, u - first, end - first, n);
    else sum += squares((const float*)in, u - first, end - first, n);
    u = end;
  }
  sum = block_sum<kClipThreads>(sum);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

constexpr int kNormThreads = 1024;
__global__ __launch_bounds__(kNormThreads) void k_norm_total(const double* __restrict__ parts, int n, float scale,
                                                             float max_norm, float eps, float* __restrict__ norm,
                                                             double* __restrict__ factor) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += kNormThreads) sum += parts[i];
  sum = block_sum<kNormThreads>(sum);
  if (threadIdx.x != 0) return;
  const double all = fabs((double)scale) * sqrt(sum);
  *norm = (float)all;
  if (factor != nullptr) {
    const double ratio = (double)max_norm / (all + (double)eps);
    *factor = (double)scale * (ratio >= 1.0 ? 1.0 : ratio);  // NaN stays
  }
}

// The product is formed in 64 bits: a factor for a norm beyond 1e38 is too small for a normal fp32 number.
template <class TI, class TO>
__device__ __forceinline__ void scaled(const TI* in, TO* out, int64_t u, int64_t end, int64_t n, double f) {
  pieces_of(u, end, n, [&](int64_t at, int left) {
    if (left == kClipPiece) {
      float x[kClipPiece];
      load8(in + at, x);
#pragma unroll
      for (int i = 0; i < kClipPiece; ++i) x[i] = (float)((double)x[i] * f);
      store8(out + at, x);
    } else {
      for (int i = 0; i < left; ++i) out[at + i] = (TO)(float)((double)(float)in[at + i] * f);
    }
  });
}

template <class TI>
__device__ __forceinline__ void scaled_to(const TI* in, void* out, int out_type, int64_t u, int64_t end, int64_t n,
                                          double f) {
  if (out_type == TT_EMB_BF16) scaled(in, (__bf16*)out, u, end, n, f);
  else if (out_type == TT_EMB_FP16) scaled(in, (_Float16*)out, u, end, n, f);
  else scaled(in, (float*)out, u, end, n, f);
}

__global__ __launch_bounds__(kClipThreads) void k_clip(ClipList list, const double* __restrict__ factor) {
  const double f = *factor;
  int64_t u = share(list.units, blockIdx.x, gridDim.x);
  const int64_t hi = share(list.units, blockIdx.x + 1, gridDim.x);
  for (int a = item_of(list, u); u < hi; ++a) {
    const int64_t first = list.item[a].first, n = list.item[a].count, end = min(hi, first + units_of(n));
    const void* in = list.item[a].in;
    void* out = list.item[a].out;
    const int type = list.item[a].type, out_type = list.item[a].out_type;
    const int64_t from = u - first;
    u = end;
    if (f == 1.0 && in == out && type == out_type) continue;  // nothing changes
    if (type == TT_EMB_BF16) scaled_to((const __bf16*)in, out, out_type, from, end - first, n, f);
    else if (type == TT_EMB_FP16) scaled_to((const _Float16*)in, out, out_type, from, end - first, n, f);
    else scaled_to((const float*)in, out, out_type, from, end - first, n, f);
  }
}

int64_t clip_units(int64_t count) { return units_of(count); }
static unsigned clip_blocks(const ClipList& list) { return (unsigned)std::min<int64_t>(list.units, kClipBlocks); }

// Returns how many parts it leaves.
int launch_norm_parts(const ClipList& list, double* parts, hipStream_t st) {
  const unsigned blocks = clip_blocks(list);
  k_norm_parts<<<blocks, kClipThreads, 0, st>>>(list, parts);
  return (int)blocks;
}
void launch_norm_total(const double* parts, int n, float scale, float max_norm, float eps, float* norm, double* factor,
                       hipStream_t st) {
  k_norm_total<<<1, kNormThreads, 0, st>>>(parts, n, scale, max_norm, eps, norm, factor);
}
void launch_clip(const ClipList& list, const double* factor, hipStream_t st) {
  k_clip<<<clip_blocks(list), kClipThreads, 0, st>>>(list, factor);
}

}  // namespace ttemb
