// The global norm of a list of gradients, and their clipping.
//
// norm = sqrt(sum g^2) over every element of every tensor, then
// g <- g max_norm / norm where the norm is larger.  Bound by memory: the
// gradients are read once for the norm and, where they are clipped, read and
// written once more.  The list travels in the kernels' arguments, kList
// tensors a launch, so nothing has to be uploaded and a captured call replays
// as it is.  Work is cut into chunks of one tensor each; a workgroup sums a
// chunk in float64 (a square of a float32 is exact there, and neither
// overflows nor vanishes) and the chunks' sums are added in a fixed order.
#include <algorithm>

#include "moce_internal.h"

namespace moce {
namespace {

constexpr int kThreads = 256;
constexpr int kSumThreads = 1024;
constexpr int kList = 128;                       // tensors a launch: 3.6 KB of arguments
constexpr int64_t kChunk = 16384;                // elements of a chunk, and
constexpr int64_t kMaxChunks = 65536;            // more of them where this many would not do

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct List {
  const void* src[kList];
  void* dst[kList];
  int64_t n[kList];         // elements; the complement (negative) for bfloat16
  int32_t first[kList + 1]; // first chunk of a tensor within the launch
  int32_t base;             // first chunk of the launch
  int32_t count;
};
static_assert(sizeof(List) <= 4000, "kernel arguments");

// The tensor of chunk q of the launch.
__device__ __forceinline__ int tensor_of(const List& l, int q) {
  int lo = 0, hi = l.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (l.first[mid] <= q)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

__device__ __forceinline__ double square(float v) { return (double)v * (double)v; }

// Gradients lie at any multiple of their element, so vector accesses are unaligned ones.
__global__ void __launch_bounds__(kThreads)
k_gradient_squares(List l, int64_t chunk, double* __restrict__ part) {
  __shared__ double s[kThreads / kWave];
  const int t = tensor_of(l, blockIdx.x);
  const bool bf16 = l.n[t] < 0;
  const int64_t n = bf16 ? ~l.n[t] : l.n[t];
  const int64_t i0 = (int64_t)(blockIdx.x - l.first[t]) * chunk, i1 = min(n, i0 + chunk);
  double a = 0., b = 0.;
  if (bf16) {
    const uint16_t* p = static_cast<const uint16_t*>(l.src[t]);
    int64_t i = i0 + threadIdx.x * 8;
    for (; i + 8 <= i1; i += kThreads * 8) {
      u32x4 v;
      __builtin_memcpy(&v, p + i, 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a += square(bf16_lo(v[e]));
        b += square(bf16_hi(v[e]));
      }
    }
    for (int e = 0; e < 8 && i + e < i1; ++e) a += square(bf16_to_f32(p[i + e]));
  } else {
    const float* p = static_cast<const float*>(l.src[t]);
    int64_t i = i0 + threadIdx.x * 4;
    for (; i + 4 <= i1; i += kThreads * 4) {
      float v[4];
      __builtin_memcpy(v, p + i, 16);
      a += square(v[0]) + square(v[1]);
      b += square(v[2]) + square(v[3]);
    }
    for (int e = 0; e < 4 && i + e < i1; ++e) a += square(p[i + e]);
  }
  a = wave_sum_f64(a + b);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = a;
  __syncthreads();
  if (threadIdx.x == 0) part[l.base + blockIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
}

// The norm, and the coefficient 1 or max_norm / norm (coef may be nullptr).
__global__ void __launch_bounds__(kSumThreads)
k_gradient_norm(const double* __restrict__ part, int chunks, float max_norm, float* __restrict__ norm,
                float* __restrict__ coef) {
  __shared__ double s[kSumThreads / kWave];
  double a = 0.;
  for (int i = threadIdx.x; i < chunks; i += kSumThreads) a += part[i];
  a = wave_sum_f64(a);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = a;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kSumThreads / kWave; ++w) a += s[w];
  a = sqrt(a);
  const float f = (float)a;
  *norm = f;
  if (coef) *coef = a > (double)max_norm && __builtin_isfinite(f) ? (float)((double)max_norm / a) : 1.f;
}

__global__ void __launch_bounds__(kThreads)
k_gradient_scale(List l, int64_t chunk, const float* __restrict__ coef) {
  const float c = *coef;
  const int t = tensor_of(l, blockIdx.x);
  if (c == 1.f && l.src[t] == l.dst[t]) return;
  const bool bf16 = l.n[t] < 0;
  const int64_t n = bf16 ? ~l.n[t] : l.n[t];
  const int64_t i0 = (int64_t)(blockIdx.x - l.first[t]) * chunk, i1 = min(n, i0 + chunk);
  if (bf16) {
    const uint16_t* p = static_cast<const uint16_t*>(l.src[t]);
    uint16_t* d = static_cast<uint16_t*>(l.dst[t]);
    int64_t i = i0 + threadIdx.x * 8;
    for (; i + 8 <= i1; i += kThreads * 8) {
      u32x4 v;
      __builtin_memcpy(&v, p + i, 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = pack_bf16x2(bf16_lo(v[e]) * c, bf16_hi(v[e]) * c);
      __builtin_memcpy(d + i, &v, 16);
    }
    for (int e = 0; e < 8 && i + e < i1; ++e) d[i + e] = f32_to_bf16(bf16_to_f32(p[i + e]) * c);
  } else {
    const float* p = static_cast<const float*>(l.src[t]);
    float* d = static_cast<float*>(l.dst[t]);
    int64_t i = i0 + threadIdx.x * 4;
    for (; i + 4 <= i1; i += kThreads * 4) {
      float v[4];
      __builtin_memcpy(v, p + i, 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= c;
      __builtin_memcpy(d + i, v, 16);
    }
    for (int e = 0; e < 4 && i + e < i1; ++e) d[i + e] = p[i + e] * c;
  }
}

// Elements of a chunk: a multiple of a workgroup's vector accesses.
int64_t chunk_size(const moce_gradient* g, int count) {
  int64_t total = 0;
  for (int i = 0; i < count; ++i) total += g[i].n;
  const int64_t want = (total + kMaxChunks - 1) / kMaxChunks;
  return std::max(kChunk, (want + 2047) / 2048 * 2048);
}
int64_t chunk_count(const moce_gradient* g, int count, int64_t chunk) {
  int64_t c = 0;
  for (int i = 0; i < count; ++i) c += (g[i].n + chunk - 1) / chunk;
  return c;
}

// f(list, chunks of it) for every kList tensors that hold anything
template <typename F>
hipError_t each_list(const moce_gradient* g, int count, int64_t chunk, F&& f) {
  List l;
  l.base = 0;
  for (int i = 0; i < count;) {
    l.count = 0;
    int32_t q = 0;
    for (; i < count && l.count < kList; ++i) {
      if (g[i].n == 0) continue;
      l.src[l.count] = g[i].src;
      l.dst[l.count] = g[i].dst;
      l.n[l.count] = g[i].dtype == MOCE_BF16 ? ~g[i].n : g[i].n;
      l.first[l.count++] = q;
      q += (int32_t)((g[i].n + chunk - 1) / chunk);
    }
    if (l.count == 0) break;
    l.first[l.count] = q;
    const hipError_t e = f(l, q);
    if (e != hipSuccess) return e;
    l.base += q;
  }
  return hipSuccess;
}

constexpr size_t kPartAt = 256;   // the workspace: the coefficient, then the chunks' sums

hipError_t norm_of(const moce_gradient* g, int count, float max_norm, float* norm, float* coef, double* part,
                   int64_t chunk, hipStream_t st) {
  const hipError_t e = each_list(g, count, chunk, [&](const List& l, int32_t chunks) {
    hipLaunchKernelGGL(k_gradient_squares, dim3(chunks), dim3(kThreads), 0, st, l, chunk, part);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_gradient_norm, dim3(1), dim3(kSumThreads), 0, st, part, (int)chunk_count(g, count, chunk),
                     max_norm, norm, coef);
  return hipGetLastError();
}

}  // namespace

size_t gradient_ws_bytes(const moce_gradient* g, int count) {
  return kPartAt + (size_t)chunk_count(g, count, chunk_size(g, count)) * sizeof(double);
}

hipError_t launch_gradient_norm(const moce_gradient* g, int count, float* norm, void* ws, hipStream_t st) {
  return norm_of(g, count, 0.f, norm, nullptr, reinterpret_cast<double*>(static_cast<char*>(ws) + kPartAt),
                 chunk_size(g, count), st);
}

hipError_t launch_gradient_clip(const moce_gradient* g, int count, float max_norm, float* norm, void* ws,
                                hipStream_t st) {
  const int64_t chunk = chunk_size(g, count);
  float* coef = static_cast<float*>(ws);
  const hipError_t e = norm_of(g, count, max_norm, norm, coef,
                               reinterpret_cast<double*>(static_cast<char*>(ws) + kPartAt), chunk, st);
  if (e != hipSuccess) return e;
  return each_list(g, count, chunk, [&](const List& l, int32_t chunks) {
    hipLaunchKernelGGL(k_gradient_scale, dim3(chunks), dim3(kThreads), 0, st, l, chunk, coef);
    return hipGetLastError();
  });
}

}  // namespace moce
