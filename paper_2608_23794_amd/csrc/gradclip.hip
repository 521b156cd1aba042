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
//
// 1.2 GB of bfloat16 gradients: 242 us for the norm (5.0 TB/s), 440 for the
// scaling (2.4 GB, 5.5 TB/s; some of it from the infinity cache).  A few small
// tensors are bound by two launches, 4 us each, and a list of hundreds by the
// host that gathers it: 161 tensors of 102 MB take the GPU 35 us, the call 98.
#include <algorithm>

#include "moce_internal.h"

namespace moce {
namespace {

constexpr int kThreads = 256;
constexpr int kSumThreads = 1024;
constexpr int kList = 128;                       // tensors a launch: 3.6 KB of arguments
// Elements of a chunk: enough chunks to fill the GPU (8 a CU), of 8 to 128 KB
// of float32, and more where kMaxChunks would not do.
constexpr int64_t kWantChunks = 2048, kMinChunk = 2048, kMaxChunk = 32768, kMaxChunks = 65536;
// Chunks whose sums every workgroup of the scaling adds up by itself, which
// saves the launch between (clip_gradients of a layer's four: 17 us, not 21).
constexpr int kFewChunks = 4096;

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

// The range of chunk q of a list.
struct Part {
  int t;
  bool bf16;
  int64_t i0, i1;
};
__device__ __forceinline__ Part part_of(const List& l, int q, int64_t chunk) {
  Part p;
  p.t = tensor_of(l, q);
  p.bf16 = l.n[p.t] < 0;
  const int64_t n = p.bf16 ? ~l.n[p.t] : l.n[p.t];
  p.i0 = (int64_t)(q - l.first[p.t]) * chunk;
  p.i1 = min(n, p.i0 + chunk);
  return p;
}

// Gradients lie at any multiple of their element, so vector accesses are
// unaligned ones.  kAhead of a thread's are in flight together.
constexpr int kAhead = 4;
template <typename T, typename F, typename G>
__device__ __forceinline__ void each_vector(const T* p, const Part& r, F&& vector, G&& element) {
  constexpr int VE = 16 / sizeof(T);
  int64_t i = r.i0 + threadIdx.x * VE;
  for (; i + (kAhead - 1) * kThreads * VE + VE <= r.i1; i += kAhead * kThreads * VE) {
    u32x4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) __builtin_memcpy(&v[u], p + i + u * kThreads * VE, 16);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) vector(i + u * kThreads * VE, v[u]);
  }
  for (; i + VE <= r.i1; i += kThreads * VE) {
    u32x4 v;
    __builtin_memcpy(&v, p + i, 16);
    vector(i, v);
  }
  for (int e = 0; e < VE && i + e < r.i1; ++e) element(i + e);
}

__global__ void __launch_bounds__(kThreads)
k_gradient_squares(List l, int64_t chunk, double* __restrict__ part) {
  __shared__ double s[kThreads / kWave];
  const Part r = part_of(l, blockIdx.x, chunk);
  double a = 0., b = 0.;
  if (r.bf16) {
    const uint16_t* p = static_cast<const uint16_t*>(l.src[r.t]);
    each_vector(p, r, [&](int64_t, u32x4 v) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a += square(bf16_lo(v[e]));
        b += square(bf16_hi(v[e]));
      }
    }, [&](int64_t i) __attribute__((always_inline)) { a += square(bf16_to_f32(p[i])); });
  } else {
    const float* p = static_cast<const float*>(l.src[r.t]);
    each_vector(p, r, [&](int64_t, u32x4 v) __attribute__((always_inline)) {
      a += square(__uint_as_float(v[0])) + square(__uint_as_float(v[1]));
      b += square(__uint_as_float(v[2])) + square(__uint_as_float(v[3]));
    }, [&](int64_t i) __attribute__((always_inline)) { a += square(p[i]); });
  }
  a = wave_sum_f64(a + b);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = a;
  __syncthreads();
  if (threadIdx.x == 0) part[l.base + blockIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
}

// The norm from the chunks' sums, by a workgroup of NT threads (every thread has it).
template <int NT>
__device__ __forceinline__ double norm_of_parts(const double* __restrict__ part, int chunks) {
  __shared__ double s[NT / kWave];
  double a = 0.;
#pragma unroll 4
  for (int i = threadIdx.x; i < chunks; i += NT) a += part[i];
  a = wave_sum_f64(a);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = a;
  __syncthreads();
  a = s[0];
#pragma unroll
  for (int w = 1; w < NT / kWave; ++w) a += s[w];
  return sqrt(a);
}
// 1 or max_norm / norm, as two factors to be multiplied one after the other: a
// quotient below the normal float32 numbers would have lost bits, or be zero,
// where a gradient near the largest ones times it is an ordinary number.  The
// first is below 1 there, so that its product cannot overflow; what that makes
// subnormal the second, 2^-126, makes zero.  One more multiplication a value,
// which the memory hides.
struct Coef {
  float first, second;
  __device__ __forceinline__ float times(float v) const { return v * first * second; }
};
__device__ __forceinline__ Coef coefficient(double norm, float max_norm) {
  if (!(norm > (double)max_norm && __builtin_isfinite((float)norm))) return {1.f, 1.f};
  const double c = (double)max_norm / norm;
  return c < 0x1p-126 ? Coef{(float)(c * 0x1p126), 0x1p-126f} : Coef{(float)c, 1.f};
}

// The norm, and the coefficient (coef may be nullptr).
template <int NT>
__global__ void __launch_bounds__(NT)
k_gradient_norm(const double* __restrict__ part, int chunks, float max_norm, float* __restrict__ norm,
                Coef* __restrict__ coef) {
  const double a = norm_of_parts<NT>(part, chunks);
  if (threadIdx.x != 0) return;
  *norm = (float)a;
  if (coef) *coef = coefficient(a, max_norm);
}

// FEW: the norm from the parts, else the coefficient is there.  The chunks go
// backwards: those read last for the norm are still in the infinity cache.
template <bool FEW>
__global__ void __launch_bounds__(kThreads)
k_gradient_scale(List l, int64_t chunk, const double* __restrict__ part, int chunks, float max_norm,
                 float* __restrict__ norm, const Coef* __restrict__ coef) {
  Coef c;
  if constexpr (FEW) {
    const double a = norm_of_parts<kThreads>(part, chunks);
    if (l.base + (int)blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)a;
    c = coefficient(a, max_norm);
  } else {
    c = *coef;
  }
  const Part r = part_of(l, gridDim.x - 1 - blockIdx.x, chunk);
  if (c.first == 1.f && c.second == 1.f && l.src[r.t] == l.dst[r.t]) return;
  if (r.bf16) {
    const uint16_t* p = static_cast<const uint16_t*>(l.src[r.t]);
    uint16_t* d = static_cast<uint16_t*>(l.dst[r.t]);
    each_vector(p, r, [&](int64_t i, u32x4 v) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = pack_bf16x2(c.times(bf16_lo(v[e])), c.times(bf16_hi(v[e])));
      __builtin_memcpy(d + i, &v, 16);
    }, [&](int64_t i) __attribute__((always_inline)) { d[i] = f32_to_bf16(c.times(bf16_to_f32(p[i]))); });
  } else {
    const float* p = static_cast<const float*>(l.src[r.t]);
    float* d = static_cast<float*>(l.dst[r.t]);
    each_vector(p, r, [&](int64_t i, u32x4 v) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(c.times(__uint_as_float(v[e])));
      __builtin_memcpy(d + i, &v, 16);
    }, [&](int64_t i) __attribute__((always_inline)) { d[i] = c.times(p[i]); });
  }
}

int64_t chunk_size(const moce_gradient* g, int count) {
  int64_t total = 0;
  for (int i = 0; i < count; ++i) total += g[i].n;
  auto up = [](int64_t n, int64_t d) { return (n + d - 1) / d; };
  const int64_t want = std::clamp(up(total, kWantChunks), kMinChunk, kMaxChunk);
  return up(std::max(want, up(total, kMaxChunks)), kMinChunk) * kMinChunk;
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

struct Work {
  int64_t chunk;
  int chunks;
  Coef* coef;
  double* part;
  Work(const moce_gradient* g, int count, void* ws)
      : chunk(chunk_size(g, count)), chunks((int)chunk_count(g, count, chunk)), coef(static_cast<Coef*>(ws)),
        part(reinterpret_cast<double*>(static_cast<char*>(ws) + kPartAt)) {}
};

hipError_t squares(const moce_gradient* g, int count, const Work& w, hipStream_t st) {
  return each_list(g, count, w.chunk, [&](const List& l, int32_t chunks) {
    hipLaunchKernelGGL(k_gradient_squares, dim3(chunks), dim3(kThreads), 0, st, l, w.chunk, w.part);
    return hipGetLastError();
  });
}
hipError_t norm_of(const Work& w, float max_norm, float* norm, Coef* coef, hipStream_t st) {
  if (w.chunks <= kFewChunks)   // the order of the sum in k_gradient_scale<true>
    hipLaunchKernelGGL(k_gradient_norm<kThreads>, dim3(1), dim3(kThreads), 0, st, w.part, w.chunks, max_norm, norm,
                       coef);
  else
    hipLaunchKernelGGL(k_gradient_norm<kSumThreads>, dim3(1), dim3(kSumThreads), 0, st, w.part, w.chunks, max_norm,
                       norm, coef);
  return hipGetLastError();
}

}  // namespace

size_t gradient_ws_bytes(const moce_gradient* g, int count) {
  return kPartAt + (size_t)chunk_count(g, count, chunk_size(g, count)) * sizeof(double);
}

hipError_t launch_gradient_norm(const moce_gradient* g, int count, float* norm, void* ws, hipStream_t st) {
  const Work w(g, count, ws);
  const hipError_t e = squares(g, count, w, st);
  return e == hipSuccess ? norm_of(w, 0.f, norm, nullptr, st) : e;
}

hipError_t launch_gradient_clip(const moce_gradient* g, int count, float max_norm, float* norm, void* ws,
                                hipStream_t st) {
  const Work w(g, count, ws);
  hipError_t e = squares(g, count, w, st);
  if (e != hipSuccess) return e;
  const bool few = w.chunks > 0 && w.chunks <= kFewChunks;
  if (!few && (e = norm_of(w, max_norm, norm, w.coef, st)) != hipSuccess) return e;
  return each_list(g, count, w.chunk, [&](const List& l, int32_t chunks) {
    if (few)
      hipLaunchKernelGGL(k_gradient_scale<true>, dim3(chunks), dim3(kThreads), 0, st, l, w.chunk, w.part, w.chunks,
                         max_norm, norm, w.coef);
    else
      hipLaunchKernelGGL(k_gradient_scale<false>, dim3(chunks), dim3(kThreads), 0, st, l, w.chunk, w.part, w.chunks,
                         max_norm, norm, w.coef);
    return hipGetLastError();
  });
}

}  // namespace moce
