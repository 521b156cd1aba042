// Group norm with an activation, and its gradients.
//
// Per image and group, mean and rstd = 1 / sqrt(variance + eps) over the
// group's channels and positions; y = act(scale (x - mean) rstd + shift).
// Bound by memory: x is read for the statistics and once more for y (dx: x and
// dy twice), which the infinity cache serves where a tensor fits it.
//
// A tensor is cut into parts: an image's positions in `chunks` of `len`.
// Sums go by channel, a part each, whatever the groups are (the gradients of
// scale and shift want them by channel anyway); a second kernel joins the parts
// and channels of a group, and a third one writes the elements.
//
// Variance: a thread sums x - p and its square about p, the first value it
// meets, so that the square of a large mean is never subtracted from a sum of
// squares: with m values S2 - S1^2 / m loses at most m roundings of the
// deviations' own sum, since p is one of them.  Threads and parts are joined
// through their means, in float64, and squared deviations.
#include "product.h"

namespace moce {
namespace {

// A part's mean and squared deviations.
struct Part {
  double mean;
  float m2;
};
// Part (b, c, k) lies at b sb + c sc + k sk, an element of V.
struct Parts {
  void* p;
  int64_t sb, sc, sk;
  template <typename V>
  __device__ __forceinline__ V& at(int64_t b, int c, int k) const {
    return static_cast<V*>(p)[b * sb + c * sc + k * sk];
  }
};

struct NormArgs {
  const void *x, *dy;
  void *y, *dx;
  const float *scale, *shift;
  float* stats;              // [2][B G] means, rstd
  Parts parts;               // of Part; of the backward float2, sums of dz and dz h
  float2* sums;              // [B][C] sums of dz and dz h
  float2* means;             // [B G] means of t and t h
  float *dscale, *dshift;
  int64_t B;
  int C, G, cg, hw, len, chunks, act;
  int tx;                    // threads across a row (channels-last), lanes a plane
  float eps;
};

// Count, mean and squared deviations of some values.
struct Moments {
  float n, m2;
  double mean;
};
__device__ __forceinline__ Moments join(const Moments& a, const Moments& b) {
  const float n = a.n + b.n;
  if (b.n == 0.f) return a;
  if (a.n == 0.f) return b;
  const double d = b.mean - a.mean;
  const float e = (float)d, f = b.n / n;
  return Moments{n, a.m2 + b.m2 + e * e * a.n * f, fma(d, (double)f, a.mean)};
}
// From n values' sums about p.
__device__ __forceinline__ Moments moments(float n, float p, float s1, float s2) {
  if (n == 0.f) return Moments{0.f, 0.f, 0.};
  const float m = s1 / n;
  return Moments{n, fmaxf(fmaf(-s1, m, s2), 0.f) + (s2 - s2), (double)p + (double)m};   // NaN and infinity stay NaN
}

// What a channel's elements go through.
struct Channel {
  float mean, rstd, scale, shift;
};
__device__ __forceinline__ Channel channel(const NormArgs& a, int64_t b, int c) {
  const int64_t at = b * a.G + c / a.cg;
  return Channel{a.stats[at], a.stats[a.B * a.G + at], a.scale ? a.scale[c] : 1.f, a.shift ? a.shift[c] : 0.f};
}
// h and dz of an element
template <typename T>
__device__ __forceinline__ float2 h_dz(const Channel& q, float x, float dy, int act) {
  const float h = (x - q.mean) * q.rstd;
  return make_float2(h, act == MOCE_ACT_NONE ? dy : act_gradient<T>(fmaf(h, q.scale, q.shift), dy, act));
}

template <typename T>
__device__ __forceinline__ void load_n(const T* p, int n, float (&v)[8]) {
  if (n == 8) {
    load8(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? Elem<T>::to_f(p[i]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store_n(T* p, int n, const float (&v)[8]) {
  if (n == 8) {
    store8(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) p[i] = Elem<T>::from_f(v[i]);
}

// ---- channels-last: a thread holds eight channels of every `down`-th row of a part ----

// f(image, part, first row, end, first channel, channels) for the parts of the launch
template <typename F>
__device__ __forceinline__ void each_rows(const NormArgs& a, F&& f) {
  const int x = threadIdx.x % a.tx, c = (blockIdx.y * a.tx + x) * 8;
  const bool in = (int)threadIdx.x / a.tx < kThreads / a.tx;
  for (int64_t u = blockIdx.x; u < a.B * a.chunks; u += gridDim.x) {
    const int64_t b = u / a.chunks;
    const int k = (int)(u - b * a.chunks), r0 = k * a.len, r1 = min(a.hw, r0 + a.len);
    f(b, k, r0 + (int)threadIdx.x / a.tx, r1, c, in ? min(8, a.C - c) : 0);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_sums_rows(NormArgs a) {
  __shared__ Moments s[kThreads][8 + 1];
  const int down = kThreads / a.tx;
  each_rows(a, [&](int64_t b, int k, int r, int r1, int c, int n) __attribute__((always_inline)) {
    const T* x = static_cast<const T*>(a.x) + (b * a.hw) * a.C + c;
    float p[8] = {}, s1[8] = {}, s2[8] = {}, m = 0.f;
    if (n > 0 && r < r1) {
      load_n(x + (int64_t)r * a.C, n, p);
      for (; r < r1; r += down, m += 1.f) {
        float v[8];
        load_n(x + (int64_t)r * a.C, n, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = v[i] - p[i];
          s1[i] += d;
          s2[i] = fmaf(d, d, s2[i]);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) s[threadIdx.x][i] = moments(m, p[i], s1[i], s2[i]);
    __syncthreads();
    for (int q = threadIdx.x; q < 8 * a.tx; q += kThreads) {
      const int cc = blockIdx.y * a.tx * 8 + q;
      if (cc >= a.C) continue;
      Moments t = s[q / 8][q % 8];
      for (int d = 1; d < down; ++d) t = join(t, s[d * a.tx + q / 8][q % 8]);
      a.parts.at<Part>(b, cc, k) = Part{t.mean, t.m2};
    }
  });
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_apply_rows(NormArgs a) {
  const int down = kThreads / a.tx;
  each_rows(a, [&](int64_t b, int, int r, int r1, int c, int n) __attribute__((always_inline)) {
    if (n <= 0) return;
    Channel q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = channel(a, b, min(c + i, a.C - 1));
    const int64_t base = b * a.hw * a.C + c;
    for (; r < r1; r += down) {
      const int64_t at = base + (int64_t)r * a.C;
      float v[8];
      load_n(static_cast<const T*>(a.x) + at, n, v);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = act_value<T>(fmaf((v[i] - q[i].mean) * q[i].rstd, q[i].scale, q[i].shift), a.act);
      store_n(static_cast<T*>(a.y) + at, n, v);
    }
  });
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_dsums_rows(NormArgs a) {
  __shared__ float2 s[kThreads][8 + 1];
  const int down = kThreads / a.tx;
  each_rows(a, [&](int64_t b, int k, int r, int r1, int c, int n) __attribute__((always_inline)) {
    float s0[8] = {}, s1[8] = {};
    if (n > 0) {
      Channel q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = channel(a, b, min(c + i, a.C - 1));
      const int64_t base = b * a.hw * a.C + c;
      for (; r < r1; r += down) {
        const int64_t at = base + (int64_t)r * a.C;
        float v[8], d[8];
        load_n(static_cast<const T*>(a.x) + at, n, v);
        load_n(static_cast<const T*>(a.dy) + at, n, d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 e = h_dz<T>(q[i], v[i], d[i], a.act);
          s0[i] += e.y;
          s1[i] = fmaf(e.x, e.y, s1[i]);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) s[threadIdx.x][i] = make_float2(s0[i], s1[i]);
    __syncthreads();
    for (int q = threadIdx.x; q < 8 * a.tx; q += kThreads) {
      const int cc = blockIdx.y * a.tx * 8 + q;
      if (cc >= a.C) continue;
      float2 t = s[q / 8][q % 8];
      for (int d = 1; d < down; ++d) {
        const float2 o = s[d * a.tx + q / 8][q % 8];
        t.x += o.x, t.y += o.y;
      }
      a.parts.at<float2>(b, cc, k) = t;
    }
  });
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_dx_rows(NormArgs a) {
  const int down = kThreads / a.tx;
  each_rows(a, [&](int64_t b, int, int r, int r1, int c, int n) __attribute__((always_inline)) {
    if (n <= 0) return;
    Channel q[8];
    float2 m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int cc = min(c + i, a.C - 1);
      q[i] = channel(a, b, cc);
      m[i] = a.means[b * a.G + cc / a.cg];
    }
    const int64_t base = b * a.hw * a.C + c;
    for (; r < r1; r += down) {
      const int64_t at = base + (int64_t)r * a.C;
      float v[8], d[8];
      load_n(static_cast<const T*>(a.x) + at, n, v);
      load_n(static_cast<const T*>(a.dy) + at, n, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 e = h_dz<T>(q[i], v[i], d[i], a.act);
        v[i] = q[i].rstd * (fmaf(q[i].scale, e.y, -m[i].x) - e.x * m[i].y);
      }
      store_n(static_cast<T*>(a.dx) + at, n, v);
    }
  });
}

// ---- channels-first: tx lanes take a plane's part, eight positions each ------------

// f(image, channel, part, first position, end) for the planes' parts of the launch;
// all lanes of a wave call it together
template <typename F>
__device__ __forceinline__ void each_planes(const NormArgs& a, F&& f) {
  const int64_t parts = a.B * a.C * a.chunks, per = kThreads / a.tx;
  for (int64_t u0 = blockIdx.x * per; u0 < parts; u0 += gridDim.x * per) {
    const int64_t u = u0 + threadIdx.x / a.tx, plane = min(u, parts - 1) / a.chunks, b = plane / a.C;
    const int k = (int)(min(u, parts - 1) - plane * a.chunks), p0 = k * a.len;
    const int p1 = u < parts ? min(a.hw, p0 + a.len) : p0;
    f(b, (int)(plane - b * a.C), k, p0 + (int)(threadIdx.x % a.tx) * 8, p1, u < parts && threadIdx.x % a.tx == 0);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_sums_planes(NormArgs a) {
  each_planes(a, [&](int64_t b, int c, int k, int p, int p1, bool first) __attribute__((always_inline)) {
    const T* x = static_cast<const T*>(a.x) + (b * a.C + c) * a.hw;
    float q = 0.f, s1 = 0.f, s2 = 0.f, m = 0.f;
    if (p < p1) q = Elem<T>::to_f(x[p]);
    for (; p < p1; p += 8 * a.tx) {
      const int n = min(8, p1 - p);
      float v[8];
      load_n(x + p, n, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = i < n ? v[i] - q : 0.f;
        s1 += d;
        s2 = fmaf(d, d, s2);
      }
      m += n;
    }
    Moments t = moments(m, q, s1, s2);
    for (int o = a.tx / 2; o > 0; o >>= 1)
      t = join(t, Moments{__shfl_xor(t.n, o, kWave), __shfl_xor(t.m2, o, kWave), __shfl_xor(t.mean, o, kWave)});
    if (first) a.parts.at<Part>(b, c, k) = Part{t.mean, t.m2};
  });
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_apply_planes(NormArgs a) {
  each_planes(a, [&](int64_t b, int c, int, int p, int p1, bool) __attribute__((always_inline)) {
    const int64_t base = (b * a.C + c) * a.hw;
    const Channel q = channel(a, b, c);
    for (; p < p1; p += 8 * a.tx) {
      const int n = min(8, p1 - p);
      float v[8];
      load_n(static_cast<const T*>(a.x) + base + p, n, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = act_value<T>(fmaf((v[i] - q.mean) * q.rstd, q.scale, q.shift), a.act);
      store_n(static_cast<T*>(a.y) + base + p, n, v);
    }
  });
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_dsums_planes(NormArgs a) {
  each_planes(a, [&](int64_t b, int c, int k, int p, int p1, bool first) __attribute__((always_inline)) {
    const int64_t base = (b * a.C + c) * a.hw;
    const Channel q = channel(a, b, c);
    float s0 = 0.f, s1 = 0.f;
    for (; p < p1; p += 8 * a.tx) {
      const int n = min(8, p1 - p);
      float v[8], d[8];
      load_n(static_cast<const T*>(a.x) + base + p, n, v);
      load_n(static_cast<const T*>(a.dy) + base + p, n, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 e = h_dz<T>(q, v[i], d[i], a.act);
        s0 += i < n ? e.y : 0.f;
        s1 += i < n ? e.x * e.y : 0.f;
      }
    }
    for (int o = a.tx / 2; o > 0; o >>= 1) {
      s0 += __shfl_xor(s0, o, kWave);
      s1 += __shfl_xor(s1, o, kWave);
    }
    if (first) a.parts.at<float2>(b, c, k) = make_float2(s0, s1);
  });
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_dx_planes(NormArgs a) {
  each_planes(a, [&](int64_t b, int c, int, int p, int p1, bool) __attribute__((always_inline)) {
    const int64_t base = (b * a.C + c) * a.hw;
    const Channel q = channel(a, b, c);
    const float2 m = a.means[b * a.G + c / a.cg];
    for (; p < p1; p += 8 * a.tx) {
      const int n = min(8, p1 - p);
      float v[8], d[8];
      load_n(static_cast<const T*>(a.x) + base + p, n, v);
      load_n(static_cast<const T*>(a.dy) + base + p, n, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 e = h_dz<T>(q, v[i], d[i], a.act);
        v[i] = q.rstd * (fmaf(q.scale, e.y, -m.x) - e.x * m.y);
      }
      store_n(static_cast<T*>(a.dx) + base + p, n, v);
    }
  });
}

// ---- groups ----------------------------------------------------------------------

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// A group's statistics from its channels' parts, a wave a group.
__global__ void __launch_bounds__(kThreads)
k_norm_stats(NormArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t groups = a.B * a.G;
  for (int64_t u = blockIdx.x * (int64_t)(kThreads / kWave) + (threadIdx.x >> 6); u < groups;
       u += (int64_t)gridDim.x * (kThreads / kWave)) {
    const int64_t b = u / a.G;
    const int c0 = (int)(u - b * a.G) * a.cg, last = a.hw - (a.chunks - 1) * a.len;
    const int64_t items = (int64_t)a.cg * a.chunks;
    const double n = (double)a.cg * a.hw;
    double mean = 0.;
    for (int64_t i = lane; i < items; i += kWave) {
      const int k = (int)(i / a.cg), c = c0 + (int)(i - (int64_t)k * a.cg);
      mean += a.parts.at<Part>(b, c, k).mean * (k + 1 < a.chunks ? a.len : last);
    }
    mean = wave_sum_f64(mean) / n;
    double m2 = 0.;
    for (int64_t i = lane; i < items; i += kWave) {
      const int k = (int)(i / a.cg), c = c0 + (int)(i - (int64_t)k * a.cg);
      const Part t = a.parts.at<Part>(b, c, k);
      const double d = t.mean - mean;
      m2 += (double)t.m2 + d * d * (k + 1 < a.chunks ? a.len : last);
    }
    m2 = wave_sum_f64(m2);
    if (lane == 0) {
      a.stats[u] = (float)mean;
      a.stats[groups + u] = (float)(1. / sqrt(m2 / n + (double)a.eps));
    }
  }
}

// The sums of dz and dz h by channel of an image, and the group's means.
__global__ void __launch_bounds__(kThreads)
k_norm_dstats(NormArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t groups = a.B * a.G;
  for (int64_t u = blockIdx.x * (int64_t)(kThreads / kWave) + (threadIdx.x >> 6); u < groups;
       u += (int64_t)gridDim.x * (kThreads / kWave)) {
    const int64_t b = u / a.G;
    const int c0 = (int)(u - b * a.G) * a.cg;
    float m0 = 0.f, m1 = 0.f;
    for (int i = lane; i < a.cg; i += kWave) {
      const int c = c0 + i;
      float2 t = make_float2(0.f, 0.f);
      for (int k = 0; k < a.chunks; ++k) {
        const float2 o = a.parts.at<float2>(b, c, k);
        t.x += o.x, t.y += o.y;
      }
      a.sums[b * a.C + c] = t;
      const float q = a.scale ? a.scale[c] : 1.f;
      m0 = fmaf(q, t.x, m0), m1 = fmaf(q, t.y, m1);
    }
    m0 = wave_sum(m0), m1 = wave_sum(m1);
    const float n = (float)a.cg * (float)a.hw;
    if (lane == 0) a.means[u] = make_float2(m0 / n, m1 / n);
  }
}

// dscale and dshift: the sums over the images, 16 channels a workgroup.
__global__ void __launch_bounds__(kThreads)
k_norm_dparams(NormArgs a) {
  __shared__ float2 s[kThreads];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;
  float2 t = make_float2(0.f, 0.f);
  if (c < a.C)
#pragma unroll 4
    for (int64_t b = y; b < a.B; b += kThreads / 16) {
      const float2 o = a.sums[b * a.C + c];
      t.x += o.x, t.y += o.y;
    }
  s[threadIdx.x] = t;
  __syncthreads();
  if (y != 0 || c >= a.C) return;
#pragma unroll
  for (int i = 1; i < kThreads / 16; ++i) t.x += s[16 * i + x].x, t.y += s[16 * i + x].y;
  if (a.dshift) a.dshift[c] = t.x;
  if (a.dscale) a.dscale[c] = t.y;
}

// ---- launches --------------------------------------------------------------------

constexpr int64_t kMaxBlocks = 1 << 20, kWantBlocks = 2048;
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

struct Layout {
  bool rows;                // channels-last
  int tx, len, chunks, across;   // across: workgroups over the channels
  size_t parts, stats, sums, means, total;
};
Layout layout_of(const GroupShape& s, bool back) {
  Layout l{};
  l.rows = s.layout == MOCE_NHWC;
  if (l.rows) {
    l.tx = 1;
    while (l.tx < 32 && l.tx * 8 < s.C) l.tx *= 2;
    l.across = (int)ceil_div(s.C, l.tx * 8);
    const int down = kThreads / l.tx;
    const int64_t want = std::max<int64_t>(1, kWantBlocks / (s.B * l.across));
    l.len = (int)std::min<int64_t>(s.HW, ceil_div(std::max<int64_t>(ceil_div(s.HW, want), 4 * down), down) * down);
  } else {
    l.tx = 1;
    while (l.tx < kWave && l.tx * 8 < s.HW) l.tx *= 2;
    l.across = 1;
    const int64_t want = std::max<int64_t>(1, 4 * kWantBlocks / (s.B * s.C)), step = 8 * l.tx;
    l.len = (int)std::min<int64_t>(s.HW, ceil_div(std::max<int64_t>(ceil_div(s.HW, want), 4 * step), step) * step);
  }
  l.chunks = (int)ceil_div(s.HW, l.len);
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += up256(n);
    return here;
  };
  l.parts = take((size_t)s.B * s.C * l.chunks * (back ? sizeof(float2) : sizeof(Part)));
  l.stats = take(back ? 0 : (size_t)2 * s.B * s.G * sizeof(float));
  l.sums = take(back ? (size_t)s.B * s.C * sizeof(float2) : 0);
  l.means = take(back ? (size_t)s.B * s.G * sizeof(float2) : 0);
  l.total = at;
  return l;
}

NormArgs args_of(const GroupShape& s, const Layout& l, const void* x, const float* scale, const float* shift, char* ws) {
  NormArgs a{};
  a.x = x, a.scale = scale, a.shift = shift, a.B = s.B, a.C = (int)s.C, a.G = (int)s.G, a.cg = (int)(s.C / s.G);
  a.hw = (int)s.HW, a.len = l.len, a.chunks = l.chunks, a.act = s.act, a.tx = l.tx, a.eps = s.eps;
  a.parts.p = ws + l.parts;
  a.parts.sb = s.C * l.chunks;
  a.parts.sc = l.rows ? 1 : l.chunks, a.parts.sk = l.rows ? s.C : 1;
  return a;
}
// the grid over the parts
dim3 part_grid(const GroupShape& s, const Layout& l) {
  const int64_t n = l.rows ? s.B * l.chunks : ceil_div(s.B * s.C * l.chunks, kThreads / l.tx);
  return dim3((unsigned)std::min(n, kMaxBlocks), (unsigned)l.across);
}
dim3 group_grid(const GroupShape& s) {
  return dim3((unsigned)std::min<int64_t>(ceil_div(s.B * s.G, kThreads / kWave), kMaxBlocks));
}

template <typename T>
hipError_t forward(const GroupShape& s, const void* x, const float* scale, const float* shift, void* y, float* stats,
                   char* ws, hipStream_t st) {
  const Layout l = layout_of(s, false);
  NormArgs a = args_of(s, l, x, scale, shift, ws);
  a.y = y, a.stats = stats ? stats : reinterpret_cast<float*>(ws + l.stats);
  const dim3 grid = part_grid(s, l), block(kThreads);
  hipLaunchKernelGGL(l.rows ? k_norm_sums_rows<T> : k_norm_sums_planes<T>, grid, block, 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_norm_stats, group_grid(s), block, 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(l.rows ? k_norm_apply_rows<T> : k_norm_apply_planes<T>, grid, block, 0, st, a);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const GroupShape& s, const void* x, const float* scale, const float* shift, const float* stats,
                    const void* dy, const moce_group_norm_grads& gr, char* ws, hipStream_t st) {
  const Layout l = layout_of(s, true);
  NormArgs a = args_of(s, l, x, scale, shift, ws);
  a.dy = dy, a.dx = gr.dx, a.dscale = gr.dscale, a.dshift = gr.dshift, a.stats = const_cast<float*>(stats);
  a.sums = reinterpret_cast<float2*>(ws + l.sums), a.means = reinterpret_cast<float2*>(ws + l.means);
  const dim3 grid = part_grid(s, l), block(kThreads);
  hipLaunchKernelGGL(l.rows ? k_norm_dsums_rows<T> : k_norm_dsums_planes<T>, grid, block, 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_norm_dstats, group_grid(s), block, 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (gr.dscale || gr.dshift) {
    hipLaunchKernelGGL(k_norm_dparams, dim3((unsigned)ceil_div(s.C, 16)), block, 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (!gr.dx) return hipSuccess;
  hipLaunchKernelGGL(l.rows ? k_norm_dx_rows<T> : k_norm_dx_planes<T>, grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace

bool group_limits(const GroupShape& s) {
  return s.C <= 1 << 20 && s.HW <= INT_MAX / s.C && s.B <= (int64_t)1 << 29 &&
         s.B <= ((int64_t)1 << 38) / (s.C * s.HW);
}

size_t group_ws_bytes(const GroupShape& s) { return layout_of(s, false).total; }
size_t group_backward_ws_bytes(const GroupShape& s) { return layout_of(s, true).total; }

hipError_t launch_group_norm(const GroupShape& s, const void* x, const float* scale, const float* shift, void* y,
                             float* stats, void* ws, hipStream_t st) {
  char* base = static_cast<char*>(ws);
  return s.elem == MOCE_F32 ? forward<float>(s, x, scale, shift, y, stats, base, st)
                            : forward<uint16_t>(s, x, scale, shift, y, stats, base, st);
}

hipError_t launch_group_norm_backward(const GroupShape& s, const void* x, const float* scale, const float* shift,
                                      const float* stats, const void* dy, const moce_group_norm_grads& gr, void* ws,
                                      hipStream_t st) {
  char* base = static_cast<char*>(ws);
  return s.elem == MOCE_F32 ? backward<float>(s, x, scale, shift, stats, dy, gr, base, st)
                            : backward<uint16_t>(s, x, scale, shift, stats, dy, gr, base, st);
}

}  // namespace moce
