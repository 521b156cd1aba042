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
// deviations' own sum, since p is one of them.  Threads are joined through
// their means, taken from the first value of the part, and squared deviations,
// parts in float64.
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
  int fold;                  // groups of a workgroup whose parts are joined by those who read them (0: by k_norm_stats)
  Parts group_parts;         // [B][chunks][G], as `parts`, where they are
  int params;                // workgroups of k_norm_dx_rows ahead of the others, for dscale and dshift
  int tx;                    // threads across a row (channels-last) or a plane
  int span, spans, each;     // groups in registers: channels of a workgroup, workgroups of an image; vectors of a plane
  float eps;
};

// Count, mean and squared deviations of some values.
// The mean is taken from some value of them all.
struct Moments {
  float n, mean, m2;
};
__device__ __forceinline__ Moments join(const Moments& a, const Moments& b) {
  const float n = a.n + b.n, d = b.mean - a.mean, f = n > 0.f ? b.n * __builtin_amdgcn_rcpf(n) : 0.f;
  return Moments{n, fmaf(d, f, a.mean), a.m2 + b.m2 + d * d * a.n * f};
}
// From n values' sums about p; off: p less the value that the means are taken from.
__device__ __forceinline__ Moments moments(float n, float off, float s1, float s2) {
  const float m = n > 0.f ? s1 * __builtin_amdgcn_rcpf(n) : 0.f;
  return Moments{n, n > 0.f ? off + m : 0.f, fmaxf(fmaf(-s1, m, s2), 0.f) + (s2 - s2)};   // NaN and infinity stay NaN
}

// A group's statistics from the sums of its n values' deviations from m and of their squares.
struct Group {
  float mean, rstd;
};
__device__ __forceinline__ Group group_of(double m, double s1, double s2, double n, float eps) {
  const double d = s1 / n, var = fmax((s2 - s1 * d) / n, 0.) + (s2 - s2);
  return Group{(float)(m + d), (float)(1. / sqrt(var + (double)eps))};
}

// What a channel's elements go through.
struct Channel {
  float mean, rstd, scale, shift;
};
__device__ __forceinline__ Channel channel(const NormArgs& a, const Group& g, int c) {
  return Channel{g.mean, g.rstd, a.scale ? a.scale[c] : 1.f, a.shift ? a.shift[c] : 0.f};
}
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
constexpr int kVE = Elem<T>::kVec;

template <typename T>
__device__ __forceinline__ void unpack(u32x4 u, float (&v)[kVE<T>]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(u[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] = bf16_lo(u[e]), v[2 * e + 1] = bf16_hi(u[e]);
  }
}
template <typename T>
__device__ __forceinline__ u32x4 pack(const float (&v)[kVE<T>]) {
  if constexpr (sizeof(T) == 4)
    return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  else
    return u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
}

// f(act as a constant)
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == MOCE_ACT_RELU)
    f(std::integral_constant<int, MOCE_ACT_RELU>{});
  else if (act == MOCE_ACT_GELU)
    f(std::integral_constant<int, MOCE_ACT_GELU>{});
  else if (act == MOCE_ACT_SILU)
    f(std::integral_constant<int, MOCE_ACT_SILU>{});
  else
    f(std::integral_constant<int, MOCE_ACT_NONE>{});
}

template <typename T>
__device__ __forceinline__ void store_vector(T* p, int n, const float (&v)[kVE<T>]) {
  if (n >= kVE<T>) {
    const u32x4 u = pack<T>(v);
    __builtin_memcpy(p, &u, 16);
    return;
  }
#pragma unroll
  for (int i = 0; i < kVE<T>; ++i)
    if (i < n) p[i] = Elem<T>::from_f(v[i]);
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

// dscale and dshift of 16 channels: their sums over the images, or (fold) over
// the images' parts.  A thread has a sixteenth of them, as many as 2^25, so the
// sums are float64 (a float32 sum of 65536 equal values a thread, of a million
// rows, was 6e-4 off; of 2^24 it stops growing).
__device__ __forceinline__ void sum_params(const NormArgs& a, int block, double2* s) {
  const float2* sums = a.fold ? static_cast<const float2*>(a.parts.p) : a.sums;
  const int64_t n = a.fold ? a.B * a.chunks : a.B;
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = block * 16 + x;
  double2 t = make_double2(0., 0.);
  if (c < a.C)
#pragma unroll 8
    for (int64_t i = y; i < n; i += kThreads / 16) {
      const float2 o = sums[i * a.C + c];
      t.x += o.x, t.y += o.y;
    }
  s[threadIdx.x] = t;
  __syncthreads();
  if (y != 0 || c >= a.C) return;
#pragma unroll
  for (int i = 1; i < kThreads / 16; ++i) t.x += s[16 * i + x].x, t.y += s[16 * i + x].y;
  if (a.dshift) a.dshift[c] = (float)t.x;
  if (a.dscale) a.dscale[c] = (float)t.y;
}

// ---- channels-last: a thread holds 16 bytes of channels of every `down`-th row of a part ----

constexpr int kAhead = 4;   // rows whose loads are in flight together

// Up to kVE channels at p, n of them there (WHOLE: all, aligned), of a row of
// ld; zeros behind them.  A row's last ones are read with those before them.
template <typename T, bool WHOLE>
__device__ __forceinline__ u32x4 load_row(const T* p, int n, int64_t ld) {
  if constexpr (WHOLE) return *reinterpret_cast<const u32x4*>(p);
  T t[kVE<T>] = {};
  u32x4 v;
  if (n >= kVE<T> || ld >= kVE<T>) {
    const int before = max(kVE<T> - n, 0);
    __builtin_memcpy(&v, p - before, 16);
    const int bytes = before * (int)sizeof(T);
    u32x4 u = bytes & 8 ? u32x4{v[2], v[3], 0u, 0u} : v;
    u = bytes & 4 ? u32x4{u[1], u[2], u[3], 0u} : u;
    if constexpr (sizeof(T) == 2) {
      const int bits = bytes & 2 ? 16 : 0;
      u = u32x4{__builtin_amdgcn_alignbit(u[1], u[0], bits), __builtin_amdgcn_alignbit(u[2], u[1], bits),
                __builtin_amdgcn_alignbit(u[3], u[2], bits), u[3] >> bits};
    }
    return u;
  }
#pragma unroll
  for (int i = 0; i < kVE<T>; ++i)
    if (i < n) t[i] = p[i];
  __builtin_memcpy(&v, t, 16);
  return v;
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void store_row(T* p, int n, const float (&v)[kVE<T>]) {
  if constexpr (WHOLE)
    __builtin_nontemporal_store(pack<T>(v), reinterpret_cast<u32x4*>(p));
  else
    store_vector(p, n, v);
}

// Bound by memory: 64 images of 256 channels at 56 x 56 in bfloat16 (103 MB a
// tensor), the backward's sums 34 us (206 MB, 6.1 TB/s, some of it from the
// infinity cache), its elements 49 (309 MB); two maps of 128 at 512 x 384, as
// large, forward 18 (5.5 TB/s) and 36.

// f(image, part, first row, end, first channel, channels) for the parts of the launch
template <typename T, typename F>
__device__ __forceinline__ void each_rows(const NormArgs& a, F&& f) {
  const int x = threadIdx.x % a.tx, c = (blockIdx.y * a.tx + x) * kVE<T>;
  for (int64_t u = blockIdx.x - a.params; u < a.B * a.chunks; u += gridDim.x - a.params) {
    const int64_t b = u / a.chunks;
    const int k = (int)(u - b * a.chunks), r0 = k * a.len, r1 = r0 + min(a.len, a.hw - r0);
    f(b, k, r0 + (int)threadIdx.x / a.tx, r1, c, min(kVE<T>, a.C - c));
  }
}
// f(row's element, vectors of M tensors) for rows r, r + down, ..; kAhead rows' loads together
template <typename T, bool WHOLE, int M, typename F>
__device__ __forceinline__ void over_rows(const T* const (&p)[M], int64_t base, int64_t ld, int r, int r1, int down,
                                          int n, F&& f) {
  for (; r + (kAhead - 1) * down < r1; r += kAhead * down) {
    u32x4 v[kAhead][M];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int m = 0; m < M; ++m) v[i][m] = load_row<T, WHOLE>(p[m] + base + (r + i * down) * ld, n, ld);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) f(base + (r + i * down) * ld, v[i]);
  }
  for (; r < r1; r += down) {
    u32x4 v[M];
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = load_row<T, WHOLE>(p[m] + base + r * ld, n, ld);
    f(base + r * ld, v);
  }
}

template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads)
k_norm_sums_rows(NormArgs a) {
  constexpr int VE = kVE<T>;
  __shared__ Moments s[kThreads][VE + 1];
  __shared__ float origin[32 * VE];   // tx is 32 at most
  __shared__ Part channels[32 * VE];
  const int down = kThreads / a.tx;
  each_rows<T>(a, [&](int64_t b, int k, int r, int r1, int c, int n) __attribute__((always_inline)) {
    const T* const x[1] = {static_cast<const T*>(a.x)};
    const int64_t base = b * a.hw * a.C + c;
    float first[VE] = {}, p[VE] = {}, s1[VE] = {}, s2[VE] = {}, m = 0.f;
    if (n > 0) unpack<T>(load_row<T, WHOLE>(x[0] + base + (int64_t)k * a.len * a.C, n, a.C), first);
    if (n > 0 && r < r1) {
      unpack<T>(load_row<T, WHOLE>(x[0] + base + (int64_t)r * a.C, n, a.C), p);
      over_rows<T, WHOLE, 1>(x, base, a.C, r, r1, down, n, [&](int64_t, const u32x4 (&q)[1]) __attribute__((always_inline)) {
        float v[VE];
        unpack<T>(q[0], v);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const float d = v[i] - p[i];
          s1[i] += d;
          s2[i] = fmaf(d, d, s2[i]);
        }
        m += 1.f;
      });
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VE; ++i) s[threadIdx.x][i] = moments(m, p[i] - first[i], s1[i], s2[i]);
    if (threadIdx.x < (unsigned)a.tx)
#pragma unroll
      for (int i = 0; i < VE; ++i) origin[threadIdx.x * VE + i] = first[i];
    __syncthreads();
    for (int q = threadIdx.x; q < VE * a.tx; q += kThreads) {
      const int cc = blockIdx.y * a.tx * VE + q;
      if (cc >= a.C) continue;
      Moments t = s[q / VE][q % VE];
      for (int d = 1; d < down; ++d) t = join(t, s[d * a.tx + q / VE][q % VE]);
      const Part o{(double)origin[q] + (double)t.mean, t.m2};
      if (a.fold)
        channels[q] = o;
      else
        a.parts.at<Part>(b, cc, k) = o;
    }
    if (!a.fold) return;
    __syncthreads();
    const int g = blockIdx.y * a.fold + threadIdx.x, rows = min(a.len, a.hw - k * a.len);
    if ((int)threadIdx.x < a.fold && g < a.G) {   // equal counts: the mean of the means
      const Part* o = channels + threadIdx.x * a.cg;
      double mean = 0., m2 = 0.;
      for (int i = 0; i < a.cg; ++i) mean += o[i].mean;
      mean /= a.cg;
      for (int i = 0; i < a.cg; ++i) m2 += (double)o[i].m2 + (o[i].mean - mean) * (o[i].mean - mean) * rows;
      a.group_parts.at<Part>(b, g, k) = Part{mean, (float)m2};
    }
  });
}

// Sums over an image's parts of the workgroup's groups, by all of its threads:
// sum(group, part, its sums so far), then done(group, sums) by one thread each.
template <typename V, typename S, typename D>
__device__ __forceinline__ void fold_groups(const NormArgs& a, V* s, S&& sum, D&& done) {
  const int per = kThreads / a.fold, x = threadIdx.x % a.fold, y = threadIdx.x / a.fold;
  const int g = blockIdx.y * a.fold + x;
  V v{};
  if (y < per && g < a.G)
    for (int k = y; k < a.chunks; k += per) sum(g, k, v);
  __syncthreads();
  s[threadIdx.x] = v;
  __syncthreads();
  if (y == 0 && g < a.G) {
    for (int i = 1; i < per; ++i) v.x += s[i * a.fold + x].x, v.y += s[i * a.fold + x].y;
    done(g, x, v);
  }
  __syncthreads();
}

template <typename T, bool WHOLE, bool FOLD>
__global__ void __launch_bounds__(kThreads)
k_norm_apply_rows(NormArgs a) {
  constexpr int VE = kVE<T>;
  __shared__ double2 s[kThreads];
  __shared__ Group groups[kThreads];
  const int down = kThreads / a.tx;
  each_rows<T>(a, [&](int64_t b, int chunk, int r, int r1, int c, int n) __attribute__((always_inline)) {
    if constexpr (FOLD) {
      const int last = a.hw - (a.chunks - 1) * a.len;
      fold_groups(a, s, [&](int g, int k, double2& v) __attribute__((always_inline)) {
        const Part t = a.group_parts.at<Part>(b, g, k);
        const double m = (double)(k + 1 < a.chunks ? a.len : last) * a.cg, d = t.mean - a.group_parts.at<Part>(b, g, 0).mean;
        v.x += d * m;
        v.y += (double)t.m2 + d * d * m;
      }, [&](int g, int x, const double2& v) __attribute__((always_inline)) {
        groups[x] = group_of(a.group_parts.at<Part>(b, g, 0).mean, v.x, v.y, (double)a.cg * a.hw, a.eps);
        if (chunk == 0) a.stats[b * a.G + g] = groups[x].mean, a.stats[(a.B + b) * a.G + g] = groups[x].rstd;
      });
    }
    if (n <= 0) return;
    float m[VE], f[VE], h[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const int cc = min(c + i, a.C - 1);
      Channel q;
      if constexpr (FOLD)
        q = channel(a, groups[cc / a.cg - blockIdx.y * a.fold], cc);
      else
        q = channel(a, b, cc);
      m[i] = q.mean, f[i] = q.rstd * q.scale, h[i] = q.shift;
    }
    const T* const x[1] = {static_cast<const T*>(a.x)};
    T* y = static_cast<T*>(a.y);
    with_act(a.act, [&](auto act) __attribute__((always_inline)) {
      over_rows<T, WHOLE, 1>(x, b * a.hw * a.C + c, a.C, r, r1, down, n,
                             [&](int64_t at, const u32x4 (&q)[1]) __attribute__((always_inline)) {
        float v[VE];
        unpack<T>(q[0], v);
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = act_value<T>(fmaf(v[i] - m[i], f[i], h[i]), decltype(act)::value);
        store_row<T, WHOLE>(y + at, n, v);
      });
    });
  });
}

template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 3)
k_norm_dsums_rows(NormArgs a) {
  constexpr int VE = kVE<T>;
  __shared__ float2 s[kThreads][VE + 1], channels[32 * VE];   // tx is 32 at most
  const int down = kThreads / a.tx;
  each_rows<T>(a, [&](int64_t b, int k, int r, int r1, int c, int n) __attribute__((always_inline)) {
    float s0[VE] = {}, s1[VE] = {};
    if (n > 0) {
      Channel q[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) q[i] = channel(a, b, min(c + i, a.C - 1));
      const T* const p[2] = {static_cast<const T*>(a.x), static_cast<const T*>(a.dy)};
      with_act(a.act, [&](auto act) __attribute__((always_inline)) {
        over_rows<T, WHOLE, 2>(p, b * a.hw * a.C + c, a.C, r, r1, down, n,
                               [&](int64_t, const u32x4 (&u)[2]) __attribute__((always_inline)) {
          float v[VE], d[VE];
          unpack<T>(u[0], v);
          unpack<T>(u[1], d);
#pragma unroll
          for (int i = 0; i < VE; ++i) {
            const float2 e = h_dz<T>(q[i], v[i], d[i], decltype(act)::value);
            s0[i] += e.y;
            s1[i] = fmaf(e.x, e.y, s1[i]);
          }
        });
      });
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VE; ++i) s[threadIdx.x][i] = make_float2(s0[i], s1[i]);
    __syncthreads();
    for (int q = threadIdx.x; q < VE * a.tx; q += kThreads) {
      const int cc = blockIdx.y * a.tx * VE + q;
      if (cc >= a.C) continue;
      float2 t = s[q / VE][q % VE];
      for (int d = 1; d < down; ++d) {
        const float2 o = s[d * a.tx + q / VE][q % VE];
        t.x += o.x, t.y += o.y;
      }
      a.parts.at<float2>(b, cc, k) = t;
      if (!a.fold) continue;
      const float f = a.scale ? a.scale[cc] : 1.f;
      channels[q] = make_float2(f * t.x, f * t.y);
    }
    if (!a.fold) return;
    __syncthreads();
    const int g = blockIdx.y * a.fold + threadIdx.x;
    if ((int)threadIdx.x < a.fold && g < a.G) {
      float2 t = make_float2(0.f, 0.f);
      for (int i = 0; i < a.cg; ++i) t.x += channels[threadIdx.x * a.cg + i].x, t.y += channels[threadIdx.x * a.cg + i].y;
      a.group_parts.at<float2>(b, g, k) = t;
    }
  });
}

template <typename T, bool WHOLE, bool FOLD>
__global__ void __launch_bounds__(kThreads, 3)
k_norm_dx_rows(NormArgs a) {
  constexpr int VE = kVE<T>;
  __shared__ double2 params[kThreads];
  __shared__ float2 groups[kThreads];
  float2* s = reinterpret_cast<float2*>(params);
  if ((int)blockIdx.x < a.params) {   // uniform
    if (blockIdx.y == 0) sum_params(a, blockIdx.x, params);
    return;
  }
  const int down = kThreads / a.tx;
  each_rows<T>(a, [&](int64_t b, int, int r, int r1, int c, int n) __attribute__((always_inline)) {
    if constexpr (FOLD)
      fold_groups(a, s, [&](int g, int k, float2& v) __attribute__((always_inline)) {
        const float2 t = a.group_parts.at<float2>(b, g, k);
        v.x += t.x, v.y += t.y;
      }, [&](int, int x, const float2& v) __attribute__((always_inline)) {
        const float count = (float)a.cg * (float)a.hw;
        groups[x] = make_float2(v.x / count, v.y / count);
      });
    if (n <= 0) return;
    Channel q[VE];
    float2 m[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const int cc = min(c + i, a.C - 1);
      q[i] = channel(a, b, cc);
      if constexpr (FOLD)
        m[i] = groups[cc / a.cg - blockIdx.y * a.fold];
      else
        m[i] = a.means[b * a.G + cc / a.cg];
    }
    const T* const p[2] = {static_cast<const T*>(a.x), static_cast<const T*>(a.dy)};
    T* dx = static_cast<T*>(a.dx);
    with_act(a.act, [&](auto act) __attribute__((always_inline)) {
      over_rows<T, WHOLE, 2>(p, b * a.hw * a.C + c, a.C, r, r1, down, n,
                             [&](int64_t at, const u32x4 (&u)[2]) __attribute__((always_inline)) {
        float v[VE], d[VE];
        unpack<T>(u[0], v);
        unpack<T>(u[1], d);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const float2 e = h_dz<T>(q[i], v[i], d[i], decltype(act)::value);
          v[i] = q[i].rstd * (fmaf(q[i].scale, e.y, -m[i].x) - e.x * m[i].y);
        }
        store_row<T, WHOLE>(dx + at, n, v);
      });
    });
  });
}

// ---- channels-first: tx lanes take a plane's part, eight positions each ------------
//
// Bound by memory, one load in flight a lane: two maps of 128 channels at 512 x
// 384 with SiLU, bfloat16 (101 MB a tensor) 66 us and their gradients 116,
// float32 157 and 240.

// f(image, channel, part, the lane's first position, positions from it to the
// part's end, none where that is not above 0) for the planes' parts of the
// launch; all lanes of a wave call it together.  A plane may have all of 2^31 - 1
// positions: what lies behind its end has no 32-bit number, so positions are
// 64 bits and ends are counts.
template <typename F>
__device__ __forceinline__ void each_planes(const NormArgs& a, F&& f) {
  const int64_t parts = a.B * a.C * a.chunks, per = kThreads / a.tx;
  for (int64_t u0 = blockIdx.x * per; u0 < parts; u0 += gridDim.x * per) {
    const int64_t u = u0 + threadIdx.x / a.tx, plane = min(u, parts - 1) / a.chunks, b = plane / a.C;
    const int k = (int)(min(u, parts - 1) - plane * a.chunks), p0 = k * a.len, x = threadIdx.x % a.tx;
    const int count = u < parts ? min(a.len, a.hw - p0) : 0;
    f(b, (int)(plane - b * a.C), k, (int64_t)p0 + x * 8, count - x * 8, u < parts && x == 0);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_sums_planes(NormArgs a) {
  each_planes(a, [&](int64_t b, int c, int k, int64_t p, int left, bool lead) __attribute__((always_inline)) {
    const T* x = static_cast<const T*>(a.x) + (b * a.C + c) * a.hw;
    float q = 0.f, s1 = 0.f, s2 = 0.f, m = 0.f;
    const float first = Elem<T>::to_f(x[min(k * a.len, a.hw - 1)]);
    if (left > 0) q = Elem<T>::to_f(x[p]);
    for (; left > 0; left -= 8 * a.tx, p += 8 * a.tx) {
      const int n = min(8, left);
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
    Moments t = moments(m, q - first, s1, s2);
    for (int o = a.tx / 2; o > 0; o >>= 1)
      t = join(t, Moments{__shfl_xor(t.n, o, kWave), __shfl_xor(t.mean, o, kWave), __shfl_xor(t.m2, o, kWave)});
    if (lead) a.parts.at<Part>(b, c, k) = Part{(double)first + (double)t.mean, t.m2};
  });
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_apply_planes(NormArgs a) {
  each_planes(a, [&](int64_t b, int c, int, int64_t p, int left, bool) __attribute__((always_inline)) {
    const int64_t base = (b * a.C + c) * a.hw;
    const Channel q = channel(a, b, c);
    for (; left > 0; left -= 8 * a.tx, p += 8 * a.tx) {
      const int n = min(8, left);
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
  each_planes(a, [&](int64_t b, int c, int k, int64_t p, int left, bool first) __attribute__((always_inline)) {
    const int64_t base = (b * a.C + c) * a.hw;
    const Channel q = channel(a, b, c);
    float s0 = 0.f, s1 = 0.f;
    for (; left > 0; left -= 8 * a.tx, p += 8 * a.tx) {
      const int n = min(8, left);
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
  each_planes(a, [&](int64_t b, int c, int, int64_t p, int left, bool) __attribute__((always_inline)) {
    const int64_t base = (b * a.C + c) * a.hw;
    const Channel q = channel(a, b, c);
    const float2 m = a.means[b * a.G + c / a.cg];
    for (; left > 0; left -= 8 * a.tx, p += 8 * a.tx) {
      const int n = min(8, left);
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

// ---- whole groups in registers -----------------------------------------------------
//
// Where a workgroup's threads can hold all elements of some groups, x (and dy)
// is read once: the sums, the groups' statistics and the results follow from
// the registers.  A thread holds N vectors of 16 bytes.  Variance: the mean
// first, then the deviations from it and their squares; the deviations' sum
// puts the mean right to the last bits, and takes its error out of the squares'.

// The vectors stay packed between the passes: without this the compiler keeps
// what one pass unpacked for the next, twice the registers.
template <int N>
__device__ __forceinline__ void keep_packed(u32x4 (&q)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(q[i]));
}

// Whether dz takes dy's place in the registers for the second pass: not in
// bfloat16, which would round it.
template <typename T>
constexpr bool kKeepDz = sizeof(T) == 4;

// A workgroup's number in the launch, neighbours on one XCD (their lines meet in its L2).
__device__ __forceinline__ int64_t neighbour() {
  return (int64_t)(blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
}

constexpr int kMaxSpan = 512;   // channels of a workgroup

// Channels-last: a workgroup takes `span` channels (whole groups, vectors) of
// an image; `tx` threads (a power of two) lie across them, `lanes` of which
// hold channels.
//
// What the threads of a column of vectors sum, VE sums each, is joined through
// LDS: m-th sum of column x, element e at get(m, x VE + e).
template <int NT, int M, int VE>
struct Columns {
  static constexpr int kWaves = NT / kWave;
  float s[kWaves][M][VE == 1 ? kWave : kMaxSpan];
  template <int L = M>
  __device__ __forceinline__ void put(float (&v)[M][VE], int tx) {
#pragma unroll
    for (int m = 0; m < L; ++m)
#pragma unroll
      for (int e = 0; e < VE; ++e)
        for (int o = tx; o < kWave; o <<= 1) v[m][e] += __shfl_xor(v[m][e], o, kWave);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane < tx) {
#pragma unroll
      for (int m = 0; m < L; ++m)
#pragma unroll
        for (int e = 0; e < VE; ++e) s[wave][m][lane * VE + e] = v[m][e];
    }
  }
  __device__ __forceinline__ float get(int m, int c) const {
    float t = s[0][m][c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) t += s[w][m][c];
    return t;
  }
};

// ONE: a vector's channels are of one group.  A thread then sums them all, and
// adds up its group's sums by itself.
//
// 64 images of 512 channels at 28 x 28 in bfloat16, 103 MB read and written, in
// 23 us from the infinity cache; of 256 at 56 x 56, a workgroup a CU, 46 so and
// 59 from memory (3.5 TB/s: one workgroup's reading does not overlap its writing).
template <typename T, int NT, int N, bool ONE>
__global__ void __launch_bounds__(NT)
k_norm_span(NormArgs a) {
  constexpr int VE = kVE<T>, kSums = ONE ? 1 : VE;
  __shared__ Columns<NT, 2, kSums> cols;
  __shared__ float sums[2][ONE ? 1 : kMaxSpan], mean[ONE ? 1 : kMaxSpan], rstd[ONE ? 1 : kMaxSpan];
  const int64_t u = neighbour();
  if (u >= a.B * a.spans) return;
  const int64_t b = u / a.spans;
  const int s0 = (int)(u - b * a.spans) * a.span, channels = min(a.span, a.C - s0);
  const int x = threadIdx.x % a.tx, r0 = threadIdx.x / a.tx, down = NT / a.tx;
  const bool in = x * VE < channels;
  const T* p = static_cast<const T*>(a.x) + b * a.hw * a.C + s0 + x * VE;
  u32x4 q[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q[i] = u32x4{0u, 0u, 0u, 0u};
    const int r = r0 + i * down;
    if (in && r < a.hw) q[i] = *reinterpret_cast<const u32x4*>(p + (int64_t)r * a.C);
  }
  const int c = threadIdx.x;   // this thread's channel of the span, where it has one
  const double n = (double)a.cg * a.hw;
  // The sums of the thread's group (ONE) or of its channel's group.  All of the workgroup calls it.
  auto group_sums = [&](auto two, float (&v)[2][kSums], float* t) __attribute__((always_inline)) {
    constexpr int M = decltype(two)::value ? 2 : 1;
    cols.template put<M>(v, a.tx);
    __syncthreads();
    if constexpr (ONE) {
      const int each = a.cg / VE, g0 = min(x, channels / VE - 1) / each * each;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        t[m] = 0.f;
        for (int k = 0; k < each; ++k) t[m] += cols.get(m, g0 + k);
      }
    } else {
#pragma unroll
      for (int m = 0; m < M; ++m)
        if (c < channels) sums[m][c] = cols.get(m, c);
      __syncthreads();
      const int g0 = c / a.cg * a.cg;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        t[m] = 0.f;
        if (c < channels)
          for (int k = 0; k < a.cg; ++k) t[m] += sums[m][g0 + k];
      }
    }
    __syncthreads();
  };
  float v[2][kSums] = {}, t[2];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float w[VE];
    unpack<T>(q[i], w);
#pragma unroll
    for (int e = 0; e < VE; ++e) v[0][ONE ? 0 : e] += w[e];
  }
  group_sums(std::false_type{}, v, t);
  keep_packed(q);
  const float near = t[0] / (float)n;   // the mean but for the sum's roundings
  if constexpr (!ONE) {
    if (c < channels) mean[c] = near;
    __syncthreads();
  }
  float m[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    m[e] = ONE ? near : in ? mean[x * VE + e] : 0.f;
    v[0][ONE ? 0 : e] = v[1][ONE ? 0 : e] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (!in || r0 + i * down >= a.hw) continue;
    float w[VE];
    unpack<T>(q[i], w);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float d = w[e] - m[e];
      v[0][ONE ? 0 : e] += d;
      v[1][ONE ? 0 : e] = fmaf(d, d, v[1][ONE ? 0 : e]);
    }
  }
  group_sums(std::true_type{}, v, t);
  const Group g = group_of((double)near, t[0], t[1], n, a.eps);
  const int at = s0 + (ONE ? x * VE : c);
  if (at % a.cg == 0 && at < s0 + channels && (!ONE || (int)threadIdx.x < a.tx)) {
    const int64_t to = b * a.G + at / a.cg;
    a.stats[to] = g.mean, a.stats[a.B * a.G + to] = g.rstd;
  }
  if constexpr (!ONE) {
    if (c < channels) mean[c] = g.mean, rstd[c] = g.rstd;
    __syncthreads();
  }
  if (!in) return;
  keep_packed(q);
  float f[VE], h[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    const int ch = s0 + x * VE + e;
    const float r = ONE ? g.rstd : rstd[x * VE + e];
    m[e] = ONE ? g.mean : mean[x * VE + e];
    f[e] = a.scale ? a.scale[ch] * r : r, h[e] = a.shift ? a.shift[ch] : 0.f;
  }
  T* y = static_cast<T*>(a.y) + b * a.hw * a.C + s0 + x * VE;
  with_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + i * down;
      if (r >= a.hw) continue;
      float w[VE];
      unpack<T>(q[i], w);
#pragma unroll
      for (int e = 0; e < VE; ++e) w[e] = act_value<T>(fmaf(w[e] - m[e], f[e], h[e]), decltype(act)::value);
      *reinterpret_cast<u32x4*>(y + (int64_t)r * a.C) = pack<T>(w);
    }
  });
}

// ONE: a vector's channels are of one group (half the registers of its channels).
template <typename T, int NT, int N, bool ONE>
__global__ void __launch_bounds__(NT)
k_norm_span_backward(NormArgs a) {
  constexpr int VE = kVE<T>;
  __shared__ Columns<NT, 2, VE> cols;
  __shared__ float sums[2][kMaxSpan], m0[kMaxSpan], m1[kMaxSpan];
  const int64_t u = neighbour();
  if (u >= a.B * a.spans) return;
  const int64_t b = u / a.spans;
  const int s0 = (int)(u - b * a.spans) * a.span, channels = min(a.span, a.C - s0);
  const int x = threadIdx.x % a.tx, r0 = threadIdx.x / a.tx, down = NT / a.tx;
  const bool in = x * VE < channels;
  const int64_t base = b * a.hw * a.C + s0 + x * VE;
  const T *p = static_cast<const T*>(a.x) + base, *d = static_cast<const T*>(a.dy) + base;
  u32x4 q[N], o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q[i] = o[i] = u32x4{0u, 0u, 0u, 0u};
    const int r = r0 + i * down;
    if (in && r < a.hw) {
      q[i] = *reinterpret_cast<const u32x4*>(p + (int64_t)r * a.C);
      o[i] = *reinterpret_cast<const u32x4*>(d + (int64_t)r * a.C);
    }
  }
  Channel ch[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    ch[e] = channel(a, b, min(s0 + x * VE + e, a.C - 1));
    if constexpr (ONE) ch[e].mean = ch[0].mean, ch[e].rstd = ch[0].rstd;
  }
  float v[2][VE] = {};
  with_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {   // what is not there has a dy of 0
      if (!in || r0 + i * down >= a.hw) continue;
      float w[VE], t[VE];
      unpack<T>(q[i], w);
      unpack<T>(o[i], t);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float2 z = h_dz<T>(ch[e], w[e], t[e], decltype(act)::value);
        v[0][e] += z.y;
        v[1][e] = fmaf(z.x, z.y, v[1][e]);
        t[e] = z.y;
      }
      if constexpr (kKeepDz<T>) o[i] = pack<T>(t);
    }
  });
  cols.put(v, a.tx);
  __syncthreads();
  const int c = threadIdx.x, g0 = c / a.cg * a.cg;
  if (c < channels) {
    const float2 t = make_float2(cols.get(0, c), cols.get(1, c));
    const float f = a.scale ? a.scale[s0 + c] : 1.f;
    a.sums[b * a.C + s0 + c] = t;
    sums[0][c] = f * t.x, sums[1][c] = f * t.y;
  }
  __syncthreads();
  if (c < channels) {
    float t0 = 0.f, t1 = 0.f;
    for (int k = 0; k < a.cg; ++k) t0 += sums[0][g0 + k], t1 += sums[1][g0 + k];
    const float n = (float)a.cg * (float)a.hw;
    m0[c] = t0 / n, m1[c] = t1 / n;
  }
  __syncthreads();
  if (!in || !a.dx) return;
  keep_packed(q), keep_packed(o);
  float k0[VE], k1[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) k0[e] = m0[x * VE + (ONE ? 0 : e)], k1[e] = m1[x * VE + (ONE ? 0 : e)];
  T* dx = static_cast<T*>(a.dx) + base;
  with_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + i * down;
      if (r >= a.hw) continue;
      float w[VE], t[VE];
      unpack<T>(q[i], w);
      unpack<T>(o[i], t);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float2 z = h_dz<T>(ch[e], w[e], t[e], kKeepDz<T> ? MOCE_ACT_NONE : decltype(act)::value);
        w[e] = ch[e].rstd * fmaf(-k1[e], z.x, fmaf(ch[e].scale, z.y, -k0[e]));
      }
      *reinterpret_cast<u32x4*>(dx + (int64_t)r * a.C) = pack<T>(w);
    }
  });
}

// Channels-first (64 images of 512 channels at 28 x 28 in bfloat16: 25 us, the
// gradients 44): a workgroup takes a group, tx threads (a power of two) a plane, `each` vectors of it; a thread's planes follow each other NT / tx
// apart.  Sums over a plane's threads are joined by its waves.
constexpr int kMaxPlanes = 1024;
template <typename T, int NT, int N, typename F>
__device__ __forceinline__ void each_vector(const NormArgs& a, F&& f) {   // f(vector, plane, position, last of the plane)
  int j = threadIdx.x / a.tx, i = 0;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    f(k, j, (i * a.tx + (int)threadIdx.x % a.tx) * kVE<T>, i + 1 == a.each);
    if (++i == a.each) i = 0, j += NT / a.tx;
  }
}
// A vector of a plane of hw elements at e; what is behind them is read where
// the tensor goes on, and is not used.
template <typename T>
__device__ __forceinline__ u32x4 load_vector(const T* p, int64_t e, int n, int64_t total) {
  u32x4 v = {0u, 0u, 0u, 0u};
  if (n <= 0) return v;
  if (e + kVE<T> <= total) {
    __builtin_memcpy(&v, p + e, 16);
    return v;
  }
  T t[kVE<T>] = {};
#pragma unroll
  for (int i = 0; i < kVE<T>; ++i)
    if (i < n) t[i] = p[e + i];
  __builtin_memcpy(&v, t, 16);
  return v;
}
// The sum over a workgroup, every thread has it.
template <int NT>
__device__ __forceinline__ float group_sum(float v, float* s) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < NT / kWave; ++w) v += s[w];
  return v;
}

template <typename T, int NT, int N>
__global__ void __launch_bounds__(NT)
k_norm_group(NormArgs a) {
  constexpr int VE = kVE<T>;
  __shared__ float s[NT / kWave];
  const int64_t u = neighbour();
  if (u >= a.B * a.G) return;
  const int64_t b = u / a.G, base = u * a.cg * a.hw, total = a.B * a.C * a.hw;
  const int c0 = (int)(u - b * a.G) * a.cg;
  const T* p = static_cast<const T*>(a.x);
  u32x4 q[N];
  each_vector<T, NT, N>(a, [&](int k, int j, int i, bool) __attribute__((always_inline)) {
    q[k] = load_vector(p, base + (int64_t)j * a.hw + i, j < a.cg ? a.hw - i : 0, total);
  });
  const double n = (double)a.cg * a.hw;
  float sum = 0.f;
  each_vector<T, NT, N>(a, [&](int k, int j, int i, bool) __attribute__((always_inline)) {
    const int left = j < a.cg ? a.hw - i : 0;
    float w[VE];
    unpack<T>(q[k], w);
#pragma unroll
    for (int e = 0; e < VE; ++e) sum += e < left ? w[e] : 0.f;
  });
  const float m = group_sum<NT>(sum, s) / (float)n;
  keep_packed(q);
  float s1 = 0.f, s2 = 0.f;
  each_vector<T, NT, N>(a, [&](int k, int j, int i, bool) __attribute__((always_inline)) {
    const int left = j < a.cg ? a.hw - i : 0;
    float w[VE];
    unpack<T>(q[k], w);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float d = e < left ? w[e] - m : 0.f;
      s1 += d;
      s2 = fmaf(d, d, s2);
    }
  });
  s1 = group_sum<NT>(s1, s), s2 = group_sum<NT>(s2, s);
  const Group g = group_of((double)m, s1, s2, n, a.eps);
  if (threadIdx.x == 0) a.stats[u] = g.mean, a.stats[a.B * a.G + u] = g.rstd;
  T* y = static_cast<T*>(a.y) + base;
  keep_packed(q);
  with_act(a.act, [&](auto act) __attribute__((always_inline)) {
    each_vector<T, NT, N>(a, [&](int k, int j, int i, bool) __attribute__((always_inline)) {
      const int left = j < a.cg ? a.hw - i : 0;
      if (left <= 0) return;
      const float f = a.scale ? a.scale[c0 + j] * g.rstd : g.rstd, h = a.shift ? a.shift[c0 + j] : 0.f;
      float w[VE];
      unpack<T>(q[k], w);
#pragma unroll
      for (int e = 0; e < VE; ++e) w[e] = act_value<T>(fmaf(w[e] - g.mean, f, h), decltype(act)::value);
      store_vector(y + (int64_t)j * a.hw + i, left, w);
    });
  });
}

template <typename T, int NT, int N>
__global__ void __launch_bounds__(NT)
k_norm_group_backward(NormArgs a) {
  constexpr int VE = kVE<T>, kParts = 2 * NT / kWave;
  __shared__ float2 part[kMaxPlanes + kParts];   // sums by plane and wave of it
  __shared__ float s[NT / kWave];
  const int64_t u = neighbour();
  if (u >= a.B * a.G) return;
  const int64_t b = u / a.G, base = u * a.cg * a.hw, total = a.B * a.C * a.hw;
  const int c0 = (int)(u - b * a.G) * a.cg;
  u32x4 q[N], o[N];
  each_vector<T, NT, N>(a, [&](int k, int j, int i, bool) __attribute__((always_inline)) {
    const int64_t e = base + (int64_t)j * a.hw + i;
    const int left = j < a.cg ? a.hw - i : 0;
    q[k] = load_vector(static_cast<const T*>(a.x), e, left, total);
    o[k] = load_vector(static_cast<const T*>(a.dy), e, left, total);
  });
  const float mean = a.stats[u], rstd = a.stats[a.B * a.G + u];
  auto of = [&](int j) __attribute__((always_inline)) {
    return Channel{mean, rstd, a.scale ? a.scale[c0 + j] : 1.f, a.shift ? a.shift[c0 + j] : 0.f};
  };
  const int waves = max(1, a.tx / kWave), lanes = min(a.tx, kWave);   // of a plane
  float s0 = 0.f, s1 = 0.f;
  with_act(a.act, [&](auto act) __attribute__((always_inline)) {
    each_vector<T, NT, N>(a, [&](int k, int j, int i, bool last) __attribute__((always_inline)) {
      const int left = j < a.cg ? a.hw - i : 0;
      const Channel ch = of(min(j, a.cg - 1));
      float w[VE], t[VE];
      unpack<T>(q[k], w);
      unpack<T>(o[k], t);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float2 z = h_dz<T>(ch, w[e], t[e], decltype(act)::value);
        s0 += e < left ? z.y : 0.f;
        s1 += e < left ? z.x * z.y : 0.f;
        t[e] = z.y;
      }
      if constexpr (kKeepDz<T>) o[k] = pack<T>(t);
      if (!last) return;
      for (int l = 1; l < lanes; l <<= 1) s0 += __shfl_xor(s0, l, kWave), s1 += __shfl_xor(s1, l, kWave);
      if (threadIdx.x % lanes == 0 && j < a.cg)
        part[j * waves + threadIdx.x % a.tx / kWave] = make_float2(s0, s1);
      s0 = s1 = 0.f;
    });
  });
  __syncthreads();
  float m0 = 0.f, m1 = 0.f;
  for (int j = threadIdx.x; j < a.cg; j += NT) {
    float2 t = part[j * waves];
    for (int w = 1; w < waves; ++w) t.x += part[j * waves + w].x, t.y += part[j * waves + w].y;
    a.sums[b * a.C + c0 + j] = t;
    const float f = a.scale ? a.scale[c0 + j] : 1.f;
    m0 = fmaf(f, t.x, m0), m1 = fmaf(f, t.y, m1);
  }
  const float n = (float)a.cg * (float)a.hw;
  m0 = group_sum<NT>(m0, s) / n, m1 = group_sum<NT>(m1, s) / n;
  if (!a.dx) return;
  keep_packed(q), keep_packed(o);
  T* dx = static_cast<T*>(a.dx) + base;
  with_act(a.act, [&](auto act) __attribute__((always_inline)) {
    each_vector<T, NT, N>(a, [&](int k, int j, int i, bool) __attribute__((always_inline)) {
      const int left = j < a.cg ? a.hw - i : 0;
      if (left <= 0) return;
      const Channel ch = of(j);
      float w[VE], t[VE];
      unpack<T>(q[k], w);
      unpack<T>(o[k], t);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float2 z = h_dz<T>(ch, w[e], t[e], kKeepDz<T> ? MOCE_ACT_NONE : decltype(act)::value);
        w[e] = rstd * (fmaf(ch.scale, z.y, -m0) - z.x * m1);
      }
      store_vector(dx + (int64_t)j * a.hw + i, left, w);
    });
  });
}

// ---- groups ----------------------------------------------------------------------

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// A group's statistics from its channels' parts, a workgroup a group: `down`
// threads (a power of two) share a channel's parts, which are taken about the
// group's first mean, in float64.
__device__ __forceinline__ double group_sum_f64(double v, double* s) {
  v = wave_sum_f64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}
__global__ void __launch_bounds__(kThreads)
k_norm_stats(NormArgs a, int down) {
  __shared__ double s[kThreads / kWave];
  const int64_t groups = a.B * a.G;
  const int last = a.hw - (a.chunks - 1) * a.len;
  const int across = kThreads / down, x = threadIdx.x % across, y = threadIdx.x / across;
  const double n = (double)a.cg * a.hw;
  for (int64_t u = blockIdx.x; u < groups; u += gridDim.x) {
    const int64_t b = u / a.G;
    const int c0 = (int)(u - b * a.G) * a.cg;
    const double p = a.parts.at<Part>(b, c0, 0).mean;
    double s1 = 0., s2 = 0.;
    for (int c = c0 + x; c < c0 + a.cg; c += across)
#pragma unroll 4
      for (int k = y; k < a.chunks; k += down) {
        const Part t = a.parts.at<Part>(b, c, k);
        const double m = k + 1 < a.chunks ? a.len : last, d = t.mean - p;
        s1 += d * m;
        s2 += (double)t.m2 + d * d * m;
      }
    s1 = group_sum_f64(s1, s), s2 = group_sum_f64(s2, s);
    if (threadIdx.x == 0) {
      const Group g = group_of(p, s1, s2, n, a.eps);
      a.stats[u] = g.mean, a.stats[groups + u] = g.rstd;
    }
  }
}

// The sums of dz and dz h by channel of an image, and the group's means, a
// workgroup a group: `down` threads (a power of two) share a channel's parts.
__global__ void __launch_bounds__(kThreads)
k_norm_dstats(NormArgs a, int down) {
  __shared__ float2 s[kThreads];
  __shared__ float sums[kThreads / kWave];
  const int64_t groups = a.B * a.G;
  const int across = kThreads / down, x = threadIdx.x % across, y = threadIdx.x / across;
  for (int64_t u = blockIdx.x; u < groups; u += gridDim.x) {
    const int64_t b = u / a.G;
    const int c0 = (int)(u - b * a.G) * a.cg;
    float m0 = 0.f, m1 = 0.f;
    for (int i0 = 0; i0 < a.cg; i0 += across) {
      const int i = i0 + x, c = c0 + i;
      float2 t = make_float2(0.f, 0.f);
      if (i < a.cg)
        for (int k = y; k < a.chunks; k += down) {
          const float2 o = a.parts.at<float2>(b, c, k);
          t.x += o.x, t.y += o.y;
        }
      if (down > 1) {
        __syncthreads();
        s[threadIdx.x] = t;
        __syncthreads();
        if (y == 0)
          for (int d = 1; d < down; ++d) t.x += s[d * across + x].x, t.y += s[d * across + x].y;
      }
      if (y == 0 && i < a.cg) {
        a.sums[b * a.C + c] = t;
        const float q = a.scale ? a.scale[c] : 1.f;
        m0 = fmaf(q, t.x, m0), m1 = fmaf(q, t.y, m1);
      }
    }
    m0 = group_sum<kThreads>(m0, sums), m1 = group_sum<kThreads>(m1, sums);
    const float n = (float)a.cg * (float)a.hw;
    if (threadIdx.x == 0) a.means[u] = make_float2(m0 / n, m1 / n);
  }
}

__global__ void __launch_bounds__(kThreads)
k_norm_dparams(NormArgs a) {
  __shared__ double2 s[kThreads];
  sum_params(a, blockIdx.x, s);
}

// ---- launches --------------------------------------------------------------------

// Rows: as many workgroups as run at once, three a CU (of 2048, whose threads had
// four rows each, 32 images of 100 channels at 64 x 64 took 40 us and not 31).
constexpr int64_t kMaxBlocks = 1 << 20, kWantBlocks = 768, kWantPlaneParts = 8192;
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

struct Layout {
  bool rows;                // channels-last
  int threads, n;           // of a workgroup that holds groups in registers, and their vectors; 0: none does
  int span, spans, each;
  int tx, len, chunks, across;   // across: workgroups over the channels
  int fold;
  size_t parts, group_parts, stats, sums, means, total;
};

// Vectors a thread, of the kernels there are: twice the registers a vector in
// the backward, 128 registers a thread in workgroups of 1024.
int up_vectors(int64_t n, int threads, bool back) {
  for (const int v : {1, 2, 4, 8, 16})
    if (n <= v && (threads < 1024 || v >= 4)) return v > (back || threads == 64 ? 8 : 16) ? 0 : v;
  return 0;
}

// Groups in registers: threads and vectors a thread, or none.
void in_registers(const GroupShape& s, bool back, Layout* l) {
  const int ve = s.elem == MOCE_F32 ? 4 : 8;
  const int64_t cg = s.C / s.G;
  if (s.layout == MOCE_NHWC) {
    if (s.C % ve != 0 || cg > kMaxSpan) return;
    int64_t least = cg;                       // whole groups and vectors
    while (least % ve != 0) least += cg;
    // Lines of 128 bytes where they fit, else of 64 or 32.  A workgroup of 1024
    // has a CU to itself: it reads, sums and writes one after the other, which
    // pays for whole lines only, and where every CU has one.  (Backward of 64
    // images of 512 channels at 28 x 28, 128 bytes: 49 us, 64 through parts; of
    // 256 at 56 x 56, 32 bytes: 118 and 102.)
    for (const int bytes : {128, 64, 32}) {
      const int64_t span = std::min(s.C, ceil_div(bytes / 16 * ve, least) * least), spans = ceil_div(s.C, span);
      int tx = 1;
      while (tx * ve < span) tx *= 2;
      if (span > kMaxSpan || tx > kWave) continue;
      for (const int threads : {256, 512, 1024}) {
        if (span > threads || s.B * spans * threads >= (int64_t)1 << 31) continue;
        const int n = up_vectors(ceil_div(s.HW, threads / tx), threads, back);
        if (n == 0 || (threads == 1024 && (bytes == 32 || s.B * spans < 256))) continue;
        // these spill registers
        if (threads == 1024 && back && n == 8 && cg % ve != 0) continue;
        l->threads = threads, l->n = n, l->tx = tx, l->span = (int)span, l->spans = (int)spans;
        return;
      }
    }
    return;
  }
  // a group of few elements is a few lanes' (each by itself, with a wave: slower)
  if (cg > kMaxPlanes || cg * s.HW < 512) return;
  for (const int threads : {64, 256, 1024}) {
    if (s.B * s.G * threads >= (int64_t)1 << 31) continue;
    int64_t best = INT_MAX;
    for (int tx = 1; tx <= threads; tx *= 2) {
      const int64_t each = ceil_div(s.HW, ve * tx), n = ceil_div(cg, threads / tx) * each;
      if (n < best) best = n, l->tx = tx, l->each = (int)each;
    }
    const int n = up_vectors(best, threads, back);
    if (n == 0) continue;
    l->threads = threads, l->n = n;
    return;
  }
}

Layout layout_of(const GroupShape& s, bool back) {
  Layout l{};
  l.rows = s.layout == MOCE_NHWC;
  in_registers(s, back, &l);
  if (l.threads == 0 && l.rows) {
    l.tx = 1;
    const int ve = s.elem == MOCE_F32 ? 4 : 8;
    while (l.tx < 32 && l.tx * ve < s.C) l.tx *= 2;
    l.across = (int)ceil_div(s.C, l.tx * ve);
    const int down = kThreads / l.tx;
    const int64_t want = std::max<int64_t>(1, kWantBlocks / (s.B * l.across));
    l.len = (int)std::min<int64_t>(s.HW, ceil_div(std::max<int64_t>(ceil_div(s.HW, want), 4 * down), down) * down);
  } else if (l.threads == 0) {
    l.tx = 1;
    while (l.tx < kWave && l.tx * 8 < s.HW) l.tx *= 2;
    l.across = 1;
    const int64_t want = std::max<int64_t>(1, kWantPlaneParts / (s.B * s.C)), step = 8 * l.tx;
    l.len = (int)std::min<int64_t>(s.HW, ceil_div(std::max<int64_t>(ceil_div(s.HW, want), 4 * step), step) * step);
  }
  l.chunks = l.threads ? 0 : (int)ceil_div(s.HW, l.len);
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += up256(n);
    return here;
  };
  // Few groups of few channels, whole ones in a workgroup, and few parts: joined
  // by the kernels that read them, which saves a launch (8 images of 64 channels
  // at 56 x 56: backward 21 to 17 us).  Each of their workgroups does so: of
  // many, the launch is cheaper (64 images of 256 channels: dx 58 us, not 48 and
  // 6 for the launch).
  if (l.rows && l.threads == 0) {
    const int64_t cg = s.C / s.G, width = l.tx * (s.elem == MOCE_F32 ? 4 : 8), groups = width / cg;
    if (cg <= 32 && width % cg == 0 && groups * ceil_div(s.HW, l.len) <= 2048 &&
        s.B * ceil_div(s.HW, l.len) * l.across <= 512)
      l.fold = (int)groups;
  }
  l.group_parts = take(l.fold ? (size_t)s.B * s.G * l.chunks * (back ? sizeof(float2) : sizeof(Part)) : 0);
  const size_t part = back ? sizeof(float2) : sizeof(Part);
  l.parts = take(!back && l.fold ? 0 : (size_t)s.B * s.C * l.chunks * part);
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
  a.span = l.span, a.spans = l.spans, a.each = l.each;
  a.fold = l.fold, a.group_parts = Parts{ws + l.group_parts, s.G * l.chunks, 1, s.G};
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
dim3 group_grid(const GroupShape& s) { return dim3((unsigned)std::min<int64_t>(s.B * s.G, kMaxBlocks)); }

// Threads that share a channel's parts.
int share(const NormArgs& a) {
  int down = 1;
  while (down < kThreads && down * 2 * a.cg <= kThreads && down < a.chunks) down *= 2;
  return down;
}

// f(threads, vectors) as constants, of the kernels there are
template <bool BACK, typename F>
void with_registers(const Layout& l, F&& f) {
  auto of = [&](auto threads) {
    constexpr int NT = decltype(threads)::value;
    switch (l.n) {
      case 1: if constexpr (NT < 1024) f(threads, std::integral_constant<int, 1>{}); break;
      case 2: if constexpr (NT < 1024) f(threads, std::integral_constant<int, 2>{}); break;
      case 4: f(threads, std::integral_constant<int, 4>{}); break;
      case 8: f(threads, std::integral_constant<int, 8>{}); break;
      case 16: if constexpr (NT > 64 && !BACK) f(threads, std::integral_constant<int, 16>{}); break;
    }
  };
  if (l.threads == 64) of(std::integral_constant<int, 64>{});
  if (l.threads == 256) of(std::integral_constant<int, 256>{});
  if (l.threads == 512) of(std::integral_constant<int, 512>{});
  if (l.threads == 1024) of(std::integral_constant<int, 1024>{});
}

template <typename T>
hipError_t forward(const GroupShape& s, const void* x, const float* scale, const float* shift, void* y, float* stats,
                   char* ws, hipStream_t st) {
  const Layout l = layout_of(s, false);
  NormArgs a = args_of(s, l, x, scale, shift, ws);
  a.y = y, a.stats = stats ? stats : reinterpret_cast<float*>(ws + l.stats);
  if (l.threads) {
    with_registers<false>(l, [&](auto threads, auto n) {
      constexpr int NT = decltype(threads)::value, N = decltype(n)::value;
      const dim3 grid((unsigned)ceil_div(s.B * (l.rows ? l.spans : s.G), 8) * 8);
      if (!l.rows)
        hipLaunchKernelGGL((k_norm_group<T, NT, N>), grid, dim3(NT), 0, st, a);
      else if constexpr (NT > 64) {
        if (a.cg % kVE<T> == 0)
          hipLaunchKernelGGL((k_norm_span<T, NT, N, true>), grid, dim3(NT), 0, st, a);
        else
          hipLaunchKernelGGL((k_norm_span<T, NT, N, false>), grid, dim3(NT), 0, st, a);
      }
    });
    return hipGetLastError();
  }
  const dim3 grid = part_grid(s, l), block(kThreads);
  const bool whole = s.C % kVE<T> == 0;
  const auto sums = !l.rows ? k_norm_sums_planes<T> : whole ? k_norm_sums_rows<T, true> : k_norm_sums_rows<T, false>;
  hipLaunchKernelGGL(sums, grid, block, 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (!l.fold) {
    hipLaunchKernelGGL(k_norm_stats, group_grid(s), block, 0, st, a, share(a));
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const auto apply = !l.rows  ? k_norm_apply_planes<T>
                     : l.fold ? (whole ? k_norm_apply_rows<T, true, true> : k_norm_apply_rows<T, false, true>)
                              : (whole ? k_norm_apply_rows<T, true, false> : k_norm_apply_rows<T, false, false>);
  hipLaunchKernelGGL(apply, grid, block, 0, st, a);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const GroupShape& s, const void* x, const float* scale, const float* shift, const float* stats,
                    const void* dy, const moce_group_norm_grads& gr, char* ws, hipStream_t st) {
  const Layout l = layout_of(s, true);
  NormArgs a = args_of(s, l, x, scale, shift, ws);
  a.dy = dy, a.dx = gr.dx, a.dscale = gr.dscale, a.dshift = gr.dshift, a.stats = const_cast<float*>(stats);
  a.sums = reinterpret_cast<float2*>(ws + l.sums), a.means = reinterpret_cast<float2*>(ws + l.means);
  const dim3 block(kThreads);
  const bool whole = s.C % kVE<T> == 0;
  hipError_t e;
  if (l.threads) {
    with_registers<true>(l, [&](auto threads, auto n) {
      constexpr int NT = decltype(threads)::value, N = decltype(n)::value;
      const dim3 grid((unsigned)ceil_div(s.B * (l.rows ? l.spans : s.G), 8) * 8);
      if (!l.rows)
        hipLaunchKernelGGL((k_norm_group_backward<T, NT, N>), grid, dim3(NT), 0, st, a);
      else if constexpr (NT > 64) {
        if (a.cg % kVE<T> == 0)
          hipLaunchKernelGGL((k_norm_span_backward<T, NT, N, true>), grid, dim3(NT), 0, st, a);
        else
          hipLaunchKernelGGL((k_norm_span_backward<T, NT, N, false>), grid, dim3(NT), 0, st, a);
      }
    });
    e = hipGetLastError();
  } else {
    const auto sums =
        !l.rows ? k_norm_dsums_planes<T> : whole ? k_norm_dsums_rows<T, true> : k_norm_dsums_rows<T, false>;
    hipLaunchKernelGGL(sums, part_grid(s, l), block, 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (!l.fold) {
      hipLaunchKernelGGL(k_norm_dstats, group_grid(s), block, 0, st, a, share(a));
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return e;
  dim3 grid = l.threads ? dim3(1) : part_grid(s, l);   // of dx, where it has a launch of its own
  if (gr.dscale || gr.dshift) {
    const unsigned params = (unsigned)ceil_div(s.C, 16);
    if (l.rows && l.threads == 0 && gr.dx) {   // beside dx
      a.params = (int)params, grid.x += params;
    } else {
      hipLaunchKernelGGL(k_norm_dparams, dim3(params), block, 0, st, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (!gr.dx || l.threads) return hipSuccess;
  const auto dx = !l.rows  ? k_norm_dx_planes<T>
                  : l.fold ? (whole ? k_norm_dx_rows<T, true, true> : k_norm_dx_rows<T, false, true>)
                           : (whole ? k_norm_dx_rows<T, true, false> : k_norm_dx_rows<T, false, false>);
  hipLaunchKernelGGL(dx, grid, block, 0, st, a);
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
