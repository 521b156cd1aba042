// The losses of a classification head, over labels or a teacher's largest
// logits, and their gradients, without the logits kept.
//
// With z = x W^T + shift and a row's scale T, both losses are lse(z / T) less
// the logits under a sparse target distribution q, and both gradients are
// g (softmax(z / T) - q).  So one set of kernels has both; a label is one entry
// of weight 1 - e (and e / V everywhere).
//
// The forward is the product x W^T (product.h) whose epilogue leaves a row's
// running maximum and sum over the tile's classes instead of the tile;
// k_head_rows joins a row's tiles and takes the logits of its targets by dot
// products of their own.  The backward forms the product again, in pieces of
// the classes; its epilogue writes g softmax, rounded, and sums it over the
// rows for dshift.  A label's element has its part taken off there; a teacher's
// k_head_targets puts right (from float32 values too, so that p - q loses no
// digits).  A piece then goes through the products of dx (whose partial sums
// are kept in float32 from piece to piece) and dweight.  8 P V C operations in
// all, 6 with the logits kept; bound by the matrix cores where C and P are large.
//
// Logits are taken in base 2: u = (z + shift) log2(e) / T, the same 32 bits in
// the forward and the backward (a logit's sum goes in the same order in every
// tile): where u is large, what a softmax is of are differences of a few steps
// of it, and u less a row's lse is above 0 nowhere.
#include "product.h"

namespace moce {
namespace {

constexpr int kMaxEntries = 1024;   // of a teacher, a row
constexpr int kWaves = kThreads / kWave;

struct Targets {
  const void *classes, *logits;
  int K, V, wide, low;       // wide: classes of 64 bits; low: logits of 16
  bool teacher;
  float c1, label;           // log2(e) / T; the weight of a label

  __device__ __forceinline__ int index(int64_t p, int k) const {   // -1: outside the classes
    const int64_t at = p * K + k;
    const int64_t v = wide ? static_cast<const int64_t*>(classes)[at] : static_cast<const int32_t*>(classes)[at];
    return v >= 0 && v < V ? (int)v : -1;
  }
  __device__ __forceinline__ float logit(int64_t p, int k) const {
    const int64_t at = p * K + k;
    return low ? bf16_to_f32(static_cast<const uint16_t*>(logits)[at]) : static_cast<const float*>(logits)[at];
  }
};

// A row as the backward's epilogue reads it.
struct alignas(16) Row {
  float lse, g;   // g of 0: the row is left out, or weighs nothing
  int label;      // -1: none, or a teacher's
  int reserved;
};
struct HeadArgs : GemmArgs {
  float c1;              // log2(e) / T
  // forward
  float2* stat;          // [R][tc] maximum and sum of 2^(u - maximum)
  float* sums;           // [R][tc] sums of z (nullptr: none)
  // backward
  const Row* info;       // [R]
  const float* top;      // the largest |g|, and 1 over it
  float even;            // e / V
  float label;           // a label's weight
  int v0;                // the piece's first class
  float* colsum;         // [rows of waves][cols_ld] sums of dz (nullptr: none)
  int64_t cols_ld;
};

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }
// u, rounded: in one step with the subtraction behind it, the backward's was not the forward's
// (logits of 2^31: infinite probabilities).
__device__ __forceinline__ float exponent(float z, float c1) {
#pragma clang fp contract(off)
  return z * c1;
}

// Maximum and sum of 2^(u - maximum); the maximum of nothing is -inf, its sum 0.
struct Soft {
  float m, s;
};
__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Soft join(Soft a, Soft b) {
  const float m = fmaxf(a.m, b.m), r = finite_or_0(m);
  return Soft{m, a.s * exp2_of(a.m - r) + b.s * exp2_of(b.m - r)};
}

// ---- forward epilogue ------------------------------------------------------------
// Bound by the products: 8192 rows of 4096 by 65536 classes in 3.24 ms, 1359
// TFLOP/s (a library product that writes its results: 1457); 3152 of 768 by
// 21841, twelve stages between the ends of a tile, 137 us, 772.
// A lane holds 4 FC classes of each of its FR rows; four lanes share a row's
// classes of the wave, WC waves the tile's.  (NaN is not a maximum, but makes
// the sum NaN.)
template <typename T, int BYTES, int FR, int FC, int WR, int WC>
struct HeadStats {
  const HeadArgs& g;
  int r0, c0, lane;
  __device__ __forceinline__ HeadStats(const HeadArgs& g, int r0, int c0, int lane) : g(g), r0(r0), c0(c0), lane(lane) {}

  template <typename L>
  __device__ __forceinline__ void run(f32x4 (&acc)[FR][FC], L&& lds, int wave, int, int) {
    static_assert(BYTES >= FR * 16 * 12, "a wave's rows");
    float sh[FC][4];
    bool in[FC][4];
#pragma unroll
    for (int j = 0; j < FC; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = c0 + 32 * (j / 2) + 8 * (lane >> 4) + 4 * (j % 2) + e;
        in[j][e] = c < g.N;
        sh[j][e] = g.shift ? g.shift[min(c, g.N - 1)] : 0.f;
      }
    float* mine = reinterpret_cast<float*>(lds(wave));
#pragma unroll
    for (int i = 0; i < FR; ++i) {
      float u[FC][4], m = -INFINITY, total = 0.f;
#pragma unroll
      for (int j = 0; j < FC; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = acc[i][j][e] + sh[j][e];
          total += in[j][e] ? z : 0.f;
          u[j][e] = in[j][e] ? exponent(z, g.c1) : -INFINITY;
          m = fmaxf(m, u[j][e]);
        }
      m = fmaxf(m, __shfl_xor(m, 16, kWave));
      m = fmaxf(m, __shfl_xor(m, 32, kWave));
      const float r = finite_or_0(m);
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < FC; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s += exp2_of(u[j][e] - r);
      s += __shfl_xor(s, 16, kWave);
      s += __shfl_xor(s, 32, kWave);
      total += __shfl_xor(total, 16, kWave);
      total += __shfl_xor(total, 32, kWave);
      if (lane < 16) {
        float* to = mine + 3 * (16 * i + lane);
        to[0] = m, to[1] = s, to[2] = total;
      }
    }
    __syncthreads();
    if (wave >= WR) return;
    const int tile = c0 / (16 * WC * FC);
    for (int r = lane; r < 16 * FR; r += kWave) {
      if (r0 + r >= g.R) break;
      Soft a{mine[3 * r], mine[3 * r + 1]};
      float total = mine[3 * r + 2];
#pragma unroll
      for (int w = 1; w < WC; ++w) {
        const float* o = reinterpret_cast<const float*>(lds(wave + w * WR)) + 3 * r;
        a = join(a, Soft{o[0], o[1]});
        total += o[2];
      }
      const int64_t at = (int64_t)(r0 + r) * g.tc + tile;
      g.stat[at] = make_float2(a.m, a.s);
      if (g.sums) g.sums[at] = total;
    }
  }
};

// ---- backward epilogue -----------------------------------------------------------
// Eight classes a lane, in rows, as Finish has them: g / G (2^(u - lse) - e / V),
// less a label's part (a teacher's is k_head_targets'), zeros behind the classes
// to the end of the line.  dz is rounded to the operands' type, which is what
// the matrix cores take beside the weight and x: in bfloat16, dx and dweight are
// 2.3e-3 off in the 2-norm for spread targets, 1.66e-3 of it their own rounding;
// two parts of bfloat16 would double the products dx and dweight, half of a
// step's time.  G, the largest |g|, comes in behind the products: with it, equal
// weights of the rows are 1, and a label's element, near -1, is rounded by its
// own small rest; within dz, the rounding of g would be one factor of all rows'
// gradients (dx and dweight of 8192 rows and 65536 classes were 3.3e-3 off in
// the 2-norm, not 1.7e-3).  The pieces of those take 3.40 ms, 5% more than the
// forward's 3.24, which has no dz.
template <typename T, int BYTES, int FR, int FC, int WR, int WC>
struct HeadGradient : Finish<T, BYTES, FR, FC, WR, WC> {
  using F = Finish<T, BYTES, FR, FC, WR, WC>;
  const HeadArgs& h;
  __device__ __forceinline__ HeadGradient(const HeadArgs& g, int r0, int c0, int lane) : F(g, r0, c0, lane), h(g) {}

  template <typename L>
  __device__ __forceinline__ void run(f32x4 (&acc)[FR][FC], L&& lds, int wave, int lane, int) {
    unsigned char* l = lds(wave);
    const int c = this->c, left = h.N - c;   // classes from the lane's first on
    float sh[8], sum[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) sh[i] = h.shift ? h.shift[min(c + i, h.N - 1)] : 0.f;
    T* y = static_cast<T*>(h.y);
    const float unit = h.top[1];
#pragma unroll
    for (int f = 0; f < FR; f += F::kFrags) {
      constexpr int kPer = 16 / F::kDown, kBatch = F::kBatch;
#pragma unroll
      for (int i = 0; i < F::kFrags; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) {
          const int r = 16 * i + (lane & 15), ch = 8 * (j / 2) + 2 * (lane >> 4) + (j & 1);
          *reinterpret_cast<f32x4*>(l + r * F::kPitch + ((ch ^ (r & 7)) << 4)) = acc[f + i][j];
        }
      for (int it = 0; it < F::kIters; it += kBatch) {
        float v[kBatch][8], lse[kBatch], g[kBatch];
        int label[kBatch];   // its place among the lane's eight
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int row = this->row(f * kPer + it + b), r = min(row, h.R - 1);
          const Row q = h.info[r];
          lse[b] = q.lse;
          g[b] = row < h.R ? q.g * unit : 0.f;
          label[b] = q.label - h.v0 - c;
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) this->value(l, it + b, v[b]);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[b][i] = exp2_of(exponent(v[b][i] + sh[i], h.c1) - lse[b]) - h.even;
          if (__any((unsigned)label[b] < 8u)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[b][i] -= label[b] == i ? h.label : 0.f;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v[b][i] = g[b] == 0.f || i >= left ? 0.f : g[b] * v[b][i];
            sum[i] += v[b][i];
          }
        }
        if (left > 0) {
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            const int row = this->row(f * kPer + it + b);
            if (row >= h.R) continue;
            T* to = y + row * h.ld + c;
            if (c + 8 <= h.ld)
              store8(to, v[b]);
            else   // float32: a line may end after four
              store4(to, v[b]);
          }
        }
      }
    }
    if (!h.colsum) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int o = F::kAcross; o < kWave; o <<= 1) sum[i] += __shfl_xor(sum[i], o, kWave);
    if (lane < F::kAcross) {
      float* to = h.colsum + (int64_t)(this->r0 / (16 * FR)) * h.cols_ld + c;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) to[i] = sum[i];
    }
  }
};

// ---- targets ---------------------------------------------------------------------

// A row's targets by one wave, kept in LDS (K of each): the classes (-1 for an
// entry that counts for nothing or whose class came before) and their
// probabilities; u is room for as many values.  False where the row is left out.
struct RowTargets {
  int* cls;
  float *q, *u;
};
__device__ __forceinline__ RowTargets targets_at(int* p, int K) {
  return RowTargets{p, reinterpret_cast<float*>(p + K), reinterpret_cast<float*>(p + 2 * K)};
}
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

template <bool TEACHER>
__device__ __forceinline__ bool take_targets(const Targets& t, int64_t p, const RowTargets& s, int lane) {
  if constexpr (!TEACHER) {
    const int i = t.index(p, 0);
    if (lane == 0) s.cls[0] = i, s.q[0] = t.label;
    wave_fence();
    return i >= 0;
  }
  float m = -INFINITY;
  for (int k = lane; k < t.K; k += kWave) {
    const int i = t.index(p, k);
    const float v = i >= 0 ? t.logit(p, k) * t.c1 : -INFINITY;
    s.cls[k] = i, s.q[k] = v;
    m = fmaxf(m, v);
  }
  m = finite_or_0(wave_max(m));
  float sum = 0.f;
  for (int k = lane; k < t.K; k += kWave) sum += s.q[k] = exp2_of(s.q[k] - m);
  sum = wave_sum(sum);
  wave_fence();
  if (sum == 0.f) return false;
  const float r = 1.f / sum;
  // the first entry of a class has the sum over all of it, the others -1
  for (int k = lane; k < t.K; k += kWave) {
    const int i = s.cls[k];
    float all = 0.f;
    bool before = false;
#pragma unroll 4
    for (int o = 0; o < t.K; ++o) {
      const bool same = s.cls[o] == i;
      before = before || (same && o < k);
      all += same ? s.q[o] : 0.f;
    }
    s.u[k] = before ? -1.f : all * r;
  }
  wave_fence();
  for (int k = lane; k < t.K; k += kWave) {
    if (s.u[k] < 0.f) s.cls[k] = -1;
    s.q[k] = s.u[k];
  }
  wave_fence();
  return true;
}

// ---- the forward's rows ----------------------------------------------------------

// A row's loss: both are at least 0, but the two logarithms that one is the
// difference of are rounded apart, and a target's logit is a sum of its own.
// (NaN stays.)
__device__ __forceinline__ float not_below_0(float l) { return l < 0.f ? 0.f : l; }

struct RowsArgs {
  Targets t;
  const void *x, *w;
  const float* shift;
  const float2* stat;
  const float* sums;
  float *rows, *code, *saved;   // code: 0 left out, 1 counts, 2 left out and not finite
  float *loss, *tail;           // of the mean, as k_head_mean has them
  bool alone;                   // one workgroup has all rows, and the mean
  int64_t P;
  int C, tc;
  float smoothing, factor;      // factor: T^2 ln 2
};

// The dot product of two rows by LANES neighbouring lanes, each of them has it.
template <typename T, int LANES>
__device__ __forceinline__ float dot_row(const T* a, const T* b, int n, int lane) {
  constexpr int kStep = 8 * LANES;
  float s[2] = {0.f, 0.f};
  int i = lane * 8;
  for (; i + kStep + 8 <= n; i += 2 * kStep) {   // two steps' loads together
    float u[2][8], v[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) load8(a + i + h * kStep, u[h]), load8(b + i + h * kStep, v[h]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[h] = fmaf(u[h][e], v[h][e], s[h]);
  }
  for (; i + 8 <= n; i += kStep) {
    float u[8], v[8];
    load8(a + i, u);
    load8(b + i, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[0] = fmaf(u[e], v[e], s[0]);
  }
  for (int e = i; e < min(i + 8, n); ++e) s[1] = fmaf(Elem<T>::to_f(a[e]), Elem<T>::to_f(b[e]), s[1]);
  return wave_sum<LANES>(s[0] + s[1]);
}

// A row's statistics over its tiles, by one wave; every lane has them.
__device__ __forceinline__ Soft row_stats(const RowsArgs& a, int64_t p, int lane, float* sum) {
  Soft m{-INFINITY, 0.f};
  float t = 0.f;
#pragma unroll 2
  for (int i = lane; i < a.tc; i += kWave) {
    const float2 o = a.stat[p * a.tc + i];
    m = join(m, Soft{o.x, o.y});
    if (a.sums) t += a.sums[p * a.tc + i];
  }
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    m = join(m, Soft{__shfl_xor(m.m, o, kWave), __shfl_xor(m.s, o, kWave)});
    t += __shfl_xor(t, o, kWave);
  }
  *sum = t;
  return m;
}

// Whether a row holds a value that is not finite, to every lane.
template <typename T>
__device__ __forceinline__ bool wild_row(const T* x, int C, int lane) {
  bool w = false;
  for (int c = lane; c < C; c += kWave) w = w || !__builtin_isfinite(Elem<T>::to_f(x[c]));
  return __any(w);
}

// The mean over the rows that count, and what the backward wants to know of all
// rows: their number, and whether a row that is left out is not finite.
template <int NT>
__device__ __forceinline__ void mean_of_rows(const float* rows, const float* code, int64_t P, float* loss, float* tail) {
  __shared__ double sums[NT / kWave], counts[NT / kWave];
  __shared__ int wild;
  if (threadIdx.x == 0) wild = 0;
  __syncthreads();
  double sum = 0., count = 0.;
  auto add = [&](float r, float c) __attribute__((always_inline)) {
    sum += r;
    count += c == 1.f;
    if (c == 2.f) wild = 1;
  };
  const int64_t whole = P / 4 * 4;
#pragma unroll 4
  for (int64_t p = threadIdx.x * 4; p < whole; p += NT * 4) {
    float r[4], c[4];
    load4(rows + p, r);
    load4(code + p, c);
#pragma unroll
    for (int i = 0; i < 4; ++i) add(r[i], c[i]);
  }
  if (whole + threadIdx.x < P) add(rows[whole + threadIdx.x], code[whole + threadIdx.x]);
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    sum += __shfl_xor(sum, o, kWave);
    count += __shfl_xor(count, o, kWave);
  }
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum, counts[threadIdx.x >> 6] = count;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < NT / kWave; ++w) sum += sums[w], count += counts[w];
  if (loss) *loss = count > 0. ? (float)(sum / count) : 0.f;
  if (tail) tail[0] = (float)count, tail[1] = (float)wild;
}
// By a launch of its own, where k_head_rows is more than one workgroup.  (Its
// last workgroup to end, found by a counter, needs a fence in all of them: 256
// rows 10.5 us, not 5.2 and 2.6.)
constexpr int kMeanThreads = 1024;
__global__ void __launch_bounds__(kMeanThreads)
k_head_mean(const float* rows, const float* code, int64_t P, float* loss, float* tail) {
  mean_of_rows<kMeanThreads>(rows, code, P, loss, tail);
}

// The rows' losses, and what the backward reads.  Labels: a wave a row.  A
// teacher: a workgroup a row, whose 16 groups of 16 lanes take the targets'
// dot products (3152 rows of 768 with 32 entries: 39 us; a wave for each: 77).
// Bound by the weight's rows: 64 entries of 4095 rows of 2048, 1.07 GB, in 167
// us, 6.4 TB/s.
template <typename T, bool TEACHER>
__global__ void __launch_bounds__(kThreads)
k_head_rows(RowsArgs a) {
  extern __shared__ int entries[];   // a teacher's: classes, probabilities, logits
  __shared__ int there, one_cls[kWaves];
  __shared__ float one_q[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = a.t.K;
  const RowTargets s = TEACHER ? targets_at(entries, K) : RowTargets{one_cls + wave, one_q + wave, nullptr};
  float* u = s.u;
  constexpr int kRows = TEACHER ? 1 : kWaves;   // of a workgroup
  for (int64_t p0 = blockIdx.x * (int64_t)kRows; p0 < a.P; p0 += (int64_t)gridDim.x * kRows) {
    const int64_t p = TEACHER ? p0 : p0 + wave;
    if (p >= a.P) break;   // a wave of labels
    const T* x = static_cast<const T*>(a.x) + p * a.C;
    bool ok;
    if constexpr (TEACHER) {
      __syncthreads();   // the last row's entries are read
      if (wave == 0) {
        const bool t = take_targets<TEACHER>(a.t, p, s, lane);
        if (lane == 0) there = t;
      }
      __syncthreads();
      ok = there;
    } else {
      ok = take_targets<TEACHER>(a.t, p, s, lane);
    }
    if (!ok) {
      const bool wild = a.saved && (!TEACHER || wave == 0) && wild_row(x, a.C, lane);
      if (lane == 0 && (!TEACHER || wave == 0)) {
        a.rows[p] = 0.f;
        a.code[p] = wild ? 2.f : 0.f;
        if (a.saved) a.saved[p * (K + 1)] = INFINITY;
      }
      continue;
    }
    float* saved = a.saved ? a.saved + p * (K + 1) : nullptr;
    if constexpr (TEACHER) {
      constexpr int kLanes = 16;
      for (int k = threadIdx.x / kLanes; k < K; k += kThreads / kLanes) {
        const int i = s.cls[k];
        if (i < 0) continue;
        const float d = dot_row<T, kLanes>(x, static_cast<const T*>(a.w) + (int64_t)i * a.C, a.C, threadIdx.x % kLanes);
        if (threadIdx.x % kLanes == 0) u[k] = (d + (a.shift ? a.shift[i] : 0.f)) * a.t.c1;
      }
      __syncthreads();
      if (wave != 0) continue;
    }
    float sum;
    const Soft m = row_stats(a, p, lane, &sum);
    const float lse = m.m + log2f(m.s);
    float l = 0.f;
    if constexpr (TEACHER) {
      for (int k = lane; k < K; k += kWave) {
        if (s.cls[k] < 0) continue;
        const float q = s.q[k];
        l += q == 0.f ? 0.f : q * (log2f(q) - u[k] + lse);
        if (saved) saved[1 + k] = u[k];
      }
      l = wave_sum(l);
    } else {
      const int i = s.cls[0];
      const float d = dot_row<T, kWave>(x, static_cast<const T*>(a.w) + (int64_t)i * a.C, a.C, lane);
      const float z = (d + (a.shift ? a.shift[i] : 0.f)) * a.t.c1;
      l = s.q[0] == 0.f ? 0.f : (lse - z) * s.q[0];   // fully smoothed: z may be infinite
      if (saved && lane == 0) saved[1] = z;
      if (a.sums && a.smoothing > 0.f) l += a.smoothing * (lse - sum / (float)a.t.V * a.t.c1);
    }
    if (lane == 0) {
      a.rows[p] = not_below_0(l) * a.factor;
      a.code[p] = 1.f;
      if (saved) saved[0] = lse;
    }
  }
  if (!a.alone) return;
  __threadfence_block();
  __syncthreads();
  mean_of_rows<kThreads>(a.rows, a.code, a.P, a.loss, a.tail);
}

// ---- few classes -------------------------------------------------------------------
//
// Where a row's targets would read more for their dot products than all of its
// logits take, written and read, the forward keeps the logits of a row until
// its loss is there: float32, bounded as a piece of the gradient is.  (32
// entries of 209 classes, 43209 rows of 2057: 73 us, not 964; a label of 16
// classes, 43810 rows of 864 float32: 27, not 43.  Few rows are faster by their
// dot products: 250 of 768, 10 entries of 1000 classes, 9 us to 6.)
constexpr int64_t kLogitClasses = 4096, kDotBytes = (int64_t)64 << 20;

// k_head_rows from the logits z [P][V], a wave a row.
template <typename T, bool TEACHER>
__global__ void __launch_bounds__(kThreads)
k_head_logits(RowsArgs a, const float* __restrict__ logits) {
  extern __shared__ int entries[];   // a wave's targets
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = a.t.K, V = a.t.V;
  const RowTargets s = targets_at(entries + wave * 3 * K, K);
  for (int64_t p = blockIdx.x * (int64_t)kWaves + wave; p < a.P; p += (int64_t)gridDim.x * kWaves) {
    float* saved = a.saved ? a.saved + p * (K + 1) : nullptr;
    wave_fence();
    if (!take_targets<TEACHER>(a.t, p, s, lane)) {
      const bool wild = saved && wild_row(static_cast<const T*>(a.x) + p * a.C, a.C, lane);
      if (lane == 0) {
        a.rows[p] = 0.f;
        a.code[p] = wild ? 2.f : 0.f;
        if (saved) saved[0] = INFINITY;
      }
      continue;
    }
    const float* z = logits + p * V;
    Soft m{-INFINITY, 0.f};
    float sum = 0.f;
    constexpr int kAt = 4;   // of a lane at a time
    for (int v = lane; v < V; v += kAt * kWave) {
      float u[kAt], top = -INFINITY, part = 0.f;
#pragma unroll
      for (int i = 0; i < kAt; ++i) {
        const int c = v + i * kWave;
        u[i] = c < V ? z[c] + (a.shift ? a.shift[c] : 0.f) : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < kAt; ++i) {
        sum += v + i * kWave < V ? u[i] : 0.f;
        u[i] = exponent(u[i], a.t.c1);
        top = fmaxf(top, u[i]);
      }
#pragma unroll
      for (int i = 0; i < kAt; ++i) part += exp2_of(u[i] - finite_or_0(top));
      m = join(m, Soft{top, part});
    }
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
      m = join(m, Soft{__shfl_xor(m.m, o, kWave), __shfl_xor(m.s, o, kWave)});
      sum += __shfl_xor(sum, o, kWave);
    }
    const float lse = m.m + log2f(m.s);
    float loss = 0.f;
    for (int k = lane; k < K; k += kWave) {
      const int i = s.cls[k];
      if (i < 0) continue;
      const float q = s.q[k], u = exponent(z[i] + (a.shift ? a.shift[i] : 0.f), a.t.c1);
      if constexpr (TEACHER)
        loss += q == 0.f ? 0.f : q * (log2f(q) - u + lse);
      else
        loss = q == 0.f ? 0.f : (lse - u) * q;
      if (saved) saved[1 + k] = u;
    }
    loss = wave_sum(loss);
    if (lane == 0) {
      if (!TEACHER && a.smoothing > 0.f) loss += a.smoothing * (lse - sum / (float)V * a.t.c1);
      a.rows[p] = not_below_0(loss) * a.factor;
      a.code[p] = 1.f;
      if (saved) saved[0] = lse;
    }
  }
}

// ---- the backward's rows ---------------------------------------------------------

constexpr int kPrepBlocks = 1024;
struct PrepArgs {
  const void* x;
  void* lines;                // x in lines of ld, rows that are left out as zeros
  int ragged;                 // written always, else only where such a row is not finite
  int64_t P;
  int C, ld, K, mean;
  float T;
  const float *saved, *dloss;
  Targets t;
  Row* info;
  float* gmax;                // [kPrepBlocks] largest |g|, finite ones, of rows' weights
  float* top;                 // G and 1 / G: here of the mean, else by k_head_top
  unsigned long long* fixed;  // [V] cleared (nullptr: none)
  int V;
};
// (Without rows that count, or of a weight that is not finite, any G will do.)
__device__ __forceinline__ void set_top(float* top, float g) {
  g = __builtin_isfinite(g) ? fmaxf(g, 0x1p-100f) : 1.f;
  top[0] = g, top[1] = 1.f / g;
}
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_head_prep(PrepArgs a) {
  __shared__ float tops[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (a.fixed)
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < a.V; i += (int64_t)gridDim.x * kThreads)
      a.fixed[i] = 0;
  const float* tail = a.saved + a.P * (a.K + 1);
  const bool copy = a.lines && (a.ragged || tail[1] != 0.f);
  float top = 0.f;
  for (int64_t p = blockIdx.x * (int64_t)kWaves + wave; p < a.P; p += (int64_t)gridDim.x * kWaves) {
    const bool there = a.saved[p * (a.K + 1)] != INFINITY;
    float g = 0.f;
    if (there) g = a.T * (a.mean ? a.dloss[0] / tail[0] : a.dloss[p]);
    if (lane == 0) a.info[p] = Row{a.saved[p * (a.K + 1)], g, a.t.teacher ? -1 : a.t.index(p, 0), 0};
    if (__builtin_isfinite(g)) top = fmaxf(top, fabsf(g));
    if (!copy) continue;
    const T* x = static_cast<const T*>(a.x) + p * a.C;
    T* to = static_cast<T*>(a.lines) + p * a.ld;
    for (int c = lane * Elem<T>::kVec; c < a.ld; c += kWave * Elem<T>::kVec) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (there) {
        if (c + Elem<T>::kVec <= a.C) {
          __builtin_memcpy(&v, x + c, 16);
        } else {
          T e[Elem<T>::kVec] = {};
#pragma unroll
          for (int i = 0; i < Elem<T>::kVec; ++i)
            if (c + i < a.C) e[i] = x[c + i];
          __builtin_memcpy(&v, e, 16);
        }
      }
      *reinterpret_cast<u32x4*>(to + c) = v;
    }
  }
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, tops[w]);
  if (!a.mean)
    a.gmax[blockIdx.x] = top;
  else if (blockIdx.x == 0)
    set_top(a.top, fabsf(a.T * a.dloss[0] / tail[0]));
}
__global__ void __launch_bounds__(kThreads)
k_head_top(const float* __restrict__ gmax, int n, float* __restrict__ top) {
  __shared__ float s[kWaves];
  float t = 0.f;
  for (int i = threadIdx.x; i < n; i += kThreads) t = fmaxf(t, gmax[i]);
  t = wave_max(t);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x == 0) set_top(top, fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
}

// A teacher's sums of (g / G) q over the rows of a class, each at most 1, go in whole
// numbers of 2^-fixed_bits: the same in any order.
__host__ __device__ inline int fixed_bits(int64_t P) {
  int n = 60;
  for (; P > 0; P >>= 1) --n;
  return n;
}

struct TargetArgs {
  Targets t;
  const Row* info;
  const float *saved, *top;
  int64_t P, ld;
  int v0, n;                  // the piece's classes
  void* dz;
  unsigned long long* fixed;  // nullptr: none
  float* colsum;              // with it: the piece's classes of one of the rows' sums of dz
};
// A teacher's elements of a piece of dz, a wave a row, from the logits that the
// forward took by dot products: g p lost digits to its rounding where p - q has
// none to spare.  Of p no more is taken from them than that rounding left open,
// since the other probabilities of the row are those of the tiles' sums.  A
// share that is not finite (of a logit that is not, or of g) has no whole number:
// it makes the class's sum of dz NaN, as it is where the two parts of dz are
// subtracted.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_head_targets(TargetArgs a) {
  extern __shared__ int entries[];   // a wave's targets
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const RowTargets s = targets_at(entries + wave * 3 * a.t.K, a.t.K);
  const int bits = fixed_bits(a.P);
  const float unit = a.top[1];
  for (int64_t p = blockIdx.x * (int64_t)kWaves + wave; p < a.P; p += (int64_t)gridDim.x * kWaves) {
    const Row row = a.info[p];
    const float g = row.g * unit;
    if (g == 0.f || !take_targets<true>(a.t, p, s, lane)) continue;
    const float* saved = a.saved + p * (a.t.K + 1);
    const float lse = row.lse;
    for (int k = lane; k < a.t.K; k += kWave) {
      const int i = s.cls[k] - a.v0;
      if (s.cls[k] < 0 || i < 0 || i >= a.n) continue;
      T* dz = static_cast<T*>(a.dz) + p * a.ld + i;
      const float q = s.q[k], tile = Elem<T>::to_f(*dz) / g;
      constexpr float kOpen = sizeof(T) == 2 ? 0x1p-8f : 0x1p-22f;   // half a step of bfloat16; float32: the division's too
      float prob = exp2_of(saved[1 + k] - lse);
      const float least = tile * (1.f - kOpen), most = fminf(tile * (1.f + kOpen), 1.f);
      prob = prob < least ? least : prob > most ? most : prob;
      *dz = Elem<T>::from_f(g * (prob - q));
      if (!a.fixed || q == 0.f) continue;
      const double w = (double)g * (double)q;
      if (__builtin_isfinite(w))
        atomicAdd(a.fixed + a.v0 + i, (unsigned long long)(long long)llrint(ldexp(w, bits)));
      else
        a.colsum[i] = __builtin_nanf("");   // all who write here write this
    }
    wave_fence();
  }
}

// dshift[v]: G times the sums over the rows' groups less the targets'.  16 classes a workgroup.
__global__ void __launch_bounds__(kThreads)
k_head_dshift(const float* __restrict__ part, int groups, int V, const unsigned long long* __restrict__ fixed,
              const float* __restrict__ top, int bits, float* __restrict__ out) {   // fixed: a teacher's
  __shared__ double s[kThreads];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, v = blockIdx.x * 16 + x;
  double t = 0.;
  if (v < V)
#pragma unroll 8
    for (int i = y; i < groups; i += kThreads / 16) t += part[(int64_t)i * V + v];
  s[threadIdx.x] = t;
  __syncthreads();
  if (y != 0 || v >= V) return;
#pragma unroll
  for (int i = 1; i < kThreads / 16; ++i) t += s[16 * i + x];
  if (fixed) t -= ldexp((double)(long long)fixed[v], -bits);
  out[v] = (float)((double)top[0] * t);
}

// ---- launches --------------------------------------------------------------------

// The gradient of the logits goes through the GPU in pieces of so many bytes,
// as many as the infinity cache has, from the product that writes them to the
// two that read them.
constexpr int64_t kPieceBytes = (int64_t)256 << 20;
constexpr int kPieceClasses = 256;   // a multiple of every tile and of whole lines
constexpr int64_t kMaxBlocks = 1 << 20;

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

struct Sizes {
  const HeadShape& s;
  int vec;
  explicit Sizes(const HeadShape& s) : s(s), vec(s.elem == MOCE_F32 ? 4 : 8) {}
  size_t el() const { return 16 / vec; }
  int64_t up(int64_t n) const { return (n + vec - 1) / vec * vec; }
  bool ragged() const { return s.C % vec != 0; }
  size_t x_bytes() const { return up256((size_t)s.P * up(s.C) * el()); }
  size_t w_bytes() const { return ragged() ? up256((size_t)s.V * up(s.C) * el()) : 0; }
};

struct FwdLayout {
  Plan p;
  bool logits;
  int tc;
  size_t x, w, part, stat, sums, rows, code, total;
};
FwdLayout fwd_layout(const HeadShape& s) {
  const Sizes z(s);
  FwdLayout l{};
  l.p = plan(s.P, s.V, s.C, s.elem, false, false, 1);
  const int64_t dots = s.K * s.C * (int64_t)z.el();   // bytes a row
  l.logits = s.V <= kLogitClasses && dots > 8 * s.V && s.P * dots >= kDotBytes && s.P * s.V * 4 <= kPieceBytes;
  l.tc = l.logits ? 0 : (int)ceil_div(s.V, kTile[l.p.tile].tc);
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += up256(n);
    return here;
  };
  l.x = take(z.ragged() ? z.x_bytes() : 0);
  l.w = take(z.w_bytes());
  l.part = take(l.logits ? part_bytes(s.P, s.V, l.p) : 0);
  l.stat = take((size_t)s.P * l.tc * sizeof(float2));
  l.sums = take(!s.teacher && s.smoothing > 0.f ? (size_t)s.P * l.tc * sizeof(float) : 0);
  l.rows = take((size_t)s.P * sizeof(float));
  l.code = take((size_t)s.P * sizeof(float));
  l.total = at;
  return l;
}

// The products of a piece of n classes.
struct Products {
  Plan z, x, w;
  double time() const { return z.time + x.time + w.time; }
};
Products products_of(const HeadShape& s, int64_t n, int most_splits = INT_MAX) {
  const bool ragged = Sizes(s).ragged();
  return Products{plan(s.P, n, s.C, s.elem, false, false, 1), plan(s.P, s.C, n, s.elem, ragged, false, most_splits),
                  plan(n, s.C, s.P, s.elem, ragged, true)};
}

struct BwdLayout {
  Products all, last;      // of a piece, of the last one
  int n, pieces, groups;   // classes of a piece, pieces; groups of rows of dshift's sums
  int64_t ld;              // of a piece of dz
  size_t x, w, info, gmax, top, fixed, cols, dz, part, dx, total;
};
// How the classes are cut: evenly, or in pieces whose 256 x 256 tiles fill the
// CUs in whole rounds, by the time of their products (4095 rows of 2048 by
// 100003 classes: 7 rounds and not 6.1, loss and gradients 6.7 ms to 6.0).
int64_t piece_of(const HeadShape& s) {
  const Sizes z(s);
  const int64_t most = std::max<int64_t>(kPieceBytes / (int64_t)(s.P * z.el()) / kPieceClasses, 1) * kPieceClasses;
  const int64_t least = ceil_div(s.V, most);   // pieces
  if (least == 1) return s.V;
  int64_t round = kPieceClasses;
  for (int64_t tiles = ceil_div(s.P, 256); tiles % 256 != 0 && round * 2 <= most; tiles *= 2) round *= 2;
  int64_t best = 0;
  double time = 1e300;
  for (const int64_t n : {ceil_div(ceil_div(s.V, least), kPieceClasses) * kPieceClasses,
                          ceil_div(ceil_div(s.V, least + 1), kPieceClasses) * kPieceClasses, most / round * round}) {
    const int64_t full = s.V / n, rest = s.V - full * n;
    const double t = full * products_of(s, n).time() + (rest ? products_of(s, rest).time() : 0.);
    if (t < time) time = t, best = n;
  }
  return best;
}
BwdLayout bwd_layout(const HeadShape& s) {
  const Sizes z(s);
  BwdLayout l{};
  l.n = (int)piece_of(s), l.pieces = (int)ceil_div(s.V, l.n), l.ld = z.up(l.n);
  l.all = l.last = products_of(s, l.n);
  const int64_t rest = s.V - (int64_t)(l.pieces - 1) * l.n;
  if (rest < l.n) l.last = products_of(s, rest, l.all.x.splits), l.last.z = l.all.z;
  l.groups = (int)ceil_div(s.P, kTile[l.all.z.tile].tr) * 2;   // every tile has two waves down
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += up256(n);
    return here;
  };
  l.x = take(z.x_bytes());
  l.w = take(z.w_bytes());
  l.info = take((size_t)s.P * sizeof(Row));
  l.gmax = take(kPrepBlocks * sizeof(float));
  l.top = take(2 * sizeof(float));
  l.fixed = take((size_t)s.V * 8);
  l.cols = take((size_t)l.groups * s.V * sizeof(float));
  l.dz = take((size_t)s.P * l.ld * z.el());
  l.dx = take(l.all.x.splits > 1 || l.pieces > 1 ? part_bytes(s.P, s.C, l.all.x) : 0);
  auto parts = [&](int64_t n, const Plan& p) { return p.splits > 1 ? part_bytes(n, s.C, p) : 0; };
  l.part = take(std::max(parts(l.n, l.all.w), parts(rest, l.last.w)));
  l.total = at;
  return l;
}

float scale_of(const HeadShape& s) { return s.teacher ? s.temperature : 1.f; }

Targets targets_of(const HeadShape& s, const HeadTargets& t) {
  Targets r{};
  r.classes = t.classes, r.logits = t.logits, r.K = s.K, r.V = (int)s.V, r.wide = s.wide;
  r.low = s.telem == MOCE_BF16, r.teacher = s.teacher, r.c1 = (float)((double)kLog2e / scale_of(s));
  r.label = 1.f - s.smoothing;
  return r;
}

// The arguments of the logits of classes v0.. v0 + n, x and w in whole lines.
HeadArgs logits(const HeadShape& s, const void* x, const void* w, const float* shift, int64_t v0, int64_t n) {
  const Sizes z(s);
  HeadArgs g{};
  g.R = (int)s.P, g.N = (int)n, g.K = (int)s.C, g.klen = (int)ceil_div(s.C, 64) * 64;
  g.a = Operand{x, z.up(s.C), 0, 0};
  g.b = Operand{static_cast<const char*>(w) + v0 * z.up(s.C) * z.el(), z.up(s.C), 0, 0};
  g.shift = shift ? shift + v0 : nullptr;
  g.c1 = (float)((double)kLog2e / scale_of(s));
  return g;
}

template <typename T>
hipError_t forward(const HeadShape& s, const void* x, const void* w, const float* shift, const HeadTargets& t,
                   float* loss, float* saved, char* ws, hipStream_t st) {
  const Sizes z(s);
  const FwdLayout l = fwd_layout(s);
  const void *xl = x, *wl = w;
  hipError_t e = hipSuccess;
  if (z.ragged()) {
    xl = ws + l.x, wl = ws + l.w;
    e = launch_weight_lines(s.elem, x, s.P, s.C, ws + l.x, st);
    if (e == hipSuccess) e = launch_weight_lines(s.elem, w, s.V, s.C, ws + l.w, st);
    if (e != hipSuccess) return e;
  }
  RowsArgs a{};
  float* z_all = reinterpret_cast<float*>(ws + l.part);
  if (l.logits) {
    LineProduct p{};
    p.a = xl, p.b = wl, p.lda = p.ldb = z.up(s.C), p.a_along = p.b_along = true;
    p.R = (int)s.P, p.N = (int)s.V, p.K = (int)s.C, p.tile = l.p.tile, p.splits = 1, p.klen = l.p.klen, p.part = z_all;
    e = launch_line_product(s.elem, p, st);
  } else {
    HeadArgs g = logits(s, xl, wl, shift, 0, s.V);
    a.stat = g.stat = reinterpret_cast<float2*>(ws + l.stat);
    a.sums = g.sums = !s.teacher && s.smoothing > 0.f ? reinterpret_cast<float*>(ws + l.sums) : nullptr;
    e = launch_product<T, true, true, HeadStats>(g, l.p, st);
  }
  if (e != hipSuccess) return e;
  a.t = targets_of(s, t);
  a.x = x, a.w = w, a.shift = shift, a.saved = saved;
  a.rows = s.mean ? reinterpret_cast<float*>(ws + l.rows) : loss;
  a.code = reinterpret_cast<float*>(ws + l.code);
  a.P = s.P, a.C = (int)s.C, a.tc = l.tc, a.smoothing = s.smoothing;
  const bool mean = s.mean || saved;
  a.loss = s.mean ? loss : nullptr, a.tail = saved ? saved + s.P * (s.K + 1) : nullptr;
  a.alone = mean && !l.logits && s.P <= (s.teacher ? 1 : kWaves);
  a.factor = (float)(0.69314718055994531 * scale_of(s) * scale_of(s));
  if (l.logits) {
    const auto rows = s.teacher ? k_head_logits<T, true> : k_head_logits<T, false>;
    hipLaunchKernelGGL(rows, dim3((unsigned)std::min(ceil_div(s.P, kWaves), kMaxBlocks)), dim3(kThreads),
                       (unsigned)(kWaves * s.K * 12), st, a, z_all);
  } else if (s.teacher)
    hipLaunchKernelGGL((k_head_rows<T, true>), dim3((unsigned)std::min(s.P, kMaxBlocks)), dim3(kThreads),
                       (unsigned)s.K * 12, st, a);
  else
    hipLaunchKernelGGL((k_head_rows<T, false>), dim3((unsigned)std::min(ceil_div(s.P, kWaves), kMaxBlocks)),
                       dim3(kThreads), 0, st, a);
  e = hipGetLastError();
  if (e != hipSuccess || !mean || a.alone) return e;
  hipLaunchKernelGGL(k_head_mean, dim3(1), dim3(kMeanThreads), 0, st, a.rows, a.code, s.P, a.loss, a.tail);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const HeadShape& s, const void* x, const void* w, const float* shift, const HeadTargets& t,
                    const float* saved, const float* dloss, const moce_head_grads& gr, char* ws, hipStream_t st) {
  const Sizes z(s);
  const BwdLayout l = bwd_layout(s);
  const int blocks = (int)std::min<int64_t>(kPrepBlocks, ceil_div(s.P, kWaves));
  Row* info = reinterpret_cast<Row*>(ws + l.info);
  float* gmax = reinterpret_cast<float*>(ws + l.gmax);
  float* top = reinterpret_cast<float*>(ws + l.top);
  unsigned long long* fixed = gr.dshift && s.teacher ? reinterpret_cast<unsigned long long*>(ws + l.fixed) : nullptr;
  float* cols = gr.dshift ? reinterpret_cast<float*>(ws + l.cols) : nullptr;
  {
    PrepArgs a{};
    a.x = x, a.lines = z.ragged() || gr.dweight ? ws + l.x : nullptr, a.ragged = z.ragged(), a.P = s.P;
    a.C = (int)s.C, a.ld = (int)z.up(s.C), a.K = s.K, a.mean = s.mean, a.T = scale_of(s);
    a.t = targets_of(s, t), a.saved = saved, a.dloss = dloss, a.info = info, a.gmax = gmax, a.top = top, a.fixed = fixed;
    a.V = (int)s.V;
    hipLaunchKernelGGL(k_head_prep<T>, dim3((unsigned)blocks), dim3(kThreads), 0, st, a);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && !s.mean) {
    hipLaunchKernelGGL(k_head_top, dim3(1), dim3(kThreads), 0, st, gmax, blocks, top);
    e = hipGetLastError();
  }
  const void *xl = x, *wl = w;
  if (z.ragged()) {
    xl = ws + l.x, wl = ws + l.w;
    if (e == hipSuccess) e = launch_weight_lines(s.elem, w, s.V, s.C, ws + l.w, st);
  }
  if (e != hipSuccess) return e;
  const float even = s.teacher ? 0.f : s.smoothing / (float)s.V;
  for (int i = 0; i < l.pieces; ++i) {
    const int64_t v0 = (int64_t)i * l.n, n = std::min<int64_t>(l.n, s.V - v0);
    const Products& plans = i + 1 < l.pieces ? l.all : l.last;
    HeadArgs g = logits(s, xl, wl, shift, v0, n);
    g.info = info, g.top = top, g.even = even, g.label = 1.f - s.smoothing, g.v0 = (int)v0;
    g.y = ws + l.dz, g.ld = l.ld, g.colsum = cols ? cols + v0 : nullptr, g.cols_ld = s.V;
    e = launch_product<T, true, true, HeadGradient>(g, plans.z, st);
    if (e != hipSuccess) return e;
    if (s.teacher) {
      TargetArgs a{};
      a.t = targets_of(s, t), a.info = info, a.saved = saved, a.top = top, a.P = s.P, a.ld = l.ld;
      a.v0 = (int)v0, a.n = (int)n, a.dz = ws + l.dz;
      a.fixed = fixed, a.colsum = cols ? cols + v0 : nullptr;
      hipLaunchKernelGGL(k_head_targets<T>, dim3((unsigned)std::min(ceil_div(s.P, kWaves), kMaxBlocks)), dim3(kThreads),
                         (unsigned)(kWaves * s.K * 12), st, a);
      e = hipGetLastError();
    }
    if (e == hipSuccess && gr.dx) {
      LineProduct p{};
      p.a = ws + l.dz, p.lda = l.ld, p.a_along = true;
      p.b = static_cast<const char*>(wl) + v0 * z.up(s.C) * z.el(), p.ldb = z.up(s.C);
      p.R = (int)s.P, p.N = (int)s.C, p.K = (int)n, p.tile = plans.x.tile, p.klen = plans.x.klen;
      p.splits = l.all.x.splits;   // those that are joined
      p.y = gr.dx, p.alpha = top;
      if (l.all.x.splits > 1 || l.pieces > 1)
        p.part = reinterpret_cast<float*>(ws + l.dx), p.add = i > 0, p.join = i + 1 == l.pieces;
      e = launch_line_product(s.elem, p, st);
    }
    if (e == hipSuccess && gr.dweight) {
      LineProduct p{};
      p.a = ws + l.dz, p.lda = l.ld, p.b = xl, p.ldb = z.up(s.C);
      if (!z.ragged()) p.pick = saved + s.P * (s.K + 1) + 1, p.other = ws + l.x;
      p.R = (int)n, p.N = (int)s.C, p.K = (int)s.P, p.tile = plans.w.tile, p.klen = plans.w.klen;
      p.splits = plans.w.splits;
      p.y = static_cast<char*>(gr.dweight) + v0 * s.C * z.el(), p.alpha = top;
      if (plans.w.splits > 1) p.part = reinterpret_cast<float*>(ws + l.part), p.join = true;
      e = launch_line_product(s.elem, p, st);
    }
    if (e != hipSuccess) return e;
  }
  if (cols)
    hipLaunchKernelGGL(k_head_dshift, dim3((unsigned)ceil_div(s.V, 16)), dim3(kThreads), 0, st, cols, l.groups,
                       (int)s.V, fixed, top, fixed_bits(s.P), gr.dshift);
  return hipGetLastError();
}

}  // namespace

bool head_limits(const HeadShape& s) {
  constexpr int64_t kCh = 1 << 20;
  return s.P <= (int64_t)1 << 24 && s.C <= kCh && s.V <= kCh && s.K <= kMaxEntries &&
         s.V <= ((int64_t)1 << 35) / s.C && s.P <= ((int64_t)1 << 35) / s.V && s.P <= ((int64_t)1 << 33) / s.C;
}

size_t head_saved_floats(const HeadShape& s) { return (size_t)s.P * (s.K + 1) + 2; }
size_t head_ws_bytes(const HeadShape& s) { return fwd_layout(s).total; }
size_t head_backward_ws_bytes(const HeadShape& s) { return bwd_layout(s).total; }

hipError_t launch_head(const HeadShape& s, const void* x, const void* w, const float* shift, const HeadTargets& t,
                       float* loss, float* saved, void* ws, hipStream_t st) {
  char* base = static_cast<char*>(ws);
  return s.elem == MOCE_F32 ? forward<float>(s, x, w, shift, t, loss, saved, base, st)
                            : forward<uint16_t>(s, x, w, shift, t, loss, saved, base, st);
}

hipError_t launch_head_backward(const HeadShape& s, const void* x, const void* w, const float* shift,
                                const HeadTargets& t, const float* saved, const float* dloss, const moce_head_grads& gr,
                                void* ws, hipStream_t st) {
  char* base = static_cast<char*>(ws);
  return s.elem == MOCE_F32 ? backward<float>(s, x, w, shift, t, saved, dloss, gr, base, st)
                            : backward<uint16_t>(s, x, w, shift, t, saved, dloss, gr, base, st);
}

}  // namespace moce
