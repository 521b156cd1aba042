// Dense pointwise projections with an epilogue, and their gradients.
//
// Every product here is out[r][c] = sum_k A[r][k] B[c][k] over matrices that
// are stored by lines, a line being contiguous in memory.  A line of an
// operand runs either along k or along r (or c), and the lines of
// channels-first tensors run over the positions of one image after the other:
//
//   product          rows r     columns c  k          A                B
//   forward, NHWC    positions  outputs    channels   x, along k       W, along k
//   forward, NCHW    outputs    positions  channels   W, along k       x, along c
//   dx, NHWC         positions  channels   outputs    dz, along k      W, along c
//   dx, NCHW         channels   positions  outputs    W, along r       dz, along c
//   dW, NHWC         outputs    channels   positions  dz, along r      x, along c
//   dW, NCHW         outputs    channels   positions  dz, along k      x, along k
//
// Outputs lie row by row (columns contiguous; for NCHW images apart), so the
// columns are the M side of the matrix instruction: a lane then holds
// neighbouring columns of one row.
#include <algorithm>
#include <climits>

#include "product.h"

namespace moce {
namespace {

// ---- few positions ---------------------------------------------------------------
//
// A handful of positions (tokens being generated) against the whole weight:
// bound by reading the weight.  A workgroup takes 16 outputs, its waves their
// shares of the channels, each straight from memory into the matrix
// instructions' operands, as many loads in flight as its share holds up to
// kFewAhead; the waves' sums meet in LDS.  Any alignment, lines of any length.
// 8 positions of 4096 by 4096 take 11 us (33.5 MB), one of 768 by 768 takes 6,
// nearly all of it a launch's own way; twice the waves or loads: the same.
constexpr int kFewWaves = 8, kFewAhead = 8;

template <typename T>
__device__ __forceinline__ u32x4 load_row(const T* row, int k, int n) {
  constexpr int VE = Elem<T>::kVec;
  u32x4 v = {0u, 0u, 0u, 0u};
  if (k + VE <= n) {
    __builtin_memcpy(&v, row + k, 16);
    return v;
  }
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    if (k + e < n) {
      if constexpr (sizeof(T) == 2)
        v[e / 2] |= (uint32_t)row[k + e] << (16 * (e & 1));
      else
        v[e] = __float_as_uint(row[k + e]);
    }
  }
  return v;
}

// x [P][K], weight [O][K], P <= 16 NB
template <typename T, int NB>
__global__ void __launch_bounds__(kFewWaves * kWave)
k_project_few(GemmArgs g) {
  constexpr int VE = Elem<T>::kVec, kStep = 4 * VE;   // channels of one load by the four lane groups
  __shared__ f32x4 sums[kFewWaves][NB][kWave];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int o0 = blockIdx.x * 16, m = lane & 15, q = lane >> 4;
  const T* w = static_cast<const T*>(g.b.p) + (int64_t)min(o0 + m, g.N - 1) * g.b.ld;
  const T* x[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) x[b] = static_cast<const T*>(g.a.p) + (int64_t)min(16 * b + m, g.R - 1) * g.a.ld;
  // whole steps are shared out; what is left behind them is the last wave's
  const int steps = g.K / kStep, each = (steps + kFewWaves - 1) / kFewWaves;
  const int s0 = wave * each, s1 = min(steps, s0 + each);
  f32x4 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = s0; s < s1; s += kFewAhead) {
    u32x4 wv[kFewAhead], xv[kFewAhead][NB];
#pragma unroll
    for (int i = 0; i < kFewAhead; ++i) {
      const int k = min(s + i, s1 - 1) * kStep + q * VE;   // past the share its last step again, not multiplied
      __builtin_memcpy(&wv[i], w + k, 16);
#pragma unroll
      for (int b = 0; b < NB; ++b) __builtin_memcpy(&xv[i][b], x[b] + k, 16);
    }
#pragma unroll
    for (int i = 0; i < kFewAhead; ++i)
      if (s + i < s1)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b] = multiply<T>(wv[i], xv[i][b], acc[b]);
  }
  if (wave == kFewWaves - 1 && steps * kStep < g.K) {
    const int k = steps * kStep + q * VE;
    const u32x4 wv = load_row(w, k, g.K);
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = multiply<T>(wv, load_row(x[b], k, g.K), acc[b]);
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) sums[wave][b][lane] = acc[b];
  __syncthreads();
  // a thread finishes four outputs of a position
  for (int u = threadIdx.x; u < NB * kWave; u += kFewWaves * kWave) {
    const int b = u / kWave, l = u % kWave, r = 16 * b + (l & 15), o = o0 + 4 * (l >> 4);
    f32x4 v = sums[0][b][l];
    for (int i = 1; i < kFewWaves; ++i) v += sums[i][b][l];
    if (r >= g.R) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (o + e >= g.N) break;
      const int64_t at = (int64_t)r * g.ld + o + e;
      float f = fmaf(v[e], g.scale ? g.scale[o + e] : 1.f, g.shift ? g.shift[o + e] : 0.f);
      if (g.res) f += Elem<T>::to_f(static_cast<const T*>(g.res)[at]);
      if (g.z) static_cast<T*>(g.z)[at] = Elem<T>::from_f(f);
      static_cast<T*>(g.y)[at] = Elem<T>::from_f(act_value<T>(f, g.act));
    }
  }
}

// Sums the splits' partial products, in a fixed order, and finishes them:
// eight columns a thread, `down` threads (a power of two) taking every
// down-th split.  Bound by memory, mostly the cache's (64 rows of 4096: 5 us).
constexpr int kJoinMany = 16;   // splits from which on eight threads share them
template <typename T, typename G>
__global__ void __launch_bounds__(kThreads)
k_project_join(G g, int splits, int down) {
  __shared__ float part[kThreads][8 + 1];
  const int across = kThreads / down, per = (g.N + 7) / 8;
  const int64_t u = (int64_t)blockIdx.x * across + threadIdx.x % across;
  const int r = (int)(u / per), c = (int)(u % per) * 8;
  float v[8] = {};
  if (r < g.R) {
    for (int s = threadIdx.x / across; s < splits; s += down) {
      const float* p = g.part + ((int64_t)s * g.R + r) * g.N + c;
      if (c + 8 <= g.N) {
        float q[8];
        load8(p, q);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += q[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < g.N) v[i] += p[i];
      }
    }
  }
  if (down > 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) part[threadIdx.x][i] = v[i];
    __syncthreads();
    if (threadIdx.x >= across) return;
    for (int d = 1; d < down; ++d)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += part[d * across + threadIdx.x][i];
  }
  if (r >= g.R) return;
  G h = g;
  h.part = nullptr;
  float sc[8], sh[8];
  column_affine(h, c, sc, sh);
  row_affine(h, r, sc, sh);
  finish8<T>(h, r, c, 0, v, sc, sh);
}

// ---- the gradients' other passes -------------------------------------------------

// out[o] = sum of the groups' partial sums part[group][o], of 16 channels o from
// o0 on and the groups g0..g1, by a workgroup; s: an element per thread.
__device__ __forceinline__ void sum_channels(const float* __restrict__ part, int64_t g0, int64_t g1, int O, int o0,
                                             float* __restrict__ out, float* s) {
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, o = o0 + x;
  float t = 0.f;
  if (o < O)
#pragma unroll 8
    for (int64_t i = g0 + y; i < g1; i += kThreads / 16) t += part[i * O + o];
  s[threadIdx.x] = t;
  __syncthreads();
  if (y == 0 && o < O) {
#pragma unroll
    for (int i = 1; i < kThreads / 16; ++i) t += s[16 * i + x];
    out[o] = t;
  }
}

// dshift, or the y-th of gridDim.y runs of its groups.
__global__ void __launch_bounds__(kThreads)
k_project_dshift(const float* __restrict__ part, int64_t groups, int O, float* __restrict__ out) {
  __shared__ float s[kThreads];
  const int64_t each = (groups + gridDim.y - 1) / gridDim.y, g0 = blockIdx.y * each;
  sum_channels(part, g0, min(groups, g0 + each), O, blockIdx.x * 16, out + (int64_t)blockIdx.y * O, s);
}

// Row o of the weight's gradient from the splits' G: dweight = scale G, dscale
// = <weight, G>.  `across` threads (a power of two) take the columns, the
// others of a workgroup their share of the splits.  Workgroups behind the O
// rows sum dshift, 16 channels each, from `groups` partial sums (a launch of
// its own: 3 us more).  768 by 768 after 50432 positions: 10 us.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_dweight(const float* __restrict__ part, int splits, int O, int C, const float* __restrict__ scale,
                  const T* __restrict__ weight, T* __restrict__ dweight, float* __restrict__ dscale, int across,
                  const float* __restrict__ sums, int64_t groups, float* __restrict__ dshift) {
  __shared__ float s[kThreads], dots[kThreads / kWave];
  if ((int)blockIdx.x >= O) {
    sum_channels(sums, 0, groups, O, (blockIdx.x - O) * 16, dshift, s);
    return;
  }
  const int o = blockIdx.x, x = threadIdx.x % across, down = kThreads / across;
  const float sc = scale ? scale[o] : 1.f;
  float dot = 0.f;
  for (int c0 = 0; c0 < C; c0 += across) {
    const int c = c0 + x;
    float v = 0.f;
    if (c < C) {
#pragma unroll 8
      for (int i = threadIdx.x / across; i < splits; i += down) v += part[((int64_t)i * O + o) * C + c];
    }
    if (down > 1) {
      __syncthreads();
      s[threadIdx.x] = v;
      __syncthreads();
      if (threadIdx.x < across)
        for (int d = 1; d < down; ++d) v += s[d * across + x];
    }
    if (threadIdx.x < across && c < C) {
      const int64_t e = (int64_t)o * C + c;
      if (dweight) dweight[e] = Elem<T>::from_f(sc * v);
      if (dscale) dot = fmaf(v, Elem<T>::to_f(weight[e]), dot);
    }
  }
  if (!dscale) return;
  dot = wave_sum(dot);
  if ((threadIdx.x & 63) == 0) dots[threadIdx.x >> 6] = dot;
  __syncthreads();
  if (threadIdx.x == 0) dscale[o] = (dots[0] + dots[1]) + (dots[2] + dots[3]);
}

// The passes over dy (and z) before the products; packing x or the weight is
// the same pass without an activation.
struct DzArgs {
  const void *z, *dy;
  void* dz;               // act'(z) dy where dy's element is (nullptr: not written)
  void* pack;             // the same, times scale where given, in lines of ld elements (nullptr: none)
  const float* scale;     // by channel
  float* part;            // [groups][O] partial sums of dz over positions (nullptr: none)
  int act, O, hw, ld;     // O channels; hw positions of a plane (channels-first)
  int rows;               // k_project_lines: not turned
  int64_t n;              // rows of positions (channels-last), images or planes (channels-first)
  int64_t per;            // rows of one group
};

// act'(z) dy of N times n neighbouring elements (up to eight; zeros behind
// them), at e[.] where there[.], stored to dz: all loads before the first
// store.  Eight are read: what lies behind a line is the next one.
template <typename T, int N>
__device__ __forceinline__ void dz_whole(const DzArgs& a, const int64_t (&e)[N], const bool (&there)[N], int n,
                                         float (&v)[N][8]) {
  const T *z = static_cast<const T*>(a.z), *dy = static_cast<const T*>(a.dy);
  T* dz = static_cast<T*>(a.dz);
  float q[N][8];
#pragma unroll
  for (int u = 0; u < N; ++u) load8(dy + e[u], v[u]);
  if (a.act != MOCE_ACT_NONE) {
#pragma unroll
    for (int u = 0; u < N; ++u) load8(z + e[u], q[u]);
    auto all = [&](int act) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = act_gradient<T>(q[u][i], v[u][i], act);
    };
    if (a.act == MOCE_ACT_RELU) all(MOCE_ACT_RELU);
    if (a.act == MOCE_ACT_GELU) all(MOCE_ACT_GELU);
    if (a.act == MOCE_ACT_SILU) all(MOCE_ACT_SILU);
  }
  if (n < 8) {
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] = i < n ? v[u][i] : 0.f;
  }
  if (!dz) return;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    if (!there[u]) continue;
    if (n == 8) {
      store8(dz + e[u], v[u]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) dz[e[u] + i] = Elem<T>::from_f(v[u][i]);
    }
  }
}
// The same of n elements at e, of a tensor of `total`.  (Its last ones go one
// by one; where every line's did, each took longer than all before it: 35972
// rows of 541, z, dy and a copy: 68 us, not 33.)
template <typename T>
__device__ __forceinline__ void dz8(const DzArgs& a, int64_t e, int n, int64_t total, float (&v)[8]) {
  using E = Elem<T>;
  if (n > 0 && e + 8 <= total) {
    const int64_t at[1] = {e};
    const bool there[1] = {true};
    dz_whole<T, 1>(a, at, there, n, reinterpret_cast<float(&)[1][8]>(v));
    return;
  }
  const T *z = static_cast<const T*>(a.z), *dy = static_cast<const T*>(a.dy);
  T* dz = static_cast<T*>(a.dz);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = 0.f;
    if (i < n) {
      v[i] = E::to_f(dy[e + i]);
      if (a.act != MOCE_ACT_NONE) v[i] = act_gradient<T>(E::to_f(z[e + i]), v[i], a.act);
      if (dz) dz[e + i] = E::from_f(v[i]);
    }
  }
}

// Channels-last: a workgroup takes 8 tx channels of a group of rows, its
// threads tx across and 256 / tx down; pack: rows of ld, zeros behind O.
// Bound by memory: 50432 rows of 768 (z, dy, dz: 232 MB) in 50 us, 4.6 TB/s.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_dz_rows(DzArgs a, int tx) {
  __shared__ float s[kThreads][8 + 1];
  const int x = threadIdx.x % tx, down = kThreads / tx;
  const int c = (blockIdx.y * tx + x) * 8, n = min(8, a.O - c);
  float sum[8] = {}, sc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) sc[i] = a.pack && a.scale ? a.scale[min(c + i, a.O - 1)] : 1.f;
  if (n > 0 && (int)threadIdx.x < down * tx) {
    const int64_t end = min(a.n, (blockIdx.x + (int64_t)1) * a.per);
    for (int64_t r = blockIdx.x * a.per + threadIdx.x / tx; r < end; r += down) {
      float v[8];
      dz8<T>(a, r * a.O + c, n, a.n * a.O, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += v[i];
      if (a.pack) {
        T* p = static_cast<T*>(a.pack) + r * a.ld + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= sc[i];
        if (c + 8 <= a.ld) {
          store8(p, v);
        } else {   // float32: a line may end after four
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c + i < a.ld) p[i] = Elem<T>::from_f(v[i]);
        }
      }
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) s[threadIdx.x][i] = sum[i];
  __syncthreads();
  for (int q = threadIdx.x; q < 8 * tx; q += kThreads) {
    const int cc = blockIdx.y * tx * 8 + q;
    float t = 0.f;
    for (int d = 0; d < down; ++d) t += s[d * tx + q / 8][q % 8];
    if (cc < a.O) a.part[blockIdx.x * (int64_t)a.O + cc] = t;
  }
}

// Channels-first, lines of whole chunks: `lanes` lanes (a power of two up to
// 64) take a plane; pack: planes as dy's.  Bound by memory: 64 images of 256
// channels by 56 x 56 (308 MB) in 57 us, 5.4 TB/s.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_dz_planes(DzArgs a, int lanes) {
  const int64_t plane = (int64_t)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes;
  float sum = 0.f;
  if (plane < a.n) {
    const float sc = a.pack && a.scale ? a.scale[plane % a.O] : 1.f;
    for (int p = (threadIdx.x % lanes) * 8; p < a.hw; p += lanes * 8) {
      float v[8];
      const int64_t e = plane * a.hw + p;
      const int n = min(8, a.hw - p);
      dz8<T>(a, e, n, a.n * a.hw, v);
      sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
      if (a.pack) {
        T* q = static_cast<T*>(a.pack) + e;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= sc;
        if (n == 8) {
          store8(q, v);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < n) q[i] = Elem<T>::from_f(v[i]);
        }
      }
    }
  }
  if (!a.part) return;
  for (int o = lanes / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
  if (plane < a.n && threadIdx.x % lanes == 0) a.part[plane] = sum;
}

// Up to three tensors brought into whole lines by one launch: planes of
// positions turned into lines of channels, [position][ld], or (rows) lines of
// hw elements, O of them, copied to lines of ld; zeros behind the elements.
// Bound by memory: the backward of 64 images of 256 to 1024 channels at 14 x
// 14 (z, dy, dz, their copies: 120 MB counted) takes 28 us, 4.3 TB/s; of three
// launches 45.
struct Lines {
  DzArgs job[3];
  int across[3];        // runs of kRun positions of an image
  unsigned end[3];      // patches of the jobs up to this one
  int jobs;
};

// A workgroup takes a patch of 64 channels by kRun positions of an image, a
// thread eight positions of a channel (a lane a position, two bytes a load,
// had taken 52 us, not 31, for the turn of dy); a patch that is turned goes
// through LDS.  Runs of 32: of 64, the last one of 196 positions is nearly
// empty (33 us for the above, not 29).  The patches of an XCD lie side by
// side, so that the lines which two of them share meet in one L2 (with every
// eighth patch 36 us, not 33).  part: a group per kRun positions.
constexpr int kRun = 32;
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_lines(Lines t) {
  using E = Elem<T>;
  constexpr int kPitch = 64 + 4 / (int)sizeof(T);   // odd words: positions on different banks
  constexpr int kLanes = kRun / 8, kDown = kThreads / kLanes, kPer = 64 / kDown;   // of a channel; channels at a time
  __shared__ __attribute__((aligned(16))) T s[kRun * kPitch];
  const unsigned each = (t.end[2] + 7) / 8;
  for (unsigned i = blockIdx.x; i < 8 * each; i += gridDim.x) {
    const unsigned v0 = (i & 7) * each + (i >> 3);
    if (v0 >= t.end[2]) continue;
    const int j = v0 >= t.end[1] ? 2 : v0 >= t.end[0] ? 1 : 0;
    const DzArgs& a = t.job[j];
    const unsigned first = v0 - (j ? t.end[j - 1] : 0), across = t.across[j], runs = (unsigned)a.n * across;
    const unsigned u = first % runs, b = u / across;
    const int p0 = (int)(u - b * across) * kRun, c0 = (int)(first / runs) * 64;
    const int pc = threadIdx.x % kLanes * 8, p = p0 + pc, n = min(8, a.hw - p), cl = threadIdx.x / kLanes;
    int64_t e[kPer];
    bool there[kPer];
    float v[kPer][8];
#pragma unroll
    for (int h = 0; h < kPer; ++h) {
      const int c = c0 + cl + h * kDown;
      there[h] = c < a.O;
      e[h] = ((int64_t)b * a.O + min(c, a.O - 1)) * a.hw + p;
    }
    const int64_t total = a.n * a.O * a.hw;
    if (n > 0 && e[kPer - 1] + 8 <= total) {
      dz_whole<T, kPer>(a, e, there, min(n, 8), v);
    } else {
#pragma unroll
      for (int h = 0; h < kPer; ++h) dz8<T>(a, e[h], there[h] ? n : 0, total, v[h]);
    }
#pragma unroll
    for (int h = 0; h < kPer; ++h) {
      const int c = c0 + cl + h * kDown;
      if (a.part) {
        float sum = ((v[h][0] + v[h][1]) + (v[h][2] + v[h][3])) + ((v[h][4] + v[h][5]) + (v[h][6] + v[h][7]));
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
        if (pc == 0 && there[h]) a.part[(int64_t)u * a.O + c] = sum;
      }
      if (!a.pack) continue;
      const float f = a.scale ? a.scale[min(c, a.O - 1)] : 1.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[h][i] = there[h] ? v[h][i] * f : 0.f;
      if (!a.rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[(pc + i) * kPitch + c - c0] = E::from_f(v[h][i]);
      } else if (there[h]) {
        T* q = static_cast<T*>(a.pack) + ((int64_t)b * a.O + c) * a.ld + p;
        if (p + 8 <= a.ld)
          store8(q, v[h]);
        else if (p < a.ld)   // float32: a line may end after four
          store4(q, v[h]);
      }
    }
    if (a.pack && !a.rows) {
      __syncthreads();
      // a thread writes 16 bytes of a position's line at a time
      constexpr int kVec = E::kVec, kAcross = 64 / kVec;
#pragma unroll
      for (int i = threadIdx.x; i < kRun * kAcross; i += kThreads) {
        const int row = i / kAcross, c = i % kAcross * kVec;
        if (p0 + row >= a.hw || c0 + c >= a.ld) continue;
        T w[kVec];
#pragma unroll
        for (int x = 0; x < kVec; ++x) w[x] = s[row * kPitch + c + x];
        __builtin_memcpy(static_cast<T*>(a.pack) + ((int64_t)b * a.hw + p0 + row) * a.ld + c0 + c, w, 16);
      }
    }
    if (i + gridDim.x < 8 * each) __syncthreads();
  }
}

// ---- launches --------------------------------------------------------------------

template <typename T, typename G>
hipError_t launch_join(const G& g, int splits, hipStream_t st) {
  const int down = splits >= kJoinMany ? 8 : 1;
  hipLaunchKernelGGL((k_project_join<T, G>), dim3((unsigned)ceil_div((int64_t)g.R * ceil_div(g.N, 8), kThreads / down)),
                     dim3(kThreads), 0, st, g, splits, down);
  return hipGetLastError();
}

// The product in one pass, or in splits and their join.
template <typename T, bool AK, bool BK>
hipError_t launch_whole(GemmArgs g, const Plan& p, float* part, hipStream_t st) {
  g.klen = p.klen;
  g.part = p.splits > 1 ? part : nullptr;
  const hipError_t e = launch_product<T, AK, BK>(g, p, st);
  if (e != hipSuccess || p.splits == 1) return e;
  return launch_join<T>(g, p.splits, st);
}

// ---- which operands are packed ---------------------------------------------------

constexpr int64_t kMaxPatches = 1 << 23;   // workgroups of k_project_lines; they go on beyond
constexpr int64_t kSpan = INT_MAX;   // bytes that a tile's offsets reach

struct Sizes {
  const ProjectShape& s;
  int vec;
  bool nhwc;
  explicit Sizes(const ProjectShape& s) : s(s), vec(s.elem == MOCE_F32 ? 4 : 8), nhwc(s.layout == MOCE_NHWC) {}
  size_t el() const { return 16 / vec; }
  int64_t P() const { return s.B * s.HW; }
  int64_t up(int64_t n) const { return (n + vec - 1) / vec * vec; }
  // Tensors whose lines are not whole chunks are packed: a weight of ragged
  // C, channels-last tensors of ragged channels, channels-first ones of
  // ragged planes (turned into lines of channels).  Offsets within a tile
  // have 31 bits: planes beyond that are turned too.
  bool weight() const { return s.C % vec != 0; }
  bool planes() const {
    const int64_t n = std::max(s.C, s.O);
    return !nhwc && (s.HW % vec != 0 || (256 * s.HW + (256 / s.HW + 2) * n * s.HW) * (int64_t)el() > kSpan);
  }
  bool rows(int64_t channels) const { return nhwc ? channels % vec != 0 : planes(); }
  size_t packed(int64_t channels) const { return (size_t)P() * up(channels) * el(); }
  // positions' lines run over images
  int images() const { return !nhwc && s.B > 1 ? (int)s.HW : 0; }
};

// Threads across a row of k_project_dz_rows: of the ways to share its chunks
// out evenly, the first that leaves no more than a
// twentieth of the threads idle (35972 rows of 544, z, dy and dz: 31 us, not 36
// with 32 across).
int row_lanes(int64_t channels) {
  const int64_t chunks = ceil_div(channels, 8);
  int best = 1, most = 0;
  for (int64_t parts = ceil_div(chunks, 128); parts <= ceil_div(chunks, 8); ++parts) {
    const int tx = (int)ceil_div(chunks, parts), used = (int)(chunks * (kThreads / tx) * 256 / (parts * kThreads));
    if (used > most) best = tx, most = used;
    if (used >= 243) break;
  }
  return best;
}
template <typename T>
hipError_t pack_rows(const void* src, int64_t rows, int64_t channels, void* out, int64_t ld, hipStream_t st) {
  DzArgs a{};
  a.dy = src, a.pack = out, a.O = (int)channels, a.ld = (int)ld, a.n = rows;
  const int tx = row_lanes(channels), down = kThreads / tx;
  a.per = ceil_div(ceil_div(rows, 2048), down) * down;
  hipLaunchKernelGGL(k_project_dz_rows<T>, dim3((unsigned)ceil_div(rows, a.per), (unsigned)ceil_div(channels, tx * 8)),
                     dim3(kThreads), 0, st, a, tx);
  return hipGetLastError();
}
// The jobs of one launch; none is no launch.
template <typename T>
struct LinesLaunch {
  Lines t{};
  int64_t patches = 0;
  void add(const DzArgs& a) {
    t.job[t.jobs] = a;
    t.across[t.jobs] = (int)ceil_div(std::max(a.hw, a.rows ? a.ld : 0), kRun);
    patches += a.n * t.across[t.jobs] * ceil_div(a.O, 64);
    for (int j = t.jobs++; j < 3; ++j) t.end[j] = (unsigned)patches;
  }
  // images of channels planes of hw positions into lines of channels, times scale (may be nullptr)
  void turn(const void* src, int64_t images, int64_t channels, int64_t hw, const float* scale, void* out, int64_t ld) {
    DzArgs a{};
    a.dy = src, a.pack = out, a.scale = scale, a.O = (int)channels, a.hw = (int)hw, a.ld = (int)ld, a.n = images;
    add(a);
  }
  // the weight as the products read it: packed into `out` where its lines are ragged or a scale goes into them
  void weight(const Sizes& z, const void** w, const float* scale, void* out) {
    if (!z.weight() && !scale) return;
    DzArgs a{};
    a.dy = *w, a.pack = out, a.scale = scale, a.O = (int)z.s.O, a.hw = (int)z.s.C, a.ld = (int)z.up(z.s.C);
    a.n = 1, a.rows = 1;
    add(a);
    *w = out;
  }
  hipError_t launch(hipStream_t st) {
    if (t.jobs == 0) return hipSuccess;
    hipLaunchKernelGGL(k_project_lines<T>, dim3((unsigned)std::min<int64_t>(ceil_div(patches, 8) * 8, kMaxPatches)), dim3(kThreads), 0,
                       st, t);
    return hipGetLastError();
  }
};
// x as the products read it: packed into `out` where its lines are ragged, by
// a launch of its own (rows) or a job of `lines`.
template <typename T>
hipError_t pack_x(const Sizes& z, const void** x, void* out, LinesLaunch<T>* lines, hipStream_t st) {
  if (!z.rows(z.s.C)) return hipSuccess;
  const void* src = *x;
  *x = out;
  if (z.nhwc) return pack_rows<T>(src, z.P(), z.s.C, out, z.up(z.s.C), st);
  lines->turn(src, z.s.B, z.s.C, z.s.HW, nullptr, out, z.up(z.s.C));
  return hipSuccess;
}

// Rows and columns of the output, of `channels` channels, as the products write it
void output(GemmArgs* g, const Sizes& z, int64_t channels) {
  const int64_t P = z.P();
  g->R = (int)(z.nhwc ? P : channels), g->N = (int)(z.nhwc ? channels : P);
  g->ld = z.nhwc ? channels : z.s.HW, g->hw = z.images(), g->img = channels * z.s.HW;
}

// Whether a tensor of so many channels has rows that are not whole 16 bytes,
// which the epilogue writes in pieces.
bool ragged_rows(const Sizes& z, int64_t channels) { return (z.nhwc ? channels : z.s.HW) % z.vec != 0; }

constexpr int kFewRows = 32;   // beyond, 64 x 64 tiles in splits are as fast (64 positions of 4096 x 4096: 17 us, not 25)
bool few_rows(const Sizes& z) { return z.nhwc && z.P() <= kFewRows; }

struct FwdLayout {
  Plan p;
  size_t x, weight, part, total;
};
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
FwdLayout fwd_layout(const ProjectShape& s) {
  const Sizes z(s);
  FwdLayout l{};
  if (few_rows(z)) return l;
  GemmArgs g{};
  output(&g, z, s.O);
  l.p = plan(g.R, g.N, s.C, s.elem, ragged_rows(z, s.O), false);
  l.x = 0;
  l.weight = l.x + (z.rows(s.C) ? up256(z.packed(s.C)) : 0);
  l.part = l.weight + (z.weight() ? up256((size_t)s.O * z.up(s.C) * z.el()) : 0);
  l.total = l.part + (l.p.splits > 1 ? part_bytes(g.R, g.N, l.p) : 0);
  return l;
}

template <typename T>
hipError_t forward(const ProjectShape& s, const void* x, const void* w, const float* scale, const float* shift,
                   const void* res, void* y, void* z_out, char* ws, hipStream_t st) {
  const Sizes z(s);
  const FwdLayout l = fwd_layout(s);
  const bool turned = !z.nhwc && z.planes();
  if (few_rows(z)) {
    GemmArgs g{};
    output(&g, z, s.O);
    g.K = (int)s.C, g.a = Operand{x, s.C, 0, 0}, g.b = Operand{w, s.C, 0, 0};
    g.scale = scale, g.shift = shift, g.res = res, g.y = y, g.z = z_out, g.act = s.act;
    const dim3 grid((unsigned)ceil_div(s.O, 16)), block(kFewWaves * kWave);
    if (g.R <= 16)
      hipLaunchKernelGGL((k_project_few<T, 1>), grid, block, 0, st, g);
    else
      hipLaunchKernelGGL((k_project_few<T, 2>), grid, block, 0, st, g);
    return hipGetLastError();
  }
  LinesLaunch<T> lines;
  lines.weight(z, &w, nullptr, ws + l.weight);
  hipError_t e = pack_x(z, &x, ws + l.x, &lines, st);
  if (e == hipSuccess) e = lines.launch(st);
  if (e != hipSuccess) return e;
  GemmArgs g{};
  output(&g, z, s.O);
  g.K = (int)s.C;
  g.scale = scale, g.shift = shift, g.res = res, g.y = y, g.z = z_out, g.act = s.act, g.per_row = !z.nhwc;
  const Operand wo{w, z.up(s.C), 0, 0}, xo{x, z.up(s.C), 0, 0};
  float* part = reinterpret_cast<float*>(ws + l.part);
  if (z.nhwc) {
    g.a = xo, g.b = wo;
    return launch_whole<T, true, true>(g, l.p, part, st);
  }
  g.a = wo;
  if (turned) {
    g.b = xo;
    return launch_whole<T, true, true>(g, l.p, part, st);
  }
  g.b = Operand{x, s.HW, s.C * s.HW, z.images()};
  return launch_whole<T, true, false>(g, l.p, part, st);
}

// Many groups' sums (small planes) are added up in kManyRuns runs, behind
// them, first.  Returns where the sums that make dshift lie, and how many.
constexpr int kManyGroups = 4096, kManyRuns = 256;
hipError_t fewer_groups(float** part, int64_t* groups, int64_t O, hipStream_t st) {
  if (*groups <= kManyGroups) return hipSuccess;
  float* runs = *part + *groups * O;
  hipLaunchKernelGGL(k_project_dshift, dim3((unsigned)ceil_div(O, 16), kManyRuns), dim3(kThreads), 0, st, *part, *groups,
                     (int)O, runs);
  *part = runs, *groups = kManyRuns;
  return hipGetLastError();
}

// Groups of positions whose sums of dz lie apart: rows (channels-last) in up
// to 1024 workgroups, images or kRun positions of them (channels-first).
struct DzPlan {
  int tx;
  int64_t per, groups;
};
DzPlan dz_plan(const Sizes& z) {
  const ProjectShape& s = z.s;
  if (!z.nhwc) return DzPlan{0, 0, z.planes() ? s.B * ceil_div(s.HW, kRun) : s.B};
  const int tx = row_lanes(s.O);
  const int64_t M = z.P(), across = ceil_div(s.O, tx * 8), down = kThreads / tx;
  const int64_t want = std::max<int64_t>(1, 1024 / across);
  // few rows are one group's, whose sums are dshift
  const int64_t per = M <= 4 * down ? M : ceil_div(ceil_div(M, want), down) * down;
  return DzPlan{tx, per, ceil_div(M, per)};
}

}  // namespace

bool project_limits(const ProjectShape& s) {
  constexpr int64_t kCh = 1 << 20;
  if (s.C > kCh || s.O > kCh || s.HW > INT_MAX / std::max(s.C, s.O)) return false;
  // positions and elements whose threads one launch holds
  if (s.O > ((int64_t)1 << 35) / s.C) return false;
  return s.B <= ((int64_t)1 << 29) / s.HW && s.B <= ((int64_t)1 << 33) / (std::max(s.C, s.O) * s.HW);
}

size_t project_ws_bytes(const ProjectShape& s) { return fwd_layout(s).total; }

hipError_t launch_project(const ProjectShape& s, const void* x, const void* w, const float* scale, const float* shift,
                          const void* res, void* y, void* z, void* ws, hipStream_t st) {
  char* base = static_cast<char*>(ws);
  return s.elem == MOCE_F32 ? forward<float>(s, x, w, scale, shift, res, y, z, base, st)
                            : forward<uint16_t>(s, x, w, scale, shift, res, y, z, base, st);
}

namespace {

struct BwdLayout {
  Plan px, pw;
  size_t dz, x, weight, shift, part, total;
};
BwdLayout bwd_layout(const ProjectShape& s) {
  const Sizes z(s);
  BwdLayout l{};
  GemmArgs g{};
  output(&g, z, s.C);
  l.px = plan(g.R, g.N, s.O, s.elem, ragged_rows(z, s.C), false);
  l.pw = plan(s.O, s.C, z.P(), s.elem, s.C % z.vec != 0, z.nhwc || z.planes());
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += up256(n);
    return here;
  };
  l.dz = take(s.act != MOCE_ACT_NONE || z.rows(s.O) ? z.packed(s.O) : 0);
  l.x = take(z.rows(s.C) ? z.packed(s.C) : 0);
  l.weight = take((size_t)std::max(s.O * z.up(s.C), z.up(s.O) * s.C) * z.el());
  const int64_t groups = dz_plan(z).groups;
  l.shift = take((size_t)(groups + (groups > kManyGroups ? kManyRuns : 0)) * s.O * sizeof(float));
  // one after the other on the stream, so both products' partial sums share their place
  l.part = take(std::max(l.px.splits > 1 ? part_bytes(g.R, g.N, l.px) : 0, part_bytes(s.O, s.C, l.pw)));
  l.total = at;
  return l;
}

template <typename T>
hipError_t backward(const ProjectShape& s, const void* x, const void* w, const float* scale, const void* z_in,
                    const void* dy, const moce_project_grads& gr, char* ws, hipStream_t st) {
  const Sizes z(s);
  const BwdLayout l = bwd_layout(s);
  const bool smooth = s.act == MOCE_ACT_GELU || s.act == MOCE_ACT_SILU;
  const bool turned = !z.nhwc && z.planes();
  // Where dz is rounded anyway, the scale goes into it before the rounding
  // (one rounding, not two); where dz is dy or 0, into the weight of dx and
  // the rows of dW.  So each bfloat16 product has one rounded operand at most,
  // whose error is as large as the result's own rounding: dx (and, of GELU and
  // SiLU, dweight) is 2.35e-3 off in the 2-norm where exact operands leave
  // 1.66e-3.  Operands in two bfloat16 parts would leave that, for products
  // twice as long: the dx of 64 images of 256 to 1024 channels at 14 x 14 takes
  // 48 us and not 31, both products of 50432 tokens of 768 by 768 another 140
  // beside a backward of 203.
  const bool fold = scale && smooth;
  const float* row_scale = fold ? nullptr : scale;
  const bool products = gr.dx || gr.dweight || gr.dscale;
  const bool ragged = z.rows(s.O);
  const void* dz = dy;
  const DzPlan dp = dz_plan(z);
  float* sums = reinterpret_cast<float*>(ws + l.shift);   // of dz, by groups of positions
  int64_t groups = dp.groups;
  LinesLaunch<T> lines;
  hipError_t e = hipSuccess;
  {
    DzArgs a{};
    a.z = z_in, a.dy = dy, a.act = s.act, a.O = (int)s.O, a.hw = (int)s.HW, a.scale = fold ? scale : nullptr;
    a.dz = gr.dresidual != dy || s.act != MOCE_ACT_NONE ? gr.dresidual : nullptr;
    a.ld = (int)(!z.nhwc && !turned ? s.HW : z.up(s.O));
    if (products && (ragged || fold)) {
      dz = a.pack = ws + l.dz;
    } else if (products && s.act != MOCE_ACT_NONE) {
      if (!a.dz) a.dz = ws + l.dz;
      dz = a.dz;
    }
    a.part = !gr.dshift ? nullptr : groups == 1 ? gr.dshift : sums;
    if (a.dz || a.pack || a.part) {
      if (z.nhwc) {
        a.n = z.P(), a.per = dp.per;
        hipLaunchKernelGGL(k_project_dz_rows<T>, dim3((unsigned)dp.groups, (unsigned)ceil_div(s.O, dp.tx * 8)),
                           dim3(kThreads), 0, st, a, dp.tx);
        e = hipGetLastError();
      } else if (turned) {
        a.n = s.B;
        lines.add(a);
      } else {
        int lanes = 1;
        while (lanes < 64 && lanes * 8 < s.HW) lanes *= 2;
        a.n = s.B * s.O;
        hipLaunchKernelGGL(k_project_dz_planes<T>, dim3((unsigned)ceil_div(a.n, kThreads / lanes)), dim3(kThreads), 0,
                           st, a, lanes);
        e = hipGetLastError();
      }
      if (e != hipSuccess) return e;
    }
  }
  // what else the products read in lines of their own
  const bool dw = gr.dweight || gr.dscale;
  const void* wp = w;
  if (gr.dx && turned) {   // the weight turned too, so that both operands run along the outputs
    lines.turn(w, 1, s.O, s.C, row_scale, ws + l.weight, z.up(s.O));
    wp = ws + l.weight;
  } else if (gr.dx) {
    lines.weight(z, &wp, row_scale, ws + l.weight);
  }
  if (dw) e = pack_x(z, &x, ws + l.x, &lines, st);
  if (e == hipSuccess) e = lines.launch(st);
  const bool shift = gr.dshift && groups > 1;   // to be summed
  if (e == hipSuccess && shift) e = fewer_groups(&sums, &groups, s.O, st);
  if (e != hipSuccess) return e;
  float* part = reinterpret_cast<float*>(ws + l.part);
  const Operand dzo{dz, z.up(s.O), 0, 0}, dzp{dz, s.HW, s.O * s.HW, z.images()};   // lines of channels, of positions
  if (gr.dx) {
    GemmArgs g{};
    output(&g, z, s.C);
    g.K = (int)s.O, g.y = gr.dx;
    const Operand wo{wp, z.up(turned ? s.O : s.C), 0, 0};
    if (turned) {
      g.a = wo, g.b = dzo;
      e = launch_whole<T, true, true>(g, l.px, part, st);
    } else if (z.nhwc) {
      g.a = dzo, g.b = wo;
      e = launch_whole<T, true, false>(g, l.px, part, st);
    } else {
      g.a = wo, g.b = dzp;
      e = launch_whole<T, false, false>(g, l.px, part, st);
    }
    if (e != hipSuccess) return e;
  }
  const bool join = dw && (row_scale || l.pw.splits > 1);
  if (dw) {
    GemmArgs g{};
    g.R = (int)s.O, g.N = (int)s.C, g.K = (int)z.P(), g.ld = s.C, g.y = gr.dweight, g.klen = l.pw.klen;
    if (join) g.part = part;
    if (z.nhwc || turned) {
      g.a = dzo, g.b = Operand{x, z.up(s.C), 0, 0};
      e = launch_product<T, false, false>(g, l.pw, st);
    } else {
      g.a = dzp, g.b = Operand{x, s.HW, s.C * s.HW, z.images()};
      e = launch_product<T, true, true>(g, l.pw, st);
    }
    if (e != hipSuccess) return e;
  }
  const unsigned shifts = shift ? (unsigned)ceil_div(s.O, 16) : 0;
  if (join) {
    int across = 32;
    while (across < kThreads && across < s.C) across *= 2;
    hipLaunchKernelGGL(k_project_dweight<T>, dim3((unsigned)s.O + shifts), dim3(kThreads), 0, st, part, l.pw.splits,
                       (int)s.O, (int)s.C, row_scale, static_cast<const T*>(w), static_cast<T*>(gr.dweight), gr.dscale,
                       across, sums, groups, gr.dshift);
  } else if (shifts) {
    hipLaunchKernelGGL(k_project_dshift, dim3(shifts), dim3(kThreads), 0, st, sums, groups, (int)s.O, gr.dshift);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t line_product(const LineProduct& p, hipStream_t st) {
  LineArgs g{};
  g.a = Operand{p.a, p.lda, 0, 0}, g.b = Operand{p.b, p.ldb, 0, 0};
  g.pick = p.pick, g.other = p.other, g.alpha = p.alpha, g.add = p.add;
  g.R = p.R, g.N = p.N, g.K = p.K, g.klen = p.klen, g.y = p.y, g.ld = p.N, g.part = p.part;
  const Plan c{p.tile, (int)ceil_div(p.K, p.klen), p.klen, 0.};
  if (p.b_along) return launch_product<T, true, true>(static_cast<const GemmArgs&>(g), c, st);   // into part, no more
  const hipError_t e = p.a_along ? launch_product<T, true, false, LineFinish>(g, c, st)
                                 : launch_product<T, false, false, LineFinish>(g, c, st);
  if (e != hipSuccess || !p.part || !p.join) return e;
  return launch_join<T>(g, p.splits, st);
}
template <typename T>
hipError_t weight_lines(const void* w, int64_t O, int64_t C, void* out, hipStream_t st) {
  const ProjectShape s{1, C, 1, O, sizeof(T) == 4 ? MOCE_F32 : MOCE_BF16, MOCE_NHWC, MOCE_ACT_NONE};
  LinesLaunch<T> lines;
  lines.weight(Sizes(s), &w, nullptr, out);
  return lines.launch(st);
}

}  // namespace

hipError_t launch_line_product(int elem, const LineProduct& p, hipStream_t st) {
  return elem == MOCE_F32 ? line_product<float>(p, st) : line_product<uint16_t>(p, st);
}
hipError_t launch_weight_lines(int elem, const void* w, int64_t O, int64_t C, void* out, hipStream_t st) {
  return elem == MOCE_F32 ? weight_lines<float>(w, O, C, out, st) : weight_lines<uint16_t>(w, O, C, out, st);
}

size_t project_backward_ws_bytes(const ProjectShape& s) { return bwd_layout(s).total; }

// What forward() and backward() launch, by the table at the file's head
// (planes that are turned are lines of channels, as channels-last ones).
moce_project_cut project_path(const ProjectShape& s, int product) {
  const Sizes z(s);
  const bool forward = product == MOCE_PRODUCT_FORWARD, turned = !z.nhwc && z.planes(), lines = z.nhwc || turned;
  moce_project_cut c{};
  c.splits = 1;
  c.a_along = forward || (product == MOCE_PRODUCT_DX ? lines : !lines);
  c.b_along = forward ? lines : product == MOCE_PRODUCT_DX ? turned : !lines;
  if (forward && few_rows(z)) return c;
  const Plan p = forward ? fwd_layout(s).p : product == MOCE_PRODUCT_DX ? bwd_layout(s).px : bwd_layout(s).pw;
  c.rows = kTile[p.tile].tr, c.columns = kTile[p.tile].tc, c.stages = kTile[p.tile].stages, c.splits = p.splits;
  c.images = product == MOCE_PRODUCT_DWEIGHT && !lines && z.images() > 0;
  return c;
}

hipError_t launch_project_backward(const ProjectShape& s, const void* x, const void* w, const float* scale,
                                   const void* z, const void* dy, const moce_project_grads& gr, void* ws,
                                   hipStream_t st) {
  char* base = static_cast<char*>(ws);
  return s.elem == MOCE_F32 ? backward<float>(s, x, w, scale, z, dy, gr, base, st)
                            : backward<uint16_t>(s, x, w, scale, z, dy, gr, base, st);
}

}  // namespace moce
