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
#include <type_traits>

#include "moce_internal.h"

namespace moce {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kThreads = 256;   // four waves, 2 x 2 over the tile
constexpr int kLine = 128;      // bytes of k that a stage holds of every row or column

// One operand: line i starts at p + i ld, its element j lies at along(j)
// (elements).  hw: positions of an image where lines run over images img
// apart, else 0.
struct Operand {
  const void* p;
  int64_t ld, img;
  int hw;
};

struct GemmArgs {
  Operand a, b;
  int R, N, K;            // rows, columns, contraction
  int klen;               // contraction of one split, a multiple of the stage's
  int tr, tc;             // tiles down and across
  // output: row r at r ld, columns as an operand's line
  void *y, *z;
  const void* res;
  int64_t ld, img;
  int hw;
  float* part;            // [split][R][N] partial products in the place of y (nullptr: none)
  const float *scale, *shift;
  int per_row;            // scale and shift by row (else by column)
  int act;
};

// ---- elements ----------------------------------------------------------------
template <typename T>
struct Elem;
template <>
struct Elem<uint16_t> {
  static constexpr int kVec = 8;   // elements of 16 bytes
  static __device__ __forceinline__ float to_f(uint16_t v) { return bf16_to_f32(v); }
  static __device__ __forceinline__ uint16_t from_f(float v) { return f32_to_bf16(v); }
};
template <>
struct Elem<float> {
  static constexpr int kVec = 4;
  static __device__ __forceinline__ float to_f(float v) { return v; }
  static __device__ __forceinline__ float from_f(float v) { return v; }
};

// 8 elements at any alignment (the hardware's unaligned vector accesses)
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  u32x4 u;
  __builtin_memcpy(&u, p, 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(u[i]);
    v[2 * i + 1] = bf16_hi(u[i]);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) { __builtin_memcpy(v, p, 32); }
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  const u32x4 u = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                   pack_bf16x2(v[6], v[7])};
  __builtin_memcpy(p, &u, 16);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) { __builtin_memcpy(p, v, 32); }

// ---- activations -------------------------------------------------------------
// The standard normal distribution function of z, and e^(-z^2 / 2) beside it.
// float32 takes the library's complementary error function.  bfloat16 takes
// the rational approximation of Abramowitz and Stegun 7.1.26 (error of the
// error function below 1.5e-7), a quarter of the instructions.
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float* e) {
  if constexpr (sizeof(T) == 4) {
    *e = expf(-0.5f * z * z);
    return 0.5f * erfcf(-z * 0.70710678118654752f);
  } else {
    const float x = fabsf(z) * 0.70710678118654752f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
    *e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z);
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    const float q = 0.5f * p * t * *e;     // half the complementary error function of x
    return z > 0.f ? 1.f - q : q;
  }
}
template <typename T>
__device__ __forceinline__ float sigmoid(float z) {
  if constexpr (sizeof(T) == 4)
    return 1.f / (1.f + expf(-z));
  else
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
}

// act(z); the products are clamped so that infinities give the limits
template <typename T>
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == MOCE_ACT_RELU) return z < 0.f ? 0.f : z;
  if (act == MOCE_ACT_GELU) {
    float e;
    return fmaxf(z, -1e4f) * normal_cdf<T>(z, &e);
  }
  if (act == MOCE_ACT_SILU) return fmaxf(z, -1e4f) * sigmoid<T>(z);
  return z;
}
template <typename T>
__device__ __forceinline__ void act_values(float (&v)[8], int act) {
  if (act == MOCE_ACT_NONE) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = act_value<T>(v[i], act);
}
// act'(z) dy; ReLU selects, so that an upstream value that is not finite stays on its own positions
template <typename T>
__device__ __forceinline__ float act_gradient(float z, float dy, int act) {
  if (act == MOCE_ACT_RELU) return z <= 0.f ? 0.f : dy;
  if (act == MOCE_ACT_GELU) {
    float e;
    const float c = normal_cdf<T>(z, &e);
    return dy * fmaf(fminf(fmaxf(z, -1e4f), 1e4f) * 0.39894228040143268f, e, c);
  }
  if (act == MOCE_ACT_SILU) {
    const float s = sigmoid<T>(z);
    return dy * (s * fmaf(fminf(fmaxf(z, -1e4f), 1e4f), 1.f - s, 1.f));
  }
  return dy;
}

// ---- epilogue ----------------------------------------------------------------
// Eight neighbouring columns c.. of row r, from the float32 products v: into
// the partial products, or through scale, shift, residual and activation into
// z and y.  sc, sh: those of the eight columns (per column only).
template <typename T>
__device__ __forceinline__ void finish8(const GemmArgs& g, int r, int c, int split, float (&v)[8],
                                        const float (&sc)[8], const float (&sh)[8]) {
  using E = Elem<T>;
  if (r >= g.R || c >= g.N) return;
  const int n = min(8, g.N - c);
  if (g.part) {
    float* p = g.part + ((int64_t)split * g.R + r) * g.N + c;
    if (n == 8) {
      store8(p, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = v[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], sc[i], sh[i]);
  int64_t base = (int64_t)r * g.ld;
  int p = c;
  if (g.hw) {
    const int b = c / g.hw;
    p = c - b * g.hw;
    base += b * g.img;
  }
  T* y = static_cast<T*>(g.y) + base;
  T* z = g.z ? static_cast<T*>(g.z) + base : nullptr;
  const T* res = g.res ? static_cast<const T*>(g.res) + base : nullptr;
  if (n == 8 && (g.hw == 0 || p + 8 <= g.hw)) {
    if (res) {
      float q[8];
      load8(res + p, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += q[i];
    }
    if (z) store8(z + p, v);
    act_values<T>(v, g.act);
    store8(y + p, v);
    return;
  }
  int64_t o = p;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i < n) {
      if (res) v[i] += E::to_f(res[o]);
      if (z) z[o] = E::from_f(v[i]);
      y[o] = E::from_f(act_value<T>(v[i], g.act));
    }
    ++o;
    if (g.hw && ++p == g.hw) {
      p = 0;
      o += g.img - g.hw;
    }
  }
}
// scale and shift of columns c.. (ones and zeros where they go by row, or are not there)
__device__ __forceinline__ void column_affine(const GemmArgs& g, int c, float (&sc)[8], float (&sh)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = min(c + i, g.N - 1);
    sc[i] = g.scale && !g.per_row ? g.scale[j] : 1.f;
    sh[i] = g.shift && !g.per_row ? g.shift[j] : 0.f;
  }
}
__device__ __forceinline__ void row_affine(const GemmArgs& g, int r, float (&sc)[8], float (&sh)[8]) {
  if (!g.per_row) return;
  const int j = min(r, g.R - 1);
  const float s = g.scale ? g.scale[j] : 1.f, t = g.shift ? g.shift[j] : 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    sc[i] = s;
    sh[i] = t;
  }
}

// ---- the tile in LDS -----------------------------------------------------------
// A stage holds 128 bytes of k (64 bfloat16 or 32 float32) of every row and
// column of the tile, in chunks of 16 bytes:
//  - an operand along k: a line of 8 chunks per row, chunk c at c ^ key(row);
//  - along rows (or columns): a line of the tile's rows per k, chunk c at
//    c ^ key(k), read as matrix operands with the transposing load (bfloat16)
//    or single words (float32).
// The keys spread the lanes that read together over the banks.  Rows are
// taken in order; columns so that a lane's eight results are neighbours:
// index m of fragment f is column 32 (f / 2) + 8 (m / 4) + 4 (f % 2) + m % 4.
template <typename T, bool ALONG_K, int TILE, bool COLS>
struct Stage {
  static constexpr int kVec = Elem<T>::kVec;
  static constexpr int kDepth = kLine / (int)sizeof(T);   // of k
  static constexpr int kBytes = TILE * kLine;
  static constexpr int kChunks = TILE * 8;
  static constexpr int kPerLine = ALONG_K ? 8 : TILE / kVec;

  static __device__ __forceinline__ int key(int line) {
    if constexpr (ALONG_K) return COLS ? (line & 3) | ((line >> 1) & 4) : line & 7;
    if constexpr (sizeof(T) == 4)
      return COLS ? ((line >> 2) & 1) | (((line >> 2) & 2) << 2) : ((line >> 2) & 3) << 2;
    if constexpr (COLS) return TILE >= 128 ? (line & 3) << 2 : ((line >> 1) & 1) << 2;
    return (TILE >= 128 ? (line & 3) | ((line >> 1) & 4) : ((line >> 1) & 1) | ((line >> 2) & 2)) << 1;
  }
  // byte of chunk c of line i
  static __device__ __forceinline__ int at(int i, int c) { return i * (kPerLine * 16) + ((c ^ key(i)) << 4); }

  // Where this lane reads fragment 0 of the 16 rows or columns from w on, step
  // 0: the others lie at an exclusive or (of bits that w leaves clear) and a
  // constant from there.
  static __device__ __forceinline__ int place(int w, int lane) {
    const int g = lane >> 4, m = lane & 15, n = w + (COLS ? 8 * (m >> 2) + (m & 3) : m);
    if constexpr (ALONG_K) return at(n, g);
    if constexpr (sizeof(T) == 4) return at(4 * g, n >> 2) + 4 * (n & 3);
    const int q = lane & 3;
    return at(8 * g + ((lane >> 2) & 3), w / 8 + (COLS ? q : q >> 1)) + (COLS ? 0 : 8 * (q & 1));
  }
  // Fragment f of step ks (64 bytes of k).
  static __device__ __forceinline__ u32x4 frag(const unsigned char* s, int place, int f, int ks) {
    const int j = f >> 1, h = f & 1;
    if constexpr (ALONG_K) {
      return *reinterpret_cast<const u32x4*>(s + (place ^ (ks << 6)) + (COLS ? 32 * j + 4 * h : 16 * f) * kLine);
    } else if constexpr (sizeof(T) == 2) {
      constexpr int W = kPerLine * 16;
      const unsigned char* p = s + (place ^ (COLS ? j << 6 : f << 5)) + (COLS ? 8 * h : 0) + 32 * ks * W;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * W));
      return __builtin_bit_cast(u32x4, s16x8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w});
    } else {
      constexpr int W = kPerLine * 16;
      const unsigned char* p = s + (place ^ (COLS ? (j << 7) | (h << 4) : f << 6)) + 16 * ks * W;
      u32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const unsigned int*>(p + e * W);
      return v;
    }
  }
};

template <typename T>
__device__ __forceinline__ f32x4 multiply(u32x4 col, u32x4 row, f32x4 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, col), __builtin_bit_cast(bf16x8, row),
                                                   acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(col[e]), __uint_as_float(row[e]), acc, 0, 0, 0);
    return acc;
  }
}

// 16 bytes from element j of line i on, of lines below ni and elements below
// nj; zeros outside.  Any alignment; a chunk may pass from one image to the
// next.
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const Operand& o, int i, int ni, int j, int nj) {
  constexpr int VE = Elem<T>::kVec;
  u32x4 v = {0u, 0u, 0u, 0u};
  if (i >= ni || j >= nj) return v;
  const T* row = static_cast<const T*>(o.p) + i * o.ld;
  int p = j;
  if (o.hw) {
    const int b = j / o.hw;
    p = j - b * o.hw;
    row += b * o.img;
  }
  if (j + VE <= nj && (o.hw == 0 || p + VE <= o.hw)) {
    __builtin_memcpy(&v, row + p, 16);
    return v;
  }
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    if (j + e < nj) {
      if constexpr (sizeof(T) == 2)
        v[e / 2] |= (uint32_t)row[p] << (16 * (e & 1));
      else
        v[e] = __float_as_uint(row[p]);
    }
    if (++p == o.hw) {
      p = 0;
      row += o.img;
    }
  }
  return v;
}

// The tile of a workgroup.  Workgroup u runs on XCD u mod 8 and takes the
// (u / 8)-th of that XCD's eighth of the tiles, which go down kGroup rows of
// tiles before they go across: the tiles that run together on an XCD share
// the lines they read in its L2.  False past the last tile.
constexpr int kGroup = 8;
__device__ __forceinline__ bool tile_of(const GemmArgs& g, int& r, int& c) {
  const int u = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  if (u >= g.tr * g.tc) return false;
  const int band = u / (kGroup * g.tc), r0 = band * kGroup, n = min(kGroup, g.tr - r0), v = u - r0 * g.tc;
  r = r0 + v % n;
  c = v / n;
  return true;
}

// Scales, shifts and stores a wave's fragments: rows r0.., columns c0...
// They pass through BYTES of LDS at l, the wave's own, so that a row is
// written (and its residual read) as one run of memory, 32 FC bytes of
// bfloat16; chunk c of a row lies at c ^ (row & 7).  Where every eight columns
// are there or not (whole), kBatch rows' residuals are in flight together.
template <typename T, int BYTES, int FR, int FC>
__device__ __forceinline__ void finish(const GemmArgs& g, int r0, int c0, int lane, f32x4 (&acc)[FR][FC],
                                       unsigned char* l) {
  constexpr int kPitch = FC * 64, kAcross = 2 * FC, kDown = kWave / kAcross;
  constexpr int kFrags = BYTES / (16 * kPitch) < FR ? BYTES / (16 * kPitch) : FR;   // fragments of rows at a time
  constexpr int kIters = kFrags * 16 / kDown, kBatch = kIters < 4 ? kIters : 4;
  static_assert(FR % kFrags == 0 && kIters % kBatch == 0, "whole parts");
  const int x = lane % kAcross, dr = lane / kAcross, c = c0 + 8 * x;
  float sc[8], sh[8];
  column_affine(g, c, sc, sh);
  const bool whole = g.N % 8 == 0 && g.hw % 8 == 0;
  int64_t at = c;   // of the lane's columns within a row
  if (whole && g.hw) at = (c / g.hw) * g.img + c % g.hw;
#pragma unroll
  for (int f = 0; f < FR; f += kFrags) {
#pragma unroll
    for (int i = 0; i < kFrags; ++i)
#pragma unroll
      for (int j = 0; j < FC; ++j) {
        const int row = 16 * i + (lane & 15), ch = 8 * (j / 2) + 2 * (lane >> 4) + (j & 1);
        *reinterpret_cast<f32x4*>(l + row * kPitch + ((ch ^ (row & 7)) << 4)) = acc[f + i][j];
      }
    auto value = [&](int row, float (&v)[8]) __attribute__((always_inline)) {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(l + row * kPitch + (((2 * x) ^ (row & 7)) << 4));
      const f32x4 hi = *reinterpret_cast<const f32x4*>(l + row * kPitch + (((2 * x + 1) ^ (row & 7)) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = lo[e];
        v[4 + e] = hi[e];
      }
    };
    const int rf = r0 + 16 * f;
    if (whole && !g.part) {
      const T* res = static_cast<const T*>(g.res);
      T *y = static_cast<T*>(g.y), *z = static_cast<T*>(g.z);
      for (int it = 0; it < kIters; it += kBatch) {
        float q[kBatch][8];
        float rsc[kBatch], rsh[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int r = min(rf + (it + u) * kDown + dr, g.R - 1);
          rsc[u] = g.per_row && g.scale ? g.scale[r] : 1.f;
          rsh[u] = g.per_row && g.shift ? g.shift[r] : 0.f;
          if (res) load8(res + r * g.ld + (c < g.N ? at : 0), q[u]);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int row = (it + u) * kDown + dr, r = rf + row;
          float v[8];
          value(row, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], g.per_row ? rsc[u] : sc[e], g.per_row ? rsh[u] : sh[e]);
          if (res)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += q[u][e];
          const bool there = r < g.R && c < g.N;
          if (z && there) store8(z + r * g.ld + at, v);
          act_values<T>(v, g.act);
          if (there) store8(y + r * g.ld + at, v);
        }
      }
    } else {
      for (int it = 0; it < kIters; ++it) {
        const int row = it * kDown + dr;
        float v[8];
        value(row, v);
        row_affine(g, rf + row, sc, sh);
        finish8<T>(g, rf + row, c, blockIdx.y, v, sc, sh);
      }
    }
  }
}

template <int FR, int FC>
__device__ __forceinline__ void clear(f32x4 (&acc)[FR][FC]) {
#pragma unroll
  for (int i = 0; i < FR; ++i)
#pragma unroll
    for (int j = 0; j < FC; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// Any alignment: one tile of 32 FR rows by 32 FC columns, staged through
// registers; AK, BK: operands along k.
template <typename T, bool AK, bool BK, int FR, int FC>
__global__ void __launch_bounds__(kThreads)
k_project_any(GemmArgs g) {
  constexpr int TR = 32 * FR, TC = 32 * FC;
  using SA = Stage<T, AK, TR, false>;
  using SB = Stage<T, BK, TC, true>;
  constexpr int kDepth = SA::kDepth;
  __shared__ __attribute__((aligned(16))) unsigned char la[SA::kBytes + SB::kBytes];
  unsigned char* lb = la + SA::kBytes;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = (wave & 1) * 16 * FR, wc = (wave >> 1) * 16 * FC;
  int r0, c0;
  if (!tile_of(g, r0, c0)) return;
  r0 *= TR, c0 *= TC;
  const int k0 = blockIdx.y * g.klen, k1 = min(g.K, k0 + g.klen);

  f32x4 acc[FR][FC];
  clear(acc);
  const int pa = SA::place(wr, lane), pb = SB::place(wc, lane);
  for (int k = k0; k < k1; k += kDepth) {
    auto fetch = [&](auto s, const Operand& o, bool along_k, int n0, int n, unsigned char* l) __attribute__((always_inline)) {
      using S = decltype(s);
#pragma unroll
      for (int u = 0; u < S::kChunks / kThreads; ++u) {
        const int q = tid + u * kThreads, i = q / S::kPerLine, c = q % S::kPerLine;
        const u32x4 v = along_k ? load_chunk<T>(o, n0 + i, n, k + c * S::kVec, k1)
                                : load_chunk<T>(o, k + i, k1, n0 + c * S::kVec, n);
        *reinterpret_cast<u32x4*>(l + S::at(i, c)) = v;
      }
    };
    __syncthreads();
    fetch(SA{}, g.a, AK, r0, g.R, la);
    fetch(SB{}, g.b, BK, c0, g.N, lb);
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4 fa[FR], fb[FC];
#pragma unroll
      for (int i = 0; i < FR; ++i) fa[i] = SA::frag(la, pa, i, ks);
#pragma unroll
      for (int j = 0; j < FC; ++j) fb[j] = SB::frag(lb, pb, j, ks);
#pragma unroll
      for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
    }
  }
  __syncthreads();
  constexpr int kPart = (SA::kBytes + SB::kBytes) / 4;
  finish<T, kPart>(g, r0 + wr, c0 + wc, lane, acc, la + wave * kPart);
}

// ---- aligned lines: stages copied by the global-to-LDS loads ---------------------
//
// Where every line starts on 16 bytes and holds whole chunks (images too), a
// stage goes to LDS without passing registers, two stages in LDS: while the
// matrix cores work on the second half of stage s, whose operands are in
// registers by then, stage s + 2 is copied over it; its own copies have the
// time of a whole stage to arrive.  One barrier a stage.  The swizzle is in
// the lane's source address.  Chunks past the contraction's end come from a
// line of zeros; rows and columns past the tensor repeat its last ones, and
// are not stored.
__device__ __align__(16) unsigned int zero_chunk[4];

typedef __attribute__((address_space(3))) unsigned char lds_byte;

// s_waitcnt operands
constexpr int vm_wait(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }
constexpr int kLgkmWait0 = 0xc07f;

// 16 bytes from a scalar base and the lane's 32-bit offset (a buffer without
// bounds), to `to` and the lanes' places behind it.  With 64-bit addresses of
// its own a lane holds two registers for each of its chunks, which the
// products need.
__device__ __forceinline__ void buffer_to_lds(const char* base, uint32_t off, lds_byte* to) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass does not know the buffer's type
  const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, -1, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, to, 16, off, 0, 0, 0);
#endif
}

// The chunks of one operand that a thread copies in every stage.  IMG: the
// lines along k run over images, so that the lanes' places in them differ;
// else the place is the same for all, and the lanes' offsets from it stay.
template <typename T, bool ALONG_K, bool IMG, int TILE, bool COLS, int NT>
struct Copier {
  using S = Stage<T, ALONG_K, TILE, COLS>;
  static constexpr int kRounds = S::kChunks / NT;
  const char* base;      // the stage to copy next
  uint32_t off[kRounds];
  int64_t step;
  // IMG
  int64_t wrap;
  int k, hw;             // the lane's first position of the stage in its image

  __device__ __forceinline__ void init(const Operand& o, int n0, int n, int k0, int tid) {
    constexpr int ES = sizeof(T);
    base = static_cast<const char*>(o.p);
    if constexpr (ALONG_K) {
      const int c = (tid & 7) ^ S::key(tid >> 3);   // the same in every round
      if constexpr (IMG) {
        hw = o.hw;
        k = k0 + c * S::kVec;
        const int b = k / hw;
        k -= b * hw;
        base += (n0 * o.ld + b * o.img + k) * ES;
        wrap = (o.img - hw) * ES;
      } else {
        base += (n0 * o.ld + k0) * ES;
      }
      step = kLine;
#pragma unroll
      for (int u = 0; u < kRounds; ++u)
        off[u] = (uint32_t)((min(n0 + u * (NT / 8) + (tid >> 3), n - 1) - n0) * o.ld * ES) + (IMG ? 0 : c * 16);
    } else {
      const int b0 = o.hw ? n0 / o.hw : 0;
      base += (k0 * o.ld + b0 * o.img) * ES;
      step = (int64_t)S::kDepth * o.ld * ES;
#pragma unroll
      for (int u = 0; u < kRounds; ++u) {
        const int q = tid + u * NT, i = q / S::kPerLine, c = (q % S::kPerLine) ^ S::key(i);
        const int j = min(n0 + c * S::kVec, n - S::kVec);
        const int64_t at = o.hw ? (j / o.hw - b0) * o.img + j % o.hw : j;
        off[u] = (uint32_t)((i * o.ld + at) * ES);
      }
    }
  }
  // Copies a stage to l; CUT: of whose k only `left` elements are there.
  template <bool CUT>
  __device__ __forceinline__ void copy(unsigned char* l, int tid, int wave, int left) {
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      lds_byte* to = (lds_byte*)(l + (u * NT + wave * kWave) * 16);
      if constexpr (CUT || IMG) {
        const char* src = base + off[u];
        if constexpr (CUT) {
          const int at = ALONG_K ? ((tid & 7) ^ S::key(tid >> 3)) * S::kVec : (tid + u * NT) / S::kPerLine;
          if (at >= left) src = reinterpret_cast<const char*>(zero_chunk);
        }
        __builtin_amdgcn_global_load_lds((const void*)src, to, 16, 0, 0);
      } else {
        buffer_to_lds(base, off[u], to);
      }
    }
    base += step;
    if constexpr (IMG) {
      k += S::kDepth;
      while (k >= hw) {
        k -= hw;
        base += wrap;
      }
    }
  }
};

// WR x WC waves of FR x FC fragments.
template <typename T, bool AK, bool BK, bool IMG, int WR, int WC, int FR, int FC>
__global__ void __launch_bounds__(64 * WR * WC, 2)
k_project_copy(GemmArgs g) {
  constexpr int NT = 64 * WR * WC, TR = 16 * WR * FR, TC = 16 * WC * FC;
  using SA = Stage<T, AK, TR, false>;
  using SB = Stage<T, BK, TC, true>;
  constexpr int kDepth = SA::kDepth;
  // four arrays, so that the compiler sees the copies and the reads apart and
  // waits for a copy only where its array is read
  __shared__ __attribute__((aligned(16))) unsigned char a0[SA::kBytes], b0[SB::kBytes], a1[SA::kBytes], b1[SB::kBytes];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % WR * 16 * FR, wc = wave / WR * 16 * FC;
  int r0, c0;
  if (!tile_of(g, r0, c0)) return;
  r0 *= TR, c0 *= TC;
  const int k0 = blockIdx.y * g.klen, length = min(g.K, k0 + g.klen) - k0;
  const int n = (length + kDepth - 1) / kDepth;

  Copier<T, AK, AK && IMG, TR, false, NT> ca;
  Copier<T, BK, BK && IMG, TC, true, NT> cb;
  ca.init(g.a, r0, g.R, k0, tid);
  cb.init(g.b, c0, g.N, k0, tid);
  f32x4 acc[FR][FC];
  clear(acc);
  // A stage goes in four phases: step 0 and 1, the upper and lower half of the
  // wave's rows; the operands of a phase are read during the one before.
  constexpr int FH = FR / 2;
  u32x4 fa[2][FH], fb[2][FC];
  int pa = SA::place(wr, lane), pb = SB::place(wc, lane);
  auto read = [&](int phase, const unsigned char* la, const unsigned char* lb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FH; ++i) fa[phase & 1][i] = SA::frag(la, pa, (phase & 1) * FH + i, phase >> 1);
    if ((phase & 1) == 0)
#pragma unroll
      for (int j = 0; j < FC; ++j) fb[phase >> 1][j] = SB::frag(lb, pb, j, phase >> 1);
  };
  auto products = [&](int phase) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FH; ++i)
#pragma unroll
      for (int j = 0; j < FC; ++j) {
        f32x4& c = acc[(phase & 1) * FH + i][j];
        c = multiply<T>(fb[phase >> 1][j], fa[phase & 1][i], c);
      }
  };
  auto publish = [&]() __attribute__((always_inline)) {   // this wave's reads and copies are done, then everyone's
    __builtin_amdgcn_s_waitcnt(kLgkmWait0);
    __builtin_amdgcn_s_waitcnt(vm_wait(0));
    __syncthreads();
  };
  // Stage s lies in (la, lb), its first phase's operands in registers; copies
  // stage s + 2 (cut: `left` of it) and leaves the next one's first operands.
  auto stage = [&](auto cut, int left, unsigned char* la, unsigned char* lb, unsigned char* na,
                   unsigned char* nb) __attribute__((always_inline)) {
    asm volatile("" : "+v"(pa), "+v"(pb));   // the places of the fragments are formed here, not kept
    read(1, la, lb);
    products(0);
    __builtin_amdgcn_sched_barrier(0);   // no phase's reads before the one ahead of it: registers
    read(2, la, lb);
    products(1);
    __builtin_amdgcn_sched_barrier(0);
    read(3, la, lb);
    products(2);
    __builtin_amdgcn_sched_barrier(0);
    publish();
    ca.template copy<decltype(cut)::value>(la, tid, wave, left);
    cb.template copy<decltype(cut)::value>(lb, tid, wave, left);
    read(0, na, nb);
    products(3);
    __builtin_amdgcn_sched_barrier(0);
  };
  const std::integral_constant<bool, true> some{};
  const std::integral_constant<bool, false> all{};
  ca.template copy<true>(a0, tid, wave, length);
  cb.template copy<true>(b0, tid, wave, length);
  publish();
  ca.template copy<true>(a1, tid, wave, length - kDepth);
  cb.template copy<true>(b1, tid, wave, length - kDepth);
  read(0, a0, b0);
  int left = length - 2 * kDepth;   // of the stage to copy next
  int s = 0;
  for (; left >= 2 * kDepth; s += 2, left -= 2 * kDepth) {
    stage(all, 0, a0, b0, a1, b1);
    stage(all, 0, a1, b1, a0, b0);
  }
  for (; s + 1 < n; s += 2, left -= 2 * kDepth) {
    stage(some, left, a0, b0, a1, b1);
    stage(some, left - kDepth, a1, b1, a0, b0);
  }
  if (s < n) stage(some, left, a0, b0, a1, b1);
  publish();
  // a wave's part of LDS for its results
  constexpr int kEach = WR * WC / 4, kPart = (SA::kBytes < SB::kBytes ? SA::kBytes : SB::kBytes) / kEach;
  const int w = wave / kEach;
  finish<T, kPart>(g, r0 + wr, c0 + wc, lane, acc, (w == 0 ? a0 : w == 1 ? b0 : w == 2 ? a1 : b1) + wave % kEach * kPart);
}

// Sums the splits' partial products, in order, and finishes them.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_join(GemmArgs g, int splits) {
  const int per = (g.N + 7) / 8;
  const int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int r = (int)(u / per), c = (int)(u % per) * 8;
  if (r >= g.R) return;
  float v[8] = {};
  for (int s = 0; s < splits; ++s) {
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
  GemmArgs h = g;
  h.part = nullptr;
  float sc[8], sh[8];
  column_affine(h, c, sc, sh);
  row_affine(h, r, sc, sh);
  finish8<T>(h, r, c, 0, v, sc, sh);
}

// ---- the gradients' other passes -------------------------------------------------

__device__ __forceinline__ float block_sum(float v) {
  __shared__ float s[kThreads / kWave];
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Row o of the weight's gradient from the splits' G: dweight = scale G, dscale = <weight, G>.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_dweight(const float* __restrict__ part, int splits, int O, int C, const float* __restrict__ scale,
                  const T* __restrict__ weight, T* __restrict__ dweight, float* __restrict__ dscale) {
  const int o = blockIdx.x;
  const float sc = scale ? scale[o] : 1.f;
  float dot = 0.f;
  for (int c = threadIdx.x; c < C; c += kThreads) {
    float v = 0.f;
    for (int s = 0; s < splits; ++s) v += part[((int64_t)s * O + o) * C + c];
    const int64_t e = (int64_t)o * C + c;
    if (dweight) dweight[e] = Elem<T>::from_f(sc * v);
    if (dscale) dot = fmaf(v, Elem<T>::to_f(weight[e]), dot);
  }
  if (!dscale) return;
  dot = block_sum(dot);
  if (threadIdx.x == 0) dscale[o] = dot;
}

struct DzArgs {
  const void *z, *dy;
  void *dz, *dzs;         // act'(z) dy, and scale times that (either may be nullptr)
  const float* scale;
  float* part;            // [groups][O] partial sums of dz over positions (nullptr: none)
  int act, O, hw;
  int64_t n;              // rows of positions (channels-last), planes (channels-first)
  int64_t per;            // rows of one group
};

// dz of eight neighbouring elements (n of them there) at e, scaled by sc for dzs
template <typename T>
__device__ __forceinline__ void dz8(const DzArgs& a, int64_t e, int n, const float (&sc)[8], float (&v)[8]) {
  using E = Elem<T>;
  const T *z = static_cast<const T*>(a.z), *dy = static_cast<const T*>(a.dy);
  T *dz = static_cast<T*>(a.dz), *dzs = static_cast<T*>(a.dzs);
  if (n == 8) {
    float q[8];
    load8(dy + e, v);
    if (a.act != MOCE_ACT_NONE) {
      load8(z + e, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = act_gradient<T>(q[i], v[i], a.act);
    }
    if (dz) store8(dz + e, v);
    if (dzs) {
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = v[i] * sc[i];
      store8(dzs + e, q);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = 0.f;
    if (i < n) {
      v[i] = E::to_f(dy[e + i]);
      if (a.act != MOCE_ACT_NONE) v[i] = act_gradient<T>(E::to_f(z[e + i]), v[i], a.act);
      if (dz) dz[e + i] = E::from_f(v[i]);
      if (dzs) dzs[e + i] = E::from_f(v[i] * sc[i]);
    }
  }
}

// Channels-last: a workgroup takes 8 tx channels of a group of rows, its
// threads tx across and 256 / tx down.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_dz_rows(DzArgs a, int tx) {
  __shared__ float s[kThreads][8 + 1];
  const int x = threadIdx.x % tx, down = kThreads / tx;
  const int c = (blockIdx.y * tx + x) * 8, n = min(8, a.O - c);
  float sum[8] = {}, sc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) sc[i] = a.dzs ? a.scale[max(0, min(c + i, a.O - 1))] : 1.f;
  if (n > 0) {
    const int64_t end = min(a.n, (blockIdx.x + (int64_t)1) * a.per);
    for (int64_t r = blockIdx.x * a.per + threadIdx.x / tx; r < end; r += down) {
      float v[8];
      dz8<T>(a, r * a.O + c, n, sc, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += v[i];
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

// Channels-first: `lanes` lanes (a power of two up to 64) take a plane.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_dz_planes(DzArgs a, int lanes) {
  const int64_t plane = (int64_t)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes;
  float sum = 0.f, sc[8];
  if (plane < a.n) {
    const float f = a.dzs ? a.scale[plane % a.O] : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sc[i] = f;
    for (int p = (threadIdx.x % lanes) * 8; p < a.hw; p += lanes * 8) {
      float v[8];
      dz8<T>(a, plane * a.hw + p, min(8, a.hw - p), sc, v);
      sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
  }
  if (!a.part) return;
  for (int o = lanes / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
  if (plane < a.n && threadIdx.x % lanes == 0) a.part[plane] = sum;
}

// dshift[o] = sum over the groups' partial sums
__global__ void __launch_bounds__(1024)
k_project_dshift(const float* __restrict__ part, int64_t groups, int O, float* __restrict__ dshift) {
  __shared__ float s[16][64];
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6, o = blockIdx.x * 64 + x;
  float t = 0.f;
  if (o < O)
    for (int64_t i = y; i < groups; i += 16) t += part[i * O + o];
  s[y][x] = t;
  __syncthreads();
  if (y == 0 && o < O) {
    t = s[0][x];
    for (int i = 1; i < 16; ++i) t += s[i][x];
    dshift[o] = t;
  }
}

// scale[o] weight[o][c], rounded to the weight's type
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_scale(const T* __restrict__ weight, const float* __restrict__ scale, int C, T* __restrict__ out) {
  const int o = blockIdx.x;
  const float s = scale[o];
  for (int c = threadIdx.x; c < C; c += kThreads)
    out[(int64_t)o * C + c] = Elem<T>::from_f(s * Elem<T>::to_f(weight[(int64_t)o * C + c]));
}

// ---- launches --------------------------------------------------------------------

constexpr int kWantTiles = 512;          // two workgroups a CU

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a product is cut: tiles of `tile` rows and columns and, where these
// make too few workgroups for the GPU, the contraction in lengths of 256 or more.
struct Plan {
  int tile, splits, klen;
};
Plan plan(int64_t R, int64_t N, int64_t K, int elem) {
  const int depth = kLine / (elem == MOCE_F32 ? 4 : 2);
  int tile = 64;
  if (ceil_div(R, 128) * ceil_div(N, 128) >= 256) tile = 128;
  if (elem == MOCE_BF16 && ceil_div(R, 256) * ceil_div(N, 256) >= 256) tile = 256;
  const int64_t tiles = ceil_div(R, tile) * ceil_div(N, tile);
  int64_t s = std::min(std::max<int64_t>(1, kWantTiles / tiles), std::max<int64_t>(1, K / 256));
  s = std::min<int64_t>(s, 256);
  const int64_t klen = ceil_div(ceil_div(K, s), depth) * depth;
  return Plan{tile, (int)ceil_div(K, klen), (int)klen};
}
size_t part_bytes(int64_t R, int64_t N, const Plan& p) { return (size_t)p.splits * R * N * sizeof(float); }

// Whether the copying kernel can read this operand: whole chunks, at offsets of 31 bits within a tile.
bool whole_chunks(const Operand& o, bool along_k, int64_t length, int elem) {
  const int es = elem == MOCE_F32 ? 4 : 2, vec = 16 / es;
  if (o.ld % vec || o.hw % vec || length % vec) return false;
  const int64_t span = along_k ? 256 * o.ld : (kLine / es) * o.ld + (o.hw ? (256 / o.hw + 2) * o.img : 0);
  return span * es < INT_MAX;
}

template <typename T, bool AK, bool BK, bool IMG, int WR, int WC, int F, int FC>
void launch_copy(GemmArgs g, int splits, hipStream_t st) {
  g.tr = (int)ceil_div(g.R, 16 * WR * F), g.tc = (int)ceil_div(g.N, 16 * WC * FC);
  const dim3 grid((unsigned)(ceil_div((int64_t)g.tr * g.tc, 8) * 8), splits);
  hipLaunchKernelGGL((k_project_copy<T, AK, BK, IMG, WR, WC, F, FC>), grid, dim3(64 * WR * WC), 0, st, g);
}

template <typename T, bool AK, bool BK, int F>
void launch_any(GemmArgs g, int splits, hipStream_t st) {
  g.tr = (int)ceil_div(g.R, 32 * F), g.tc = (int)ceil_div(g.N, 32 * F);
  const dim3 grid((unsigned)(ceil_div((int64_t)g.tr * g.tc, 8) * 8), splits);
  hipLaunchKernelGGL((k_project_any<T, AK, BK, F, F>), grid, dim3(kThreads), 0, st, g);
}

template <typename T, bool AK, bool BK>
hipError_t launch_product(const GemmArgs& g, const Plan& p, hipStream_t st) {
  const int elem = sizeof(T) == 4 ? MOCE_F32 : MOCE_BF16;
  const bool whole = whole_chunks(g.a, AK, AK ? g.K : g.R, elem) && whole_chunks(g.b, BK, BK ? g.K : g.N, elem);
  auto copy = [&](auto img) {
    constexpr bool IMG = decltype(img)::value;
    if (p.tile == 64)
      launch_copy<T, AK, BK, IMG, 2, 2, 2, 2>(g, p.splits, st);
    else if (p.tile == 128 || sizeof(T) == 4)
      launch_copy<T, AK, BK, IMG, 2, 2, 4, 4>(g, p.splits, st);
    else if constexpr (sizeof(T) == 2)
      launch_copy<T, AK, BK, IMG, 2, 4, 8, 4>(g, p.splits, st);
  };
  if (!whole) {
    if (p.tile == 64)
      launch_any<T, AK, BK, 2>(g, p.splits, st);
    else
      launch_any<T, AK, BK, 4>(g, p.splits, st);
  } else if constexpr (AK && BK) {
    if (g.a.hw)
      copy(std::true_type{});
    else
      copy(std::false_type{});
  } else {
    copy(std::false_type{});
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_join(const GemmArgs& g, int splits, hipStream_t st) {
  hipLaunchKernelGGL(k_project_join<T>, dim3((unsigned)ceil_div((int64_t)g.R * ceil_div(g.N, 8), kThreads)),
                     dim3(kThreads), 0, st, g, splits);
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

// The positions' part of a channels-first tensor of n channels
int images(const ProjectShape& s) { return s.layout == MOCE_NCHW && s.B > 1 ? (int)s.HW : 0; }

template <typename T>
hipError_t forward(const ProjectShape& s, const void* x, const void* w, const float* scale, const float* shift,
                   const void* res, void* y, void* z, float* part, hipStream_t st) {
  const int P = (int)(s.B * s.HW), hw = images(s);
  GemmArgs g{};
  g.K = (int)s.C;
  g.scale = scale, g.shift = shift, g.res = res, g.y = y, g.z = z, g.act = s.act;
  const Operand wo{w, s.C, 0, 0};
  if (s.layout == MOCE_NHWC) {
    g.a = Operand{x, s.C, 0, 0}, g.b = wo, g.R = P, g.N = (int)s.O, g.ld = s.O;
    return launch_whole<T, true, true>(g, plan(g.R, g.N, g.K, s.elem), part, st);
  }
  g.a = wo, g.b = Operand{x, s.HW, s.C * s.HW, hw}, g.R = (int)s.O, g.N = P, g.per_row = 1;
  g.ld = s.HW, g.img = s.O * s.HW, g.hw = hw;
  return launch_whole<T, true, false>(g, plan(g.R, g.N, g.K, s.elem), part, st);
}

// Groups of positions whose sums of dz lie apart: rows (channels-last) in up
// to 1024 workgroups, images (channels-first).
struct DzPlan {
  int tx;
  int64_t per, groups;
};
DzPlan dz_plan(const ProjectShape& s) {
  if (s.layout == MOCE_NCHW) return DzPlan{0, 0, s.B};
  int tx = 1;
  while (tx < 32 && tx * 8 < s.O) tx *= 2;
  const int64_t M = s.B * s.HW, across = ceil_div(s.O, tx * 8), down = kThreads / tx;
  const int64_t want = std::max<int64_t>(1, 1024 / across);
  const int64_t per = ceil_div(ceil_div(M, want), down) * down;
  return DzPlan{tx, per, ceil_div(M, per)};
}

}  // namespace

bool project_limits(const ProjectShape& s) {
  constexpr int64_t kCh = 1 << 20;
  if (s.C > kCh || s.O > kCh || s.HW > INT_MAX / std::max(s.C, s.O)) return false;
  // positions and elements whose threads one launch holds
  return s.B <= ((int64_t)1 << 29) / s.HW && s.B <= ((int64_t)1 << 33) / (std::max(s.C, s.O) * s.HW);
}

size_t project_ws_bytes(const ProjectShape& s) {
  const bool nhwc = s.layout == MOCE_NHWC;
  const int64_t P = s.B * s.HW, R = nhwc ? P : s.O, N = nhwc ? s.O : P;
  const Plan p = plan(R, N, s.C, s.elem);
  return p.splits > 1 ? part_bytes(R, N, p) : 0;
}

hipError_t launch_project(const ProjectShape& s, const void* x, const void* w, const float* scale, const float* shift,
                          const void* res, void* y, void* z, void* ws, hipStream_t st) {
  float* part = static_cast<float*>(ws);
  return s.elem == MOCE_F32 ? forward<float>(s, x, w, scale, shift, res, y, z, part, st)
                            : forward<uint16_t>(s, x, w, scale, shift, res, y, z, part, st);
}

ProjectBwdSizes project_backward_sizes(const ProjectShape& s) {
  const size_t el = s.elem == MOCE_F32 ? 4 : 2;
  const int64_t P = s.B * s.HW;
  const bool nhwc = s.layout == MOCE_NHWC;
  const Plan px = nhwc ? plan(P, s.C, s.O, s.elem) : plan(s.C, P, s.O, s.elem);
  const Plan pw = plan(s.O, s.C, P, s.elem);
  ProjectBwdSizes z{};
  z.dz = s.act == MOCE_ACT_NONE ? 0 : (size_t)P * s.O * el;
  z.weight = (size_t)s.O * s.C * el;
  z.shift = (size_t)dz_plan(s).groups * s.O * sizeof(float);
  // one after the other on the stream, so both products' partial sums share their place
  z.part = std::max(px.splits > 1 ? part_bytes(P, s.C, px) : 0, part_bytes(s.O, s.C, pw));
  return z;
}

namespace {

template <typename T>
hipError_t backward(const ProjectShape& s, const void* x, const void* w, const float* scale, const void* z,
                    const void* dy, const moce_project_grads& gr, const ProjectBwdWs& ws, hipStream_t st) {
  const int P = (int)(s.B * s.HW), hw = images(s);
  const bool nhwc = s.layout == MOCE_NHWC;
  const bool smooth = s.act == MOCE_ACT_GELU || s.act == MOCE_ACT_SILU;
  // Where dz is rounded anyway, the scale goes into it before the rounding
  // (one rounding, not two); where dz is dy or 0, into the weight of dx and
  // the rows of dW.
  const bool fold = scale && smooth;
  const bool products = gr.dx || gr.dweight || gr.dscale;
  const void* dz = dy;
  hipError_t e;
  {
    DzArgs a{};
    a.z = z, a.dy = dy, a.act = s.act, a.O = (int)s.O, a.hw = (int)s.HW, a.scale = scale;
    a.dz = gr.dresidual != dy || s.act != MOCE_ACT_NONE ? gr.dresidual : nullptr;
    if (fold) {
      if (products) dz = a.dzs = ws.dz;
    } else if (s.act != MOCE_ACT_NONE && products) {
      if (!a.dz) a.dz = ws.dz;
      dz = a.dz;
    }
    a.part = gr.dshift ? ws.shift : nullptr;
    const DzPlan dp = dz_plan(s);
    if (a.dz || a.dzs || a.part) {
      if (nhwc) {
        a.n = P, a.per = dp.per;
        hipLaunchKernelGGL(k_project_dz_rows<T>, dim3((unsigned)dp.groups, (unsigned)ceil_div(s.O, dp.tx * 8)),
                           dim3(kThreads), 0, st, a, dp.tx);
      } else {
        int lanes = 1;
        while (lanes < 64 && lanes * 8 < s.HW) lanes *= 2;
        a.n = s.B * s.O;
        hipLaunchKernelGGL(k_project_dz_planes<T>, dim3((unsigned)ceil_div(a.n, kThreads / lanes)), dim3(kThreads), 0,
                           st, a, lanes);
      }
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (gr.dshift) {
      hipLaunchKernelGGL(k_project_dshift, dim3((unsigned)ceil_div(s.O, 64)), dim3(1024), 0, st, ws.shift, dp.groups,
                         (int)s.O, gr.dshift);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  const float* row_scale = fold ? nullptr : scale;
  if (gr.dx) {
    if (row_scale) {
      hipLaunchKernelGGL(k_project_scale<T>, dim3((unsigned)s.O), dim3(kThreads), 0, st, static_cast<const T*>(w),
                         scale, (int)s.C, static_cast<T*>(ws.weight));
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    GemmArgs g{};
    const Operand wo{row_scale ? ws.weight : w, s.C, 0, 0};
    g.K = (int)s.O, g.y = gr.dx;
    if (nhwc) {
      g.a = Operand{dz, s.O, 0, 0}, g.b = wo, g.R = P, g.N = (int)s.C, g.ld = s.C;
      e = launch_whole<T, true, false>(g, plan(g.R, g.N, g.K, s.elem), ws.part, st);
    } else {
      g.a = wo, g.b = Operand{dz, s.HW, s.O * s.HW, hw}, g.R = (int)s.C, g.N = P;
      g.ld = s.HW, g.img = s.C * s.HW, g.hw = hw;
      e = launch_whole<T, false, false>(g, plan(g.R, g.N, g.K, s.elem), ws.part, st);
    }
    if (e != hipSuccess) return e;
  }
  if (gr.dweight || gr.dscale) {
    GemmArgs g{};
    const Plan p = plan(s.O, s.C, P, s.elem);
    g.R = (int)s.O, g.N = (int)s.C, g.K = P, g.ld = s.C, g.y = gr.dweight, g.klen = p.klen;
    const bool join = row_scale || p.splits > 1;
    if (join) g.part = ws.part;
    if (nhwc) {
      g.a = Operand{dz, s.O, 0, 0}, g.b = Operand{x, s.C, 0, 0};
      e = launch_product<T, false, false>(g, p, st);
    } else {
      g.a = Operand{dz, s.HW, s.O * s.HW, hw}, g.b = Operand{x, s.HW, s.C * s.HW, hw};
      e = launch_product<T, true, true>(g, p, st);
    }
    if (e != hipSuccess) return e;
    if (join) {
      hipLaunchKernelGGL(k_project_dweight<T>, dim3((unsigned)s.O), dim3(kThreads), 0, st, ws.part, p.splits, (int)s.O,
                         (int)s.C, row_scale, static_cast<const T*>(w), static_cast<T*>(gr.dweight), gr.dscale);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_project_backward(const ProjectShape& s, const void* x, const void* w, const float* scale,
                                   const void* z, const void* dy, const moce_project_grads& gr,
                                   const ProjectBwdWs& ws, hipStream_t st) {
  return s.elem == MOCE_F32 ? backward<float>(s, x, w, scale, z, dy, gr, ws, st)
                            : backward<uint16_t>(s, x, w, scale, z, dy, gr, ws, st);
}

}  // namespace moce
