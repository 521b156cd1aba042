// The tiled matrix product of the dense projections and of the heads' losses:
// operands by lines, tiles in LDS, the model that cuts a product into tiles, and
// the epilogue that writes it.  project.hip's head says which operand lies how.
#pragma once

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
  int tr, tc, splits;     // tiles down and across, parts of the contraction
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
// A product of the heads' gradients.  (In GemmArgs these cost the projections 2
// to 4%: 50432 tokens of 768 by 768, 97 us and not 93.)
struct LineArgs : GemmArgs {
  int add;                // to what the partial products hold
  const float* alpha;     // a factor of everything (nullptr: 1)
  const float* pick;      // where *pick is not 0, b lies at `other` (nullptr: no choice)
  const void* other;
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

// Two values rounded to bfloat16 by one conversion (of one value each they
// take two, and two more to join).
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

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
  const u32x4 u = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
  __builtin_memcpy(p, &u, 16);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) { __builtin_memcpy(p, v, 32); }

__device__ __forceinline__ void load4(const uint16_t* p, float* v) {
  uint32_t u[2];
  __builtin_memcpy(u, p, 8);
  v[0] = bf16_lo(u[0]), v[1] = bf16_hi(u[0]), v[2] = bf16_lo(u[1]), v[3] = bf16_hi(u[1]);
}
__device__ __forceinline__ void load4(const float* p, float* v) { __builtin_memcpy(v, p, 16); }
__device__ __forceinline__ void store4(uint16_t* p, const float* v) {
  const uint32_t u[2] = {pack2(v[0], v[1]), pack2(v[2], v[3])};
  __builtin_memcpy(p, u, 8);
}
__device__ __forceinline__ void store4(float* p, const float* v) { __builtin_memcpy(p, v, 16); }

// The same past the caches, for results in whole aligned rows.
__device__ __forceinline__ void stream8(uint16_t* p, const float (&v)[8]) {
  const u32x4 u = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
  __builtin_nontemporal_store(u, reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ void stream8(float* p, const float (&v)[8]) {
  __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4*>(p));
  __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4*>(p + 4));
}

// ---- activations -------------------------------------------------------------
// The standard normal distribution function of z, and e^(-z^2 / 2) beside it
// (the derivative of GELU, whose float32 sums keep its error).  float32 takes
// the library's complementary error function; bfloat16 the rational
// approximation of Abramowitz and Stegun 7.1.26 (error of the error function
// below 1.5e-7), a quarter of the instructions.
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
    if constexpr (sizeof(T) == 4) {
      float e;
      return fmaxf(z, -1e4f) * normal_cdf<T>(z, &e);
    }
    // max(z, 0) - x Q(x) with x = |z| and Q(x) = P(Z > x) for a normal Z: log2
    // Q is smooth, and this polynomial (a minimax fit in log2 Q up to x = 13,
    // where x Q leaves the normal numbers) leaves 4e-6 of Q at x < 1, 2.1e-5
    // at x < 3 and 1.1e-4 everywhere: 1/35 of a rounding to bfloat16.  Beyond
    // 13 it only falls.
    const float x = fabsf(z);
    float p = fmaf(-1.696558005e-9f, x, 1.301394263e-7f);
    p = fmaf(p, x, -4.336038273e-6f);
    p = fmaf(p, x, 8.308103133e-5f);
    p = fmaf(p, x, -1.025861013e-3f);
    p = fmaf(p, x, 8.733066730e-3f);
    p = fmaf(p, x, -5.423573032e-2f);
    p = fmaf(p, x, -4.583052695e-1f);
    p = fmaf(p, x, -1.151285052f);
    p = fmaf(p, x, -9.999940991e-1f);
    return fmaf(-fminf(x, 1e4f), __builtin_amdgcn_exp2f(p), fmaxf(z, 0.f));
  }
  if (act == MOCE_ACT_SILU) return fmaxf(z, -1e4f) * sigmoid<T>(z);
  return z;
}
template <typename T, int N>
__device__ __forceinline__ void act_values(float (&v)[N][8], int act) {
  auto all = [&](int a) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] = act_value<T>(v[u][i], a);
  };
  if (act == MOCE_ACT_RELU) all(MOCE_ACT_RELU);
  if (act == MOCE_ACT_GELU) all(MOCE_ACT_GELU);
  if (act == MOCE_ACT_SILU) all(MOCE_ACT_SILU);
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
template <typename T, typename G>
__device__ __forceinline__ void finish8(const G& g, int r, int c, int split, float (&v)[8],
                                        const float (&sc)[8], const float (&sh)[8]) {
  using E = Elem<T>;
  if (r >= g.R || c >= g.N) return;
  const int n = min(8, g.N - c);
  if (g.part) {
    float* p = g.part + ((int64_t)split * g.R + r) * g.N + c;
    if constexpr (std::is_same_v<G, LineArgs>) {
      if (g.add) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) v[i] += p[i];
      }
    }
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
  T *y = static_cast<T*>(g.y), *z = static_cast<T*>(g.z);
  const T* res = static_cast<const T*>(g.res);
#pragma unroll
  for (int h = 0; h < 8; h += 4) {   // halves: planes of four positions and their multiples have them whole
    if (h >= n) break;
    int64_t at = (int64_t)r * g.ld + c + h;
    int p = c + h;
    if (g.hw) {
      const int b = p / g.hw;
      at += b * (g.img - g.hw);
      p -= b * g.hw;
    }
    if (h + 4 <= n && (g.hw == 0 || p + 4 <= g.hw)) {
      if (res) {
        float q[4];
        load4(res + at, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[h + i] += q[i];
      }
      if (z) store4(z + at, v + h);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[h + i] = act_value<T>(v[h + i], g.act);
      store4(y + at, v + h);
      continue;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (h + i < n) {
        if (res) v[h + i] += E::to_f(res[at]);
        if (z) z[at] = E::from_f(v[h + i]);
        y[at] = E::from_f(act_value<T>(v[h + i], g.act));
      }
      ++at;
      if (g.hw && ++p == g.hw) {
        p = 0;
        at += g.img - g.hw;
      }
    }
  }
}
// scale and shift of columns c.. (ones and zeros where they go by row, or are not there)
template <typename G>
__device__ __forceinline__ void column_affine(const G& g, int c, float (&sc)[8], float (&sh)[8]) {
  if constexpr (std::is_same_v<G, LineArgs>) {   // no scale and shift
    const float a = g.alpha ? *g.alpha : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sc[i] = a, sh[i] = 0.f;
    return;
  }
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

  static constexpr __host__ __device__ int key(int line) {
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

// The tile and the split of a workgroup.  Workgroup u runs on XCD u mod 8 and
// takes the (u / 8)-th of that XCD's eighth of the work, which goes through the
// tiles of one split after the other, down kGroup rows of tiles before it goes
// across: what runs together on an XCD shares the lines it reads in its L2.
// (With a split's tiles spread over the XCDs each of them read both operands
// whole: the weight's gradient of 50432 tokens, 768 by 768, took a tenth
// more.)  False past the last.
constexpr int kGroup = 8;
__device__ __forceinline__ bool tile_of(const GemmArgs& g, int& r, int& c, int& split) {
  const int n = g.tr * g.tc, w = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  split = w / n;
  if (split >= g.splits) return false;
  const int u = w - split * n;
  const int band = u / (kGroup * g.tc), r0 = band * kGroup, down = min(kGroup, g.tr - r0), v = u - r0 * g.tc;
  r = r0 + v % down;
  c = v / down;
  return true;
}

// The epilogue of a wave's FR x FC fragments: rows r0.., columns c0...  The
// results pass through BYTES of LDS, the wave's own, so that a row is written
// (and its residual read) as one run of memory, 32 FC bytes of bfloat16; chunk
// c of a row lies at c ^ (row & 7).  A lane takes eight columns c of one row
// in kDown; those that are not all there, or pass from one image to the next,
// go through finish8.
template <typename G, typename T, int BYTES, int FR, int FC, int WR, int WC>
struct FinishOf {
  static constexpr int kPitch = FC * 64, kAcross = 2 * FC, kDown = kWave / kAcross, kAll = FR * 16 / kDown;
  static constexpr int kFrags = BYTES / (16 * kPitch) < FR ? BYTES / (16 * kPitch) : FR;   // of rows at a time
  static constexpr int kIters = kFrags * 16 / kDown, kBatch = kIters < 4 ? kIters : 4;
  static_assert(FR % kFrags == 0 && kIters % kBatch == 0, "whole parts");
  // Small tiles read their residual before the products: its way from memory
  // is as long as theirs (64 to 256 channels at 56 x 56: 94 to 75 us).
  static constexpr bool kAhead = FR * FC * sizeof(T) <= 32;
  typedef T T8 __attribute__((ext_vector_type(8)));

  const G& g;
  int x, down, r0, c;
  bool fit;        // the lane's eight columns lie side by side
  int64_t at;      // of the first within a row
  T8 ahead[kAhead ? kAll : 1];

  __device__ __forceinline__ FinishOf(const G& g, int r0, int c0, int lane)
      : g(g), x(lane % kAcross), down(lane / kAcross), r0(r0), c(c0 + 8 * x) {
    at = c;
    fit = c + 8 <= g.N;
    if (g.hw) {
      const int b = c / g.hw, p = c - b * g.hw;
      at += b * (g.img - g.hw);
      fit = fit && p + 8 <= g.hw;
    }
    if constexpr (kAhead) {
      if (g.res && !g.part && fit) {
#pragma unroll
        for (int i = 0; i < kAll; ++i) ahead[i] = residual(i);
      }
    }
  }
  __device__ __forceinline__ int row(int i) const { return r0 + i * kDown + down; }
  // the residual of iteration i (only where fit)
  __device__ __forceinline__ T8 residual(int i) const {
    T8 v;
    __builtin_memcpy(&v, static_cast<const T*>(g.res) + min(row(i), g.R - 1) * g.ld + at, sizeof(T8));
    return v;
  }
  __device__ __forceinline__ void value(const unsigned char* l, int i, float (&v)[8]) const {
    const int r = i * kDown + down;
    const f32x4 lo = *reinterpret_cast<const f32x4*>(l + r * kPitch + (((2 * x) ^ (r & 7)) << 4));
    const f32x4 hi = *reinterpret_cast<const f32x4*>(l + r * kPitch + (((2 * x + 1) ^ (r & 7)) << 4));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = lo[e];
      v[4 + e] = hi[e];
    }
  }
  // lds(w): the part of wave w
  template <typename L>
  __device__ __forceinline__ void run(f32x4 (&acc)[FR][FC], L&& lds, int wave, int lane, int split) {
    unsigned char* l = lds(wave);
    float sc[8], sh[8];
    column_affine(g, c, sc, sh);
    T *y = static_cast<T*>(g.y), *z = static_cast<T*>(g.z);
    // rows of whole 16 bytes go past the caches (ViT projection 84 to 76 us);
    // rows at 8 bytes do not: their pieces meet in L2 (stage 3: 28 us, not 34)
    const bool stream = g.ld % 8 == 0 && g.hw % 8 == 0;
#pragma unroll
    for (int f = 0; f < FR; f += kFrags) {
      constexpr int kPer = 16 / kDown;   // iterations of a fragment
#pragma unroll
      for (int i = 0; i < kFrags; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) {
          const int r = 16 * i + (lane & 15), ch = 8 * (j / 2) + 2 * (lane >> 4) + (j & 1);
          *reinterpret_cast<f32x4*>(l + r * kPitch + ((ch ^ (r & 7)) << 4)) = acc[f + i][j];
        }
      if (!g.part && fit) {
        // each step over the whole batch: one decision for 8 kBatch values,
        // and as many independent chains
        auto batch = [&](int it) __attribute__((always_inline)) {
          const int i0 = f * kPer + it;
          float v[kBatch][8];
          T8 q[kBatch];
          if (g.res)
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              if constexpr (kAhead)
                q[u] = ahead[i0 + u];
              else
                q[u] = residual(i0 + u);
            }
#pragma unroll
          for (int u = 0; u < kBatch; ++u) value(l, it + u, v[u]);
          if (!g.per_row) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
              for (int e = 0; e < 8; ++e) v[u][e] = fmaf(v[u][e], sc[e], sh[e]);
          } else {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              const int r = min(row(i0 + u), g.R - 1);
              const float a = g.scale ? g.scale[r] : 1.f, b = g.shift ? g.shift[r] : 0.f;
#pragma unroll
              for (int e = 0; e < 8; ++e) v[u][e] = fmaf(v[u][e], a, b);
            }
          }
          if (g.res)
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
              for (int e = 0; e < 8; ++e) v[u][e] += Elem<T>::to_f(q[u][e]);
          auto store = [&](T* to) __attribute__((always_inline)) {
            T* p = to + at + row(i0) * g.ld;
            if (stream) {
#pragma unroll
              for (int u = 0; u < kBatch; ++u)
                if (row(i0 + u) < g.R) stream8(p + u * kDown * g.ld, v[u]);
            } else {
#pragma unroll
              for (int u = 0; u < kBatch; ++u)
                if (row(i0 + u) < g.R) store8(p + u * kDown * g.ld, v[u]);
            }
          };
          if (z) store(z);
          act_values<T>(v, g.act);
          store(y);
        };
        if constexpr (kAhead) {   // the residual's registers by constant places
#pragma unroll
          for (int it = 0; it < kIters; it += kBatch) batch(it);
        } else {
          for (int it = 0; it < kIters; it += kBatch) batch(it);
        }
      }
      if (g.part || !fit) {
        for (int it = 0; it < kIters; ++it) {
          float v[8];
          value(l, it, v);
          row_affine(g, row(f * kPer + it), sc, sh);
          finish8<T>(g, row(f * kPer + it), c, split, v, sc, sh);
        }
      }
    }
  }
};

template <typename T, int BYTES, int FR, int FC, int WR, int WC>
using Finish = FinishOf<GemmArgs, T, BYTES, FR, FC, WR, WC>;
template <typename T, int BYTES, int FR, int FC, int WR, int WC>
using LineFinish = FinishOf<LineArgs, T, BYTES, FR, FC, WR, WC>;

template <int FR, int FC>
__device__ __forceinline__ void clear(f32x4 (&acc)[FR][FC]) {
#pragma unroll
  for (int i = 0; i < FR; ++i)
#pragma unroll
    for (int j = 0; j < FC; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// ---- the product -----------------------------------------------------------------
//
// Operands' lines start on 16 bytes and hold whole chunks (images too; where
// a tensor's do not, it is packed into lines that do first).  A stage goes to
// LDS without passing registers, two stages in LDS: while the matrix cores
// work on the last quarter of stage s, whose operands are in registers by
// then, stage s + 2 is copied over it; its own copies have the time of a
// whole stage to arrive.  One barrier a stage.  The swizzle is in the lane's
// source address.  Chunks past the contraction's end come from a line of
// zeros; rows and columns past the tensor repeat its last ones, and are not
// stored.
__device__ __align__(16) unsigned int zero_chunk[4];

typedef __attribute__((address_space(3))) unsigned char lds_byte;

// the operand of s_waitcnt for at most n memory accesses in flight
constexpr int vm_wait(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }

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
        const int j = min(n0 + c * S::kVec, (n - 1) / S::kVec * S::kVec);   // a packed line's last chunk is whole too
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

// The barrier behind which stages are published: it waits for this wave's own
// LDS accesses and then for every wave, but not for its copies in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// WR x WC waves of FR x FC fragments, D stages in LDS.
//
// Bound by the matrix cores where the contraction is long (16384 positions of
// 4096 by 4096: 429 us, 1281 TFLOP/s, of the 1466 that a large product of the
// library reaches here; the cores are busy 62% of the cycles of a burst, whose
// clock falls to 2 GHz), by memory where it is short (64 to 256 channels over
// 64 images of 56 x 56 with their residual: 50 us, 4.6 TB/s).  Between (50432
// positions of 768 by 768, GELU, z written too: 86 us, for 46 of memory and 41
// of products; cores busy 26%, 125 MB read for 79) the two do not overlap: a
// workgroup's results leave while only its neighbours on the CU multiply.  Tried and slower there: a wave of its
// own that only copies, stages ahead of the product's end (persistent
// workgroups), and prefetches of the stage after next into L2 (86 to 89 us).
//
// F is the epilogue, over arguments G (GemmArgs and what else it needs).
template <typename T, bool AK, bool BK, bool IMG, int WR, int WC, int FR, int FC, int D, typename G = GemmArgs,
          template <typename, int, int, int, int, int> class F = Finish>
__global__ void __launch_bounds__(64 * WR * WC, 2)
k_project(G g) {
  constexpr int NT = 64 * WR * WC, TR = 16 * WR * FR, TC = 16 * WC * FC;
  using SA = Stage<T, AK, TR, false>;
  using SB = Stage<T, BK, TC, true>;
  constexpr int kDepth = SA::kDepth, kA = SA::kBytes, kB = SB::kBytes;
  // arrays of their own, so that the compiler sees the copies and the reads
  // apart and waits for a copy only where its array is read
  __shared__ __attribute__((aligned(16))) unsigned char a0[kA], b0[kB], a1[D > 1 ? kA : 16], b1[D > 1 ? kB : 16],
      a2[D > 2 ? kA : 16], b2[D > 2 ? kB : 16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % WR * 16 * FR, wc = wave / WR * 16 * FC;
  int r0, c0, split;
  if (!tile_of(g, r0, c0, split)) return;
  r0 *= TR, c0 *= TC;
  const int k0 = split * g.klen, length = min(g.K, k0 + g.klen) - k0;
  const int n = (length + kDepth - 1) / kDepth;

  // a wave's part of LDS for its results
  constexpr int kArrays = D == 1 ? 2 : 4, kEach = WR * WC / kArrays, kPart = (kA < kB ? kA : kB) / kEach;
  F<T, kPart, FR, FC, WR, WC> fin(g, r0 + wr, c0 + wc, lane);

  Copier<T, AK, AK && IMG, TR, false, NT> ca;
  Copier<T, BK, BK && IMG, TC, true, NT> cb;
  constexpr int kRounds = ca.kRounds + cb.kRounds;
  ca.init(g.a, r0, g.R, k0, tid);
  if constexpr (std::is_same_v<G, LineArgs>) {
    Operand b = g.b;
    if (g.pick && *g.pick != 0.f) b.p = g.other;
    cb.init(b, c0, g.N, k0, tid);
  } else {
    cb.init(g.b, c0, g.N, k0, tid);
  }
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
  // Copies the next stage to (la, lb); `left` elements of k are there from it on.
  auto copy = [&](auto cut, int left, unsigned char* la, unsigned char* lb) __attribute__((always_inline)) {
    ca.template copy<decltype(cut)::value>(la, tid, wave, left);
    cb.template copy<decltype(cut)::value>(lb, tid, wave, left);
  };
  // Stage s lies in (la, lb), its first phase's operands in registers; copies
  // stage s + D over it and leaves the first operands of the next, in (na, nb).
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
    if constexpr (D > 1) {
      __builtin_amdgcn_s_waitcnt(vm_wait((D - 2) * kRounds));   // the next stage is here
      lds_barrier();
      copy(cut, left, la, lb);
      read(0, na, nb);
    }
    products(3);
    __builtin_amdgcn_sched_barrier(0);
  };
  const std::integral_constant<bool, true> some{};
  const std::integral_constant<bool, false> all{};
  copy(some, length, a0, b0);
  if constexpr (D > 1) copy(some, length - kDepth, a1, b1);
  if constexpr (D > 2) copy(some, length - 2 * kDepth, a2, b2);
  __builtin_amdgcn_s_waitcnt(vm_wait((D - 1) * kRounds));
  lds_barrier();
  read(0, a0, b0);
  int left = length - D * kDepth;   // of the stage to copy next
  if constexpr (D == 1) {
    stage(some, 0, a0, b0, a0, b0);
  } else if constexpr (D == 2) {
    int s = 0;
    for (; left >= D * kDepth; s += D, left -= D * kDepth) {
      stage(all, 0, a0, b0, a1, b1);
      stage(all, 0, a1, b1, a0, b0);
    }
    for (; s + 1 < n; s += D, left -= D * kDepth) {
      stage(some, left, a0, b0, a1, b1);
      stage(some, left - kDepth, a1, b1, a0, b0);
    }
    if (s < n) stage(some, left, a0, b0, a1, b1);
  } else {
    int s = 0;
    for (; left >= D * kDepth; s += D, left -= D * kDepth) {
      stage(all, 0, a0, b0, a1, b1);
      stage(all, 0, a1, b1, a2, b2);
      stage(all, 0, a2, b2, a0, b0);
    }
    for (; s + 2 < n; s += D, left -= D * kDepth) {
      stage(some, left, a0, b0, a1, b1);
      stage(some, left - kDepth, a1, b1, a2, b2);
      stage(some, left - 2 * kDepth, a2, b2, a0, b0);
    }
    if (s < n) stage(some, left, a0, b0, a1, b1);
    if (s + 1 < n) stage(some, left - kDepth, a1, b1, a2, b2);
  }
  // the stages' LDS is taken for the results: no wave reads, nothing is copied any more
  __builtin_amdgcn_s_waitcnt(vm_wait(0));
  __syncthreads();
  auto part = [&](int u) __attribute__((always_inline)) {
    const int w = u / kEach;
    return (w == 0 ? a0 : w == 1 ? b0 : w == 2 ? a1 : b1) + u % kEach * kPart;
  };
  fin.run(acc, part, wave, lane, split);
}

// ---- launches --------------------------------------------------------------------

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The tiles there are: tr x tc, stages in LDS, workgroups a CU, and the
// microseconds of a bfloat16 stage on a CU that is full (a workgroup's share)
// and on one of its own.  These times and those of plan() are fitted to
// measured cuts (forward, dx and dW from one position to 360000, 32 to 4096
// channels).  Of 225 products in both types, 5657 cuts measured again, the cut
// they pick is 1.6% slower than the best one on average, 22% at worst, and more
// than 5% for 20 of them.
struct Tile {
  int tr, tc, stages, per_cu;
  double busy, alone;
};
enum { kT256, kT128, kT128x64, kT64x128, kT128x64Deep, kT64x128Deep, kT64, kT128x64Once, kT64x128Once, kTiles };
constexpr Tile kTile[kTiles] = {
    {256, 256, 2, 1, 1.81, 1.45},  // the most products for an LDS read: 1350 TFLOP/s where it fills the GPU
    {128, 128, 2, 2, 0.48, 0.70},  // 1130
    {128, 64, 2, 3, 0.30, 0.69},   // 890; three workgroups a CU hide each other's ends
    {64, 128, 2, 3, 0.30, 0.69},
    {128, 64, 3, 2, 0.36, 0.34},   // few tiles, long contractions: 1024 x 2048 over 2048 in 15 us, not 20
    {64, 128, 3, 2, 0.36, 0.34},
    {64, 64, 3, 3, 0.20, 0.24},    // few outputs
    {128, 64, 1, 4, 0.30, 0.86},   // contractions of one stage: 56 x 56 x 64, 64 to 256 channels, 54 us, not 66
    {64, 128, 1, 4, 0.30, 0.86},
};
// Parts of the contraction: above eight in multiples of the dies.
constexpr int kSplits[] = {1, 2, 3, 4, 6, 8, 16, 24, 32, 48, 64, 96, 128, 192, 256};

// How a product is cut: its tile and, where the tiles are too few for the GPU,
// the contraction in `splits` lengths whose sums are joined by another kernel.
struct Plan {
  int tile, splits, klen;
  double time;   // microseconds, by the model
};
// ragged: the output's rows are not whole chunks; turned: both operands lie
// across the contraction (more LDS reads); most: splits.
inline Plan plan(int64_t R, int64_t N, int64_t K, int elem, bool ragged, bool turned, int most = INT_MAX) {
  constexpr int kCUs = 256;
  const int depth = kLine / (elem == MOCE_F32 ? 4 : 2), stages = (int)ceil_div(K, depth);
  // The time of a cut: rounds of workgroups over the CUs, each as long as its
  // stages and its ends (the way of the first operands and of the results,
  // 12.9 KB a microsecond and CU); then the join.
  Plan best{};
  double least = 1e300;
  for (int t = 0; t < kTiles; ++t) {
    const Tile& c = kTile[t];
    if (c.stages == 1 ? stages != 1 : elem == MOCE_F32 && (t == kT256 || c.stages == 3) && t != kT64) continue;
    const int64_t tiles = ceil_div(R, c.tr) * ceil_div(N, c.tc), slots = (int64_t)kCUs * c.per_cu;
    // float32: bound by its matrix instructions
    const double busy = elem == MOCE_F32 ? 0.68 / 4096 * c.tr * c.tc : turned ? 1.16 * c.busy : c.busy;
    const double alone = std::max(c.alone, elem == MOCE_F32 ? 1.03 * busy : busy);
    for (const int s : kSplits) {
      if (s > most) break;
      if (s > 1 && (stages / s < 2 || tiles * (s - 1) >= 2 * slots)) break;
      const int64_t each = ceil_div(stages, s), splits = ceil_div(stages, each);
      const int64_t rounds = tiles * splits / slots, k = ceil_div(tiles * splits % slots, kCUs);
      // rows in pieces; short runs of memory
      const double pieces = splits > 1 ? 1. : ragged ? 2.65 : c.tc == 64 ? 1.05 : 1.;
      const double end = c.tr * c.tc * (splits > 1 || elem == MOCE_F32 ? 4 : 2) * pieces / 12900., begin = 4.7 / c.per_cu;
      double time = rounds * (each * c.per_cu * busy + begin + end * c.per_cu);
      if (k > 0) time += each * std::max(alone, k * busy) + begin + end * k;
      if (splits > 1) {
        if (splits % 8) time *= 1.125;   // splits that lie on two dies are read by both
        time += 6.8 + (double)splits * R * N * 4 / 2.9e6;
      }
      if (time < least) {
        least = time;
        best = Plan{t, (int)splits, (int)(each * depth), time};
      }
    }
  }
  return best;
}
inline size_t part_bytes(int64_t R, int64_t N, const Plan& p) { return (size_t)p.splits * R * N * sizeof(float); }

template <typename T, bool AK, bool BK, bool IMG, int WR, int WC, int FR, int FC, int D,
          template <typename, int, int, int, int, int> class F, typename G>
void launch_tiles(G g, int splits, hipStream_t st) {
  g.tr = (int)ceil_div(g.R, 16 * WR * FR), g.tc = (int)ceil_div(g.N, 16 * WC * FC);
  g.splits = splits;
  const dim3 grid((unsigned)(ceil_div((int64_t)g.tr * g.tc * splits, 8) * 8));
  hipLaunchKernelGGL((k_project<T, AK, BK, IMG, WR, WC, FR, FC, D, G, F>), grid, dim3(64 * WR * WC), 0, st, g);
}

template <typename T, bool AK, bool BK, template <typename, int, int, int, int, int> class F = Finish,
          typename G = GemmArgs>
hipError_t launch_product(const G& g, const Plan& p, hipStream_t st) {
  auto copy = [&](auto img) {
    constexpr bool IMG = decltype(img)::value;
    constexpr bool low = sizeof(T) == 2;
    switch (p.tile) {
      case kT256: if constexpr (low) launch_tiles<T, AK, BK, IMG, 2, 4, 8, 4, 2, F>(g, p.splits, st); break;
      case kT128: launch_tiles<T, AK, BK, IMG, 2, 2, 4, 4, 2, F>(g, p.splits, st); break;
      case kT128x64: launch_tiles<T, AK, BK, IMG, 2, 2, 4, 2, 2, F>(g, p.splits, st); break;
      case kT64x128: launch_tiles<T, AK, BK, IMG, 2, 2, 2, 4, 2, F>(g, p.splits, st); break;
      case kT128x64Deep: if constexpr (low) launch_tiles<T, AK, BK, IMG, 2, 2, 4, 2, 3, F>(g, p.splits, st); break;
      case kT64x128Deep: if constexpr (low) launch_tiles<T, AK, BK, IMG, 2, 2, 2, 4, 3, F>(g, p.splits, st); break;
      case kT64: launch_tiles<T, AK, BK, IMG, 2, 2, 2, 2, 3, F>(g, p.splits, st); break;
      case kT128x64Once: launch_tiles<T, AK, BK, IMG, 2, 2, 4, 2, 1, F>(g, p.splits, st); break;
      case kT64x128Once: launch_tiles<T, AK, BK, IMG, 2, 2, 2, 4, 1, F>(g, p.splits, st); break;
    }
  };
  if constexpr (AK && BK && std::is_same_v<G, GemmArgs>) {
    if (g.a.hw)
      copy(std::true_type{});
    else
      copy(std::false_type{});
  } else {
    copy(std::false_type{});
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace moce
