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
template <typename T, int BYTES, int FR, int FC>
struct Finish {
  static constexpr int kPitch = FC * 64, kAcross = 2 * FC, kDown = kWave / kAcross, kAll = FR * 16 / kDown;
  static constexpr int kFrags = BYTES / (16 * kPitch) < FR ? BYTES / (16 * kPitch) : FR;   // of rows at a time
  static constexpr int kIters = kFrags * 16 / kDown, kBatch = kIters < 4 ? kIters : 4;
  static_assert(FR % kFrags == 0 && kIters % kBatch == 0, "whole parts");
  // Small tiles read their residual before the products: its way from memory
  // is as long as theirs (64 to 256 channels at 56 x 56: 94 to 75 us).
  static constexpr bool kAhead = FR * FC * sizeof(T) <= 32;
  typedef T T8 __attribute__((ext_vector_type(8)));

  const GemmArgs& g;
  int x, down, r0, c;
  bool fit;        // the lane's eight columns lie side by side
  int64_t at;      // of the first within a row
  T8 ahead[kAhead ? kAll : 1];

  __device__ __forceinline__ Finish(const GemmArgs& g, int r0, int c0, int lane)
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
  __device__ __forceinline__ void run(f32x4 (&acc)[FR][FC], unsigned char* l, int lane, int split) {
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
template <typename T, bool AK, bool BK, bool IMG, int WR, int WC, int FR, int FC, int D>
__global__ void __launch_bounds__(64 * WR * WC, 2)
k_project(GemmArgs g) {
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
  Finish<T, kPart, FR, FC> fin(g, r0 + wr, c0 + wc, lane);

  Copier<T, AK, AK && IMG, TR, false, NT> ca;
  Copier<T, BK, BK && IMG, TC, true, NT> cb;
  constexpr int kRounds = ca.kRounds + cb.kRounds;
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
  const int w = wave / kEach;
  fin.run(acc, (w == 0 ? a0 : w == 1 ? b0 : w == 2 ? a1 : b1) + wave % kEach * kPart, lane, split);
}

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
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_join(GemmArgs g, int splits, int down) {
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
  GemmArgs h = g;
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

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

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
};
// ragged: the output's rows are not whole chunks; turned: both operands lie
// across the contraction (more LDS reads).
Plan plan(int64_t R, int64_t N, int64_t K, int elem, bool ragged, bool turned) {
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
        best = Plan{t, (int)splits, (int)(each * depth)};
      }
    }
  }
  return best;
}
size_t part_bytes(int64_t R, int64_t N, const Plan& p) { return (size_t)p.splits * R * N * sizeof(float); }

template <typename T, bool AK, bool BK, bool IMG, int WR, int WC, int FR, int FC, int D>
void launch_tiles(GemmArgs g, int splits, hipStream_t st) {
  g.tr = (int)ceil_div(g.R, 16 * WR * FR), g.tc = (int)ceil_div(g.N, 16 * WC * FC);
  g.splits = splits;
  const dim3 grid((unsigned)(ceil_div((int64_t)g.tr * g.tc * splits, 8) * 8));
  hipLaunchKernelGGL((k_project<T, AK, BK, IMG, WR, WC, FR, FC, D>), grid, dim3(64 * WR * WC), 0, st, g);
}

template <typename T, bool AK, bool BK>
hipError_t launch_product(const GemmArgs& g, const Plan& p, hipStream_t st) {
  auto copy = [&](auto img) {
    constexpr bool IMG = decltype(img)::value;
    constexpr bool low = sizeof(T) == 2;
    switch (p.tile) {
      case kT256: if constexpr (low) launch_tiles<T, AK, BK, IMG, 2, 4, 8, 4, 2>(g, p.splits, st); break;
      case kT128: launch_tiles<T, AK, BK, IMG, 2, 2, 4, 4, 2>(g, p.splits, st); break;
      case kT128x64: launch_tiles<T, AK, BK, IMG, 2, 2, 4, 2, 2>(g, p.splits, st); break;
      case kT64x128: launch_tiles<T, AK, BK, IMG, 2, 2, 2, 4, 2>(g, p.splits, st); break;
      case kT128x64Deep: if constexpr (low) launch_tiles<T, AK, BK, IMG, 2, 2, 4, 2, 3>(g, p.splits, st); break;
      case kT64x128Deep: if constexpr (low) launch_tiles<T, AK, BK, IMG, 2, 2, 2, 4, 3>(g, p.splits, st); break;
      case kT64: launch_tiles<T, AK, BK, IMG, 2, 2, 2, 2, 3>(g, p.splits, st); break;
      case kT128x64Once: launch_tiles<T, AK, BK, IMG, 2, 2, 4, 2, 1>(g, p.splits, st); break;
      case kT64x128Once: launch_tiles<T, AK, BK, IMG, 2, 2, 2, 4, 1>(g, p.splits, st); break;
    }
  };
  if constexpr (AK && BK) {
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
  const int down = splits >= kJoinMany ? 8 : 1;
  hipLaunchKernelGGL(k_project_join<T>, dim3((unsigned)ceil_div((int64_t)g.R * ceil_div(g.N, 8), kThreads / down)),
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

}  // namespace

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
