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
#include <cstdio>
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

// The passes over dy (and z) before the products; packing x or the weight is
// the same pass without an activation.
struct DzArgs {
  const void *z, *dy;
  void* dz;               // act'(z) dy where dy's element is (nullptr: not written)
  void* pack;             // the same, times scale where given, in lines of ld elements (nullptr: none)
  const float* scale;     // by channel
  float* part;            // [groups][O] partial sums of dz over positions (nullptr: none)
  int act, O, hw, ld;     // O channels; hw positions of a plane (channels-first)
  int64_t n;              // rows of positions (channels-last), images or planes (channels-first)
  int64_t per;            // rows of one group
};

// act'(z) dy of eight neighbouring elements (n of them there) at e, stored to dz
template <typename T>
__device__ __forceinline__ void dz8(const DzArgs& a, int64_t e, int n, float (&v)[8]) {
  using E = Elem<T>;
  const T *z = static_cast<const T*>(a.z), *dy = static_cast<const T*>(a.dy);
  T* dz = static_cast<T*>(a.dz);
  if (n == 8) {
    load8(dy + e, v);
    if (a.act != MOCE_ACT_NONE) {
      float q[8];
      load8(z + e, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = act_gradient<T>(q[i], v[i], a.act);
    }
    if (dz) store8(dz + e, v);
    return;
  }
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
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_dz_rows(DzArgs a, int tx) {
  __shared__ float s[kThreads][8 + 1];
  const int x = threadIdx.x % tx, down = kThreads / tx;
  const int c = (blockIdx.y * tx + x) * 8, n = min(8, a.O - c);
  float sum[8] = {}, sc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) sc[i] = a.pack && a.scale ? a.scale[min(c + i, a.O - 1)] : 1.f;
  if (n > 0) {
    const int64_t end = min(a.n, (blockIdx.x + (int64_t)1) * a.per);
    for (int64_t r = blockIdx.x * a.per + threadIdx.x / tx; r < end; r += down) {
      float v[8];
      dz8<T>(a, r * a.O + c, n, v);
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
// 64) take a plane; pack: planes as dy's.
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
      dz8<T>(a, e, n, v);
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

// Channels-first to lines of channels: a workgroup turns 64 channels by 64
// positions of an image through LDS, a wave 16 channels, a lane a position;
// pack: [position][ld], zeros behind O.  part: a group per 64 positions.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_turn(DzArgs a, int across) {
  using E = Elem<T>;
  constexpr int kPitch = 64 + 4 / (int)sizeof(T) * 1;   // odd words: lanes down a column on different banks
  __shared__ T s[64 * kPitch];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t u = blockIdx.x;                         // image and run of positions
  const int64_t b = u / across;
  const int p = (int)(u % across) * 64 + lane, c0 = blockIdx.y * 64;
  const T *z = static_cast<const T*>(a.z), *dy = static_cast<const T*>(a.dy);
  T* dz = static_cast<T*>(a.dz);
  float v[16], q[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int c = c0 + 16 * wave + i;
    const int64_t e = (b * a.O + min(c, a.O - 1)) * a.hw + min(p, a.hw - 1);
    v[i] = E::to_f(dy[e]);
    q[i] = a.act != MOCE_ACT_NONE ? E::to_f(z[e]) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int c = c0 + 16 * wave + i;
    const bool there = c < a.O && p < a.hw;
    v[i] = there ? act_gradient<T>(q[i], v[i], a.act) : 0.f;
    if (dz && there) dz[(b * a.O + c) * a.hw + p] = E::from_f(v[i]);
    if (a.part) {
      const float t = wave_sum(v[i]);
      if (lane == 0 && c < a.O) a.part[u * a.O + c] = t;
    }
    if (a.pack) s[lane * kPitch + 16 * wave + i] = E::from_f(a.scale ? v[i] * a.scale[min(c, a.O - 1)] : v[i]);
  }
  if (!a.pack) return;
  __syncthreads();
  // a thread writes 16 bytes of a position's line at a time
  constexpr int kVec = E::kVec, kLanes = 64 / kVec;
#pragma unroll
  for (int i = threadIdx.x; i < 64 * kLanes; i += kThreads) {
    const int row = i / kLanes, c = i % kLanes * kVec, at = (int)(u % across) * 64 + row;
    if (at >= a.hw || c0 + c >= a.ld) continue;
    T w[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) w[j] = s[row * kPitch + c + j];
    __builtin_memcpy(static_cast<T*>(a.pack) + (b * a.hw + at) * a.ld + c0 + c, w, 16);
  }
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

// scale[o] weight[o][c] (scale may be nullptr), rounded to the weight's type, in lines of ld, zeros behind C
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_project_weight(const T* __restrict__ weight, const float* __restrict__ scale, int C, int ld, T* __restrict__ out) {
  const int o = blockIdx.x;
  const float s = scale ? scale[o] : 1.f;
  for (int c = threadIdx.x; c < ld; c += kThreads)
    out[(int64_t)o * ld + c] = c < C ? Elem<T>::from_f(s * Elem<T>::to_f(weight[(int64_t)o * C + c])) : (T)0;
}

// ---- launches --------------------------------------------------------------------

constexpr int kWantTiles = 512;          // two workgroups a CU

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a product is cut: tiles of tr rows and tc columns and, where these
// make too few workgroups for the GPU, the contraction in lengths of 256 or more.
struct Plan {
  int tr, tc, splits, klen;
};
Plan split_plan(int tr, int tc, int64_t s, int64_t K, int elem) {
  const int depth = kLine / (elem == MOCE_F32 ? 4 : 2);
  s = std::min<int64_t>(std::max<int64_t>(s, 1), 256);
  const int64_t klen = ceil_div(ceil_div(K, s), depth) * depth;
  return Plan{tr, tc, (int)ceil_div(K, klen), (int)klen};
}
Plan sweep_plan(int64_t R, int64_t N, int64_t K, int elem, const char* e) {
  int tr = 64, tc = 64, s = 0;
  sscanf(e, "%dx%d/%d", &tr, &tc, &s);
  if (s == 0) s = (int)std::min(std::max<int64_t>(1, kWantTiles / (ceil_div(R, tr) * ceil_div(N, tc))), std::max<int64_t>(1, K / 256));
  return split_plan(tr, tc, s, K, elem);
}
Plan plan(int64_t R, int64_t N, int64_t K, int elem) {
  // sweep
  int tile = 64;
  if (ceil_div(R, 128) * ceil_div(N, 128) >= 256) tile = 128;
  if (elem == MOCE_BF16 && ceil_div(R, 256) * ceil_div(N, 256) >= 256) tile = 256;
  const int64_t tiles = ceil_div(R, tile) * ceil_div(N, tile);
  return split_plan(tile, tile, std::min(std::max<int64_t>(1, kWantTiles / tiles), std::max<int64_t>(1, K / 256)), K, elem);
}
size_t part_bytes(int64_t R, int64_t N, const Plan& p) { return (size_t)p.splits * R * N * sizeof(float); }

template <typename T, bool AK, bool BK, bool IMG, int WR, int WC, int F, int FC>
void launch_copy(GemmArgs g, int splits, hipStream_t st) {
  g.tr = (int)ceil_div(g.R, 16 * WR * F), g.tc = (int)ceil_div(g.N, 16 * WC * FC);
  const dim3 grid((unsigned)(ceil_div((int64_t)g.tr * g.tc, 8) * 8), splits);
  hipLaunchKernelGGL((k_project_copy<T, AK, BK, IMG, WR, WC, F, FC>), grid, dim3(64 * WR * WC), 0, st, g);
}

template <typename T, bool AK, bool BK>
hipError_t launch_product(const GemmArgs& g, const Plan& p, hipStream_t st) {
  auto copy = [&](auto img) {
    constexpr bool IMG = decltype(img)::value;
    const int t = p.tr * 1000 + p.tc;
    if (t == 64064) launch_copy<T, AK, BK, IMG, 2, 2, 2, 2>(g, p.splits, st);
    else if (t == 128128 || sizeof(T) == 4) launch_copy<T, AK, BK, IMG, 2, 2, 4, 4>(g, p.splits, st);
    else if constexpr (sizeof(T) == 2) {
      if (t == 256256) launch_copy<T, AK, BK, IMG, 2, 4, 8, 4>(g, p.splits, st);
      if (t == 128064) launch_copy<T, AK, BK, IMG, 2, 2, 4, 2>(g, p.splits, st);
      if (t == 64128) launch_copy<T, AK, BK, IMG, 2, 2, 2, 4>(g, p.splits, st);
      if (t == 256128) launch_copy<T, AK, BK, IMG, 4, 2, 4, 4>(g, p.splits, st);
      if (t == 128256) launch_copy<T, AK, BK, IMG, 2, 4, 4, 4>(g, p.splits, st);
      if (t == 256064) launch_copy<T, AK, BK, IMG, 4, 1, 4, 4>(g, p.splits, st);
      if (t == 64256) launch_copy<T, AK, BK, IMG, 1, 4, 4, 4>(g, p.splits, st);
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

// ---- which operands are packed ---------------------------------------------------

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

template <typename T>
hipError_t pack_rows(const void* src, int64_t rows, int64_t channels, void* out, int64_t ld, hipStream_t st) {
  DzArgs a{};
  a.dy = src, a.pack = out, a.O = (int)channels, a.ld = (int)ld, a.n = rows;
  int tx = 1;
  while (tx < 32 && tx * 8 < channels) tx *= 2;
  a.per = ceil_div(ceil_div(rows, 2048), kThreads / tx) * (kThreads / tx);
  hipLaunchKernelGGL(k_project_dz_rows<T>, dim3((unsigned)ceil_div(rows, a.per), (unsigned)ceil_div(channels, tx * 8)),
                     dim3(kThreads), 0, st, a, tx);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_turn(const DzArgs& a, hipStream_t st) {
  const int across = (int)ceil_div(a.hw, 64);
  return image_slices(a.n, (int64_t)across * kThreads, 1, [&](int64_t b, int64_t n) {
    DzArgs p = a;
    const int64_t at = b * a.O * a.hw;
    auto on = [&](const void* q) { return const_cast<T*>(static_cast<const T*>(q) + at); };
    p.dy = on(a.dy);
    if (a.z) p.z = on(a.z);
    if (a.dz) p.dz = on(a.dz);
    if (a.pack) p.pack = static_cast<T*>(a.pack) + b * a.hw * a.ld;
    if (a.part) p.part = a.part + b * across * a.O;
    hipLaunchKernelGGL(k_project_turn<T>, dim3((unsigned)(n * across), (unsigned)ceil_div(a.O, 64)), dim3(kThreads), 0,
                       st, p, across);
    return hipGetLastError();
  });
}
// Images of channels planes of hw positions into lines of channels, times scale (may be nullptr).
template <typename T>
hipError_t turn(const void* src, int64_t images, int64_t channels, int64_t hw, const float* scale, void* out,
                int64_t ld, hipStream_t st) {
  DzArgs a{};
  a.dy = src, a.pack = out, a.scale = scale, a.O = (int)channels, a.hw = (int)hw, a.ld = (int)ld, a.n = images;
  return launch_turn<T>(a, st);
}
// x (or dy) as the products read it: packed into `out` where its lines are ragged.
template <typename T>
hipError_t pack_tensor(const Sizes& z, const void** t, int64_t channels, void* out, hipStream_t st) {
  if (!z.rows(channels)) return hipSuccess;
  const void* src = *t;
  *t = out;
  return z.nhwc ? pack_rows<T>(src, z.P(), channels, out, z.up(channels), st)
                : turn<T>(src, z.s.B, channels, z.s.HW, nullptr, out, z.up(channels), st);
}
template <typename T>
hipError_t pack_weight(const Sizes& z, const void** w, const float* scale, void* out, hipStream_t st) {
  if (!z.weight() && !scale) return hipSuccess;
  hipLaunchKernelGGL(k_project_weight<T>, dim3((unsigned)z.s.O), dim3(kThreads), 0, st, static_cast<const T*>(*w), scale,
                     (int)z.s.C, (int)z.up(z.s.C), static_cast<T*>(out));
  *w = out;
  return hipGetLastError();
}

// Rows and columns of the output, of `channels` channels, as the products write it
void output(GemmArgs* g, const Sizes& z, int64_t channels) {
  const int64_t P = z.P();
  g->R = (int)(z.nhwc ? P : channels), g->N = (int)(z.nhwc ? channels : P);
  g->ld = z.nhwc ? channels : z.s.HW, g->hw = z.images(), g->img = channels * z.s.HW;
}

struct FwdLayout {
  Plan p;
  size_t x, weight, part, total;
};
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
FwdLayout fwd_layout(const ProjectShape& s) {
  const Sizes z(s);
  FwdLayout l{};
  GemmArgs g{};
  output(&g, z, s.O);
  l.p = plan(g.R, g.N, s.C, s.elem);
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
  hipError_t e = pack_tensor<T>(z, &x, s.C, ws + l.x, st);
  if (e == hipSuccess) e = pack_weight<T>(z, &w, nullptr, ws + l.weight, st);
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

// Groups of positions whose sums of dz lie apart: rows (channels-last) in up
// to 1024 workgroups, images or 64 positions of them (channels-first).
struct DzPlan {
  int tx;
  int64_t per, groups;
};
DzPlan dz_plan(const Sizes& z) {
  const ProjectShape& s = z.s;
  if (!z.nhwc) return DzPlan{0, 0, z.planes() ? s.B * ceil_div(s.HW, 64) : s.B};
  int tx = 1;
  while (tx < 32 && tx * 8 < s.O) tx *= 2;
  const int64_t M = z.P(), across = ceil_div(s.O, tx * 8), down = kThreads / tx;
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
  l.px = plan(g.R, g.N, s.O, s.elem);
  l.pw = plan(s.O, s.C, z.P(), s.elem);
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += up256(n);
    return here;
  };
  l.dz = take(s.act != MOCE_ACT_NONE || z.rows(s.O) ? z.packed(s.O) : 0);
  l.x = take(z.rows(s.C) ? z.packed(s.C) : 0);
  l.weight = take((size_t)std::max(s.O * z.up(s.C), z.up(s.O) * s.C) * z.el());
  l.shift = take((size_t)dz_plan(z).groups * s.O * sizeof(float));
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
  // the rows of dW.
  const bool fold = scale && smooth;
  const float* row_scale = fold ? nullptr : scale;
  const bool products = gr.dx || gr.dweight || gr.dscale;
  const bool ragged = z.rows(s.O);
  const void* dz = dy;
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
    a.part = gr.dshift ? reinterpret_cast<float*>(ws + l.shift) : nullptr;
    const DzPlan dp = dz_plan(z);
    if (a.dz || a.pack || a.part) {
      if (z.nhwc) {
        a.n = z.P(), a.per = dp.per;
        hipLaunchKernelGGL(k_project_dz_rows<T>, dim3((unsigned)dp.groups, (unsigned)ceil_div(s.O, dp.tx * 8)),
                           dim3(kThreads), 0, st, a, dp.tx);
        e = hipGetLastError();
      } else if (turned) {
        a.n = s.B;
        e = launch_turn<T>(a, st);
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
    if (gr.dshift) {
      hipLaunchKernelGGL(k_project_dshift, dim3((unsigned)ceil_div(s.O, 64)), dim3(1024), 0, st, a.part, dp.groups,
                         (int)s.O, gr.dshift);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  float* part = reinterpret_cast<float*>(ws + l.part);
  const Operand dzo{dz, z.up(s.O), 0, 0}, dzp{dz, s.HW, s.O * s.HW, z.images()};   // lines of channels, of positions
  if (gr.dx) {
    GemmArgs g{};
    output(&g, z, s.C);
    g.K = (int)s.O, g.y = gr.dx;
    if (turned) {
      // the weight turned too, so that both operands run along the outputs
      e = turn<T>(w, 1, s.O, s.C, row_scale, ws + l.weight, z.up(s.O), st);
      if (e != hipSuccess) return e;
      g.a = Operand{ws + l.weight, z.up(s.O), 0, 0}, g.b = dzo;
      e = launch_whole<T, true, true>(g, l.px, part, st);
    } else {
      const void* wp = w;
      e = pack_weight<T>(z, &wp, row_scale, ws + l.weight, st);
      if (e != hipSuccess) return e;
      const Operand wo{wp, z.up(s.C), 0, 0};
      if (z.nhwc) {
        g.a = dzo, g.b = wo;
        e = launch_whole<T, true, false>(g, l.px, part, st);
      } else {
        g.a = wo, g.b = dzp;
        e = launch_whole<T, false, false>(g, l.px, part, st);
      }
    }
    if (e != hipSuccess) return e;
  }
  if (gr.dweight || gr.dscale) {
    e = pack_tensor<T>(z, &x, s.C, ws + l.x, st);
    if (e != hipSuccess) return e;
    GemmArgs g{};
    g.R = (int)s.O, g.N = (int)s.C, g.K = (int)z.P(), g.ld = s.C, g.y = gr.dweight, g.klen = l.pw.klen;
    const bool join = row_scale || l.pw.splits > 1;
    if (join) g.part = part;
    if (z.nhwc || turned) {
      g.a = dzo, g.b = Operand{x, z.up(s.C), 0, 0};
      e = launch_product<T, false, false>(g, l.pw, st);
    } else {
      g.a = dzp, g.b = Operand{x, s.HW, s.C * s.HW, z.images()};
      e = launch_product<T, true, true>(g, l.pw, st);
    }
    if (e != hipSuccess) return e;
    if (join) {
      hipLaunchKernelGGL(k_project_dweight<T>, dim3((unsigned)s.O), dim3(kThreads), 0, st, part, l.pw.splits, (int)s.O,
                         (int)s.C, row_scale, static_cast<const T*>(w), static_cast<T*>(gr.dweight), gr.dscale);
      e = hipGetLastError();
    }
  }
  return e;
}

}  // namespace

size_t project_backward_ws_bytes(const ProjectShape& s) { return bwd_layout(s).total; }

hipError_t launch_project_backward(const ProjectShape& s, const void* x, const void* w, const float* scale,
                                   const void* z, const void* dy, const moce_project_grads& gr, void* ws,
                                   hipStream_t st) {
  char* base = static_cast<char*>(ws);
  return s.elem == MOCE_F32 ? backward<float>(s, x, w, scale, z, dy, gr, base, st)
                            : backward<uint16_t>(s, x, w, scale, z, dy, gr, base, st);
}

}  // namespace moce
