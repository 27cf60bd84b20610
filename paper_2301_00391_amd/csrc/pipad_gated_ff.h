// The gated feed-forward block on node rows, and its gradients (pipad_gated_ff, pipad_gated_ff_backward in include/pipad.h).
//
//   G = X Wg + bg,  U = X Wu + bu,  H = act(G) * U,  Y = H Wd + bd
//
// G, U and H are several times as wide as the rows and are never written: a wave keeps 32 node rows, walks the hidden columns 32 at
// a time, and its share of H goes from the registers where the matrix instructions left it straight into the next product.  The
// backward pass makes G and U again, which is two products out of eleven, where keeping them would be 8 bytes a hidden column and row.
//
// Products of 32-bit floats from matrix instructions on bf16: x = x1 + x2 + x3, each piece the nearest with 8 bits to what is left, so
// that the sum has all 24 bits of x.  Of the nine products of pieces the three smallest are left out: x2 y3 and x3 y2 are below 2^-8 2^-17 of
// the whole each, with either sign.  Six instructions of 32 cycles for 32 x 32 x 16 are 2.7 times as fast as the matrix instructions on floats.
// A value that is not finite (or above 3.389e38, which rounds to none that is) has no such pieces: its row's results are NaN where floats would
// give an infinity.
//
// The sums are 32-bit floats.  An instruction aligns what it adds to the largest of it and cuts off, so a sum comes out low by some 8e-9
// of its terms' size; over millions of rows that would be seen, and the weights' gradients are taken with every other tile of rows negated,
// where it comes out high.  Over 1024 terms of one sign accumulated by the instructions alone it was 4e-7; the gradients' sums are therefore made
// of sums of 32 rows by additions that round to the nearest.
//
// How a 32 x 32 x 16 instruction lies in a wave, m = lane % 32, g = lane / 32: the left operand's lane holds row m, the right one's
// column m, both the depth 8 g .. 8 g + 7; register r of the result is row 8 (r / 4) + 4 g + r % 4, column m.  So the registers
// 8 s .. 8 s + 7 of a result are, without moving between lanes, an operand of the next product whose depth runs over
// 16 s + 8 (j / 4) + 4 g + j % 4, j = 0 .. 7: the other operand is laid out in the same order ("depth of a result" below).
#ifndef PIPAD_GATED_FF_H_
#define PIPAD_GATED_FF_H_

#include "pipad_internal.h"

namespace pipad {
namespace ff {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32, kDepth = 16;
constexpr int kFragment = 3 * kWave;  // the three pieces of a 32 x 16 operand, in 16-byte words
__host__ __device__ constexpr int gu_words(int fq) { return fq * 2 * kFragment + kWave; }  // of a hidden tile

__host__ __device__ constexpr int64_t tiles(int64_t x, int64_t t) { return (x + t - 1) / t; }

__device__ inline int result_depth(int s, int g, int j) { return 16 * s + 8 * (j / 4) + 4 * g + j % 4; }

struct Split {
  u32x4 p[3];
};
__device__ inline Split split8(const float (&v)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  Split s;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      const uint32_t ab = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
      s.p[q][i] = ab;
      a -= __uint_as_float(ab << 16);
      b -= __uint_as_float(ab & 0xffff0000u);
    }
  }
  return s;
}

__device__ inline Split split8(float (&v)[8], float sign) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= sign;
  return split8(v);
}

__device__ inline f32x16 mfma(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// c + a b, the small products first.
__device__ inline f32x16 product(const Split &a, const Split &b, f32x16 c) {
  c = mfma(a.p[2], b.p[0], c);
  c = mfma(a.p[0], b.p[2], c);
  c = mfma(a.p[1], b.p[1], c);
  c = mfma(a.p[1], b.p[0], c);
  c = mfma(a.p[0], b.p[1], c);
  return mfma(a.p[0], b.p[0], c);
}
__device__ inline Split fragment(const u32x4 *at, int64_t index) {
  at += index * kFragment + (threadIdx.x & (kWave - 1));
  return Split{{at[0], at[kWave], at[2 * kWave]}};
}

// ---- the activations ----------------------------------------------------------------------------
struct Sigmoid {
  float s, rest;  // sigmoid and 1 - sigmoid, each to its own last bits
};
__device__ inline Sigmoid sigmoid2(float x) {
  const float e = __expf(-fabsf(x)), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
  return x >= 0.f ? Sigmoid{big, small} : Sigmoid{small, big};
}
// The normal distribution's Phi(x), and its density times sqrt(2 pi).  The tail Q(t) = 1 - Phi(t), t >= 0, is exp(-t^2 / 2) times a function
// that falls like 1 / t: a polynomial in k = 1 / (1 + 0.3 t) without a constant term, fitted for the least relative error (1.5e-7 over t <= 14,
// 4.3e-7 with the arithmetic's own), so that both tails keep their last bits, where 1 + erf loses the lower one.
struct Normal {
  float cdf, density;
};
__device__ inline Normal normal_of(float x) {
  const float t = fabsf(x), k = __builtin_amdgcn_rcpf(fmaf(0.3f, t, 1.f)), e = __expf(-0.5f * x * x);
  float q = 0.03567368909716606f;
  q = fmaf(q, k, -0.15719902515411377f);
  q = fmaf(q, k, 0.2063472718000412f);
  q = fmaf(q, k, -0.05367852374911308f);
  q = fmaf(q, k, 0.12855921685695648f);
  q = fmaf(q, k, 0.09991414099931717f);
  q = fmaf(q, k, 0.12075386196374893f);
  q = fmaf(q, k, 0.11962930113077164f);
  q *= k * e;
  return {x < 0.f ? q : 1.f - q, e};
}

template <int ACT>
__device__ inline float activate(float x) {
  if (ACT == PIPAD_ACT_RELU) return x < 0.f ? 0.f : x;  // (NaN stays)
  if (ACT == PIPAD_ACT_GELU) return x * normal_of(x).cdf;
  const float s = __builtin_amdgcn_rcpf(1.f + __expf(-x));
  return ACT == PIPAD_ACT_SIGMOID ? s : x * s;
}
// act(x) and its slope
template <int ACT>
__device__ inline float2 activate_slope(float x) {
  if (ACT == PIPAD_ACT_RELU) return make_float2(x < 0.f ? 0.f : x, x > 0.f ? 1.f : 0.f);
  if (ACT == PIPAD_ACT_GELU) {
    const Normal p = normal_of(x);
    return make_float2(x * p.cdf, fmaf(x * 0.39894228f, p.density, p.cdf));
  }
  const Sigmoid s = sigmoid2(x);
  if (ACT == PIPAD_ACT_SIGMOID) return make_float2(s.s, s.s * s.rest);
  return make_float2(x * s.s, s.s * fmaf(x, s.rest, 1.f));
}

// ---- arguments ----------------------------------------------------------------------------------
struct FfArgs {
  const float *X[PIPAD_MAX_K], *dY[PIPAD_MAX_K];
  float *out[PIPAD_MAX_K];  // Y or dX
  int64_t ldx, lddy, ldo, rows;
  int32_t n, k, F, hidden, Fo;
  int32_t ht, fq, oq, ft, ot;  // 32-column tiles of the hidden columns, 16- and 32-column tiles of X's and Y's
  bool vec_x, vec_dy, vec_o;
  // Weights as fragments.  gu: [ht], each [fq][Wg, Wu], m = hidden column, depth = X's columns, and behind them the biases of the tile's
  // hidden columns (32 floats of bg, 32 of bu, 256 bytes unused), 0 where there are none.  down: [ht][ot][2], m = Y's column, depth of a
  // result = hidden.  up: [ht][oq], m = hidden, depth = Y's columns (Wd).  back: [ht][ft][2][Wg, Wu], m = X's column, depth of a result = hidden.
  const u32x4 *gu, *down, *up, *back;
  const float *bd;  // padded with zeros to whole tiles
  const float *Wg, *Wu, *Wd, *bg, *bu;  // as they came
  int64_t ldwg, ldwu, ldwd;
  // weight gradients: partial sums of `parts` ranges of rows, each [dWg F x hidden | dWu | dWd hidden x Fo | dbg | dbu | dbd]
  float *partial;
  int64_t part_floats, tiles_per_part;
};

struct RowAt {
  int32_t t, i;
};
__device__ inline RowAt row_at(const FfArgs &a, int64_t base, int offset) {  // row base + offset, or the last one
  const int64_t last = a.rows - 1 - base;
  int64_t i = base % a.n + (offset < last ? offset : last);
  int32_t t = (int32_t)(base / a.n);
  while (i >= a.n) i -= a.n, ++t;
  return {t, (int32_t)i};
}

// Columns c .. c + 7 of a row; 0 behind the last one.
__device__ inline void load8(float (&v)[8], const float *p, int c, int F, bool vec) {
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    if (vec && c + h + 4 <= F) {
      const float4 t = *reinterpret_cast<const float4 *>(p + c + h);
      v[h] = t.x, v[h + 1] = t.y, v[h + 2] = t.z, v[h + 3] = t.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[h + e] = c + h + e < F ? p[c + h + e] : 0.f;
    }
  }
}
__device__ inline f32x16 zeros() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
__device__ inline void add(f32x16 &c, float sign, const f32x16 &x) {
#pragma unroll
  for (int r = 0; r < 16; ++r) c[r] = fmaf(sign, x[r], c[r]);
}
// A column vector, one value a row of a result.
__device__ inline f32x16 per_row(const float *p, int g) {
  f32x16 z;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float4 t = *reinterpret_cast<const float4 *>(p + 8 * q + 4 * g);
    z[4 * q] = t.x, z[4 * q + 1] = t.y, z[4 * q + 2] = t.z, z[4 * q + 3] = t.w;
  }
  return z;
}
__device__ inline Split half(const f32x16 &r, int s) {  // the registers 8 s .. 8 s + 7 as an operand
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = r[8 * s + j];
  return split8(v);
}
// A result's rows are columns c0 .. of a matrix, its column m a row of it.
__device__ inline void store_tile(const f32x16 &r, float *row, int c0, int F, bool vec, int g) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = c0 + 8 * q + 4 * g;
    if (vec && c + 4 <= F) {
      *reinterpret_cast<float4 *>(row + c) = make_float4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < F) row[c + e] = r[4 * q + e];
    }
  }
}

// Copies whole 1024-byte pieces to LDS past the registers; staged() waits for them, and for the other waves.
template <int WAVES, int WORDS>
__device__ inline void stage(const u32x4 *from, u32x4 *to) {
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * kWave;
#pragma unroll
  for (int i = 0; i < WORDS; i += WAVES * kWave)
    if (i + WAVES * kWave <= WORDS || i + wave < WORDS)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from + i + wave + lane),
                                       (__attribute__((address_space(3))) void *)(to + i + wave), 16, 0, 0);
}
__device__ inline void staged() {
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  __syncthreads();
}

// A kernel for rows of few columns, by its tiles of them, and the waves of its workgroups.
struct Kept {
  void (*kernel)(FfArgs);
  int waves;
};
Kept kept_forward(int act, int fq, int ot);
Kept kept_backward(int act, int fq, int oq);
Kept kept_weights(int act, int fd, int od);  // tiles of 32 columns

}  // namespace ff
}  // namespace pipad

#endif  // PIPAD_GATED_FF_H_
