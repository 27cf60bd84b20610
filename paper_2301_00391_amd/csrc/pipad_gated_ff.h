// The gated feed-forward block on node rows, and its gradients (pipad_gated_ff, pipad_gated_ff_backward in include/pipad.h): what its kernels share.
//
//   G = X Wg + bg,  U = X Wu + bu,  H = act(G) * U,  Y = H Wd + bd
//
// G, U and H are several times as wide as the rows and are never written: a wave keeps 32 node rows, walks the hidden columns 32 at
// a time, and its share of H goes from the registers where the matrix instructions left it straight into the next product.  The
// backward pass makes G and U again, which is two products out of eleven, where keeping them would be 8 bytes a hidden column and row.
//
// Products of 32-bit floats from matrix instructions on 16-bit ones: x s = h1 + h2, each piece the nearest with 11 bits to what is left; h1 k1 +
// h1 k2 + h2 k1, the fourth product being below 2^-22 of the whole, summed in 32 bits.  Pieces hold 22 bits and a sign, so an operand is off by
// 2^-22 at most and 2^-24 on average; the error of a sum of 64 products came out as 1.0e-7 of its size (1.4e-7 for a chain of 32-bit
// multiply-adds, whose roundings are more).  Three instructions of 32 cycles for 32 x 32 x 16 are 5.3 times as fast as the matrix instructions on
// floats; bf16 pieces hold the last two bits, too, and reach as far as floats do, but take three each and six products, and issue and the card's
// power are what bounds these kernels: 8 million rows of 64 through 171 columns took 2.85 ms with them and take 2.21 now.
//
// A 16-bit float reaches from 2^-24 to 2^16, so operands are scaled, by powers of two: rows of X and dY by their largest value, weights by the
// largest of the column that a result sees (Wg's and Wu's columns for G and U, Wd's rows for dH, Wd's columns for Y, and for dX the rows of Wg and
// Wu, which share one), so that a huge or infinite weight is a matter of its own column; H, dG and dU by the largest of a node's (or in the weights'
// gradients a hidden column's) 32 values at a time, whose products are added up outside.  Largest values come to 2^14 .. 2^15.  h2 is kept 2^11
// larger and its products are summed apart, so that values down to 2^-29 of the largest have all their bits, and smaller ones an error of 2^-51 of
// it.  With h2 as it is and one sum they have them down to 2^-18, and an error of 2^-40 below, which columns of X at 2^-20 of the others, or gates that
// are nearly closed, come to: 7 % less time forward and 10 % backward (64 columns through 256) do not pay for that.
// A value that is not finite makes its row NaN (or infinite).
//
// An instruction aligns what it adds to the largest of it and cuts off, so a sum comes out low by some 1e-8 of its terms' size; over millions of
// rows that would be seen, and the weights' gradients are taken with every other tile of rows negated, where it comes out high.  They are sums
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

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32, kDepth = 16;
constexpr int kFragment = 2 * kWave;  // the two pieces of a 32 x 16 operand, in 16-byte words
constexpr float kWide = 2048.f;       // what h2 is multiplied by
// Wg's and Wu's fragments of a hidden tile, and its vectors behind them (struct TileVectors).
__host__ __device__ constexpr int gu_words(int fq) { return fq * 2 * kFragment + kWave; }
struct TileVectors {
  float bg[kTile], bu[kTile];
  float inv_g[kTile], inv_u[kTile], inv_d[kTile];  // 1 over the scales of Wg's and Wu's columns, and of Wd's rows
};
static_assert(sizeof(TileVectors) <= kWave * sizeof(u32x4), "fits behind the fragments");

__host__ __device__ constexpr int64_t tiles(int64_t x, int64_t t) { return (x + t - 1) / t; }

__device__ inline int result_depth(int s, int g, int j) { return 16 * s + 8 * (j / 4) + 4 * g + j % 4; }

// ---- scales and pieces --------------------------------------------------------------------------
struct Scale {
  float to, inv;  // powers of two, 1 / to
};
// Brings the largest magnitude to 2^14 .. 2^15; below 2^-100, and for 0, by 2^114 all the same, so that both factors are ordinary floats.
__device__ inline Scale scale_for(float largest) {
  const uint32_t e = min(max(__float_as_uint(largest) >> 23, 27u), 254u);
  return {__uint_as_float((268u - e) << 23), __uint_as_float((e - 14u) << 23)};
}
__device__ inline float max_of(float a, float b) { return fmaxf(a, fabsf(b)); }
template <int N>
__device__ inline float largest_of(const float (&v)[N], float so_far = 0.f) {
#pragma unroll
  for (int j = 0; j < N; ++j) so_far = max_of(so_far, v[j]);
  return so_far;
}
// Largest of a lane and the one 32, or 16, lanes away.
__device__ inline float max_over_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_over_16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_of_wave(float x) {
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) x = fmaxf(x, __shfl_xor(x, d));
  return max_over_32(max_over_16(x));
}

struct Split {
  u32x4 p[2];
};
__device__ inline Split split8(const float (&v)[8], float scale) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  Split s;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = v[2 * i] * scale, b = v[2 * i + 1] * scale;
    const f16x2 h = __builtin_convertvector((f32x2{a, b}), f16x2);
    const f16x2 rest = __builtin_convertvector((f32x2{fmaf((float)h[0], -kWide, a * kWide), fmaf((float)h[1], -kWide, b * kWide)}), f16x2);
    s.p[0][i] = __builtin_bit_cast(uint32_t, h);
    s.p[1][i] = __builtin_bit_cast(uint32_t, rest);
  }
  return s;
}

// ---- products -----------------------------------------------------------------------------------
__device__ inline f32x16 zeros() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
__device__ inline f32x16 mfma(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
struct Sums {  // main + cross / kWide
  f32x16 main, cross;
};
__device__ inline Sums no_sums() { return {zeros(), zeros()}; }
__device__ inline void add_product(Sums &c, const Split &a, const Split &b) {
  c.cross = mfma(a.p[1], b.p[0], c.cross);
  c.main = mfma(a.p[0], b.p[0], c.main);
  c.cross = mfma(a.p[0], b.p[1], c.cross);
}
__device__ inline Split fragment(const u32x4 *at, int64_t index) {
  at += index * kFragment + (threadIdx.x & (kWave - 1));
  return Split{{at[0], at[kWave]}};
}
// The sums times what was divided out, of the result's column and of its row, and a vector with one value a row.
__device__ inline float sum_of(const Sums &c, int r) { return fmaf(c.cross[r], 1.f / kWide, c.main[r]); }
__device__ inline f32x16 value_of(const Sums &c, float inv, const float *inv_row, const float *per_row, int g) {
  f32x16 z;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float4 t = *reinterpret_cast<const float4 *>(per_row + 8 * q + 4 * g), u = *reinterpret_cast<const float4 *>(inv_row + 8 * q + 4 * g);
    const float b[4] = {t.x, t.y, t.z, t.w}, f[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) z[4 * q + e] = fmaf(sum_of(c, 4 * q + e), inv * f[e], b[e]);
  }
  return z;
}
__device__ inline f32x16 value_of(const Sums &c, float inv, const float *inv_row, int g) {
  f32x16 z;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float4 u = *reinterpret_cast<const float4 *>(inv_row + 8 * q + 4 * g);
    const float f[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) z[4 * q + e] = sum_of(c, 4 * q + e) * (inv * f[e]);
  }
  return z;
}
__device__ inline void add(f32x16 &c, float factor, const Sums &x) {
#pragma unroll
  for (int r = 0; r < 16; ++r) c[r] = fmaf(factor, sum_of(x, r), c[r]);
}
__device__ inline float largest_of(const f32x16 &x, float so_far = 0.f) {
#pragma unroll
  for (int r = 0; r < 16; ++r) so_far = max_of(so_far, x[r]);
  return so_far;
}
__device__ inline Split half(const f32x16 &r, int s, float scale) {  // the registers 8 s .. 8 s + 7 as an operand
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = r[8 * s + j];
  return split8(v, scale);
}

// A sum of many terms that carries what the additions round off (over thousands of tiles a plain one is off by more than 1e-6).
struct Total {
  float sum = 0.f, lost = 0.f;
  __device__ void add(float x) {
    x -= lost;
    const float s = sum + x;
    lost = (s - sum) - x;
    sum = s;
  }
};

// ---- the activations ----------------------------------------------------------------------------
// The normal distribution's tail Q(|x|) = 1 - Phi(|x|), and its density times sqrt(2 pi), exp(-x^2 / 2).  Q is that times a function that falls like
// 1 / |x|: a polynomial in k = 1 / (1 + 0.275 |x|) without a constant term, which is the form of formula 26.2.17 in Abramowitz and Stegun's handbook,
// fitted here for the least error of |x| Q (1.1e-8, 6.9e-8 with the arithmetic's own; of Q itself 4e-5 of it at most up to |x| = 4).
// x Phi(x) = max(x, 0) - |x| Q(|x|) for either sign.
struct Normal {
  float tail, density;
};
__device__ inline Normal normal_of(float x) {
  const float k = __builtin_amdgcn_rcpf(fmaf(0.275f, fabsf(x), 1.f)), e = __builtin_amdgcn_exp2f(x * x * -0.72134752f);
  float q = -0.11416427046060562f;
  q = fmaf(q, k, 0.44915953278541565f);
  q = fmaf(q, k, -0.3263809084892273f);
  q = fmaf(q, k, 0.3302135169506073f);
  q = fmaf(q, k, 0.04359893128275871f);
  q = fmaf(q, k, 0.11757319420576096f);
  return {q * (k * e), e};
}
__device__ inline float relu_of(float x) { return x < 0.f ? 0.f : x; }  // (NaN stays)

template <int ACT>
__device__ inline float activate(float x) {
  if (ACT == PIPAD_ACT_RELU) return relu_of(x);
  if (ACT == PIPAD_ACT_GELU) return fmaf(-fabsf(x), normal_of(x).tail, relu_of(x));
  const float s = __builtin_amdgcn_rcpf(1.f + __expf(-x));
  return ACT == PIPAD_ACT_SIGMOID ? s : x * s;
}
// act(x) and its slope
template <int ACT>
__device__ inline float2 activate_slope(float x) {
  if (ACT == PIPAD_ACT_RELU) return make_float2(relu_of(x), x > 0.f ? 1.f : 0.f);
  if (ACT == PIPAD_ACT_GELU) {
    const Normal p = normal_of(x);
    return make_float2(fmaf(-fabsf(x), p.tail, relu_of(x)), fmaf(x * 0.39894228f, p.density, x < 0.f ? p.tail : 1.f - p.tail));
  }
  // 1 - s = exp(-x) s: the difference would lose it where the gate is wide open.  Where the exponential has no end, s is 0 and the product is no
  // number, of which the least is 1.
  const float e = __expf(-x), s = __builtin_amdgcn_rcpf(1.f + e), rest = fminf(e * s, 1.f);
  if (ACT == PIPAD_ACT_SIGMOID) return make_float2(s, s * rest);
  const float a = x * s;
  return make_float2(a, fmaf(a, rest, s));
}

// ---- arguments ----------------------------------------------------------------------------------
struct FfArgs {
  const float *X[PIPAD_MAX_K], *dY[PIPAD_MAX_K];
  float *out[PIPAD_MAX_K];  // Y or dX
  int64_t ldx, lddy, ldo, rows;
  int32_t n, k, F, hidden, Fo;
  int32_t ht, fq, oq, ft, ot;  // 32-column tiles of the hidden columns, 16- and 32-column tiles of X's and Y's
  bool vec_x, vec_dy, vec_o;
  // Weights as fragments.  gu: [ht], each [fq][Wg, Wu], m = hidden column, depth = X's columns, and a TileVectors behind them.
  // up: [ht][oq], m = hidden, depth = Y's columns (Wd).  down: [ht][ot][2], m = Y's column, depth of a result = hidden.
  // back: [ht][ft][2][Wg, Wu], m = X's column, depth of a result = hidden.
  const u32x4 *gu, *down, *up, *back;
  const float *inv_out, *bd;  // 1 over the scales of down's or back's columns, over kToOne, and bd; padded to whole tiles
  const float *Wg, *Wu, *Wd, *bg, *bu, *bd_in;  // as they came
  int64_t ldwg, ldwu, ldwd;
  // weight gradients: partial sums of `parts` ranges of rows, each [dWg F x hidden | dWu | dWd hidden x Fo | dbg | dbu | dbd]
  float *partial;
  int64_t part_floats, tiles_per_part;
};
__device__ inline const TileVectors &vectors_of(const u32x4 *gu, int fq) { return *reinterpret_cast<const TileVectors *>(gu + fq * 2 * kFragment); }

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
// A row of up to 16 N columns, whose other half lane m + 32 has, as pieces; returns 1 over its scale.
template <int N>
__device__ inline float load_row(Split (&x)[N], const float *row, int g, int F, bool vec) {
  float v[N][8], largest = 0.f;
#pragma unroll
  for (int q = 0; q < N; ++q) load8(v[q], row, q * kDepth + 8 * g, F, vec);
#pragma unroll
  for (int q = 0; q < N; ++q) largest = largest_of(v[q], largest);
  const Scale s = scale_for(max_over_32(largest));
#pragma unroll
  for (int q = 0; q < N; ++q) x[q] = split8(v[q], s.to);
  return s.inv;
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
// Sums of Y's and dX's columns are kept for weights that come to 1 .. 2, not to 2^14 .. 2^15: they are about as large as H's, or dG's and dU's, sums then,
// and end where those do.
constexpr float kToOne = 1.f / 16384.f;
// Y's or dX's columns c0 .. as they are: times 1 over their scales, and Y's bias.
__device__ inline f32x16 unscaled(const f32x16 &sums, const float *inv, const float *bias, int g) {
  f32x16 z = per_row(inv, g), b = zeros();
  if (bias) b = per_row(bias, g);
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = fmaf(sums[r], z[r], b[r]);
  return z;
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
template <int ACT>
Kept kept_forward(int fq, int ot);
template <int ACT>
Kept kept_backward(int fq, int oq);
Kept split_forward(int act, int ot);  // 32 rows a workgroup
Kept split_backward(int act, int ft);
template <int ACT>
Kept kept_weights(int fd, int od, int waves);  // tiles of 32 columns; 4 waves, or up to 2 tiles 8

}  // namespace ff
}  // namespace pipad

#endif  // PIPAD_GATED_FF_H_
