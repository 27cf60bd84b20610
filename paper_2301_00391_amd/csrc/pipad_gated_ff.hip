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
#include "pipad_internal.h"

namespace pipad {

namespace {

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
  int32_t n, F, hidden, Fo;
  int32_t ht, fq, oq, ft, ot;  // 32-column tiles of the hidden columns, 16- and 32-column tiles of X's and Y's
  bool vec_x, vec_dy, vec_o;
  // Weights as fragments.  gu: [ht], each [fq][Wg, Wu], m = hidden column, depth = X's columns, and behind them the biases of the tile's
  // hidden columns (32 floats of bg, 32 of bu, 256 bytes unused), 0 where there are none.  down: [ht][ot][2], m = Y's column, depth of a
  // result = hidden.  up: [ht][oq], m = hidden, depth = Y's columns (Wd).  back: [ht][ft][2][Wg, Wu], m = X's column, depth of a result = hidden.
  const u32x4 *gu, *down, *up, *back;
  const float *bd;  // padded with zeros to whole tiles
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

// ---- weights as fragments -----------------------------------------------------------------------
struct PackArgs {
  const float *Wg, *Wu, *Wd, *bg, *bu, *bd;
  int64_t ldwg, ldwu, ldwd;
  int32_t F, hidden, Fo, ht, fq, oq, ft, ot;
  int64_t n_gu, n_down, n_up, n_back;  // fragments of each kind (0: not wanted)
  u32x4 *gu, *down, *up, *back;
  float *pbd;
};
__global__ void __launch_bounds__(kBlock) k_ff_pack(PackArgs a) {
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5;
  int64_t at = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kWave;
  if (at == 0)  // the last bias, by the first wave
    for (int c = lane; c < a.ot * kTile; c += kWave) a.pbd[c] = a.bd && c < a.Fo ? a.bd[c] : 0.f;
  float v[8];
  u32x4 *to;
  if (at < a.n_gu) {
    const int w = (int)(at % 2), q = (int)(at / 2 % a.fq), h = (int)(at / 2 / a.fq);
    const float *W = w ? a.Wu : a.Wg;
    const int64_t ld = w ? a.ldwu : a.ldwg;
    const int hid = h * kTile + m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int f = q * kDepth + 8 * g + j;
      v[j] = f < a.F && hid < a.hidden ? W[f * ld + hid] : 0.f;
    }
    to = a.gu + (int64_t)h * gu_words(a.fq) + (at - (int64_t)h * a.fq * 2) * kFragment;
    if (at == (int64_t)h * a.fq * 2) {  // the tile's biases, by the wave of its first fragment
      const float *const b = g ? a.bu : a.bg;
      reinterpret_cast<float *>(a.gu + (int64_t)h * gu_words(a.fq) + a.fq * 2 * kFragment)[lane] = b && hid < a.hidden ? b[hid] : 0.f;
    }
  } else if ((at -= a.n_gu) < a.n_down) {
    const int s = (int)(at % 2), o = (int)(at / 2 % a.ot), h = (int)(at / 2 / a.ot), fo = o * kTile + m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int hid = h * kTile + result_depth(s, g, j);
      v[j] = hid < a.hidden && fo < a.Fo ? a.Wd[hid * a.ldwd + fo] : 0.f;
    }
    to = a.down + at * kFragment;
  } else if ((at -= a.n_down) < a.n_up) {
    const int q = (int)(at % a.oq), h = (int)(at / a.oq), hid = h * kTile + m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int fo = q * kDepth + 8 * g + j;
      v[j] = hid < a.hidden && fo < a.Fo ? a.Wd[hid * a.ldwd + fo] : 0.f;
    }
    to = a.up + at * kFragment;
  } else if ((at -= a.n_up) < a.n_back) {
    const int w = (int)(at % 2), s = (int)(at / 2 % 2), t = (int)(at / 4 % a.ft), h = (int)(at / 4 / a.ft), f = t * kTile + m;
    const float *W = w ? a.Wu : a.Wg;
    const int64_t ld = w ? a.ldwu : a.ldwg;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int hid = h * kTile + result_depth(s, g, j);
      v[j] = hid < a.hidden && f < a.F ? W[f * ld + hid] : 0.f;
    }
    to = a.back + at * kFragment;
  } else {
    return;
  }
  const Split s = split8(v);
#pragma unroll
  for (int q = 0; q < 3; ++q) to[q * kWave + lane] = s.p[q];
}

// ---- forward ------------------------------------------------------------------------------------
// A wave: 32 node rows, OT tiles of Y's columns from tile blockIdx.y * OT on.  Results lie transposed (a node row is a lane's column).
template <int ACT, int OT>
__global__ void __launch_bounds__(kBlock, 2) k_ff_rows(FfArgs a) {
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5;
  const int64_t base = ((int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / kWave) * kTile;
  if (base >= a.rows) return;
  const RowAt at = row_at(a, base, m);
  const float *const x = a.X[at.t] + at.i * a.ldx;
  const int o0 = blockIdx.y * OT;
  f32x16 y[OT];
#pragma unroll
  for (int o = 0; o < OT; ++o) y[o] = o0 + o < a.ot ? per_row(a.bd + (o0 + o) * kTile, g) : zeros();
  for (int h = 0; h < a.ht; ++h) {
    const u32x4 *const gu = a.gu + (int64_t)h * gu_words(a.fq);
    const float *const bias = reinterpret_cast<const float *>(gu + a.fq * 2 * kFragment);
    f32x16 G = per_row(bias, g), U = per_row(bias + kTile, g);
    for (int q = 0; q < a.fq; ++q) {
      float v[8];
      load8(v, x, q * kDepth + 8 * g, a.F, a.vec_x);
      const Split b = split8(v);
      G = product(fragment(gu, 2 * q), b, G);
      U = product(fragment(gu, 2 * q + 1), b, U);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) G[r] = activate<ACT>(G[r]) * U[r];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const Split b = half(G, s);
#pragma unroll
      for (int o = 0; o < OT; ++o)
        if (o0 + o < a.ot) y[o] = product(fragment(a.down, ((int64_t)h * a.ot + o0 + o) * 2 + s), b, y[o]);
    }
  }
  if (base + m >= a.rows) return;
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int o = 0; o < OT; ++o) store_tile(y[o], out, (o0 + o) * kTile, a.Fo, a.vec_o, g);
}

// The same where a row's columns, and those of its result, are 128 at most: X's pieces stay in registers, and the waves of a workgroup, 32 node
// rows each, share the weights through LDS.  A hidden tile's weights come in two phases, [Wg, Wu, biases] and [Wd], each into a buffer of its
// own while the other is multiplied: loaded past the registers, one barrier a phase.  What is in flight is waited for before the barrier.
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

template <int ACT, int FQ, int OT, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, 2) k_ff_kept(FfArgs a) {
  constexpr int kGu = gu_words(FQ), kDown = OT * 2 * kFragment;
  __shared__ u32x4 gu[kGu], down[kDown];  // (two arrays: what is read of one does not wait for what is loaded into the other)
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5;
  const int64_t base = ((int64_t)blockIdx.x * WAVES + threadIdx.x / kWave) * kTile;
  stage<WAVES, kGu>(a.gu, gu);
  const RowAt at = row_at(a, base < a.rows ? base : a.rows - 1, m);
  Split x[FQ];
  {
    const float *const row = a.X[at.t] + at.i * a.ldx;
    float v[FQ][8];
#pragma unroll
    for (int q = 0; q < FQ; ++q) load8(v[q], row, q * kDepth + 8 * g, a.F, a.vec_x);
#pragma unroll
    for (int q = 0; q < FQ; ++q) x[q] = split8(v[q]);
  }
  f32x16 y[OT];
#pragma unroll
  for (int o = 0; o < OT; ++o) y[o] = per_row(a.bd + o * kTile, g);
  const float *const bias = reinterpret_cast<const float *>(gu + FQ * 2 * kFragment);
  for (int h = 0; h < a.ht; ++h) {
    staged();
    stage<WAVES, kDown>(a.down + (int64_t)h * kDown, down);
    f32x16 G = per_row(bias, g), U = per_row(bias + kTile, g);
#pragma unroll
    for (int q = 0; q < FQ; ++q) {
      G = product(fragment(gu, 2 * q), x[q], G);
      U = product(fragment(gu, 2 * q + 1), x[q], U);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) G[r] = activate<ACT>(G[r]) * U[r];
    staged();
    if (h + 1 < a.ht) stage<WAVES, kGu>(a.gu + (int64_t)(h + 1) * kGu, gu);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const Split b = half(G, s);
#pragma unroll
      for (int o = 0; o < OT; ++o) y[o] = product(fragment(down, 2 * o + s), b, y[o]);
    }
  }
  if (base + m >= a.rows) return;
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int o = 0; o < OT; ++o) store_tile(y[o], out, o * kTile, a.Fo, a.vec_o, g);
}

// ---- the gradient of X --------------------------------------------------------------------------
template <int ACT, int FT>
__global__ void __launch_bounds__(kBlock, 2) k_ff_rows_backward(FfArgs a) {
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5;
  const int64_t base = ((int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / kWave) * kTile;
  if (base >= a.rows) return;
  const RowAt at = row_at(a, base, m);
  const float *const x = a.X[at.t] + at.i * a.ldx, *const dy = a.dY[at.t] + at.i * a.lddy;
  const int f0 = blockIdx.y * FT;
  f32x16 dx[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) dx[f] = zeros();
  for (int h = 0; h < a.ht; ++h) {
    const u32x4 *const gu = a.gu + (int64_t)h * gu_words(a.fq);
    const float *const bias = reinterpret_cast<const float *>(gu + a.fq * 2 * kFragment);
    f32x16 G = per_row(bias, g), U = per_row(bias + kTile, g), dH = zeros();
    float v[8];
    for (int q = 0; q < a.fq; ++q) {
      load8(v, x, q * kDepth + 8 * g, a.F, a.vec_x);
      const Split b = split8(v);
      G = product(fragment(gu, 2 * q), b, G);
      U = product(fragment(gu, 2 * q + 1), b, U);
    }
    for (int q = 0; q < a.oq; ++q) {
      load8(v, dy, q * kDepth + 8 * g, a.Fo, a.vec_dy);
      dH = product(fragment(a.up, (int64_t)h * a.oq + q), split8(v), dH);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float2 c = activate_slope<ACT>(G[r]);
      G[r] = dH[r] * U[r] * c.y;
      U[r] = dH[r] * c.x;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const Split dg = half(G, s), du = half(U, s);
#pragma unroll
      for (int f = 0; f < FT; ++f)
        if (f0 + f < a.ft) {
          const int64_t w = (((int64_t)h * a.ft + f0 + f) * 2 + s) * 2;
          dx[f] = product(fragment(a.back, w), dg, dx[f]);
          dx[f] = product(fragment(a.back, w + 1), du, dx[f]);
        }
    }
  }
  if (base + m >= a.rows) return;
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int f = 0; f < FT; ++f) store_tile(dx[f], out, (f0 + f) * kTile, a.F, a.vec_o, g);
}

// ---- the gradients of the weights ---------------------------------------------------------------
// A wave: one tile of hidden columns, the rows of one part, T tiles of X's and of Y's columns from tile blockIdx.z * T on.  Results
// lie as they are (a hidden column is a lane's column), so dG, dU and H are operands of products whose depth is the node rows.
template <int ACT, int T>
__global__ void __launch_bounds__(kBlock, 1) k_ff_weights_backward(FfArgs a) {
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5;
  const int h = blockIdx.x * kWavesPerBlock + threadIdx.x / kWave;
  if (h >= a.ht) return;
  const int t0 = blockIdx.z * T;
  f32x16 dwg[T], dwu[T], dwd[T];
#pragma unroll
  for (int t = 0; t < T; ++t) dwg[t] = dwu[t] = dwd[t] = zeros();
  float dbg = 0.f, dbu = 0.f, dbd[T] = {};
  const u32x4 *const gu = a.gu + (int64_t)h * gu_words(a.fq);
  const float *const bias = reinterpret_cast<const float *>(gu + a.fq * 2 * kFragment);
  const float bg = bias[m], bu = bias[kTile + m];
  const int64_t first = blockIdx.y * a.tiles_per_part * kTile;
  const int64_t end = first + a.tiles_per_part * kTile < a.rows ? first + a.tiles_per_part * kTile : a.rows;
  for (int64_t base = first; base < end; base += kTile) {
    const bool there = base + m < end;
    const RowAt at = row_at(a, base, m);
    const float *const x = a.X[at.t] + at.i * a.ldx, *const dy = a.dY[at.t] + at.i * a.lddy;
    const float sign = base / kTile % 2 ? -1.f : 1.f;
    f32x16 G, U, dH = zeros();
#pragma unroll
    for (int r = 0; r < 16; ++r) G[r] = sign * bg, U[r] = sign * bu;
    float v[8];
    for (int q = 0; q < a.fq; ++q) {
      load8(v, x, q * kDepth + 8 * g, there ? a.F : 0, a.vec_x);
      const Split b = split8(v, sign);
      G = product(b, fragment(gu, 2 * q), G);
      U = product(b, fragment(gu, 2 * q + 1), U);
    }
    for (int q = 0; q < a.oq; ++q) {
      load8(v, dy, q * kDepth + 8 * g, there ? a.Fo : 0, a.vec_dy);
      dH = product(split8(v, sign), fragment(a.up, (int64_t)h * a.oq + q), dH);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float2 c = activate_slope<ACT>(sign * G[r]);
      const float u = sign * U[r], d = sign * dH[r];
      G[r] = d * u * c.y;
      U[r] = d * c.x;
      dH[r] = c.x * u;
      dbg += G[r];
      dbu += U[r];
    }
    Split dg[2], du[2], hh[2];
    RowAt rows[2][8];
    bool in[2][8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      dg[s] = half(G, s), du[s] = half(U, s), hh[s] = half(dH, s);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int d = result_depth(s, g, j);
        rows[s][j] = row_at(a, base, d);
        in[s][j] = base + d < end;
      }
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int c = (t0 + t) * kTile + m;
      if (t0 + t < a.ft) {
        f32x16 g_sum = zeros(), u_sum = zeros();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = in[s][j] && c < a.F ? a.X[rows[s][j].t][rows[s][j].i * a.ldx + c] : 0.f;
          const Split xs = split8(v, sign);
          g_sum = product(xs, dg[s], g_sum);
          u_sum = product(xs, du[s], u_sum);
        }
        add(dwg[t], sign, g_sum);
        add(dwu[t], sign, u_sum);
      }
      if (t0 + t < a.ot) {
        f32x16 d_sum = zeros();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            v[j] = in[s][j] && c < a.Fo ? a.dY[rows[s][j].t][rows[s][j].i * a.lddy + c] : 0.f;
            dbd[t] += v[j];
          }
          d_sum = product(hh[s], split8(v, sign), d_sum);
        }
        add(dwd[t], sign, d_sum);
      }
    }
  }
  float *const to = a.partial + blockIdx.y * a.part_floats, *const to_d = to + 2 * (int64_t)a.F * a.hidden;
  const int hid = h * kTile + m;
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = result_depth(r / 8, g, r % 8), f = (t0 + t) * kTile + row;
      if (f < a.F && hid < a.hidden) {
        to[(int64_t)f * a.hidden + hid] = dwg[t][r];
        to[((int64_t)a.F + f) * a.hidden + hid] = dwu[t][r];
      }
      const int fo = (t0 + t) * kTile + m;
      if (h * kTile + row < a.hidden && fo < a.Fo) to_d[(int64_t)(h * kTile + row) * a.Fo + fo] = dwd[t][r];
    }
  float *const to_b = to_d + (int64_t)a.hidden * a.Fo;
  dbg += __shfl_xor(dbg, 32);
  dbu += __shfl_xor(dbu, 32);
  if (blockIdx.z == 0 && g == 0 && hid < a.hidden) {
    to_b[hid] = dbg;
    to_b[a.hidden + hid] = dbu;
  }
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const float b = dbd[t] + __shfl_xor(dbd[t], 32);
    const int fo = (t0 + t) * kTile + m;
    if (h == 0 && g == 0 && fo < a.Fo) to_b[2 * a.hidden + fo] = b;
  }
}

struct SumArgs {
  const float *partial;
  int64_t part_floats;
  int32_t parts, F, hidden, Fo;
  pipad_gated_ff_grads_t out;
};
// The parts added up, always in the same order, each value to its place.
__global__ void __launch_bounds__(kBlock) k_ff_sums(SumArgs a) {
  __shared__ float part[4][kWave];
  const int x = threadIdx.x & (kWave - 1), y = threadIdx.x / kWave;
  const int64_t e = (int64_t)blockIdx.x * kWave + x;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (e < a.part_floats) {
    int p = y;
    for (; p + 12 < a.parts; p += 16) {
#pragma unroll
      for (int u = 0; u < 4; ++u) s[u] += a.partial[(p + 4 * u) * a.part_floats + e];
    }
    for (; p < a.parts; p += 4) s[0] += a.partial[p * a.part_floats + e];
  }
  part[y][x] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (y != 0 || e >= a.part_floats) return;
  const float v = (part[0][x] + part[1][x]) + (part[2][x] + part[3][x]);
  const int64_t in = (int64_t)a.F * a.hidden, down = (int64_t)a.hidden * a.Fo;
  int64_t q = e;
  const auto put = [&](float *to, int64_t ld, int64_t columns) {
    if (to) to[q / columns * ld + q % columns] = v;
  };
  if (q < in) return put(a.out.dWg, a.out.lddwg, a.hidden);
  if ((q -= in) < in) return put(a.out.dWu, a.out.lddwu, a.hidden);
  if ((q -= in) < down) return put(a.out.dWd, a.out.lddwd, a.Fo);
  if ((q -= down) < a.hidden) return put(a.out.dbg, 0, a.hidden);
  if ((q -= a.hidden) < a.hidden) return put(a.out.dbu, 0, a.hidden);
  q -= a.hidden;
  put(a.out.dbd, 0, a.Fo);
}

// ---- host ---------------------------------------------------------------------------------------
bool aligned(const float *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 4 == 0; }

// Tiles of up to 128 columns: as many as one of the kernels that keep a row has; behind the columns that there are the fragments hold 0.
constexpr int kKept = 128;
int32_t column_tiles(int32_t F) {
  const int32_t t = (int32_t)tiles(F, kTile);
  return F > kKept || t <= 2 ? t : 4;
}
int32_t depth_tiles(int32_t F) {
  const int32_t t = (int32_t)tiles(F, kDepth);
  return F > kKept || t <= 2 ? t : t <= 4 ? 4 : t <= 6 ? 6 : 8;
}

// What lies where in the workspace (bytes), the same for the size query and the calls.
struct Plan {
  int32_t ht, fq, oq, ft, ot;
  int64_t n_gu, n_down, n_up, n_back;
  size_t gu, down, up, back, bd, partial, total;
  int64_t rows, part_floats, parts, tiles_per_part;
  Plan(const pipad_gated_ff_t &c, int32_t n, int32_t k, bool backward) {
    ht = (int32_t)tiles(c.hidden, kTile);
    fq = depth_tiles(c.F), ft = column_tiles(c.F), oq = depth_tiles(c.Fo), ot = column_tiles(c.Fo);
    n_gu = (int64_t)ht * fq * 2;
    n_down = backward ? 0 : (int64_t)ht * ot * 2;
    n_up = backward ? (int64_t)ht * oq : 0;
    n_back = backward ? (int64_t)ht * ft * 4 : 0;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
      const size_t here = at;
      at += align_up(bytes, 256);
      return here;
    };
    const size_t fragment_bytes = kFragment * sizeof(u32x4);
    gu = take((size_t)ht * gu_words(fq) * sizeof(u32x4)), down = take(n_down * fragment_bytes);
    up = take(n_up * fragment_bytes), back = take(n_back * fragment_bytes);
    bd = take(ot * kTile * sizeof(float));
    // about two waves a SIMD for the weights' gradients, and four tiles of rows at least for each
    rows = (int64_t)n * k;
    part_floats = 2 * (int64_t)c.F * c.hidden + (int64_t)c.hidden * c.Fo + 2 * (int64_t)c.hidden + c.Fo;
    const int64_t row_tiles = tiles(rows, kTile);
    const int64_t most = std::max<int64_t>(1, 2048 / ht);
    tiles_per_part = std::max<int64_t>(4, tiles(row_tiles, most));
    parts = tiles(row_tiles, tiles_per_part);
    partial = take(backward ? (size_t)parts * part_floats * sizeof(float) : 0);
    total = at;
  }
};

FfArgs arguments(const pipad_gated_ff_t &c, const Plan &p, int32_t n, int32_t k, const float *const *X, int64_t ldx, const float *const *dY,
                 int64_t lddy, float *const *out, int64_t ldo, char *ws) {
  FfArgs a{};
  a.vec_x = a.vec_dy = a.vec_o = true;
  for (int t = 0; t < k; ++t) {
    a.X[t] = X[t];
    a.vec_x = a.vec_x && aligned(X[t], ldx);
    if (dY) a.dY[t] = dY[t], a.vec_dy = a.vec_dy && aligned(dY[t], lddy);
    if (out) a.out[t] = out[t], a.vec_o = a.vec_o && aligned(out[t], ldo);
  }
  a.ldx = ldx, a.lddy = lddy, a.ldo = ldo, a.rows = p.rows, a.n = n, a.F = c.F, a.hidden = c.hidden, a.Fo = c.Fo;
  a.ht = p.ht, a.fq = p.fq, a.oq = p.oq, a.ft = p.ft, a.ot = p.ot;
  a.gu = reinterpret_cast<const u32x4 *>(ws + p.gu), a.down = reinterpret_cast<const u32x4 *>(ws + p.down);
  a.up = reinterpret_cast<const u32x4 *>(ws + p.up), a.back = reinterpret_cast<const u32x4 *>(ws + p.back);
  a.bd = reinterpret_cast<const float *>(ws + p.bd);
  a.partial = reinterpret_cast<float *>(ws + p.partial), a.part_floats = p.part_floats, a.tiles_per_part = p.tiles_per_part;
  return a;
}

int pack(const pipad_gated_ff_t &c, const Plan &p, char *ws, hipStream_t st) {
  PackArgs a{c.Wg,   c.Wu,   c.Wd,     c.bg,   c.bu,
             c.bd,   c.ldwg, c.ldwu,   c.ldwd, c.F,
             c.hidden, c.Fo, p.ht,     p.fq,   p.oq,
             p.ft,   p.ot,   p.n_gu,   p.n_down, p.n_up,
             p.n_back, reinterpret_cast<u32x4 *>(ws + p.gu), reinterpret_cast<u32x4 *>(ws + p.down), reinterpret_cast<u32x4 *>(ws + p.up),
             reinterpret_cast<u32x4 *>(ws + p.back), reinterpret_cast<float *>(ws + p.bd)};
  const int64_t waves = p.n_gu + p.n_down + p.n_up + p.n_back;
  hipLaunchKernelGGL(k_ff_pack, dim3((unsigned)tiles(waves, kWavesPerBlock)), dim3(kBlock), 0, st, a);
  PIPAD_HIP(hipGetLastError());
  return PIPAD_OK;
}

// A kernel by activation and by the tiles of columns that a wave keeps: 1, 2 or 4.
#define PIPAD_FF_KERNELS(name)                                                                                                        \
  using name##_fn = void (*)(FfArgs);                                                                                                 \
  constexpr name##_fn name##_of[4][3] = {{name<0, 1>, name<0, 2>, name<0, 4>},                                                        \
                                         {name<1, 1>, name<1, 2>, name<1, 4>},                                                        \
                                         {name<2, 1>, name<2, 2>, name<2, 4>},                                                        \
                                         {name<3, 1>, name<3, 2>, name<3, 4>}};
PIPAD_FF_KERNELS(k_ff_rows)
PIPAD_FF_KERNELS(k_ff_rows_backward)
PIPAD_FF_KERNELS(k_ff_weights_backward)
#undef PIPAD_FF_KERNELS

struct Kept {
  void (*kernel)(FfArgs);
  int waves;
};
template <int ACT, int FQ, int OT>
Kept kept_of() {
  constexpr int kWaves = FQ <= 4 && OT <= 2 ? 4 : 8;
  return {k_ff_kept<ACT, FQ, OT, kWaves>, kWaves};
}
template <int ACT, int FQ>
Kept kept_of(int ot) {
  return ot == 1 ? kept_of<ACT, FQ, 1>() : ot == 2 ? kept_of<ACT, FQ, 2>() : kept_of<ACT, FQ, 4>();
}
template <int ACT>
Kept kept_of(int fq, int ot) {
  switch (fq) {
    case 1: return kept_of<ACT, 1>(ot);
    case 2: return kept_of<ACT, 2>(ot);
    case 4: return kept_of<ACT, 4>(ot);
    case 6: return kept_of<ACT, 6>(ot);
    default: return kept_of<ACT, 8>(ot);
  }
}
Kept kept(int act, int fq, int ot) {
  switch (act) {
    case PIPAD_ACT_SIGMOID: return kept_of<PIPAD_ACT_SIGMOID>(fq, ot);
    case PIPAD_ACT_RELU: return kept_of<PIPAD_ACT_RELU>(fq, ot);
    case PIPAD_ACT_GELU: return kept_of<PIPAD_ACT_GELU>(fq, ot);
    default: return kept_of<PIPAD_ACT_SILU>(fq, ot);
  }
}

int width(int t) { return t <= 1 ? 0 : t <= 2 ? 1 : 2; }  // which of 1, 2, 4 tiles

}  // namespace

size_t gated_ff_workspace(const pipad_gated_ff_t &c, int32_t n, int32_t k, bool backward) { return Plan(c, n, k, backward).total; }

int gated_ff_launch(const pipad_gated_ff_t &c, int32_t n, int32_t k, const float *const *X, int64_t ldx, float *const *Y, int64_t ldy,
                    void *workspace, hipStream_t st) {
  const Plan p(c, n, k, false);
  char *const ws = static_cast<char *>(workspace);
  const int rc = pack(c, p, ws, st);
  if (rc != PIPAD_OK) return rc;
  const FfArgs a = arguments(c, p, n, k, X, ldx, nullptr, 0, Y, ldy, ws);
  if (c.F <= kKept && c.Fo <= kKept) {
    const Kept f = kept(c.activation, p.fq, p.ot);
    hipLaunchKernelGGL(f.kernel, dim3((unsigned)tiles(p.rows, kTile * f.waves)), dim3(f.waves * kWave), 0, st, a);
    PIPAD_HIP(hipGetLastError());
    return PIPAD_OK;
  }
  const int w = width(p.ot);
  hipLaunchKernelGGL(k_ff_rows_of[c.activation][w], dim3((unsigned)tiles(p.rows, kTile * kWavesPerBlock), (unsigned)tiles(p.ot, 1 << w)),
                     dim3(kBlock), 0, st, a);
  PIPAD_HIP(hipGetLastError());
  return PIPAD_OK;
}

int gated_ff_backward_launch(const pipad_gated_ff_t &c, int32_t n, int32_t k, const float *const *X, int64_t ldx, const float *const *dY,
                             int64_t lddy, float *const *dX, int64_t lddx, const pipad_gated_ff_grads_t *grads, void *workspace, hipStream_t st) {
  const Plan p(c, n, k, true);
  char *const ws = static_cast<char *>(workspace);
  if (p.rows > 0) {
    const int rc = pack(c, p, ws, st);
    if (rc != PIPAD_OK) return rc;
    const FfArgs a = arguments(c, p, n, k, X, ldx, dY, lddy, dX, lddx, ws);
    if (dX) {
      const int w = width(p.ft);
      hipLaunchKernelGGL(k_ff_rows_backward_of[c.activation][w],
                         dim3((unsigned)tiles(p.rows, kTile * kWavesPerBlock), (unsigned)tiles(p.ft, 1 << w)), dim3(kBlock), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    }
    if (grads) {
      const int most = std::max(p.ft, p.ot), w = width(most);
      hipLaunchKernelGGL(k_ff_weights_backward_of[c.activation][w],
                         dim3((unsigned)tiles(p.ht, kWavesPerBlock), (unsigned)p.parts, (unsigned)tiles(most, 1 << w)), dim3(kBlock), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    }
  }
  if (grads) {
    const SumArgs s{reinterpret_cast<const float *>(ws + p.partial), p.part_floats, (int32_t)p.parts, c.F, c.hidden, c.Fo, *grads};
    hipLaunchKernelGGL(k_ff_sums, dim3((unsigned)tiles(p.part_floats, kWave)), dim3(kBlock), 0, st, s);
    PIPAD_HIP(hipGetLastError());
  }
  return PIPAD_OK;
}

}  // namespace pipad
