// The gated feed-forward block, the gradient of X, on rows of up to 128 columns.
#include "pipad_gated_ff.h"

namespace pipad {
namespace ff {

namespace {

// The same where rows are 128 columns at most (see k_ff_kept): X's and dY's pieces stay in registers; the phases of a hidden tile are
// [Wg, Wu, biases, Wd] and [Wg, Wu] laid out for the way back.
template <int ACT, int FQ, int OQ, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, FQ + OQ <= 8 ? 2 : 1) k_ff_kept_backward(FfArgs a) {
  constexpr int FT = FQ <= 2 ? 1 : FQ / 2;
  constexpr int kGu = gu_words(FQ), kUp = OQ * kFragment, kBack = FT * 4 * kFragment;
  __shared__ u32x4 in[kGu + kUp], back[kBack];
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5;
  const int64_t base = ((int64_t)blockIdx.x * WAVES + threadIdx.x / kWave) * kTile;
  stage<WAVES, kGu>(a.gu, in);
  stage<WAVES, kUp>(a.up, in + kGu);
  const RowAt at = row_at(a, base < a.rows ? base : a.rows - 1, m);
  Split x[FQ], dy[OQ];
  {
    const float *const row = a.X[at.t] + at.i * a.ldx;
    float v[FQ][8];
#pragma unroll
    for (int q = 0; q < FQ; ++q) load8(v[q], row, q * kDepth + 8 * g, a.F, a.vec_x);
#pragma unroll
    for (int q = 0; q < FQ; ++q) x[q] = split8(v[q]);
  }
  {
    const float *const row = a.dY[at.t] + at.i * a.lddy;
    float v[OQ][8];
#pragma unroll
    for (int q = 0; q < OQ; ++q) load8(v[q], row, q * kDepth + 8 * g, a.Fo, a.vec_dy);
#pragma unroll
    for (int q = 0; q < OQ; ++q) dy[q] = split8(v[q]);
  }
  f32x16 dx[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) dx[f] = zeros();
  const float *const bias = reinterpret_cast<const float *>(in + FQ * 2 * kFragment);
  for (int h = 0; h < a.ht; ++h) {
    staged();
    stage<WAVES, kBack>(a.back + (int64_t)h * kBack, back);
    f32x16 G = per_row(bias, g), U = per_row(bias + kTile, g), dH = zeros();
#pragma unroll
    for (int q = 0; q < FQ; ++q) {
      G = product(fragment(in, 2 * q), x[q], G);
      U = product(fragment(in, 2 * q + 1), x[q], U);
    }
#pragma unroll
    for (int q = 0; q < OQ; ++q) dH = product(fragment(in + kGu, q), dy[q], dH);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float2 c = activate_slope<ACT>(G[r]);
      G[r] = dH[r] * U[r] * c.y;
      U[r] = dH[r] * c.x;
    }
    staged();
    if (h + 1 < a.ht) {
      stage<WAVES, kGu>(a.gu + (int64_t)(h + 1) * kGu, in);
      stage<WAVES, kUp>(a.up + (int64_t)(h + 1) * kUp, in + kGu);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const Split dg = half(G, s), du = half(U, s);
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        dx[f] = product(fragment(back, (f * 2 + s) * 2), dg, dx[f]);
        dx[f] = product(fragment(back, (f * 2 + s) * 2 + 1), du, dx[f]);
      }
    }
  }
  if (base + m >= a.rows) return;
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int f = 0; f < FT; ++f) store_tile(dx[f], out, f * kTile, a.F, a.vec_o, g);
}

template <int ACT, int FQ>
Kept kept_backward_of(int oq) {
  switch (oq) {
    case 1: return {k_ff_kept_backward<ACT, FQ, 1, 4>, 4};
    case 2: return {k_ff_kept_backward<ACT, FQ, 2, 4>, 4};
    case 4: return {k_ff_kept_backward<ACT, FQ, 4, 4>, 4};
    default: return {k_ff_kept_backward<ACT, FQ, 8, 4>, 4};
  }
}
template <int ACT>
Kept kept_backward_of(int fq, int oq) {
  return fq == 1 ? kept_backward_of<ACT, 1>(oq) : fq == 2 ? kept_backward_of<ACT, 2>(oq) : fq == 4 ? kept_backward_of<ACT, 4>(oq) : kept_backward_of<ACT, 8>(oq);
}
}  // namespace

Kept kept_backward(int act, int fq, int oq) {
  switch (act) {
    case PIPAD_ACT_SIGMOID: return kept_backward_of<PIPAD_ACT_SIGMOID>(fq, oq);
    case PIPAD_ACT_RELU: return kept_backward_of<PIPAD_ACT_RELU>(fq, oq);
    case PIPAD_ACT_GELU: return kept_backward_of<PIPAD_ACT_GELU>(fq, oq);
    default: return kept_backward_of<PIPAD_ACT_SILU>(fq, oq);
  }
}

}  // namespace ff
}  // namespace pipad
