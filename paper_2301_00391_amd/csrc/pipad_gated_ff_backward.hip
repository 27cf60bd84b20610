// The gated feed-forward block, the gradient of X, on rows of up to 256 columns.
//
// 1.6 million rows of 64 through 256: 0.95 ms (277 TFLOP/s of its five products), the matrix instructions 44 % and the vector ones 66 % of
// the cycles.  More than 64 columns leave one wave a SIMD, which waits for its own instructions: 312 thousand rows of 128 through 341, 0.67 ms, 28 %
// and 38 %.
#include "pipad_gated_ff.h"

namespace pipad {
namespace ff {

namespace {

// As the forward kernel: X's and dY's pieces stay in registers; the phases of a hidden tile are [Wg, Wu, vectors, Wd] and [Wg, Wu] laid out for
// the way back.  Of more than 128 columns of X a workgroup makes the gradient of 128, and another G, U and dH once more for the rest.
template <int ACT, int FQ, int OQ, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, FQ + OQ <= 8 ? 2 : 1) k_ff_kept_backward(FfArgs a) {
  constexpr int kAll = FQ <= 2 ? 1 : FQ / 2, FT = kAll < 4 ? kAll : 4;
  constexpr int kGu = gu_words(FQ), kUp = OQ * kFragment, kBack = FT * 4 * kFragment;
  const int f0 = kAll > FT ? blockIdx.y * FT : 0;
  __shared__ u32x4 in[kGu + kUp], back[kBack];
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5;
  const int64_t base = ((int64_t)blockIdx.x * WAVES + threadIdx.x / kWave) * kTile;
  stage<WAVES, kGu>(a.gu, in);
  stage<WAVES, kUp>(a.up, in + kGu);
  const RowAt at = row_at(a, base < a.rows ? base : a.rows - 1, m);
  Split x[FQ], dy[OQ];
  const float inv_x = load_row(x, a.X[at.t] + at.i * a.ldx, g, a.F, a.vec_x);
  const float inv_dy = load_row(dy, a.dY[at.t] + at.i * a.lddy, g, a.Fo, a.vec_dy);
  f32x16 dx[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) dx[f] = zeros();
  for (int h = 0; h < a.ht; ++h) {
    staged();
    stage<WAVES, kBack>(a.back + ((int64_t)h * kAll + f0) * 4 * kFragment, back);
    Sums sg = no_sums(), su = no_sums();
#pragma unroll
    for (int q = 0; q < FQ; ++q) {
      add_product(sg, fragment(in, 2 * q), x[q]);
      add_product(su, fragment(in, 2 * q + 1), x[q]);
    }
    const TileVectors &v = vectors_of(in, FQ);
    f32x16 G = value_of(sg, inv_x, v.inv_g, v.bg, g), U = value_of(su, inv_x, v.inv_u, v.bu, g);
    Sums sd = no_sums();
#pragma unroll
    for (int q = 0; q < OQ; ++q) add_product(sd, fragment(in + kGu, q), dy[q]);
    const f32x16 dH = value_of(sd, inv_dy, v.inv_d, g);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float2 c = activate_slope<ACT>(G[r]);
      G[r] = dH[r] * U[r] * c.y;
      U[r] = dH[r] * c.x;
    }
    const Scale scale = scale_for(max_over_32(largest_of(U, largest_of(G))));
    const Split dg[2] = {half(G, 0, scale.to), half(G, 1, scale.to)}, du[2] = {half(U, 0, scale.to), half(U, 1, scale.to)};
    staged();
    if (h + 1 < a.ht) {
      stage<WAVES, kGu>(a.gu + (int64_t)(h + 1) * kGu, in);
      stage<WAVES, kUp>(a.up + (int64_t)(h + 1) * kUp, in + kGu);
    }
#pragma unroll
    for (int f = 0; f < FT; ++f) {
      Sums sum = no_sums();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        add_product(sum, fragment(back, (f * 2 + s) * 2), dg[s]);
        add_product(sum, fragment(back, (f * 2 + s) * 2 + 1), du[s]);
      }
      add(dx[f], scale.inv * kToOne, sum);
    }
  }
  if (base + m >= a.rows) return;
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int f = 0; f < FT; ++f) store_tile(unscaled(dx[f], a.inv_out + (f0 + f) * kTile, nullptr, g), out, (f0 + f) * kTile, a.F, a.vec_o, g);
}

template <int ACT, int FQ>
Kept kept_backward_of(int oq) {
  switch (oq) {
    case 1: return {k_ff_kept_backward<ACT, FQ, 1, 4>, 4};
    case 2: return {k_ff_kept_backward<ACT, FQ, 2, 4>, 4};
    case 4: return {k_ff_kept_backward<ACT, FQ, 4, 4>, 4};
    case 8: return {k_ff_kept_backward<ACT, FQ, 8, 4>, 4};
    default: return {k_ff_kept_backward<ACT, FQ, 16, 4>, 4};
  }
}
template <int ACT>
Kept kept_backward_of(int fq, int oq) {
  return fq == 1 ? kept_backward_of<ACT, 1>(oq) : fq == 2 ? kept_backward_of<ACT, 2>(oq) : fq == 4 ? kept_backward_of<ACT, 4>(oq) : fq == 8 ? kept_backward_of<ACT, 8>(oq) : kept_backward_of<ACT, 16>(oq);
}
}  // namespace

// (a source of its own for each activation: a quarter of the kernels each, compiled side by side)
template <>
Kept kept_backward<PIPAD_FF_ACT>(int fq, int oq) {
  return kept_backward_of<PIPAD_FF_ACT>(fq, oq);
}

}  // namespace ff
}  // namespace pipad
