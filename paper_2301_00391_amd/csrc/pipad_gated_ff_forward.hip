// The gated feed-forward block, forward, on rows of up to 256 columns.
//
// Bound by issue and power: activations, scales and pieces of H are 87 % of the cycles in vector instructions (1.6 million rows of 64 through 256 with
// gelu), the matrix instructions 40 % beside them, at 1.8 GHz.  That takes 650 us, 242 TFLOP/s of the block's own products; 8 million rows of 64
// through 171 with silu, 77 % and 45 % at 1.6 GHz, 2.21 ms, 238 TFLOP/s and 1.9 TB/s.
#include "pipad_gated_ff.h"

namespace pipad {
namespace ff {

namespace {

// X's pieces stay in registers, and the waves of a workgroup, 32 node rows each, share the weights through LDS.  A hidden tile's weights come in
// two phases, [Wg, Wu, vectors] and [Wd], each into a buffer of its own while the other is multiplied: loaded past the registers, one
// barrier a phase.
template <int ACT, int FQ, int OT, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, FQ + 2 * OT <= 16 ? 2 : 1) k_ff_kept(FfArgs a) {
  constexpr int kGu = gu_words(FQ), kDown = OT * 2 * kFragment;
  __shared__ u32x4 gu[kGu], down[kDown];  // (two arrays: what is read of one does not wait for what is loaded into the other)
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5;
  const int64_t base = ((int64_t)blockIdx.x * WAVES + threadIdx.x / kWave) * kTile;
  stage<WAVES, kGu>(a.gu, gu);
  const RowAt at = row_at(a, base < a.rows ? base : a.rows - 1, m);
  Split x[FQ];
  const float inv_x = load_row(x, a.X[at.t] + at.i * a.ldx, g, a.F, a.vec_x);
  f32x16 y[OT];
#pragma unroll
  for (int o = 0; o < OT; ++o) y[o] = zeros();
  for (int h = 0; h < a.ht; ++h) {
    staged();
    stage<WAVES, kDown>(a.down + (int64_t)h * kDown, down);
    Sums sg = no_sums(), su = no_sums();
#pragma unroll
    for (int q = 0; q < FQ; ++q) {
      add_product(sg, fragment(gu, 2 * q), x[q]);
      add_product(su, fragment(gu, 2 * q + 1), x[q]);
    }
    const TileVectors &v = vectors_of(gu, FQ);
    f32x16 G = value_of(sg, inv_x, v.inv_g, v.bg, g);
    const f32x16 U = value_of(su, inv_x, v.inv_u, v.bu, g);
#pragma unroll
    for (int r = 0; r < 16; ++r) G[r] = activate<ACT>(G[r]) * U[r];
    const Scale scale = scale_for(max_over_32(largest_of(G)));
    const Split b[2] = {half(G, 0, scale.to), half(G, 1, scale.to)};
    staged();
    if (h + 1 < a.ht) stage<WAVES, kGu>(a.gu + (int64_t)(h + 1) * kGu, gu);
#pragma unroll
    for (int o = 0; o < OT; ++o) {
      Sums sum = no_sums();
#pragma unroll
      for (int s = 0; s < 2; ++s) add_product(sum, fragment(down, 2 * o + s), b[s]);
      add(y[o], scale.inv * kToOne, sum);
    }
  }
  if (base + m >= a.rows) return;
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int o = 0; o < OT; ++o) store_tile(unscaled(y[o], a.inv_out + o * kTile, a.bd + o * kTile, g), out, o * kTile, a.Fo, a.vec_o, g);
}

template <int ACT, int FQ, int OT>
Kept kept_of() {
  // two workgroups a compute unit, or where LDS holds one, twice the waves; above 256 registers a wave it is four again
  constexpr int kWaves = (FQ <= 4 && OT <= 2) || FQ + 2 * OT > 16 ? 4 : 8;
  return {k_ff_kept<ACT, FQ, OT, kWaves>, kWaves};
}
template <int ACT, int FQ>
Kept kept_of(int ot) {
  return ot == 1 ? kept_of<ACT, FQ, 1>() : ot == 2 ? kept_of<ACT, FQ, 2>() : ot == 4 ? kept_of<ACT, FQ, 4>() : kept_of<ACT, FQ, 8>();
}
template <int ACT>
Kept kept_of(int fq, int ot) {
  switch (fq) {
    case 1: return kept_of<ACT, 1>(ot);
    case 2: return kept_of<ACT, 2>(ot);
    case 4: return kept_of<ACT, 4>(ot);
    case 6: return kept_of<ACT, 6>(ot);
    case 8: return kept_of<ACT, 8>(ot);
    default: return kept_of<ACT, 16>(ot);
  }
}
}  // namespace

// (a source of its own for each activation: a quarter of the kernels each, compiled side by side)
template <>
Kept kept_forward<PIPAD_FF_ACT>(int fq, int ot) {
  return kept_of<PIPAD_FF_ACT>(fq, ot);
}

}  // namespace ff
}  // namespace pipad
