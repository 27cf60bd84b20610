// The gated feed-forward block, forward and the gradient of X, on few rows.  A wave for 32 rows, as in the kernels for many, goes through all
// hidden tiles alone, and what it takes is the latency of its chain of loads and products, however few rows there are.  Here eight waves have
// the same 32 rows and every eighth hidden tile each, and their results are added up in LDS, always in the same order.  The rows' pieces lie
// in LDS, where every wave needs them; a tile's weights are read by one wave only and come straight from the caches.  At 4096 rows of 64
// columns through 256 that is 13.7 us instead of 20.5 (the gradient 20.0 instead of 30.5), of which packing the weights takes 5 to 7.
#include "pipad_gated_ff.h"

namespace pipad {
namespace ff {

namespace {

constexpr int kWaves = 8, kMostDepth = 16;  // tiles of 16 columns that a row has at most

// Rows base .. base + 31 as pieces; returns 1 over the scale of the lane's row.  The waves have a tile of 16 columns each, of more than 8
// tiles two.
__device__ inline float share_rows(u32x4 *to, float (&largest)[kWaves][kTile], const float *row, int tiles_, int F, bool vec) {
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  float v[2][8], x = 0.f;
#pragma unroll
  for (int s = 0; s < 2; ++s)
    if (wave + s * kWaves < tiles_) {
      load8(v[s], row, (wave + s * kWaves) * kDepth + 8 * g, F, vec);
      x = largest_of(v[s], x);
    }
  x = max_over_32(x);
  if (g == 0) largest[wave][m] = x;
  __syncthreads();
  x = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x = fmaxf(x, largest[w][m]);
  const Scale scale = scale_for(x);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int q = wave + s * kWaves;
    if (q < tiles_) {
      const Split p = split8(v[s], scale.to);
      to[q * kFragment + lane] = p.p[0], to[q * kFragment + kWave + lane] = p.p[1];
    }
  }
  return scale.inv;
}

// Columns c0 .. c0 + 31 of the rows: the waves' results added up, times 1 over the columns' scales, and a vector; the first four waves store 8
// columns each.
__device__ inline void store_sum(float (&part)[kWaves][16][kWave], const f32x16 &mine, const float *inv, const float *bias, float *row, bool there, int c0, int F, bool vec) {
  const int lane = threadIdx.x & (kWave - 1), g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
  for (int r = 0; r < 16; ++r) part[wave][r][lane] = mine[r];
  __syncthreads();
  if (wave < 4 && there) {
    const int c = c0 + 8 * wave + 4 * g;
    float s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s[e] += part[w][4 * wave + e][lane];
      s[e] = fmaf(s[e], inv[c + e], bias ? bias[c + e] : 0.f);
    }
    if (vec && c + 4 <= F) {
      *reinterpret_cast<float4 *>(row + c) = make_float4(s[0], s[1], s[2], s[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < F) row[c + e] = s[e];
    }
  }
  __syncthreads();
}

template <int ACT, int OT>
__global__ void __launch_bounds__(kWaves *kWave, 2) k_ff_split(FfArgs a) {
  __shared__ u32x4 xs[kMostDepth * kFragment];
  __shared__ float part[kWaves][16][kWave], largest[kWaves][kTile];
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t base = (int64_t)blockIdx.x * kTile;
  const RowAt at = row_at(a, base, m);
  const float inv_x = share_rows(xs, largest, a.X[at.t] + at.i * a.ldx, a.fq, a.F, a.vec_x);
  __syncthreads();
  f32x16 y[OT];
#pragma unroll
  for (int o = 0; o < OT; ++o) y[o] = zeros();
  for (int h = wave; h < a.ht; h += kWaves) {
    const u32x4 *const gu = a.gu + (int64_t)h * gu_words(a.fq), *const down = a.down + (int64_t)h * a.ot * 2 * kFragment;
    const TileVectors &v = vectors_of(gu, a.fq);
    Sums sg = no_sums(), su = no_sums();
#pragma unroll 4
    for (int q = 0; q < a.fq; ++q) {
      const Split x = fragment(xs, q);
      add_product(sg, fragment(gu, 2 * q), x);
      add_product(su, fragment(gu, 2 * q + 1), x);
    }
    f32x16 G = value_of(sg, inv_x, v.inv_g, v.bg, g);
    const f32x16 U = value_of(su, inv_x, v.inv_u, v.bu, g);
#pragma unroll
    for (int r = 0; r < 16; ++r) G[r] = activate<ACT>(G[r]) * U[r];
    const Scale scale = scale_for(max_over_32(largest_of(G)));
    const Split b[2] = {half(G, 0, scale.to), half(G, 1, scale.to)};
#pragma unroll
    for (int o = 0; o < OT; ++o) {
      Sums sum = no_sums();
#pragma unroll
      for (int s = 0; s < 2; ++s) add_product(sum, fragment(down, 2 * o + s), b[s]);
      add(y[o], scale.inv * kToOne, sum);
    }
  }
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int o = 0; o < OT; ++o) store_sum(part, y[o], a.inv_out, a.bd, out, base + m < a.rows, o * kTile, a.Fo, a.vec_o);
}

// FT tiles of X's columns from tile blockIdx.y * FT on.
template <int ACT, int FT>
__global__ void __launch_bounds__(kWaves *kWave, 2) k_ff_split_backward(FfArgs a) {
  __shared__ u32x4 xs[kMostDepth * kFragment], dys[kMostDepth * kFragment];
  __shared__ float part[kWaves][16][kWave], largest[2][kWaves][kTile];
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t base = (int64_t)blockIdx.x * kTile;
  const int f0 = blockIdx.y * FT;
  const RowAt at = row_at(a, base, m);
  const float inv_x = share_rows(xs, largest[0], a.X[at.t] + at.i * a.ldx, a.fq, a.F, a.vec_x);
  const float inv_dy = share_rows(dys, largest[1], a.dY[at.t] + at.i * a.lddy, a.oq, a.Fo, a.vec_dy);
  __syncthreads();
  f32x16 dx[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) dx[f] = zeros();
  for (int h = wave; h < a.ht; h += kWaves) {
    const u32x4 *const gu = a.gu + (int64_t)h * gu_words(a.fq), *const up = a.up + (int64_t)h * a.oq * kFragment;
    const u32x4 *const back = a.back + ((int64_t)h * a.ft + f0) * 4 * kFragment;
    const TileVectors &v = vectors_of(gu, a.fq);
    Sums sg = no_sums(), su = no_sums();
#pragma unroll 4
    for (int q = 0; q < a.fq; ++q) {
      const Split x = fragment(xs, q);
      add_product(sg, fragment(gu, 2 * q), x);
      add_product(su, fragment(gu, 2 * q + 1), x);
    }
    f32x16 G = value_of(sg, inv_x, v.inv_g, v.bg, g), U = value_of(su, inv_x, v.inv_u, v.bu, g);
    Sums sd = no_sums();
#pragma unroll 4
    for (int q = 0; q < a.oq; ++q) add_product(sd, fragment(up, q), fragment(dys, q));
    const f32x16 dH = value_of(sd, inv_dy, v.inv_d, g);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float2 c = activate_slope<ACT>(G[r]);
      G[r] = dH[r] * U[r] * c.y;
      U[r] = dH[r] * c.x;
    }
    const Scale scale = scale_for(max_over_32(largest_of(U, largest_of(G))));
    const Split dg[2] = {half(G, 0, scale.to), half(G, 1, scale.to)}, du[2] = {half(U, 0, scale.to), half(U, 1, scale.to)};
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
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int f = 0; f < FT; ++f) store_sum(part, dx[f], a.inv_out, nullptr, out, base + m < a.rows, (f0 + f) * kTile, a.F, a.vec_o);
}

template <int ACT>
Kept split_of(int ot) {
  return {ot == 1 ? k_ff_split<ACT, 1> : ot == 2 ? k_ff_split<ACT, 2> : ot == 4 ? k_ff_split<ACT, 4> : k_ff_split<ACT, 8>, kWaves};
}
template <int ACT>
Kept split_backward_of(int ft) {
  return {ft == 1 ? k_ff_split_backward<ACT, 1> : ft == 2 ? k_ff_split_backward<ACT, 2> : k_ff_split_backward<ACT, 4>, kWaves};
}
}  // namespace

Kept split_forward(int act, int ot) {
  switch (act) {
    case PIPAD_ACT_SIGMOID: return split_of<PIPAD_ACT_SIGMOID>(ot);
    case PIPAD_ACT_RELU: return split_of<PIPAD_ACT_RELU>(ot);
    case PIPAD_ACT_GELU: return split_of<PIPAD_ACT_GELU>(ot);
    default: return split_of<PIPAD_ACT_SILU>(ot);
  }
}
Kept split_backward(int act, int ft) {
  switch (act) {
    case PIPAD_ACT_SIGMOID: return split_backward_of<PIPAD_ACT_SIGMOID>(ft);
    case PIPAD_ACT_RELU: return split_backward_of<PIPAD_ACT_RELU>(ft);
    case PIPAD_ACT_GELU: return split_backward_of<PIPAD_ACT_GELU>(ft);
    default: return split_backward_of<PIPAD_ACT_SILU>(ft);
  }
}

}  // namespace ff
}  // namespace pipad
