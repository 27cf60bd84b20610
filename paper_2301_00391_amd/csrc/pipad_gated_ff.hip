// The gated feed-forward block: weights as fragments, the kernels for rows of any width, and the host side.  How the products are
// made stands in pipad_gated_ff.h; rows of up to 256 columns have kernels of their own in pipad_gated_ff_forward.hip, _backward.hip, _weights.hip
// and, for few rows, _split.hip.  The kernels here for wider ones hold no row, but read it again for every hidden tile, and the waves of a workgroup make
// a tile of H (dG and dU) each for all of them; of more than 512 columns another workgroup makes them again.  65536 rows of 512 through 2048: 2.4 ms
// forward and 3.9 the gradient of X, where three and five products of float matrices take 2.7 and 4.5 and write H in between; 29 the gradients of the
// weights, where six take 5.4: a column of X is loaded and split again for every hidden tile.
#include "pipad_gated_ff.h"

namespace pipad {
using namespace ff;

namespace {

// ---- weights as fragments -----------------------------------------------------------------------
struct PackArgs {
  const float *Wg, *Wu, *Wd, *bg, *bu, *bd;
  int64_t ldwg, ldwu, ldwd;
  int32_t F, hidden, Fo, ht, fq, oq, ft, ot;
  u32x4 *gu, *down, *up, *back;  // (all but gu: null where they are not wanted)
  float *inv_out, *pbd;          // (pbd with down only)
  int32_t tiles;                 // hidden tiles that a workgroup has of down or back
};
// A workgroup a hidden tile (gu, up) or, behind these, some hidden tiles of 32 columns of Y (down) or X (back): the largest of each column, then a
// wave a fragment.  What a fragment's m is has a scale of its own, the lane's.
constexpr int kPackWaves = 16;

// Largest of the columns c0 .. c0 + 31 of N matrices, column m in lanes m and m + 32, of this wave's rows.
template <int N>
__device__ inline void largest_of_columns(float (&x)[N], const float *const (&W)[N], const int64_t (&ld)[N], int rows, int c, bool there, int wave, int g) {
#pragma unroll
  for (int q = 0; q < N; ++q) x[q] = 0.f;
  if (there) {
#pragma unroll 4
    for (int r = 2 * wave + g; r < rows; r += 2 * kPackWaves)
#pragma unroll
      for (int q = 0; q < N; ++q) x[q] = max_of(x[q], W[q][r * ld[q] + c]);
  }
#pragma unroll
  for (int q = 0; q < N; ++q) x[q] = max_over_32(x[q]);
}
// Largest of rows `wave` and `wave` + 16 of 32 in N matrices together; behind the last row the last one's (no branch: all loads are on the way at once).
template <int N>
__device__ inline void largest_of_rows(float (&to)[kTile], const float *const (&W)[N], const int64_t (&ld)[N], int first, int rows, int columns, int lane, int wave) {
  float x[2] = {0.f, 0.f};
  const int64_t r[2] = {min(first + wave, rows - 1), min(first + wave + kPackWaves, rows - 1)};
#pragma unroll 4
  for (int c = lane; c < columns; c += kWave)
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int q = 0; q < N; ++q) x[s] = max_of(x[s], W[q][r[s] * ld[q] + c]);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    x[s] = max_of_wave(x[s]);
    if (lane == 0) to[wave + s * kPackWaves] = x[s];
  }
}

// The scales of m's column, of what the waves have found.
__device__ inline Scale scale_of(const float (&found)[kPackWaves][kTile], int m) {
  float x = 0.f;
#pragma unroll
  for (int w = 0; w < kPackWaves; ++w) x = fmaxf(x, found[w][m]);
  return scale_for(x);
}

__device__ inline void pack_hidden(const PackArgs &a, int h, float (&found)[2][kPackWaves][kTile], float (&rows)[kTile]) {
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h0 = h * kTile;
  const bool there = h0 + m < a.hidden;
  float largest[2];
  largest_of_columns<2>(largest, {a.Wg, a.Wu}, {a.ldwg, a.ldwu}, a.F, h0 + m, there, wave, g);
  if (g == 0) found[0][wave][m] = largest[0], found[1][wave][m] = largest[1];
  if (a.up) largest_of_rows<1>(rows, {a.Wd}, {a.ldwd}, h0, a.hidden, a.Fo, lane, wave);
  __syncthreads();
  const Scale scale_g = scale_of(found[0], m), scale_u = scale_of(found[1], m), scale_d = scale_for(a.up ? rows[m] : 0.f);
  u32x4 *const tile = a.gu + (int64_t)h * gu_words(a.fq);
  if (threadIdx.x < kTile) {
    TileVectors &t = *reinterpret_cast<TileVectors *>(tile + a.fq * 2 * kFragment);
    t.bg[m] = a.bg && there ? a.bg[h0 + m] : 0.f;
    t.bu[m] = a.bu && there ? a.bu[h0 + m] : 0.f;
    t.inv_g[m] = scale_g.inv, t.inv_u[m] = scale_u.inv, t.inv_d[m] = scale_d.inv;
  }
  const int n_gu = 2 * a.fq, n_up = a.up ? a.oq : 0;
  for (int at = wave; at < n_gu + n_up; at += kPackWaves) {
    float v[8];
    Split s;
    u32x4 *to;
    if (at < n_gu) {  // [fq][Wg, Wu]
      const float *W = at % 2 ? a.Wu : a.Wg;
      const int64_t ld = at % 2 ? a.ldwu : a.ldwg;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int f = at / 2 * kDepth + 8 * g + j;
        v[j] = f < a.F && there ? W[f * ld + h0 + m] : 0.f;
      }
      s = split8(v, at % 2 ? scale_u.to : scale_g.to);
      to = tile + at * kFragment;
    } else {  // [oq]
      load8(v, a.Wd + (there ? h0 + m : 0) * a.ldwd, (at - n_gu) * kDepth + 8 * g, there ? a.Fo : 0, false);
      s = split8(v, scale_d.to);
      to = a.up + ((int64_t)h * n_up + at - n_gu) * kFragment;
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) to[p * kWave + lane] = s.p[p];
  }
}

__device__ inline void pack_down(const PackArgs &a, int o, int first, float (&found)[kPackWaves][kTile]) {
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = o * kTile + m;
  const bool there = c < a.Fo;
  float largest[1];
  largest_of_columns<1>(largest, {a.Wd}, {a.ldwd}, a.hidden, c, there, wave, g);
  if (g == 0) found[wave][m] = largest[0];
  __syncthreads();
  const Scale scale = scale_of(found, m);
  if (first == 0 && threadIdx.x < kTile) a.inv_out[c] = scale.inv / kToOne, a.pbd[c] = a.bd && there ? a.bd[c] : 0.f;
  const int count = 2 * min(a.ht - first, a.tiles);
  for (int at = wave; at < count; at += kPackWaves) {  // [2]
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int hid = (first + at / 2) * kTile + result_depth(at % 2, g, j);
      v[j] = hid < a.hidden && there ? a.Wd[hid * a.ldwd + c] : 0.f;
    }
    const Split s = split8(v, scale.to);
    u32x4 *const to = a.down + (((int64_t)(first + at / 2) * a.ot + o) * 2 + at % 2) * kFragment;
#pragma unroll
    for (int p = 0; p < 2; ++p) to[p * kWave + lane] = s.p[p];
  }
}

__device__ inline void pack_back(const PackArgs &a, int t, int first, float (&rows)[kTile]) {
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int f = t * kTile + m;
  largest_of_rows<2>(rows, {a.Wg, a.Wu}, {a.ldwg, a.ldwu}, t * kTile, a.F, a.hidden, lane, wave);
  __syncthreads();
  const Scale scale = scale_for(rows[m]);
  if (first == 0 && threadIdx.x < kTile) a.inv_out[f] = scale.inv / kToOne;
  const int count = 4 * min(a.ht - first, a.tiles);
  for (int at = wave; at < count; at += kPackWaves) {  // [2][Wg, Wu]
    const float *W = at % 2 ? a.Wu : a.Wg;
    const int64_t ld = at % 2 ? a.ldwu : a.ldwg;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int hid = (first + at / 4) * kTile + result_depth(at / 2 % 2, g, j);
      v[j] = hid < a.hidden && f < a.F ? W[f * ld + hid] : 0.f;
    }
    const Split s = split8(v, scale.to);
    u32x4 *const to = a.back + (((int64_t)(first + at / 4) * a.ft + t) * 4 + at % 4) * kFragment;
#pragma unroll
    for (int p = 0; p < 2; ++p) to[p * kWave + lane] = s.p[p];
  }
}

__global__ void __launch_bounds__(kPackWaves *kWave) k_ff_pack(PackArgs a) {
  __shared__ float found[2][kPackWaves][kTile], rows[kTile];
  const int b = (int)blockIdx.x - a.ht;
  if (b < 0) return pack_hidden(a, blockIdx.x, found, rows);
  if (a.down) return pack_down(a, b % a.ot, b / a.ot * a.tiles, found[0]);
  pack_back(a, b % a.ft, b / a.ft * a.tiles, rows);
}

// ---- forward ------------------------------------------------------------------------------------
// Scale of a row of any width, of which lane m + 32 has the other half of every 16 columns.
__device__ inline Scale scale_of_row(const float *row, int F, int g, bool vec) {
  float largest = 0.f, v[8];
  for (int c = 8 * g; c < F; c += kDepth) {
    load8(v, row, c, F, vec);
    largest = largest_of(v, largest);
  }
  return scale_for(max_over_32(largest));
}

// A workgroup: 32 node rows, OT tiles of Y's columns a wave.  The waves make a tile of H each, lay its pieces in LDS (in two places by turns, for one
// barrier), and all multiply all of these, each into its own columns.  Results lie transposed (a node row is a lane's column).
template <int PIECES>
struct Shared {  // what a wave gives the others: operands of 16 deep, and a lane's factor
  u32x4 piece[2][kWavesPerBlock][PIECES * kFragment];
  float inv[2][kWavesPerBlock][kWave];
};
__device__ inline void lay(u32x4 *to, int index, const Split &s, int lane) {
  to[index * kFragment + lane] = s.p[0], to[index * kFragment + kWave + lane] = s.p[1];
}
template <int ACT, int OT>
__global__ void __launch_bounds__(kBlock, 2) k_ff_rows(FfArgs a) {
  __shared__ Shared<2> hs;
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t base = (int64_t)blockIdx.x * kTile;
  const RowAt at = row_at(a, base, m);
  const float *const x = a.X[at.t] + at.i * a.ldx;
  const Scale scale_x = scale_of_row(x, a.F, g, a.vec_x);
  const int o0 = (blockIdx.y * kWavesPerBlock + wave) * OT;
  f32x16 y[OT];
#pragma unroll
  for (int o = 0; o < OT; ++o) y[o] = zeros();
  for (int h0 = 0, turn = 0; h0 < a.ht; h0 += kWavesPerBlock, turn ^= 1) {
    if (h0 + wave < a.ht) {
      const u32x4 *const gu = a.gu + (int64_t)(h0 + wave) * gu_words(a.fq);
      const TileVectors &vectors = vectors_of(gu, a.fq);
      Sums sg = no_sums(), su = no_sums();
      for (int q = 0; q < a.fq; ++q) {
        float v[8];
        load8(v, x, q * kDepth + 8 * g, a.F, a.vec_x);
        const Split b = split8(v, scale_x.to);
        add_product(sg, fragment(gu, 2 * q), b);
        add_product(su, fragment(gu, 2 * q + 1), b);
      }
      f32x16 G = value_of(sg, scale_x.inv, vectors.inv_g, vectors.bg, g);
      const f32x16 U = value_of(su, scale_x.inv, vectors.inv_u, vectors.bu, g);
#pragma unroll
      for (int r = 0; r < 16; ++r) G[r] = activate<ACT>(G[r]) * U[r];
      const Scale scale = scale_for(max_over_32(largest_of(G)));
#pragma unroll
      for (int s = 0; s < 2; ++s) lay(hs.piece[turn][wave], s, half(G, s, scale.to), lane);
      hs.inv[turn][wave][lane] = scale.inv * kToOne;
    }
    __syncthreads();
    const int count = min(a.ht - h0, kWavesPerBlock);
    for (int w = 0; w < count; ++w) {
      const Split b[2] = {fragment(hs.piece[turn][w], 0), fragment(hs.piece[turn][w], 1)};
      const float inv = hs.inv[turn][w][lane];
#pragma unroll
      for (int o = 0; o < OT; ++o)
        if (o0 + o < a.ot) {
          const int64_t at_w = ((int64_t)(h0 + w) * a.ot + o0 + o) * 2;
          Sums sum = no_sums();
#pragma unroll
          for (int s = 0; s < 2; ++s) add_product(sum, fragment(a.down, at_w + s), b[s]);
          add(y[o], inv, sum);
        }
    }
  }
  if (base + m >= a.rows) return;
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int o = 0; o < OT; ++o)
    if (o0 + o < a.ot) store_tile(unscaled(y[o], a.inv_out + (o0 + o) * kTile, a.bd + (o0 + o) * kTile, g), out, (o0 + o) * kTile, a.Fo, a.vec_o, g);
}

// Few rows: a workgroup a row, in 32-bit floats, straight from the weights as they are.  What counts is the time from the first load to the last
// store: no launch for fragments, and every wave has its loads on the way at once.  Columns lie along the lanes; the sum over the rows
// of a matrix is shared by as many waves as there are left, and added up in LDS, always in the same order.  One row of 64 through 256: 8.0 us, of which a
// launch and two round trips to memory are most (13.8 with fragments and eight waves).
constexpr int kFewThreads = 1024, kFewWaves = kFewThreads / kWave, kFewColumns = 1024, kFewMostF = 2048, kFewMostFo = 8192;
template <int ACT>
__global__ void __launch_bounds__(kFewThreads) k_ff_few(FfArgs a) {
  __shared__ float x[kFewMostF], sum_g[kFewThreads], sum_u[kFewThreads], hidden[kFewColumns], sums[kFewMostFo];  // (sums: of more than kFewColumns hidden columns)
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const RowAt at = row_at(a, blockIdx.x, 0);
  const float *const row = a.X[at.t] + at.i * a.ldx;
  for (int f = threadIdx.x; f < a.F; f += kFewThreads) x[f] = row[f];
  float *const out = a.out[at.t] + at.i * a.ldo;
  __syncthreads();
  for (int h0 = 0; h0 < a.hidden; h0 += kFewColumns) {
    const int columns = min(a.hidden - h0, kFewColumns), blocks = (columns + kWave - 1) / kWave, groups = kFewWaves / blocks;
    {
      const int group = wave / blocks, c = wave % blocks * kWave + lane;
      float g = 0.f, u = 0.f;
      if (group < groups && c < columns) {
        const float *const wg = a.Wg + h0 + c, *const wu = a.Wu + h0 + c;
#pragma unroll 16
        for (int f = group; f < a.F; f += groups) {
          g = fmaf(x[f], wg[f * a.ldwg], g);
          u = fmaf(x[f], wu[f * a.ldwu], u);
        }
      }
      sum_g[threadIdx.x] = g, sum_u[threadIdx.x] = u;
    }
    __syncthreads();
    if (threadIdx.x < columns) {
      float g = a.bg ? a.bg[h0 + threadIdx.x] : 0.f, u = a.bu ? a.bu[h0 + threadIdx.x] : 0.f;
      for (int q = 0; q < groups; ++q) g += sum_g[q * blocks * kWave + threadIdx.x], u += sum_u[q * blocks * kWave + threadIdx.x];
      hidden[threadIdx.x] = activate<ACT>(g) * u;
    }
    __syncthreads();
    for (int o0 = 0; o0 < a.Fo; o0 += kFewColumns) {
      const int outs = min(a.Fo - o0, kFewColumns), oblocks = (outs + kWave - 1) / kWave, ogroups = kFewWaves / oblocks;
      const int group = wave / oblocks, c = wave % oblocks * kWave + lane;
      float y = 0.f;
      if (group < ogroups && c < outs) {
        const float *const wd = a.Wd + h0 * a.ldwd + o0 + c;
#pragma unroll 16
        for (int h = group; h < columns; h += ogroups) y = fmaf(hidden[h], wd[h * a.ldwd], y);
      }
      sum_g[threadIdx.x] = y;
      __syncthreads();
      if (threadIdx.x < outs) {
        const int o = o0 + threadIdx.x;
        float s = h0 ? sums[o] : a.bd_in ? a.bd_in[o] : 0.f;
        for (int q = 0; q < ogroups; ++q) s += sum_g[q * oblocks * kWave + threadIdx.x];
        if (h0 + kFewColumns < a.hidden) sums[o] = s;
        else out[o] = s;
      }
      __syncthreads();
    }
  }
}

// ---- the gradient of X --------------------------------------------------------------------------
// As k_ff_rows, with dG and dU in the place of H.
template <int ACT, int FT>
__global__ void __launch_bounds__(kBlock, 2) k_ff_rows_backward(FfArgs a) {
  __shared__ Shared<4> ds;
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t base = (int64_t)blockIdx.x * kTile;
  const RowAt at = row_at(a, base, m);
  const float *const x = a.X[at.t] + at.i * a.ldx, *const dy = a.dY[at.t] + at.i * a.lddy;
  const Scale scale_x = scale_of_row(x, a.F, g, a.vec_x), scale_dy = scale_of_row(dy, a.Fo, g, a.vec_dy);
  const int f0 = (blockIdx.y * kWavesPerBlock + wave) * FT;
  f32x16 dx[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) dx[f] = zeros();
  for (int h0 = 0, turn = 0; h0 < a.ht; h0 += kWavesPerBlock, turn ^= 1) {
    if (h0 + wave < a.ht) {
      const int h = h0 + wave;
      const u32x4 *const gu = a.gu + (int64_t)h * gu_words(a.fq);
      const TileVectors &vectors = vectors_of(gu, a.fq);
      Sums sg = no_sums(), su = no_sums(), sd = no_sums();
      float v[8];
      for (int q = 0; q < a.fq; ++q) {
        load8(v, x, q * kDepth + 8 * g, a.F, a.vec_x);
        const Split b = split8(v, scale_x.to);
        add_product(sg, fragment(gu, 2 * q), b);
        add_product(su, fragment(gu, 2 * q + 1), b);
      }
      for (int q = 0; q < a.oq; ++q) {
        load8(v, dy, q * kDepth + 8 * g, a.Fo, a.vec_dy);
        add_product(sd, fragment(a.up, (int64_t)h * a.oq + q), split8(v, scale_dy.to));
      }
      f32x16 G = value_of(sg, scale_x.inv, vectors.inv_g, vectors.bg, g), U = value_of(su, scale_x.inv, vectors.inv_u, vectors.bu, g);
      const f32x16 dH = value_of(sd, scale_dy.inv, vectors.inv_d, g);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float2 c = activate_slope<ACT>(G[r]);
        G[r] = dH[r] * U[r] * c.y;
        U[r] = dH[r] * c.x;
      }
      const Scale scale = scale_for(max_over_32(largest_of(U, largest_of(G))));
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        lay(ds.piece[turn][wave], s, half(G, s, scale.to), lane);
        lay(ds.piece[turn][wave], 2 + s, half(U, s, scale.to), lane);
      }
      ds.inv[turn][wave][lane] = scale.inv * kToOne;
    }
    __syncthreads();
    const int count = min(a.ht - h0, kWavesPerBlock);
    for (int w = 0; w < count; ++w) {
      Split dg[2], du[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) dg[s] = fragment(ds.piece[turn][w], s), du[s] = fragment(ds.piece[turn][w], 2 + s);
      const float inv = ds.inv[turn][w][lane];
#pragma unroll
      for (int f = 0; f < FT; ++f)
        if (f0 + f < a.ft) {
          Sums sum = no_sums();
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const int64_t at_w = (((int64_t)(h0 + w) * a.ft + f0 + f) * 2 + s) * 2;
            add_product(sum, fragment(a.back, at_w), dg[s]);
            add_product(sum, fragment(a.back, at_w + 1), du[s]);
          }
          add(dx[f], inv, sum);
        }
    }
  }
  if (base + m >= a.rows) return;
  float *const out = a.out[at.t] + at.i * a.ldo;
#pragma unroll
  for (int f = 0; f < FT; ++f)
    if (f0 + f < a.ft) store_tile(unscaled(dx[f], a.inv_out + (f0 + f) * kTile, nullptr, g), out, (f0 + f) * kTile, a.F, a.vec_o, g);
}

// ---- the gradients of the weights ---------------------------------------------------------------
// A workgroup: one tile of hidden columns, the rows of one part, T tiles of X's and of Y's columns a wave.  The waves make dG, dU and H of 32 rows each,
// lay their pieces in LDS, and all multiply all of these, each with its own columns of X and dY.  Results lie as they are (a hidden column is a
// lane's column), so dG, dU and H are operands of products whose depth is the node rows; X and dY keep their rows' scales there, by whose
// inverses dG, dU and H are multiplied before they get a scale of their own, a hidden column each.
template <int ACT, int T>
__global__ void __launch_bounds__(kBlock, 1) k_ff_weights_backward(FfArgs a) {
  __shared__ Shared<6> shared;
  __shared__ float inv_of[2][kWavesPerBlock][2][kWave], to_of[2][kWavesPerBlock][2][kTile], bias[2][kWavesPerBlock][kTile];
  const int lane = threadIdx.x & (kWave - 1), m = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = blockIdx.x, t0 = (blockIdx.z * kWavesPerBlock + wave) * T;
  f32x16 dwg[T], dwu[T], dwd[T];  // dwd transposed: its rows are Y's columns
#pragma unroll
  for (int t = 0; t < T; ++t) dwg[t] = dwu[t] = dwd[t] = zeros();
  Total dbg, dbu, dbd[T];
  const u32x4 *const gu = a.gu + (int64_t)h * gu_words(a.fq);
  const TileVectors &vectors = vectors_of(gu, a.fq);
  const float bg = vectors.bg[m], bu = vectors.bu[m], inv_g = vectors.inv_g[m], inv_u = vectors.inv_u[m], inv_d = vectors.inv_d[m];
  const int64_t first = blockIdx.y * a.tiles_per_part * kTile;
  const int64_t end = first + a.tiles_per_part * kTile < a.rows ? first + a.tiles_per_part * kTile : a.rows;
  const auto sign_of = [](int64_t base) { return base / kTile % 2 ? -1.f : 1.f; };
  int turn = 0;
  for (int64_t batch = first; batch < end; batch += kWavesPerBlock * kTile, turn ^= 1) {
    const int64_t mine = batch + wave * kTile;
    if (mine < end) {
      const bool there = mine + m < end;
      const RowAt at = row_at(a, mine, m);
      const float *const x = a.X[at.t] + at.i * a.ldx, *const dy = a.dY[at.t] + at.i * a.lddy;
      const float sign = sign_of(mine);
      const Scale scale_x = scale_of_row(x, there ? a.F : 0, g, a.vec_x), scale_dy = scale_of_row(dy, there ? a.Fo : 0, g, a.vec_dy);
      Sums sg = no_sums(), su = no_sums(), sd = no_sums();
      float v[8];
      for (int q = 0; q < a.fq; ++q) {
        load8(v, x, q * kDepth + 8 * g, there ? a.F : 0, a.vec_x);
        const Split b = split8(v, sign * scale_x.to);
        add_product(sg, b, fragment(gu, 2 * q));
        add_product(su, b, fragment(gu, 2 * q + 1));
      }
      for (int q = 0; q < a.oq; ++q) {
        load8(v, dy, q * kDepth + 8 * g, there ? a.Fo : 0, a.vec_dy);
        add_product(sd, split8(v, sign * scale_dy.to), fragment(a.up, (int64_t)h * a.oq + q));
      }
      float vg[16], vu[16], vh[16], tile_g = 0.f, tile_u = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = result_depth(r / 8, g, r % 8);
        const float inv_x = __shfl(scale_x.inv, d), inv_dy = __shfl(scale_dy.inv, d);
        const float sx = sign * inv_x;
        const float2 c = activate_slope<ACT>(fmaf(sum_of(sg, r), sx * inv_g, bg));
        const float u = fmaf(sum_of(su, r), sx * inv_u, bu), e = sum_of(sd, r) * (sign * inv_dy * inv_d);
        vg[r] = e * u * c.y;
        vu[r] = e * c.x;
        tile_g += vg[r];
        tile_u += vu[r];
        vg[r] *= inv_x;
        vu[r] *= inv_x;
        vh[r] = c.x * u * inv_dy;
      }
      dbg.add(tile_g), dbu.add(tile_u);
      const auto pieces = [&](const float (&from)[16], int index) {
        const Scale scale = scale_for(max_over_32(largest_of(from)));
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = from[8 * s + j];
          lay(shared.piece[turn][wave], index + s, split8(v, scale.to), lane);
        }
        return sign * scale.inv;
      };
      shared.inv[turn][wave][lane] = pieces(vg, 0);
      inv_of[turn][wave][0][lane] = pieces(vu, 2);
      inv_of[turn][wave][1][lane] = pieces(vh, 4);
      if (g == 0) to_of[turn][wave][0][m] = sign * scale_x.to, to_of[turn][wave][1][m] = sign * scale_dy.to;
    }
    __syncthreads();
    for (int w = 0; w < kWavesPerBlock && batch + w * kTile < end; ++w) {
      const int64_t base = batch + w * kTile;
      const u32x4 *const of = shared.piece[turn][w];
      const float cg = shared.inv[turn][w][lane], cu = inv_of[turn][w][0][lane], ch = inv_of[turn][w][1][lane];
      float v[8];
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const int c = (t0 + t) * kTile + m;
        const auto transposed = [&](const float *const *X, int64_t ld, int F, const float (&to)[kTile], int s) {
          float scaled[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int d = result_depth(s, g, j);
            const RowAt r = row_at(a, base, d);
            v[j] = base + d < end && c < F ? X[r.t][r.i * ld + c] : 0.f;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) scaled[j] = v[j] * to[result_depth(s, g, j)];
          return split8(scaled, 1.f);
        };
        if (t0 + t < a.ft) {
          Sums g_sum = no_sums(), u_sum = no_sums();
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const Split xs = transposed(a.X, a.ldx, a.F, to_of[turn][w][0], s);
            add_product(g_sum, xs, fragment(of, s));
            add_product(u_sum, xs, fragment(of, 2 + s));
          }
          add(dwg[t], cg, g_sum);
          add(dwu[t], cu, u_sum);
        }
        if (t0 + t < a.ot) {
          Sums d_sum = no_sums();
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const Split dys = transposed(a.dY, a.lddy, a.Fo, to_of[turn][w][1], s);
#pragma unroll
            for (int j = 0; j < 8; ++j) dbd[t].add(v[j]);
            add_product(d_sum, dys, fragment(of, 4 + s));
          }
          add(dwd[t], ch, d_sum);
        }
      }
    }
  }
  float *const to = a.partial + blockIdx.y * a.part_floats, *const to_d = to + 2 * (int64_t)a.F * a.hidden;
  const int hid = h * kTile + m;
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int c = (t0 + t) * kTile + result_depth(r / 8, g, r % 8);
      if (c < a.F && hid < a.hidden) {
        to[(int64_t)c * a.hidden + hid] = dwg[t][r];
        to[((int64_t)a.F + c) * a.hidden + hid] = dwu[t][r];
      }
      if (c < a.Fo && hid < a.hidden) to_d[(int64_t)hid * a.Fo + c] = dwd[t][r];
    }
  float *const to_b = to_d + (int64_t)a.hidden * a.Fo;
  const float sum_g = dbg.sum + __shfl_xor(dbg.sum, 32), sum_u = dbu.sum + __shfl_xor(dbu.sum, 32);
  if (g == 0) bias[0][wave][m] = sum_g, bias[1][wave][m] = sum_u;
  __syncthreads();
  if (blockIdx.z == 0 && wave == 0 && g == 0 && hid < a.hidden) {
    to_b[hid] = (bias[0][0][m] + bias[0][1][m]) + (bias[0][2][m] + bias[0][3][m]);
    to_b[a.hidden + hid] = (bias[1][0][m] + bias[1][1][m]) + (bias[1][2][m] + bias[1][3][m]);
  }
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const float b = dbd[t].sum + __shfl_xor(dbd[t].sum, 32);
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
__device__ inline void sum_parts(const SumArgs &a, int64_t first, float (&part)[4][kWave]) {
  const int x = threadIdx.x & (kWave - 1), y = threadIdx.x / kWave;
  const int64_t e = first + x;
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
constexpr int64_t kMostSums = (int64_t)1 << 22;  // workgroups (a launch has fewer than 2^32 threads along x)
__global__ void __launch_bounds__(kBlock) k_ff_sums(SumArgs a) {
  __shared__ float part[4][kWave];
  for (int64_t first = (int64_t)blockIdx.x * kWave; first < a.part_floats; first += (int64_t)gridDim.x * kWave) {
    sum_parts(a, first, part);
    __syncthreads();
  }
}

// ---- host ---------------------------------------------------------------------------------------
bool aligned(const float *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 4 == 0; }

// Tiles of up to 256 columns: as many as one of the kernels that keep a row has; behind the columns that there are the fragments hold 0.
constexpr int kKept = 256;
constexpr int kUnits = 256;    // compute units
constexpr int kKeptTiles = 4;  // of the gradient of X that one workgroup has
int32_t column_tiles(int32_t F) {
  const int32_t t = (int32_t)tiles(F, kTile);
  return F > kKept || t <= 2 ? t : t <= 4 ? 4 : 8;
}
int32_t depth_tiles(int32_t F, bool backward) {
  const int32_t t = (int32_t)tiles(F, kDepth);
  return F > kKept || t <= 2 ? t : t <= 4 ? 4 : t <= 6 && !backward ? 6 : t <= 8 ? 8 : 16;
}

// What lies where in the workspace (bytes), the same for the size query and the calls.
struct Plan {
  int32_t ht, fq, oq, ft, ot;
  int64_t n_gu, n_down, n_up, n_back;
  size_t gu, down, up, back, inv_out, bd, partial, total;
  int64_t rows, part_floats, parts, tiles_per_part;
  bool kept, few, split;
  int weight_waves;
  Plan(const pipad_gated_ff_t &c, int32_t n, int32_t k, bool backward) {
    ht = (int32_t)tiles(c.hidden, kTile);
    fq = depth_tiles(c.F, backward), ft = column_tiles(c.F), oq = depth_tiles(c.Fo, backward), ot = column_tiles(c.Fo);
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
    inv_out = take((backward ? ft : ot) * kTile * sizeof(float)), bd = take(backward ? 0 : ot * kTile * sizeof(float));
    rows = (int64_t)n * k;
    part_floats = 2 * (int64_t)c.F * c.hidden + (int64_t)c.hidden * c.Fo + 2 * (int64_t)c.hidden + c.Fo;
    // Parts of the rows for the weights' gradients.  Rows of any width: a thousand workgroups, a tile of rows a wave at least.  Up to
    // 256 columns, where the tiles are of one snapshot each: as many workgroups (64 hidden columns each) as run at a time, and one tile each
    // of up to 64, two of more, where there are few (64 columns through 256, these gradients alone: 19.7 us instead of 28.0 with four at 256 rows, 27.6
    // instead of 30.6 at 4096, with one 28.7).
    kept = c.F <= kKept && c.Fo <= kKept;
    const int64_t row_tiles = kept ? tiles(n, kTile) * k : tiles(rows, kTile);
    // Eight waves share the rows' splitting where they are all of use (64 columns at most, for the registers): 0.84 of the time of
    // four twice at 32 columns, 0.92 at 64 (1.6 million rows, 128 and 256 hidden columns: 471 us, four 560; 1336, four 1451).
    const int64_t four = tiles(c.hidden, 64), eight = tiles(c.hidden, 128);
    weight_waves = std::max(ft, ot) <= 2 && 2 * eight * 87 < four * 100 ? 8 : 4;
    const int64_t at_a_time = weight_waves == 8 ? 256 : std::max(ft, ot) <= 2 ? 512 : std::max(ft, ot) <= 4 ? 256 : 128;
    const int64_t most = std::max<int64_t>(1, kept ? at_a_time / (weight_waves == 8 ? eight : four) : 1024 / ht);
    tiles_per_part = std::max<int64_t>(!kept ? 4 : row_tiles <= 64 ? 1 : 2, tiles(row_tiles, most));
    parts = tiles(row_tiles, tiles_per_part);
    // A workgroup a row takes as long for 256 rows, one a compute unit, as for one, and then for every further 256: 64 columns through 256,
    // 8.1 us at 1 row, 8.5 at 256, 15.1 at 512; eight waves to 32 rows 13.8 to 14.1 throughout (32 through 128: 6.7, 7.0, 11.7 and 9.8 to
    // 10.1; 256 through 1024: 47, 48, 95 and 89 to 92).  The kernels for more than 256 columns take longer for the same rows: 512 rows there (512
    // through 2048: 185, 183, 363 at 512, 725 at 1024, in tiles 530 to 556; 40 through 600 to 512: 28, 29, 55, 109, in tiles 83 to 86).
    few = !backward && rows <= (kept ? 256 : 512) && c.F <= kFewMostF && (c.hidden <= kFewColumns || c.Fo <= kFewMostFo);  // (LDS holds a row, its sums)
    // Eight waves to 32 rows instead of one, as long as that is one round of workgroups: two a compute unit forward, one for the gradient of X,
    // of which 256 columns need two for the same rows.  64 through 256, both with the packing of the weights: 13.7 us instead of 20.5 at
    // 4096 rows, 16.6 instead of 21.0 at 16384, 26.0 instead of 21.9 at 32768; the gradient 20.0 instead of 30.5 at 4096, 29.1 instead of 30.9 and
    // 46.5 instead of 32.3.  256 through 1024 at 4096 rows: 84 instead of 186, the gradient 111 instead of 231.  Fewer than four tiles of
    // hidden columns are too little to share: 16 through 64 took 8.8 instead of 8.2.
    const int64_t groups = backward ? tiles(rows, kTile) * tiles(ft, kKeptTiles) : tiles(rows, 2 * kTile);
    split = kept && ht >= 4 && groups <= kUnits;
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
  a.ldx = ldx, a.lddy = lddy, a.ldo = ldo, a.rows = p.rows, a.n = n, a.k = k, a.F = c.F, a.hidden = c.hidden, a.Fo = c.Fo;
  a.ht = p.ht, a.fq = p.fq, a.oq = p.oq, a.ft = p.ft, a.ot = p.ot;
  a.gu = reinterpret_cast<const u32x4 *>(ws + p.gu), a.down = reinterpret_cast<const u32x4 *>(ws + p.down);
  a.up = reinterpret_cast<const u32x4 *>(ws + p.up), a.back = reinterpret_cast<const u32x4 *>(ws + p.back);
  a.inv_out = reinterpret_cast<const float *>(ws + p.inv_out), a.bd = reinterpret_cast<const float *>(ws + p.bd);
  a.Wg = c.Wg, a.Wu = c.Wu, a.Wd = c.Wd, a.bg = c.bg, a.bu = c.bu, a.bd_in = c.bd, a.ldwg = c.ldwg, a.ldwu = c.ldwu, a.ldwd = c.ldwd;
  a.partial = reinterpret_cast<float *>(ws + p.partial), a.part_floats = p.part_floats, a.tiles_per_part = p.tiles_per_part;
  return a;
}

int pack(const pipad_gated_ff_t &c, const Plan &p, bool dx, char *ws, hipStream_t st) {
  const auto at = [&](size_t offset, int64_t count) { return count ? reinterpret_cast<u32x4 *>(ws + offset) : nullptr; };
  // A fragment a wave and one round of loads for it, where the hidden tiles are 64 at most; each workgroup looks for the largest of its columns itself.
  const int32_t most = std::max<int32_t>(p.n_down ? 8 : 4, (int32_t)tiles(p.ht, 16));
  const PackArgs a{c.Wg,   c.Wu,   c.Wd, c.bg, c.bu, c.bd, c.ldwg, c.ldwu, c.ldwd, c.F, c.hidden, c.Fo,
                   p.ht,   p.fq,   p.oq, p.ft, p.ot, at(p.gu, p.n_gu), at(p.down, p.n_down), at(p.up, p.n_up), at(p.back, p.n_back),
                   reinterpret_cast<float *>(ws + p.inv_out), reinterpret_cast<float *>(ws + p.bd), most};
  const int64_t columns = p.n_down ? p.ot : dx ? p.ft : 0;
  hipLaunchKernelGGL(k_ff_pack, dim3((unsigned)(p.ht + columns * tiles(p.ht, most))), dim3(kPackWaves * kWave), 0, st, a);
  PIPAD_HIP(hipGetLastError());
  return PIPAD_OK;
}

// A kernel by activation and by the tiles of columns that a wave keeps: 1, 2 or 4 (the weights' gradients, three matrices of them: 1 or 2).
using FfKernel = void (*)(FfArgs);
#define PIPAD_FF_KERNELS(name, ...) \
  constexpr FfKernel name##_of[4][3] = {{name<0, 1>, name<0, 2>, name<0, __VA_ARGS__>}, {name<1, 1>, name<1, 2>, name<1, __VA_ARGS__>}, \
                                        {name<2, 1>, name<2, 2>, name<2, __VA_ARGS__>}, {name<3, 1>, name<3, 2>, name<3, __VA_ARGS__>}};
static_assert(PIPAD_ACT_SIGMOID == 0 && PIPAD_ACT_RELU == 1 && PIPAD_ACT_GELU == 2 && PIPAD_ACT_SILU == 3, "the order below");
constexpr Kept (*kept_forward_of[4])(int, int) = {kept_forward<0>, kept_forward<1>, kept_forward<2>, kept_forward<3>};
constexpr Kept (*kept_backward_of[4])(int, int) = {kept_backward<0>, kept_backward<1>, kept_backward<2>, kept_backward<3>};
constexpr Kept (*kept_weights_of[4])(int, int, int) = {kept_weights<0>, kept_weights<1>, kept_weights<2>, kept_weights<3>};
constexpr FfKernel k_ff_few_of[4] = {k_ff_few<0>, k_ff_few<1>, k_ff_few<2>, k_ff_few<3>};
PIPAD_FF_KERNELS(k_ff_rows, 4)
PIPAD_FF_KERNELS(k_ff_rows_backward, 4)
PIPAD_FF_KERNELS(k_ff_weights_backward, 2)
#undef PIPAD_FF_KERNELS

// Which of 1, 2, 4 tiles a wave, of the four that share t
int width(int t) { return t <= kWavesPerBlock ? 0 : t <= 2 * kWavesPerBlock ? 1 : 2; }

}  // namespace

size_t gated_ff_workspace(const pipad_gated_ff_t &c, int32_t n, int32_t k, bool backward) { return Plan(c, n, k, backward).total; }

int gated_ff_launch(const pipad_gated_ff_t &c, int32_t n, int32_t k, const float *const *X, int64_t ldx, float *const *Y, int64_t ldy,
                    void *workspace, hipStream_t st) {
  const Plan p(c, n, k, false);
  char *const ws = static_cast<char *>(workspace);
  const FfArgs a = arguments(c, p, n, k, X, ldx, nullptr, 0, Y, ldy, ws);
  if (p.few) {
    hipLaunchKernelGGL(k_ff_few_of[c.activation], dim3((unsigned)p.rows), dim3(kFewThreads), 0, st, a);
    PIPAD_HIP(hipGetLastError());
    return PIPAD_OK;
  }
  const int rc = pack(c, p, false, ws, st);
  if (rc != PIPAD_OK) return rc;
  if (p.kept) {
    const Kept f = p.split ? split_forward(c.activation, p.ot) : kept_forward_of[c.activation](p.fq, p.ot);
    hipLaunchKernelGGL(f.kernel, dim3((unsigned)tiles(p.rows, p.split ? kTile : kTile * f.waves)), dim3(f.waves * kWave), 0, st, a);
    PIPAD_HIP(hipGetLastError());
    return PIPAD_OK;
  }
  const int w = width(p.ot);
  hipLaunchKernelGGL(k_ff_rows_of[c.activation][w], dim3((unsigned)tiles(p.rows, kTile), (unsigned)tiles(p.ot, kWavesPerBlock << w)),
                     dim3(kBlock), 0, st, a);
  PIPAD_HIP(hipGetLastError());
  return PIPAD_OK;
}

int gated_ff_backward_launch(const pipad_gated_ff_t &c, int32_t n, int32_t k, const float *const *X, int64_t ldx, const float *const *dY,
                             int64_t lddy, float *const *dX, int64_t lddx, const pipad_gated_ff_grads_t *grads, void *workspace, hipStream_t st) {
  const Plan p(c, n, k, true);
  char *const ws = static_cast<char *>(workspace);
  if (p.rows > 0) {
    // The kernel for the weights' gradients of rows of up to 256 columns reads the weights as they are.
    const int rc = dX || !p.kept ? pack(c, p, dX != nullptr, ws, st) : PIPAD_OK;
    if (rc != PIPAD_OK) return rc;
    const FfArgs a = arguments(c, p, n, k, X, ldx, dY, lddy, dX, lddx, ws);
    if (dX && p.kept) {
      const Kept f = p.split ? split_backward(c.activation, p.ft) : kept_backward_of[c.activation](p.fq, p.oq);
      hipLaunchKernelGGL(f.kernel, dim3((unsigned)tiles(p.rows, p.split ? kTile : kTile * f.waves), (unsigned)tiles(p.ft, kKeptTiles)),
                         dim3(f.waves * kWave), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    } else if (dX) {
      const int w = width(p.ft);
      hipLaunchKernelGGL(k_ff_rows_backward_of[c.activation][w],
                         dim3((unsigned)tiles(p.rows, kTile), (unsigned)tiles(p.ft, kWavesPerBlock << w)), dim3(kBlock), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    }
    if (grads && p.kept) {
      const Kept f = kept_weights_of[c.activation](p.ft, p.ot, p.weight_waves);
      hipLaunchKernelGGL(f.kernel, dim3((unsigned)tiles(c.hidden, 16 * f.waves), (unsigned)p.parts, (unsigned)tiles(std::max(p.ft, p.ot), kKeptTiles)),
                         dim3(f.waves * kWave), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    } else if (grads) {
      const int most = std::max(p.ft, p.ot), w = std::min(width(most), 1);
      hipLaunchKernelGGL(k_ff_weights_backward_of[c.activation][w],
                         dim3((unsigned)p.ht, (unsigned)p.parts, (unsigned)tiles(most, kWavesPerBlock << w)), dim3(kBlock), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    }
  }
  if (grads) {
    const SumArgs s{reinterpret_cast<const float *>(ws + p.partial), p.part_floats, (int32_t)p.parts, c.F, c.hidden, c.Fo, *grads};
    hipLaunchKernelGGL(k_ff_sums, dim3((unsigned)std::min(tiles(p.part_floats, kWave), kMostSums)), dim3(kBlock), 0, st, s);
    PIPAD_HIP(hipGetLastError());
  }
  return PIPAD_OK;
}

}  // namespace pipad
