// The gated feed-forward block: weights as fragments, the kernels for rows of any width, and the host side.  How the products are
// made stands in pipad_gated_ff.h; rows of few columns have kernels of their own in pipad_gated_ff_forward.hip, _backward.hip and _weights.hip.
#include "pipad_gated_ff.h"

namespace pipad {
using namespace ff;

namespace {

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
int32_t depth_tiles(int32_t F, bool backward) {
  const int32_t t = (int32_t)tiles(F, kDepth);
  return F > kKept || t <= 2 ? t : t <= 4 ? 4 : t <= 6 && !backward ? 6 : 8;
}

// What lies where in the workspace (bytes), the same for the size query and the calls.
struct Plan {
  int32_t ht, fq, oq, ft, ot;
  int64_t n_gu, n_down, n_up, n_back;
  size_t gu, down, up, back, bd, partial, total;
  int64_t rows, part_floats, parts, tiles_per_part;
  bool kept;
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
    bd = take(ot * kTile * sizeof(float));
    rows = (int64_t)n * k;
    part_floats = 2 * (int64_t)c.F * c.hidden + (int64_t)c.hidden * c.Fo + 2 * (int64_t)c.hidden + c.Fo;
    // Parts of the rows for the weights' gradients, four tiles of rows at least in each.  Rows of any width: about two waves a SIMD.  Up to
    // 128 columns, where the tiles are of one snapshot each: as many workgroups (64 hidden columns each) as run at a time.
    kept = c.F <= kKept && c.Fo <= kKept;
    const int64_t row_tiles = kept ? tiles(n, kTile) * k : tiles(rows, kTile);
    const int64_t at_a_time = std::max(ft, ot) <= 2 ? 512 : 256;
    const int64_t most = std::max<int64_t>(1, kept ? at_a_time / tiles(c.hidden, 16 * kWavesPerBlock) : 2048 / ht);
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
  a.ldx = ldx, a.lddy = lddy, a.ldo = ldo, a.rows = p.rows, a.n = n, a.k = k, a.F = c.F, a.hidden = c.hidden, a.Fo = c.Fo;
  a.ht = p.ht, a.fq = p.fq, a.oq = p.oq, a.ft = p.ft, a.ot = p.ot;
  a.gu = reinterpret_cast<const u32x4 *>(ws + p.gu), a.down = reinterpret_cast<const u32x4 *>(ws + p.down);
  a.up = reinterpret_cast<const u32x4 *>(ws + p.up), a.back = reinterpret_cast<const u32x4 *>(ws + p.back);
  a.bd = reinterpret_cast<const float *>(ws + p.bd);
  a.Wg = c.Wg, a.Wu = c.Wu, a.Wd = c.Wd, a.bg = c.bg, a.bu = c.bu, a.ldwg = c.ldwg, a.ldwu = c.ldwu, a.ldwd = c.ldwd;
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
  if (p.kept) {
    const Kept f = kept_forward(c.activation, p.fq, p.ot);
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
    if (dX && p.kept) {
      const Kept f = kept_backward(c.activation, p.fq, p.oq);
      hipLaunchKernelGGL(f.kernel, dim3((unsigned)tiles(p.rows, kTile * f.waves)), dim3(f.waves * kWave), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    } else if (dX) {
      const int w = width(p.ft);
      hipLaunchKernelGGL(k_ff_rows_backward_of[c.activation][w],
                         dim3((unsigned)tiles(p.rows, kTile * kWavesPerBlock), (unsigned)tiles(p.ft, 1 << w)), dim3(kBlock), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    }
    if (grads && p.kept) {
      const Kept f = kept_weights(c.activation, p.ft, p.ot);
      hipLaunchKernelGGL(f.kernel, dim3((unsigned)tiles(c.hidden, 16 * f.waves), (unsigned)p.parts), dim3(f.waves * kWave), 0, st, a);
      PIPAD_HIP(hipGetLastError());
    } else if (grads) {
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
