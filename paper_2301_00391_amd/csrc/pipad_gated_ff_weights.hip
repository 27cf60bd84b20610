// The gated feed-forward block, the gradients of the weights, on rows of up to 128 columns.
//
// A wave owns 16 hidden columns: it keeps their weights' pieces in registers and accumulates their gradients there.  The four waves of a
// workgroup share the node rows, 32 of one snapshot at a time, whose pieces lie in LDS row by row in two slots, so that one barrier
// a tile is enough: while a tile is multiplied the next one is split and laid down.  G, U and dH are made with a node row a result row, so that
// dG, dU and H are operands of products whose depth is the node rows; the other operand, X or dY with its columns along the lanes, comes from
// the same LDS rows by loads that transpose.
//
// Everything is in 16 x 16 x 32 instructions: 16 columns a wave rather than 32 halve the registers for weights and gradients, so that two
// waves share a SIMD (64 columns: 244 registers) and the one's elementwise work, some 1900 cycles a tile, runs beside the other's 2304 of matrix
// instructions.  With 32 columns and one wave a SIMD it took 3.5 ms on 1.6 million rows of 64 through 256 columns.
// l = lane % 16, g = lane / 16: an operand's lane holds row (column) l, depth 8 g .. 8 g + 7; register r of the result is row 4 g + r, column l.
// Two results one below the other are an operand whose depth runs over 16 (j / 4) + 4 g + j % 4; a load that transposes gives lane l of 16 the
// 16-bit values of column l in four rows, whose 8-byte pieces the lanes 4 j + c address (row j, columns 4 c ..).
#include "pipad_gated_ff.h"

namespace pipad {
namespace ff {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ inline f32x4 mfma16(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ inline f32x4 product16(const Split &a, const Split &b, f32x4 c) {  // as product()
  c = mfma16(a.p[2], b.p[0], c);
  c = mfma16(a.p[0], b.p[2], c);
  c = mfma16(a.p[1], b.p[1], c);
  c = mfma16(a.p[1], b.p[0], c);
  c = mfma16(a.p[0], b.p[1], c);
  return mfma16(a.p[0], b.p[0], c);
}

// The pieces of 32 rows of 32 D columns: three planes, rows 16 bytes further apart than they are long, so that 16 lanes that read 16 bytes of a
// row each, or 8 bytes of four rows each, meet all banks once.
template <int D>
struct Slot {
  static constexpr int kStride = 64 * D + 16;
  char plane[3][kTile * kStride];
  __device__ void put(int row, int chunk, const Split &s) {  // columns 8 chunk ..
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4 *>(plane[p] + row * kStride + 16 * chunk) = s.p[p];
  }
  // rows 16 sub .., columns 32 d ..
  __device__ Split plain(int sub, int d, int lane) const {
    const int at = (16 * sub + lane % 16) * kStride + 64 * d + 16 * (lane / 16);
    Split s;
#pragma unroll
    for (int p = 0; p < 3; ++p) s.p[p] = *reinterpret_cast<const u32x4 *>(plane[p] + at);
    return s;
  }
  // columns 16 t .., all 32 rows
  __device__ Split transposed(int t, int lane) const {
    const int at = (4 * (lane / 16) + lane % 16 / 4) * kStride + 32 * t + 8 * (lane % 4);
    Split s;
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      typedef const __attribute__((address_space(3))) s16x4 *Lds;
      union {
        s16x4 h[2];
        u32x4 w;
      } both;
#pragma unroll
      for (int half = 0; half < 2; ++half)
        both.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(Lds)(plane[p] + at + 16 * half * kStride));
      s.p[p] = both.w;
    }
    return s;
  }
};

// A thread's share of the rows that come next: 8 columns at a time, D of them 8 rows apart ... D (32 rows are 128 D pieces of 8 columns).
template <int D>
struct Share {
  static constexpr int kMine = kTile * 4 * D / kBlock > 0 ? kTile * 4 * D / kBlock : 1, kChunks = 4 * D;
  float v[kMine][8];
  __device__ static bool there() { return kTile * kChunks >= kBlock || threadIdx.x < kTile * kChunks; }
  __device__ static int row(int q) { return (q * kBlock + threadIdx.x) / kChunks; }
  __device__ static int chunk() { return threadIdx.x % kChunks; }
  __device__ void load(const float *first, int64_t ld, int F, bool vec, int count) {  // rows behind `count` are 0
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      const int r = row(q);
      load8(v[q], first + (r < count ? r : 0) * ld, 8 * chunk(), there() && r < count ? F : 0, vec);
    }
  }
  __device__ void lay_down(Slot<D> &slot, float sign) {
    if (!there()) return;
#pragma unroll
    for (int q = 0; q < kMine; ++q) slot.put(row(q), chunk(), split8(v[q], sign));
  }
};

template <int ACT, int FD, int OD>
__global__ void __launch_bounds__(kBlock, FD + OD <= 4 ? 2 : 1) k_ff_kept_weights(FfArgs a) {
  __shared__ Slot<FD> xs[2];
  __shared__ Slot<OD> dys[2];
  const int lane = threadIdx.x & (kWave - 1), l = lane & 15, g = lane >> 4;
  const int hid = (blockIdx.x * kWavesPerBlock + threadIdx.x / kWave) * 16 + l;  // this lane's hidden column; none: weights of 0
  const bool there = hid < a.hidden;

  Split wg[FD], wu[FD], wd[OD];
  {
    float v[8];
#pragma unroll
    for (int q = 0; q < FD; ++q) {
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const float *const W = w ? a.Wu : a.Wg;
        const int64_t ld = w ? a.ldwu : a.ldwg;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int f = 32 * q + 8 * g + j;
          v[j] = there && f < a.F ? W[f * ld + hid] : 0.f;
        }
        (w ? wu : wg)[q] = split8(v);
      }
    }
#pragma unroll
    for (int q = 0; q < OD; ++q) {
      load8(v, a.Wd + (there ? hid : 0) * a.ldwd, 32 * q + 8 * g, there ? a.Fo : 0, false);
      wd[q] = split8(v);
    }
  }
  const float bg = there && a.bg ? a.bg[hid] : 0.f, bu = there && a.bu ? a.bu[hid] : 0.f;
  f32x4 dwg[2 * FD], dwu[2 * FD], dwd[2 * OD];
#pragma unroll
  for (int t = 0; t < 2 * FD; ++t) dwg[t] = dwu[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < 2 * OD; ++t) dwd[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float dbg = 0.f, dbu = 0.f, dbd[8] = {};

  // the part's tiles, of each snapshot a whole number, and the place of the one that is loaded next
  const int64_t of_snapshot = ((int64_t)a.n + kTile - 1) / kTile, every = of_snapshot * a.k;
  const int64_t first = blockIdx.y * a.tiles_per_part, left = every - first, count = left < a.tiles_per_part ? left : a.tiles_per_part;
  int t = (int)(first / of_snapshot);
  int64_t i0 = first % of_snapshot * kTile, loaded = 0;
  Share<FD> x;
  Share<OD> dy;
  const auto load_next = [&] {
    const int rows = loaded < count ? (int)(a.n - i0 < kTile ? a.n - i0 : kTile) : 0;
    if (rows > 0) {
      x.load(a.X[t] + i0 * a.ldx, a.ldx, a.F, a.vec_x, rows);
      dy.load(a.dY[t] + i0 * a.lddy, a.lddy, a.Fo, a.vec_dy, rows);
    }
    ++loaded;
    i0 += kTile;
    if (i0 >= a.n) i0 = 0, ++t;
  };
  const auto lay_down = [&](int slot, float sign) {
    x.lay_down(xs[slot], sign);
    if (blockIdx.x == 0)
#pragma unroll
      for (int q = 0; q < Share<OD>::kMine; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) dbd[j] += dy.v[q][j];
    dy.lay_down(dys[slot], sign);
  };

  load_next();
  lay_down(0, 1.f);
  load_next();
  __syncthreads();
  float sign = 1.f;
  for (int64_t i = 0; i < count; ++i) {
    const Slot<FD> &X = xs[i & 1];
    const Slot<OD> &dY = dys[i & 1];
    f32x4 G[2], U[2], dH[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float b = sign * bg, c = sign * bu;
      G[s] = f32x4{b, b, b, b}, U[s] = f32x4{c, c, c, c}, dH[s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < FD; ++q) {
        const Split p = X.plain(s, q, lane);
        G[s] = product16(p, wg[q], G[s]);
        U[s] = product16(p, wu[q], U[s]);
      }
#pragma unroll
      for (int q = 0; q < OD; ++q) dH[s] = product16(dY.plain(s, q, lane), wd[q], dH[s]);
    }
    if (i + 1 < count) {
      lay_down((int)(i + 1) & 1, -sign);
      load_next();
    }
    // X and dY have this tile's sign, which cancels in the product of dH and U
    float vg[8], vu[8], vh[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 c = activate_slope<ACT>(sign * G[j / 4][j % 4]);
      const float u = U[j / 4][j % 4], d = dH[j / 4][j % 4], as = sign * c.x;
      vg[j] = d * u * c.y;
      vu[j] = d * as;
      vh[j] = as * u;
      dbg += vg[j];
      dbu += vu[j];
    }
    const Split dg = split8(vg), du = split8(vu), hh = split8(vh);
    const f32x4 zero{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 2 * FD; ++q) {
      const Split p = X.transposed(q, lane);
      const f32x4 gs = product16(p, dg, zero), us = product16(p, du, zero);
#pragma unroll
      for (int r = 0; r < 4; ++r) dwg[q][r] = fmaf(sign, gs[r], dwg[q][r]), dwu[q][r] = fmaf(sign, us[r], dwu[q][r]);
    }
#pragma unroll
    for (int q = 0; q < 2 * OD; ++q) {
      const f32x4 ds = product16(hh, dY.transposed(q, lane), zero);
#pragma unroll
      for (int r = 0; r < 4; ++r) dwd[q][r] = fmaf(sign, ds[r], dwd[q][r]);
    }
    __syncthreads();
    sign = -sign;
  }

  float *const to = a.partial + blockIdx.y * a.part_floats, *const to_d = to + 2 * (int64_t)a.F * a.hidden, *const to_b = to_d + (int64_t)a.hidden * a.Fo;
  if (blockIdx.x == 0) {  // dbd: every thread has its columns' sums over its rows
    float *const sums = reinterpret_cast<float *>(dys);
    constexpr int kThreads = kBlock / Share<OD>::kChunks;  // threads of a chunk of columns
    if (Share<OD>::there())
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[(threadIdx.x / Share<OD>::kChunks) * 32 * OD + 8 * Share<OD>::chunk() + j] = dbd[j];
    __syncthreads();
    for (int c = threadIdx.x; c < a.Fo; c += kBlock) {
      float s = 0.f;
      for (int w = 0; w < (kThreads < kTile ? kThreads : kTile); ++w) s += sums[w * 32 * OD + c];
      to_b[2 * a.hidden + c] = s;
    }
  }
  // (all lanes have to take part before those without a column leave)
  dbg += __shfl_xor(dbg, 16);
  dbu += __shfl_xor(dbu, 16);
  dbg += __shfl_xor(dbg, 32);
  dbu += __shfl_xor(dbu, 32);
  if (there) {
#pragma unroll
    for (int q = 0; q < 2 * FD; ++q)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int f = 16 * q + 4 * g + r;
        if (f < a.F) {
          to[(int64_t)f * a.hidden + hid] = dwg[q][r];
          to[((int64_t)a.F + f) * a.hidden + hid] = dwu[q][r];
        }
      }
    if (g == 0) to_b[hid] = dbg, to_b[a.hidden + hid] = dbu;
  }
#pragma unroll
  for (int q = 0; q < 2 * OD; ++q)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = hid - l + 4 * g + r, fo = 16 * q + l;
      if (row < a.hidden && fo < a.Fo) to_d[(int64_t)row * a.Fo + fo] = dwd[q][r];
    }
}

template <int ACT, int FD>
Kept kept_weights_of(int od) {
  switch (od) {
    case 1: return {k_ff_kept_weights<ACT, FD, 1>, kWavesPerBlock};
    case 2: return {k_ff_kept_weights<ACT, FD, 2>, kWavesPerBlock};
    default: return {k_ff_kept_weights<ACT, FD, 4>, kWavesPerBlock};
  }
}
template <int ACT>
Kept kept_weights_of(int fd, int od) {
  return fd == 1 ? kept_weights_of<ACT, 1>(od) : fd == 2 ? kept_weights_of<ACT, 2>(od) : kept_weights_of<ACT, 4>(od);
}
}  // namespace

Kept kept_weights(int act, int fd, int od) {
  switch (act) {
    case PIPAD_ACT_SIGMOID: return kept_weights_of<PIPAD_ACT_SIGMOID>(fd, od);
    case PIPAD_ACT_RELU: return kept_weights_of<PIPAD_ACT_RELU>(fd, od);
    case PIPAD_ACT_GELU: return kept_weights_of<PIPAD_ACT_GELU>(fd, od);
    default: return kept_weights_of<PIPAD_ACT_SILU>(fd, od);
  }
}

}  // namespace ff
}  // namespace pipad
