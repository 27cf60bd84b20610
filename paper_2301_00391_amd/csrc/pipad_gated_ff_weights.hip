// The gated feed-forward block, the gradients of the weights, on rows of up to 256 columns.
//
// A wave owns 16 hidden columns: it keeps their weights' pieces in registers and accumulates their gradients there.  The four waves of a
// workgroup share the node rows, 32 of one snapshot at a time, whose pieces lie in LDS row by row in two slots, so that one barrier
// a tile is enough: while a tile is multiplied the next one is split and laid down.  G, U and dH are made with a node row a result row, so that
// dG, dU and H are operands of products whose depth is the node rows; the other operand, X or dY with its columns along the lanes, comes from
// the same LDS rows by loads that transpose.  It keeps its rows' scales there, by whose inverses dG, dU and H are multiplied before they get a
// scale of their own: a lane's, since a lane is a hidden column of theirs and of the result.
//
// Of more than 128 columns a workgroup accumulates the gradients that go with 128 of X's and 128 of Y's, and another makes G, U and dH once more
// for the rest: all of them do not fit the registers.
//
// 1.6 million rows of 64 through 256: 1.33 ms (236 TFLOP/s of its six products), the vector instructions 71 % of the cycles, the matrix instructions
// 30 %.  312 thousand rows of 128 through 341, where one wave a SIMD waits for itself: 1.25 ms, 50 % and 19 %.
//
// Everything is in 16 x 16 x 32 instructions: 16 columns a wave rather than 32 halve the registers for weights and gradients, so that two
// waves share a SIMD and one's elementwise work runs beside the other's matrix instructions.
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
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
struct Sums16 {  // as Sums
  f32x4 main, cross;
};
__device__ inline Sums16 no_sums16() { return {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}; }
__device__ inline void add_product16(Sums16 &c, const Split &a, const Split &b) {
  c.cross = mfma16(a.p[1], b.p[0], c.cross);
  c.main = mfma16(a.p[0], b.p[0], c.main);
  c.cross = mfma16(a.p[0], b.p[1], c.cross);
}
__device__ inline float sum_of(const Sums16 &c, int r) { return fmaf(c.cross[r], 1.f / kWide, c.main[r]); }

// The pieces of 32 rows of 32 D columns, two planes, and 1 over the rows' scales.  The 16-byte chunks of a row are permuted by its number, so that
// 16 neighbouring lanes that read a chunk of a row each, and 32 that read 8 bytes of eight rows, meet all 64 banks once: rows of 64 D bytes are 4 / D
// to the 256 of all banks, and the chunks of those that lie on the same banks have to differ, for the loads that transpose in pairs.  26 to 28 % of
// the LDS cycles are counted as conflicts all the same, so that some access is not taken 16, or 32, neighbouring lanes at a time.
template <int D>
struct Slot {
  char plane[2][kTile * 64 * D];
  float inv[kTile];
  __device__ static int place(int row, int chunk) {
    const int high = row >> 3 & 1;
    const int f = D == 1 ? (row >> 2 & 1) * 2 + high : D == 2 ? (row >> 1 & 3) * 2 + high : (row & 7) * 2 + high;
    return row * 64 * D + ((chunk ^ f) << 4);
  }
  __device__ void put(int row, int chunk, const Split &s) {  // columns 8 chunk ..
#pragma unroll
    for (int p = 0; p < 2; ++p) *reinterpret_cast<u32x4 *>(plane[p] + place(row, chunk)) = s.p[p];
  }
  // rows 16 sub .., columns 32 d ..
  __device__ Split plain(int sub, int d, int lane) const {
    const int at = place(16 * sub + lane % 16, 4 * d + lane / 16);
    Split s;
#pragma unroll
    for (int p = 0; p < 2; ++p) s.p[p] = *reinterpret_cast<const u32x4 *>(plane[p] + at);
    return s;
  }
  // columns 16 t .., all 32 rows
  __device__ Split transposed(int t, int lane) const {
    const int row = 4 * (lane / 16) + lane % 16 / 4, c = lane % 4;
    const int at = place(row, 2 * t + c / 2) + 8 * (c % 2);  // (16 rows further on the chunks lie alike)
    Split s;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      union {
        s16x4 h[2];
        u32x4 w;
      } both;
#pragma unroll
      for (int half = 0; half < 2; ++half)
        both.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(plane[p] + at + 16 * half * 64 * D));
      s.p[p] = both.w;
    }
    return s;
  }
};

// A thread's share of the rows that come next, 8 columns at a time: 4 D consecutive threads have a row.  Where there are threads enough X's are the
// first of a workgroup's THREADS and dY's come behind them, at AT.
template <int D, int AT, int THREADS>
struct Share {
  static constexpr int kChunks = 4 * D, kUnits = kTile * kChunks, kMine = kUnits > THREADS ? kUnits / THREADS : 1;
  float v[kMine][8];
  __device__ static int me() {
    int at = (int)threadIdx.x - AT;
    if (D > 4) asm("" : "+v"(at));  // (of 256 columns: what follows from it is made again each time, for the registers)
    return at;
  }
  __device__ static bool there() { return AT + kUnits >= THREADS ? AT == 0 || me() >= 0 : me() >= 0 && me() < kUnits; }
  __device__ static int row(int q) { return (q * THREADS + me()) / kChunks; }
  __device__ static int chunk() { return me() % kChunks; }
  __device__ void load(const float *first, int64_t ld, int F, bool vec, int count) {  // rows behind `count` are 0
    if (!there()) return;
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      const int r = row(q);
      const float *const at = first + (r < count ? r : 0) * ld;
      if (vec && F % 8 == 0) {  // (no column is left out of a piece)
        float4 t[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
        if (r < count && 8 * chunk() < F) {
          t[0] = *reinterpret_cast<const float4 *>(at + 8 * chunk());
          t[1] = *reinterpret_cast<const float4 *>(at + 8 * chunk() + 4);
        }
        v[q][0] = t[0].x, v[q][1] = t[0].y, v[q][2] = t[0].z, v[q][3] = t[0].w;
        v[q][4] = t[1].x, v[q][5] = t[1].y, v[q][6] = t[1].z, v[q][7] = t[1].w;
      } else {
        load8(v[q], at, 8 * chunk(), r < count ? F : 0, vec);
      }
    }
  }
  __device__ void lay_down(Slot<D> &slot, float sign) {
    if (!there()) return;
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      uint32_t x = __float_as_uint(largest_of(v[q]));  // of a row: its lanes are 4 to 32 neighbours (not negative: floats compare as integers)
      x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));   // quad_perm: lane ^ 1
      x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));   // quad_perm: lane ^ 2
      if (kChunks >= 8) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));   // row_half_mirror: the other four
      if (kChunks >= 16) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, false));  // row_mirror: the other eight
      if (kChunks >= 32) x = __float_as_uint(max_over_16(__uint_as_float(x)));
      const Scale scale = scale_for(__uint_as_float(x));
      slot.put(row(q), chunk(), split8(v[q], sign * scale.to));
      if (chunk() == 0) slot.inv[row(q)] = scale.inv;
    }
  }
};

// A lane's 8 values, a hidden column in four lanes, as pieces; returns 1 over their scale.
__device__ inline float pieces_of(const float (&v)[8], Split *to) {
  const Scale scale = scale_for(max_over_32(max_over_16(largest_of(v))));
  *to = split8(v, scale.to);
  return scale.inv;
}

template <int ACT, int FD, int OD, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, FD + OD <= 4 ? 2 : 1) k_ff_kept_weights(FfArgs a) {
  constexpr int kThreads = WAVES * kWave;
  using ShareX = Share<FD, 0, kThreads>;
  using ShareDY = Share<OD, kTile * 4 * (FD + OD) <= kThreads ? kTile * 4 * FD : 0, kThreads>;
  constexpr int FS = FD < 4 ? FD : 4, OS = OD < 4 ? OD : 4;  // tiles of 32 columns whose gradients are accumulated here, from f0 and o0 on
  const int f0 = FD > FS ? blockIdx.z * FS : 0, o0 = OD > OS ? blockIdx.z * OS : 0;
  const bool mine_f = FD > FS || blockIdx.z == 0, mine_o = OD > OS || blockIdx.z == 0;
  __shared__ Slot<FD> xs[2];
  __shared__ Slot<OD> dys[2];
  const int lane = threadIdx.x & (kWave - 1), l = lane & 15, g = lane >> 4;
  const int hid = (blockIdx.x * WAVES + threadIdx.x / kWave) * 16 + l;  // this lane's hidden column; none: weights of 0
  const bool there = hid < a.hidden;

  Split wg[FD], wu[FD], wd[OD];
  float inv_g, inv_u, inv_d;  // 1 over the scales of the lane's column of Wg and Wu and row of Wd, which four lanes share
  const auto columns_of = [&](const float *W, int64_t ld, Split (&to)[FD], float *inv) {
    float v[FD][8], largest = 0.f;
#pragma unroll
    for (int q = 0; q < FD; ++q) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int f = 32 * q + 8 * g + j;
        v[q][j] = there && f < a.F ? W[f * ld + hid] : 0.f;
      }
      largest = largest_of(v[q], largest);
    }
    const Scale scale = scale_for(max_over_32(max_over_16(largest)));
    *inv = scale.inv;
#pragma unroll
    for (int q = 0; q < FD; ++q) to[q] = split8(v[q], scale.to);
  };
  columns_of(a.Wg, a.ldwg, wg, &inv_g);
  columns_of(a.Wu, a.ldwu, wu, &inv_u);
  {
    float v[OD][8], largest = 0.f;
#pragma unroll
    for (int q = 0; q < OD; ++q) {
      load8(v[q], a.Wd + (there ? hid : 0) * a.ldwd, 32 * q + 8 * g, there ? a.Fo : 0, false);
      largest = largest_of(v[q], largest);
    }
    const Scale scale = scale_for(max_over_32(max_over_16(largest)));
    inv_d = scale.inv;
#pragma unroll
    for (int q = 0; q < OD; ++q) wd[q] = split8(v[q], scale.to);
  }
  const float bg = there && a.bg ? a.bg[hid] : 0.f, bu = there && a.bu ? a.bu[hid] : 0.f;
  f32x4 dwg[2 * FS], dwu[2 * FS], dwd[2 * OS];  // dwd transposed: its rows are Y's columns
#pragma unroll
  for (int t = 0; t < 2 * FS; ++t) dwg[t] = dwu[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < 2 * OS; ++t) dwd[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  Total dbg, dbu, dbd[8];

  // the part's tiles, of each snapshot a whole number, and the place of the one that is loaded next
  const int64_t of_snapshot = ((int64_t)a.n + kTile - 1) / kTile, every = of_snapshot * a.k;
  const int64_t first = blockIdx.y * a.tiles_per_part, left = every - first, count = left < a.tiles_per_part ? left : a.tiles_per_part;
  int t = (int)(first / of_snapshot);
  int64_t i0 = first % of_snapshot * kTile, loaded = 0;
  ShareX x;
  ShareDY dy;
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
    if (blockIdx.x == 0 && blockIdx.z == 0 && ShareDY::there())
#pragma unroll
      for (int q = 0; q < ShareDY::kMine; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) dbd[j].add(dy.v[q][j]);
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
    int at = lane;
    if (FD + OD > 12) asm("" : "+v"(at));  // (where there are not the registers to keep what follows from the lane: places in LDS)
    Sums16 sg[2] = {no_sums16(), no_sums16()}, su[2] = {no_sums16(), no_sums16()}, sd[2] = {no_sums16(), no_sums16()};
    // an operand's loads are on the way while the one before is multiplied (one wave a SIMD waits for each of them otherwise)
    constexpr int kPlain = 2 * (FD + OD);
    const auto plain = [&](int p) { return p < 2 * FD ? X.plain(p % 2, p / 2, at) : dY.plain(p % 2, (p - 2 * FD) / 2, at); };
    Split now = plain(0);
#pragma unroll
    for (int p = 0; p < kPlain; ++p) {
      const Split next = plain(p + 1 < kPlain ? p + 1 : 0);
      if (p < 2 * FD) {
        add_product16(sg[p % 2], now, wg[p / 2]);
        add_product16(su[p % 2], now, wu[p / 2]);
      } else {
        add_product16(sd[p % 2], now, wd[(p - 2 * FD) / 2]);
      }
      now = next;
      __builtin_amdgcn_sched_barrier(0);
    }
    if (i + 1 < count) {
      lay_down((int)(i + 1) & 1, -sign);
      load_next();
    }
    // X and dY have this tile's sign
    const float sign_g = sign * inv_g, sign_u = sign * inv_u, sign_d = sign * inv_d;
    float vg[8], vu[8], vh[8], tile_g = 0.f, tile_u = 0.f;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const f32x4 inv_x = *reinterpret_cast<const f32x4 *>(X.inv + 16 * s + 4 * g), inv_dy = *reinterpret_cast<const f32x4 *>(dY.inv + 16 * s + 4 * g);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 4 * s + r;
        const float2 c = activate_slope<ACT>(fmaf(sum_of(sg[s], r), sign_g * inv_x[r], bg));
        const float u = fmaf(sum_of(su[s], r), sign_u * inv_x[r], bu), d = sum_of(sd[s], r) * (sign_d * inv_dy[r]);
        vg[j] = d * u * c.y;
        vu[j] = d * c.x;
        tile_g += vg[j];
        tile_u += vu[j];
        vg[j] *= inv_x[r];
        vu[j] *= inv_x[r];
        vh[j] = c.x * u * inv_dy[r];
      }
    }
    dbg.add(tile_g), dbu.add(tile_u);
    Split dg, du, hh;
    const float cg = sign * pieces_of(vg, &dg), cu = sign * pieces_of(vu, &du), ch = sign * pieces_of(vh, &hh);
    const auto add = [](f32x4 &to, float factor, const Sums16 &x) {
#pragma unroll
      for (int r = 0; r < 4; ++r) to[r] = fmaf(sum_of(x, r), factor, to[r]);
    };
    // likewise, and a product's sums are added while the next one is made
    constexpr int kTransposed = 2 * (FS + OS);
    const auto transposed = [&](int p) { return p < 2 * FS ? X.transposed(2 * f0 + p, at) : dY.transposed(2 * o0 + p - 2 * FS, at); };
    Sums16 sums[2];
    const auto add_sums = [&](int p) {
      if (p < 2 * FS) {
        add(dwg[p], cg, sums[0]);
        add(dwu[p], cu, sums[1]);
      } else {
        add(dwd[p - 2 * FS], ch, sums[0]);
      }
    };
    now = transposed(0);
#pragma unroll
    for (int p = 0; p < kTransposed; ++p) {
      const Split next = transposed(p + 1 < kTransposed ? p + 1 : 0);
      Sums16 made[2] = {no_sums16(), no_sums16()};
      add_product16(made[0], now, p < 2 * FS ? dg : hh);
      if (p < 2 * FS) add_product16(made[1], now, du);
      if (p > 0) add_sums(p - 1);
      sums[0] = made[0], sums[1] = made[1];
      now = next;
      __builtin_amdgcn_sched_barrier(0);
    }
    add_sums(kTransposed - 1);
    __syncthreads();
    sign = -sign;
  }

  float *const to = a.partial + blockIdx.y * a.part_floats, *const to_d = to + 2 * (int64_t)a.F * a.hidden, *const to_b = to_d + (int64_t)a.hidden * a.Fo;
  if (blockIdx.x == 0 && blockIdx.z == 0) {  // dbd: every thread has its columns' sums over its rows
    float *const sums = reinterpret_cast<float *>(dys);
    constexpr int kSets = (ShareDY::kMine > 1 ? kThreads : ShareDY::kUnits) / ShareDY::kChunks;  // threads that have a chunk of columns
    if (ShareDY::there())
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[ShareDY::me() / ShareDY::kChunks * 32 * OD + 8 * ShareDY::chunk() + j] = dbd[j].sum;
    __syncthreads();
    for (int c = threadIdx.x; c < a.Fo; c += kThreads) {
      float s = 0.f;
      for (int w = 0; w < kSets; ++w) s += sums[w * 32 * OD + c];
      to_b[2 * a.hidden + c] = s;
    }
  }
  // (all lanes have to take part before those without a column leave)
  const auto over_rows = [](float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
  };
  const float sum_g = over_rows(dbg.sum), sum_u = over_rows(dbu.sum);
  if (there) {
#pragma unroll
    for (int q = 0; q < 2 * FS; ++q)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int f = 32 * f0 + 16 * q + 4 * g + r;
        if (mine_f && f < a.F) {
          to[(int64_t)f * a.hidden + hid] = dwg[q][r];
          to[((int64_t)a.F + f) * a.hidden + hid] = dwu[q][r];
        }
      }
#pragma unroll
    for (int q = 0; q < 2 * OS; ++q)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int fo = 32 * o0 + 16 * q + 4 * g + r;
        if (mine_o && fo < a.Fo) to_d[(int64_t)hid * a.Fo + fo] = dwd[q][r];
      }
    if (g == 0 && blockIdx.z == 0) to_b[hid] = sum_g, to_b[a.hidden + hid] = sum_u;
  }
}

template <int ACT, int FD, int OD>
Kept kept_weights_of(int waves) {
  if constexpr (FD <= 2 && OD <= 2) {
    if (waves == 8) return {k_ff_kept_weights<ACT, FD, OD, 8>, 8};
  }
  return {k_ff_kept_weights<ACT, FD, OD, 4>, 4};
}
template <int ACT, int FD>
Kept kept_weights_of(int od, int waves) {
  switch (od) {
    case 1: return kept_weights_of<ACT, FD, 1>(waves);
    case 2: return kept_weights_of<ACT, FD, 2>(waves);
    case 4: return kept_weights_of<ACT, FD, 4>(waves);
    default: return kept_weights_of<ACT, FD, 8>(waves);
  }
}
template <int ACT>
Kept kept_weights_of(int fd, int od, int waves) {
  switch (fd) {
    case 1: return kept_weights_of<ACT, 1>(od, waves);
    case 2: return kept_weights_of<ACT, 2>(od, waves);
    case 4: return kept_weights_of<ACT, 4>(od, waves);
    default: return kept_weights_of<ACT, 8>(od, waves);
  }
}
}  // namespace

// (a source of its own for each activation: a quarter of the kernels each, compiled side by side)
template <>
Kept kept_weights<PIPAD_FF_ACT>(int fd, int od, int waves) {
  return kept_weights_of<PIPAD_FF_ACT>(fd, od, waves);
}

}  // namespace ff
}  // namespace pipad
