// The norms around a block of a model, fused with its gate and residual scale, and their gradients (pipad_residual_norm,
// pipad_residual_norm_backward in include/pipad.h).
//
//   P = post(B),  R' = R + scale * sigmoid(gate) * P,  Z = pre(R')       post, pre: none, root mean square, or layer norm
//
// Everything about a node row is local to the row but the gradients of the vectors that all rows share, so one pass over the
// matrices does it: a row lies in the registers of LPR lanes, its sums go over these lanes, and nothing is kept from the
// forward pass but R' itself.  What is read and written once is all that there is to move: 5 matrices forward, 8 backward.
// Memory bounds it: 8 million rows of 64, forward, 1.61 ms, 6.4 TB/s (a sum of two large arrays reaches 6.1); 4 million of 128, backward, 3.11 ms,
// 5.3 TB/s from five matrices to three; 150 thousand of 253, column by column, 5.2 TB/s.
#include "pipad_internal.h"

namespace pipad {

namespace {

struct NormArgs {
  const float *R[PIPAD_MAX_K], *B[PIPAD_MAX_K], *gate[PIPAD_MAX_K];      // R: R' in the backward pass
  const float *dRout[PIPAD_MAX_K], *dZ[PIPAD_MAX_K];                     // backward
  float *out0[PIPAD_MAX_K], *out1[PIPAD_MAX_K], *out2[PIPAD_MAX_K];      // R', Z; or dR, dB, dgate
  int64_t ldr, ldb, ldg, lddro, lddz, ld0, ld1, ld2;
  int64_t first;  // row of the launch's first workgroup
  int32_t n, F, post, pre;
  float eps, inv_f;
  const float *scale, *w_post, *b_post, *w_pre, *b_pre;
  bool has_b, has_gate, has_drout, has_dz, want0, want1, want2;
  float *partial;  // [block][kSums][F], or null
};

constexpr int kSums = 5;  // dscale, dw_post, db_post, dw_pre, db_pre

// Sum over the LPR lanes of a row, the same bits in all of them: lanes add what their neighbours have, quads, eights and sixteens what the mirror
// image has, by register moves (a row needs four such sums one after the other: through LDS they are 150 cycles and more each).  256: the whole
// workgroup, through `lds`, whose turns alternate between two halves so that one barrier a sum is enough.
template <int CTRL>
__device__ inline float plus_moved(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LPR>
__device__ inline float row_sum(float x, float *lds, int &turn) {
  if (LPR >= 2) x = plus_moved<0xb1>(x);    // quad_perm: lane ^ 1
  if (LPR >= 4) x = plus_moved<0x4e>(x);    // quad_perm: lane ^ 2
  if (LPR >= 8) x = plus_moved<0x141>(x);   // row_half_mirror
  if (LPR >= 16) x = plus_moved<0x140>(x);  // row_mirror
  if (LPR >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (LPR >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (LPR == 256) {
    float *const at = lds + 4 * turn;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
    __syncthreads();
    x = (at[0] + at[1]) + (at[2] + at[3]);
  }
  return x;
}

__device__ inline float sigmoid_of(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }

typedef float f32x4 __attribute__((ext_vector_type(4)));

// The columns of a lane: VEC consecutive ones, NV times, LPR * VEC apart.
template <int VEC, int LPR, int NV>
struct Row {
  static constexpr int kElems = VEC * NV;
  float v[kElems];
  __device__ static int column(int lane, int j) { return (j / VEC) * LPR * VEC + lane * VEC + j % VEC; }
  __device__ void fill(float x) {
#pragma unroll
    for (int j = 0; j < kElems; ++j) v[j] = x;
  }
  // Vectors, which all rows read, by ordinary loads; matrices in 16-byte pieces are read, and written, once: past the caches.  Column by column
  // the loads of a lane share cache lines with each other and with the next row's: 34 columns at 4.6 TB/s forward and 4.1 backward, past the
  // caches 3.4 and 2.9.
  template <bool ONCE = false>
  __device__ void load(const float *p, int lane, int F) {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int c = column(lane, q * VEC);
      if (VEC == 4) {
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
        if (c < F) t = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p + c)) : *reinterpret_cast<const f32x4 *>(p + c);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[q * VEC + e] = t[e];
      } else {
        v[q] = 0.f;
        if (c < F) v[q] = p[c];
      }
    }
  }
  __device__ void load_or(const float *p, int lane, int F, float otherwise) {
    if (p) load(p, lane, F);
    else fill(otherwise);
  }
  __device__ void store(float *p, int lane, int F) const {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int c = column(lane, q * VEC);
      if (c < F) {
        if (VEC == 4) {
          f32x4 t;
#pragma unroll
          for (int e = 0; e < VEC; ++e) t[e] = v[q * VEC + e];
          __builtin_nontemporal_store(t, reinterpret_cast<f32x4 *>(p + c));
        } else {
          p[c] = v[q];
        }
      }
    }
  }
};

// x becomes x normalised; columns that are not there stay 0.  Returns the factor.  The layer norm's variance is that of the
// centred values (a second pass over registers), never a difference of two large sums.
template <int VEC, int LPR, int NV>
__device__ inline float normalise(Row<VEC, LPR, NV> &x, int kind, int lane, int F, float inv_f, float eps, float *lds, int &turn) {
  constexpr int E = VEC * NV;
  if (kind == PIPAD_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < E; ++j) s += x.v[j];
    const float mean = row_sum<LPR>(s, lds, turn) * inv_f;
#pragma unroll
    for (int j = 0; j < E; ++j) x.v[j] = x.column(lane, j) < F ? x.v[j] - mean : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < E; ++j) s = fmaf(x.v[j], x.v[j], s);
  const float r = rsqrtf(fmaf(row_sum<LPR>(s, lds, turn), inv_f, eps));
#pragma unroll
  for (int j = 0; j < E; ++j) x.v[j] *= r;
  return r;
}

// d (the gradient of the normalised x) becomes that of what was normalised with factor r.
template <int VEC, int LPR, int NV>
__device__ inline void normalise_back(Row<VEC, LPR, NV> &d, const Row<VEC, LPR, NV> &x, float r, int kind, float inv_f, float *lds, int &turn) {
  constexpr int E = VEC * NV;
  float s = 0.f, m = 0.f;
#pragma unroll
  for (int j = 0; j < E; ++j) s = fmaf(d.v[j], x.v[j], s);
  s = row_sum<LPR>(s, lds, turn) * inv_f;
  if (kind == PIPAD_NORM_LAYER) {
#pragma unroll
    for (int j = 0; j < E; ++j) m += d.v[j];
    m = row_sum<LPR>(m, lds, turn) * inv_f;
  }
#pragma unroll
  for (int j = 0; j < E; ++j) d.v[j] = (d.v[j] - m - x.v[j] * s) * r;
}

template <int VEC, int LPR, int NV>
__global__ void __launch_bounds__(kBlock) k_residual_norm(NormArgs a) {
  using R = Row<VEC, LPR, NV>;
  constexpr int E = R::kElems, kRows = kBlock / LPR;
  __shared__ float lds[8];
  int turn = 0;
  const int lane = threadIdx.x % LPR, t = blockIdx.y, F = a.F;
  R scale, w_post, b_post, w_pre, b_pre;
  if (a.has_b) {
    scale.load_or(a.scale, lane, F, 1.f);
    w_post.load_or(a.w_post, lane, F, 1.f);
    b_post.load_or(a.b_post, lane, F, 0.f);
  }
  if (a.want1) {
    w_pre.load_or(a.w_pre, lane, F, 1.f);
    b_pre.load_or(a.b_pre, lane, F, 0.f);
  }
  const int64_t i = a.first + (int64_t)blockIdx.x * kRows + threadIdx.x / LPR;
  if (i >= a.n) return;  // (with LPR == 256 all of a workgroup's threads, else all lanes of a row)
  {
    R r, p, gate;
    r.template load<true>(a.R[t] + i * a.ldr, lane, F);
    if (a.has_b) {
      p.template load<true>(a.B[t] + i * a.ldb, lane, F);
      if (a.has_gate) gate.template load<true>(a.gate[t] + i * a.ldg, lane, F);
      if (a.post != PIPAD_NORM_NONE) {
        normalise(p, a.post, lane, F, a.inv_f, a.eps, lds, turn);
#pragma unroll
        for (int j = 0; j < E; ++j) p.v[j] = fmaf(p.v[j], w_post.v[j], b_post.v[j]);
      }
      if (a.has_gate) {
#pragma unroll
        for (int j = 0; j < E; ++j) p.v[j] *= sigmoid_of(gate.v[j]);
      }
#pragma unroll
      for (int j = 0; j < E; ++j) r.v[j] = r.column(lane, j) < F ? fmaf(scale.v[j], p.v[j], r.v[j]) : 0.f;
      if (a.want0) r.store(a.out0[t] + i * a.ld0, lane, F);
    }
    if (a.want1) {
      normalise(r, a.pre, lane, F, a.inv_f, a.eps, lds, turn);
#pragma unroll
      for (int j = 0; j < E; ++j) r.v[j] = fmaf(r.v[j], w_pre.v[j], b_pre.v[j]);
      r.store(a.out1[t] + i * a.ld1, lane, F);
    }
  }
}

// The sums over all rows: every lane adds up those of its rows, then the lanes of one column are added, within the waves and then over them, in a
// fixed order, and go to the workgroup's own place in `partial`; k_norm_sums adds the workgroups.
template <int VEC, int LPR, int NV>
__global__ void __launch_bounds__(kBlock) k_residual_norm_backward(NormArgs a) {
  using R = Row<VEC, LPR, NV>;
  constexpr int E = R::kElems, kRows = kBlock / LPR;
  constexpr bool kAhead = E <= 4;  // a row's loads are on the way while the one before is computed
  __shared__ float lds[8];
  __shared__ float sums[2][kWavesPerBlock][LPR < 256 ? E * LPR : 1];  // (more than one row a workgroup; in turns: one barrier a sum)
  int turn = 0;
  const int lane = threadIdx.x % LPR, t = blockIdx.y, F = a.F;
  R scale, w_post, b_post, w_pre, acc[kSums], rest[kSums];
  scale.load_or(a.scale, lane, F, 1.f);
  w_post.load_or(a.w_post, lane, F, 1.f);
  b_post.load_or(a.b_post, lane, F, 0.f);
  w_pre.load_or(a.w_pre, lane, F, 1.f);
#pragma unroll
  for (int q = 0; q < kSums; ++q) acc[q].fill(0.f), rest[q].fill(0.f);
  // A plain chain of additions would be off by more the more rows a lane has (4 million rows of 128: 3.5e-7 of the sums' size, so 1.4e-7).  A sum of few
  // columns a lane carries what its additions round off, in `rest`, at no cost; of more columns, whose registers are short, 64 rows are added up by
  // themselves and then to `rest` (256 MB a matrix, as plain chains, so, and carried: 512 columns 398, 420 and 422 us, 1022 columns 612, 621 and 663,
  // 4096 columns 632, 595 and 636, 4094 columns 687, 760 and 813).
  constexpr bool kCarry = E <= 4;
  constexpr int kChain = 64;
  int chain = 0;
  const auto add = [&](int q, int j, float x, float y) {
    float &sum = acc[q].v[j], &lost = rest[q].v[j];
    if (!kCarry) {
      sum = fmaf(x, y, sum);
      return;
    }
    const float z = fmaf(x, y, -lost), s = sum + z;
    lost = (s - sum) - z;
    sum = s;
  };
  const auto end_chain = [&] {
#pragma unroll
    for (int q = 0; q < kSums; ++q)
#pragma unroll
      for (int j = 0; j < E; ++j) rest[q].v[j] += acc[q].v[j], acc[q].v[j] = 0.f;
    chain = 0;
  };
  struct Loaded {
    R b, gate, g, x, d;
  };
  const auto load = [&](Loaded &q, int64_t i) {
    if (a.has_b) q.b.template load<true>(a.B[t] + i * a.ldb, lane, F);
    if (a.has_gate) q.gate.template load<true>(a.gate[t] + i * a.ldg, lane, F);
    if (a.has_drout) q.g.template load<true>(a.dRout[t] + i * a.lddro, lane, F);
    else q.g.fill(0.f);
    if (a.has_dz) {
      q.x.template load<true>(a.R[t] + i * a.ldr, lane, F);
      q.d.template load<true>(a.dZ[t] + i * a.lddz, lane, F);
    }
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t i = (int64_t)blockIdx.x * kRows + threadIdx.x / LPR;
  Loaded next;
  if (kAhead && i < a.n) load(next, i);
  for (; i < a.n; i += step) {
    if (!kAhead) load(next, i);
    R d = next.d, b = next.b, gate = next.gate, g = next.g, x = next.x;
    if (kAhead && i + step < a.n) load(next, i + step);
    if (a.has_dz) {
      const float r = normalise(x, a.pre, lane, F, a.inv_f, a.eps, lds, turn);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        add(3, j, d.v[j], x.v[j]);
        add(4, j, d.v[j], 1.f);
        d.v[j] *= w_pre.v[j];
      }
      normalise_back(d, x, r, a.pre, a.inv_f, lds, turn);
#pragma unroll
      for (int j = 0; j < E; ++j) g.v[j] += d.v[j];
    }
    if (a.want0) g.store(a.out0[t] + i * a.ld0, lane, F);
    if (a.has_b) {
      float r = 1.f;
      if (a.post != PIPAD_NORM_NONE) r = normalise(b, a.post, lane, F, a.inv_f, a.eps, lds, turn);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const float p = a.post != PIPAD_NORM_NONE ? fmaf(b.v[j], w_post.v[j], b_post.v[j]) : b.v[j];
        float gs = g.v[j] * scale.v[j];
        if (a.has_gate) {
          // (1 - sigmoid) from the same exponential: their difference would lose it where the gate is wide open
          const float e = __expf(-fabsf(gate.v[j])), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
          const float sig = gate.v[j] >= 0.f ? big : small;
          add(0, j, g.v[j], sig * p);
          gate.v[j] = gs * p * big * small;
          gs *= sig;
        } else {
          add(0, j, g.v[j], p);
        }
        d.v[j] = gs;
      }
      if (a.has_gate && a.want2) gate.store(a.out2[t] + i * a.ld2, lane, F);
      if (a.post != PIPAD_NORM_NONE) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
          add(1, j, d.v[j], b.v[j]);
          add(2, j, d.v[j], 1.f);
          d.v[j] = d.column(lane, j) < F ? d.v[j] * w_post.v[j] : 0.f;
        }
        normalise_back(d, b, r, a.post, a.inv_f, lds, turn);
      }
      if (a.want1) d.store(a.out1[t] + i * a.ld1, lane, F);
    }
    if (!kCarry && ++chain == kChain) end_chain();
  }
  if (!a.partial) return;
  if (!kCarry) end_chain();
  const R *const total = kCarry ? acc : rest;
  float *const to = a.partial + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kSums * F;
#pragma unroll
  for (int q = 0; q < kSums; ++q) {
    if (LPR == 256) {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (total[q].column(lane, j) < F) to[q * F + total[q].column(lane, j)] = total[q].v[j];
      continue;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
      float x = total[q].v[j];
#pragma unroll
      for (int d = LPR; d < kWave; d *= 2) x += __shfl_xor(x, d);
      if (threadIdx.x % kWave < LPR) sums[q & 1][threadIdx.x / kWave][total[q].column(lane, j)] = x;
    }
    __syncthreads();
    const auto &of = sums[q & 1];
    for (int c = threadIdx.x; c < F; c += kBlock) to[q * F + c] = (of[0][c] + of[1][c]) + (of[2][c] + of[3][c]);
  }
}

struct SumOut {
  float *out[kSums];
};
// out[q][c] = the sum of the workgroups' partial[.][q][c], always in the same order: 64 of its lanes take every 64th each.
constexpr int kSumThreads = 1024, kSumLanes = kSumThreads / 16;
__global__ void __launch_bounds__(kSumThreads) k_norm_sums(const float *partial, int64_t count, int32_t F, SumOut o) {
  __shared__ float part[kSumLanes][17];
  const int x = threadIdx.x % 16, y = threadIdx.x / 16;
  const int64_t c = (int64_t)blockIdx.x * 16 + x, columns = (int64_t)kSums * F;
  float s[8] = {};
  if (c < columns) {
    int64_t b = y;
    for (; b + 7 * kSumLanes < count; b += 8 * kSumLanes) {
#pragma unroll
      for (int u = 0; u < 8; ++u) s[u] += partial[(b + kSumLanes * u) * columns + c];
    }
    for (; b < count; b += kSumLanes) s[0] += partial[b * columns + c];
  }
  part[y][x] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
  for (int d = kSumLanes / 2; d >= 1; d /= 2) {
    __syncthreads();
    if (y < d) part[y][x] += part[y + d][x];
  }
  if (y != 0 || c >= columns) return;
  const int q = (int)(c / F);
  if (o.out[q]) o.out[q][c - (int64_t)q * F] = part[0][x];
}

using NormKernel = void (*)(NormArgs);
struct NormPlan {
  NormKernel forward, backward;
  int lanes;  // of a row: LPR
};

template <int VEC, int LPR, int NV>
NormPlan plan_of() {
  return {k_residual_norm<VEC, LPR, NV>, k_residual_norm_backward<VEC, LPR, NV>, LPR};
}

// In 16-byte pieces the fewest lanes that hold a row with one load each, up to a wave; then up to four pieces a lane; then the whole workgroup.
// `vec`: every row of the call starts on 16 bytes and is a multiple of 4 long.  Others go column by column (150 thousand rows of 253 took
// 118 us so and 155 in 16-byte pieces off their boundaries), two to four columns a lane: what a row costs is mostly its sums over lanes,
// so that few lanes idle and several rows share a wave.  256 MB a matrix, with one column a lane up to 64: 3 columns 395 us forward and 569
// backward, now 292 and 451; 17 columns 583 and 908, now 293 and 549; 34 columns 603 and 948, now 278 and 531.
NormPlan plan(int32_t F, bool vec) {
  if (vec) {
    if (F <= 4) return plan_of<4, 1, 1>();
    if (F <= 8) return plan_of<4, 2, 1>();
    if (F <= 16) return plan_of<4, 4, 1>();
    if (F <= 32) return plan_of<4, 8, 1>();
    if (F <= 64) return plan_of<4, 16, 1>();
    if (F <= 128) return plan_of<4, 32, 1>();
    if (F <= 256) return plan_of<4, 64, 1>();
    if (F <= 512) return plan_of<4, 64, 2>();
    if (F <= 1024) return plan_of<4, 64, 4>();
    return plan_of<4, 256, 4>();
  }
  if (F <= 1) return plan_of<1, 1, 1>();
  if (F <= 2) return plan_of<1, 1, 2>();
  if (F <= 4) return plan_of<1, 2, 2>();
  if (F <= 8) return plan_of<1, 4, 2>();
  if (F <= 12) return plan_of<1, 4, 3>();
  if (F <= 16) return plan_of<1, 8, 2>();
  if (F <= 24) return plan_of<1, 8, 3>();
  if (F <= 32) return plan_of<1, 16, 2>();
  if (F <= 48) return plan_of<1, 16, 3>();
  if (F <= 64) return plan_of<1, 16, 4>();
  if (F <= 96) return plan_of<1, 32, 3>();
  if (F <= 128) return plan_of<1, 32, 4>();
  if (F <= 256) return plan_of<1, 64, 4>();
  if (F <= 512) return plan_of<1, 64, 8>();
  if (F <= 1024) return plan_of<1, 64, 16>();
  return plan_of<1, 256, 16>();
}

bool aligned(const float *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 4 == 0; }

// Workgroups a snapshot.  Forward: one for every kBlock / lanes rows, which keeps more loads on the way than fewer that go on and on (8 million rows
// of 64: 1.67 ms, 2.00 with 2048).  Backward, where each has partial sums: at most 2048 over all snapshots
// (4 million rows of 128: 3.18 ms with 1024, 3.13 with 2048, 3.22 with 4096).
constexpr int kMostGroups = 2048;
int64_t all_groups(int32_t n, int lanes) {
  const int64_t rows = kBlock / lanes;
  return ((int64_t)n + rows - 1) / rows;
}
int64_t groups(int32_t n, int32_t k, int lanes) { return std::max<int64_t>(1, std::min<int64_t>(all_groups(n, lanes), (kMostGroups + k - 1) / k)); }

}  // namespace

size_t residual_norm_workspace(int32_t F, int32_t n, int32_t k) {
  if (n == 0) return 0;
  // (the rows' alignment is not known here: the more workgroups)
  return (size_t)std::max(groups(n, k, plan(F, true).lanes), groups(n, k, plan(F, false).lanes)) * k * kSums * F * sizeof(float);
}

// Returns whether every row is one for 16-byte pieces.
static bool fill(NormArgs *a, const pipad_residual_norm_t &c, int32_t n, int32_t k, const NormRows &m) {
  a->n = n, a->F = c.F, a->post = c.post, a->pre = c.pre, a->eps = c.eps, a->inv_f = 1.f / (float)c.F;
  a->scale = c.scale, a->w_post = c.w_post, a->b_post = c.b_post, a->w_pre = c.w_pre, a->b_pre = c.b_pre;
  a->has_b = m.B != nullptr, a->has_gate = m.gate != nullptr, a->has_drout = m.dRout != nullptr, a->has_dz = m.dZ != nullptr;
  a->want0 = m.out0 != nullptr, a->want1 = m.out1 != nullptr, a->want2 = m.out2 != nullptr;
  a->ldr = m.ldr, a->ldb = m.ldb, a->ldg = m.ldg, a->lddro = m.lddro, a->lddz = m.lddz, a->ld0 = m.ld0, a->ld1 = m.ld1, a->ld2 = m.ld2;
  bool vec = c.F % 4 == 0;
  for (const float *v : {c.scale, c.w_post, c.b_post, c.w_pre, c.b_pre}) vec = vec && aligned(v, 0);
  const auto take = [&](auto *const *from, auto *to, int64_t ld) {
    for (int t = 0; from && t < k; ++t) {
      to[t] = from[t];
      vec = vec && aligned(from[t], ld);
    }
  };
  take(m.R, a->R, m.ldr), take(m.B, a->B, m.ldb), take(m.gate, a->gate, m.ldg), take(m.dRout, a->dRout, m.lddro), take(m.dZ, a->dZ, m.lddz);
  take(m.out0, a->out0, m.ld0), take(m.out1, a->out1, m.ld1), take(m.out2, a->out2, m.ld2);
  return vec;
}

int residual_norm_launch(const pipad_residual_norm_t &c, int32_t n, int32_t k, const NormRows &m, hipStream_t st) {
  NormArgs a{};
  const NormPlan p = plan(c.F, fill(&a, c, n, k, m));
  constexpr int64_t kMostLaunched = (int64_t)1 << 22;  // (a launch has fewer than 2^32 threads along x)
  const int64_t all = all_groups(n, p.lanes);
  for (int64_t at = 0; at < all; at += kMostLaunched) {
    a.first = at * (kBlock / p.lanes);
    hipLaunchKernelGGL(p.forward, dim3((unsigned)std::min(all - at, kMostLaunched), (unsigned)k), dim3(kBlock), 0, st, a);
    PIPAD_HIP(hipGetLastError());
  }
  return PIPAD_OK;
}

int residual_norm_backward_launch(const pipad_residual_norm_t &c, int32_t n, int32_t k, const NormRows &m, float *const (&sums)[5], void *workspace,
                                  hipStream_t st) {
  bool any = false;
  SumOut o{};
  for (int q = 0; q < kSums; ++q) {
    o.out[q] = sums[q];
    any = any || sums[q];
  }
  int64_t count = 0;
  if (n > 0) {
    NormArgs a{};
    const NormPlan p = plan(c.F, fill(&a, c, n, k, m));
    const int64_t g = groups(n, k, p.lanes);
    a.partial = any ? static_cast<float *>(workspace) : nullptr;
    count = g * k;
    hipLaunchKernelGGL(p.backward, dim3((unsigned)g, (unsigned)k), dim3(kBlock), 0, st, a);
    PIPAD_HIP(hipGetLastError());
  }
  if (any) {
    hipLaunchKernelGGL(k_norm_sums, dim3((unsigned)((kSums * (int64_t)c.F + 15) / 16)), dim3(kSumThreads), 0, st,
                       static_cast<const float *>(workspace), count, c.F, o);
    PIPAD_HIP(hipGetLastError());
  }
  return PIPAD_OK;
}

}  // namespace pipad
