// C ABI of libpipad: argument checks and dispatch.  See include/pipad.h for the contract.
#include <cstdio>
#include <cstring>
#include <string>

#include "pipad_internal.h"

namespace pipad {

static thread_local std::string g_hip_error;

int hip_fail(hipError_t e, const char *what) {
  g_hip_error = std::string(hipGetErrorString(e)) + " in " + what;
  (void)hipGetLastError();  // clear the sticky error so that later calls are not blamed
  return PIPAD_ERR_HIP;
}

Options &options() {
  static Options o;
  return o;
}

int build_overlap(int32_t n, int32_t k, const pipad_csr_t *snaps, uint32_t flags,
                  pipad_alloc_fn alloc, void *alloc_ctx, hipStream_t st, pipad_frame **out);
void destroy_frame(pipad_frame *f);
int transpose_frame(const pipad_frame *f, pipad_alloc_fn alloc, void *alloc_ctx, hipStream_t st,
                    pipad_frame **out);

// k matrices of n rows of F columns: PIPAD_OK, or what is wrong with them.  `at` null where that is allowed is not looked at.
template <class T>
static int check_rows(int32_t n, int32_t k, int32_t F, T *const *at, int64_t ld) {
  if (!at || ld < F) return PIPAD_ERR_INVALID_ARG;
  if (n > 0)
    for (int t = 0; t < k; ++t)
      if (!at[t]) return PIPAD_ERR_INVALID_ARG;
  return (int64_t)n * ld >= (int64_t)1 << 40 || ld >= (int64_t)1 << 40 ? PIPAD_ERR_TOO_LARGE : PIPAD_OK;
}

}  // namespace pipad

extern "C" {

int pipad_frame_build_overlap(int32_t n, int32_t k, const pipad_csr_t *snaps, uint32_t flags,
                              pipad_alloc_fn alloc, void *alloc_ctx, void *stream,
                              pipad_frame_t **out) {
  if (!out || !snaps || n < 0 || k < 1 || k > PIPAD_MAX_K) return PIPAD_ERR_INVALID_ARG;
  if (flags & ~PIPAD_VALIDATE) return PIPAD_ERR_INVALID_ARG;
  for (int t = 0; t < k; ++t) {
    if (snaps[t].n != n || snaps[t].nnz < 0 || !snaps[t].rowptr) return PIPAD_ERR_INVALID_ARG;
    if (snaps[t].nnz > 0 && !snaps[t].colidx) return PIPAD_ERR_INVALID_ARG;
    if (n == 0 && snaps[t].nnz != 0) return PIPAD_ERR_INVALID_ARG;
  }
  pipad_frame *f = nullptr;
  const int rc = pipad::build_overlap(n, k, snaps, flags, alloc, alloc_ctx,
                                      static_cast<hipStream_t>(stream), &f);
  if (rc != PIPAD_OK) return rc;
  *out = f;
  return PIPAD_OK;
}

int pipad_frame_common(const pipad_frame_t *f, pipad_csr_t *view) {
  if (!f || !view) return PIPAD_ERR_INVALID_ARG;
  view->n = f->n;
  view->nnz = f->nnz_c;
  view->rowptr = f->rowptr_c;
  view->colidx = f->col_c;
  return PIPAD_OK;
}

int pipad_frame_delta(const pipad_frame_t *f, int32_t t, pipad_csr_t *view) {
  if (!f || !view || t < 0 || t >= f->k) return PIPAD_ERR_INVALID_ARG;
  view->n = f->n;
  view->nnz = f->nnz_d[t];
  view->rowptr = f->rowptr_d[t];
  view->colidx = f->col_d[t];
  return PIPAD_OK;
}

int pipad_frame_dinv(const pipad_frame_t *f, const float **dinv, int64_t *ld_node,
                     int64_t *ld_snap) {
  if (!f || !dinv || !ld_node || !ld_snap) return PIPAD_ERR_INVALID_ARG;
  *dinv = f->dinv;
  *ld_node = 1;
  *ld_snap = f->n;
  return PIPAD_OK;
}

int pipad_frame_shape(const pipad_frame_t *f, int32_t *n, int32_t *k) {
  if (!f) return PIPAD_ERR_INVALID_ARG;
  if (n) *n = f->n;
  if (k) *k = f->k;
  return PIPAD_OK;
}

int pipad_frame_aggregate(pipad_frame_t *frame, int32_t F, const float *const *X, int64_t ldx,
                          float *const *Y, int64_t ldy, void *stream) {
  if (!frame || !X || !Y || F < 1 || ldx < F || ldy < F) return PIPAD_ERR_INVALID_ARG;
  if (frame->n > 0)
    for (int t = 0; t < frame->k; ++t)
      if (!X[t] || !Y[t]) return PIPAD_ERR_INVALID_ARG;
  if ((int64_t)frame->n * ldx >= ((int64_t)1 << 40) || (int64_t)frame->n * ldy >= ((int64_t)1 << 40))
    return PIPAD_ERR_TOO_LARGE;
  if (frame->n > 0) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return pipad::hip_fail(hipGetLastError(), "hipGetDevice");
    if (dev != frame->device) return PIPAD_ERR_INVALID_ARG;  // frames are tied to their GPU
  }
  // the frame's scratch buffers are the only state an aggregation changes
  return pipad::aggregate_launch(frame, F, X, ldx, Y, ldy, static_cast<hipStream_t>(stream),
                                 pipad::ScratchRef{&frame->partial, &frame->partial_floats, frame});
}

int pipad_frame_aggregate_subset(pipad_frame_t *frame, int32_t nsel, const int32_t *snapshots,
                                 int32_t F, const float *const *X, int64_t ldx, float *const *Y,
                                 int64_t ldy, void *stream) {
  if (!frame || !X || !Y || F < 1 || ldx < F || ldy < F || nsel < 0 || nsel > frame->k ||
      (nsel > 0 && !snapshots))
    return PIPAD_ERR_INVALID_ARG;
  uint32_t seen = 0;
  for (int q = 0; q < nsel; ++q) {
    const int32_t t = snapshots[q];
    if (t < 0 || t >= frame->k || (seen >> t & 1u)) return PIPAD_ERR_INVALID_ARG;
    seen |= 1u << t;
    if (frame->n > 0 && (!X[t] || !Y[t])) return PIPAD_ERR_INVALID_ARG;
  }
  if ((int64_t)frame->n * ldx >= ((int64_t)1 << 40) || (int64_t)frame->n * ldy >= ((int64_t)1 << 40))
    return PIPAD_ERR_TOO_LARGE;
  if (frame->n == 0 || nsel == 0) return PIPAD_OK;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return pipad::hip_fail(hipGetLastError(), "hipGetDevice");
  if (dev != frame->device) return PIPAD_ERR_INVALID_ARG;
  // the aggregation only ever looks at the pointers of the chosen snapshots
  const float *xs[PIPAD_MAX_K] = {};
  float *ys[PIPAD_MAX_K] = {};
  for (int q = 0; q < nsel; ++q) {
    xs[snapshots[q]] = X[snapshots[q]];
    ys[snapshots[q]] = Y[snapshots[q]];
  }
  return pipad::aggregate_launch(frame, F, xs, ldx, ys, ldy, static_cast<hipStream_t>(stream),
                                 pipad::ScratchRef{&frame->partial, &frame->partial_floats, frame},
                                 nullptr, snapshots, nsel);
}

int pipad_frame_aggregate_static(const pipad_frame_t *frame, int32_t F, const float *const *X,
                                 int64_t ldx, float *const *Y, int64_t ldy, void *stream) {
  if (!frame || !X || !Y || F < 1 || ldx < F || ldy < F) return PIPAD_ERR_INVALID_ARG;
  if (frame->n > 0)
    for (int t = 0; t < frame->k; ++t)
      if (!X[t] || !Y[t]) return PIPAD_ERR_INVALID_ARG;
  if ((int64_t)frame->n * ldx >= ((int64_t)1 << 40) || (int64_t)frame->n * ldy >= ((int64_t)1 << 40))
    return PIPAD_ERR_TOO_LARGE;
  if (frame->n == 0) return PIPAD_OK;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return pipad::hip_fail(hipGetLastError(), "hipGetDevice");
  if (dev != frame->device) return PIPAD_ERR_INVALID_ARG;
  float *scratch_ptr = nullptr;
  size_t scratch_floats = 0;
  const int rc = pipad::static_scratch(&scratch_ptr, &scratch_floats);
  if (rc != PIPAD_OK) return rc;
  return pipad::aggregate_launch(frame, F, X, ldx, Y, ldy, static_cast<hipStream_t>(stream),
                                 pipad::ScratchRef{&scratch_ptr, &scratch_floats, nullptr});
}

int pipad_frame_aggregate_update(pipad_frame_t *frame, int32_t F, const float *const *X,
                                 int64_t ldx, const float *W, int64_t ldw, const float *bias,
                                 int32_t Fo, float *const *A, int64_t lda, float *const *H,
                                 int64_t ldh, void *stream) {
  if (!frame || !X || !H || !W || F < 1 || Fo < 1 || ldx < F || ldw < Fo || ldh < Fo)
    return PIPAD_ERR_INVALID_ARG;
  if (A && lda < F) return PIPAD_ERR_INVALID_ARG;
  if (frame->n > 0)
    for (int t = 0; t < frame->k; ++t)
      if (!X[t] || !H[t] || (A && !A[t])) return PIPAD_ERR_INVALID_ARG;
  const int64_t lim = (int64_t)1 << 40;
  if ((int64_t)frame->n * ldx >= lim || (int64_t)frame->n * ldh >= lim ||
      (A && (int64_t)frame->n * lda >= lim))
    return PIPAD_ERR_TOO_LARGE;
  if (frame->n > 0) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return pipad::hip_fail(hipGetLastError(), "hipGetDevice");
    if (dev != frame->device) return PIPAD_ERR_INVALID_ARG;
  }
  pipad::UpdateSpec u{W, ldw, bias, Fo, H, ldh};
  return pipad::aggregate_launch(frame, F, X, ldx, A, A ? lda : F, static_cast<hipStream_t>(stream),
                                 pipad::ScratchRef{&frame->partial, &frame->partial_floats, frame}, &u);
}

int pipad_frame_transpose(const pipad_frame_t *frame, pipad_alloc_fn alloc, void *alloc_ctx,
                          void *stream, pipad_frame_t **out) {
  if (!frame || !out) return PIPAD_ERR_INVALID_ARG;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return pipad::hip_fail(hipGetLastError(), "hipGetDevice");
  if (dev != frame->device) return PIPAD_ERR_INVALID_ARG;
  pipad_frame *g = nullptr;
  const int rc = pipad::transpose_frame(frame, alloc, alloc_ctx, static_cast<hipStream_t>(stream), &g);
  if (rc != PIPAD_OK) return rc;
  *out = g;
  return PIPAD_OK;
}

// ---- operators on node rows ---------------------------------------------------------------------
#define PIPAD_ROWS(F, at, ld)                                     \
  do {                                                            \
    const int rc__ = pipad::check_rows(n, k, (F), (at), (ld));           \
    if (rc__ != PIPAD_OK) return rc__;                            \
  } while (0)

static int check_norm(const pipad_residual_norm_t *c, int32_t n, int32_t k, bool has_b, bool has_gate) {
  if (!c || n < 0 || k < 1 || k > PIPAD_MAX_K || c->F < 1 || !(c->eps >= 0.f)) return PIPAD_ERR_INVALID_ARG;
  for (int32_t kind : {c->post, c->pre})
    if (kind != PIPAD_NORM_NONE && kind != PIPAD_NORM_RMS && kind != PIPAD_NORM_LAYER) return PIPAD_ERR_INVALID_ARG;
  if (c->post == PIPAD_NORM_NONE && (c->w_post || c->b_post)) return PIPAD_ERR_INVALID_ARG;
  if (c->pre == PIPAD_NORM_NONE && (c->w_pre || c->b_pre)) return PIPAD_ERR_INVALID_ARG;
  if (!has_b && (has_gate || c->scale || c->post != PIPAD_NORM_NONE)) return PIPAD_ERR_INVALID_ARG;
  return c->F > PIPAD_NORM_MAX_F ? PIPAD_ERR_TOO_LARGE : PIPAD_OK;
}

static int check_workspace(const void *workspace, size_t have, size_t need) {
  if (need == 0) return PIPAD_OK;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return PIPAD_ERR_INVALID_ARG;
  return have < need ? PIPAD_ERR_SCRATCH : PIPAD_OK;
}

int pipad_residual_norm(const pipad_residual_norm_t *norm, int32_t n, int32_t k, const float *const *R, int64_t ldr,
                        const float *const *B, int64_t ldb, const float *const *gate, int64_t ldg, float *const *R_out,
                        int64_t ldro, float *const *Z, int64_t ldz, void *stream) {
  int rc = check_norm(norm, n, k, B != nullptr, gate != nullptr);
  if (rc != PIPAD_OK) return rc;
  if ((!R_out && !Z) || (R_out && !B) || (Z && norm->pre == PIPAD_NORM_NONE)) return PIPAD_ERR_INVALID_ARG;
  PIPAD_ROWS(norm->F, R, ldr);
  if (B) PIPAD_ROWS(norm->F, B, ldb);
  if (gate) PIPAD_ROWS(norm->F, gate, ldg);
  if (R_out) PIPAD_ROWS(norm->F, R_out, ldro);
  if (Z) PIPAD_ROWS(norm->F, Z, ldz);
  if (n == 0) return PIPAD_OK;
  return pipad::residual_norm_launch(*norm, n, k, pipad::NormRows{R, B, gate, nullptr, nullptr, R_out, Z, nullptr, ldr, ldb, ldg, 0, 0, ldro, ldz, 0},
                                     static_cast<hipStream_t>(stream));
}

int pipad_residual_norm_workspace(int32_t F, int32_t n, int32_t k, size_t *bytes) {
  if (!bytes || F < 1 || n < 0 || k < 1 || k > PIPAD_MAX_K) return PIPAD_ERR_INVALID_ARG;
  if (F > PIPAD_NORM_MAX_F) return PIPAD_ERR_TOO_LARGE;
  *bytes = pipad::residual_norm_workspace(F, n, k);
  return PIPAD_OK;
}

int pipad_residual_norm_backward(const pipad_residual_norm_t *norm, int32_t n, int32_t k, const float *const *R, int64_t ldr,
                                 const float *const *B, int64_t ldb, const float *const *gate, int64_t ldg,
                                 const float *const *dR_out, int64_t lddro, const float *const *dZ, int64_t lddz,
                                 float *const *dR, int64_t lddr, float *const *dB, int64_t lddb, float *const *dgate,
                                 int64_t lddg, const pipad_residual_norm_grads_t *grads, void *workspace,
                                 size_t workspace_bytes, void *stream) {
  int rc = check_norm(norm, n, k, B != nullptr, gate != nullptr);
  if (rc != PIPAD_OK) return rc;
  if ((!dR_out && !dZ) || (dZ && norm->pre == PIPAD_NORM_NONE) || (dB && !B) || (dgate && !gate) || (!dR && !dB && !dgate && !grads))
    return PIPAD_ERR_INVALID_ARG;
  PIPAD_ROWS(norm->F, R, ldr);
  if (B) PIPAD_ROWS(norm->F, B, ldb);
  if (gate) PIPAD_ROWS(norm->F, gate, ldg);
  if (dR_out) PIPAD_ROWS(norm->F, dR_out, lddro);
  if (dZ) PIPAD_ROWS(norm->F, dZ, lddz);
  if (dR) PIPAD_ROWS(norm->F, dR, lddr);
  if (dB) PIPAD_ROWS(norm->F, dB, lddb);
  if (dgate) PIPAD_ROWS(norm->F, dgate, lddg);
  float *sums[5] = {};
  if (grads) {
    if ((rc = check_workspace(workspace, workspace_bytes, pipad::residual_norm_workspace(norm->F, n, k))) != PIPAD_OK) return rc;
    sums[0] = grads->dscale, sums[1] = grads->dw_post, sums[2] = grads->db_post, sums[3] = grads->dw_pre, sums[4] = grads->db_pre;
  }
  return pipad::residual_norm_backward_launch(*norm, n, k,
                                              pipad::NormRows{R, B, gate, dR_out, dZ, dR, dB, dgate, ldr, ldb, ldg, lddro, lddz, lddr, lddb, lddg},
                                              sums, workspace, static_cast<hipStream_t>(stream));
}

static int check_ff_sizes(const pipad_gated_ff_t *c, int32_t n, int32_t k) {
  if (!c || n < 0 || k < 1 || k > PIPAD_MAX_K || c->F < 1 || c->hidden < 1 || c->Fo < 1) return PIPAD_ERR_INVALID_ARG;
  if (c->activation < PIPAD_ACT_SIGMOID || c->activation > PIPAD_ACT_SILU) return PIPAD_ERR_INVALID_ARG;
  const int32_t lim = 1 << 16;
  const bool many = (int64_t)n * k > (int64_t)1 << (c->F > 256 || c->Fo > 256 ? 28 : 30);  // (rows that a launch's threads can be counted for)
  return many || c->F >= lim || c->hidden >= lim || c->Fo >= lim ? PIPAD_ERR_TOO_LARGE : PIPAD_OK;
}
static int check_ff(const pipad_gated_ff_t *c, int32_t n, int32_t k) {
  const int rc = check_ff_sizes(c, n, k);
  if (rc != PIPAD_OK) return rc;
  if (!c->Wg || !c->Wu || !c->Wd || c->ldwg < c->hidden || c->ldwu < c->hidden || c->ldwd < c->Fo) return PIPAD_ERR_INVALID_ARG;
  const int64_t lim = (int64_t)1 << 40;
  return c->ldwg >= lim || c->ldwu >= lim || c->ldwd >= lim ? PIPAD_ERR_TOO_LARGE : PIPAD_OK;
}

int pipad_gated_ff_workspace(const pipad_gated_ff_t *block, int32_t n, int32_t k, int32_t backward, size_t *bytes) {
  const int rc = check_ff_sizes(block, n, k);
  if (rc != PIPAD_OK) return rc;
  if (!bytes || (backward != 0 && backward != 1)) return PIPAD_ERR_INVALID_ARG;
  *bytes = pipad::gated_ff_workspace(*block, n, k, backward != 0);
  return PIPAD_OK;
}

int pipad_gated_ff(const pipad_gated_ff_t *block, int32_t n, int32_t k, const float *const *X, int64_t ldx, float *const *Y,
                   int64_t ldy, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = check_ff(block, n, k);
  if (rc != PIPAD_OK) return rc;
  PIPAD_ROWS(block->F, X, ldx);
  PIPAD_ROWS(block->Fo, Y, ldy);
  if (n == 0) return PIPAD_OK;
  if ((rc = check_workspace(workspace, workspace_bytes, pipad::gated_ff_workspace(*block, n, k, false))) != PIPAD_OK) return rc;
  return pipad::gated_ff_launch(*block, n, k, X, ldx, Y, ldy, workspace, static_cast<hipStream_t>(stream));
}

int pipad_gated_ff_backward(const pipad_gated_ff_t *block, int32_t n, int32_t k, const float *const *X, int64_t ldx,
                            const float *const *dY, int64_t lddy, float *const *dX, int64_t lddx,
                            const pipad_gated_ff_grads_t *grads, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = check_ff(block, n, k);
  if (rc != PIPAD_OK) return rc;
  PIPAD_ROWS(block->F, X, ldx);
  PIPAD_ROWS(block->Fo, dY, lddy);
  if (dX) PIPAD_ROWS(block->F, dX, lddx);
  if (!dX && !grads) return PIPAD_ERR_INVALID_ARG;
  if (grads) {
    const int64_t lim = (int64_t)1 << 40;
    if ((grads->dWg && grads->lddwg < block->hidden) || (grads->dWu && grads->lddwu < block->hidden) || (grads->dWd && grads->lddwd < block->Fo))
      return PIPAD_ERR_INVALID_ARG;
    if ((grads->dWg && grads->lddwg >= lim) || (grads->dWu && grads->lddwu >= lim) || (grads->dWd && grads->lddwd >= lim)) return PIPAD_ERR_TOO_LARGE;
  }
  if (n > 0 && (rc = check_workspace(workspace, workspace_bytes, pipad::gated_ff_workspace(*block, n, k, true))) != PIPAD_OK) return rc;
  return pipad::gated_ff_backward_launch(*block, n, k, X, ldx, dY, lddy, dX, lddx, grads, workspace, static_cast<hipStream_t>(stream));
}
#undef PIPAD_ROWS

int64_t pipad_recommended_row_stride(int32_t F) {
  if (F < 1) return PIPAD_ERR_INVALID_ARG;
  if (F <= 32) {  // within one line: the next power of two, so that no row straddles two lines
    int64_t p = 1;
    while (p < F) p <<= 1;
    return p;
  }
  int64_t lines = ((int64_t)F * 4 + 127) / 128;  // 128-byte lines that hold a row
  if (lines % 2 == 0) ++lines;                    // ... made odd
  return lines * 32;
}

int pipad_frame_temporaries(pipad_frame_t *frame, void **ptr, size_t *bytes) {
  if (!frame || !ptr || !bytes) return PIPAD_ERR_INVALID_ARG;
  *ptr = frame->temp_ptr;
  *bytes = frame->temp_bytes;
  frame->temp_ptr = nullptr;
  frame->temp_bytes = 0;
  return PIPAD_OK;
}

void pipad_frame_destroy(pipad_frame_t *frame) { pipad::destroy_frame(frame); }

const char *pipad_strerror(int status) {
  switch (status) {
    case PIPAD_OK: return "ok";
    case PIPAD_ERR_INVALID_ARG: return "invalid argument";
    case PIPAD_ERR_BAD_CSR: return "snapshot is not a canonical CSR pattern";
    case PIPAD_ERR_ALLOC: return "device allocation failed";
    case PIPAD_ERR_TOO_LARGE: return "size exceeds the int32 index space";
    case PIPAD_ERR_HIP: return "HIP runtime error";
    case PIPAD_ERR_SCRATCH: return "the fixed scratch array is too small for this frame and F, or a workspace for its call";
    default: return "unknown status";
  }
}

const char *pipad_last_hip_error(void) { return pipad::g_hip_error.c_str(); }

static int64_t *option_slot(const char *key, int64_t *max_value) {
  pipad::Options &o = pipad::options();
  if (!key) return nullptr;
  const int64_t len_max = (int64_t)1 << 30;  // thresholds on row lengths
  struct Slot { const char *name; int64_t *value; int64_t max; };
  const Slot slots[] = {
      {"short_max", &o.short_max, len_max},     {"mid_max", &o.mid_max, len_max},
      {"hub_threshold", &o.hub_threshold, len_max}, {"hub_segment", &o.hub_segment, len_max},
      {"sub_classes", &o.sub_classes, 4},       {"agg_order", &o.agg_order, 2},
      {"agg_nt", &o.agg_nt, 3},                 {"agg_generic", &o.agg_generic, 1},
      {"slice_cols", &o.slice_cols, 64},        {"agg_coalescent", &o.agg_coalescent, 2},
      {"scale_codes", &o.scale_codes, 2},
  };
  for (const Slot &sl : slots)
    if (!std::strcmp(key, sl.name)) {
      *max_value = sl.max;
      return sl.value;
    }
  return nullptr;
}

int pipad_set_option(const char *key, int64_t value) {
  int64_t max_value = 0;
  int64_t *slot = option_slot(key, &max_value);
  if (!slot || value < 0 || value > max_value) return PIPAD_ERR_INVALID_ARG;
  *slot = value;
  return PIPAD_OK;
}

int pipad_get_option(const char *key, int64_t *value) {
  int64_t max_value = 0;
  int64_t *slot = option_slot(key, &max_value);
  if (!slot || !value) return PIPAD_ERR_INVALID_ARG;
  *value = *slot;
  return PIPAD_OK;
}

}  // extern "C"
