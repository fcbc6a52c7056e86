// C ABI of the layer norm (optorch_matrix.h): argument checks, then the kernels of k_norm.hip on the caller's stream.
#include "args.h"

using namespace oseq;

static int norm_check(const optorch_layer_norm_t* a, bool backward) {
  if (!a) return oseq_mat_err(OPTORCH_E_INVALID, "null arguments");
  if (!precision_ok(a->precision)) return oseq_mat_err(OPTORCH_E_INVALID, "unknown precision");
  if (a->rows < 0 || a->rows > 0x7fffff00) return oseq_mat_err(OPTORCH_E_INVALID, "rows must be 0 .. 2^31 - 256");
  if (a->cols < 1 || a->cols > kMaxFeatures) return oseq_mat_err(OPTORCH_E_INVALID, "cols must be 1 .. 2^22 - 8");
  const int esize = bytes_of(a->precision);
  const bool some = a->rows > 0;  // (an empty batch has no matrices of its own)
  int rc = OPTORCH_OK;
  auto matrix = [&](const void* p, int64_t ld, const char* name) {
    if (some && rc == OPTORCH_OK) rc = check_matrix(p, ld, a->cols, esize, name);
  };
  auto vector = [&](const float* p, const char* name) {
    if (rc == OPTORCH_OK) rc = check_vector(p, name);
  };
  if (!backward) {
    if (!(a->eps >= 0.f) || !std::isfinite(a->eps)) return oseq_mat_err(OPTORCH_E_INVALID, "eps must be finite and not negative");
    matrix(a->x, a->ldx, "x");
    matrix(a->y, a->ldy, "y");
    vector(a->bias, "bias");
    if (rc == OPTORCH_OK && some && !a->mean != !a->rstd) rc = oseq_mat_err(OPTORCH_E_INVALID, "mean and rstd are kept together or not at all");
  } else {
    if (!a->dx && !a->dweight && !a->dbias) return oseq_mat_err(OPTORCH_E_INVALID, "no gradient asked for");
    matrix(a->dy, a->lddy, "dy");
    if (a->dx || a->dweight) {
      matrix(a->x, a->ldx, "x");
      if (rc == OPTORCH_OK && some && (!a->mean || !a->rstd)) rc = oseq_mat_err(OPTORCH_E_INVALID, "null mean or rstd");
    }
    if (a->dx) {
      matrix(a->dx, a->lddx, "dx");
      if (a->residual) matrix(a->residual, a->ldr, "residual");
    }
    vector(a->dweight, "dweight");
    vector(a->dbias, "dbias");
  }
  vector(a->weight, "weight");
  vector(a->mean, "mean");
  vector(a->rstd, "rstd");
  return rc;
}

static int norm_overlaps(const optorch_layer_norm_t* a, bool backward, uint64_t workspace_bytes) {
  Operands o;
  const int e = bytes_of(a->precision);
  const int64_t rows = a->rows, cols = a->cols;
  if (!backward || a->dx || a->dweight) {
    o.add("x", a->x, rows, cols, a->ldx, e, false);
    o.vector("weight", a->weight, cols, 4, false);
    o.vector("mean", a->mean, rows, 4, !backward);
    o.vector("rstd", a->rstd, rows, 4, !backward);
  }
  if (!backward) {
    o.vector("bias", a->bias, cols, 4, false);
    o.add("y", a->y, rows, cols, a->ldy, e, true);
  } else {
    o.add("dy", a->dy, rows, cols, a->lddy, e, false);
    if (a->dx) o.add("residual", a->residual, rows, cols, a->ldr, e, false);
    o.add("dx", a->dx, rows, cols, a->lddx, e, true);
    o.vector("dweight", a->dweight, cols, 4, true);
    o.vector("dbias", a->dbias, cols, 4, true);
    o.vector("workspace", workspace_bytes ? a->workspace : nullptr, (int64_t)workspace_bytes, 1, true);
  }
  return o.apart([](const Operands::Named& p, const Operands::Named& q) {
    return p.is("residual") && q.is("dx") && same_place(p.p, q.p);
  });
}

extern "C" int64_t optorch_layer_norm_workspace(const optorch_layer_norm_t* a) {
  return guarded([&]() -> int64_t {
    const int rc = norm_check(a, true);
    if (rc != OPTORCH_OK) return rc;
    return a->rows ? (int64_t)plan_norm_backward(*a).bytes : 0;
  });
}

extern "C" int optorch_layer_norm_forward(const optorch_layer_norm_t* a) {
  return guarded([&]() -> int {
    int rc = norm_check(a, false);
    if (rc == OPTORCH_OK) rc = norm_overlaps(a, false, 0);
    if (rc != OPTORCH_OK) return rc;
    if (a->rows) launch_norm_forward(*a);
    return mat_launched("layer_norm_forward");
  });
}

extern "C" int optorch_layer_norm_backward(const optorch_layer_norm_t* a) {
  return guarded([&]() -> int {
    int rc = norm_check(a, true);
    if (rc != OPTORCH_OK) return rc;
    NormPlan p = {};
    if (a->rows) {
      p = plan_norm_backward(*a);
      rc = check_workspace(a->workspace, a->workspace_bytes, p.bytes);
      if (rc != OPTORCH_OK) return rc;
    }
    rc = norm_overlaps(a, true, p.bytes);
    if (rc != OPTORCH_OK) return rc;
    launch_norm_backward(*a, p);
    return mat_launched("layer_norm_backward");
  });
}
