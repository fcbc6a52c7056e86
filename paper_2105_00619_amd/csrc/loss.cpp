// C ABI of the losses over many classes (optorch_matrix.h): argument checks, then the kernels of k_loss.hip and k_loss_grad.hip on the
// caller's stream.
#include "args.h"

using namespace oseq;

static int loss_check(const optorch_softmax_loss_t* a, bool backward) {
  if (!a) return oseq_mat_err(OPTORCH_E_INVALID, "null arguments");
  if (!precision_ok(a->precision)) return oseq_mat_err(OPTORCH_E_INVALID, "unknown precision");
  if (a->rows < 0 || a->rows > 0x7fffff00) return oseq_mat_err(OPTORCH_E_INVALID, "rows must be 0 .. 2^31 - 256");
  if (a->in_features < 1 || a->classes < 1 || a->in_features > kMaxFeatures || a->classes > kMaxFeatures)
    return oseq_mat_err(OPTORCH_E_INVALID, "in_features and classes must be 1 .. 2^22 - 8");
  if (a->precision == OPTORCH_FP32 && (a->in_features > kMaxFeatures32 || a->classes > kMaxFeatures32))
    return oseq_mat_err(OPTORCH_E_INVALID, "in fp32 in_features and classes must be 1 .. 2^20 - 16");
  const int esize = bytes_of(a->precision);
  const bool some = a->rows > 0;  // (an empty batch has no matrices of its own)
  int rc = OPTORCH_OK;
  auto matrix = [&](const void* p, int64_t ld, int64_t cols, int size, const char* name) {
    if (rc == OPTORCH_OK) rc = check_matrix(p, ld, cols, size, name);
  };
  auto vector = [&](const void* p, bool wanted, const char* name) {
    if (rc == OPTORCH_OK && wanted && !p) rc = oseq_mat_err(OPTORCH_E_INVALID, std::string("null ") + name);
    if (rc == OPTORCH_OK) rc = check_vector(p, name);
  };
  if (backward && !a->dx && !a->dw && !a->dbias) return oseq_mat_err(OPTORCH_E_INVALID, "no gradient asked for");
  if (a->labels) {
    if (a->indices || a->teacher) return oseq_mat_err(OPTORCH_E_INVALID, "labels and a teacher exclude each other");
    if (!(a->label_smoothing >= 0.f && a->label_smoothing <= 1.f)) return oseq_mat_err(OPTORCH_E_INVALID, "label_smoothing must be 0 .. 1");
    if (!(a->z_loss >= 0.f) || !std::isfinite(a->z_loss)) return oseq_mat_err(OPTORCH_E_INVALID, "z_loss must be finite and not negative");
    vector(a->labels, true, "labels");
  } else if (a->indices || a->teacher || some) {
    if (some && !a->indices && !a->teacher) return oseq_mat_err(OPTORCH_E_INVALID, "neither labels nor a teacher");
    if (!precision_ok(a->teacher_precision)) return oseq_mat_err(OPTORCH_E_INVALID, "unknown teacher_precision");
    if (a->top < 1 || a->top > 1024) return oseq_mat_err(OPTORCH_E_INVALID, "top must be 1 .. 1024");
    if (!(a->temperature > 0.f) || !std::isfinite(a->temperature) || !std::isfinite(1.f / a->temperature))
      return oseq_mat_err(OPTORCH_E_INVALID, "temperature must be finite and above 0");
    if (a->label_smoothing != 0.f || a->z_loss != 0.f) return oseq_mat_err(OPTORCH_E_INVALID, "label_smoothing and z_loss go with labels");
    if (some) matrix(a->indices, a->ldi, a->top, 4, "indices");
    if (some) matrix(a->teacher, a->ldt, a->top, bytes_of(a->teacher_precision), "teacher");
  }
  if (some) matrix(a->x, a->ldx, a->in_features, esize, "x");
  if (some) matrix(a->w, a->ldw, a->in_features, esize, "w");
  vector(a->bias, false, "bias");
  vector(a->lse, some, "lse");
  if (!backward) {
    vector(a->loss, some, "loss");
  } else {
    vector(a->dloss, some, "dloss");
    if (some && a->dx) matrix(a->dx, a->lddx, a->in_features, esize, "dx");
    if (a->dw) matrix(a->dw, a->lddw, a->in_features, esize, "dw");
    vector(a->dbias, false, "dbias");
  }
  return rc;
}

static int loss_overlaps(const optorch_softmax_loss_t* a, bool backward, uint64_t workspace_bytes) {
  Operands o;
  const int e = bytes_of(a->precision);
  const int64_t rows = a->rows, in = a->in_features, classes = a->classes;
  if (rows) {
    o.add("x", a->x, rows, in, a->ldx, e, false);
    o.add("w", a->w, classes, in, a->ldw, e, false);
    o.vector("bias", a->bias, classes, 4, false);
    o.vector("labels", a->labels, rows, 4, false);
    o.add("indices", a->indices, rows, a->top, a->ldi, 4, false);
    o.add("teacher", a->teacher, rows, a->top, a->ldt, bytes_of(a->teacher_precision), false);
    o.vector("lse", a->lse, rows, 4, !backward);
  }
  if (!backward) {
    o.vector("loss", a->loss, rows, 4, true);
  } else {
    o.vector("dloss", a->dloss, rows, 4, false);
    o.add("dx", a->dx, rows, in, a->lddx, e, true);
    o.add("dw", a->dw, classes, in, a->lddw, e, true);
    o.vector("dbias", a->dbias, classes, 4, true);
  }
  o.vector("workspace", workspace_bytes ? a->workspace : nullptr, (int64_t)workspace_bytes, 1, true);
  return o.apart([](const Operands::Named&, const Operands::Named&) { return false; });
}

extern "C" int64_t optorch_softmax_loss_workspace(const optorch_softmax_loss_t* a, int32_t backward) {
  return guarded([&]() -> int64_t {
    const int rc = loss_check(a, backward != 0);
    if (rc != OPTORCH_OK) return rc;
    return a->rows ? (int64_t)plan_loss(*a, backward != 0).bytes : 0;
  });
}

static int loss_run(const optorch_softmax_loss_t* a, bool backward) {
  int rc = loss_check(a, backward);
  if (rc != OPTORCH_OK) return rc;
  LossPlan p = {};
  if (a->rows) {
    p = plan_loss(*a, backward);
    rc = check_workspace(a->workspace, a->workspace_bytes, p.bytes);
    if (rc != OPTORCH_OK) return rc;
  }
  rc = loss_overlaps(a, backward, p.bytes);
  if (rc != OPTORCH_OK) return rc;
  if (!backward && a->rows) launch_loss_forward(*a, p);
  if (backward) launch_loss_backward(*a, p);
  return mat_launched(backward ? "softmax_loss_backward" : "softmax_loss_forward");
}

extern "C" int optorch_softmax_loss_forward(const optorch_softmax_loss_t* a) { return guarded([&] { return loss_run(a, false); }); }
extern "C" int optorch_softmax_loss_backward(const optorch_softmax_loss_t* a) { return guarded([&] { return loss_run(a, true); }); }

// How a call is cut, for the tests that name a kernel by its tile (not part of the API): the values of a logits tile's edge, pieces of the
// classes, then 1000 * values of the edge + parts for dx and dw
namespace oseq {
void loss_shape(const optorch_softmax_loss_t* a, bool backward, int32_t out[4]);
void loss_shape(const optorch_softmax_loss_t* a, bool backward, int32_t out[4]) {
  const LossPlan p = plan_loss(*a, backward);
  out[0] = 2 * p.wave;
  out[1] = (a->classes + p.piece - 1) / p.piece;
  out[2] = 2000 * p.dx.wave + p.dx.parts;
  out[3] = 2000 * p.dw.wave + p.dw.parts;
}
// ... and which kernel makes the forward pass' logits: 0 tiles, 1 weights straight from memory, otherwise the blocks that stream them
int32_t loss_path(const optorch_softmax_loss_t* a);
int32_t loss_path(const optorch_softmax_loss_t* a) {
  const LossPlan p = plan_loss(*a, false);
  return p.few ? 1 : p.stream;
}
}  // namespace oseq
