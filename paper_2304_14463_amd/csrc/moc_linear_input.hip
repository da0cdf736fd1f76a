// The linear layer's gradient with regard to its input, and through the activation before it.
#include "moc_linear.h"

extern "C" int moc_linear_backward_input(int64_t rows, int64_t cin, int64_t cout, const moc_matrix* dy, const moc_matrix* w, int32_t act,
                                         const moc_matrix* pre, const moc_matrix* dx, void* work, int64_t work_bytes, void* hip_stream) {
  if (!sizes_ok(rows, cin) || !sizes_ok(rows, cout) || act < MOC_ACT_NONE || act > MOC_ACT_SILU || (!pre && act != MOC_ACT_NONE)) return MOC_EINVAL;
  if (!matrix_ok(dy, rows, cout, true, false) || dy->type == MOC_F32 || !matrix_ok(w, cout, cin, true, false) || w->type != dy->type) return MOC_EINVAL;
  if (!matrix_ok(dx, rows, cin, true, false) || (dx->type != dy->type && dx->type != MOC_F32)) return MOC_EINVAL;
  if (pre && (!matrix_ok(pre, rows, cin, true, true) || (is_value(pre->type) && pre->type != dy->type && pre->type != MOC_F32))) return MOC_EINVAL;
  if (rows == 0 || cin == 0) return MOC_OK;
  LinearArgs g = {};
  g.a = operand_of(dy);
  g.b = operand_of(w);
  g.m = (int)rows;
  g.n = (int)cin;
  g.k = (int)cout;
  Epilogue& e = g.e;
  e.act = act;
  if (pre && act != MOC_ACT_NONE) {
    e.extra = pre->data;
    e.extra_scales = pre->scales;
    e.extra_type = pre->type;
    e.extra_stride = pre->stride;
    e.extra_scale_stride = pre->scale_stride;
    e.slope = 1;
  }
  set_out(e, dx);
  int units = 0;
  LinearPlan p;
  int rc = moc_compute_units(&units);
  if (rc == MOC_OK) rc = cut_linear<kRow, kCol>(g, loading_of(direct_ok(dy, cout) && direct_ok(w, cin), cout, cin), units, work, work_bytes, p);
  return rc == MOC_OK ? queue_linear<kRow, kCol, false>(g, p, dy->type, dy->type, hip_stream) : rc;
}
