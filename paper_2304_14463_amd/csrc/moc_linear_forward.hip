// The linear layer: act(x w^T + bias) + residual, with the checkpoint of the activation's argument.
#include "moc_linear.h"

extern "C" {

int moc_linear_forward(int64_t rows, int64_t cin, int64_t cout, const moc_matrix* x, const moc_matrix* w, const void* bias, int32_t bias_type,
                       int32_t act, const moc_matrix* residual, const moc_matrix* y, const moc_matrix* kept, void* work, int64_t work_bytes,
                       void* hip_stream) {
  if (!sizes_ok(rows, cin) || !sizes_ok(rows, cout) || act < MOC_ACT_NONE || act > MOC_ACT_SILU) return MOC_EINVAL;
  if (!matrix_ok(x, rows, cin, true, false) || x->type == MOC_F32 || !matrix_ok(w, cout, cin, true, false) || w->type != x->type) return MOC_EINVAL;
  if (!matrix_ok(y, rows, cout, true, false) || (y->type != x->type && y->type != MOC_F32) || !params_ok(bias, bias_type)) return MOC_EINVAL;
  if (residual && (!matrix_ok(residual, rows, cout, true, false) || (residual->type != x->type && residual->type != MOC_F32))) return MOC_EINVAL;
  if (kept && !matrix_ok(kept, rows, cout, false, true)) return MOC_EINVAL;
  if (rows == 0 || cout == 0) return MOC_OK;
  LinearArgs g = {};
  g.a = operand_of(x);
  g.b = operand_of(w);
  g.m = (int)rows;
  g.n = (int)cout;
  g.k = (int)cin;
  Epilogue& e = g.e;
  e.bias = bias;
  e.bias_type = bias_type;
  e.act = act;
  if (residual) {
    e.extra = residual->data;
    e.extra_type = residual->type;
    e.extra_stride = residual->stride;
  }
  set_out(e, y);
  if (kept) {
    e.codes = static_cast<uint8_t*>(kept->data);
    e.scales = kept->scales;
    e.kept_type = kept->type;
    e.code_stride = kept->stride;
    e.scale_stride = kept->scale_stride;
    e.most = most_kept(kept->type, x->type);
  }
  int units = 0;
  LinearPlan p;
  int rc = moc_compute_units(&units);
  if (rc == MOC_OK) rc = cut_linear<kRow, kRow>(g, loading_of(direct_ok(x, cin) && direct_ok(w, cin), cin, cin), units, work, work_bytes, p);
  return rc == MOC_OK ? queue_linear<kRow, kRow, false>(g, p, x->type, x->type, hip_stream) : rc;
}

int64_t moc_linear_work(int64_t rows, int64_t cin, int64_t cout) {
  if (!sizes_ok(rows, cin) || !sizes_ok(rows, cout)) return MOC_EINVAL;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  int64_t most = cout > 0 ? moc_bias_stretches(rows, cout, units) * cout * (int64_t)sizeof(float) : 0;
  for (const Loading how : {kDirect, kThroughRegisters, kNarrow}) {
    const int64_t sizes[3][3] = {{rows, cout, cin}, {rows, cin, cout}, {cout, cin, rows}};
    for (int cols = 0; cols < 3; ++cols) {
      const int64_t bytes = linear_plan(sizes[cols][0], sizes[cols][1], sizes[cols][2], cols, how, units).work_bytes;
      most = bytes > most ? bytes : most;
    }
  }
  return most;
}

int moc_linear_parts(int32_t product, int64_t rows, int64_t cin, int64_t cout, int32_t aligned, int32_t units, int64_t* out) {
  if (!sizes_ok(rows, cin) || !sizes_ok(rows, cout) || product < MOC_LINEAR_FORWARD || product > MOC_LINEAR_BACKWARD_WEIGHT || units < 0 || !out) return MOC_EINVAL;
  int there = units;
  const int rc = units > 0 ? MOC_OK : moc_compute_units(&there);
  if (rc != MOC_OK) return rc;
  const int64_t sizes[3][3] = {{rows, cout, cin}, {rows, cin, cout}, {cout, cin, rows}}, along = product == MOC_LINEAR_FORWARD ? cin : cout;
  const Loading how = loading_of(aligned && along % 8 == 0 && cin % 8 == 0, along, cin);
  const int64_t* const s = sizes[product];
  const LinearPlan p = linear_plan(s[0], s[1], s[2], product, how, there);   // as many operands lie in columns
  const int last = (p.splits - 1) * p.split_k;
  out[0] = kShapes[p.shape].tile;
  out[1] = p.shape == kDirect128 || p.shape == kDirect256;
  out[2] = p.splits;
  out[3] = p.split_k;
  out[4] = part_end((int)s[2], last, p.split_k) - last;
  return MOC_OK;
}

}  // extern "C"
