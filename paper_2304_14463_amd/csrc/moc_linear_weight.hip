// The linear layer's gradients with regard to its weight, from a tensor or a checkpoint, and its bias.
#include "moc_linear.h"

namespace {

// db: a column sum of dy.  64 columns a workgroup of 16 x 64 threads, rows in one order.
__global__ __launch_bounds__(1024) void bias_grad_kernel(const void* dy, int type, int64_t stride, int64_t rows, int cols, float* db) {
  __shared__ float stage[16][64];
  const int col = blockIdx.x * 64 + (threadIdx.x & 63), mine = threadIdx.x >> 6;
  float s = 0.0f;
  if (col < cols) {
    for (int64_t row = mine; row < rows; row += 16) {
      const uint16_t* p = static_cast<const uint16_t*>(dy) + row * stride + col;
      s += type == MOC_BF16 ? (float)__builtin_bit_cast(__bf16, *p) : (float)__builtin_bit_cast(_Float16, *p);
    }
  }
  stage[mine][threadIdx.x & 63] = s;
  __syncthreads();
  if (mine == 0 && col < cols) {
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += stage[i][threadIdx.x];
    db[col] = s;
  }
}

}  // namespace

extern "C" int moc_linear_backward_weight(int64_t rows, int64_t cin, int64_t cout, const moc_matrix* dy, const moc_matrix* x, const moc_matrix* dw,
                                          float* db, void* work, int64_t work_bytes, void* hip_stream) {
  if (!sizes_ok(rows, cin) || !sizes_ok(rows, cout)) return MOC_EINVAL;
  if (!matrix_ok(dy, rows, cout, true, false) || dy->type == MOC_F32) return MOC_EINVAL;
  if (!matrix_ok(x, rows, cin, true, true) || (is_value(x->type) && x->type != dy->type)) return MOC_EINVAL;
  if (!matrix_ok(dw, cout, cin, true, false) || (dw->type != dy->type && dw->type != MOC_F32) || !aligned_to(db, 4)) return MOC_EINVAL;
  if (cout == 0) return MOC_OK;
  if (cin > 0) {
    LinearArgs g = {};
    g.a = operand_of(dy);
    g.b = operand_of(x);
    g.m = (int)cout;
    g.n = (int)cin;
    g.k = (int)rows;
    set_out(g.e, dw);
    const bool direct = direct_ok(dy, cout) && (is_kept(x->type) || direct_ok(x, cin));
    const int rc = queue_linear<kCol, kCol, true>(g, dy->type, x->type, direct, work, work_bytes, hip_stream);
    if (rc != MOC_OK) return rc;
  }
  if (db) {
    hipLaunchKernelGGL(bias_grad_kernel, dim3((unsigned)((cout + 63) / 64)), dim3(1024), 0, static_cast<hipStream_t>(hip_stream), dy->data, dy->type,
                       dy->stride, rows, (int)cout, db);
    MOC_HIP(hipGetLastError());
  }
  return MOC_OK;
}
