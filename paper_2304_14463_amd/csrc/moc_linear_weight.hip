// The linear layer's gradients with regard to its weight, from a tensor or a checkpoint, and its bias.
#include "moc_linear.h"

namespace {

// db where the product does not take it along: a column sum of dy, bound by memory.  A workgroup has 512 columns, eight a lane, and a stretch of
// rows, which its four waves take in turn, four at a time; where the rows are cut into several
// stretches their sums meet in the workspace and are added in order.
constexpr int kBiasCols = kWave * kRun, kBiasWaves = 4;

struct BiasArgs {
  const void* dy;
  int type;
  int64_t stride, rows, each;   // rows of a stretch
  int cols;
  float* out;                   // [stretches][cols]
};

template <int TYPE>
__global__ __launch_bounds__(kBiasWaves * kWave) void bias_grad_kernel(BiasArgs g) {
  __shared__ float stage[kBiasWaves][kRun][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int col = blockIdx.x * kBiasCols + lane * kRun, n = g.cols - col;
  const int64_t begin = blockIdx.y * g.each, end = begin + g.each < g.rows ? begin + g.each : g.rows;
  float s[kRun] = {};
  constexpr int kAt = 4;
  for (int64_t row = begin + wave; row < end; row += kAt * kBiasWaves) {
    float v[kAt][kRun];
#pragma unroll
    for (int i = 0; i < kAt; ++i) {
      const int64_t r = row + i * kBiasWaves;
      load_run<TYPE>(static_cast<const uint16_t*>(g.dy) + (r < end ? r : row) * g.stride, n > 0 ? col : 0, r < end ? n : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kAt; ++i)
#pragma unroll
      for (int j = 0; j < kRun; ++j) s[j] += v[i][j];
  }
#pragma unroll
  for (int j = 0; j < kRun; ++j) stage[wave][j][lane] = s[j];
  __syncthreads();
  if (wave != 0 || n <= 0) return;
#pragma unroll
  for (int j = 0; j < kRun; ++j) s[j] = stage[0][j][lane] + stage[1][j][lane] + stage[2][j][lane] + stage[3][j][lane];
  store_run<MOC_F32>(g.out + (int64_t)blockIdx.y * g.cols, col, n, s);
}

}  // namespace

extern "C" int moc_linear_backward_weight(int64_t rows, int64_t cin, int64_t cout, const moc_matrix* dy, const moc_matrix* x, const moc_matrix* dw,
                                          float* db, void* work, int64_t work_bytes, void* hip_stream) {
  if (!sizes_ok(rows, cin) || !sizes_ok(rows, cout)) return MOC_EINVAL;
  if (!matrix_ok(dy, rows, cout, true, false) || dy->type == MOC_F32) return MOC_EINVAL;
  if (!matrix_ok(x, rows, cin, true, true) || (is_value(x->type) && x->type != dy->type)) return MOC_EINVAL;
  if (!matrix_ok(dw, cout, cin, true, false) || (dw->type != dy->type && dw->type != MOC_F32) || !aligned_to(db, 4)) return MOC_EINVAL;
  if (cout == 0) return MOC_OK;
  int units = 0;
  const int asked = moc_compute_units(&units);
  if (asked != MOC_OK) return asked;
  // Everything is checked before the product is queued: the bias's gradient has a need of its own where the product does not
  // take it along.
  LinearArgs product = {};
  LinearPlan plan;
  if (cin > 0) {
    LinearArgs& g = product;
    g.sums = db;
    g.a = operand_of(dy);
    g.b = operand_of(x);
    g.m = (int)cout;
    g.n = (int)cin;
    g.k = (int)rows;
    set_out(g.e, dw);
    const bool direct = direct_ok(dy, cout) && (is_kept(x->type) ? kept_direct_ok(x, cin) : direct_ok(x, cin));
    const int rc = cut_linear<kCol, kCol>(g, loading_of(direct, cout, cin), units, work, work_bytes, plan);
    if (rc != MOC_OK) return rc;
  }
  const bool apart = db && !product.sums;
  const int64_t stretches = apart ? moc_bias_stretches(rows, cout, units) : 1;
  if (stretches > 1 && (!work || !aligned_to(work, 16) || work_bytes < stretches * cout * (int64_t)sizeof(float))) return MOC_EINVAL;
  if (cin > 0) {
    const int rc = queue_linear<kCol, kCol, true>(product, plan, dy->type, x->type, hip_stream);
    if (rc != MOC_OK) return rc;
  }
  if (apart) {
    BiasArgs g = {};
    g.dy = dy->data;
    g.type = dy->type;
    g.stride = dy->stride;
    g.rows = rows;
    g.each = (rows + stretches - 1) / stretches;
    g.cols = (int)cout;
    g.out = stretches > 1 ? static_cast<float*>(work) : db;   // the product is done with the workspace: one stream
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const dim3 grid((unsigned)((cout + kBiasCols - 1) / kBiasCols), (unsigned)stretches);
    hipLaunchKernelGGL(dy->type == MOC_BF16 ? bias_grad_kernel<MOC_BF16> : bias_grad_kernel<MOC_F16>, grid, dim3(kBiasWaves * kWave), 0, stream, g);
    MOC_HIP(hipGetLastError());
    if (stretches > 1) {
      hipLaunchKernelGGL(join_sums_kernel, dim3((unsigned)((cout + 63) / 64)), dim3(1024), 0, stream, g.out, (int)stretches, cout, cout, db);
      MOC_HIP(hipGetLastError());
    }
  }
  return MOC_OK;
}
