// The residual connection, forward: what a block has computed goes through a norm and a gate, is added to the scaled stream,
// and the norm before the next block is taken of the sum, in one pass.
#include "moc_residual.h"

namespace {

// ---- forward ------------------------------------------------------------------------------------

// Mean (0 of a norm by the root of the squares alone) and 1 / deviation of a row of values that are 0 beyond it.
template <int T, int CH, class Sums>
__device__ __forceinline__ void statistics(const RowNorm& norm, Sums& sums, int cols, int lane, const Runs<CH>& v, float& mean, float& rstd) {
  float s[1] = {0.0f};
  mean = 0.0f;
  if (norm.layer) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < kRun; ++i) s[0] += v[c][i];
    sums(s);
    mean = s[0] / (float)cols;   // a division, so that equal values leave no difference
  }
  s[0] = 0.0f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int n = asked_again(cols - (c * T + lane) * kRun);
    s[0] = n >= kRun ? squares(v[c], mean, kRun, s[0]) : squares(v[c], mean, n, s[0]);
  }
  sums(s);
  rstd = inverse_root(s[0] / (float)cols + norm.eps);
}

// S, B, D: what x and r, the block's output and n hold.  A workgroup goes over rows with the parameters in registers
// and the next row on its way.
template <int S, int B, int D, int T, int CH, bool AFTER>
__global__ __launch_bounds__(T < 256 ? 256 : T) void residual_forward_kernel(ResidualArgs g) {
  constexpr int kRows = T < 256 ? 256 / T : 1;
  using Sums = RowSums<T, 1>;
  __shared__ float room[Sums::kRoom];
  Sums sums{room};
  const int lane = threadIdx.x % T, mine = kRows > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / T) : 0;
  const bool whole = S != kAny || (g.cols >= kRun && !g.parts);   // which S says: see forward_shape
  const uint32_t step = gridDim.x * kRows;
  uint32_t row = blockIdx.x * kRows + mine;
  Raw wb[CH], wx[CH], wg[CH];
  const auto load = [&](uint32_t at) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * T + lane) * kRun;
      wb[c] = load_run_of<B>(g.block, at, col, g.cols, whole);
      if (g.x.data) wx[c] = load_run_of<S>(g.x, at, col, g.cols, whole);
      if (g.gates > 1) wg[c] = load_run_of<kTensor>(g.gate, at / g.rows_per_gate, col, g.cols, whole);
    }
  };
  if (row < g.rows) load(row);
  constexpr bool kHold = CH == 1 || T < kMaxThreads;
  Runs<CH> gamma1, beta1, gate, gamma2, beta2;
  if constexpr (AFTER && kHold) {
    hold_param<T, CH>(g.after.gamma, g.after.param_type, lane, g.cols, 1.0f, gamma1);
    hold_param<T, CH>(g.after.beta, g.after.param_type, lane, g.cols, 0.0f, beta1);
  }
  if (g.gates <= 1) hold_gate<T, CH>(g, 0, lane, gate);
  if constexpr (kHold) {
    hold_param<T, CH>(g.before.gamma, g.before.param_type, lane, g.cols, 1.0f, gamma2);
    hold_param<T, CH>(g.before.beta, g.before.param_type, lane, g.cols, 0.0f, beta2);
  }
  for (; row < g.rows; row += step) {
    Runs<CH> v;
    Raw x[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = asked_again((c * T + lane) * kRun);
      values_of_run<B>(g.block, wb[c], col, g.cols, whole, v[c]);
      if (g.gates > 1) values_of_run<kTensor>(g.gate, wg[c], col, g.cols, whole, gate[c]);
      x[c] = wx[c];
    }
    if (row + step < g.rows) load(row + step);
    if constexpr (AFTER) {
      float mean, rstd;
      statistics<T, CH>(g.after, sums, g.cols, lane, v, mean, rstd);
      if (lane == 0) {
        if (g.after.layer) g.after.mean[row] = mean;
        g.after.rstd[row] = rstd;
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = asked_again((c * T + lane) * kRun);
        float ga[kRun], be[kRun];
        normalise(v[c], mean, rstd, param_of<kHold>(gamma1[c], g.after.gamma, g.after.param_type, col, g.cols, 1.0f, ga),
                  param_of<kHold>(beta1[c], g.after.beta, g.after.param_type, col, g.cols, 0.0f, be));
      }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = asked_again((c * T + lane) * kRun), n = g.cols - col;
#pragma unroll
      for (int i = 0; i < kRun; ++i) v[c][i] *= gate[c][i];
      if (g.x.data) {
        float more[kRun];
        values_of_run<S>(g.x, x[c], col, g.cols, whole, more);
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[c][i] = __builtin_fmaf(g.scale, more[i], v[c][i]);
      }
      if (n < kRun) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[c][i] = i < n ? v[c][i] : 0.0f;   // a norm has made something of them
      }
      if (g.r.data) store_run_of<S>(g.r, row, col, n, v[c]);
    }
    if (!g.before.on) continue;
    float mean, rstd;
    statistics<T, CH>(g.before, sums, g.cols, lane, v, mean, rstd);
    if (lane == 0) {
      if (g.before.layer) g.before.mean[row] = mean;
      g.before.rstd[row] = rstd;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = asked_again((c * T + lane) * kRun), n = g.cols - col;
      float ga[kRun], be[kRun];
      normalise(v[c], mean, rstd, param_of<kHold>(gamma2[c], g.before.gamma, g.before.param_type, col, g.cols, 1.0f, ga),
                param_of<kHold>(beta2[c], g.before.beta, g.before.param_type, col, g.cols, 0.0f, be));
      store_run_of<D>(g.n, row, col, n, v[c]);
      if (!g.kept.data) continue;
      if (n < kRun) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[c][i] = i < n ? v[c][i] : 0.0f;
      }
      keep_any(g.kept.type, v[c], col, n, g.most, reinterpret_cast<uint8_t*>(row_at(g.kept, row)), g.kept.scales + (uint64_t)row * g.kept.scale_step);
    }
  }
}

// ---- dispatch -----------------------------------------------------------------------------------

using Kernel = void (*)(ResidualArgs);
struct Shape {
  Kernel kern;
  int threads, rows;   // of a workgroup
};
template <int S, int B, int D, bool AFTER>
Shape forward_shape(int64_t cols) {
  if (cols <= 512) return {residual_forward_kernel<S, B, D, 64, 1, AFTER>, 256, 4};
  if (cols <= 1024) return {residual_forward_kernel<S, B, D, 64, 2, AFTER>, 256, 4};
  if (cols <= 2048) return {residual_forward_kernel<S, B, D, 256, 1, AFTER>, 256, 1};
  if (cols <= 4096) return {residual_forward_kernel<S, B, D, 512, 1, AFTER>, 512, 1};
  if (cols <= 8192) return {residual_forward_kernel<S, B, D, 1024, 1, AFTER>, 1024, 1};
  return {residual_forward_kernel<S, B, D, 1024, 2, AFTER>, 1024, 1};
}
template <bool AFTER>
Shape forward_shape(int s, int b, int d, int64_t cols) {
  if (s == MOC_BF16 && b == MOC_BF16 && d == MOC_BF16) return forward_shape<MOC_BF16, MOC_BF16, MOC_BF16, AFTER>(cols);
  if (s == MOC_F32 && b == MOC_BF16 && d == MOC_BF16) return forward_shape<MOC_F32, MOC_BF16, MOC_BF16, AFTER>(cols);
  if (s == MOC_F16 && b == MOC_F16 && d == MOC_F16) return forward_shape<MOC_F16, MOC_F16, MOC_F16, AFTER>(cols);
  if (s == MOC_F32 && b == MOC_F16 && d == MOC_F16) return forward_shape<MOC_F32, MOC_F16, MOC_F16, AFTER>(cols);
  return forward_shape<kAny, kAny, kAny, AFTER>(cols);
}

}  // namespace

extern "C" {

int moc_residual_forward(int64_t rows, int64_t cols, const moc_matrix* x, const moc_matrix* block, const moc_matrix* gate, int64_t gates, float scale, const moc_row_norm* after,
                         const moc_row_norm* before, const moc_matrix* r, const moc_matrix* n, const moc_matrix* kept, void* hip_stream) {
  if (!residual_sizes_ok(rows, cols, gates) || !(scale - scale == 0.0f)) return MOC_EINVAL;
  if ((x && !matrix_ok(x, rows, cols, true, false)) || !matrix_ok(block, rows, cols, true, true) || (gates > 0) != (gate != nullptr) || (gate && !matrix_ok(gate, gates, cols, true, false))) return MOC_EINVAL;
  if (!norm_ok(after, rows) || !norm_ok(before, rows)) return MOC_EINVAL;
  const bool last = before && before->kind != MOC_NORM_NONE;
  if ((r && !matrix_ok(r, rows, cols, true, false)) || last != (n != nullptr) || (n && !matrix_ok(n, rows, cols, true, false)) || (kept && (!n || !matrix_ok(kept, rows, cols, false, true))))
    return MOC_EINVAL;
  if (!r && !n) return MOC_EINVAL;
  if (rows == 0) return MOC_OK;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  ResidualArgs g = {};
  g.x = mat_of(x); g.block = mat_of(block); g.gate = mat_of(gate); g.r = mat_of(r); g.n = mat_of(n); g.kept = mat_of(kept);
  g.after = row_norm_of(after); g.before = row_norm_of(before);
  g.rows = (uint32_t)rows; g.cols = (int)cols; g.gates = (uint32_t)gates; g.rows_per_gate = (uint32_t)(gates > 0 ? rows / gates : rows);
  g.scale = scale;
  if (kept) g.most = most_kept(kept->type, n->type);
  g.parts = lies_over(r, {x, block, gate}) || lies_over(n, {x, block, gate});
  // kernels made for some types, where all matrices are of them and a row's last run may be loaded whole
  const bool ragged = cols < kRun || (g.parts && cols % kRun != 0);
  const int ks = ragged ? kAny : agreed({x, r}, kind_of(block->type)), kb = kind_of(block->type), kd = agreed({n}, kb);
  const Shape s = g.after.on ? forward_shape<true>(ks, kb, kd, cols) : forward_shape<false>(ks, kb, kd, cols);
  const int64_t there = (rows + s.rows - 1) / s.rows, wanted = (int64_t)units * (2 * kMaxThreads / s.threads);
  hipLaunchKernelGGL(s.kern, dim3((unsigned)std::min(there, wanted)), dim3(s.threads), 0, static_cast<hipStream_t>(hip_stream), g);
  MOC_HIP(hipGetLastError());
  return MOC_OK;
}

}  // extern "C"
