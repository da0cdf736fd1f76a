// The residual connection: what a block has computed goes through a norm and a gate, is added to the scaled stream, and the
// norm before the next block is taken of the sum, in one pass; and the gradients of all of it.
//
// Bound by memory: every value is read once and written once, 8 bytes of the forward and 12 of the backward pass where all are
// 16 bits wide.  T threads take a row and hold it in registers, CH runs of eight values each, as in moc_norm.hip; the
// parameters' gradients are held in registers over a workgroup's rows and added over workgroups by a second kernel, in their order.
#include <algorithm>

#include "moc_rows.h"

namespace {

constexpr int kMaxThreads = 1024;

struct Mat {
  void* data;
  uint8_t* scales;
  int64_t stride, scale_stride;
  int type;
};
struct RowNorm {
  const void *gamma, *beta;
  int param_type;
  float eps;
  bool on, layer;
  float *mean, *rstd;
};
struct ResidualArgs {
  Mat x, block, gate, r, n, kept;
  Mat dr, dn, dx, dblock;
  RowNorm after, before;
  int64_t rows, gates, rows_per_gate;
  int cols;
  float scale, most;
  bool parts;         // rows are loaded value by value where they end in a run: an output lies over an input
  // backward
  float* sums;        // [workgroups][kinds][cols]
  float* gate_sums;   // [gates][chunks][cols]; with one chunk the result itself
  int kinds;          // of sums: bits of kBeforeGamma ..
  bool want_gate, own_gates;   // own: a gate for every row
  int64_t chunks, chunk_rows, groups;   // workgroups of a gate's rows, and their rows; or gates of a workgroup
};
constexpr int kBeforeGamma = 1, kBeforeBeta = 2, kAfterGamma = 4, kAfterBeta = 8;

__device__ __forceinline__ char* row_at(const Mat& m, int64_t row) {
  const int bytes = m.type == MOC_F32 ? 4 : m.type == MOC_E4M3 || m.type == MOC_I8 ? 1 : 2;
  return static_cast<char*>(m.data) + row * m.stride * bytes;
}

// A run of a row on its way; `whole`: of a row of eight columns at least (see load_raw_whole).
__device__ __forceinline__ Raw load_run_of(const Mat& m, int64_t row, int col, int cols, bool whole) {
  const void* const at = row_at(m, row);
  const uint8_t* const scales = m.scales + row * m.scale_stride;
  if (whole) {
    if (m.type == MOC_BF16 || m.type == MOC_F16) return load_raw_whole<MOC_BF16>(at, nullptr, col, cols);
    if (m.type == MOC_F32) return load_raw_whole<MOC_F32>(at, nullptr, col, cols);
    return load_raw_whole<MOC_E4M3>(at, scales, col, cols);
  }
  return load_raw_any(m.type, at, scales, col, cols - col);
}
// Its values, 0 beyond the row.
__device__ __forceinline__ void values_of_run(const Mat& m, Raw w, int col, int cols, bool whole, float (&v)[kRun]) {
  const int n = cols - col;
  if (whole && cols % kRun != 0) {
    if (m.type == MOC_BF16 || m.type == MOC_F16) settle<MOC_BF16>(w, col, cols);
    else if (m.type == MOC_F32) settle<MOC_F32>(w, col, cols);
    else settle<MOC_E4M3>(w, col, cols);
  }
  values_of_any(m.type, w, v);
  if (n < kRun) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = i < n ? v[i] : 0.0f;
  }
}

__device__ __forceinline__ void store_run_of(const Mat& m, int64_t row, int col, int n, const float (&v)[kRun]) {
  if (n > 0) store_any(m.type, row_at(m, row), col, n, v);
}

template <int CH>
using Runs = float[CH][kRun];

template <int T, int CH>
__device__ __forceinline__ void hold_param(const void* p, int type, int lane, int cols, float other, Runs<CH>& v) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = (c * T + lane) * kRun;
    load_param(p, type, min(col, cols - 1), cols - col, other, v[c]);
  }
}
// 1 where there is no gate.
template <int T, int CH>
__device__ __forceinline__ void hold_gate(const ResidualArgs& g, int64_t gate, int lane, Runs<CH>& v) {
  hold_param<T, CH>(g.gates ? row_at(g.gate, gate) : nullptr, g.gate.type, lane, g.cols, 1.0f, v);
}

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
    const int n = cols - (c * T + lane) * kRun;
#pragma unroll
    for (int i = 0; i < kRun; ++i) s[0] += i < n ? (v[c][i] - mean) * (v[c][i] - mean) : 0.0f;
  }
  sums(s);
  rstd = inverse_root(s[0] / (float)cols + norm.eps);
}

template <int T, int CH, bool AFTER>
__global__ __launch_bounds__(T < 256 ? 256 : T) void residual_forward_kernel(ResidualArgs g) {
  constexpr int kRows = T < 256 ? 256 / T : 1;
  using Sums = RowSums<T, 1>;
  __shared__ float room[Sums::kRoom];
  Sums sums{room};
  const int lane = threadIdx.x % T, mine = kRows > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / T) : 0;
  const bool whole = g.cols >= kRun && !g.parts;
  Runs<CH> gamma1, beta1, gate, gamma2, beta2;
  if constexpr (AFTER) {
    hold_param<T, CH>(g.after.gamma, g.after.param_type, lane, g.cols, 1.0f, gamma1);
    hold_param<T, CH>(g.after.beta, g.after.param_type, lane, g.cols, 0.0f, beta1);
  }
  if (g.gates <= 1) hold_gate<T, CH>(g, 0, lane, gate);
  hold_param<T, CH>(g.before.gamma, g.before.param_type, lane, g.cols, 1.0f, gamma2);
  hold_param<T, CH>(g.before.beta, g.before.param_type, lane, g.cols, 0.0f, beta2);
  for (int64_t row = (int64_t)blockIdx.x * kRows + mine; row < g.rows; row += (int64_t)gridDim.x * kRows) {
    Runs<CH> v;
    Raw wx[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * T + lane) * kRun;
      const Raw w = load_run_of(g.block, row, col, g.cols, whole);
      if (g.x.data) wx[c] = load_run_of(g.x, row, col, g.cols, whole);
      values_of_run(g.block, w, col, g.cols, whole, v[c]);
    }
    if (g.gates > 1) hold_gate<T, CH>(g, row / g.rows_per_gate, lane, gate);
    if constexpr (AFTER) {
      float mean, rstd;
      statistics<T, CH>(g.after, sums, g.cols, lane, v, mean, rstd);
      if (lane == 0) {
        if (g.after.layer) g.after.mean[row] = mean;
        g.after.rstd[row] = rstd;
      }
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[c][i] = (v[c][i] - mean) * rstd * gamma1[c][i] + beta1[c][i];
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * T + lane) * kRun, n = g.cols - col;
#pragma unroll
      for (int i = 0; i < kRun; ++i) v[c][i] *= gate[c][i];
      if (g.x.data) {
        float x[kRun];
        values_of_run(g.x, wx[c], col, g.cols, whole, x);
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[c][i] = __builtin_fmaf(g.scale, x[i], v[c][i]);
      }
#pragma unroll
      for (int i = 0; i < kRun; ++i) v[c][i] = i < n ? v[c][i] : 0.0f;   // a norm's beta is not
      if (g.r.data) store_run_of(g.r, row, col, n, v[c]);
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
      const int col = (c * T + lane) * kRun, n = g.cols - col;
#pragma unroll
      for (int i = 0; i < kRun; ++i) v[c][i] = (v[c][i] - mean) * rstd * gamma2[c][i] + beta2[c][i];
      store_run_of(g.n, row, col, n, v[c]);
      if (!g.kept.data) continue;
      if (n < kRun) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[c][i] = i < n ? v[c][i] : 0.0f;
      }
      keep_any(g.kept.type, v[c], col, n, g.most, static_cast<uint8_t*>(g.kept.data) + row * g.kept.stride, g.kept.scales + row * g.kept.scale_stride);
    }
  }
}

// ---- backward -----------------------------------------------------------------------------------

// The sums of a workgroup's kRows groups of T lanes, added in their order, to a row of floats.  By all threads.
template <int T, int kRows, int CH>
__device__ __forceinline__ void put_sums(const Runs<CH>& s, float* out, int cols, float* stage) {
  const int lane = threadIdx.x % T, mine = threadIdx.x / T;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = (c * T + lane) * kRun;
    float a[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) a[i] = s[c][i];
    if constexpr (kRows > 1) {   // stage: [kRows][8][T]
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRun; ++i) stage[(mine * kRun + i) * T + lane] = a[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        a[i] = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) a[i] += stage[(r * kRun + i) * T + lane];
      }
    }
    if (mine == 0 && cols > col) store_run<MOC_F32>(out, col, cols - col, a);
  }
}

template <int T, int CH, bool AFTER>
__global__ __launch_bounds__(T < 256 ? 256 : T) void residual_backward_kernel(ResidualArgs g) {
  constexpr int kRows = T < 256 ? 256 / T : 1;
  using Sums = RowSums<T, 2>;
  __shared__ float room[Sums::kRoom];
  __shared__ float stage[kRows > 1 ? kRows * kRun * T : 1];
  Sums sums{room};
  const int lane = threadIdx.x % T, mine = kRows > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / T) : 0;
  const bool whole = g.cols >= kRun && !g.parts;
  const float part = 1.0f / (float)g.cols;
  Runs<CH> gamma1, beta1, gate, gamma2;
  Runs<CH> sg1, sb1, sgate, sg2, sb2;
  if constexpr (AFTER) {
    hold_param<T, CH>(g.after.gamma, g.after.param_type, lane, g.cols, 1.0f, gamma1);
    hold_param<T, CH>(g.after.beta, g.after.param_type, lane, g.cols, 0.0f, beta1);
  }
  hold_param<T, CH>(g.before.gamma, g.before.param_type, lane, g.cols, 1.0f, gamma2);
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < kRun; ++i) sg1[c][i] = sb1[c][i] = sgate[c][i] = sg2[c][i] = sb2[c][i] = 0.0f;
  // the gates of this workgroup, and its rows of them
  const int64_t from = g.chunks > 1 ? blockIdx.x / g.chunks : blockIdx.x * g.groups, last = min(g.chunks > 1 ? from + 1 : from + g.groups, g.own_gates ? (int64_t)1 : max(g.gates, (int64_t)1));
  const int64_t chunk = g.chunks > 1 ? blockIdx.x - from * g.chunks : 0;
  for (int64_t which = from; which < last; ++which) {
    const int64_t first = which * g.rows_per_gate + chunk * g.chunk_rows, end = min(first + g.chunk_rows, (which + 1) * g.rows_per_gate);
    if (!g.own_gates) hold_gate<T, CH>(g, which, lane, gate);
    for (int64_t at = first; at < end; at += kRows) {
      const int64_t row = at + mine;
      if (row >= end) break;   // of groups of lanes that share no barrier
      Raw wr[CH], wn[CH], wd[CH], wb[CH];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = (c * T + lane) * kRun;
        if (g.before.on) {
          wr[c] = load_run_of(g.r, row, col, g.cols, whole);
          wn[c] = load_run_of(g.dn, row, col, g.cols, whole);
        }
        if (g.dr.data) wd[c] = load_run_of(g.dr, row, col, g.cols, whole);
        if (g.block.data) wb[c] = load_run_of(g.block, row, col, g.cols, whole);
      }
      if (g.own_gates) hold_gate<T, CH>(g, row, lane, gate);
      Runs<CH> d;
      if (g.before.on) {
        const float mean = g.before.layer ? g.before.mean[row] : 0.0f, rstd = g.before.rstd[row];
        Runs<CH> h;
        float m[2] = {0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int col = (c * T + lane) * kRun, n = g.cols - col;
          values_of_run(g.r, wr[c], col, g.cols, whole, h[c]);
          values_of_run(g.dn, wn[c], col, g.cols, whole, d[c]);
#pragma unroll
          for (int i = 0; i < kRun; ++i) {
            h[c][i] = i < n ? (h[c][i] - mean) * rstd : 0.0f;
            sg2[c][i] += d[c][i] * h[c][i];
            sb2[c][i] += d[c][i];
            d[c][i] *= gamma2[c][i];
            m[0] += d[c][i];
            m[1] += d[c][i] * h[c][i];
          }
        }
        sums(m);
        const float a = g.before.layer ? m[0] * part : 0.0f, b = m[1] * part;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < kRun; ++i) d[c][i] = rstd * (d[c][i] - a - h[c][i] * b);
      } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < kRun; ++i) d[c][i] = 0.0f;
      }
      Runs<CH> h;   // what the gate is multiplied with
      float mean = 0.0f, rstd = 1.0f, m[2] = {0.0f, 0.0f};
      if constexpr (AFTER) {
        mean = g.after.layer ? g.after.mean[row] : 0.0f;
        rstd = g.after.rstd[row];
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = (c * T + lane) * kRun, n = g.cols - col;
        if (g.dr.data) {
          float more[kRun];
          values_of_run(g.dr, wd[c], col, g.cols, whole, more);
#pragma unroll
          for (int i = 0; i < kRun; ++i) d[c][i] += more[i];
        }
        if (g.dx.data) {
          float o[kRun];
#pragma unroll
          for (int i = 0; i < kRun; ++i) o[i] = g.scale * d[c][i];
          store_run_of(g.dx, row, col, n, o);
        }
        if (!g.dblock.data && !g.block.data) continue;
        if (g.block.data) {
          values_of_run(g.block, wb[c], col, g.cols, whole, h[c]);
        } else {
#pragma unroll
          for (int i = 0; i < kRun; ++i) h[c][i] = 0.0f;
        }
        float own[kRun];
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          if (i >= n) d[c][i] = 0.0f;
          float y = h[c][i];
          if constexpr (AFTER) {
            h[c][i] = i < n ? (h[c][i] - mean) * rstd : 0.0f;
            y = h[c][i] * gamma1[c][i] + beta1[c][i];
          }
          own[i] = d[c][i] * y;
          sgate[c][i] += own[i];
          d[c][i] *= gate[c][i];
          if constexpr (AFTER) {
            sg1[c][i] += d[c][i] * h[c][i];
            sb1[c][i] += d[c][i];
            d[c][i] *= gamma1[c][i];
            m[0] += d[c][i];
            m[1] += d[c][i] * h[c][i];
          }
        }
        if (g.own_gates && g.want_gate && n > 0) store_run<MOC_F32>(g.gate_sums + row * g.cols, col, n, own);
      }
      if constexpr (AFTER) {
        sums(m);
        const float a = g.after.layer ? m[0] * part : 0.0f, b = m[1] * part;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < kRun; ++i) d[c][i] = rstd * (d[c][i] - a - h[c][i] * b);
      }
      if (g.dblock.data) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int col = (c * T + lane) * kRun;
          store_run_of(g.dblock, row, col, g.cols - col, d[c]);
        }
      }
    }
    if (g.want_gate && !g.own_gates) {
      put_sums<T, kRows, CH>(sgate, g.gate_sums + (which * g.chunks + chunk) * g.cols, g.cols, stage);
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < kRun; ++i) sgate[c][i] = 0.0f;
    }
  }
  float* out = g.sums + (int64_t)blockIdx.x * __builtin_popcount(g.kinds) * g.cols;
  if (g.kinds & kBeforeGamma) {
    put_sums<T, kRows, CH>(sg2, out, g.cols, stage);
    out += g.cols;
  }
  if (g.kinds & kBeforeBeta) {
    put_sums<T, kRows, CH>(sb2, out, g.cols, stage);
    out += g.cols;
  }
  if constexpr (AFTER) {
    if (g.kinds & kAfterGamma) {
      put_sums<T, kRows, CH>(sg1, out, g.cols, stage);
      out += g.cols;
    }
    if (g.kinds & kAfterBeta) put_sums<T, kRows, CH>(sb1, out, g.cols, stage);
  }
}

// ---- sums over workgroups -----------------------------------------------------------------------

struct JoinArgs {
  const float *sums, *gate_sums;
  float* out[4];      // of the kinds of sums, in their order
  float* gate;        // null: nothing to add up
  int kinds;
  int64_t parts, chunks, gates;
  int cols;
};

// 64 columns of one result a workgroup, a wave every sixteenth part.
__global__ __launch_bounds__(1024) void residual_join_kernel(JoinArgs g) {
  __shared__ float stage[16][kWave];
  const int lane = threadIdx.x % kWave, mine = threadIdx.x / kWave, col = blockIdx.x * kWave + lane;
  const int64_t which = blockIdx.y;
  const float* from;
  float* to;
  int64_t parts, stride;
  if (which < g.kinds) {
    from = g.sums + which * g.cols;
    stride = (int64_t)g.kinds * g.cols;
    parts = g.parts;
    to = g.out[which];
  } else {
    const int64_t gate = which - g.kinds;
    from = g.gate_sums + gate * g.chunks * g.cols;
    stride = g.cols;
    parts = g.chunks;
    to = g.gate + gate * g.cols;
  }
  float s = 0.0f;
  if (col < g.cols) {
    int64_t p = mine;
    for (; p + 48 < parts; p += 64) {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = from[(p + 16 * i) * stride + col];
      s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    for (; p < parts; p += 16) s += from[p * stride + col];
  }
  stage[mine][lane] = s;
  __syncthreads();
  if (mine == 0 && col < g.cols) {
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += stage[i][lane];
    to[col] = s;
  }
}

__global__ __launch_bounds__(256) void zero_kernel(float* out, int64_t count) {
  const int64_t at = block_of() * 256 + threadIdx.x;
  if (at < count) out[at] = 0.0f;
}

// ---- dispatch -----------------------------------------------------------------------------------

using Kernel = void (*)(ResidualArgs);
struct Shape {
  Kernel kern;
  int threads, rows;   // of a workgroup
};
template <bool AFTER>
Shape forward_shape(int64_t cols) {
  if (cols <= 512) return {residual_forward_kernel<64, 1, AFTER>, 256, 4};
  if (cols <= 1024) return {residual_forward_kernel<64, 2, AFTER>, 256, 4};
  if (cols <= 2048) return {residual_forward_kernel<256, 1, AFTER>, 256, 1};
  if (cols <= 4096) return {residual_forward_kernel<512, 1, AFTER>, 512, 1};
  if (cols <= 8192) return {residual_forward_kernel<1024, 1, AFTER>, 1024, 1};
  return {residual_forward_kernel<1024, 2, AFTER>, 1024, 1};
}
template <bool AFTER>
Shape backward_shape(int64_t cols) {
  if (cols <= 512) return {residual_backward_kernel<64, 1, AFTER>, 256, 4};
  if (cols <= 1024) return {residual_backward_kernel<64, 2, AFTER>, 256, 4};
  if (cols <= 2048) return {residual_backward_kernel<256, 1, AFTER>, 256, 1};
  if (cols <= 4096) return {residual_backward_kernel<512, 1, AFTER>, 512, 1};
  if (cols <= 8192) return {residual_backward_kernel<1024, 1, AFTER>, 1024, 1};
  return {residual_backward_kernel<1024, 2, AFTER>, 1024, 1};
}

// Which rows a workgroup of the backward pass takes.
struct Cut {
  int64_t chunks, chunk_rows, groups, workgroups;
  bool own;
};
Cut cut_of(const Shape& s, int64_t rows, int64_t gates, int units) {
  Cut c = {};
  c.own = gates > 1 && gates == rows;
  const int64_t apart = c.own || gates < 1 ? 1 : gates, each = rows / apart;
  const int64_t most = (int64_t)units * (kMaxThreads / s.threads), few = std::max<int64_t>(units, (rows + 8 * s.rows - 1) / (8 * s.rows));
  const int64_t wanted = std::max<int64_t>(1, std::min(most, few));
  const int64_t chunks = std::max<int64_t>(1, wanted / apart);
  c.chunk_rows = (each + chunks - 1) / chunks;
  c.chunk_rows = (c.chunk_rows + s.rows - 1) / s.rows * s.rows;
  c.chunks = (each + c.chunk_rows - 1) / c.chunk_rows;
  c.groups = c.chunks > 1 ? 1 : (apart + wanted - 1) / wanted;
  c.workgroups = c.chunks > 1 ? apart * c.chunks : (apart + c.groups - 1) / c.groups;
  return c;
}
int64_t sums_bytes(const Cut& c, int kinds, int64_t gates, bool gate_too, int64_t cols) {
  const int64_t rows = c.workgroups * __builtin_popcount(kinds) + (gate_too && !c.own && c.chunks > 1 ? gates * c.chunks : 0);
  return rows * cols * (int64_t)sizeof(float);
}

Mat mat_of(const moc_matrix* m) { return m ? Mat{m->data, m->scales, m->stride, m->scale_stride, m->type} : Mat{}; }

bool residual_sizes_ok(int64_t rows, int64_t cols, int64_t gates) {
  return sizes_ok(rows, cols) && cols >= 1 && cols <= MOC_RESIDUAL_MAX_COLS && gates >= 0 && gates <= std::max<int64_t>(rows, 1) && (gates < 1 || rows % gates == 0);
}
bool norm_ok(const moc_row_norm* n, int64_t rows) {
  if (!n || n->kind == MOC_NORM_NONE) return true;
  if (n->reserved != 0 || (n->kind != MOC_NORM_LAYER && n->kind != MOC_NORM_RMS) || !(n->eps >= 0.0f) || !params_ok(n->gamma, n->param_type) || !params_ok(n->beta, n->param_type)) return false;
  if (n->beta && n->kind == MOC_NORM_RMS) return false;
  if (rows == 0) return true;
  return n->rstd && aligned_to(n->rstd, 4) && (n->kind == MOC_NORM_RMS || (n->mean && aligned_to(n->mean, 4)));
}
RowNorm row_norm_of(const moc_row_norm* n) {
  RowNorm r = {};
  if (!n || n->kind == MOC_NORM_NONE) return r;
  r.gamma = n->gamma; r.beta = n->beta; r.param_type = n->param_type; r.eps = n->eps;
  r.on = true; r.layer = n->kind == MOC_NORM_LAYER; r.mean = n->mean; r.rstd = n->rstd;
  return r;
}
bool lies_over(const moc_matrix* out, std::initializer_list<const moc_matrix*> in) {
  if (!out || !out->data) return false;
  for (const moc_matrix* m : in)
    if (m && m->data == out->data) return true;
  return false;
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
  g.rows = rows; g.cols = (int)cols; g.gates = gates; g.rows_per_gate = gates > 0 ? rows / gates : rows;
  g.scale = scale;
  if (kept) g.most = most_kept(kept->type, n->type);
  g.parts = lies_over(r, {x, block, gate}) || lies_over(n, {x, block, gate});
  const Shape s = g.after.on ? forward_shape<true>(cols) : forward_shape<false>(cols);
  const int64_t there = (rows + s.rows - 1) / s.rows, wanted = (int64_t)units * (2 * kMaxThreads / s.threads);
  hipLaunchKernelGGL(s.kern, dim3((unsigned)std::min(there, wanted)), dim3(s.threads), 0, static_cast<hipStream_t>(hip_stream), g);
  MOC_HIP(hipGetLastError());
  return MOC_OK;
}

int64_t moc_residual_backward_work(int64_t rows, int64_t cols, int64_t gates) {
  if (!residual_sizes_ok(rows, cols, gates)) return MOC_EINVAL;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  if (rows == 0) return 0;
  const Cut c = cut_of(backward_shape<true>(cols), rows, gates, units);
  return sums_bytes(c, kBeforeGamma | kBeforeBeta | kAfterGamma | kAfterBeta, gates, true, cols);
}

int moc_residual_backward(int64_t rows, int64_t cols, const moc_matrix* dr, const moc_matrix* dn, const moc_matrix* r, const moc_matrix* block, const moc_matrix* gate, int64_t gates, float scale,
                          const moc_row_norm* after, const moc_row_norm* before, const moc_matrix* dx, const moc_matrix* dblock, const moc_residual_grads* grads, void* work,
                          int64_t work_bytes, void* hip_stream) {
  if (!residual_sizes_ok(rows, cols, gates) || !(scale - scale == 0.0f)) return MOC_EINVAL;
  if (!norm_ok(after, rows) || !norm_ok(before, rows)) return MOC_EINVAL;
  const bool first = after && after->kind != MOC_NORM_NONE, last = before && before->kind != MOC_NORM_NONE;
  if ((dr && !matrix_ok(dr, rows, cols, true, false)) || last != (dn != nullptr) || (dn && !matrix_ok(dn, rows, cols, true, false)) || (!dr && !dn)) return MOC_EINVAL;
  if (last && !matrix_ok(r, rows, cols, true, true)) return MOC_EINVAL;
  if ((gates > 0) != (gate != nullptr) || (gate && !matrix_ok(gate, gates, cols, true, false))) return MOC_EINVAL;
  const moc_residual_grads none = {}, &d = grads ? *grads : none;
  const bool needed = first || d.gate;   // the block's output
  if (needed && !matrix_ok(block, rows, cols, true, true)) return MOC_EINVAL;
  if ((dx && !matrix_ok(dx, rows, cols, true, false)) || (dblock && !matrix_ok(dblock, rows, cols, true, false))) return MOC_EINVAL;
  if ((d.gate && gates < 1) || (d.before_gamma && !last) || (d.after_gamma && !first)) return MOC_EINVAL;
  if ((d.before_beta && (!last || before->kind != MOC_NORM_LAYER)) || (d.after_beta && (!first || after->kind != MOC_NORM_LAYER))) return MOC_EINVAL;
  float* const out[4] = {d.before_gamma, d.before_beta, d.after_gamma, d.after_beta};
  for (const float* p : out)
    if (!aligned_to(p, 4)) return MOC_EINVAL;
  if (!aligned_to(d.gate, 4)) return MOC_EINVAL;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  int kinds = 0;
  for (int i = 0; i < 4; ++i) kinds |= out[i] ? 1 << i : 0;
  if (rows == 0) {
    for (float* p : out) {
      if (!p) continue;
      hipLaunchKernelGGL(zero_kernel, grid_of((cols + 255) / 256), dim3(256), 0, stream, p, cols);
      MOC_HIP(hipGetLastError());
    }
    if (d.gate) {
      hipLaunchKernelGGL(zero_kernel, grid_of((gates * cols + 255) / 256), dim3(256), 0, stream, d.gate, gates * cols);
      MOC_HIP(hipGetLastError());
    }
    return MOC_OK;
  }
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  const Shape s = first ? backward_shape<true>(cols) : backward_shape<false>(cols);
  const Cut c = cut_of(s, rows, gates, units);
  const bool gate_parts = d.gate && !c.own && c.chunks > 1;
  const int64_t need = sums_bytes(c, kinds, gates, d.gate != nullptr, cols);
  if (need > 0 && (!work || !aligned_to(work, 16) || work_bytes < need)) return MOC_EINVAL;
  ResidualArgs g = {};
  g.dr = mat_of(dr); g.dn = mat_of(dn); g.gate = mat_of(gate); g.dx = mat_of(dx); g.dblock = mat_of(dblock);
  if (last) g.r = mat_of(r);
  if (needed) g.block = mat_of(block);
  g.after = row_norm_of(after); g.before = row_norm_of(before);
  g.rows = rows; g.cols = (int)cols; g.gates = gates; g.rows_per_gate = gates > 0 && !c.own ? rows / gates : rows;
  g.scale = scale;
  g.parts = lies_over(dx, {dr, dn, r, block, gate}) || lies_over(dblock, {dr, dn, r, block, gate});
  g.kinds = kinds;
  g.sums = static_cast<float*>(work);
  g.want_gate = d.gate != nullptr; g.own_gates = c.own;
  float* const gate_room = gate_parts ? static_cast<float*>(work) + c.workgroups * __builtin_popcount(kinds) * cols : d.gate;
  g.gate_sums = gate_room;
  g.chunks = c.chunks; g.chunk_rows = c.chunk_rows; g.groups = c.groups;
  hipLaunchKernelGGL(s.kern, dim3((unsigned)c.workgroups), dim3(s.threads), 0, stream, g);
  MOC_HIP(hipGetLastError());
  JoinArgs j = {};
  j.sums = static_cast<const float*>(work); j.gate_sums = gate_room; j.gate = d.gate;
  for (int i = 0; i < 4; ++i)
    if (out[i]) j.out[j.kinds++] = out[i];
  j.parts = c.workgroups; j.chunks = c.chunks; j.gates = gate_parts ? gates : 0; j.cols = (int)cols;
  if (j.kinds + j.gates > 0) {
    hipLaunchKernelGGL(residual_join_kernel, dim3((unsigned)((cols + kWave - 1) / kWave), (unsigned)(j.kinds + j.gates)), dim3(1024), 0, stream, j);
    MOC_HIP(hipGetLastError());
  }
  return MOC_OK;
}

}  // extern "C"
