// Layer norm, forward and backward, with the reduction of the parameters' gradients.
//
// Bound by memory: every value is read once and written once.  T threads take a row and hold it in
// registers, CH runs of eight values each, so the variance is that of the differences from the mean
// and nothing is read again; rows longer than 16384 columns are read again from cache.  A wave a row
// up to 1024 columns (no barrier: 65536 x 1024 forward 77 -> 53 us, 5.0 TB/s), then 256 threads, then two
// runs a thread in the forward pass (32768 x 4096 bf16 116 us, 4.6 TB/s, and 139, 4.9, with an e4m3
// checkpoint; one run and two rows at a time 124 and 174).  The backward pass has no registers for two:
// 153 us, 5.3 TB/s, against 226.  Of 8193 to 16384 columns it has them all the same and spills 56 to 152 bytes a lane: 8192 x
// 16384 248 us, 3.3 TB/s, from int8 308, 2.2 (a quarter of a gigabyte read and a tenth written for it).  The last run of a ragged row is loaded whole and moved down when it is
// used, since a load in parts would be waited for (4999 x 1247, backward from int8: 32 -> 25 us).
// Workgroups go over many rows: gamma and beta stay in registers, and in the backward pass so do a
// column's two sums; they meet in the workspace, one row of sums a workgroup, and a second kernel adds
// those in their order.
#include <algorithm>

#include "moc_rows.h"

namespace {

constexpr int kMaxThreads = 1024;

struct NormArgs {
  const void* x;          // tensor or codes
  const uint8_t* x_scales;
  int64_t x_stride, x_scale_stride;
  const void *gamma, *beta;
  int param_type;
  float eps;
  float *mean, *rstd;
  // forward
  void* y;
  int y_type;
  int64_t y_stride;
  uint8_t *codes, *scales;
  int64_t code_stride, scale_stride;
  int kept_type;          // -1: none
  float most;
  // backward
  const void *dy, *residual;   // residual may be null
  int64_t dy_stride, residual_stride;
  float* sums;            // [gridDim][2][cols], null: no parameter gradients
  int64_t rows;
  int cols;
};

template <int X>
__device__ __forceinline__ const void* row_of(const void* x, int64_t row, int64_t stride) {
  return static_cast<const typename Stored<X>::type*>(x) + row * stride;
}
__device__ __forceinline__ char* row_any(const void* x, int type, int64_t row, int64_t stride) {
  return const_cast<char*>(static_cast<const char*>(x)) + row * stride * (type == MOC_F32 ? 4 : 2);
}

template <int X>
__device__ __forceinline__ void load_x(const NormArgs& g, int64_t row, int col, int n, float (&v)[kRun]) {
  load_held<X>(row_of<X>(g.x, row, g.x_stride), g.x_scales + row * g.x_scale_stride, col, n, v);
}
__device__ __forceinline__ bool whole_runs(const NormArgs& g) { return g.cols % kRun == 0; }

// ---- forward ------------------------------------------------------------------------------------

// y and its checkpoint of one run.
__device__ __forceinline__ void finish_run(const NormArgs& g, int64_t row, int col, int n, float mean, float rstd, const float (&ga)[kRun], const float (&be)[kRun],
                                           float (&v)[kRun]) {
#pragma unroll
  for (int i = 0; i < kRun; ++i) v[i] = (v[i] - mean) * rstd * ga[i] + be[i];
  if (n > 0) store_any(g.y_type, row_any(g.y, g.y_type, row, g.y_stride), col, n, v);
  if (g.kept_type < 0) return;
  if (n < kRun) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = i < n ? v[i] : 0.0f;
  }
  keep_any(g.kept_type, v, col, n, g.most, g.codes + row * g.code_stride, g.scales + row * g.scale_stride);
}

template <int X, int T, int CH>
__device__ __forceinline__ void load_row(const NormArgs& g, int64_t row, int lane, Raw (&w)[CH]) {
  const void* const x = row_of<X>(g.x, row, g.x_stride);
  const uint8_t* const scales = g.x_scales + row * g.x_scale_stride;
  if (g.cols >= kRun) {
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c] = load_raw_whole<X>(x, scales, (c * T + lane) * kRun, g.cols);
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c] = load_raw<X>(x, scales, (c * T + lane) * kRun, g.cols - (c * T + lane) * kRun);
  }
}

// Workgroups go over rows with gamma and beta in registers (from cache they would be four times the
// bytes of a row), R rows at a time, whose sums are taken together, and the next R on their way.  16
// waves a compute unit; 32 gain 6 % at 1024 columns and lose 10 % at 2048.
template <int X, int T, int CH, int R>
__global__ __launch_bounds__(T < 256 ? 256 : T, 4) void norm_forward_kernel(NormArgs g) {
  constexpr int kRows = T < 256 ? 256 / T : 1;   // groups of R rows of a workgroup at a time
  static_assert(T <= kWave || kRows == 1);
  using Sums = RowSums<T, R>;
  __shared__ float room[Sums::kRoom];
  Sums sums{room};
  const int lane = threadIdx.x % T;
  float ga[CH][kRun], be[CH][kRun];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = (c * T + lane) * kRun;
    load_param(g.gamma, g.param_type, min(col, g.cols - 1), g.cols - col, 1.0f, ga[c]);
    load_param(g.beta, g.param_type, min(col, g.cols - 1), g.cols - col, 0.0f, be[c]);
  }
  const float part = 1.0f / (float)g.cols;
  const bool whole = whole_runs(g);
  const int64_t step = (int64_t)gridDim.x * kRows * R;
  int64_t row = ((int64_t)blockIdx.x * kRows + (kRows > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / T) : 0)) * R;
  Raw w[R][CH];
  const auto load = [&](int64_t from) {   // beyond the last row it is read again
#pragma unroll
    for (int r = 0; r < R; ++r) load_row<X, T, CH>(g, min(from + r, g.rows - 1), lane, w[r]);
  };
  if (row < g.rows) load(row);
  for (; row < g.rows; row += step) {
    float v[R][CH][kRun], mean[R], rstd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] = 0.0f;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if (!whole) settle<X>(w[r][c], (c * T + lane) * kRun, g.cols);
        values_of<X>(w[r][c], v[r][c]);
        float s = 0.0f;   // 0 where a row ends inside a run
#pragma unroll
        for (int i = 0; i < kRun; ++i) s += v[r][c][i];
        mean[r] += (c * T + lane) * kRun < g.cols ? s : 0.0f;
      }
    }
    load(row + step);
    sums(mean);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] /= (float)g.cols;   // a division, so that equal values leave no difference
      rstd[r] = 0.0f;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int n = g.cols - (c * T + lane) * kRun;
        float q = 0.0f;
        if (whole) {
#pragma unroll
          for (int i = 0; i < kRun; ++i) q += (v[r][c][i] - mean[r]) * (v[r][c][i] - mean[r]);
        } else {
#pragma unroll
          for (int i = 0; i < kRun; ++i) q += i < n ? (v[r][c][i] - mean[r]) * (v[r][c][i] - mean[r]) : 0.0f;
        }
        rstd[r] += n > 0 ? q : 0.0f;
      }
    }
    sums(rstd);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= g.rows) break;
      rstd[r] = inverse_root(rstd[r] * part + g.eps);
      if (lane == 0) {
        g.mean[row + r] = mean[r];
        g.rstd[row + r] = rstd[r];
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = (c * T + lane) * kRun;
        finish_run(g, row + r, col, g.cols - col, mean[r], rstd[r], ga[c], be[c], v[r][c]);
      }
    }
  }
}

// Rows that do not fit the registers of a workgroup: read three times.
template <int X>
__global__ __launch_bounds__(kMaxThreads) void norm_forward_long_kernel(NormArgs g) {
  constexpr int T = kMaxThreads;
  using Sums = RowSums<T, 1>;
  __shared__ float room[Sums::kRoom];
  Sums sums{room};
  const int blocks = (g.cols + MOC_BLOCK - 1) / MOC_BLOCK * MOC_BLOCK;   // quads stay together
  for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
    float v[kRun], s[1] = {0.0f};
    for (int col = threadIdx.x * kRun; col < g.cols; col += T * kRun) {
      load_x<X>(g, row, col, g.cols - col, v);
#pragma unroll
      for (int i = 0; i < kRun; ++i) s[0] += v[i];
    }
    const float count = (float)g.cols;
    sums(s);
    const float mean = s[0] / count;
    float q[1] = {0.0f};
    for (int col = threadIdx.x * kRun; col < g.cols; col += T * kRun) {
      load_x<X>(g, row, col, g.cols - col, v);
#pragma unroll
      for (int i = 0; i < kRun; ++i) q[0] += i < g.cols - col ? (v[i] - mean) * (v[i] - mean) : 0.0f;
    }
    sums(q);
    const float rstd = inverse_root(q[0] / count + g.eps);
    if (threadIdx.x == 0) {
      g.mean[row] = mean;
      g.rstd[row] = rstd;
    }
    for (int col = threadIdx.x * kRun; col < blocks; col += T * kRun) {
      float ga[kRun], be[kRun];
      load_x<X>(g, row, min(col, g.cols - 1), g.cols - col, v);
      load_param(g.gamma, g.param_type, min(col, g.cols - 1), g.cols - col, 1.0f, ga);
      load_param(g.beta, g.param_type, min(col, g.cols - 1), g.cols - col, 0.0f, be);
      finish_run(g, row, col, g.cols - col, mean, rstd, ga, be, v);
    }
  }
}

// ---- backward -----------------------------------------------------------------------------------

// A row's run of x, dy and the residual, on its way or there.
struct GradRaw {
  Raw x, d, r;
};
template <int X, int D, bool WHOLE>
__device__ __forceinline__ GradRaw load_grad(const NormArgs& g, int64_t row, int col) {
  const void *const x = row_of<X>(g.x, row, g.x_stride), *const d = row_of<D>(g.dy, row, g.dy_stride), *const r = row_of<D>(g.residual, row, g.residual_stride);
  const uint8_t* const scales = g.x_scales + row * g.x_scale_stride;
  GradRaw w = {};
  if constexpr (WHOLE) {
    w.x = load_raw_whole<X>(x, scales, col, g.cols);
    w.d = load_raw_whole<D>(d, nullptr, col, g.cols);
    if (g.residual) w.r = load_raw_whole<D>(r, nullptr, col, g.cols);
  } else {
    w.x = load_raw<X>(x, scales, col, g.cols - col);
    w.d = load_raw<D>(d, nullptr, col, g.cols - col);
    if (g.residual) w.r = load_raw<D>(r, nullptr, col, g.cols - col);
  }
  return w;
}
template <int X, int D, int T, int CH>
__device__ __forceinline__ void load_grads(const NormArgs& g, int64_t row, int lane, GradRaw (&w)[CH]) {
  if (g.cols >= kRun) {
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c] = load_grad<X, D, true>(g, row, (c * T + lane) * kRun);
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c] = load_grad<X, D, false>(g, row, (c * T + lane) * kRun);
  }
}

// To the compiler, another value from here on.
__device__ __forceinline__ void opaque(Raw& w) {
  asm("" : "+v"(w.a));
  asm("" : "+v"(w.b));
}

// h and dy of a run, 0 beyond the row.
template <int X, int D>
__device__ __forceinline__ void values_of_grad(const NormArgs& g, const GradRaw& w, int col, float mean, float rstd, float (&h)[kRun], float (&d)[kRun]) {
  values_of<X>(w.x, h);
  values_of<D>(w.d, d);
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    h[i] = i < g.cols - col ? (h[i] - mean) * rstd : 0.0f;
    d[i] = i < g.cols - col ? d[i] : 0.0f;
  }
}

template <int D>
__device__ __forceinline__ void store_dx(const NormArgs& g, int64_t row, int col, float rstd, float a, float b, const float (&h)[kRun], const float (&d)[kRun],
                                         const float (&ga)[kRun], const Raw& residual) {
  const int n = g.cols - col;
  if (n <= 0) return;
  float o[kRun];
#pragma unroll
  for (int i = 0; i < kRun; ++i) o[i] = rstd * (d[i] * ga[i] - a - h[i] * b);
  if (g.residual) {
    float r[kRun];
    values_of<D>(residual, r);
#pragma unroll
    for (int i = 0; i < kRun; ++i) o[i] += r[i];
  }
  store_run<D>(const_cast<void*>(row_of<D>(g.y, row, g.y_stride)), col, n, o);
}

// The sums of a workgroup's rows groups (kRows of T lanes), added in their order, into its row of the
// workspace.
template <int T, int kRows, int CH>
__device__ __forceinline__ void store_sums(const NormArgs& g, const float (&sg)[CH][kRun], const float (&sb)[CH][kRun], float* stage) {
  const int lane = threadIdx.x % T, mine = threadIdx.x / T;
  float* const out = g.sums + (int64_t)blockIdx.x * 2 * g.cols;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float a[kRun], b[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      a[i] = sg[c][i];
      b[i] = sb[c][i];
    }
    if constexpr (kRows > 1) {   // stage: [kRows][16][T]
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        stage[(mine * 16 + i) * T + lane] = a[i];
        stage[(mine * 16 + 8 + i) * T + lane] = b[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRun; ++i) a[i] = b[i] = 0.0f;
      if (mine == 0) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
          for (int i = 0; i < kRun; ++i) {
            a[i] += stage[(r * 16 + i) * T + lane];
            b[i] += stage[(r * 16 + 8 + i) * T + lane];
          }
      }
    }
    const int col = (c * T + lane) * kRun, n = g.cols - col;
    if (mine == 0 && n > 0) {
      store_run<MOC_F32>(out, col, n, a);
      store_run<MOC_F32>(out + g.cols, col, n, b);
    }
  }
}

// 16 waves a compute unit, 128 registers a thread; a wave a row with two runs a lane has 12, or 8 where x is float32 or
// a checkpoint (65536 x 1024 float32 168 us, 310 with 12 and what that spills).  The next row is on its way while the
// sums over this one are taken.
template <int X, int D, int T, int CH>
__global__ __launch_bounds__(T < 256 ? 256 : T, CH > 1 && T == kWave ? (X == MOC_F32 || X == MOC_E4M3 || X == MOC_I8 ? 2 : 3) : 4) void norm_backward_kernel(NormArgs g) {
  constexpr int kRows = T < 256 ? 256 / T : 1;
  static_assert(T <= kWave || kRows == 1);
  using Sums = RowSums<T, 2>;
  __shared__ float room[Sums::kRoom];
  Sums sums{room};
  __shared__ float stage[kRows > 1 ? kRows * 16 * T : 1];
  const int lane = threadIdx.x % T;
  constexpr bool kHold = CH == 1 || T == kWave;   // gamma, in registers; from cache where two runs leave none
  float held[CH][kRun], sg[CH][kRun], sb[CH][kRun];
  const auto gamma_of = [&](int c, float(&ga)[kRun]) {
    const int col = (c * T + lane) * kRun;
    load_param(g.gamma, g.param_type, min(col, g.cols - 1), g.cols - col, 1.0f, ga);
  };
  if constexpr (kHold) {
#pragma unroll
    for (int c = 0; c < CH; ++c) gamma_of(c, held[c]);
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) sg[c][i] = sb[c][i] = 0.0f;
  }
  const float part = 1.0f / (float)g.cols;
  const bool whole = whole_runs(g);
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + (kRows > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / T) : 0);
  constexpr bool kAhead = CH == 1 || T == kWave;   // two runs a thread: no registers for it
  GradRaw w[CH];
  float mean = 0.0f, rstd = 0.0f;
  if (kAhead && row < g.rows) {
    load_grads<X, D, T, CH>(g, row, lane, w);
    mean = g.mean[row];
    rstd = g.rstd[row];
  }
  while (row < g.rows) {
    if constexpr (!kAhead) {
      load_grads<X, D, T, CH>(g, row, lane, w);
      mean = g.mean[row];
      rstd = g.rstd[row];
    }
    // the row stays as it was loaded, and is converted once more after the sums: fewer registers
    GradRaw now[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) now[c] = w[c];
    if (!whole) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = (c * T + lane) * kRun;
        settle<X>(now[c].x, col, g.cols);
        settle<D>(now[c].d, col, g.cols);
        settle<D>(now[c].r, col, g.cols);
      }
    }
    const float mu = mean, scale = rstd;
    const int64_t next = row + step;
    if (kAhead && next < g.rows) {
      load_grads<X, D, T, CH>(g, next, lane, w);
      mean = g.mean[next];
      rstd = g.rstd[next];
    }
    float m[2] = {0.0f, 0.0f};   // of p, of p * h
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float h[kRun], d[kRun], ga[kRun];
      values_of_grad<X, D>(g, now[c], (c * T + lane) * kRun, mu, scale, h, d);
      if constexpr (!kHold) gamma_of(c, ga);
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        if constexpr (kHold) ga[i] = held[c][i];
        const float p = d[i] * ga[i];
        m[0] += p;
        m[1] += p * h[i];
        sg[c][i] += d[i] * h[i];
        sb[c][i] += d[i];
      }
    }
    sums(m);
    const float a = m[0] * part, b = m[1] * part;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float h[kRun], d[kRun], ga[kRun];
      if constexpr (CH > 1) {   // or both conversions become one, and kept
        opaque(now[c].x);
        opaque(now[c].d);
      }
      values_of_grad<X, D>(g, now[c], (c * T + lane) * kRun, mu, scale, h, d);
      if constexpr (!kHold) gamma_of(c, ga);
#pragma unroll
      for (int i = 0; i < kRun; ++i)
        if constexpr (kHold) ga[i] = held[c][i];
      store_dx<D>(g, row, (c * T + lane) * kRun, scale, a, b, h, d, ga, now[c].r);
    }
    row = next;
  }
  if (g.sums) store_sums<T, kRows, CH>(g, sg, sb, stage);
}

// Rows that do not fit the registers: two passes a row; the sums go to the workspace as they grow
// (a workgroup's own row of it, zeroed first).
template <int X, int D>
__global__ __launch_bounds__(kMaxThreads) void norm_backward_long_kernel(NormArgs g) {
  constexpr int T = kMaxThreads;
  using Sums = RowSums<T, 2>;
  __shared__ float room[Sums::kRoom];
  Sums over_row{room};
  float* const sums = g.sums ? g.sums + (int64_t)blockIdx.x * 2 * g.cols : nullptr;
  const float count = (float)g.cols;
  if (sums) {
    const float zero[kRun] = {};
    for (int col = threadIdx.x * kRun; col < g.cols; col += T * kRun) {
      store_run<MOC_F32>(sums, col, g.cols - col, zero);
      store_run<MOC_F32>(sums + g.cols, col, g.cols - col, zero);
    }
  }
  for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
    const float mean = g.mean[row], rstd = g.rstd[row];
    float h[kRun], d[kRun], ga[kRun], m[2] = {0.0f, 0.0f};
    for (int col = threadIdx.x * kRun; col < g.cols; col += T * kRun) {
      const int n = g.cols - col;
      values_of_grad<X, D>(g, load_grad<X, D, false>(g, row, col), col, mean, rstd, h, d);
      load_param(g.gamma, g.param_type, col, n, 1.0f, ga);
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        m[0] += d[i] * ga[i];
        m[1] += d[i] * ga[i] * h[i];
      }
      if (sums) {   // the same thread's columns in every row
        float s[kRun], t[kRun];
        load_run<MOC_F32>(sums, col, n, s);
        load_run<MOC_F32>(sums + g.cols, col, n, t);
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          s[i] += d[i] * h[i];
          t[i] += d[i];
        }
        store_run<MOC_F32>(sums, col, n, s);
        store_run<MOC_F32>(sums + g.cols, col, n, t);
      }
    }
    over_row(m);
    const float a = m[0] / count, b = m[1] / count;
    for (int col = threadIdx.x * kRun; col < g.cols; col += T * kRun) {
      const GradRaw w = load_grad<X, D, false>(g, row, col);
      values_of_grad<X, D>(g, w, col, mean, rstd, h, d);
      load_param(g.gamma, g.param_type, col, g.cols - col, 1.0f, ga);
      store_dx<D>(g, row, col, rstd, a, b, h, d, ga, w.r);
    }
  }
}

// ---- dispatch -----------------------------------------------------------------------------------

using NormKernel = void (*)(NormArgs);
struct Shape {
  NormKernel kern;
  int threads, rows;   // of a workgroup
};

template <int X>
Shape forward_shape(int64_t cols) {
  if (cols <= 512) return {norm_forward_kernel<X, 64, 1, 2>, 256, 8};
  if (cols <= 1024) return {norm_forward_kernel<X, 64, 2, X == MOC_F32 ? 1 : 2>, 256, X == MOC_F32 ? 4 : 8};   // two rows of float32 do not fit the registers
  if (cols <= 2048) return {norm_forward_kernel<X, 256, 1, 2>, 256, 2};
  if (cols <= 4096) return {norm_forward_kernel<X, 256, 2, 1>, 256, 1};
  if (cols <= 8192) return {norm_forward_kernel<X, 512, 2, 1>, 512, 1};
  if (cols <= 16384) return {norm_forward_kernel<X, 1024, 2, 1>, 1024, 1};
  return {norm_forward_long_kernel<X>, kMaxThreads, 1};
}
Shape forward_shape_of(int type, int64_t cols) {
  switch (type) {
    case MOC_F32: return forward_shape<MOC_F32>(cols);
    case MOC_F16: return forward_shape<MOC_F16>(cols);
    case MOC_BF16: return forward_shape<MOC_BF16>(cols);
    case MOC_E4M3: return forward_shape<MOC_E4M3>(cols);
    default: return forward_shape<MOC_I8>(cols);
  }
}
template <int X, int D>
Shape backward_shape(int64_t cols) {
  if (cols <= 512) return {norm_backward_kernel<X, D, 64, 1>, 256, 4};
  if (cols <= 1024) return {norm_backward_kernel<X, D, 64, 2>, 256, 4};
  if (cols <= 2048) return {norm_backward_kernel<X, D, 256, 1>, 256, 1};
  if (cols <= 4096) return {norm_backward_kernel<X, D, 512, 1>, 512, 1};
  if (cols <= 8192) return {norm_backward_kernel<X, D, 1024, 1>, 1024, 1};
  if (cols <= 16384) return {norm_backward_kernel<X, D, 1024, 2>, 1024, 1};
  return {norm_backward_long_kernel<X, D>, kMaxThreads, 1};
}
// x of dy's type, or a checkpoint
template <int D>
Shape backward_shape_of(int type, int64_t cols) {
  return type == MOC_E4M3 ? backward_shape<MOC_E4M3, D>(cols) : type == MOC_I8 ? backward_shape<MOC_I8, D>(cols) : backward_shape<D, D>(cols);
}
Shape backward_shape_of(int type, int dy_type, int64_t cols) {
  return dy_type == MOC_BF16 ? backward_shape_of<MOC_BF16>(type, cols) : dy_type == MOC_F16 ? backward_shape_of<MOC_F16>(type, cols) : backward_shape_of<MOC_F32>(type, cols);
}

// Workgroups: what the compute units hold at a time, no more (the backward pass writes the sums of each
// and reads them again).
int64_t groups_of(const Shape& s, int64_t rows, int units) {
  const int64_t wanted = (int64_t)units * (kMaxThreads / s.threads), there = (rows + s.rows - 1) / s.rows;
  return there < wanted ? there : wanted;
}
// In the backward pass eight rows for each that a workgroup takes at a time, where that leaves every unit one: the sums
// of fewer rows cost as much as the rows (1000 x 1247 18.5 -> 10.7 us, 5000 x 1000 20.9 -> 14.4; sixteen gain nothing more
// and cost 4999 x 1247 3 us).
int64_t backward_groups(int64_t rows, int64_t cols, int units) {
  const Shape s = backward_shape<MOC_BF16, MOC_BF16>(cols);   // does not depend on the types
  const int64_t most = groups_of(s, rows, units), few = (rows + 8 * s.rows - 1) / (8 * s.rows);
  return std::min(most, std::max<int64_t>(few, units));
}

}  // namespace

extern "C" {

int moc_norm_forward(int64_t rows, int64_t cols, const moc_matrix* x, const void* gamma, const void* beta, int32_t param_type, float eps,
                     const moc_matrix* y, const moc_matrix* kept, float* mean, float* rstd, void* hip_stream) {
  if (!sizes_ok(rows, cols) || cols < 1 || !(eps >= 0.0f)) return MOC_EINVAL;
  if (!matrix_ok(x, rows, cols, true, true) || !matrix_ok(y, rows, cols, true, false) || (kept && !matrix_ok(kept, rows, cols, false, true))) return MOC_EINVAL;
  if (!params_ok(gamma, param_type) || !params_ok(beta, param_type)) return MOC_EINVAL;
  if (rows == 0) return MOC_OK;
  if (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return MOC_EINVAL;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  NormArgs g = {};
  g.x = x->data; g.x_scales = x->scales; g.x_stride = x->stride; g.x_scale_stride = x->scale_stride;
  g.gamma = gamma; g.beta = beta; g.param_type = param_type; g.eps = eps;
  g.mean = mean; g.rstd = rstd;
  g.y = y->data; g.y_type = y->type; g.y_stride = y->stride;
  g.kept_type = -1;
  if (kept) {
    g.codes = static_cast<uint8_t*>(kept->data); g.scales = kept->scales;
    g.code_stride = kept->stride; g.scale_stride = kept->scale_stride;
    g.kept_type = kept->type;
    g.most = most_kept(kept->type, y->type);
  }
  g.rows = rows; g.cols = (int)cols;
  const Shape s = forward_shape_of(x->type, cols);
  hipLaunchKernelGGL(s.kern, dim3((unsigned)groups_of(s, rows, units)), dim3(s.threads), 0, static_cast<hipStream_t>(hip_stream), g);
  MOC_HIP(hipGetLastError());
  return MOC_OK;
}

int64_t moc_norm_backward_work(int64_t rows, int64_t cols) {
  if (!sizes_ok(rows, cols) || cols < 1) return MOC_EINVAL;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  return backward_groups(rows, cols, units) * 2 * cols * (int64_t)sizeof(float);
}

int moc_norm_backward(int64_t rows, int64_t cols, const moc_matrix* dy, const moc_matrix* x, const void* gamma, int32_t param_type,
                      const float* mean, const float* rstd, const moc_matrix* residual, const moc_matrix* dx, float* dgamma, float* dbeta,
                      void* work, int64_t work_bytes, void* hip_stream) {
  if (!sizes_ok(rows, cols) || cols < 1) return MOC_EINVAL;
  if (!matrix_ok(dy, rows, cols, true, false) || !matrix_ok(x, rows, cols, true, true) || !matrix_ok(dx, rows, cols, true, false)) return MOC_EINVAL;
  if ((residual && !matrix_ok(residual, rows, cols, true, false)) || !params_ok(gamma, param_type)) return MOC_EINVAL;
  if (dx->type != dy->type || (residual && residual->type != dy->type) || (is_value(x->type) && x->type != dy->type)) return MOC_EINVAL;
  if ((dgamma == nullptr) != (dbeta == nullptr) || !aligned_to(dgamma, 4) || !aligned_to(dbeta, 4)) return MOC_EINVAL;
  if (rows > 0 && (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4))) return MOC_EINVAL;
  if (rows == 0 && !dgamma) return MOC_OK;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  const int64_t groups = backward_groups(rows, cols, units);
  if (dgamma && groups > 0 && (!work || !aligned_to(work, 16) || work_bytes < groups * 2 * cols * (int64_t)sizeof(float))) return MOC_EINVAL;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (rows > 0) {
    NormArgs g = {};
    g.x = x->data; g.x_scales = x->scales; g.x_stride = x->stride; g.x_scale_stride = x->scale_stride;
    g.gamma = gamma; g.param_type = param_type;
    g.mean = const_cast<float*>(mean); g.rstd = const_cast<float*>(rstd);
    g.y = dx->data; g.y_stride = dx->stride;
    g.dy = dy->data; g.dy_stride = dy->stride;
    if (residual) {
      g.residual = residual->data; g.residual_stride = residual->stride;
    }
    g.sums = dgamma ? static_cast<float*>(work) : nullptr;
    g.rows = rows; g.cols = (int)cols;
    const Shape s = backward_shape_of(x->type, dy->type, cols);
    hipLaunchKernelGGL(s.kern, dim3((unsigned)groups), dim3(s.threads), 0, stream, g);
    MOC_HIP(hipGetLastError());
  }
  if (dgamma) {
    // the sums of a workgroup are dgamma's and dbeta's one after the other, and so they may be wanted
    const float* const sums = static_cast<const float*>(work);
    const bool together = dbeta == dgamma + cols;
    for (int i = 0; i < (together ? 1 : 2); ++i) {
      const int64_t wide = together ? 2 * cols : cols;
      hipLaunchKernelGGL(join_sums_kernel, dim3((unsigned)((wide + 63) / 64)), dim3(1024), 0, stream, sums + i * cols, (int)groups, wide, 2 * cols, i ? dbeta : dgamma);
      MOC_HIP(hipGetLastError());
    }
  }
  return MOC_OK;
}

}  // extern "C"
