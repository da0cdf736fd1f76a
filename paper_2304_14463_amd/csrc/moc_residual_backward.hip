// The residual connection's gradients, with the reductions of the gate's and the parameters' gradients.
#include "moc_residual_backward.h"

namespace {

// ---- backward -----------------------------------------------------------------------------------

// For anything: what a matrix holds is asked at every run.  The next row is on its way where registers are left for it.
template <int T, int CH, bool AFTER>
__global__ __launch_bounds__(T < 256 ? 256 : T) void residual_backward_any_kernel(ResidualArgs g) {
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
  const uint32_t from = g.chunks > 1 ? blockIdx.x / g.chunks : blockIdx.x * g.groups, last = min(from + (g.chunks > 1 ? 1 : g.groups), g.own_gates ? 1 : max(g.gates, 1u));
  const uint32_t chunk = g.chunks > 1 ? blockIdx.x - from * g.chunks : 0;
  constexpr bool kAhead = CH == 1 || T <= 512;
  Raw wr[CH], wn[CH], wd[CH], wb[CH], wg[CH];
  float next_mean2 = 0.0f, next_rstd2 = 0.0f, next_mean1 = 0.0f, next_rstd1 = 1.0f;
  const auto load = [&](uint32_t row) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * T + lane) * kRun;
      if (g.before.on) {
        wr[c] = load_run_of<kAny>(g.r, row, col, g.cols, whole);
        wn[c] = load_run_of<kAny>(g.dn, row, col, g.cols, whole);
      }
      if (g.dr.data) wd[c] = load_run_of<kAny>(g.dr, row, col, g.cols, whole);
      if (g.block.data) wb[c] = load_run_of<kAny>(g.block, row, col, g.cols, whole);
      if (g.own_gates) wg[c] = load_run_of<kTensor>(g.gate, row, col, g.cols, whole);
    }
    if (g.before.on) {
      next_rstd2 = g.before.rstd[row];
      if (g.before.layer) next_mean2 = g.before.mean[row];
    }
    if constexpr (AFTER) {
      next_rstd1 = g.after.rstd[row];
      if (g.after.layer) next_mean1 = g.after.mean[row];
    }
  };
  for (uint32_t which = from; which < last; ++which) {
    const uint32_t first = which * g.rows_per_gate + chunk * g.chunk_rows, end = min(first + g.chunk_rows, (which + 1) * g.rows_per_gate);
    if (!g.own_gates) hold_gate<T, CH>(g, which, lane, gate);
    uint32_t row = first + mine;
    if (kAhead && row < end) load(row);
    for (; row < end; row += kRows) {   // groups of lanes that end earlier share no barrier
      if (!kAhead) load(row);
      Raw r[CH], n_[CH], s_[CH], b[CH];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        r[c] = wr[c];
        n_[c] = wn[c];
        s_[c] = wd[c];
        b[c] = wb[c];
        if (g.own_gates) values_of_run<kTensor>(g.gate, wg[c], (c * T + lane) * kRun, g.cols, whole, gate[c]);
      }
      const float mean2 = next_mean2, rstd2 = next_rstd2, mean1 = next_mean1, rstd1 = next_rstd1;
      if (kAhead && row + kRows < end) load(row + kRows);
      Runs<CH> d;
      if (g.before.on) {
        Runs<CH> h;
        float m[2] = {0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int col = asked_again((c * T + lane) * kRun);
          values_of_run<kAny>(g.r, r[c], col, g.cols, whole, h[c]);
          values_of_run<kAny>(g.dn, n_[c], col, g.cols, whole, d[c]);
          before_run(h[c], d[c], mean2, rstd2, gamma2[c], sg2[c], sb2[c], m);   // beyond the row h meets zeros
        }
        sums(m);
        const float ma = g.before.layer ? m[0] * part : 0.0f, mb = m[1] * part;
#pragma unroll
        for (int c = 0; c < CH; ++c) norm_gradient(d[c], h[c], rstd2, ma, mb);
      } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < kRun; ++i) d[c][i] = 0.0f;
      }
      Runs<CH> h;   // what the gate is multiplied with
      float m[2] = {0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = asked_again((c * T + lane) * kRun), n = g.cols - col;
        if (g.dr.data) {
          float more[kRun];
          values_of_run<kAny>(g.dr, s_[c], col, g.cols, whole, more);
          add_run(d[c], more);
        }
        if (g.dx.data) {
          float o[kRun];
#pragma unroll
          for (int i = 0; i < kRun; ++i) o[i] = g.scale * d[c][i];
          store_run_of<kAny>(g.dx, row, col, n, o);
        }
        if (!g.dblock.data && !g.block.data) continue;
        if (g.block.data) {
          values_of_run<kAny>(g.block, b[c], col, g.cols, whole, h[c]);
        } else {
#pragma unroll
          for (int i = 0; i < kRun; ++i) h[c][i] = 0.0f;
        }
        if (n < kRun) {
#pragma unroll
          for (int i = 0; i < kRun; ++i) d[c][i] = i < n ? d[c][i] : 0.0f;
        }
        float own[kRun];
        gate_run<AFTER>(h[c], d[c], own, mean1, rstd1, gamma1[c], beta1[c], gate[c], sg1[c], sb1[c], m);
        add_run(sgate[c], own);
        if (g.own_gates && g.want_gate && n > 0) store_run<MOC_F32>(g.gate_sums + (uint64_t)row * g.cols, col, n, own);
      }
      if constexpr (AFTER) {
        sums(m);
        const float ma = g.after.layer ? m[0] * part : 0.0f, mb = m[1] * part;
#pragma unroll
        for (int c = 0; c < CH; ++c) norm_gradient(d[c], h[c], rstd1, ma, mb);
      }
      if (g.dblock.data) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int col = asked_again((c * T + lane) * kRun);
          store_run_of<kAny>(g.dblock, row, col, g.cols - col, d[c]);
        }
      }
    }
    if (g.want_gate && !g.own_gates) {
      put_sums<T, kRows, CH>(sgate, g.gate_sums + (uint64_t)(which * g.chunks + chunk) * g.cols, g.cols, stage);
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

template <bool AFTER>
ResidualShape any_shape(int64_t cols) {
  if (cols <= 512) return {residual_backward_any_kernel<64, 1, AFTER>, 256, 4};
  if (cols <= 1024) return {residual_backward_any_kernel<64, 2, AFTER>, 256, 4};
  if (cols <= 2048) return {residual_backward_any_kernel<256, 1, AFTER>, 256, 1};
  if (cols <= 4096) return {residual_backward_any_kernel<512, 1, AFTER>, 512, 1};
  if (cols <= 8192) return {residual_backward_any_kernel<512, 2, AFTER>, 512, 1};
  return {residual_backward_any_kernel<1024, 2, AFTER>, 1024, 1};
}
ResidualShape any_shape(bool after, int64_t cols) { return after ? any_shape<true>(cols) : any_shape<false>(cols); }

constexpr int kFewWaves = 8, kManyWaves = 16;   // 256 and 128 registers a lane

// Which rows a workgroup of the backward pass takes.
struct Cut {
  int64_t chunks, chunk_rows, groups, workgroups;
  bool own;
};
// `waves`: of a compute unit, by the kernels' registers.
Cut cut_of(const ResidualShape& s, int64_t rows, int64_t gates, int units, int waves) {
  Cut c = {};
  c.own = gates > 1 && gates == rows;
  const int64_t apart = c.own || gates < 1 ? 1 : gates, each = rows / apart;
  const int64_t most = (int64_t)units * std::max(1, waves * kWave / s.threads), few = std::max<int64_t>(units, (rows + 8 * s.rows - 1) / (8 * s.rows));
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

}  // namespace

extern "C" {

int64_t moc_residual_backward_work(int64_t rows, int64_t cols, int64_t gates) {
  if (!residual_sizes_ok(rows, cols, gates)) return MOC_EINVAL;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  if (rows == 0) return 0;
  const auto bytes = [&](int waves) { return sums_bytes(cut_of(any_shape(true, cols), rows, gates, units, waves), kBeforeGamma | kBeforeBeta | kAfterGamma | kAfterBeta, gates, true, cols); };
  return std::max(bytes(kFewWaves), bytes(kManyWaves));
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
  ResidualArgs g = {};
  g.parts = lies_over(dx, {dr, dn, r, block, gate}) || lies_over(dblock, {dr, dn, r, block, gate});
  // kernels made for some types, where all matrices are of them and a row's last run may be loaded whole
  const bool ragged = cols < kRun || (g.parts && cols % kRun != 0), usual = dblock && !ragged, own = gates > 1 && gates == rows;
  const int kd = agreed({dn, dblock}, kAny), ks = agreed({dr, last ? r : nullptr, dx}, kAny), kb = needed ? kind_of(block->type) : kd;
  const int mode = (last ? kBefore : 0) | (dr ? kStream : 0) | (needed ? kBlock : 0) | (first ? kAfter : 0) | (!needed && (gate || !last) ? kGate : 0);
  ResidualShape s = {};
  if (usual) {
    if (kd == MOC_F32) s = moc_residual_backward_f32(ks, kb, mode, own, cols);
    if (kd == MOC_BF16) s = moc_residual_backward_bf16(ks, kb, mode, own, cols);
    if (kd == MOC_F16) s = moc_residual_backward_f16(ks, kb, mode, own, cols);
  }
  if (!s.kern) s = any_shape(first, cols);
  const Cut c = cut_of(s, rows, gates, units, !needed && !gate && cols <= 4096 ? kManyWaves : kFewWaves);
  const bool gate_parts = d.gate && !c.own && c.chunks > 1;
  const int64_t need = sums_bytes(c, kinds, gates, d.gate != nullptr, cols);
  if (need > 0 && (!work || !aligned_to(work, 16) || work_bytes < need)) return MOC_EINVAL;
  g.dr = mat_of(dr); g.dn = mat_of(dn); g.gate = mat_of(gate); g.dx = mat_of(dx); g.dblock = mat_of(dblock);
  if (last) g.r = mat_of(r);
  if (needed) g.block = mat_of(block);
  g.after = row_norm_of(after); g.before = row_norm_of(before);
  g.cols = (int)cols; g.gates = (uint32_t)gates; g.rows_per_gate = (uint32_t)(gates > 0 && !c.own ? rows / gates : rows);
  g.scale = scale;
  g.kinds = kinds;
  g.sums = static_cast<float*>(work);
  g.want_gate = d.gate != nullptr; g.own_gates = c.own;
  float* const gate_room = gate_parts ? static_cast<float*>(work) + c.workgroups * __builtin_popcount(kinds) * cols : d.gate;
  g.gate_sums = gate_room;
  g.chunks = (uint32_t)c.chunks; g.chunk_rows = (uint32_t)c.chunk_rows; g.groups = (uint32_t)c.groups;
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
