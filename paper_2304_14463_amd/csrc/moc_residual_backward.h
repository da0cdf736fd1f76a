// The residual connection's gradients: kernels made for types, and which of them a size takes.
#pragma once

#include "moc_residual.h"

using ResidualKernel = void (*)(ResidualArgs);
struct ResidualShape {
  ResidualKernel kern;
  int threads, rows;   // of a workgroup
};
// What a kernel is made for: a norm before the next block, a gradient of the stream, the block's output looked at, a norm behind it;
// a gate, without a look at the block's output.
constexpr int kBefore = 1, kStream = 2, kBlock = 4, kAfter = 8, kGate = 16;

// In a source file of its own for each type of the norm's and the block's gradients; kern is null where there is none.
ResidualShape moc_residual_backward_bf16(int stream, int block, int mode, bool own, int64_t cols);
ResidualShape moc_residual_backward_f16(int stream, int block, int mode, bool own, int64_t cols);
ResidualShape moc_residual_backward_f32(int stream, int block, int mode, bool own, int64_t cols);

namespace {

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

// Where a workgroup's parameters are: a run's in registers; all in LDS, of which a lane reads what it has written, where with both
// norms two runs a lane do not fit (8192 x 8192 bf16 180 us, 249 with registers spilled, float32 407 and 729; with one run a lane
// 261 and 576); or in cache.  Of 1025 to 2048 columns LDS leaves room for three workgroups a unit for two: 4998 x 1247 37 us, 35 without.
constexpr int kRegisters = 0, kLds = 1, kCache = 2;
template <int WHERE>
__device__ __forceinline__ const float (&param_at(const float (&held)[kRun], const float* lds, const void* p, int type, int col, int cols, float other, float (&room)[kRun]))[kRun] {
  if constexpr (WHERE == kLds) {
    __builtin_memcpy(room, lds + col, sizeof room);
    return room;
  } else {
    return param_of<WHERE == kRegisters>(held, p, type, col, cols, other, room);
  }
}
template <int T, int CH, int WHERE>
__device__ __forceinline__ void place_param(const void* p, int type, int lane, int cols, float other, Runs<CH>& v, float* lds) {
  hold_param<T, CH>(p, type, lane, cols, other, v);
  if constexpr (WHERE == kLds) {
#pragma unroll
    for (int c = 0; c < CH; ++c) __builtin_memcpy(lds + (c * T + lane) * kRun, v[c], sizeof v[c]);
  }
}

// Made for types, of a call with dblock.  MODE: what there is; the gate of kBlock, kAfter and kGate may be ones.
// OWN: a gate for every row.  Lanes beyond the row take no part but in the sums.
template <int S, int B, int D, int T, int CH, int MODE, bool OWN>
__global__ __launch_bounds__(T < 256 ? 256 : T) void residual_backward_kernel(ResidualArgs g) {
  constexpr int kRows = T < 256 ? 256 / T : 1;
  constexpr bool kAhead = CH == 1 || T <= 512;
  constexpr bool BEFORE = (MODE & kBefore) != 0, STREAM = (MODE & kStream) != 0, BLOCK = (MODE & kBlock) != 0, AFTER = (MODE & kAfter) != 0, GATE = BLOCK || (MODE & kGate) != 0;
  constexpr int kWhere = !kAhead ? kCache : T == 512 && CH == 2 && BEFORE && AFTER ? kLds : kRegisters, kPlaces = kWhere == kLds ? T * CH * kRun : 0;
  using Sums = RowSums<T, 2>;
  __shared__ float room[Sums::kRoom];
  __shared__ __attribute__((aligned(16))) float params[kWhere == kLds ? 4 * kPlaces : 1];
  __shared__ float stage[kRows > 1 ? kRows * kRun * T : 1];
  Sums sums{room};
  const uint32_t lane = threadIdx.x % T, mine = kRows > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / T) : 0, cols = g.cols;
  // a norm without a mean has 0 for it
  const float part = 1.0f / (float)cols, part2 = g.before.layer ? part : 0.0f, part1 = g.after.layer ? part : 0.0f;
  const float *const means2 = g.before.layer ? g.before.mean : g.before.rstd, *const means1 = g.after.layer ? g.after.mean : g.after.rstd;
  const float layer2 = g.before.layer ? 1.0f : 0.0f, layer1 = g.after.layer ? 1.0f : 0.0f;
  Runs<CH> gamma1, beta1, gate, gamma2;
  Runs<CH> sg1, sb1, sgate, sg2, sb2;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < kRun; ++i) sg1[c][i] = sb1[c][i] = sgate[c][i] = sg2[c][i] = sb2[c][i] = 0.0f;
  const uint32_t from = g.chunks > 1 ? blockIdx.x / g.chunks : blockIdx.x * g.groups, last = min(from + (g.chunks > 1 ? 1 : g.groups), OWN ? 1 : max(g.gates, 1u));
  const uint32_t chunk = g.chunks > 1 ? blockIdx.x - from * g.chunks : 0;
  Raw wr[CH], wn[CH], wd[CH], wb[CH], wg[CH];
  float stats[4];
  const auto load = [&](uint32_t row) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const uint32_t col = (c * T + lane) * kRun;
      if constexpr (BEFORE) {
        wr[c] = fetch<S>(g.r, row, col, cols);
        wn[c] = fetch<D>(g.dn, row, col, cols);
      }
      if constexpr (STREAM) wd[c] = fetch<S>(g.dr, row, col, cols);
      if constexpr (BLOCK) wb[c] = fetch<B>(g.block, row, col, cols);
      if constexpr (OWN) wg[c] = load_run_of<kTensor>(g.gate, row, (int)col, g.cols, true);
    }
    if constexpr (BEFORE) {
      stats[0] = of_row(means2, row);
      stats[1] = of_row(g.before.rstd, row);
    }
    if constexpr (AFTER) {
      stats[2] = of_row(means1, row);
      stats[3] = of_row(g.after.rstd, row);
    }
  };
  for (uint32_t which = from; which < last; ++which) {
    const uint32_t first = which * g.rows_per_gate + chunk * g.chunk_rows, end = min(first + g.chunk_rows, (which + 1) * g.rows_per_gate);
    uint32_t row = first + mine;
    if (kAhead && row < end) load(row);
    if (kWhere != kCache && which == from) {   // with the first row on its way
      if constexpr (AFTER) {
        place_param<T, CH, kWhere>(g.after.gamma, g.after.param_type, lane, cols, 1.0f, gamma1, params);
        place_param<T, CH, kWhere>(g.after.beta, g.after.param_type, lane, cols, 0.0f, beta1, params + kPlaces);
      }
      if constexpr (BEFORE) place_param<T, CH, kWhere>(g.before.gamma, g.before.param_type, lane, cols, 1.0f, gamma2, params + 2 * kPlaces);
    }
    if constexpr (GATE && kWhere != kCache && !OWN) place_param<T, CH, kWhere>(g.gates ? row_at(g.gate, which) : nullptr, g.gate.type, lane, cols, 1.0f, gate, params + 3 * kPlaces);
    for (; row < end; row += kRows) {   // groups of lanes that end earlier share no barrier
      if (!kAhead) load(row);
      Runs<CH> h, d;
      Raw cr[CH], cn[CH], cd[CH], cb[CH], cg[CH];
      const float mean2 = BEFORE ? stats[0] * layer2 : 0.0f, rstd2 = BEFORE ? stats[1] : 1.0f, mean1 = AFTER ? stats[2] * layer1 : 0.0f, rstd1 = AFTER ? stats[3] : 1.0f;
      float m[2] = {0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if constexpr (BEFORE) {
          cr[c] = wr[c];
          cn[c] = wn[c];
        }
        if constexpr (STREAM) cd[c] = wd[c];
        if constexpr (BLOCK) cb[c] = wb[c];
        if constexpr (OWN) cg[c] = wg[c];
      }
      if (kAhead) load(min(row + kRows, end - 1));   // behind the last row it once more
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const uint32_t col = (c * T + lane) * kRun;
        if (col < cols && col + kRun > cols) {
          if constexpr (BEFORE) {
            settle_run<S>(cr[c], col, cols);
            settle_run<D>(cn[c], col, cols);
          }
          if constexpr (STREAM) settle_run<S>(cd[c], col, cols);
          if constexpr (BLOCK) settle_run<B>(cb[c], col, cols);
        }
        if (BEFORE && col < cols) {
          values_fetched<S>(g.r, cr[c], h[c]);
          values_fetched<D>(g.dn, cn[c], d[c]);
          float ga[kRun];   // where the row has ended h meets zeros
          before_run(h[c], d[c], mean2, rstd2, param_at<kWhere>(gamma2[c], params + 2 * kPlaces, g.before.gamma, g.before.param_type, (int)col, g.cols, 1.0f, ga), sg2[c], sb2[c], m);
        }
      }
      if constexpr (BEFORE) sums(m);
      const float a2 = m[0] * part2, b2 = m[1] * part;
      m[0] = m[1] = 0.0f;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const uint32_t col = (c * T + lane) * kRun;
        if (col < cols) {
          float v[kRun];
          if constexpr (BEFORE) norm_gradient(d[c], h[c], rstd2, a2, b2);
          if constexpr (STREAM) values_fetched<S>(g.dr, cd[c], v);
          if constexpr (BEFORE && STREAM) add_run(d[c], v);
          if constexpr (!BEFORE) {
#pragma unroll
            for (int i = 0; i < kRun; ++i) d[c][i] = v[i];
          }
          if (g.dx.data) {
#pragma unroll
            for (int i = 0; i < kRun; ++i) v[i] = g.scale * d[c][i];
            put<S>(g.dx, row, col, cols, v);
          }
          if constexpr (GATE && !BLOCK) {
            float of[kRun];
            const float(&by)[kRun] = param_at<kWhere>(gate[c], params + 3 * kPlaces, g.gates ? row_at(g.gate, which) : nullptr, g.gate.type, (int)col, g.cols, 1.0f, of);
#pragma unroll
            for (int i = 0; i < kRun; ++i) d[c][i] *= by[i];
          }
          if constexpr (BLOCK) {
            if (col + kRun > cols) {
#pragma unroll
              for (uint32_t i = 0; i < kRun; ++i) d[c][i] = col + i < cols ? d[c][i] : 0.0f;
            }
            values_fetched<B>(g.block, cb[c], h[c]);
            float ga[kRun], be[kRun], of[kRun];
            if constexpr (OWN) values_of_run<kTensor>(g.gate, cg[c], (int)col, g.cols, true, of);
            gate_run<AFTER>(h[c], d[c], v, mean1, rstd1, param_at<AFTER ? kWhere : kRegisters>(gamma1[c], params, g.after.gamma, g.after.param_type, (int)col, g.cols, 1.0f, ga),
                                      param_at<AFTER ? kWhere : kRegisters>(beta1[c], params + kPlaces, g.after.beta, g.after.param_type, (int)col, g.cols, 0.0f, be),
                                      OWN ? of : param_at<kWhere>(gate[c], params + 3 * kPlaces, g.gates ? row_at(g.gate, which) : nullptr, g.gate.type, (int)col, g.cols, 1.0f, of), sg1[c], sb1[c], m);
            if constexpr (!OWN) add_run(sgate[c], v);
            else if (g.want_gate) put<MOC_F32>(Mat{reinterpret_cast<char*>(g.gate_sums), nullptr, cols * 4, 0, MOC_F32}, row, col, cols, v);
          }
        }
      }
      if constexpr (AFTER) sums(m);
      const float a1 = m[0] * part1, b1 = m[1] * part;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const uint32_t col = (c * T + lane) * kRun;
        if (col < cols) {
          if constexpr (AFTER) norm_gradient(d[c], h[c], rstd1, a1, b1);
          put<D>(g.dblock, row, col, cols, d[c]);
        }
      }
    }
    if (BLOCK && !OWN && g.want_gate) {
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

// T and CH by the columns alone: moc_residual_backward_work does not know the rest.
template <int S, int B, int D, int MODE, bool OWN>
ResidualShape backward_shape(int64_t cols) {
  if (cols <= 512) return {residual_backward_kernel<S, B, D, 64, 1, MODE, OWN>, 256, 4};
  if (cols <= 1024) return {residual_backward_kernel<S, B, D, 64, 2, MODE, OWN>, 256, 4};
  if (cols <= 2048) return {residual_backward_kernel<S, B, D, 256, 1, MODE, OWN>, 256, 1};
  if (cols <= 4096) return {residual_backward_kernel<S, B, D, 512, 1, MODE, OWN>, 512, 1};
  if (cols <= 8192) return {residual_backward_kernel<S, B, D, 512, 2, MODE, OWN>, 512, 1};
  return {residual_backward_kernel<S, B, D, 1024, 2, MODE, OWN>, 1024, 1};
}
template <int S, int B, int D>
ResidualShape backward_shape(int mode, bool own, int64_t cols) {
  switch (mode) {
    case kBefore: return backward_shape<S, D, D, kBefore, false>(cols);
    case kBefore | kStream: return backward_shape<S, D, D, kBefore | kStream, false>(cols);
    case kBefore | kStream | kBlock: return own ? backward_shape<S, B, D, kBefore | kStream | kBlock, true>(cols) : backward_shape<S, B, D, kBefore | kStream | kBlock, false>(cols);
    case kBefore | kStream | kBlock | kAfter:
      return own ? backward_shape<S, B, D, kBefore | kStream | kBlock | kAfter, true>(cols) : backward_shape<S, B, D, kBefore | kStream | kBlock | kAfter, false>(cols);
  }
  if (own) return {};
  switch (mode) {
    case kBefore | kBlock: return backward_shape<S, B, D, kBefore | kBlock, false>(cols);
    case kBefore | kBlock | kAfter: return backward_shape<S, B, D, kBefore | kBlock | kAfter, false>(cols);
    case kStream | kGate: return backward_shape<S, D, D, kStream | kGate, false>(cols);
    case kBefore | kStream | kGate: return backward_shape<S, D, D, kBefore | kStream | kGate, false>(cols);
    case kStream | kBlock: return backward_shape<S, B, D, kStream | kBlock, false>(cols);
    case kStream | kBlock | kAfter: return backward_shape<S, B, D, kStream | kBlock | kAfter, false>(cols);
  }
  return {};
}
template <int D>
ResidualShape backward_shape_of(int s, int b, int mode, bool own, int64_t cols) {
  if (s == D && b == D) return backward_shape<D, D, D>(mode, own, cols);
  if (s == D && b == kKept) return backward_shape<D, kKept, D>(mode, own, cols);
  if constexpr (D != MOC_F32) {
    if (s == MOC_F32 && b == D) return backward_shape<MOC_F32, D, D>(mode, own, cols);
    if (s == MOC_F32 && b == kKept) return backward_shape<MOC_F32, kKept, D>(mode, own, cols);
  }
  return {};
}

}  // namespace
