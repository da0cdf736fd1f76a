// Activation checkpoints in 8 bits: written, and read back (through an activation).
//
// Both are one pass over the data and bound by memory: 2 + 1.03 bytes a value of 16 bits one way.  A
// thread takes eight values of a row (kRun), a quad of lanes a block of 32, whose largest magnitude
// goes round by two lane permutations; nothing is staged.  16384 x 4096 bf16: written in 39 us (5.2 TB/s), read
// back in 30 (6.7, what was written last being in cache); 8192 x 16384 through gelu 68 us, 5.9 TB/s.
#include "moc_training.h"

namespace {

constexpr int kThreads = 256, kTurns = 4, kAtOnce = kThreads * kTurns;

struct CheckpointArgs {
  void* values;          // [rows][stride]
  uint8_t *codes, *scales;
  int64_t rows, stride, code_stride, scale_stride;
  int64_t cols;
  int64_t runs;          // runs of eight in a row, a multiple of four
  int group;             // rows of a workgroup
  int act;
  float most;
};

// Where a thread is.  FLAT: a matrix without gaps, of whole blocks, is one row of any length, and a
// workgroup has kAtOnce runs of it.  Otherwise a workgroup has `group` rows, laid end to end so that
// narrow ones fill its waves too; quads never straddle rows (runs % 4 == 0).  All lanes of a quad make
// the same number of turns.
struct Place {
  int64_t row, col;
};
template <bool FLAT>
__device__ __forceinline__ Place place(const CheckpointArgs& g, uint32_t i) {
  if constexpr (FLAT) return Place{0, (block_of() * kAtOnce + i) * kRun};
  const uint32_t row = i / (uint32_t)g.runs;
  return Place{block_of() * g.group + row, (int64_t)(i - row * (uint32_t)g.runs) * kRun};
}

// fetch(turn, place) and use(turn, place) for the runs of a thread.  Of a flat matrix four are fetched
// before the first is used, without a branch (134 M values read back: 115 us one at a time, 72 so).
template <bool FLAT, class Fetch, class Use>
__device__ __forceinline__ void go_over(const CheckpointArgs& g, const Fetch& fetch, const Use& use) {
  if constexpr (FLAT) {
    const int64_t left = g.runs - block_of() * kAtOnce;
    if (left >= kAtOnce) {
#pragma unroll
      for (int t = 0; t < kTurns; ++t) fetch(t, place<true>(g, threadIdx.x + t * kThreads));
#pragma unroll
      for (int t = 0; t < kTurns; ++t) use(t, place<true>(g, threadIdx.x + t * kThreads));
      return;
    }
#pragma unroll 1
    for (uint32_t i = threadIdx.x; (int64_t)i < left; i += kThreads) {
      fetch(0, place<true>(g, i));
      use(0, place<true>(g, i));
    }
  } else {
    const int64_t left = g.rows - block_of() * g.group, rows = left < g.group ? left : g.group;
    const uint32_t total = rows > 0 ? (uint32_t)rows * (uint32_t)g.runs : 0;
    for (uint32_t i = threadIdx.x; i < total; i += kThreads) {
      const Place at = place<false>(g, i);
      fetch(0, at);
      use(0, at);
    }
  }
}

template <bool FLAT>
__device__ __forceinline__ int values_there(const CheckpointArgs& g, const Place& at) {
  if constexpr (FLAT) return kRun;
  const int64_t n = g.cols - at.col;
  return n < kRun ? (int)n : kRun;
}

template <int TYPE, int FMT, bool FLAT>
__global__ __launch_bounds__(kThreads) void checkpoint_write_kernel(CheckpointArgs g) {
  using T = typename Stored<TYPE>::type;
  Raw w[kTurns];
  go_over<FLAT>(
      g,
      [&](int t, const Place& at) { w[t] = load_raw<TYPE>(static_cast<const T*>(g.values) + at.row * g.stride + at.col, nullptr, 0, values_there<FLAT>(g, at)); },
      [&](int t, const Place& at) {
        float v[kRun];
        values_of<TYPE>(w[t], v);
        keep_run<FMT>(v, at.col, values_there<FLAT>(g, at), g.most, g.codes + at.row * g.code_stride, g.scales + at.row * g.scale_stride);
      });
}

template <int TYPE, int FMT, bool FLAT>
__global__ __launch_bounds__(kThreads) void checkpoint_read_kernel(CheckpointArgs g) {
  Raw w[kTurns];
  go_over<FLAT>(
      g,
      [&](int t, const Place& at) {
        const uint2 c = load_codes(g.codes + at.row * g.code_stride + at.col, values_there<FLAT>(g, at));
        w[t].a[0] = c.x;
        w[t].a[1] = c.y;
        w[t].scale = g.scales[at.row * g.scale_stride + at.col / MOC_BLOCK];
      },
      [&](int t, const Place& at) {
        const int n = values_there<FLAT>(g, at);
        if (n <= 0) return;
        float v[kRun];
        values_of<FMT>(w[t], v);
        act_run(g.act, v);
        store_run<TYPE>(static_cast<typename Stored<TYPE>::type*>(g.values) + at.row * g.stride, at.col, n, v);
      });
}

using CheckpointKernel = void (*)(CheckpointArgs);
template <int TYPE, int FMT>
CheckpointKernel pick(bool write, bool flat) {
  if (write) return flat ? checkpoint_write_kernel<TYPE, FMT, true> : checkpoint_write_kernel<TYPE, FMT, false>;
  return flat ? checkpoint_read_kernel<TYPE, FMT, true> : checkpoint_read_kernel<TYPE, FMT, false>;
}
template <int FMT>
CheckpointKernel pick(bool write, bool flat, int type) {
  return type == MOC_BF16 ? pick<MOC_BF16, FMT>(write, flat) : type == MOC_F16 ? pick<MOC_F16, FMT>(write, flat) : pick<MOC_F32, FMT>(write, flat);
}

int queue(bool write, int64_t rows, int64_t cols, const moc_matrix* values, const moc_matrix* kept, int act, void* stream) {
  CheckpointArgs g = {};
  g.values = values->data;
  g.codes = static_cast<uint8_t*>(kept->data);
  g.scales = kept->scales;
  g.rows = rows;
  g.stride = values->stride;
  g.code_stride = kept->stride;
  g.scale_stride = kept->scale_stride;
  g.cols = cols;
  g.act = act;
  g.most = most_kept(kept->type, values->type);
  // Without gaps and with whole blocks, all rows are one: no places to work out.
  const bool flat = values->stride == cols && kept->stride == cols && cols % MOC_BLOCK == 0 && kept->scale_stride == cols / MOC_BLOCK;
  if (flat) {
    g.cols = rows * cols;
    g.rows = 1;
  }
  g.runs = (g.cols + MOC_BLOCK - 1) / MOC_BLOCK * (MOC_BLOCK / kRun);
  const int64_t group = kAtOnce / g.runs;
  g.group = (int)(group < 1 ? 1 : group);
  const int64_t blocks = flat ? (g.runs + kAtOnce - 1) / kAtOnce : (rows + g.group - 1) / g.group;
  const CheckpointKernel kern = kept->type == MOC_E4M3 ? pick<MOC_E4M3>(write, flat, values->type) : pick<MOC_I8>(write, flat, values->type);
  hipLaunchKernelGGL(kern, grid_of(blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream), g);
  MOC_HIP(hipGetLastError());
  return MOC_OK;
}

}  // namespace

int moc_compute_units(int* out) {
  static std::atomic<int> known[64];
  int dev = -1;
  MOC_HIP(hipGetDevice(&dev));
  const bool kept = dev >= 0 && dev < 64;
  int n = kept ? known[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    MOC_HIP(hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev));
    if (kept) known[dev].store(n, std::memory_order_relaxed);
  }
  *out = n;
  return MOC_OK;
}

extern "C" {

int moc_training_version(void) { return MOC_TRAINING_VERSION; }

int moc_checkpoint_write(int64_t rows, int64_t cols, const moc_matrix* x, const moc_matrix* kept, void* hip_stream) {
  if (!sizes_ok(rows, cols) || !matrix_ok(x, rows, cols, true, false) || !matrix_ok(kept, rows, cols, false, true)) return MOC_EINVAL;
  if (rows == 0 || cols == 0) return MOC_OK;
  return queue(true, rows, cols, x, kept, MOC_ACT_NONE, hip_stream);
}

int moc_checkpoint_read(int64_t rows, int64_t cols, const moc_matrix* kept, int32_t act, const moc_matrix* out, void* hip_stream) {
  if (!sizes_ok(rows, cols) || act < MOC_ACT_NONE || act > MOC_ACT_SILU) return MOC_EINVAL;
  if (!matrix_ok(kept, rows, cols, false, true) || !matrix_ok(out, rows, cols, true, false)) return MOC_EINVAL;
  if (rows == 0 || cols == 0) return MOC_OK;
  return queue(false, rows, cols, out, kept, act, hip_stream);
}

}  // extern "C"
