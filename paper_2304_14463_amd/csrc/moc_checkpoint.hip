// Activation checkpoints in 8 bits: written, and read back (through an activation).
//
// Both are one pass over the data and bound by memory: 2 + 1.03 bytes a value of 16 bits one way.  A
// thread takes eight values of a row (kRun), a quad of lanes a block of 32, whose largest magnitude
// goes round by two lane permutations; nothing is staged.
#include "moc_training.h"

namespace {

constexpr int kThreads = 256;

struct CheckpointArgs {
  void* values;          // [rows][stride]
  uint8_t *codes, *scales;
  int64_t rows, stride, code_stride, scale_stride;
  int cols, runs;        // runs of eight in a row, a multiple of four
  int group;             // rows of a workgroup
  int act;
  float most;
};

// A workgroup has `group` rows, laid end to end so that narrow ones fill its waves too.  Quads never
// straddle rows (runs % 4 == 0), and all lanes of one make the same number of turns.
struct Place {
  int64_t row;
  int col;
};
__device__ __forceinline__ Place place(uint32_t i, const CheckpointArgs& g) {
  const uint32_t row = i / (uint32_t)g.runs;
  return Place{block_of() * g.group + row, (int)(i - row * (uint32_t)g.runs) * kRun};
}
__device__ __forceinline__ uint32_t runs_of_group(const CheckpointArgs& g) {
  const int64_t left = g.rows - block_of() * g.group;
  return left <= 0 ? 0 : (uint32_t)(left < g.group ? (int)left : g.group) * (uint32_t)g.runs;
}

template <int TYPE, int FMT>
__global__ __launch_bounds__(kThreads) void checkpoint_write_kernel(CheckpointArgs g) {
  const uint32_t total = runs_of_group(g);
  for (uint32_t i = threadIdx.x; i < total; i += kThreads) {
    const Place at = place(i, g);
    const int n = g.cols - at.col;
    float v[kRun];
    load_run<TYPE>(static_cast<const typename Stored<TYPE>::type*>(g.values) + at.row * g.stride, at.col, n, v);
    keep_run<FMT>(v, at.col, n, g.most, g.codes + at.row * g.code_stride, g.scales + at.row * g.scale_stride);
  }
}

template <int TYPE, int FMT>
__global__ __launch_bounds__(kThreads) void checkpoint_read_kernel(CheckpointArgs g) {
  const uint32_t total = runs_of_group(g);
  for (uint32_t i = threadIdx.x; i < total; i += kThreads) {
    const Place at = place(i, g);
    const int n = g.cols - at.col;
    if (n <= 0) continue;
    float v[kRun];
    load_held<FMT>(g.codes + at.row * g.code_stride, g.scales + at.row * g.scale_stride, at.col, n, v);
    act_run(g.act, v);
    store_run<TYPE>(static_cast<typename Stored<TYPE>::type*>(g.values) + at.row * g.stride, at.col, n, v);
  }
}

using CheckpointKernel = void (*)(CheckpointArgs);
template <template <int, int> class K>
CheckpointKernel pick(int type, int fmt) {
  if (fmt == MOC_E4M3) return type == MOC_BF16 ? K<MOC_BF16, MOC_E4M3>::kernel() : type == MOC_F16 ? K<MOC_F16, MOC_E4M3>::kernel() : K<MOC_F32, MOC_E4M3>::kernel();
  return type == MOC_BF16 ? K<MOC_BF16, MOC_I8>::kernel() : type == MOC_F16 ? K<MOC_F16, MOC_I8>::kernel() : K<MOC_F32, MOC_I8>::kernel();
}
template <int TYPE, int FMT> struct Write { static CheckpointKernel kernel() { return checkpoint_write_kernel<TYPE, FMT>; } };
template <int TYPE, int FMT> struct Read { static CheckpointKernel kernel() { return checkpoint_read_kernel<TYPE, FMT>; } };

int queue(CheckpointKernel kern, int64_t rows, int64_t cols, const moc_matrix* values, const moc_matrix* kept, int act, void* stream) {
  CheckpointArgs g = {};
  g.values = values->data;
  g.codes = static_cast<uint8_t*>(kept->data);
  g.scales = kept->scales;
  g.rows = rows;
  g.stride = values->stride;
  g.code_stride = kept->stride;
  g.scale_stride = kept->scale_stride;
  g.cols = (int)cols;
  g.runs = (int)((cols + MOC_BLOCK - 1) / MOC_BLOCK) * (MOC_BLOCK / kRun);
  g.act = act;
  g.most = most_kept(kept->type, values->type);
  // Four turns a workgroup where there is enough to fill the card with that, fewer below.
  int64_t turns = rows * g.runs / (kThreads * 2048);
  turns = turns < 1 ? 1 : turns > 4 ? 4 : turns;
  const int64_t group = turns * kThreads / g.runs;
  g.group = (int)(group < 1 ? 1 : group);
  hipLaunchKernelGGL(kern, grid_of((rows + g.group - 1) / g.group), dim3(kThreads), 0, static_cast<hipStream_t>(stream), g);
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
  return queue(pick<Write>(x->type, kept->type), rows, cols, x, kept, MOC_ACT_NONE, hip_stream);
}

int moc_checkpoint_read(int64_t rows, int64_t cols, const moc_matrix* kept, int32_t act, const moc_matrix* out, void* hip_stream) {
  if (!sizes_ok(rows, cols) || act < MOC_ACT_NONE || act > MOC_ACT_SILU) return MOC_EINVAL;
  if (!matrix_ok(kept, rows, cols, false, true) || !matrix_ok(out, rows, cols, true, false)) return MOC_EINVAL;
  if (rows == 0 || cols == 0) return MOC_OK;
  return queue(pick<Read>(out->type, kept->type), rows, cols, out, kept, act, hip_stream);
}

}  // extern "C"
