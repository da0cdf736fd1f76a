// Shared by the kernels that hold a row in the registers of a group of threads: sums over such a row, parameters by
// column.
#pragma once

#include "moc_training.h"

namespace {

// The sum over the wave, in all lanes: inside rows of 16 by shifts of the vector ALU, then across them.
template <int CTRL, int ROWS>
__device__ __forceinline__ float add_shifted(float a) {
  return a + bits_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)float_bits(a), CTRL, ROWS, 0xF, true));
}
__device__ __forceinline__ float wave_sum(float a) {
  a = add_shifted<0x111, 0xF>(a);   // row_shr:1, 2, 4, 8
  a = add_shifted<0x112, 0xF>(a);
  a = add_shifted<0x114, 0xF>(a);
  a = add_shifted<0x118, 0xF>(a);
  a = add_shifted<0x142, 0xA>(a);   // row_bcast:15 into rows 1 and 3, :31 into rows 2 and 3
  a = add_shifted<0x143, 0xC>(a);
  return bits_float((uint32_t)__builtin_amdgcn_readlane((int)float_bits(a), kWave - 1));
}

// The sum over the first W lanes, a power of two up to 16, in all lanes.
template <int W>
__device__ __forceinline__ float first_sum(float a) {
  if constexpr (W > 1) a = add_shifted<0x111, 0xF>(a);
  if constexpr (W > 2) a = add_shifted<0x112, 0xF>(a);
  if constexpr (W > 4) a = add_shifted<0x114, 0xF>(a);
  if constexpr (W > 8) a = add_shifted<0x118, 0xF>(a);
  return bits_float((uint32_t)__builtin_amdgcn_readlane((int)float_bits(a), W - 1));
}

// Sums over the T threads that share a row, N of them at a time, in all of the threads.  `room`: two
// halves of N x T / 64 floats, used in turn, so that one barrier does: what was written two sums ago
// has been read when all waves have come to the sums in between.  Called by whole workgroups where T > 64.
template <int T, int N>
struct RowSums {
  static constexpr int kWaves = T / kWave, kRoom = 2 * N * kWaves;
  float* room;
  int half = 0;
  __device__ __forceinline__ void operator()(float (&a)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = wave_sum(a[i]);
    if constexpr (T > kWave) {
      float* const mine = room + half * N * kWaves;
      const int lane = threadIdx.x % kWave;
      if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) mine[i * kWaves + (threadIdx.x % T) / kWave] = a[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) a[i] = first_sum<kWaves>(mine[i * kWaves + lane % kWaves]);
      half ^= 1;
    }
  }
};

__device__ __forceinline__ void load_param(const void* p, int type, int col, int n, float other, float (&v)[kRun]) {
  if (p) {
    load_any(type, p, col, n, v);
  } else {
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = other;
  }
}

// 1 / sqrt(x), subnormal arguments too: the hardware's, 1 ulp off, and a step of Newton's method, which leaves
// little but the last rounding (an error of rstd moves a whole row's values, and codes of its checkpoint with them).
__device__ __forceinline__ float inverse_root(float x) {
  const bool small = x < 0x1p-100f;
  const float a = small ? x * 0x1p64f : x, r = __builtin_amdgcn_rsqf(a);
  const float better = __builtin_fmaf(0.5f * r, __builtin_fmaf(-a * r, r, 1.0f), r), root = r > 0.0f && r < kInf ? better : r;
  return small ? root * 0x1p32f : root;
}

}  // namespace
