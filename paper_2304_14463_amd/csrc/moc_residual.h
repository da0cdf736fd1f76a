// Shared by the two passes of the residual connection: what a block has computed goes through a norm and a gate, is added to the scaled stream, and the
// norm before the next block is taken of the sum, in one pass; and the gradients of all of it.
//
// Bound by memory: every value is read once and written once, 8 bytes of the forward and 12 of the backward pass where all are
// 16 bits wide.  T threads take a row and hold it in registers, CH runs of eight values each, as in moc_norm.hip: a wave a row up
// to 1024 columns, then 256, 512 and 1024 threads.  Parameters stay in registers over a workgroup's rows, and in the backward
// pass so do their gradients' sums, which a second kernel adds over workgroups, in their order; the next row is on its
// way meanwhile.  Kernels are made for types: with types asked at every run, code and scalar registers grew until those spilled
// (4998 x 1247 backward from int8 94 us, 36 so; 8192 x 8192 bf16 with a gate alone 274 and 115, float32 647 and 334).  bf16, both norms and a gate: 32768 x 4096 forward 206 us (5.2 TB/s), backward
// 319 (5.1); a copy of 1 GiB reaches 5.0.  Of 8193 to 16384 columns the backward pass with both norms spills half a kilobyte a lane
// (8192 x 16384: 866 us, 1.9 TB/s); without the norm behind the block it is 283 us, 4.8 TB/s.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "moc_rows.h"

struct ResidualMat {
  char* data;
  uint8_t* scales;
  uint32_t step, scale_step;   // bytes from one row to the next
  int type;
};
struct ResidualNorm {
  const void *gamma, *beta;
  int param_type;
  float eps;
  bool on, layer;
  float *mean, *rstd;
};
struct ResidualArgs {
  ResidualMat x, block, gate, r, n, kept;
  ResidualMat dr, dn, dx, dblock;
  ResidualNorm after, before;
  uint32_t rows;      // forward
  uint32_t gates, rows_per_gate;
  int cols;
  float scale, most;
  bool parts;         // runs at a row's end are loaded value by value: an output lies over an input
  // backward
  float* sums;        // [workgroups][kinds][cols]
  float* gate_sums;   // [gates][chunks][cols]; with one chunk the result itself
  int kinds;          // of sums: bits of kBeforeGamma ..
  bool want_gate, own_gates;   // own: a gate for every row
  uint32_t chunks, chunk_rows, groups;   // workgroups of a gate's rows, and their rows; or gates of a workgroup
};

namespace {

constexpr int kMaxThreads = 1024;

using Mat = ResidualMat;
using RowNorm = ResidualNorm;

constexpr int kBeforeGamma = 1, kBeforeBeta = 2, kAfterGamma = 4, kAfterBeta = 8;

__device__ __forceinline__ char* row_at(const Mat& m, uint32_t row) { return m.data + (uint64_t)row * m.step; }

// What a kernel is made for a matrix to hold, beside one type of values: a checkpoint of either format, values of any type, or
// anything, which is then asked at every run.
constexpr int kKept = -1, kTensor = -2, kAny = -3;
constexpr bool is_half(int k) { return k == MOC_BF16 || k == MOC_F16; }

// A run of a row on its way; `whole`: of a row of eight columns at least (see load_raw_whole).
template <int K>
__device__ __forceinline__ Raw load_run_of(const Mat& m, uint32_t row, int col, int cols, bool whole) {
  const void* const at = row_at(m, row);
  if constexpr (is_half(K)) {
    return whole ? load_raw_whole<MOC_BF16>(at, nullptr, col, cols) : load_raw<MOC_BF16>(at, nullptr, col, cols - col);
  } else if constexpr (K == MOC_F32) {
    return whole ? load_raw_whole<MOC_F32>(at, nullptr, col, cols) : load_raw<MOC_F32>(at, nullptr, col, cols - col);
  } else if constexpr (K == kKept) {
    const uint8_t* const scales = m.scales + (uint64_t)row * m.scale_step;
    return whole ? load_raw_whole<MOC_E4M3>(at, scales, col, cols) : load_raw<MOC_E4M3>(at, scales, col, cols - col);
  } else {
    if (m.type == MOC_BF16 || m.type == MOC_F16) return load_run_of<MOC_BF16>(m, row, col, cols, whole);
    if (K == kTensor || m.type == MOC_F32) return load_run_of<MOC_F32>(m, row, col, cols, whole);
    return load_run_of<kKept>(m, row, col, cols, whole);
  }
}
// Its values, 0 beyond the row.
template <int K>
__device__ __forceinline__ void values_of_run(const Mat& m, Raw w, int col, int cols, bool whole, float (&v)[kRun]) {
  if constexpr (K == kTensor || K == kAny) {
    if (m.type == MOC_BF16) values_of_run<MOC_BF16>(m, w, col, cols, whole, v);
    else if (m.type == MOC_F16) values_of_run<MOC_F16>(m, w, col, cols, whole, v);
    else if (K == kTensor || m.type == MOC_F32) values_of_run<MOC_F32>(m, w, col, cols, whole, v);
    else values_of_run<kKept>(m, w, col, cols, whole, v);
    return;
  } else {
    const int n = cols - col;
    if (n < kRun && whole) settle<K == kKept ? MOC_E4M3 : K>(w, col, cols);
    if constexpr (K == kKept) {
      if (m.type == MOC_E4M3) values_of<MOC_E4M3>(w, v);
      else values_of<MOC_I8>(w, v);
    } else {
      values_of<K>(w, v);
    }
    if (n < kRun) {
#pragma unroll
      for (int i = 0; i < kRun; ++i) v[i] = i < n ? v[i] : 0.0f;
    }
  }
}

// Rounded to 32 bits before it is rounded to 16: the compiler makes one instruction of a product, a sum and a conversion to
// float16, with one rounding, where it sees all three.
__device__ __forceinline__ void rounded(const float (&v)[kRun], float (&w)[kRun]) {
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    w[i] = v[i];
    asm("" : "+v"(w[i]));
  }
}

// The same in kernels made for a type, of rows of eight columns at least: always from within the row, without a branch, so that
// the waits for it are for nothing else.  Lanes beyond the row have its last eight values.
template <int K>
__device__ __forceinline__ Raw fetch(const Mat& m, uint32_t row, uint32_t col, uint32_t cols) {
  constexpr uint32_t kBytes = K == MOC_F32 ? 4 : K == kKept ? 1 : 2;
  const char* const at = row_at(m, row);
  const uint32_t place = min(col, cols - kRun) * kBytes;
  Raw x = {};
  if constexpr (K == kKept) {
    uint2 c;
    __builtin_memcpy(&c, at + place, 8);
    x.a[0] = c.x;
    x.a[1] = c.y;
    x.scale = (m.scales + (uint64_t)row * m.scale_step)[min(col, cols - 1) / MOC_BLOCK];
  } else {
    __builtin_memcpy(&x.a, at + place, 16);
    if constexpr (K == MOC_F32) __builtin_memcpy(&x.b, at + place + 16, 16);
  }
  return x;
}
// A row's last run, where it is none of eight: moved down, zeros behind it.
template <int K>
__device__ __forceinline__ void settle_run(Raw& w, uint32_t col, uint32_t cols) { settle<K == kKept ? MOC_E4M3 : K>(w, (int)col, (int)cols); }
template <int K>
__device__ __forceinline__ void values_fetched(const Mat& m, const Raw& w, float (&v)[kRun]) {
  if constexpr (K == kKept) {
    if (m.type == MOC_E4M3) values_of<MOC_E4M3>(w, v);
    else values_of<MOC_I8>(w, v);
  } else {
    values_of<K>(w, v);
  }
}
// The first n < 8 of eight values: four, two and one of them, as n has them.
template <class T>
__device__ __forceinline__ void put_part(char* at, const T (&t)[kRun], uint32_t n) {
  constexpr int kWords = sizeof(T) * kRun / 4, kFour = kWords / 2;
  uint32_t w[kWords];
  __builtin_memcpy(w, t, sizeof w);
  if (n & 4) {
    __builtin_memcpy(at, w, kFour * 4);
    at += kFour * 4;
#pragma unroll
    for (int i = 0; i < kFour; ++i) w[i] = w[kFour + i];
  }
  if (n & 2) {
    __builtin_memcpy(at, w, kFour * 2);
    at += kFour * 2;
#pragma unroll
    for (int i = 0; i < kFour / 2; ++i) w[i] = w[kFour / 2 + i];
  }
  if (n & 1) __builtin_memcpy(at, w, sizeof(T));
}
template <int K>
__device__ __forceinline__ void put(const Mat& m, uint32_t row, uint32_t col, uint32_t cols, const float (&of)[kRun]) {
  using T = typename Stored<K>::type;
  float v[kRun];
  rounded(of, v);
  char* const at = row_at(m, row) + col * (uint32_t)sizeof(T);
  T t[kRun];
#pragma unroll
  for (int i = 0; i < kRun; ++i) t[i] = (T)v[i];
  if (col + kRun <= cols) {
    __builtin_memcpy(at, t, sizeof t);
  } else {
    put_part(at, t, cols - col);
  }
}

template <int K>
__device__ __forceinline__ void store_run_of(const Mat& m, uint32_t row, int col, int n, const float (&of)[kRun]) {
  if (n <= 0) return;
  if constexpr (K >= 0) {
    put<K>(m, row, (uint32_t)col, (uint32_t)(col + n), of);
  } else {
    float v[kRun];
    rounded(of, v);
    store_any(m.type, row_at(m, row), col, n, v);
  }
}

// To the compiler, another number in each row: what a ragged row's end is asked is not kept over rows in scalar registers.
__device__ __forceinline__ int asked_again(int n) {
  asm volatile("" : "+v"(n));
  return n;
}

template <int CH>
using Runs = float[CH][kRun];

// Parameters by column, `other` where there are none.  A ragged row's last ones are loaded whole, too: in parts each of them
// would be waited for.
template <int T, int CH>
__device__ __forceinline__ void hold_param(const void* p, int type, int lane, int cols, float other, Runs<CH>& v) {
  const Mat m{static_cast<char*>(const_cast<void*>(p)), nullptr, 0, 0, type};
  const bool whole = cols >= kRun;
  if (p) {
    Raw w[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c] = load_run_of<kTensor>(m, 0, (c * T + lane) * kRun, cols, whole);
#pragma unroll
    for (int c = 0; c < CH; ++c) values_of_run<kTensor>(m, w[c], (c * T + lane) * kRun, cols, whole, v[c]);
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < kRun; ++i) v[c][i] = other;
  }
}
// 1 where there is no gate.
template <int T, int CH>
__device__ __forceinline__ void hold_gate(const ResidualArgs& g, uint32_t gate, int lane, Runs<CH>& v) {
  hold_param<T, CH>(g.gates ? row_at(g.gate, gate) : nullptr, g.gate.type, lane, g.cols, 1.0f, v);
}

// A row's number, which all lanes share, through the scalar cache: it is not waited for with the rows.
__device__ __forceinline__ float of_row(const float* p, uint32_t row) {
  using Constant = const float __attribute__((address_space(4)))*;
  return reinterpret_cast<Constant>(reinterpret_cast<uintptr_t>(p))[row];
}

// A parameter's run: as it is held, or read again from cache in kernels that have no registers for it.
template <bool HOLD>
__device__ __forceinline__ const float (&param_of(const float (&held)[kRun], const void* p, int type, int col, int cols, float other, float (&room)[kRun]))[kRun] {
  if constexpr (HOLD) return held;
  if (p) {
    const Mat m{static_cast<char*>(const_cast<void*>(p)), nullptr, 0, 0, type};
    values_of_run<kTensor>(m, load_run_of<kTensor>(m, 0, col, cols, cols >= kRun), col, cols, cols >= kRun, room);
  } else {
#pragma unroll
    for (int i = 0; i < kRun; ++i) room[i] = other;
  }
  return room;
}

// ---- arithmetic ---------------------------------------------------------------------------------

// Operations as they are written, none of them fused by the compiler: every kernel gives the same bits.
__device__ __forceinline__ float squares(const float (&v)[kRun], float mean, int n, float s) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    const float d = i < n ? v[i] - mean : 0.0f;
    s = __builtin_fmaf(d, d, s);
  }
  return s;
}
__device__ __forceinline__ void normalise(float (&v)[kRun], float mean, float rstd, const float (&gamma)[kRun], const float (&beta)[kRun]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < kRun; ++i) v[i] = __builtin_fmaf((v[i] - mean) * rstd, gamma[i], beta[i]);
}
// h: the stream's run, then normalised; d: n's gradient, then times gamma.
__device__ __forceinline__ void before_run(float (&h)[kRun], float (&d)[kRun], float mean, float rstd, const float (&gamma)[kRun], float (&sg)[kRun], float (&sb)[kRun], float (&m)[2]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    h[i] = (h[i] - mean) * rstd;
    sg[i] = __builtin_fmaf(d[i], h[i], sg[i]);
    sb[i] += d[i];
    d[i] *= gamma[i];
    m[0] += d[i];
    m[1] = __builtin_fmaf(d[i], h[i], m[1]);
  }
}
// A norm's gradient from d times gamma, the normalised h and their means.
__device__ __forceinline__ void norm_gradient(float (&d)[kRun], const float (&h)[kRun], float rstd, float a, float b) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < kRun; ++i) d[i] = rstd * (__builtin_fmaf(-h[i], b, d[i]) - a);
}
// h: the block's run, then normalised; d: the gradient of what the gate is multiplied with, then on its way through it.
template <bool NORMED>
__device__ __forceinline__ void gate_run(float (&h)[kRun], float (&d)[kRun], float (&own)[kRun], float mean, float rstd, const float (&gamma)[kRun], const float (&beta)[kRun], const float (&gate)[kRun],
                                         float (&sg)[kRun], float (&sb)[kRun], float (&m)[2]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    if constexpr (NORMED) {
      h[i] = (h[i] - mean) * rstd;
      own[i] = d[i] * __builtin_fmaf(h[i], gamma[i], beta[i]);
    } else {
      own[i] = d[i] * h[i];
    }
    d[i] *= gate[i];
    if constexpr (NORMED) {
      sg[i] = __builtin_fmaf(d[i], h[i], sg[i]);
      sb[i] += d[i];
      d[i] *= gamma[i];
      m[0] += d[i];
      m[1] = __builtin_fmaf(d[i], h[i], m[1]);
    }
  }
}
__device__ __forceinline__ void add_run(float (&s)[kRun], const float (&v)[kRun]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < kRun; ++i) s[i] += v[i];
}

// ---- host ---------------------------------------------------------------------------------------

inline int kind_of(int type) { return is_value(type) ? type : kKept; }

// What all the matrices that are there hold, kAny where they differ, `otherwise` where there are none.
inline int agreed(std::initializer_list<const moc_matrix*> of, int otherwise) {
  int k = kAny;
  for (const moc_matrix* m : of) {
    if (!m) continue;
    if (k != kAny && k != kind_of(m->type)) return kAny;
    k = kind_of(m->type);
  }
  return k == kAny ? otherwise : k;
}

inline Mat mat_of(const moc_matrix* m) {
  if (!m) return Mat{};
  return Mat{static_cast<char*>(m->data), m->scales, (uint32_t)(m->stride * type_bytes(m->type)), (uint32_t)m->scale_stride, m->type};
}

inline bool residual_sizes_ok(int64_t rows, int64_t cols, int64_t gates) {
  return sizes_ok(rows, cols) && cols >= 1 && cols <= MOC_RESIDUAL_MAX_COLS && gates >= 0 && gates <= std::max<int64_t>(rows, 1) && (gates < 1 || rows % gates == 0);
}
inline bool norm_ok(const moc_row_norm* n, int64_t rows) {
  if (!n || n->kind == MOC_NORM_NONE) return true;
  if (n->reserved != 0 || (n->kind != MOC_NORM_LAYER && n->kind != MOC_NORM_RMS) || !(n->eps >= 0.0f) || !params_ok(n->gamma, n->param_type) || !params_ok(n->beta, n->param_type)) return false;
  if (n->beta && n->kind == MOC_NORM_RMS) return false;
  if (rows == 0) return true;
  return n->rstd && aligned_to(n->rstd, 4) && (n->kind == MOC_NORM_RMS || (n->mean && aligned_to(n->mean, 4)));
}
inline RowNorm row_norm_of(const moc_row_norm* n) {
  RowNorm r = {};
  if (!n || n->kind == MOC_NORM_NONE) return r;
  r.gamma = n->gamma; r.beta = n->beta; r.param_type = n->param_type; r.eps = n->eps;
  r.on = true; r.layer = n->kind == MOC_NORM_LAYER; r.mean = n->mean; r.rstd = n->rstd;
  return r;
}
inline bool lies_over(const moc_matrix* out, std::initializer_list<const moc_matrix*> in) {
  if (!out || !out->data) return false;
  for (const moc_matrix* m : in)
    if (m && m->data == out->data) return true;
  return false;
}

}  // namespace
