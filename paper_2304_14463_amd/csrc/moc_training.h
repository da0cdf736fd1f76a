// Shared by the kernels of include/moccasin_training.h: runs of eight values loaded, stored and
// converted, activations, blocks of a checkpoint, and the checks of descriptors.
#pragma once

#include "moc_internal.h"
#include "moccasin_training.h"

namespace {

using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using f16x2 = _Float16 __attribute__((ext_vector_type(2)));
using f32x2 = float __attribute__((ext_vector_type(2)));

constexpr float kInf = __builtin_inff();
constexpr int kMinExp = -111;   // smallest exponent of a scale

// What a thread takes at a time: eight values next to each other in a row, from a column that is a
// multiple of eight.  16-bit types: 16 bytes, the widest load; four neighbouring lanes hold the 32
// columns that share a scale.  `n` of them exist (all eight where n >= 8).  Addresses are aligned to
// the element only: gfx950 takes vector loads at any address, and memcpy says so to the compiler.
constexpr int kRun = 8;

__device__ __forceinline__ float bits_float(uint32_t b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ uint32_t float_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

template <int TYPE> struct Stored;
template <> struct Stored<MOC_F32> { using type = float; };
template <> struct Stored<MOC_F16> { using type = _Float16; };
template <> struct Stored<MOC_BF16> { using type = __bf16; };
template <> struct Stored<MOC_E4M3> { using type = uint8_t; };
template <> struct Stored<MOC_I8> { using type = uint8_t; };

template <int TYPE>
__device__ __forceinline__ void load_run(const void* row, int64_t col, int n, float (&v)[kRun]) {
  using T = typename Stored<TYPE>::type;
  const T* p = static_cast<const T*>(row) + col;
  T t[kRun];
  if (n >= kRun) {
    __builtin_memcpy(t, p, sizeof t);
  } else {
#pragma unroll
    for (int i = 0; i < kRun; ++i) t[i] = i < n ? p[i] : T(0.0f);
  }
#pragma unroll
  for (int i = 0; i < kRun; ++i) v[i] = (float)t[i];
}

template <int TYPE>
__device__ __forceinline__ void store_run(void* row, int64_t col, int n, const float (&v)[kRun]) {
  using T = typename Stored<TYPE>::type;
  T* p = static_cast<T*>(row) + col;
  T t[kRun];
#pragma unroll
  for (int i = 0; i < kRun; ++i) t[i] = (T)v[i];
  if (n >= kRun) {
    __builtin_memcpy(p, t, sizeof t);
  } else {
#pragma unroll
    for (int i = 0; i < kRun; ++i)
      if (i < n) p[i] = t[i];
  }
}

// The same with the type known at run time only (uniform over the wave).
__device__ __forceinline__ void load_any(int type, const void* row, int64_t col, int n, float (&v)[kRun]) {
  if (type == MOC_BF16) load_run<MOC_BF16>(row, col, n, v);
  else if (type == MOC_F16) load_run<MOC_F16>(row, col, n, v);
  else load_run<MOC_F32>(row, col, n, v);
}
__device__ __forceinline__ void store_any(int type, void* row, int64_t col, int n, const float (&v)[kRun]) {
  if (type == MOC_BF16) store_run<MOC_BF16>(row, col, n, v);
  else if (type == MOC_F16) store_run<MOC_F16>(row, col, n, v);
  else store_run<MOC_F32>(row, col, n, v);
}

// ---- checkpoints --------------------------------------------------------------------------------

__device__ __forceinline__ float scale_of(uint8_t byte) { return bits_float((uint32_t)byte << 23); }

// Eight codes, as two words, to the values they stand for.
template <int FMT>
__device__ __forceinline__ void decode_run(uint2 c, float scale, float (&v)[kRun]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (FMT == MOC_E4M3) {
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
      v[4 * h] = lo[0] * scale;
      v[4 * h + 1] = lo[1] * scale;
      v[4 * h + 2] = hi[0] * scale;
      v[4 * h + 3] = hi[1] * scale;
    } else {
      const uint32_t u = w[h] ^ 0x80808080u;   // code + 128: a byte of it is converted in one instruction
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * h + i] = ((float)(u >> (8 * i) & 0xFF) - 128.0f) * scale;
      if (((u - 0x01010101u) & ~u & 0x80808080u) != 0) {   // a byte is 0: a code is NaN's
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if ((u >> (8 * i) & 0xFF) == 0) v[4 * h + i] = bits_float(0x7FC00000u);
      }
    }
  }
}

__device__ __forceinline__ uint2 load_codes(const uint8_t* p, int n) {
  uint2 c = {0, 0};
  if (n >= kRun) {
    __builtin_memcpy(&c, p, 8);
  } else {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kRun - 1; ++i)
      if (i < n) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    c = {w[0], w[1]};
  }
  return c;
}

__device__ __forceinline__ void store_codes(uint8_t* p, int n, uint2 c) {
  if (n >= kRun) {
    __builtin_memcpy(p, &c, 8);
  } else {
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < kRun - 1; ++i)
      if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}

// A row of a matrix that is a tensor or a checkpoint.
template <int TYPE>
__device__ __forceinline__ void load_held(const void* row, const uint8_t* scales, int64_t col, int n, float (&v)[kRun]) {
  if constexpr (TYPE == MOC_E4M3 || TYPE == MOC_I8) {
    decode_run<TYPE>(load_codes(static_cast<const uint8_t*>(row) + col, n), scale_of(scales[col / MOC_BLOCK]), v);
  } else {
    load_run<TYPE>(row, col, n, v);
  }
}

// Magnitudes above this are taken for it (what a code stands for stays finite in the values' type).
inline float most_kept(int fmt, int type) {
  const float top = type == MOC_F16 ? 32768.0f : 1.7014118346046923e38f;   // 2^15, 2^127
  return (fmt == MOC_E4M3 ? 1.875f : 1.96875f) * top;
}

// Whether a run has values that are not finite or above `most`; its largest finite magnitude, `most` at
// most.  Both are rare: the maximum takes no notice of NaN, and what is not finite times 0 is NaN.
__device__ __forceinline__ bool run_peak(const float (&v)[kRun], float most, float& peak) {
  float a = 0.0f, odd = 0.0f;
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    a = fmaxf(a, __builtin_fabsf(v[i]));
    odd = __builtin_fmaf(v[i], 0.0f, odd);
  }
  const bool special = odd != odd || a > most;
  if (special) {
    a = 0.0f;
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const float m = __builtin_fabsf(v[i]);
      a = m < kInf && m > a ? m : a;
    }
    a = fminf(a, most);
  }
  peak = a;
  return special;
}

// The exponent of a block's scale from its peak: the peak's own exponent less the format's, one more
// where its fraction is above that of the format's largest value.
template <int FMT>
__device__ __forceinline__ int scale_exp(float peak) {
  const uint32_t b = float_bits(peak);
  const int k = (int)(b >> 23) - 127 - (FMT == MOC_E4M3 ? 8 : 6) + ((b & 0x7FFFFFu) > (FMT == MOC_E4M3 ? 0x600000u : 0x7E0000u) ? 1 : 0);
  return max(k, kMinExp);
}

// Four finite values within the format's range, scaled, to four codes.
template <int FMT>
__device__ __forceinline__ uint32_t encode_four(const float* q) {
  if constexpr (FMT == MOC_E4M3) {
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], r, true);
  } else {
    // 1.5 * 2^23 rounds to whole numbers, ties to even, and leaves them in the lowest byte
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = float_bits(q[i] + 12582912.0f);
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000C0Cu);
    return lo | hi;
  }
}

template <int FMT>
__device__ __forceinline__ uint2 encode_run(const float (&v)[kRun], int k, float most, bool special) {
  const float inv = bits_float((uint32_t)(127 - k) << 23);
  float q[kRun];
#pragma unroll
  for (int i = 0; i < kRun; ++i) q[i] = v[i] * inv;
  if (special) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) q[i] = __builtin_fabsf(v[i]) < kInf ? fminf(fmaxf(v[i], -most), most) * inv : FMT == MOC_E4M3 ? kInf : -128.0f;   // infinity has no code of its own: 0x7F
  }
  return uint2{encode_four<FMT>(q), encode_four<FMT>(q + 4)};
}

// The maximum over the quad of lanes that holds a block's 32 columns.
__device__ __forceinline__ float quad_max(float a) {
  a = fmaxf(a, bits_float((uint32_t)__builtin_amdgcn_mov_dpp((int)float_bits(a), 0xB1, 0xF, 0xF, true)));   // quad_perm 1 0 3 2
  return fmaxf(a, bits_float((uint32_t)__builtin_amdgcn_mov_dpp((int)float_bits(a), 0x4E, 0xF, 0xF, true)));   // quad_perm 2 3 0 1
}

// A run of a row into a checkpoint; all four lanes of the quad come here together, those beyond the
// row with n <= 0 and values of 0.
template <int FMT>
__device__ __forceinline__ void keep_run(const float (&v)[kRun], int64_t col, int n, float most, uint8_t* codes, uint8_t* scales) {
  float peak;
  const bool special = run_peak(v, most, peak);
  const int k = scale_exp<FMT>(quad_max(peak));
  if (n > 0) {
    store_codes(codes + col, n, encode_run<FMT>(v, k, most, special));
    if ((col & (MOC_BLOCK - 1)) == 0) scales[col / MOC_BLOCK] = (uint8_t)(k + 127);
  }
}
__device__ __forceinline__ void keep_any(int fmt, const float (&v)[kRun], int64_t col, int n, float most, uint8_t* codes, uint8_t* scales) {
  if (fmt == MOC_E4M3) keep_run<MOC_E4M3>(v, col, n, most, codes, scales);
  else keep_run<MOC_I8>(v, col, n, most, codes, scales);
}

// ---- activations --------------------------------------------------------------------------------

// exp2 and the reciprocal are the hardware's (1 ulp each), and exp2's argument z is rounded to 32 bits: a value is off by 2^-21 +
// 2^-22 |z| of itself.  Next to a rounding to 16 bits that is nothing; float32 outputs hold 2^-16 where gelu or silu is
// smallest (gelu at -9: 2^-16.8).
__device__ __forceinline__ float over_one_plus(float u, float e) { return u * __builtin_amdgcn_rcpf(1.0f + e); }
__device__ __forceinline__ float exp_minus(float z) { return __builtin_amdgcn_exp2f(z * -1.4426950408889634f); }

constexpr float kGelu1 = 1.5957691216057308f;            // 2 sqrt(2 / pi)
constexpr float kGelu3 = 1.5957691216057308f * 0.044715f;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ void act_run(int act, float (&v)[kRun]) {
  if (act == MOC_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = v[i] <= 0.0f ? 0.0f : v[i];
  } else if (act == MOC_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = over_one_plus(v[i], __builtin_amdgcn_exp2f(v[i] * __builtin_fmaf(v[i] * v[i], -kLog2e * kGelu3, -kLog2e * kGelu1)));
  } else if (act == MOC_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = over_one_plus(v[i], exp_minus(v[i]));
  }
}

// d times the activation's derivative at u.
__device__ __forceinline__ void slope_run(int act, float (&d)[kRun], const float (&u)[kRun]) {
  if (act == MOC_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) d[i] = u[i] <= 0.0f ? 0.0f : u[i] > 0.0f ? d[i] : bits_float(0x7FC00000u);
  } else if (act == MOC_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      // beyond +-16 the derivative is 0 or 1 in 32 bits; the squares of larger arguments would overflow
      const float c = u[i] < -16.0f ? -16.0f : u[i] > 16.0f ? 16.0f : u[i];   // keeps a NaN
      const float q = c * c, s = over_one_plus(1.0f, __builtin_amdgcn_exp2f(c * __builtin_fmaf(q, -kLog2e * kGelu3, -kLog2e * kGelu1)));
      d[i] *= __builtin_fmaf(c * s * (1.0f - s), __builtin_fmaf(q, 3.0f * kGelu3, kGelu1), s);
    }
  } else if (act == MOC_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const float s = over_one_plus(1.0f, exp_minus(u[i]));
      d[i] *= s * __builtin_fmaf(u[i], 1.0f - s, 1.0f);
    }
  }
}

// ---- a run as it lies in memory -----------------------------------------------------------------

// Loaded early, converted when it is used: codes and their scale, 16-bit values, or floats.
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
struct Raw {
  u32x4 a, b;
  uint32_t scale;
};

template <int TYPE>
__device__ __forceinline__ Raw load_raw(const void* row, const uint8_t* scales, int col, int n) {
  Raw x = {};
  if constexpr (TYPE == MOC_E4M3 || TYPE == MOC_I8) {
    if (n <= 0) return x;
    const uint2 c = load_codes(static_cast<const uint8_t*>(row) + col, n);
    x.a[0] = c.x;
    x.a[1] = c.y;
    x.scale = scales[col / MOC_BLOCK];
  } else if constexpr (TYPE == MOC_F32) {
    const float* f = static_cast<const float*>(row) + col;
    if (n >= kRun) {
      __builtin_memcpy(&x.a, f, 16);
      __builtin_memcpy(&x.b, f + 4, 16);
    } else {
#pragma unroll
      for (int i = 0; i < kRun - 1; ++i)
        if (i < n) (i < 4 ? x.a : x.b)[i & 3] = float_bits(f[i]);
    }
  } else {
    const uint16_t* h = static_cast<const uint16_t*>(row) + col;
    if (n >= kRun) {
      __builtin_memcpy(&x.a, h, 16);
    } else {
#pragma unroll
      for (int i = 0; i < kRun - 1; ++i)
        if (i < n) x.a[i >> 1] |= (uint32_t)h[i] << (16 * (i & 1));
    }
  }
  return x;
}

// Of a row of eight columns at least: no branch, so that many are under way at once.  Beyond the row its
// last eight are read, and not used; where it ends in a run, too, and settle() moves them down.
template <int TYPE>
__device__ __forceinline__ Raw load_raw_whole(const void* row, const uint8_t* scales, int col, int cols) {
  Raw x = load_raw<TYPE>(row, scales, min(col, cols - kRun), kRun);
  if constexpr (TYPE == MOC_E4M3 || TYPE == MOC_I8) x.scale = scales[min(col, cols - 1) / MOC_BLOCK];
  return x;
}

// What load_raw_whole has loaded for `col` becomes that run, with zeros beyond the row.
template <int TYPE>
__device__ __forceinline__ void settle(Raw& x, int col, int cols) {
  const int n = cols - col;
  if (n >= kRun || n <= 0 || cols < kRun) return;
  const int down = kRun - n;
  if constexpr (TYPE == MOC_F32) {
    uint32_t w[2 * kRun] = {x.a[0], x.a[1], x.a[2], x.a[3], x.b[0], x.b[1], x.b[2], x.b[3]};   // and zeros
#pragma unroll
    for (int by = 1; by < kRun; by *= 2)
#pragma unroll
      for (int i = 0; i < 2 * kRun - by; ++i) w[i] = down & by ? w[i + by] : w[i];
#pragma unroll
    for (int i = 0; i < kRun; ++i) (i < 4 ? x.a : x.b)[i & 3] = w[i];
  } else {
    uint64_t lo = x.a[0] | (uint64_t)x.a[1] << 32, hi = x.a[2] | (uint64_t)x.a[3] << 32;
    if constexpr (TYPE == MOC_E4M3 || TYPE == MOC_I8) {
      lo >>= 8 * down;
    } else {
      const int bits = 16 * down;   // 16 .. 112
      lo = bits >= 64 ? hi >> (bits - 64) : lo >> bits | hi << (64 - bits);
      hi = bits >= 64 ? 0 : hi >> bits;
    }
    x.a = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
  }
}

template <int TYPE>
__device__ __forceinline__ void values_of(const Raw& x, float (&v)[kRun]) {
  if constexpr (TYPE == MOC_E4M3 || TYPE == MOC_I8) {
    decode_run<TYPE>(uint2{x.a[0], x.a[1]}, scale_of((uint8_t)x.scale), v);
  } else if constexpr (TYPE == MOC_F32) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = bits_float(i < 4 ? x.a[i & 3] : x.b[i & 3]);
  } else {
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const uint16_t h = (uint16_t)(x.a[i >> 1] >> (16 * (i & 1)));
      v[i] = TYPE == MOC_BF16 ? bits_float((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
    }
  }
}

// The same with the type known at run time only (uniform over the wave).
__device__ __forceinline__ Raw load_raw_any(int type, const void* row, const uint8_t* scales, int col, int n) {
  if (type == MOC_BF16 || type == MOC_F16) return load_raw<MOC_BF16>(row, scales, col, n);
  if (type == MOC_F32) return load_raw<MOC_F32>(row, scales, col, n);
  return load_raw<MOC_E4M3>(row, scales, col, n);
}
__device__ __forceinline__ void values_of_any(int type, const Raw& x, float (&v)[kRun]) {
  if (type == MOC_BF16) values_of<MOC_BF16>(x, v);
  else if (type == MOC_F16) values_of<MOC_F16>(x, v);
  else if (type == MOC_F32) values_of<MOC_F32>(x, v);
  else if (type == MOC_E4M3) values_of<MOC_E4M3>(x, v);
  else values_of<MOC_I8>(x, v);
}

// ---- sums over parts ----------------------------------------------------------------------------

// out[col] = sum over `parts` rows of `width` floats, `stride` apart, in one order: 64 columns a workgroup, a wave every
// sixteenth row, four of them under way.
[[maybe_unused]] __global__ __launch_bounds__(1024) void join_sums_kernel(const float* sums, int parts, int64_t width, int64_t stride, float* out) {
  __shared__ float stage[16][64];
  const int64_t col = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
  const int mine = threadIdx.x >> 6;
  float s = 0.0f;
  if (col < width) {
    int p = mine;
    for (; p + 48 < parts; p += 64) {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = sums[(p + 16 * i) * stride + col];
      s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    for (; p < parts; p += 16) s += sums[p * stride + col];
  }
  stage[mine][threadIdx.x & 63] = s;
  __syncthreads();
  if (mine == 0 && col < width) {
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += stage[i][threadIdx.x];
    out[col] = s;
  }
}

// ---- grids --------------------------------------------------------------------------------------

// A launch has fewer than 2^32 threads along x: more workgroups than that go on along y.
inline dim3 grid_of(int64_t blocks) {
  const int64_t x = blocks < (1 << 21) ? blocks : 1 << 21;
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}
__device__ __forceinline__ int64_t block_of() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// ---- descriptors --------------------------------------------------------------------------------

inline bool is_kept(int type) { return type == MOC_E4M3 || type == MOC_I8; }
inline bool is_value(int type) { return type == MOC_F32 || type == MOC_F16 || type == MOC_BF16; }
inline int type_bytes(int type) { return type == MOC_F32 ? 4 : is_kept(type) ? 1 : 2; }

inline bool sizes_ok(int64_t rows, int64_t cols) { return rows >= 0 && rows <= MOC_MAX_ROWS && cols >= 0 && cols <= MOC_MAX_COLS; }

// A tensor (values only) or a checkpoint (kept only) of rows x cols, with memory unless it is empty.
inline bool matrix_ok(const moc_matrix* x, int64_t rows, int64_t cols, bool values, bool kept) {
  if (!x || x->reserved != 0) return false;
  const bool ckpt = is_kept(x->type);
  if (!(ckpt ? kept : values && is_value(x->type))) return false;
  if (x->stride < cols || x->stride > MOC_MAX_STRIDE) return false;
  if (ckpt && (x->scale_stride < (cols + MOC_BLOCK - 1) / MOC_BLOCK || x->scale_stride > MOC_MAX_STRIDE)) return false;
  if (rows == 0 || cols == 0) return true;
  if (!x->data || (ckpt && !x->scales)) return false;
  return reinterpret_cast<uintptr_t>(x->data) % type_bytes(x->type) == 0;
}

inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline bool params_ok(const void* p, int type) { return !p || (is_value(type) && aligned_to(p, type_bytes(type))); }

}  // namespace

// Compute units of the current device (asked for once each), or an error code.
int moc_compute_units(int* out);
