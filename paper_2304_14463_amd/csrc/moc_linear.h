// The matrix product behind the linear layer and its gradients: out[m][n] = sum over k of A(m, k) B(n, k),
// 16-bit operands, 32-bit sums, on the matrix cores.
//
// Operands lie in memory either with k running along a row ("row": x and w of the forward pass, dy of
// the input's gradient) or with m or n running along it ("col": w of the input's gradient, dy and x of
// the weight's).  Both go to LDS as they lie, 16 bytes a lane, and come out of it as the matrix cores
// want them: a lane holds eight consecutive k of one m or n, which a row operand has next to each
// other (one 16-byte read) and a col operand below each other (two reads that transpose 4 x 16 values
// among 16 lanes, ds_read_b64_tr_b16).
//
// A workgroup computes BM x BN of the output, 64 of k at a time, in two buffers.  Two kernels: one whose
// loads run straight into LDS while the other buffer is multiplied, for large products of aligned
// operands, and one whose loads wait in registers, for everything else.
#pragma once

#include <algorithm>

#include "moc_training.h"

namespace {

constexpr int kStepK = 64;                      // k of a step
constexpr int kRowBytes = kStepK * 2;           // of a row operand's row in LDS
constexpr int kWindow = 0x7FFFFFF0;             // bytes a buffer descriptor covers; an offset of this reads as 0

using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using s16x4 = short __attribute__((ext_vector_type(4)));
using s16x8 = short __attribute__((ext_vector_type(8)));

// S x S of the result, 512 / S of k: with operands in registers and normally distributed values 16 x 16 x 32 reaches
// 2.0 PFLOP/s and 32 x 32 x 16, which reads and writes the sums twice as often, 1.3; but it needs half the registers for
// operands, so it is taken where a loader needs them.
template <int S> struct Sums;
template <> struct Sums<16> { using type = float __attribute__((ext_vector_type(4))); };
template <> struct Sums<32> { using type = float __attribute__((ext_vector_type(16))); };

template <int TYPE>
__device__ __forceinline__ Sums<16>::type mfma(s16x8 a, s16x8 b, Sums<16>::type c) {
  if constexpr (TYPE == MOC_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int TYPE>
__device__ __forceinline__ Sums<32>::type mfma(s16x8 a, s16x8 b, Sums<32>::type c) {
  if constexpr (TYPE == MOC_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <class V>
__device__ __forceinline__ void clear(V& x) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof x / 4); ++i) x[i] = 0.0f;
}

enum { kRow = 0, kCol = 1 };                       // how an operand lies
enum Loading { kDirect, kThroughRegisters, kNarrow };   // how operands can get to LDS; kNarrow: some have rows of fewer than eight

struct Operand {
  const void* data;
  const uint8_t* scales;     // a checkpoint's
  int64_t stride, scale_stride;
};

struct Epilogue {
  const void* bias;
  int bias_type;
  int act;
  // A matrix of the output's sizes: the residual, or the activation's argument, through whose
  // derivative the sum goes then (`slope`).  Null: none.
  const void* extra;
  const uint8_t* extra_scales;
  int extra_type, slope;
  int64_t extra_stride, extra_scale_stride;
  void* out;
  int out_type;
  int64_t out_stride;
  uint8_t *codes, *scales;    // the checkpoint of what the activation is taken of; null: none
  int kept_type;
  int64_t code_stride, scale_stride;
  float most;
};

// Where the part of k ends that starts at `begin` < k: begin + each can be past 2^31 where k is a weight gradient's rows.
__host__ __device__ inline int part_end(int k, int begin, int each) { return k - begin < each ? k : begin + each; }

struct LinearArgs {
  Operand a, b;
  int m, n, k;
  int tiles_m, tiles_n, splits, split_k;   // split_k: k of a split, a multiple of kStepK
  float* partial;                          // [splits][m][partial_stride], then [splits][m] of `sums`; splits > 1 only
  int64_t partial_stride;                  // n up to a multiple of MOC_BLOCK
  float* sums;                             // [m]: of a over k (the bias's gradient), col operands only; null: none
  Epilogue e;
};

// ---- epilogue -----------------------------------------------------------------------------------

__device__ __forceinline__ const char* row_at(const void* x, int type, int64_t row, int64_t stride) {
  return static_cast<const char*>(x) + row * stride * (type == MOC_F32 ? 4 : type == MOC_BF16 || type == MOC_F16 ? 2 : 1);
}

__device__ __forceinline__ Raw load_extra(const Epilogue& e, int64_t row, int col, int n) {
  if (!e.extra || n <= 0) return Raw{};
  return load_raw_any(e.extra_type, row_at(e.extra, e.extra_type, row, e.extra_stride), e.extra_scales + row * e.extra_scale_stride, col, n);
}

// A run of finished sums; the four lanes of a quad have a block of a row, n <= 0 beyond the row.
__device__ __forceinline__ void finish_sum(const Epilogue& e, int64_t row, int col, int n, const float (&bias)[kRun], const Raw& extra, float (&v)[kRun]) {
#pragma unroll
  for (int r = 0; r < kRun; ++r) v[r] = r < n ? v[r] + bias[r] : 0.0f;
  if (e.codes) keep_any(e.kept_type, v, col, n, e.most, e.codes + row * e.code_stride, e.scales + row * e.scale_stride);
  if (n <= 0) return;
  if (e.slope) {
    float u[kRun];
    values_of_any(e.extra_type, extra, u);
    slope_run(e.act, v, u);
  } else {
    act_run(e.act, v);
    if (e.extra) {
      float r[kRun];
      values_of_any(e.extra_type, extra, r);
#pragma unroll
      for (int i = 0; i < kRun; ++i) v[i] += r[i];
    }
  }
  store_any(e.out_type, const_cast<char*>(row_at(e.out, e.out_type, row, e.out_stride)), col, n, v);
}

// ---- operands to LDS ----------------------------------------------------------------------------

using Lds = __attribute__((address_space(3))) uint8_t;

// Which 16 bytes of its row of the tile lie at place `pos` of row `row` in LDS.  Reads of one
// instruction then meet all banks evenly: 16 rows of a row operand at one k, 4 rows of a col operand.
template <int LAY, int WIDTH>
__device__ __forceinline__ int swizzle(int row) {
  if constexpr (LAY == kRow) return (row >> 1) & 7;
  else if constexpr (WIDTH >= 128) return (row & 3) << 2;
  else if constexpr (WIDTH == 64) return ((row >> 1) & 1) << 2;
  else return 0;
}

// The part of an operand that a workgroup goes through: WIDTH of m or n from `first`, k from `begin`.
template <int LAY, int WIDTH, int THREADS>
struct Tile {
  static constexpr int kPieces = WIDTH * 8;                    // 16 bytes each
  static constexpr int kEach = kPieces / THREADS;              // of a thread
  static constexpr int kPerRow = LAY == kRow ? 8 : WIDTH / 8;  // of a row in LDS
  static_assert(kPieces % THREADS == 0);
  // the row in LDS, and the 16 bytes of the tile's row, of piece i of this thread
  static __device__ __forceinline__ int row(int i) { return (i * THREADS + (int)threadIdx.x) / kPerRow; }
  static __device__ __forceinline__ int piece(int i) {
    return ((i * THREADS + (int)threadIdx.x) % kPerRow) ^ swizzle<LAY, WIDTH>(row(i));
  }
};

// Straight into LDS by buffer loads, which read 0 beyond their window: offsets are set once, the
// window's base moves with k.  Rows, and runs of eight along a row, are whole here.
template <int LAY, int WIDTH, int THREADS>
struct DirectLoader {
  using T = Tile<LAY, WIDTH, THREADS>;
  static constexpr int kLoads = T::kEach;
  const char* base;       // of the window: the tile's first row and k
  int64_t left;           // bytes from there to the operand's end
  int64_t step;           // bytes the base moves by
  int offset[T::kEach];
  int k_left;

  __device__ __forceinline__ DirectLoader(const Operand& x, int first, int extent, int begin, int end) {
    const int64_t rb = x.stride * 2;
    const char* const data = static_cast<const char*>(x.data);
    if constexpr (LAY == kRow) {
      base = data + first * rb + (int64_t)begin * 2;
      left = (int64_t)(extent - first - 1) * rb + (int64_t)(end - begin) * 2;
      step = kRowBytes;
    } else {
      base = data + begin * rb + (int64_t)first * 2;
      left = (int64_t)(end - begin - 1) * rb + (int64_t)(extent - first) * 2;
      step = kStepK * rb;
    }
    k_left = end - begin;
#pragma unroll
    for (int i = 0; i < T::kEach; ++i) {
      const int row = T::row(i), piece = T::piece(i);
      offset[i] = (int)(row * rb) + piece * 16;
      if (LAY == kCol && first + piece * 8 >= extent) offset[i] = kWindow;
    }
  }
  __device__ __forceinline__ void load(Lds* to) {
    const __amdgpu_buffer_rsrc_t window =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (int)(left < kWindow ? (left > 0 ? left : 0) : kWindow), 0x00020000);
    const bool last = LAY == kRow && k_left < kStepK;
#pragma unroll
    for (int i = 0; i < T::kEach; ++i) {
      int at = offset[i];
      if (last && T::piece(i) * 8 >= k_left) at = kWindow;
      const int wave = (i * THREADS + ((int)threadIdx.x & ~(kWave - 1))) * 16;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(window, (__attribute__((address_space(3))) void*)(to + __builtin_amdgcn_readfirstlane(wave)), 16, at, 0, 0, 0);
    }
    base += step;
    left -= step;
    k_left -= kStepK;
  }
  static constexpr int kWork = 0, kWrites = 0;
  __device__ __forceinline__ void put(Lds*, int) {}
  __device__ __forceinline__ void mend(Lds*) {}
};

// Through registers: any alignment and size, and checkpoints, whose codes become values on the way.
// Loads have no branch: of a run that the row ends in, the row's last eight are loaded and moved down
// when they are put; rows beyond the last are the last one, put as zeros where they are k.  NARROW: rows
// of fewer than eight.
template <int LAY, int WIDTH, int THREADS, int TYPE, int HELD, bool NARROW = false>
struct RegisterLoader {
  using T = Tile<LAY, WIDTH, THREADS>;
  using V = typename Stored<TYPE>::type;
  static constexpr bool kKept = HELD == MOC_E4M3 || HELD == MOC_I8;
  // A step's part of this thread: 16-bit values, or eight codes and their scale.
  struct Set {
    uint32_t w[T::kEach][kKept ? 2 : 4];
    uint8_t scale[kKept ? T::kEach : 1];
  };
  static constexpr int kBytes = kKept ? 1 : 2;   // of a value
  Operand x;
  int first, extent, end;
  // Where pieces lie from the tile's first row on, for k = 0 and in 32 bits: the address of a load is then
  // one in scalar registers that moves with k, and this.  Room for a run that is moved down (kRow).
  static constexpr uint32_t kRoom = kRun * kBytes;
  uint32_t place[T::kEach], scale_place[kKept ? T::kEach : 1];

  __device__ __forceinline__ RegisterLoader(const Operand& x_, int first_, int extent_, int end_) : x(x_), first(first_), extent(extent_), end(end_) {
    static_assert(!kKept || LAY == kCol);
#pragma unroll
    for (int i = 0; i < T::kEach; ++i) {
      const int row = T::row(i);
      if constexpr (LAY == kRow) {
        place[i] = (uint32_t)min(row, extent - 1 - first) * row_bytes() + kRoom;
      } else {
        place[i] = (uint32_t)row * row_bytes() + column(i);
        if constexpr (kKept) scale_place[i] = (uint32_t)row * (uint32_t)x.scale_stride + scale_column(i);
      }
    }
  }

  // values of the memory's rows, their bytes, and where in them a piece lies (kCol)
  __device__ __forceinline__ int length() const { return LAY == kRow ? end : extent; }
  __device__ __forceinline__ uint32_t row_bytes() const { return (uint32_t)x.stride * kBytes; }
  __device__ __forceinline__ uint32_t column(int i) const { return (uint32_t)min(first + T::piece(i) * kRun, extent - kRun) * kBytes; }
  __device__ __forceinline__ uint32_t scale_column(int i) const { return (uint32_t)min(first + T::piece(i) * kRun, extent - 1) / MOC_BLOCK; }

  // k < end
  __device__ __forceinline__ void load(Set& s, int k) const {
    const char* const data = static_cast<const char*>(x.data);
    if constexpr (NARROW) {
#pragma unroll
      for (int i = 0; i < T::kEach; ++i) {
        const int row = min((LAY == kRow ? first : k) + T::row(i), (LAY == kRow ? extent : end) - 1), c = (LAY == kRow ? k : first) + T::piece(i) * kRun, n = length() - c;
        const char* const at = data + row * x.stride * kBytes;
        if constexpr (kKept) {
          const uint2 codes = load_codes(reinterpret_cast<const uint8_t*>(at) + c, n);
          s.w[i][0] = codes.x;
          s.w[i][1] = codes.y;
          s.scale[i] = x.scales[row * x.scale_stride + scale_column(i)];
        } else {
          const Raw r = load_raw<TYPE>(at, nullptr, c, n);
#pragma unroll
          for (int j = 0; j < 4; ++j) s.w[i][j] = r.a[j];
        }
      }
    } else if constexpr (LAY == kRow) {
      const char* const from = data + first * x.stride * kBytes + (int64_t)k * kBytes - kRoom;
      const int most = end - kRun - k;   // -7 at least
#pragma unroll
      for (int i = 0; i < T::kEach; ++i) __builtin_memcpy(s.w[i], from + (place[i] + (uint32_t)(min(T::piece(i) * kRun, most) * kBytes)), sizeof s.w[i]);
    } else {
      const char* const from = data + k * x.stride * kBytes;
      const uint32_t below = (uint32_t)min(end - 1 - k, kStepK - 1), most = below * row_bytes();   // the last row
#pragma unroll
      for (int i = 0; i < T::kEach; ++i) {
        __builtin_memcpy(s.w[i], from + min(place[i], most + column(i)), sizeof s.w[i]);
        if constexpr (kKept) s.scale[i] = (x.scales + k * x.scale_stride)[min(scale_place[i], below * (uint32_t)x.scale_stride + scale_column(i))];
      }
    }
  }
  // What was loaded for k.
  __device__ __forceinline__ void put(const Set& s, int k, Lds* lds) const {
    const bool edge = k + kStepK > end || (LAY == kCol && first + WIDTH > extent);   // the same for all
    if (!edge) {
#pragma unroll
      for (int i = 0; i < T::kEach; ++i) put_piece(s, i, s.w[i], lds);
      return;
    }
#pragma unroll
    for (int i = 0; i < T::kEach; ++i) {
      uint64_t v[kKept ? 1 : 2];
      __builtin_memcpy(v, s.w[i], sizeof v);
      const int n = LAY == kCol && k + T::row(i) >= end ? 0 : length() - (LAY == kRow ? k : first) - T::piece(i) * kRun;   // that exist
      const int down = NARROW || n >= kRun ? 0 : kRun - n;
      if (n <= 0) {
#pragma unroll
        for (uint64_t& p : v) p = 0;
      } else if (down > 0) {
        if constexpr (kKept) {
          v[0] >>= 8 * down;
        } else {
          const int bits = 16 * down;
          v[0] = bits >= 64 ? v[1] >> (bits - 64) : v[0] >> bits | v[1] << (64 - bits);
          v[1] = bits >= 64 ? 0 : v[1] >> bits;
        }
      }
      uint32_t w[kKept ? 2 : 4];
      __builtin_memcpy(w, v, sizeof w);
      put_piece(s, i, w, lds);
    }
  }
  template <int N>
  __device__ __forceinline__ void put_piece(const Set& s, int i, const uint32_t (&w)[N], Lds* lds) const {
    u32x4 out;
    if constexpr (kKept) {
      float f[kRun];
      decode_run<HELD>(uint2{w[0], w[1]}, scale_of(s.scale[i]), f);
      V t[kRun];
#pragma unroll
      for (int j = 0; j < kRun; ++j) t[j] = (V)f[j];
      __builtin_memcpy(&out, t, 16);
    } else {
      __builtin_memcpy(&out, w, 16);
    }
    *(__attribute__((address_space(3))) u32x4*)(lds + (i * THREADS + (int)threadIdx.x) * 16) = out;
  }
};

// A checkpoint whose rows and strides are multiples of 16: a thread has the 32 values of a block in one
// row, that is two loads and one scale a step, and turns them into 16-bit values between the products.
template <int WIDTH, int THREADS, int TYPE, int FMT>
struct KeptLoader {
  static_assert(WIDTH * kStepK / MOC_BLOCK == THREADS);
  static constexpr int kPer = WIDTH / MOC_BLOCK;   // blocks of a row of the tile
  static constexpr int kLoads = 3;
  static constexpr int kWork = FMT == MOC_E4M3 ? 3 : 8;   // vector instructions for each product
  static constexpr int kWrites = 4;
  const uint8_t *base, *scale_base;
  int64_t left, scale_left, step, scale_step;
  int offset[2], scale_offset, place;
  u32x4 codes[2];
  uint8_t scale;
  uint32_t rare = 0;

  __device__ __forceinline__ KeptLoader(const Operand& x, int first, int extent, int begin, int end) {
    const int row = threadIdx.x / kPer, block = threadIdx.x % kPer;
    base = static_cast<const uint8_t*>(x.data) + begin * x.stride + first;
    left = (int64_t)(end - begin - 1) * x.stride + (extent - first);
    step = kStepK * x.stride;
    scale_base = x.scales + begin * x.scale_stride + first / MOC_BLOCK;
    scale_left = (int64_t)(end - begin - 1) * x.scale_stride + (extent - first + MOC_BLOCK - 1) / MOC_BLOCK;
    scale_step = kStepK * x.scale_stride;
#pragma unroll
    for (int h = 0; h < 2; ++h) offset[h] = first + block * MOC_BLOCK + 16 * h < extent ? (int)(row * x.stride) + block * MOC_BLOCK + 16 * h : kWindow;
    scale_offset = first + block * MOC_BLOCK < extent ? (int)(row * x.scale_stride) + block : kWindow;
    place = (row * (WIDTH / 8) + ((block * 4) ^ swizzle<kCol, WIDTH>(row))) * 16;   // moves whole blocks only
  }
  static __device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const uint8_t* base, int64_t left) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, (int)(left < kWindow ? (left > 0 ? left : 0) : kWindow), 0x00020000);
  }
  __device__ __forceinline__ void load(Lds*) {
    const __amdgpu_buffer_rsrc_t w = window(base, left);
    scale = __builtin_amdgcn_raw_buffer_load_b8(window(scale_base, scale_left), scale_offset, 0, 0);
#pragma unroll
    for (int h = 0; h < 2; ++h) codes[h] = __builtin_amdgcn_raw_buffer_load_b128(w, offset[h], 0, 0);
    base += step;
    left -= step;
    scale_base += scale_step;
    scale_left -= scale_step;
  }
  __device__ __forceinline__ void put(Lds* to, int h) {
    const float s = scale_of(scale);
    u32x4 out[2];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t w = codes[h][q];
      if constexpr (FMT == MOC_E4M3) {   // a power of two is exact, as the conversion is
        if constexpr (TYPE == MOC_BF16) {
          out[q >> 1][2 * q & 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, s, false));
          out[q >> 1][(2 * q & 3) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, s, true));
        } else {
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
          out[q >> 1][2 * q & 3] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)(lo[0] * s), (_Float16)(lo[1] * s)});
          out[q >> 1][(2 * q & 3) + 1] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)(hi[0] * s), (_Float16)(hi[1] * s)});
        }
      } else {
        // code + 128, of which a byte is taken in one instruction; exact unless 128 * s overflows
        const uint32_t u = w ^ 0x80808080u;
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __builtin_fmaf((float)(u >> (8 * i) & 0xFF), s, s * -128.0f);
        rare |= (u - 0x01010101u) & ~u & 0x80808080u;   // a byte of it is 0 (and perhaps, for nothing, a 1 above one)
        if constexpr (TYPE == MOC_BF16) {
          out[q >> 1][2 * q & 3] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)f[0], (__bf16)f[1]});
          out[q >> 1][(2 * q & 3) + 1] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)f[2], (__bf16)f[3]});
        } else {
          out[q >> 1][2 * q & 3] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)f[0], (_Float16)f[1]});
          out[q >> 1][(2 * q & 3) + 1] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)f[2], (_Float16)f[3]});
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) *(__attribute__((address_space(3))) u32x4*)(to + place + (2 * h + i) * 16) = out[i];
  }
  // What put() does not look at, behind it: codes of NaN, and scales of 2^121 and above.
  __device__ __forceinline__ void mend(Lds* to) {
    if constexpr (FMT == MOC_I8) {
      if (rare != 0 || scale >= 127 + 121) {
        using V = typename Stored<TYPE>::type;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 c = codes[i >> 1];
          float v[kRun];
          decode_run<FMT>(i & 1 ? uint2{c[2], c[3]} : uint2{c[0], c[1]}, scale_of(scale), v);
          V t[kRun];
#pragma unroll
          for (int j = 0; j < kRun; ++j) t[j] = (V)v[j];
          u32x4 out;
          __builtin_memcpy(&out, t, 16);
          *(__attribute__((address_space(3))) u32x4*)(to + place + i * 16) = out;
        }
      }
      rare = 0;
    }
  }
};

// ---- LDS to the matrix cores --------------------------------------------------------------------

// S x 512 / S pieces of an operand for one wave, whose m or n start at `first` in the tile: a lane has eight k
// of one m or n, lane % S.
template <int S, int LAY, int WIDTH, int COUNT>
struct Reader {
  static constexpr int kK = 512 / S, kParts = kStepK / kK;
  static constexpr int kEach = LAY == kRow ? 1 : 2;   // instructions of a read
  static constexpr int kSame = 32 / S;                // pieces that lie alike: the swizzle moves 32 columns at least
  int at[LAY == kRow ? 1 : (COUNT + kSame - 1) / kSame][LAY == kRow ? kParts : 1];

  __device__ __forceinline__ explicit Reader(int first) {
    const int lane = threadIdx.x & (kWave - 1);
    if constexpr (LAY == kRow) {   // 16 rows further on the swizzle is the same
      const int row = first + lane % S;
#pragma unroll
      for (int s = 0; s < kParts; ++s) at[0][s] = row * kRowBytes + ((kK / 8 * s + lane / S) ^ swizzle<LAY, WIDTH>(row)) * 16;
    } else {
      const int in = lane & 15, k = lane / S * 8 + (in >> 2);   // swizzle() looks at k % 4 only
#pragma unroll
      for (int c = 0; c < COUNT; c += kSame) {
        const int col = first + S * c + (lane & (S - 16)) + (in & 3) * 4;
        at[c / kSame][0] = k * WIDTH * 2 + ((col >> 3) ^ swizzle<LAY, WIDTH>(in >> 2)) * 16 + (col & 7) * 2;
      }
    }
  }
  // k of kK * s and on
  __device__ __forceinline__ s16x8 read(const Lds* from, int c, int s) const {
    if constexpr (LAY == kRow) {
      return *(const __attribute__((address_space(3))) s16x8*)(from + at[0][s] + S * c * kRowBytes);
    } else {
      using P = __attribute__((address_space(3))) s16x4*;
      const Lds* const p = from + at[c / kSame][0] + c % kSame * S * 2 + kK * s * WIDTH * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 4 * WIDTH * 2));
      return s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    }
  }
};

// ---- tiles --------------------------------------------------------------------------------------

struct TileAt {
  int m0, n0;
};
// Workgroups go round the eight XCDs: each XCD takes a stretch of neighbouring tiles, in groups of
// eight rows of tiles, so that what its L2 holds is used again.
template <int BM, int BN>
__device__ __forceinline__ TileAt tile_of(const LinearArgs& g) {
  int64_t tile = blockIdx.x;
  const int tiles = g.tiles_m * g.tiles_n, per = tiles / 8, more = tiles % 8, xcd = (int)(tile % 8);
  tile = (int64_t)xcd * per + (xcd < more ? xcd : more) + tile / 8;
  const int band = 8 * g.tiles_n, first_m = (int)(tile / band) * 8, height = min(8, g.tiles_m - first_m), in = (int)(tile % band);
  return TileAt{(first_m + in % height) * BM, in / height * BN};
}

// Out by way of LDS, so that lanes next to each other have runs next to each other and a quad has a
// block of 32.  A lane has runs of four n of one m, lane % S.  Every
// wave stages its own outputs, 64 rows at a time, in memory of its own; 16 bytes of a row are moved
// by the row's number, so that writes (16 rows at once) and reads (whole rows) meet all banks.
// s0 .. s3: BN, BN, BM and BM rows of an operand's tile, nothing in them still wanted.
template <int S, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void write_out(const LinearArgs& g, const typename Sums<S>::type (&acc)[BM / WM / S][BN / WN / S], int m0, int n0, Lds* s0, Lds* s1, Lds* s2, Lds* s3) {
  constexpr int TM = BM / WM / S, TN = BN / WN / S;
  constexpr int TH = TM < 64 / S ? TM : 64 / S, kCols = TN * S, kChunks = kCols / 4, kMove = kChunks < 16 ? kChunks - 1 : 15;
  constexpr int kStage = TH * S * kCols * 4, kPer = BN * kRowBytes / kStage;   // waves that one of the arrays has room for
  static_assert(kPer >= 1 && (kPer >= WM * WN || (2 * kPer >= WM * WN && BM <= BN) || (BM >= BN && 4 * kPer >= WM * WN)));
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  const int array = wave / kPer;
  Lds* const stage = (array == 0 ? s0 : array == 1 ? s1 : array == 2 ? s2 : s3) + wave % kPer * kStage;
  const int lane = threadIdx.x & (kWave - 1);
  constexpr int kRuns = kCols / kRun, kRowsAt = kWave / kRuns;   // runs of a row, rows at a time
  const int col = n0 + wn + lane % kRuns * kRun, n = g.n - col;
  float bias[kRun];
#pragma unroll
  for (int r = 0; r < kRun; ++r) bias[r] = 0.0f;
  if (g.e.bias && g.splits == 1 && n > 0) load_any(g.e.bias_type, g.e.bias, col, n, bias);
  constexpr int kAhead = 3;   // rows of the extra operand on their way
  Raw ahead[kAhead];
#pragma unroll
  for (int half = 0; half < TM / TH; ++half) {
    const int row0 = m0 + wm + half * TH * S + lane / kRuns;
    const auto extra = [&](int at) { return row0 + at * kRowsAt < g.m && at * kRowsAt < TH * S && g.splits == 1 ? load_extra(g.e, row0 + at * kRowsAt, col, n) : Raw{}; };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i] = extra(i);
#pragma unroll
    for (int i = 0; i < TH; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < S * S / 256; ++q) {   // 64 / S lanes have the next runs
          const int m = S * i + lane % S, chunk = S / 4 * j + 64 / S * q + lane / S;
          const auto& c = acc[half * TH + i][j];
          *(__attribute__((address_space(3))) f32x4*)(stage + m * (kCols * 4) + (chunk ^ (m & kMove)) * 16) = f32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
        }
#pragma unroll 1
    for (int at = 0; at < TH * S / kRowsAt; ++at) {
      const int row = row0 + at * kRowsAt, m = lane / kRuns + at * kRowsAt;
      if (row >= g.m) break;   // all lanes of a row, and of a quad
      const Raw now = ahead[0];
#pragma unroll
      for (int i = 0; i + 1 < kAhead; ++i) ahead[i] = ahead[i + 1];
      ahead[kAhead - 1] = extra(at + kAhead);
      float v[kRun];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 c = *(const __attribute__((address_space(3))) f32x4*)(stage + m * (kCols * 4) + ((lane % kRuns * 2 + h) ^ (m & kMove)) * 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[4 * h + r] = c[r];
      }
      if (g.splits > 1) {
        if (col < g.partial_stride) store_run<MOC_F32>(g.partial + ((int64_t)blockIdx.y * g.m + row) * g.partial_stride, col, kRun, v);
      } else {
        finish_sum(g.e, row, col, n, bias, now, v);
      }
    }
  }
}

// ---- the kernel ---------------------------------------------------------------------------------

template <int TYPE, int LAY, int WIDTH, int THREADS, int HELD>
struct PickB;
template <int TYPE, int LAY, int WIDTH, int THREADS>
struct PickB<TYPE, LAY, WIDTH, THREADS, TYPE> { using type = DirectLoader<LAY, WIDTH, THREADS>; };
template <int TYPE, int WIDTH, int THREADS>
struct PickB<TYPE, kCol, WIDTH, THREADS, MOC_E4M3> { using type = KeptLoader<WIDTH, THREADS, TYPE, MOC_E4M3>; };
template <int TYPE, int WIDTH, int THREADS>
struct PickB<TYPE, kCol, WIDTH, THREADS, MOC_I8> { using type = KeptLoader<WIDTH, THREADS, TYPE, MOC_I8>; };

// Has the scheduler put a read from LDS behind each product, as long as there are any, then the loads
// into it, evenly; and `WORK` vector instructions and the writes to LDS that follow from them.
template <int MFMA, int READS, int LOADS, int WORK, int WRITES, int I = 0>
__device__ __forceinline__ void interleave() {
  if constexpr (I < MFMA) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    constexpr int kAt = (READS + MFMA - 1) / MFMA, kReads = READS < kAt ? READS : kAt;
    constexpr int kLoads = (LOADS + MFMA - I - 1) / (MFMA - I), kWrites = I * 2 < MFMA ? 0 : (WRITES + MFMA - I - 1) / (MFMA - I);
    if constexpr (kReads > 0) __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
    if constexpr (kLoads > 0) __builtin_amdgcn_sched_group_barrier(0x020, kLoads, 0);
    if constexpr (WORK > 0) __builtin_amdgcn_sched_group_barrier(0x002, WORK, 0);
    if constexpr (kWrites > 0) __builtin_amdgcn_sched_group_barrier(0x200, kWrites, 0);
    interleave<MFMA, READS - kReads, LOADS - kLoads, WORK, WRITES - kWrites, I + 1>();
  }
}

// TYPE of the operands; HELD: of b, TYPE or a checkpoint's.  256 x 256 by eight waves, two on a SIMD, 128 x 64
// each: 64 KB come from L2 for every 8 MFLOP.  16384 x 4096 x 16384 in bf16: 1.76 to 1.83 ms (1.22 PFLOP/s; a library's
// product 1.49 to 1.58 beside it), by columns 1.69 (w) and 1.65 (both), from e4m3 1.93, int8 2.12.  The matrix cores are busy
// 63 % of the clocks (w by columns 70, both 73, e4m3 57, int8 52), of which power leaves 1.8 to 1.9 GHz (x all zeros: 10 %
// less time).  The rest: one workgroup has a compute unit's LDS, so nothing is multiplied while 256 x 256 results go out (the
// input's gradient 1.69 ms with 4096 columns of output, 1.71 to 2.0 with 16384); reads by columns conflict in LDS for 25 %
// (one operand) and 50 % (both) of its clocks; 52 bytes a lane are spilled where w lies by columns.  Tried and slower: four
// waves of 128 x 128, lines brought to L2 a step ahead.
template <int TYPE, int ALAY, int BLAY, int BM, int BN, int WM, int WN, int HELD>
__global__ __launch_bounds__(WM* WN* kWave, 2) void linear_kernel(LinearArgs g) {
  constexpr int kThreads = WM * WN * kWave;
  constexpr int S = HELD == TYPE ? 16 : 32;
  constexpr int TM = BM / WM / S, TN = BN / WN / S;   // S x S outputs of a wave
  constexpr int kParts = S == 16 ? 2 : 4, TH = TM * kParts / 4;   // of k in a step; outputs down of a quarter of a step
  __shared__ __attribute__((aligned(1024))) uint8_t a0[BM * kRowBytes], a1[BM * kRowBytes], b0[BN * kRowBytes], b1[BN * kRowBytes];

  const TileAt at = tile_of<BM, BN>(g);
  const int m0 = at.m0, n0 = at.n0;
  const int begin = blockIdx.y * g.split_k, end = part_end(g.k, begin, g.split_k);

  using LoadA = DirectLoader<ALAY, BM, kThreads>;
  using LoadB = typename PickB<TYPE, BLAY, BN, kThreads, HELD>::type;
  LoadA la(g.a, m0, g.m, begin, end);
  LoadB lb(g.b, n0, g.n, begin, end);

  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  const Reader<S, ALAY, BM, TM> ra(wm);
  const Reader<S, BLAY, BN, TN> rb(wn);

  typename Sums<S>::type acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) clear(acc[i][j]);

  // A quarter of a step: 16 of k, or 32 of k by half of the wave's rows.
  s16x8 fa[2][TH], fb[2][TN];
  const auto part = [](int q) { return q * kParts / 4; };
  const auto fetch = [&](const Lds* a, const Lds* b, int q) {
    if (q * kParts % 4 == 0) {
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[part(q) & 1][j] = rb.read(b, j, part(q));
    }
#pragma unroll
    for (int i = 0; i < TH; ++i) fa[q & 1][i] = ra.read(a, q * TH % TM + i, part(q));
  };
  const auto multiply = [&](int q) {
#pragma unroll
    for (int i = 0; i < TH; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        auto& c = acc[q * TH % TM + i][j];
        c = mfma<TYPE>(fb[part(q) & 1][j], fa[q & 1][i], c);   // rows of the result: n
      }
  };
  const auto load = [&](Lds* a, Lds* b) {
    la.load(a);
    lb.load(b);
  };
  const auto put = [&](Lds* a, Lds* b, int h) {
    la.put(a, h);
    lb.put(b, h);
  };
  const auto arrived = [] {
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0), lgkmcnt(0): this wave's loads into LDS, its reads and writes
    __syncthreads();
  };
  constexpr int kReadsA = TH * decltype(ra)::kEach, kReads = kReadsA + TN * decltype(rb)::kEach;   // with a's part of k the same, and another
  // A step on what lies in (a, b), with the next step's operands on their way to (c, d): every quarter
  // is read while the one before is multiplied.  The last multiplication comes after the barrier, to
  // cover the first reads of the next step; (a, b), all read, take the step after that.  What lies
  // beyond the last step is not read from memory (its window is empty) and not used.
  const auto step = [&](Lds* a, Lds* b, Lds* c, Lds* d) {
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      fetch(a, b, q + 1);
      multiply(q);
      if (q == 0) {
        interleave<TH * TN, kParts == 4 ? kReads : kReadsA, 0, 0, 0>();
      } else {
        put(c, d, q - 1);
        if (q == 1) interleave<TH * TN, kReads, 0, LoadB::kWork, LoadB::kWrites / 2>();
        else interleave<TH * TN, kParts == 4 ? kReads : kReadsA, 0, LoadB::kWork, LoadB::kWrites / 2>();
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    lb.mend(d);
    arrived();
    fetch(c, d, 0);
    load(a, b);
    multiply(3);
    interleave<TH * TN, kReads, LoadA::kLoads + LoadB::kLoads, 0, 0>();
    __builtin_amdgcn_sched_barrier(0);
  };
  // Steps in pairs, so that each buffer has its own code (and the compiler sees that the loads do not
  // touch what is read); an odd one comes first.
  Lds *const pa0 = (Lds*)a0, *const pa1 = (Lds*)a1, *const pb0 = (Lds*)b0, *const pb1 = (Lds*)b1;
  const int steps = end > begin ? (end - begin + kStepK - 1) / kStepK : 0;
  if (steps & 1) {
    load(pa1, pb1);
    put(pa1, pb1, 0);
    put(pa1, pb1, 1);
    lb.mend(pb1);
    arrived();
    fetch(pa1, pb1, 0);
    load(pa0, pb0);
    step(pa1, pb1, pa0, pb0);
  } else if (steps > 0) {
    load(pa0, pb0);
    put(pa0, pb0, 0);
    put(pa0, pb0, 1);
    lb.mend(pb0);
    arrived();
    fetch(pa0, pb0, 0);
    load(pa1, pb1);
  }
  for (int pair = steps / 2; pair > 0; --pair) {
    step(pa0, pb0, pa1, pb1);
    step(pa1, pb1, pa0, pb0);
  }

  arrived();   // the last reads; and the loads of nothing that write zeros
  write_out<S, BM, BN, WM, WN>(g, acc, m0, n0, pb0, pb1, pa0, pa1);
}

// Whether a kernel takes the sums of a along: where its registers have room.
constexpr bool sums_along(int alay, int bm) { return alay == kCol && bm == 64; }

// For products of few or ragged tiles, which wait for memory: every operand goes through registers, kRing
// steps of it on their way, so that any alignment does and a short sum is all loaded at once.  1247 x 442 x 1000
// 9.8 us (23.8 with one step on its way), 1 x 4096 x 16384 31 us, 4.3 TB/s of weights; 9001 x 5001 x 5003 in tiles of
// 256 x 256 530 us, 0.85 PFLOP/s (from checkpoints 28 and 16 bytes a lane are spilled).  Bound by what L2 hands out in
// 64 x 64 (11 TB/s).  128 x 128 through registers is not among the shapes: of twenty sizes in three layouts it was more than 6 %
// faster than both others at one (4099 x 4097 x 1027 84 us against 94, its input gradient 87 against 96), 128 x 64 at none;
// eight steps on their way are 5 to 10 % slower.
template <int TYPE, int ALAY, int BLAY, int BM, int BN, int WM, int WN, int kRing, int HELD, bool NARROW>
__global__ __launch_bounds__(WM* WN* kWave, 2) void linear_ring_kernel(LinearArgs g) {
  constexpr int kThreads = WM * WN * kWave;
  constexpr int S = 32, TM = BM / WM / S, TN = BN / WN / S;
  __shared__ __attribute__((aligned(1024))) uint8_t a0[BM * kRowBytes], a1[BM * kRowBytes], b0[BN * kRowBytes], b1[BN * kRowBytes];
  const TileAt at = tile_of<BM, BN>(g);
  const int begin = blockIdx.y * g.split_k, end = part_end(g.k, begin, g.split_k);
  using LoadA = RegisterLoader<ALAY, BM, kThreads, TYPE, TYPE, NARROW>;
  using LoadB = RegisterLoader<BLAY, BN, kThreads, TYPE, HELD, NARROW>;
  const LoadA la(g.a, at.m0, g.m, end);
  const LoadB lb(g.b, at.n0, g.n, end);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  const Reader<S, ALAY, BM, TM> ra(wm);
  const Reader<S, BLAY, BN, TN> rb(wn);

  typename Sums<S>::type acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) clear(acc[i][j]);

  typename LoadA::Set sa[kRing];
  typename LoadB::Set sb[kRing];
  Lds *const pa[2] = {(Lds*)a0, (Lds*)a1}, *const pb[2] = {(Lds*)b0, (Lds*)b1};
  // Beyond the last step it is loaded again: without a branch the compiler knows how many loads are under
  // way, and waits for one step's only.
  const int last = begin + (end - begin - 1) / kStepK * kStepK;
  const auto load = [&](int i, int k) {
    la.load(sa[i], min(k, last));
    lb.load(sb[i], min(k, last));
  };
  if (begin < end) {
#pragma unroll
    for (int i = 0; i < kRing; ++i) load(i, begin + i * kStepK);
  }
  // Two buffers and a barrier a step: what is put into one was last read before the barrier in between.
  const auto put = [&](int i, int k) {
    la.put(sa[i], k, pa[i & 1]);
    lb.put(sb[i], k, pb[i & 1]);
  };
  // Sums of a over k, by products with ones: in the first column of tiles, of the waves at its start.
  constexpr bool kSums = sums_along(ALAY, BM);
  const bool summing = kSums && g.sums && at.n0 == 0 && wn == 0;
  const uint16_t one = TYPE == MOC_BF16 ? 0x3F80 : 0x3C00;
  const s16x8 ones = {(short)one, (short)one, (short)one, (short)one, (short)one, (short)one, (short)one, (short)one};
  typename Sums<S>::type sums[kSums ? TM : 1];
#pragma unroll
  for (auto& x : sums) clear(x);
  const auto multiply = [&](int i) {
    constexpr int kParts = decltype(ra)::kParts;
    s16x8 fa[kParts][TM];
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
      s16x8 fb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = rb.read(pb[i & 1], j, s);
#pragma unroll
      for (int c = 0; c < TM; ++c) fa[s][c] = ra.read(pa[i & 1], c, s);
#pragma unroll
      for (int c = 0; c < TM; ++c)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[c][j] = mfma<TYPE>(fb[j], fa[s][c], acc[c][j]);
    }
    if constexpr (kSums) {
      if (summing) {
#pragma unroll
        for (int s = 0; s < kParts; ++s)
#pragma unroll
          for (int c = 0; c < TM; ++c) sums[c] = mfma<TYPE>(ones, fa[s][c], sums[c]);
      }
    }
  };
  // A step is put while the one before is multiplied.
  const auto step = [&](int i, int k, bool more) {
    const int next = (i + 1) % kRing;
    if (more) {
      put(next, k + kStepK);
      load(next, k + (kRing + 1) * kStepK);
    }
    multiply(i);
    __syncthreads();   // waits for what was put, not for loads
  };
  int k = begin;
  if (begin < end) {
    put(0, begin);
    load(0, begin + kRing * kStepK);
    __syncthreads();
  }
  for (; k + kRing * kStepK < end; k += kRing * kStepK) {
#pragma unroll
    for (int i = 0; i < kRing; ++i) step(i, k + i * kStepK, true);
  }
#pragma unroll
  for (int i = 0; i < kRing; ++i) {
    if (k + i * kStepK >= end) break;
    step(i, k + i * kStepK, k + (i + 1) * kStepK < end);
  }
  if constexpr (kSums) {
    const int lane = threadIdx.x & (kWave - 1);
    if (summing && lane < S) {   // a lane has one m, every n alike
      float* const to = g.splits > 1 ? g.partial + (int64_t)g.splits * g.m * g.partial_stride + (int64_t)blockIdx.y * g.m : g.sums;
#pragma unroll
      for (int c = 0; c < TM; ++c) {
        const int m = at.m0 + wm + S * c + lane;
        if (m < g.m) to[m] = sums[c][0];
      }
    }
  }
  write_out<S, BM, BN, WM, WN>(g, acc, at.m0, at.n0, pb[0], pb[1], pa[0], pa[1]);
}

// The sum of the splits, in their order, and the epilogue; a thread has a run, a quad a block.
__global__ __launch_bounds__(256) void linear_join_kernel(LinearArgs g) {
  const Epilogue& e = g.e;
  const int runs = (int)(g.partial_stride / kRun);
  const int64_t total = (int64_t)g.m * runs, i = block_of() * 256 + threadIdx.x;
  if (i >= total) {   // whole quads
    const int64_t m = i - total;
    if (g.sums && m < g.m) {
      const float* const from = g.partial + (int64_t)g.splits * g.m * g.partial_stride + m;
      float sum = 0.0f;
      for (int s = 0; s < g.splits; ++s) sum += from[(int64_t)s * g.m];
      g.sums[m] = sum;
    }
    return;
  }
  const int64_t row = i / runs;
  const int col = (int)(i - row * runs) * kRun, n = g.n - col;
  float v[kRun] = {};
  const float* from = g.partial + row * g.partial_stride + col;
  for (int s = 0; s < g.splits; ++s, from += g.m * g.partial_stride) {
    float p[kRun];
    load_run<MOC_F32>(from, 0, kRun, p);
#pragma unroll
    for (int r = 0; r < kRun; ++r) v[r] += p[r];
  }
  float bias[kRun] = {};
  if (e.bias && n > 0) load_any(e.bias_type, e.bias, col, n, bias);
  finish_sum(e, row, col, n, bias, load_extra(e, row, col, n), v);
}

// ---- dispatch -----------------------------------------------------------------------------------

// The kernels: linear_kernel (operands straight into LDS) and linear_ring_kernel (through registers).
enum Shape { kDirect128, kDirect256, kRing64, kRing256, kRingNarrow };
struct ShapeSize {
  int tile, threads;
};
constexpr ShapeSize kShapes[] = {{128, 256}, {256, 512}, {64, 256}, {256, 512}, {64, 256}};

// How a product is cut up.
struct LinearPlan {
  Shape shape;
  int tiles_m, tiles_n, splits, split_k;
  int64_t partial_stride, work_bytes;
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Microseconds that a product takes in tiles of a shape with k cut into `splits`, as measured over 30 sizes from 1 x 1000 x
// 1000 to 16384 x 8192 x 2048 in all three layouts (`cols`: how many operands lie in columns).  The smallest k of a weight
// gradient among them is 442, and the output's bytes are not counted: of few rows, whose gradient is bound by what it writes,
// the choice is not measured (8 rows, 8192 x 8192: 82 us in 256 x 256, 3.3 TB/s written).  A step of a workgroup of
// 64 x 64 takes 0.27 us and 0.1 more for an operand in columns, waiting for memory, or 0.25 (0.36 of ragged rows) for each
// of those that share a compute unit; of 128 x 128 0.65 (two in columns: 0.95) and 0.7 (1.0); 256 x 256 have a unit to
// themselves, 1.85 (2.0), through registers 2.2 (2.8).  Cutting k costs a launch and the sums, written and read.
inline double linear_cost(Shape shape, int64_t m, int64_t n, int64_t k, int cols, bool ragged, int64_t splits, int units) {
  const double groups = (double)(ceil_div(m, kShapes[shape].tile) * ceil_div(n, kShapes[shape].tile) * splits) / units;
  const double steps = (double)ceil_div(ceil_div(k, kStepK), splits), rounds = groups > (int64_t)groups ? (double)((int64_t)groups + 1) : groups;
  const bool columns = cols == 2;
  double at = 0.0;
  switch (shape) {
    case kDirect128: at = steps * std::max(columns ? 0.95 : 0.65, (columns ? 1.0 : 0.7) * groups); break;
    case kDirect256: at = steps * rounds * (columns ? 2.0 : 1.85); break;
    case kRing256: at = steps * rounds * (columns ? 2.8 : 2.2); break;
    default: at = steps * std::max(0.27 + 0.1 * cols, (ragged ? 0.36 : 0.25) * groups); break;
  }
  at = std::max(at, ((double)m * k + (double)n * k) * 2 / 5.5e6);   // memory
  return at + (splits > 1 ? 5.0 + (double)splits * m * n * 8 / 4e6 : 0.0);
}

inline LinearPlan linear_plan(int64_t m, int64_t n, int64_t k, int cols, Loading how, int units) {
  LinearPlan p = {};
  const int64_t steps = ceil_div(k, kStepK);
  double best = 0.0;
  p.splits = 0;
  for (const Shape shape : {kDirect256, kDirect128, kRing256, kRing64, kRingNarrow}) {
    if ((shape == kRingNarrow) != (how == kNarrow) || (shape <= kDirect256 && how != kDirect) || (shape == kRing256 && how == kDirect)) continue;
    for (int64_t splits = 1; splits <= 32 && (splits == 1 || steps / splits >= 4); splits += splits < 4 ? 1 : splits / 2) {
      const double cost = linear_cost(shape, m, n, k, cols, how != kDirect, splits, units);
      if (p.splits && cost >= best) continue;
      best = cost;
      p.shape = shape;
      p.splits = (int)splits;
    }
  }
  p.tiles_m = (int)ceil_div(m, kShapes[p.shape].tile);
  p.tiles_n = (int)ceil_div(n, kShapes[p.shape].tile);
  const int64_t each = ceil_div(steps, p.splits);
  p.splits = (int)(steps ? ceil_div(steps, each) : 1);
  p.split_k = (int)(each * kStepK);
  p.partial_stride = ceil_div(n, MOC_BLOCK) * MOC_BLOCK;
  p.work_bytes = p.splits > 1 ? p.splits * m * (p.partial_stride + 1) * (int64_t)sizeof(float) : 0;
  return p;
}

// Whether an operand of 16-bit values can go straight into LDS, `along` values of it in a row.
inline bool direct_ok(const moc_matrix* x, int64_t along) { return aligned_to(x->data, 16) && x->stride % 8 == 0 && along % 8 == 0; }

// Whether a checkpoint can take KeptLoader.
inline bool kept_direct_ok(const moc_matrix* x, int64_t along) { return aligned_to(x->data, 16) && x->stride % 16 == 0 && along % 16 == 0; }

// How operands go to LDS, whose rows have `along_a` and `along_b` values.
inline Loading loading_of(bool direct, int64_t along_a, int64_t along_b) { return along_a < kRun || along_b < kRun ? kNarrow : direct ? kDirect : kThroughRegisters; }

inline Operand operand_of(const moc_matrix* x) { return Operand{x->data, x->scales, x->stride, x->scale_stride}; }

inline void set_out(Epilogue& e, const moc_matrix* out) {
  e.out = out->data;
  e.out_type = out->type;
  e.out_stride = out->stride;
}

// Stretches of rows that the bias's gradient is summed over: two workgroups a compute unit, at least 64
// rows each (their sums are written and read again).
inline int64_t moc_bias_stretches(int64_t rows, int64_t cout, int units) {
  const int64_t across = ceil_div(cout, 512), wanted = 2 * (int64_t)units / across, most = rows / 64;
  const int64_t n = wanted < most ? wanted : most;
  return n < 1 ? 1 : n;
}

using LinearKernel = void (*)(LinearArgs);

template <int TYPE, int ALAY, int BLAY, int HELD>
LinearKernel pick_linear(Shape shape) {
  switch (shape) {
    case kDirect128: return linear_kernel<TYPE, ALAY, BLAY, 128, 128, 2, 2, HELD>;
    case kDirect256: return linear_kernel<TYPE, ALAY, BLAY, 256, 256, 2, 4, HELD>;
    case kRing64: return linear_ring_kernel<TYPE, ALAY, BLAY, 64, 64, 2, 2, 4, HELD, false>;
    case kRing256: return linear_ring_kernel<TYPE, ALAY, BLAY, 256, 256, 2, 4, 2, HELD, false>;
    case kRingNarrow: return linear_ring_kernel<TYPE, ALAY, BLAY, 64, 64, 2, 2, 4, HELD, true>;
  }
  return nullptr;
}

// Cuts the product up, as far as its workspace and a launch go: `g` has the operands, sizes and epilogue.  g.sums is set
// to null where the kernel does not take them.
template <int ALAY, int BLAY>
int cut_linear(LinearArgs& g, Loading how, int units, void* work, int64_t work_bytes, LinearPlan& p) {
  p = linear_plan(g.m, g.n, g.k, (ALAY == kCol) + (BLAY == kCol), how, units);
  if (p.work_bytes > 0 && (!work || !aligned_to(work, 16) || work_bytes < p.work_bytes)) return MOC_EINVAL;
  if ((int64_t)p.tiles_m * p.tiles_n > (1 << 22)) return MOC_EOVERFLOW;   // a launch's threads
  g.tiles_m = p.tiles_m;
  g.tiles_n = p.tiles_n;
  g.splits = p.splits;
  g.split_k = p.split_k;
  g.partial = static_cast<float*>(work);
  g.partial_stride = p.partial_stride;
  if (kShapes[p.shape].tile != 64) g.sums = nullptr;
  return MOC_OK;
}

// Queues what cut_linear has cut up; held: b's type.
template <int ALAY, int BLAY, bool KEPT>
int queue_linear(const LinearArgs& g, const LinearPlan& p, int type, int held, void* hip_stream) {
  LinearKernel kern = nullptr;
  if constexpr (KEPT) {
    if (type == MOC_BF16) {
      kern = held == MOC_E4M3 ? pick_linear<MOC_BF16, ALAY, BLAY, MOC_E4M3>(p.shape)
             : held == MOC_I8 ? pick_linear<MOC_BF16, ALAY, BLAY, MOC_I8>(p.shape)
                              : pick_linear<MOC_BF16, ALAY, BLAY, MOC_BF16>(p.shape);
    } else {
      kern = held == MOC_E4M3 ? pick_linear<MOC_F16, ALAY, BLAY, MOC_E4M3>(p.shape)
             : held == MOC_I8 ? pick_linear<MOC_F16, ALAY, BLAY, MOC_I8>(p.shape)
                              : pick_linear<MOC_F16, ALAY, BLAY, MOC_F16>(p.shape);
    }
  } else {
    kern = type == MOC_BF16 ? pick_linear<MOC_BF16, ALAY, BLAY, MOC_BF16>(p.shape) : pick_linear<MOC_F16, ALAY, BLAY, MOC_F16>(p.shape);
  }
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  hipLaunchKernelGGL(kern, dim3((unsigned)(p.tiles_m * p.tiles_n), (unsigned)p.splits), dim3(kShapes[p.shape].threads), 0, stream, g);
  MOC_HIP(hipGetLastError());
  if (p.splits > 1) {
    hipLaunchKernelGGL(linear_join_kernel, grid_of(ceil_div(g.m * (p.partial_stride / kRun) + (g.sums ? g.m : 0), 256)), dim3(256), 0, stream, g);
    MOC_HIP(hipGetLastError());
  }
  return MOC_OK;
}

}  // namespace
