// AdamW over many tensors at once, with moments in 32 bits or in 8, and what moments stand for.
//
// One pass over a tensor's values, bound by memory: 28 bytes a value with moments and gradients in 32 bits, 14 to 16 with
// moments in 8: the kernel over 150 M parameters in 32 bits with copies 834 us (5.4 TB/s), 537 M with moments in 8 bits 1660 us (5.2), their reading
// back 626.  A launch takes up to kTensors tensors, whose descriptors travel in its arguments: nothing is copied to
// the device first, and a captured launch keeps them.
#include <type_traits>

#include "moc_training.h"

namespace {

// A thread takes four values at a time, so that neighbouring lanes load and store next to each other whatever the type is,
// and `turns` times four, all of them on their way before the first is used: 12 blocks of 1247 in 32 bits 836 us with one
// turn and 891 with two, 16 blocks of 2048 in 8 bits 2630 with one, 2381 with two, 2348 with four.
constexpr int kThreads = 256, kFew = 4, kTurn = kThreads * kFew;
constexpr int turns(bool eight) { return eight ? 2 : 1; }
constexpr int kReadTurns = 4;
constexpr int chunk(bool eight) { return kTurn * turns(eight); }   // values of a workgroup
using Four = float[kFew];
constexpr int kTensors = 40;                              // of a launch: its arguments have to stay below 4 KB

struct Entry {
  void *param, *m, *v, *copy;
  const void* grad;
  uint8_t *m_scales, *v_scales;
  int64_t count;
  uint32_t number;            // place in the caller's list
  float decay;
  uint8_t param_type, grad_type, copy_type;
};
struct Factors {
  float lr, away, root, grad_scale;   // away = lr / (1 - beta1^step), root = 1 / sqrt(1 - beta2^step)
};
struct AdamwArgs {
  uint32_t first[kTensors];   // the workgroup that a tensor begins with; ~0 behind the last
  Entry entry[kTensors];
  Factors f;
  float beta1, beta2, rest1, rest2, eps;   // rest = 1 - beta
  float log1, log2;                        // natural logarithms of the betas
  uint32_t step_low, seed_key;             // seed_key: the seed mixed
  const float *lr_at, *grad_scale_at;
  const int64_t* step_at;
};
static_assert(sizeof(AdamwArgs) <= 4096);

// Two odd factors out of 150 pairs drawn at random: the pair by which a bit of the argument, flipped, most evenly flips each bit of
// the result (0.9 points off one in two at the worst of all pairs of bits, over 200000 arguments).
constexpr uint32_t mix(uint32_t h) {
  h ^= h >> 16;
  h *= 0xF704BB15u;
  h ^= h >> 15;
  h *= 0x371E2E67u;
  return h ^ h >> 16;
}

// ---- moments in 8 bits --------------------------------------------------------------------------

// Exponent of the smallest normal code: of m as in MOC_E4M3, of v, which has no sign, 16 lower.
constexpr int first_exp(bool second) { return second ? -22 : -6; }

// How many of a thread's four values there are.  (With `left` and 0 to max(), the compiler loses the case of all four.)
__device__ __forceinline__ int there(int64_t left) { return left >= kFew ? kFew : left > 0 ? (int)left : 0; }

// Four values from a place on.  A tensor's last ones are loaded whole, from within it, and moved down: without a branch, so
// that all of a thread's loads are under way at once.  Threads beyond it have its last four.
struct Raw4 {
  u32x4 a;
};
template <int BYTES>
__device__ __forceinline__ Raw4 load_four(const void* p, int64_t place, int64_t count) {
  const char* const at = static_cast<const char*>(p);
  Raw4 r = {};
  if (count >= kFew) {
    const char* const from = at + min(place, count - kFew) * BYTES;
    if constexpr (BYTES == 4) {
      __builtin_memcpy(&r.a, from, 16);
    } else if constexpr (BYTES == 2) {
      uint2 w;
      __builtin_memcpy(&w, from, 8);
      r.a[0] = w.x;
      r.a[1] = w.y;
    } else {
      uint32_t w;
      __builtin_memcpy(&w, from, 4);
      r.a[0] = w;
    }
  } else if (place == 0) {   // a tensor of less than four
    for (int i = 0; i < (int)count; ++i) {
      uint32_t w = 0;
      if constexpr (BYTES == 4) w = reinterpret_cast<const uint32_t*>(at)[i];
      else if constexpr (BYTES == 2) w = reinterpret_cast<const uint16_t*>(at)[i];
      else w = reinterpret_cast<const uint8_t*>(at)[i];
      const int word = i * BYTES / 4, up = i * BYTES % 4 * 8;
      r.a[0] |= word == 0 ? w << up : 0;
      r.a[1] |= word == 1 ? w << up : 0;
      r.a[2] |= word == 2 ? w << up : 0;
    }
  }
  return r;
}
template <int BYTES>
__device__ __forceinline__ void settle_four(Raw4& r, int64_t place, int64_t count) {
  const int64_t n = count - place;
  if (n >= kFew || n <= 0 || count < kFew) return;
  const int down = kFew - (int)n;
  if constexpr (BYTES == 4) {
    if (down & 1) r.a = u32x4{r.a[1], r.a[2], r.a[3], 0};
    if (down & 2) r.a = u32x4{r.a[2], r.a[3], 0, 0};
  } else if constexpr (BYTES == 2) {
    const uint64_t w = (r.a[0] | (uint64_t)r.a[1] << 32) >> (16 * down);
    r.a[0] = (uint32_t)w;
    r.a[1] = (uint32_t)(w >> 32);
  } else {
    r.a[0] >>= 8 * down;
  }
}
__device__ __forceinline__ Raw4 load_four_any(int type, const void* p, int64_t place, int64_t count) {
  return type == MOC_F32 ? load_four<4>(p, place, count) : load_four<2>(p, place, count);
}
__device__ __forceinline__ void settle_four_any(int type, Raw4& r, int64_t place, int64_t count) {
  if (type == MOC_F32) settle_four<4>(r, place, count);
  else settle_four<2>(r, place, count);
}
__device__ __forceinline__ void values_of_four(int type, const Raw4& r, Four& v) {
#pragma unroll
  for (int i = 0; i < kFew; ++i) {
    const uint16_t h = (uint16_t)(r.a[i >> 1] >> (16 * (i & 1)));
    v[i] = type == MOC_F32 ? bits_float(r.a[i]) : type == MOC_BF16 ? bits_float((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
  }
}
template <class T>
__device__ __forceinline__ void store_four(void* p, int64_t place, int n, const T (&t)[kFew]) {
  T* const at = static_cast<T*>(p) + place;
  if (n >= kFew) {
    __builtin_memcpy(at, t, sizeof t);
  } else {
#pragma unroll
    for (int i = 0; i < kFew - 1; ++i)
      if (i < n) at[i] = t[i];
  }
}
__device__ __forceinline__ void store_four_any(int type, void* p, int64_t place, int n, const Four& v) {
  if (type == MOC_F32) {
    store_four(p, place, n, v);
  } else if (type == MOC_BF16) {
    const __bf16 t[kFew] = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    store_four(p, place, n, t);
  } else {
    const _Float16 t[kFew] = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
    store_four(p, place, n, t);
  }
}

template <bool SECOND>
__device__ __forceinline__ void moment_values(uint32_t c, uint8_t scale, Four& x) {
  if constexpr (!SECOND) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    const float by = scale_of(scale);
    x[0] = lo[0] * by;
    x[1] = lo[1] * by;
    x[2] = hi[0] * by;
    x[3] = hi[1] * by;
  } else {
    // a code is the top of a float whose exponents are 104 lower
    const int up = (int)scale - 127 + 104;
#pragma unroll
    for (int i = 0; i < kFew; ++i) x[i] = __builtin_ldexpf(bits_float((c >> (8 * i) & 0xFF) << 20), up);
    if (((~c - 0x01010101u) & c & 0x80808080u) != 0) {   // a code is NaN's
#pragma unroll
      for (int i = 0; i < kFew; ++i)
        if ((c >> (8 * i) & 0xFF) == 0xFF) x[i] = bits_float(0x7FC00000u);
    }
  }
}

// The maximum over the eight lanes that hold a block's 32 values.
__device__ __forceinline__ float block_max(float a) {
  a = quad_max(a);
  return fmaxf(a, bits_float((uint32_t)__builtin_amdgcn_mov_dpp((int)float_bits(a), 0x141, 0xF, 0xF, true)));   // row_half_mirror
}

// Four values' codes and their block's scale; all eight lanes of a block come here together, those beyond the tensor with zeros.
// The distance from the lower code is what lies below a code's last bit in the scaled value's 32: random bits added there
// carry into the code.  Below the smallest normal code, that code's value is added first, which makes it so there, too.
template <bool SECOND>
__device__ __forceinline__ uint32_t moment_codes(const Four& x, const uint32_t (&random)[kFew], uint8_t& scale) {
  constexpr float kMost = 1.875f * 0x1p127f;
  float peak = 0.0f, odd = 0.0f;
#pragma unroll
  for (int i = 0; i < kFew; ++i) {
    peak = fmaxf(peak, __builtin_fabsf(x[i]));
    odd = __builtin_fmaf(x[i], 0.0f, odd);   // what is not finite times 0 is NaN
  }
  const bool special = odd != odd || peak > kMost;
  if (special) {
    peak = 0.0f;
#pragma unroll
    for (int i = 0; i < kFew; ++i) {
      const float m = __builtin_fabsf(x[i]);
      peak = m < kInf && m > peak ? m : peak;
    }
    peak = fminf(peak, kMost);
  }
  const int k = scale_exp<MOC_E4M3>(block_max(peak));
  scale = (uint8_t)(k + 127);
  const float inv = bits_float((uint32_t)(127 - k) << 23), first = SECOND ? 0x1p-22f : 0x1p-6f;
  constexpr uint32_t kBase = (uint32_t)(first_exp(SECOND) + 127) << 3;
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < kFew; ++i) {
    const float mag = __builtin_fabsf(x[i]), q = (special ? fminf(mag, kMost) : mag) * inv;
    const bool small = q < first;
    const uint32_t bits = float_bits(small ? q + first : q) + ((SECOND ? random[i] >> 16 : random[i] & 0xFFFF) << 4 | 8);
    uint32_t c = (bits >> 20) - (small ? kBase : kBase - 8);
    if (SECOND) c = x[i] > 0.0f ? max(c, 1u) : c;
    if (special) c = mag < kInf ? c : SECOND ? 0xFF : 0x7F;
    if (!SECOND) c |= float_bits(x[i]) >> 24 & (special && !(mag < kInf) ? 0 : 0x80);
    w |= c << (8 * i);
  }
  return w;
}

// ---- kernels ------------------------------------------------------------------------------------

// Which tensor the workgroup is in.
__device__ __forceinline__ int entry_of(const uint32_t* first, uint32_t block) {
  const uint32_t mine = first[min((int)(threadIdx.x % kWave), kTensors - 1)];
  const uint64_t begun = __builtin_amdgcn_ballot_w64(threadIdx.x % kWave < kTensors && mine <= block);
  return __builtin_popcountll(begun) - 1;
}

template <bool EIGHT>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamwArgs g) {
  constexpr int kTurns = turns(EIGHT), kChunk = chunk(EIGHT);
  const uint32_t block = (uint32_t)block_of();
  const int at = entry_of(g.first, block);
  const Entry& e = g.entry[at];
  const int64_t start = (int64_t)(block - g.first[at]) * kChunk + threadIdx.x * kFew;
  const int64_t last = e.count - 1;
  Raw4 wp[kTurns], wd[kTurns], wm[kTurns], wv[kTurns];
  uint8_t ms[kTurns], vs[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int64_t place = start + t * kTurn;
    wp[t] = load_four_any(e.param_type, e.param, place, e.count);
    wd[t] = load_four_any(e.grad_type, e.grad, place, e.count);
    if constexpr (EIGHT) {
      wm[t] = load_four<1>(e.m, place, e.count);
      wv[t] = load_four<1>(e.v, place, e.count);
      ms[t] = e.m_scales[min(place, last) / MOC_BLOCK];
      vs[t] = e.v_scales[min(place, last) / MOC_BLOCK];
    } else {
      wm[t] = load_four<4>(e.m, place, e.count);
      wv[t] = load_four<4>(e.v, place, e.count);
    }
  }
  Factors f = g.f;
  uint32_t step = g.step_low;
  if (g.lr_at) f.lr = *g.lr_at;
  if (g.grad_scale_at) f.grad_scale = *g.grad_scale_at;
  if (g.step_at) {
    const int64_t t = *g.step_at;
    step = (uint32_t)t;
    f.root = 1.0f / __builtin_sqrtf(-expm1f((float)t * g.log2));
    f.away = f.lr / -expm1f((float)t * g.log1);
  } else if (g.lr_at) {
    f.away *= f.lr;
  }
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int64_t place = start + t * kTurn, left = e.count - place;
    const int n = there(left);
    if (!EIGHT && n <= 0) break;
    if (n < kFew) {
      settle_four_any(e.param_type, wp[t], place, e.count);
      settle_four_any(e.grad_type, wd[t], place, e.count);
      settle_four<EIGHT ? 1 : 4>(wm[t], place, e.count);
      settle_four<EIGHT ? 1 : 4>(wv[t], place, e.count);
    }
    Four p, d, m, v;
    values_of_four(e.param_type, wp[t], p);
    values_of_four(e.grad_type, wd[t], d);
    if constexpr (EIGHT) {
      moment_values<false>(wm[t].a[0], ms[t], m);
      moment_values<true>(wv[t].a[0], vs[t], v);
    } else {
      values_of_four(MOC_F32, wm[t], m);
      values_of_four(MOC_F32, wv[t], v);
    }
#pragma unroll
    for (int i = 0; i < kFew; ++i) {
      d[i] *= f.grad_scale;
      m[i] = __builtin_fmaf(g.beta1, m[i], g.rest1 * d[i]);
      v[i] = __builtin_fmaf(g.beta2, v[i], g.rest2 * (d[i] * d[i]));
      const float away = f.away * m[i] * __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_sqrtf(v[i]), f.root, g.eps));
      p[i] -= __builtin_fmaf(f.lr * e.decay, p[i], away);
    }
    if constexpr (EIGHT) {
      if (n < kFew) {
#pragma unroll
        for (int i = 0; i < kFew; ++i) {
          m[i] = i < n ? m[i] : 0.0f;
          v[i] = i < n ? v[i] : 0.0f;
        }
      }
      uint32_t random[kFew];
      const uint32_t key = mix((uint32_t)(place >> 32) ^ mix(e.number ^ mix(step ^ g.seed_key)));
#pragma unroll
      for (int i = 0; i < kFew; ++i) random[i] = mix((uint32_t)(place + i) ^ key);
      uint8_t m_scale, v_scale;
      uint8_t mc[kFew], vc[kFew];
      const uint32_t mw = moment_codes<false>(m, random, m_scale), vw = moment_codes<true>(v, random, v_scale);
      __builtin_memcpy(mc, &mw, 4);
      __builtin_memcpy(vc, &vw, 4);
      if (n <= 0) break;   // from here on no lane of the others' blocks is asked
      store_four(e.m, place, n, mc);
      store_four(e.v, place, n, vc);
      if ((place & (MOC_BLOCK - 1)) == 0) {
        e.m_scales[place / MOC_BLOCK] = m_scale;
        e.v_scales[place / MOC_BLOCK] = v_scale;
      }
    } else {
      store_four(e.m, place, n, m);
      store_four(e.v, place, n, v);
    }
    store_four_any(e.param_type, e.param, place, n, p);
    if (e.copy) store_four_any(e.copy_type, e.copy, place, n, p);
  }
}

__global__ __launch_bounds__(kThreads) void moments_read_kernel(AdamwArgs g) {
  constexpr int kTurns = kReadTurns, kChunk = kTurn * kTurns;
  const uint32_t block = (uint32_t)block_of();
  const int at = entry_of(g.first, block);
  const Entry& e = g.entry[at];
  const int64_t start = (int64_t)(block - g.first[at]) * kChunk + threadIdx.x * kFew;
  Raw4 wm[kTurns], wv[kTurns];
  uint8_t ms[kTurns], vs[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int64_t place = start + t * kTurn;
    if (e.m_scales) {
      wm[t] = load_four<1>(e.m, place, e.count);
      wv[t] = load_four<1>(e.v, place, e.count);
      ms[t] = e.m_scales[min(place, e.count - 1) / MOC_BLOCK];
      vs[t] = e.v_scales[min(place, e.count - 1) / MOC_BLOCK];
    } else {
      wm[t] = load_four<4>(e.m, place, e.count);
      wv[t] = load_four<4>(e.v, place, e.count);
    }
  }
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int64_t place = start + t * kTurn, left = e.count - place;
    const int n = there(left);
    if (n <= 0) break;
    if (n < kFew) {
      if (e.m_scales) {
        settle_four<1>(wm[t], place, e.count);
        settle_four<1>(wv[t], place, e.count);
      } else {
        settle_four<4>(wm[t], place, e.count);
        settle_four<4>(wv[t], place, e.count);
      }
    }
    Four m, v;
    if (e.m_scales) {
      moment_values<false>(wm[t].a[0], ms[t], m);
      moment_values<true>(wv[t].a[0], vs[t], v);
    } else {
      values_of_four(MOC_F32, wm[t], m);
      values_of_four(MOC_F32, wv[t], v);
    }
    store_four_any(e.param_type, e.param, place, n, m);
    store_four_any(e.param_type, e.copy, place, n, v);
  }
}

using Kernel = void (*)(AdamwArgs);

// The tensors of one kind of moments, kTensors a launch, `values` of them a workgroup; fill(i, e) fills in e and says whether tensor i is one of them.
template <class Fill>
int queue(Kernel kern, int values, AdamwArgs& g, int64_t tensors, hipStream_t stream, const Fill& fill) {
  int held = 0;
  int64_t blocks = 0;
  const auto launch = [&]() -> int {
    for (int i = held; i < kTensors; ++i) g.first[i] = ~0u;
    hipLaunchKernelGGL(kern, grid_of(blocks), dim3(kThreads), 0, stream, g);
    MOC_HIP(hipGetLastError());
    held = 0;
    blocks = 0;
    return MOC_OK;
  };
  for (int64_t i = 0; i < tensors; ++i) {
    Entry e = {};
    if (!fill(i, e)) continue;
    const int64_t more = (e.count + values - 1) / values;
    if (held == kTensors || (held > 0 && blocks + more > 0x7FFFFFFF)) {
      const int rc = launch();
      if (rc != MOC_OK) return rc;
    }
    g.first[held] = (uint32_t)blocks;
    g.entry[held++] = e;
    blocks += more;
  }
  return held > 0 ? launch() : MOC_OK;
}

bool moments_ok(const void* m, const void* v, const uint8_t* ms, const uint8_t* vs, int64_t count, int type) {
  if (count < 0 || count > (int64_t)1 << 40 || (type != MOC_F32 && type != MOC_E4M3)) return false;
  if (count == 0) return true;
  if (!m || !v) return false;
  return type == MOC_E4M3 ? ms && vs : aligned_to(m, 4) && aligned_to(v, 4);
}

}  // namespace

extern "C" {

int moc_adamw_step(int64_t tensors, const moc_adamw_tensor* tensor, const moc_adamw_rule* rule, void* hip_stream) {
  if (tensors < 0 || tensors > INT32_MAX || (tensors > 0 && !tensor) || !rule) return MOC_EINVAL;
  const auto finite = [](double x) { return x - x == 0.0; };
  if (!finite((float)rule->lr) || !finite((float)rule->grad_scale) || !finite((float)rule->eps) || !((float)rule->eps >= 0x1p-126f) || rule->step < 1) return MOC_EINVAL;
  if (!(rule->beta1 >= 0.0 && rule->beta1 < 1.0) || !(rule->beta2 >= 0.0 && rule->beta2 < 1.0)) return MOC_EINVAL;
  if (!aligned_to(rule->lr_at, 4) || !aligned_to(rule->grad_scale_at, 4) || !aligned_to(rule->step_at, 8)) return MOC_EINVAL;
  bool kinds[2] = {false, false};
  for (int64_t i = 0; i < tensors; ++i) {
    const moc_adamw_tensor& t = tensor[i];
    if (t.reserved != 0 || !is_value(t.param_type) || !is_value(t.grad_type) || !(t.decay >= 0.0f) || !finite(t.decay)) return MOC_EINVAL;
    if (!moments_ok(t.m, t.v, t.m_scales, t.v_scales, t.count, t.moment_type)) return MOC_EINVAL;
    if (t.copy && t.copy_type != MOC_F16 && t.copy_type != MOC_BF16) return MOC_EINVAL;
    if (t.count == 0) continue;
    if (!t.param || !t.grad || !aligned_to(t.param, type_bytes(t.param_type)) || !aligned_to(t.grad, type_bytes(t.grad_type)) || !aligned_to(t.copy, 2)) return MOC_EINVAL;
    kinds[t.moment_type == MOC_E4M3] = true;
  }
  AdamwArgs g = {};
  const double rest1 = -expm1((double)rule->step * log(rule->beta1)), rest2 = -expm1((double)rule->step * log(rule->beta2));   // 1 where beta is 0
  g.f.lr = (float)rule->lr;
  g.f.away = (float)((rule->lr_at ? 1.0 : rule->lr) / rest1);
  g.f.root = (float)(1.0 / sqrt(rest2));
  g.f.grad_scale = (float)rule->grad_scale;
  g.beta1 = (float)rule->beta1; g.beta2 = (float)rule->beta2;
  g.rest1 = (float)(1.0 - rule->beta1); g.rest2 = (float)(1.0 - rule->beta2);
  g.eps = (float)rule->eps;
  g.log1 = (float)log(rule->beta1); g.log2 = (float)log(rule->beta2);
  g.step_low = (uint32_t)rule->step;
  g.seed_key = mix((uint32_t)(rule->seed >> 32) ^ mix((uint32_t)rule->seed));
  g.lr_at = rule->lr_at; g.grad_scale_at = rule->grad_scale_at; g.step_at = rule->step_at;
  for (const bool eight : {false, true}) {
    if (!kinds[eight]) continue;
    const int rc = queue(eight ? adamw_kernel<true> : adamw_kernel<false>, chunk(eight), g, tensors, static_cast<hipStream_t>(hip_stream), [&](int64_t i, Entry& e) {
      const moc_adamw_tensor& t = tensor[i];
      if (t.count == 0 || (t.moment_type == MOC_E4M3) != eight) return false;
      e.param = t.param; e.grad = t.grad; e.m = t.m; e.v = t.v; e.copy = t.copy;
      e.m_scales = t.m_scales; e.v_scales = t.v_scales;
      e.count = t.count; e.number = (uint32_t)i; e.decay = t.decay;
      e.param_type = (uint8_t)t.param_type; e.grad_type = (uint8_t)t.grad_type; e.copy_type = (uint8_t)t.copy_type;
      return true;
    });
    if (rc != MOC_OK) return rc;
  }
  return MOC_OK;
}

int moc_moments_read(int64_t tensors, const moc_moments_tensor* tensor, void* hip_stream) {
  if (tensors < 0 || tensors > INT32_MAX || (tensors > 0 && !tensor)) return MOC_EINVAL;
  for (int64_t i = 0; i < tensors; ++i) {
    const moc_moments_tensor& t = tensor[i];
    if (!moments_ok(t.m, t.v, t.m_scales, t.v_scales, t.count, t.moment_type) || !is_value(t.value_type)) return MOC_EINVAL;
    if (t.count > 0 && (!t.m_values || !t.v_values || !aligned_to(t.m_values, type_bytes(t.value_type)) || !aligned_to(t.v_values, type_bytes(t.value_type)))) return MOC_EINVAL;
  }
  AdamwArgs g = {};
  return queue(moments_read_kernel, kTurn * kReadTurns, g, tensors, static_cast<hipStream_t>(hip_stream), [&](int64_t i, Entry& e) {
    const moc_moments_tensor& t = tensor[i];
    if (t.count == 0) return false;
    e.m = const_cast<void*>(t.m); e.v = const_cast<void*>(t.v);
    if (t.moment_type == MOC_E4M3) {
      e.m_scales = const_cast<uint8_t*>(t.m_scales);
      e.v_scales = const_cast<uint8_t*>(t.v_scales);
    }
    e.param = t.m_values; e.copy = t.v_values; e.count = t.count;
    e.param_type = (uint8_t)t.value_type;
    return true;
  });
}

}  // extern "C"
