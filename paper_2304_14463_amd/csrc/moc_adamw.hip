// AdamW over many tensors at once, with moments in 32 bits or in 8, and what moments stand for.
//
// One pass over a tensor's values, bound by memory: 28 bytes a value with moments and gradients in 32 bits, 14 to 16 with
// moments in 8.  A launch takes up to kTensors tensors, whose descriptors travel in its arguments: nothing is copied to
// the device first, and a captured launch keeps them.
#include "moc_training.h"

namespace {

constexpr int kThreads = 256, kChunk = kThreads * kRun;   // values of a workgroup
constexpr int kTensors = 40;                              // of a launch: its arguments have to stay below 4 KB

struct Entry {
  void *param, *m, *v, *copy;
  const void* grad;
  uint8_t *m_scales, *v_scales;
  int64_t count;
  uint32_t number;            // place in the caller's list
  float decay;
  uint8_t param_type, grad_type, copy_type, whole;   // whole: of 8 bits
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

template <bool SECOND>
__device__ __forceinline__ void moment_values(uint2 c, uint8_t scale, float (&x)[kRun]) {
  if constexpr (!SECOND) {
    decode_run<MOC_E4M3>(c, scale_of(scale), x);
  } else {
    // a code is the top of a float whose exponents are 104 lower
    const uint32_t w[2] = {c.x, c.y};
    const int up = (int)scale - 127 + 104;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = __builtin_ldexpf(bits_float((w[h] >> (8 * i) & 0xFF) << 20), up);
      if ((((~w[h]) - 0x01010101u) & w[h] & 0x80808080u) != 0) {   // a code is NaN's
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if ((w[h] >> (8 * i) & 0xFF) == 0xFF) x[4 * h + i] = bits_float(0x7FC00000u);
      }
    }
  }
}

// A run's codes and its block's scale; all four lanes of a quad come here together, those beyond the tensor with zeros.
// The distance from the lower code is what lies below a code's last bit in the scaled value's 32: random bits added there
// carry into the code.  Below the smallest normal code, that code's value is added first, which makes it so there, too.
template <bool SECOND>
__device__ __forceinline__ uint2 moment_codes(const float (&x)[kRun], const uint32_t (&random)[kRun], uint8_t& scale) {
  constexpr float kMost = 1.875f * 0x1p127f;
  float peak;
  const bool special = run_peak(x, kMost, peak);
  const int k = scale_exp<MOC_E4M3>(quad_max(peak));
  scale = (uint8_t)(k + 127);
  const float inv = bits_float((uint32_t)(127 - k) << 23), first = SECOND ? 0x1p-22f : 0x1p-6f;
  constexpr uint32_t kBase = (uint32_t)(first_exp(SECOND) + 127) << 3;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    const float mag = __builtin_fabsf(x[i]), q = (special ? fminf(mag, kMost) : mag) * inv;
    const bool small = q < first;
    const uint32_t bits = float_bits(small ? q + first : q) + ((SECOND ? random[i] >> 16 : random[i] & 0xFFFF) << 4 | 8);
    uint32_t c = (bits >> 20) - (small ? kBase : kBase - 8);
    if (SECOND) c = x[i] > 0.0f ? max(c, 1u) : c;
    if (special) c = mag < kInf ? c : SECOND ? 0xFF : 0x7F;
    if (!SECOND) c |= float_bits(x[i]) >> 24 & (special && !(mag < kInf) ? 0 : 0x80);
    w[i >> 2] |= c << (8 * (i & 3));
  }
  return uint2{w[0], w[1]};
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
  const uint32_t block = (uint32_t)block_of();
  const int at = entry_of(g.first, block);
  const Entry& e = g.entry[at];
  const int64_t place = (int64_t)(block - g.first[at]) * kChunk + threadIdx.x * kRun, left = e.count - place;
  const int n = left < kRun ? (int)left : kRun;
  Factors f = g.f;
  uint32_t step = g.step_low;
  if (g.lr_at) f.lr = *g.lr_at;
  if (g.grad_scale_at) f.grad_scale = *g.grad_scale_at;
  if (g.lr_at || g.step_at) {
    const int64_t t = g.step_at ? *g.step_at : (int64_t)step;
    if (g.step_at) {
      step = (uint32_t)t;
      f.root = 1.0f / __builtin_sqrtf(-expm1f((float)t * g.log2));
    }
    f.away = g.step_at ? f.lr / -expm1f((float)t * g.log1) : f.lr * f.away;
  }
  if (!EIGHT && n <= 0) return;
  float p[kRun], d[kRun], m[kRun], v[kRun];
  load_any(e.param_type, e.param, place, n, p);
  load_any(e.grad_type, e.grad, place, n, d);
  if constexpr (EIGHT) {
    uint8_t ms = 0, vs = 0;
    if (n > 0) {
      ms = e.m_scales[place / MOC_BLOCK];
      vs = e.v_scales[place / MOC_BLOCK];
    }
    moment_values<false>(load_codes(static_cast<const uint8_t*>(e.m) + place, n), ms, m);
    moment_values<true>(load_codes(static_cast<const uint8_t*>(e.v) + place, n), vs, v);
  } else {
    load_run<MOC_F32>(e.m, place, n, m);
    load_run<MOC_F32>(e.v, place, n, v);
  }
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    d[i] *= f.grad_scale;
    m[i] = __builtin_fmaf(g.beta1, m[i], g.rest1 * d[i]);
    v[i] = __builtin_fmaf(g.beta2, v[i], g.rest2 * (d[i] * d[i]));
    const float away = f.away * m[i] * __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_sqrtf(v[i]), f.root, g.eps));
    p[i] -= __builtin_fmaf(f.lr * e.decay, p[i], away);
  }
  if constexpr (EIGHT) {
    if (n < kRun) {
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        m[i] = i < n ? m[i] : 0.0f;
        v[i] = i < n ? v[i] : 0.0f;
      }
    }
    uint32_t random[kRun];
    const uint32_t key = mix((uint32_t)(place >> 32) ^ mix(e.number ^ mix(step ^ g.seed_key)));
#pragma unroll
    for (int i = 0; i < kRun; ++i) random[i] = mix((uint32_t)(place + i) ^ key);
    uint8_t ms, vs;
    const uint2 mc = moment_codes<false>(m, random, ms), vc = moment_codes<true>(v, random, vs);
    if (n <= 0) return;
    store_codes(static_cast<uint8_t*>(e.m) + place, n, mc);
    store_codes(static_cast<uint8_t*>(e.v) + place, n, vc);
    if ((place & (MOC_BLOCK - 1)) == 0) {
      e.m_scales[place / MOC_BLOCK] = ms;
      e.v_scales[place / MOC_BLOCK] = vs;
    }
  } else {
    store_run<MOC_F32>(e.m, place, n, m);
    store_run<MOC_F32>(e.v, place, n, v);
  }
  store_any(e.param_type, e.param, place, n, p);
  if (e.copy) store_any(e.copy_type, e.copy, place, n, p);
}

__global__ __launch_bounds__(kThreads) void moments_read_kernel(AdamwArgs g) {
  const uint32_t block = (uint32_t)block_of();
  const int at = entry_of(g.first, block);
  const Entry& e = g.entry[at];
  const int64_t place = (int64_t)(block - g.first[at]) * kChunk + threadIdx.x * kRun, left = e.count - place;
  const int n = left < kRun ? (int)left : kRun;
  if (n <= 0) return;
  float m[kRun], v[kRun];
  if (e.m_scales) {
    moment_values<false>(load_codes(static_cast<const uint8_t*>(e.m) + place, n), e.m_scales[place / MOC_BLOCK], m);
    moment_values<true>(load_codes(static_cast<const uint8_t*>(e.v) + place, n), e.v_scales[place / MOC_BLOCK], v);
  } else {
    load_run<MOC_F32>(e.m, place, n, m);
    load_run<MOC_F32>(e.v, place, n, v);
  }
  store_any(e.param_type, e.param, place, n, m);
  store_any(e.param_type, e.copy, place, n, v);
}

using Kernel = void (*)(AdamwArgs);

// The tensors of one kind of moments, kTensors a launch; entry(i, e) fills in e and says whether tensor i is one of them.
template <class Fill>
int queue(Kernel kern, AdamwArgs& g, int64_t tensors, hipStream_t stream, const Fill& fill) {
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
    const int64_t more = (e.count + kChunk - 1) / kChunk;
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
    const int rc = queue(eight ? adamw_kernel<true> : adamw_kernel<false>, g, tensors, static_cast<hipStream_t>(hip_stream), [&](int64_t i, Entry& e) {
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
  return queue(moments_read_kernel, g, tensors, static_cast<hipStream_t>(hip_stream), [&](int64_t i, Entry& e) {
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
