// Log probabilities of given tokens with the entropy and the most likely alternatives, and their gradient.
//
// Forward: one pass over a row.  A lane holds the largest logit m it has met, s = sum of e and w = sum of e t with
// t = scale (x - m) / ln 2 and e = 2^t; a larger one scales both, s' = f s and w' = f (w + d s) with d = scale (m - m') / ln 2 and
// f = 2^d, and so do lanes that are joined.  Then log sum exp = scale m + ln s and the entropy ln s - ln 2 w / s.
// The alternatives: a wave keeps its 64 best, one a lane in falling order, as whole numbers that order by value and
// then by place; a value above the last one wanted moves those below it one lane on.
// Backward: a pass over the logits and their gradient.
#include "moc_training.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kMostTop = kWave;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFar = -200.0f;   // 2^kFar is 0: a value further below the largest adds nothing, an infinite one neither

struct LogprobArgs {
  const void* logits;
  int64_t stride;
  int64_t rows;
  int vocab, top, token_bytes;
  float scale, scale2;   // scale2 = scale / ln 2
  const void* tokens;
  float *logp, *lse, *entropy, *top_logp;
  int64_t* top_tokens;
  // backward
  const float *lse_of, *entropy_of, *dlogp, *dentropy;
  void* out;
  int64_t out_stride;
  int out_type;
};

// To a number or NaN where one of the two is NaN.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ int64_t token_of(const LogprobArgs& g, int64_t row) {
  return g.token_bytes == 8 ? static_cast<const int64_t*>(g.tokens)[row] : static_cast<const int32_t*>(g.tokens)[row];
}

// ---- sums ---------------------------------------------------------------------------------------

struct Sums {
  float m;      // the largest logit
  float at;     // scale2 * m, or what anchor() makes of it: terms are 2^(scale2 x - at)
  float s, w;
};

// Logits of the type's lowest value (a mask's) times scale2 pass float32's range; where nothing else has been met, `at`
// stays above them and they count as nothing.  A row of nothing else is taken again by row_again().
__device__ __forceinline__ float anchor(float m, float scale2) { return fmaxf(m * scale2, -0x1p127f); }

// Terms relative to `to` instead of x.at.
__device__ __forceinline__ void move_to(Sums& x, float to) {
  if (x.s == 0.0f) {   // and w
    x.at = to;
    return;
  }
  const float d = x.at - to, f = exp2_of(d);
  x.w = f * __builtin_fmaf(d, x.s, x.w);
  x.s *= f;
  x.at = to;
}

template <int N>
__device__ __forceinline__ void add_values(Sums& x, const float (&v)[N], float scale2) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
  if (m > x.m) {
    x.m = m;
    move_to(x, anchor(m, scale2));
  }
  float s[2] = {0.0f, 0.0f}, w[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float t = larger(__builtin_fmaf(v[i], scale2, -x.at), kFar), e = exp2_of(t);
    s[i & 1] += e;
    w[i & 1] = __builtin_fmaf(e, t, w[i & 1]);
  }
  x.s += s[0] + s[1];
  x.w += w[0] + w[1];
}

__device__ __forceinline__ void join(Sums& a, Sums b) {
  // one that holds nothing has no say in where the terms are relative to
  const float to = a.s == 0.0f ? b.at : b.s == 0.0f ? a.at : fmaxf(a.at, b.at);
  move_to(a, to);
  move_to(b, to);
  a.m = fmaxf(a.m, b.m);
  a.s += b.s;
  a.w += b.w;
}

__device__ __forceinline__ Sums from_lane(const Sums& x, int offset) {
  return Sums{__shfl_xor(x.m, offset), __shfl_xor(x.at, offset), __shfl_xor(x.s, offset), __shfl_xor(x.w, offset)};
}

// ---- alternatives -------------------------------------------------------------------------------

using Key = uint64_t;   // a logit's order in the upper half, the complement of its place in the lower; 0: none
__device__ __forceinline__ Key key_of(float x, uint32_t place) {
  const uint32_t b = float_bits(x + 0.0f);   // -0 is 0
  return (Key)((b ^ (uint32_t)((int32_t)b >> 31 & 0x7FFFFFFF)) ^ 0x80000000u) << 32 | (uint32_t)~place;
}
__device__ __forceinline__ float logit_of(Key k) {
  const uint32_t b = (uint32_t)(k >> 32) ^ 0x80000000u;
  return bits_float(b ^ (uint32_t)((int32_t)b >> 31 & 0x7FFFFFFF));
}
__device__ __forceinline__ uint32_t place_of(Key k) { return ~(uint32_t)k; }

__device__ __forceinline__ Key lane_key(Key k, int lane) {
  return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}
// The key of the lane before.
__device__ __forceinline__ Key key_before(Key k) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)k, 0x138, 0xF, 0xF, false), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(k >> 32), 0x138, 0xF, 0xF, false);
  return (Key)hi << 32 | lo;
}

struct Best {
  Key key = 0;            // of this lane; falling over the wave
  Key last = 0;           // the last one wanted
  float above = -kInf;    // its logit
  bool full = false;      // as many as are wanted are there

  __device__ __forceinline__ void insert(Key c, int lane, int top) {   // c: the same in all lanes
    const int before = __builtin_popcountll(__builtin_amdgcn_ballot_w64(key > c));
    const Key moved = key_before(key);
    key = lane < before ? key : lane == before ? c : moved;
    last = lane_key(key, top - 1);
  }
  // The run of each lane, from column `col` on, `n` of it in the row.  `over` lets values through: above it, or at it too
  // where `with`.
  __device__ __forceinline__ void offer(const float (&v)[kRun], int col, int n, float over, bool with, int lane, int top) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      uint64_t some = __builtin_amdgcn_ballot_w64(i < n && (v[i] > over || (with && v[i] == over)));
      if (some == 0) continue;
      const Key k = key_of(v[i], (uint32_t)(col + i));
      while (some != 0) {
        const int from = __builtin_ctzll(some);
        some &= some - 1;
        const Key c = lane_key(k, from);
        if (c > last) insert(c, lane, top);
      }
    }
  }
  __device__ __forceinline__ void settle() {
    full = last != 0;
    above = full ? logit_of(last) : -kInf;
  }
};

// The value that `top` lanes reach with their x: one that many values of a first batch are not below.
__device__ __forceinline__ float reached(float x, int lane, int top) {
  int before = 0;
#pragma unroll
  for (int j = 0; j < kWave; ++j) {
    const float other = bits_float((uint32_t)__builtin_amdgcn_readlane((int)float_bits(x), j));
    before += other > x || (other == x && j < lane) ? 1 : 0;
  }
  const uint64_t me = __builtin_amdgcn_ballot_w64(before == top - 1);
  return bits_float((uint32_t)__builtin_amdgcn_readlane((int)float_bits(x), me ? __builtin_ctzll(me) : 0));
}

// The best 64 of two falling lists, falling.
__device__ __forceinline__ Key merge(Key a, Key reversed, int lane) {
  Key k = a > reversed ? a : reversed;
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) {
    const Key other = __shfl_xor((unsigned long long)k, d);
    k = ((lane & d) == 0) == (k > other) ? k : other;
  }
  return k;
}

// ---- forward ------------------------------------------------------------------------------------

// A row whose largest logit times scale2 leaves float32's range: differences first.  In all threads.
template <int TYPE>
__device__ Sums row_again(const LogprobArgs& g, const void* row, float m, float* room) {
  float s = 0.0f, w = 0.0f;
  for (int col = threadIdx.x * kRun; col < g.vocab; col += kThreads * kRun) {
    float v[kRun];
    load_run<TYPE>(row, col, g.vocab - col, v);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      if (i >= g.vocab - col) continue;
      const float t = larger((v[i] - m) * g.scale2, kFar), e = exp2_of(t);
      s += e;
      w = __builtin_fmaf(e, t, w);
    }
  }
  __syncthreads();
  for (int d = 1; d < kWave; d *= 2) {
    s += __shfl_xor(s, d);
    w += __shfl_xor(w, d);
  }
  if (threadIdx.x % kWave == 0) {
    room[threadIdx.x / kWave] = s;
    room[kWaves + threadIdx.x / kWave] = w;
  }
  __syncthreads();
  Sums x{m, 0.0f, 0.0f, 0.0f};
  for (int i = 0; i < kWaves; ++i) {
    x.s += room[i];
    x.w += room[kWaves + i];
  }
  return x;
}

// What a row's sums say; by == again: sums of differences.
struct Row {
  Sums x;
  float log;      // log2 of s
  bool again, none, empty;
  __device__ Row(const Sums& sums, bool differences) : x(sums), again(differences) {
    empty = x.m == -kInf && x.s == 0.0f;
    none = !(x.s > 0.0f && x.s < kInf) && !empty;   // NaN or an infinite logit
    log = log2f(x.s);
  }
  __device__ float logp(float logit, const LogprobArgs& g) const {
    if (none) return bits_float(0x7FC00000u);
    if (empty) return -kInf;
    const float p = kLn2 * ((again ? (logit - x.m) * g.scale2 : __builtin_fmaf(logit, g.scale2, -x.at)) - log);
    if (p == -kInf && logit > -kInf) return __builtin_fmaf(logit, g.scale, -lse(g));   // the logit times scale2 has left the range
    return fminf(p, 0.0f);   // a rounding of scale2 * m may leave 2^-24 above
  }
  __device__ float lse(const LogprobArgs& g) const {
    if (none) return bits_float(0x7FC00000u);
    if (empty) return -kInf;
    return again ? __builtin_fmaf(kLn2, log, g.scale * x.m) : kLn2 * (x.at + log);
  }
  __device__ float entropy() const { return none ? bits_float(0x7FC00000u) : empty ? 0.0f : fmaxf(kLn2 * (log - x.w / x.s), 0.0f); }
};

template <int TYPE>
__device__ __forceinline__ void write_row(const LogprobArgs& g, int64_t row, const Row& r) {
  using T = typename Stored<TYPE>::type;
  g.lse[row] = r.lse(g);
  g.entropy[row] = r.entropy();
  if (!g.logp) return;
  const int64_t t = token_of(g, row);
  float p = 0.0f;
  if (t >= g.vocab) p = bits_float(0x7FC00000u);
  else if (t >= 0) p = r.logp((float)(static_cast<const T*>(g.logits) + row * g.stride)[t], g);
  g.logp[row] = p;
}

__device__ __forceinline__ void write_top(const LogprobArgs& g, int64_t row, const Row& r, Key k, int lane) {
  if (lane >= g.top) return;
  g.top_logp[row * g.top + lane] = r.logp(logit_of(k), g);
  g.top_tokens[row * g.top + lane] = r.none ? -1 : (int64_t)place_of(k);
}

template <int TYPE, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_forward_kernel(LogprobArgs g) {
  using T = typename Stored<TYPE>::type;
  constexpr int kAhead = 4;
  __shared__ Sums sums[kWaves];
  __shared__ float room[2 * kWaves];
  __shared__ Key keys[TOP ? kWaves : 1][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t row = block_of();
  if (row >= g.rows) return;
  const void* const at = static_cast<const T*>(g.logits) + row * g.stride;
  Sums x{-kInf, 0.0f, 0.0f, 0.0f};
  Best best;
  bool first = true;
  int col = threadIdx.x * kRun;
  const auto take = [&](auto& v, int n) {   // N / 8 runs, kThreads * 8 columns apart; the last of n values
    constexpr int N = sizeof(v) / sizeof(float);
    float largest = -kInf;
    if constexpr (TOP) {
#pragma unroll
      for (int i = 0; i < N; ++i) largest = fmaxf(largest, v[i]);
    }
    add_values(x, v, g.scale2);
    if constexpr (TOP) {
      const float over = first ? reached(largest, lane, g.top) : best.above;
      const bool with = first || !best.full;
      if (__builtin_amdgcn_ballot_w64(with || largest > over) != 0) {
#pragma unroll
        for (int u = 0; u < N / kRun; ++u) {
          float run[kRun];
#pragma unroll
          for (int i = 0; i < kRun; ++i) run[i] = v[u * kRun + i];
          best.offer(run, col + u * kThreads * kRun, u == N / kRun - 1 ? n : kRun, over, with, lane, g.top);
        }
        best.settle();
      }
      first = false;
    }
  };
  for (; col - threadIdx.x * kRun + kAhead * kThreads * kRun <= g.vocab; col += kAhead * kThreads * kRun) {
    Raw w[kAhead];
    float v[kAhead * kRun];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) w[u] = load_raw<TYPE>(at, nullptr, col + u * kThreads * kRun, kRun);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float run[kRun];
      values_of<TYPE>(w[u], run);
#pragma unroll
      for (int i = 0; i < kRun; ++i) v[u * kRun + i] = run[i];
    }
    take(v, kRun);
  }
  for (; col - threadIdx.x * kRun < g.vocab; col += kThreads * kRun) {
    const int n = g.vocab - col;
    float v[kRun];
    load_run<TYPE>(at, col, n, v);
#pragma unroll
    for (int i = 0; i < kRun; ++i) v[i] = i < n ? v[i] : -kInf;
    take(v, n);
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) join(x, from_lane(x, d));
  if (lane == 0) sums[wave] = x;
  if constexpr (TOP) keys[wave][lane] = best.key;
  __syncthreads();
  x = sums[0];
  for (int i = 1; i < kWaves; ++i) join(x, sums[i]);
  // beyond float32's range, or with its largest logit there, which then counted as nothing
  const bool again = x.m > -kInf && (!(x.s > 0.0f && x.s < kInf) || x.at != anchor(x.m, g.scale2));
  if (again) x = row_again<TYPE>(g, at, x.m, room);
  if (wave != 0) return;
  const Row r(x, again);
  if (lane == 0) write_row<TYPE>(g, row, r);
  if constexpr (TOP) {
    Key k = best.key;
    for (int i = 1; i < kWaves; ++i) k = merge(k, keys[i][kWave - 1 - lane], lane);
    write_top(g, row, r, k, lane);
  }
}

// ---- backward -----------------------------------------------------------------------------------

constexpr int kTurns = 4, kAtOnce = kThreads * kTurns * kRun;   // columns of a workgroup

template <int TYPE, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void logprob_backward_kernel(LogprobArgs g, int pieces) {
  using T = typename Stored<TYPE>::type;
  const int64_t block = block_of(), row = block / pieces;
  if (row >= g.rows) return;
  const int from = (int)(block - row * pieces) * kAtOnce;
  const void* const at = static_cast<const T*>(g.logits) + row * g.stride;
  char* const out = static_cast<char*>(g.out) + row * g.out_stride * (g.out_type == MOC_F32 ? 4 : 2);
  const float lse = g.lse_of[row], entropy = ENTROPY ? g.entropy_of[row] : 0.0f, dh = ENTROPY ? g.dentropy[row] : 0.0f;
  const int64_t token = g.dlogp ? token_of(g, row) : -1;
  const float dl = token < 0 ? 0.0f : token < g.vocab ? g.dlogp[row] : bits_float(0x7FC00000u);
  const bool empty = lse == -kInf;
  Raw w[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int col = from + (t * kThreads + threadIdx.x) * kRun;
    w[t] = load_raw<TYPE>(at, nullptr, col, g.vocab - col);
  }
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int col = from + (t * kThreads + threadIdx.x) * kRun, n = g.vocab - col;
    if (n <= 0) break;
    float v[kRun];
    values_of<TYPE>(w[t], v);
    const int64_t mine = token - col;
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const float z = larger(__builtin_fmaf(v[i], g.scale, -lse), kFar), p = exp2_of(z * kLog2e);
      float d = dl * ((mine == i ? 1.0f : 0.0f) - p);
      if (ENTROPY) d -= dh * p * (z + entropy);
      v[i] = empty ? 0.0f : g.scale * d;
    }
    store_any(g.out_type, out, col, n, v);
  }
}

using Forward = void (*)(LogprobArgs);
using Backward = void (*)(LogprobArgs, int);
template <bool TOP>
Forward forward_of(int type) {
  return type == MOC_BF16 ? logprob_forward_kernel<MOC_BF16, TOP> : type == MOC_F16 ? logprob_forward_kernel<MOC_F16, TOP> : logprob_forward_kernel<MOC_F32, TOP>;
}
template <bool ENTROPY>
Backward backward_of(int type) {
  return type == MOC_BF16 ? logprob_backward_kernel<MOC_BF16, ENTROPY> : type == MOC_F16 ? logprob_backward_kernel<MOC_F16, ENTROPY> : logprob_backward_kernel<MOC_F32, ENTROPY>;
}

bool scale_ok(float scale) { return scale > 0.0f && scale <= 0x1p64f && scale >= 0x1p-64f; }
bool tokens_ok(const void* tokens, int bytes) { return !tokens || ((bytes == 4 || bytes == 8) && aligned_to(tokens, bytes)); }

}  // namespace

extern "C" {

int64_t moc_logprob_forward_work(int64_t rows, int64_t vocab, int32_t top) {
  if (!sizes_ok(rows, vocab) || vocab < 1 || top < 0 || top > kMostTop || top > vocab) return MOC_EINVAL;
  return 0;
}

int moc_logprob_forward(int64_t rows, int64_t vocab, const moc_matrix* logits, const void* tokens, int32_t token_bytes, float scale, int32_t top, float* logp, float* lse,
                        float* entropy, float* top_logp, int64_t* top_tokens, void* work, int64_t work_bytes, void* hip_stream) {
  if (!sizes_ok(rows, vocab) || vocab < 1 || top < 0 || top > kMostTop || top > vocab || !scale_ok(scale)) return MOC_EINVAL;
  if (!matrix_ok(logits, rows, vocab, true, false) || !tokens_ok(tokens, token_bytes)) return MOC_EINVAL;
  if (rows == 0) return MOC_OK;
  if ((tokens == nullptr) != (logp == nullptr) || !lse || !entropy || !aligned_to(logp, 4) || !aligned_to(lse, 4) || !aligned_to(entropy, 4)) return MOC_EINVAL;
  if (top > 0 && (!top_logp || !top_tokens || !aligned_to(top_logp, 4) || !aligned_to(top_tokens, 8))) return MOC_EINVAL;
  LogprobArgs g = {};
  g.logits = logits->data; g.stride = logits->stride;
  g.rows = rows; g.vocab = (int)vocab; g.top = top; g.token_bytes = token_bytes;
  g.scale = scale; g.scale2 = (float)((double)scale * 1.4426950408889634);
  g.tokens = tokens; g.logp = logp; g.lse = lse; g.entropy = entropy; g.top_logp = top_logp; g.top_tokens = top_tokens;
  hipLaunchKernelGGL(top > 0 ? forward_of<true>(logits->type) : forward_of<false>(logits->type), grid_of(rows), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), g);
  MOC_HIP(hipGetLastError());
  return MOC_OK;
}

int moc_logprob_backward(int64_t rows, int64_t vocab, const moc_matrix* logits, const float* lse, const float* entropy, const void* tokens, int32_t token_bytes, const float* dlogp,
                         const float* dentropy, float scale, const moc_matrix* out, void* hip_stream) {
  if (!sizes_ok(rows, vocab) || vocab < 1 || !scale_ok(scale)) return MOC_EINVAL;
  if (!matrix_ok(logits, rows, vocab, true, false) || !matrix_ok(out, rows, vocab, true, false) || !tokens_ok(tokens, token_bytes)) return MOC_EINVAL;
  if (out->type != logits->type && out->type != MOC_F32) return MOC_EINVAL;
  if (rows == 0) return MOC_OK;
  if (!lse || !aligned_to(lse, 4) || (tokens == nullptr) != (dlogp == nullptr) || !aligned_to(dlogp, 4)) return MOC_EINVAL;
  if ((dentropy && !entropy) || !aligned_to(entropy, 4) || !aligned_to(dentropy, 4)) return MOC_EINVAL;
  LogprobArgs g = {};
  g.logits = logits->data; g.stride = logits->stride;
  g.rows = rows; g.vocab = (int)vocab; g.token_bytes = token_bytes;
  g.scale = scale;
  g.tokens = tokens; g.lse_of = lse; g.entropy_of = entropy; g.dlogp = dlogp; g.dentropy = dentropy;
  g.out = out->data; g.out_stride = out->stride; g.out_type = out->type;
  const int pieces = (int)((vocab + kAtOnce - 1) / kAtOnce);
  hipLaunchKernelGGL(dentropy ? backward_of<true>(logits->type) : backward_of<false>(logits->type), grid_of(rows * pieces), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), g,
                     pieces);
  MOC_HIP(hipGetLastError());
  return MOC_OK;
}

}  // extern "C"
