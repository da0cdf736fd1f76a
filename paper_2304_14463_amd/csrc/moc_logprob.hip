// Log probabilities of given tokens with the entropy and the most likely alternatives, and their gradient.
//
// Forward: one pass over a row.  A lane holds the largest logit m it has met, s = sum of e and w = sum of e t with
// t = scale (x - m) / ln 2 and e = 2^t; a larger one scales both, s' = f s and w' = f (w + d s) with d = scale (m - m') / ln 2 and
// f = 2^d, and so do lanes that are joined.  Then log sum exp = scale m + ln s and the entropy ln s - ln 2 w / s.
// The alternatives: the wanted number of lanes have a largest logit that is not below some value, so nothing below it is among
// them; the few lanes whose largest is not below it have their columns read again, what is not below it goes to LDS, and its
// places in the order are counted.  Few rows are cut into parts, whose sums and alternatives a second kernel joins.  A
// workgroup a row of 8192 x 131072 bf16: 359 us, 6.0 TB/s, the vector ALU busy beside it (eight instructions a logit, exp2 at a
// quarter of the rate); 4999 x 32003 fp16 with five alternatives 69 us, 64 of them 96 (391 with lists that waves hold); one row
// of 131072 with twenty 12 us (51 by one workgroup).
// Backward: a pass over the logits and their gradient, 8192 columns a workgroup, runs at aligned addresses: 8192 x 131072 bf16
// 690 us, 6.2 TB/s (843 where each load had a branch); four float32 values a lane (1247 x 32003 63 us, 83 with eight).
// Times of one input again and again; where inputs change from pass to pass, 4999 x 32003 takes 72 us, the gradient of 1247 x 32003 69.
#include <algorithm>

#include "moc_rows.h"
#include "moc_wave.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kMostTop = kWave, kMostParts = kWave;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFar = -200.0f;   // 2^kFar is 0: a value further below the largest adds nothing, an infinite one neither

struct Sums;
struct LogprobArgs {
  const void* logits;
  int64_t stride;
  int64_t rows;
  int vocab, top, token_bytes;
  float scale, scale2;   // scale2 = scale / ln 2
  const void* tokens;
  float *logp, *lse, *entropy, *top_logp;
  int64_t* top_tokens;
  int parts, part_cols;
  Sums* part_sums;   // [rows][parts]
  uint64_t* part_keys;      // [rows][parts][top]
  // backward
  const float *lse_of, *entropy_of, *dlogp, *dentropy;
  void* out;
  int64_t out_stride;
  int out_type;
};

// NaN where one of the two is NaN.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ int64_t token_of(const LogprobArgs& g, int64_t row) {
  return g.token_bytes == 8 ? static_cast<const int64_t*>(g.tokens)[row] : static_cast<const int32_t*>(g.tokens)[row];
}

// ---- sums ---------------------------------------------------------------------------------------

struct Sums {
  float m;      // the largest logit
  float at;     // scale2 * m, rounded, or what anchor() makes of it: terms are 2^(scale2 x - at)
  float s, w;
};

// Up to kReach either way, scale2 * m is rounded by a quarter at most, so that the largest term is 2^(+-1/4) and all sums stay
// in range.  Beyond it the rounding grows without bound (2^100 and more for masks of -1e9 or -1e30, and their w not a number
// where a real logit comes after): what lies below counts as nothing beside whatever lies above, and a row of nothing else, or one with
// logits above kReach, is taken again by row_again().  4999 x 32000 fp32 masked by -1e9 or -1e30 106 us as by -infinity, 180
// where the mask leaves nothing.
constexpr float kReach = 0x1p23f;
__device__ __forceinline__ float anchor(float m, float scale2) { return fmaxf(m * scale2, -kReach); }

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

// Over the wave, in lane 63: shifts of the vector ALU inside rows of 16 lanes, then across them.
template <int CTRL, int ROWS>
__device__ __forceinline__ float shifted(float a, float otherwise) {
  return bits_float((uint32_t)__builtin_amdgcn_update_dpp((int)float_bits(otherwise), (int)float_bits(a), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float wave_largest(float a) {
  a = fmaxf(a, shifted<0x111, 0xF>(a, -kInf));
  a = fmaxf(a, shifted<0x112, 0xF>(a, -kInf));
  a = fmaxf(a, shifted<0x114, 0xF>(a, -kInf));
  a = fmaxf(a, shifted<0x118, 0xF>(a, -kInf));
  a = fmaxf(a, shifted<0x142, 0xA>(a, -kInf));
  a = fmaxf(a, shifted<0x143, 0xC>(a, -kInf));
  return bits_float((uint32_t)__builtin_amdgcn_readlane((int)float_bits(a), kWave - 1));
}
__device__ __forceinline__ Sums join_wave(Sums x) {
  move_to(x, wave_largest(x.s == 0.0f ? -kInf : x.at));   // one that holds nothing has no say; where none holds any, s and w are 0 all the same
  return Sums{wave_largest(x.m), x.at, wave_sum(x.s), wave_sum(x.w)};
}

// ---- columns ------------------------------------------------------------------------------------

// The columns lo .. hi - 1 of a row, taken in runs of eight from `first` on, where runs begin at aligned addresses: up to seven
// columns before lo.
constexpr int kStep = kThreads * kRun;
struct Columns {
  int first, lo, hi;
};
// Runs begin at addresses that are multiples of 16 bytes.
template <int TYPE>
__device__ __forceinline__ int before_row(const void* row) {
  return (int)(reinterpret_cast<uintptr_t>(row) % 16) / (int)sizeof(typename Stored<TYPE>::type);
}
__device__ __forceinline__ bool whole_run(const Columns& c, int col) { return col >= c.lo && col + kRun <= c.hi; }
// A run that is not wholly there, `otherwise` for what is not: loads without a branch, none of which is waited for alone.
template <int TYPE>
__device__ __forceinline__ void load_edge(const void* row, const Columns& c, int col, float otherwise, float (&v)[kRun]) {
  using T = typename Stored<TYPE>::type;
  T t[kRun];
#pragma unroll
  for (int i = 0; i < kRun; ++i) t[i] = static_cast<const T*>(row)[min(max(col + i, c.lo), c.hi - 1)];
#pragma unroll
  for (int i = 0; i < kRun; ++i) v[i] = col + i >= c.lo && col + i < c.hi ? (float)t[i] : otherwise;
}
template <int TYPE>
__device__ __forceinline__ void load_columns(const void* row, const Columns& c, int col, float otherwise, float (&v)[kRun]) {
  if (whole_run(c, col)) load_run<TYPE>(row, col, kRun, v);
  else load_edge<TYPE>(row, c, col, otherwise, v);
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

// A number that `top` keys or more are not below, EACH of them a thread: the last of the best, or one with as many of its upper
// bits as leave few keys.  Its bits one after the other, down to `lowest`.  By all threads.
constexpr int kFewKeys = 2 * kMostTop;
struct CutRoom {
  uint32_t counts[2][kWaves], left;
};
template <int EACH>
__device__ __forceinline__ Key bound_of(const Key (&k)[EACH], int top, int lowest, CutRoom& r) {
  Key t = 0;
#pragma unroll 1
  for (int bit = 63, half = 0; bit >= lowest; --bit, half ^= 1) {
    const Key next = t | (Key)1 << bit;
    int count = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k[i] >= next));
    if (threadIdx.x % kWave == 0) r.counts[half][threadIdx.x / kWave] = (uint32_t)count;
    __syncthreads();
    count = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) count += (int)r.counts[half][i];
    if (count < top) continue;
    t = next;
    if (count <= kFewKeys) break;
  }
  return t;
}
template <int EACH>
__device__ __forceinline__ void keys_of(const Key* keys, uint32_t n, Key (&k)[EACH]) {
#pragma unroll
  for (int i = 0; i < EACH; ++i) k[i] = i * kThreads + threadIdx.x < n ? keys[i * kThreads + threadIdx.x] : 0;
}
// Of n keys in LDS, more than a few, those that can be among the first `top`, in their place; how many those are, in all threads.
template <int EACH>
__device__ __forceinline__ uint32_t cut_keys(Key* keys, uint32_t n, int top, CutRoom& r) {
  Key k[EACH];
  keys_of(keys, n, k);
  if (threadIdx.x == 0) r.left = 0;
  const Key least = bound_of(k, top, 0, r);
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (k[i] >= least) keys[atomicAdd(&r.left, 1u)] = k[i];
  __syncthreads();
  return r.left;
}

// A logit that at least `top` of the lanes reach with their largest, in all threads: the largest number of 16 bits that as many
// of the upper halves of their orders are not below.
constexpr int kRoom = 1024;
struct TopRoom {
  float largest[kThreads];
  uint16_t lanes[kThreads];
  uint32_t reach, found, again;   // one for each step: a wave may read what it went by after another went on
  float least;
  Key keys[kRoom], best[kMostTop];
  CutRoom cut;
};
__device__ __forceinline__ void find_least(TopRoom& r, int top) {
  if (threadIdx.x < kWave) {
    uint32_t half[kWaves], t = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) half[i] = (uint32_t)(key_of(r.largest[i * kWave + threadIdx.x], 0) >> 48);
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
      const uint32_t next = t | 1u << bit;
      int count = 0;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(half[i] >= next));
      if (count >= top) t = next;
    }
    const float least = logit_of((Key)t << 48);
    if (threadIdx.x == 0) r.least = least == least ? least : -kInf;
  }
}

// What is above `least`, or not below it (`with`), of the columns of lanes that reach it, to r.keys; no further than there is room
// for.  4999 x 32000 fp16 with equal logits: 170 us, 578 where each logit asked for its own place and all were counted.
template <int TYPE>
__device__ __forceinline__ void gather(const void* row, const Columns& c, float least, bool with, TopRoom& r) {
  const uint32_t lanes = r.reach, total = lanes * (uint32_t)((c.hi - c.first + kStep - 1) / kStep);
  for (uint32_t i = threadIdx.x; i < total; i += kThreads) {
    const int col = c.first + (int)(i / lanes * kThreads + r.lanes[i % lanes]) * kRun;
    if (col >= c.hi) continue;
    float v[kRun];
    load_columns<TYPE>(row, c, col, bits_float(0x7FC00000u), v);
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      const uint64_t some = __builtin_amdgcn_ballot_w64(with ? v[j] >= least : v[j] > least);
      if (some == 0) continue;
      // one lane asks for all
      const int first = __builtin_ctzll(some);
      uint32_t begin = 0;
      if ((int)(threadIdx.x % kWave) == first) begin = atomicAdd(&r.found, (uint32_t)__builtin_popcountll(some));
      begin = (uint32_t)__builtin_amdgcn_readlane((int)begin, first);
      const uint32_t at = begin + __builtin_amdgcn_mbcnt_hi((uint32_t)(some >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)some, 0));
      if (at < kRoom && (some >> (threadIdx.x % kWave) & 1)) r.keys[at] = key_of(v[j], (uint32_t)(col + j));
      if (begin > kRoom) return;   // more than there is room for, in any case
    }
  }
}

// More logits than there is room for: the last of the best among those that are there, or little below it, is a better bound.  What is above it, and of
// those that equal it the first ones by column, as many as are missing; or all over again from there, as every key there is
// above the bound then.  By all threads, as all of these.
template <int TYPE>
__device__ __attribute__((noinline)) uint32_t gather_again(const void* row, Columns c, int top, TopRoom* room) {
  TopRoom& r = *room;
  for (uint32_t above = kRoom;;) {
    __syncthreads();
    Key k[kRoom / kThreads];
    keys_of(r.keys, above, k);
    float least = logit_of(bound_of(k, top, 32, r.cut));
    least = least == least ? least : -kInf;
    if (threadIdx.x == 0) r.found = 0;
    __syncthreads();
    gather<TYPE>(row, c, least, false, r);
    __syncthreads();
    above = min(r.found, (uint32_t)kRoom);
    if (above > kRoom - kMostTop) continue;   // at least `top` of what is above the bound: it rises
    if (threadIdx.x < kWave) {
      uint32_t have = above;
      for (int at = c.lo; at < c.hi && have < (uint32_t)top; at += kWave * kRun) {
        const int col = at + (int)threadIdx.x * kRun;
        float v[kRun];
        uint32_t equal = 0;
        if (col < c.hi) {
          load_columns<TYPE>(row, c, col, bits_float(0x7FC00000u), v);
#pragma unroll
          for (int j = 0; j < kRun; ++j) equal |= v[j] == least ? 1u << j : 0;
        }
        const int mine = __builtin_popcount(equal), up_to = scan_sum(mine);
        uint32_t place = have + (uint32_t)(up_to - mine);
        for (; equal != 0 && place < (uint32_t)top; equal &= equal - 1, ++place) r.keys[place] = key_of(least, (uint32_t)(col + __builtin_ctz(equal)));
        have += (uint32_t)__builtin_amdgcn_readlane(up_to, kWave - 1);
      }
      if (threadIdx.x == 0) r.again = min(max((uint32_t)top, above), have);
    }
    __syncthreads();
    return r.again;
  }
}

// The first `top` of n keys in LDS, in falling order, to best; 0 behind the last.  Takes time by the square of n: few lanes with many
// candidates 242 us where they were cut to a few first, 762 without; one row of 131072 equal logits 43, 886 without.  Ends with
// a barrier.
__device__ __forceinline__ void order(const Key* keys, uint32_t n, int top, Key* best) {
  if (threadIdx.x < kMostTop) best[threadIdx.x] = 0;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
    const Key k = keys[i];
    int before = 0;
    for (uint32_t j = 0; j < n; ++j) before += keys[j] > k ? 1 : 0;
    if (before < top) best[before] = k;
  }
  __syncthreads();
}

// The best of some columns, of which `mine` is the largest of this thread's, to r.best.
template <int TYPE>
__device__ __forceinline__ void select_top(const void* row, const Columns& c, float mine, int top, TopRoom& r) {
  r.largest[threadIdx.x] = mine;
  if (threadIdx.x == 0) r.reach = r.found = 0;
  __syncthreads();
  find_least(r, top);
  __syncthreads();
  const float least = r.least;
  if (mine >= least) r.lanes[atomicAdd(&r.reach, 1u)] = (uint16_t)threadIdx.x;
  __syncthreads();
  gather<TYPE>(row, c, least, true, r);
  __syncthreads();
  uint32_t found = r.found;
  if (found > kRoom) found = gather_again<TYPE>(row, c, top, &r);
  if (found > kFewKeys) found = cut_keys<kRoom / kThreads>(r.keys, found, top, r.cut);
  order(r.keys, found, top, r.best);
}

// ---- forward ------------------------------------------------------------------------------------

// A row whose largest logit times scale2 lies beyond kReach: differences first.  In all threads.
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

// What a row's sums say; `again`: they are sums of differences.
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
    return smaller(p, 0.0f);   // a rounding of scale2 * m may leave 2^-24 above
  }
  __device__ float lse(const LogprobArgs& g) const {
    if (none) return bits_float(0x7FC00000u);
    if (empty) return -kInf;
    return again ? __builtin_fmaf(kLn2, log, g.scale * x.m) : kLn2 * (x.at + log);
  }
  __device__ float entropy() const { return none ? bits_float(0x7FC00000u) : empty ? 0.0f : larger(kLn2 * (log - x.w / x.s), 0.0f); }
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

// In all threads: the row's sums, and in lane i the best but i.
template <int TYPE, bool TOP>
__device__ __forceinline__ void finish_row(const LogprobArgs& g, int64_t row, Sums x, Key k, float* room) {
  using T = typename Stored<TYPE>::type;
  const bool again = x.m > -kInf && (!(x.s > 0.0f && x.s < kInf) || !(__builtin_fabsf(x.m * g.scale2) <= kReach));
  if (again) x = row_again<TYPE>(g, static_cast<const T*>(g.logits) + row * g.stride, x.m, room);
  if (threadIdx.x >= kWave) return;
  const Row r(x, again);
  if (threadIdx.x == 0) write_row<TYPE>(g, row, r);
  if constexpr (TOP) write_top(g, row, r, k, threadIdx.x);
}

template <int TYPE, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_forward_kernel(LogprobArgs g) {
  using T = typename Stored<TYPE>::type;
  constexpr int kAhead = 4;
  __shared__ Sums sums[kWaves];
  __shared__ float room[2 * kWaves];
  __shared__ __attribute__((aligned(8))) char top_room[TOP ? sizeof(TopRoom) : 8];
  const int64_t block = block_of(), row = block / g.parts;
  if (row >= g.rows) return;
  const void* const at = static_cast<const T*>(g.logits) + row * g.stride;
  const int begin = (int)(block - row * g.parts) * g.part_cols - before_row<TYPE>(at);
  const Columns c{begin, max(begin, 0), min(begin + g.part_cols, g.vocab)};
  Sums x{-kInf, 0.0f, 0.0f, 0.0f};
  // kAhead runs of a lane on their way at a time; at both ends they may not all be there
  for (int first = c.first; first < c.hi; first += kAhead * kStep) {
    const int col = first + threadIdx.x * kRun;
    Raw w[kAhead];
    float v[kAhead * kRun];
    if (first >= c.lo && first + kAhead * kStep <= c.hi) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) w[u] = load_raw<TYPE>(at, nullptr, col + u * kStep, kRun);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        float run[kRun];
        values_of<TYPE>(w[u], run);
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[u * kRun + i] = run[i];
      }
      add_values(x, v, g.scale2);
    } else {
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (whole_run(c, col + u * kStep)) w[u] = load_raw<TYPE>(at, nullptr, col + u * kStep, kRun);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (first + u * kStep >= c.hi) break;
        if (col + u * kStep >= c.hi) continue;
        float run[kRun];
        if (whole_run(c, col + u * kStep)) values_of<TYPE>(w[u], run);
        else load_edge<TYPE>(at, c, col + u * kStep, -kInf, run);
        add_values(x, run, g.scale2);
      }
    }
  }
  if constexpr (TOP) select_top<TYPE>(at, c, x.m, g.top, *reinterpret_cast<TopRoom*>(top_room));
  x = join_wave(x);
  if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = x;
  __syncthreads();
  x = sums[0];
  for (int i = 1; i < kWaves; ++i) join(x, sums[i]);
  Key k = 0;
  if constexpr (TOP) k = reinterpret_cast<TopRoom*>(top_room)->best[threadIdx.x % kMostTop];
  if (g.parts > 1) {
    if (threadIdx.x == 0) g.part_sums[block] = x;
    if (TOP && threadIdx.x < g.top) g.part_keys[block * g.top + threadIdx.x] = k;
    return;
  }
  finish_row<TYPE, TOP>(g, row, x, k, room);
}

// A row's parts joined.
template <int TYPE, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_join_kernel(LogprobArgs g) {
  __shared__ float room[2 * kWaves];
  __shared__ Sums sums;
  __shared__ Key keys[TOP ? kMostParts * kMostTop : 1], best[TOP ? kMostTop : 1];
  __shared__ Key least;
  __shared__ uint32_t found;
  __shared__ CutRoom cut;
  const int64_t row = block_of();
  if (row >= g.rows) return;
  const int lane = threadIdx.x % kWave;
  const Key* const from = g.part_keys + row * g.parts * g.top;
  if (threadIdx.x < kWave) {
    Sums x{-kInf, 0.0f, 0.0f, 0.0f};
    if (lane < g.parts) x = g.part_sums[row * g.parts + lane];
    x = join_wave(x);
    if (lane == 0) sums = x;
  } else if (TOP && threadIdx.x < 2 * kWave) {
    // `each` keys of a part are not below its each-th; of those, as many as it takes are not below the largest number of 16 bits
    // that so many of their upper ends are not below
    const int each = (g.top + g.parts - 1) / g.parts, needed = (g.top + each - 1) / each;
    const uint32_t upper = lane < g.parts ? (uint32_t)(from[lane * g.top + each - 1] >> 48) : 0;
    uint32_t t = 0;
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
      const uint32_t next = t | 1u << bit;
      if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(upper >= next)) >= needed) t = next;
    }
    if (lane == 0) {
      least = (Key)t << 48;
      found = 0;
    }
  }
  __syncthreads();
  const Sums x = sums;
  Key k = 0;
  if constexpr (TOP) {
    const Key bound = least;
    for (int i = threadIdx.x; i < g.parts * g.top; i += kThreads) {
      const Key one = from[i];
      if (one != 0 && one >= bound) keys[atomicAdd(&found, 1u)] = one;
    }
    __syncthreads();
    uint32_t n = found;
    if (n > kFewKeys) n = cut_keys<kMostParts * kMostTop / kThreads>(keys, n, g.top, cut);
    order(keys, n, g.top, best);
    k = best[threadIdx.x % kMostTop];
  }
  finish_row<TYPE, TOP>(g, row, x, k, room);
}

// ---- backward -----------------------------------------------------------------------------------

constexpr int kTurns = 4, kAtOnce = kThreads * kTurns * kRun;   // columns of a workgroup

// p = exp(z - lse) is off by what lse is, of itself: of rows beyond this, where half a step of lse is 2^-14 or more, the sum is taken
// again by differences from the largest logit.  All of a row masked by -1e9 has lse = -1e9, every p 1 by it, not one of the columns'.
constexpr float kFarLse = 1024.0f;

// Such a row, by one workgroup (the logits may be overwritten, so that no other may read them): the largest logit, the sum, the gradient.
// A value a lane, so that there is little code: 8192 x 131072 fp32 3.9 ms, 1.6 where no row is far; one row of 131072 87 us and 5.
template <int TYPE, class F>
__device__ __forceinline__ void each_value(const void* row, int vocab, const F& f) {
  constexpr int kEach = 8;   // on their way at a time
#pragma unroll 1
  for (int first = threadIdx.x; first < vocab; first += kEach * kThreads) {
    typename Stored<TYPE>::type t[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) t[u] = static_cast<const typename Stored<TYPE>::type*>(row)[min(first + u * kThreads, vocab - 1)];
#pragma unroll
    for (int u = 0; u < kEach; ++u)
      if (first + u * kThreads < vocab) f(first + u * kThreads, (float)t[u]);
  }
}
template <int TYPE, bool ENTROPY>
__device__ __forceinline__ void far_row(const LogprobArgs& g, const void* row, char* out, int64_t token, float dl, float dh, float entropy, float* room) {
  float m = -kInf, s = 0.0f;
  each_value<TYPE>(row, g.vocab, [&](int, float x) { m = fmaxf(m, x); });
  m = wave_largest(m);
  if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = m;
  __syncthreads();
  for (int i = 0; i < kWaves; ++i) m = fmaxf(m, room[i]);
  each_value<TYPE>(row, g.vocab, [&](int, float x) { s += exp2_of(larger((x - m) * g.scale2, kFar)); });
  s = wave_sum(s);
  if (threadIdx.x % kWave == 0) room[kWaves + threadIdx.x / kWave] = s;
  __syncthreads();
  s = 0.0f;
  for (int i = 0; i < kWaves; ++i) s += room[kWaves + i];
  const float log = log2f(s);
  const bool empty = m == -kInf;
  each_value<TYPE>(row, g.vocab, [&](int col, float x) {
    const float t = larger((x - m) * g.scale2 - log, kFar), p = exp2_of(t);
    float d = dl * ((token == col ? 1.0f : 0.0f) - p);
    if (ENTROPY) d -= dh * p * __builtin_fmaf(kLn2, t, entropy);
    d = empty ? 0.0f : g.scale * d;
    if (g.out_type == MOC_F32) reinterpret_cast<float*>(out)[col] = d;
    else reinterpret_cast<typename Stored<TYPE>::type*>(out)[col] = (typename Stored<TYPE>::type)d;
  });
}

// Six waves a SIMD: with the question for far rows and eight of them 8192 x 131072 bf16 takes 740 us, 690 so, 1247 x 32003 fp32 64 and 63.
template <int TYPE, bool ENTROPY>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 6))) void logprob_backward_kernel(LogprobArgs g, int pieces) {
  using T = typename Stored<TYPE>::type;
  __shared__ float room[2 * kWaves];
  const int64_t block = block_of(), row = block / pieces;
  if (row >= g.rows) return;
  const int from = (int)(block - row * pieces) * kAtOnce;
  const void* const at = static_cast<const T*>(g.logits) + row * g.stride;
  char* const out = static_cast<char*>(g.out) + row * g.out_stride * (g.out_type == MOC_F32 ? 4 : 2);
  const float lse = g.lse_of[row], entropy = ENTROPY ? g.entropy_of[row] : 0.0f, dh = ENTROPY ? g.dentropy[row] : 0.0f;
  const int64_t token = g.dlogp ? token_of(g, row) : -1;
  const float dl = token < 0 ? 0.0f : token < g.vocab ? g.dlogp[row] : bits_float(0x7FC00000u);
  const bool empty = !ENTROPY && token < 0;   // no gradient, whatever the logits are
  // In all of a row's workgroups; NaN is not.  Asked with the logits on their way, which are not looked at then.
  const auto far = [&] {
    if (!__builtin_amdgcn_readfirstlane(!empty && __builtin_fabsf(lse) > kFarLse)) return false;
    if ((uint32_t)(block - row * pieces) == (uint32_t)row % (uint32_t)pieces) far_row<TYPE, ENTROPY>(g, at, out, token, dl, dh, entropy, room);   // not all of them on one XCD
    return true;
  };
  const auto gradient = [&](float x, int col) {
    const float z = larger(__builtin_fmaf(x, g.scale, -lse), kFar), p = exp2_of(z * kLog2e);
    float d = dl * ((token == col ? 1.0f : 0.0f) - p);
    if (ENTROPY) d -= dh * p * (z + entropy);
    return empty ? 0.0f : g.scale * d;
  };
  if constexpr (TYPE == MOC_F32) {   // four values a lane: 16 bytes, next to the neighbour's
    constexpr int kFew = 4;
    u32x4 w[2 * kTurns];
#pragma unroll
    for (int t = 0; t < 2 * kTurns; ++t) {
      const int col = from + (t * kThreads + threadIdx.x) * kFew;
      if (col + kFew <= g.vocab) __builtin_memcpy(&w[t], static_cast<const float*>(at) + col, 16);
    }
    if (far()) return;
#pragma unroll
    for (int t = 0; t < 2 * kTurns; ++t) {
      const int col = from + (t * kThreads + threadIdx.x) * kFew;
      if (col + kFew <= g.vocab) {
#pragma unroll
        for (int i = 0; i < kFew; ++i) w[t][i] = float_bits(gradient(bits_float(w[t][i]), col + i));
        __builtin_memcpy(reinterpret_cast<float*>(out) + col, &w[t], 16);
      } else {
        for (int c = col; c < g.vocab; ++c) reinterpret_cast<float*>(out)[c] = gradient(static_cast<const float*>(at)[c], c);
      }
    }
  } else {
    // Runs begin where the output is 16 bytes apart from an aligned address: rows of an odd size do not (4999 x 32003 fp16
    // 166 us at 2-byte addresses, 124 so).  The first run of a row may begin before it.
    const int shift = g.out_type == TYPE ? before_row<TYPE>(out) : 0;
    Raw w[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int col = from + (t * kThreads + threadIdx.x) * kRun - shift;
      if (col >= 0 && col + kRun <= g.vocab) w[t] = load_raw<TYPE>(at, nullptr, col, kRun);
    }
    if (far()) return;
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int col = from + (t * kThreads + threadIdx.x) * kRun - shift;
      if (col >= 0 && col + kRun <= g.vocab) {
        float v[kRun];
        values_of<TYPE>(w[t], v);
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[i] = gradient(v[i], col + i);
        store_any(g.out_type, out, col, kRun, v);
      } else {
        for (int c = max(col, 0); c < min(col + kRun, g.vocab); ++c) {
          const float v[kRun] = {gradient((float)static_cast<const T*>(at)[c], c)};
          store_any(g.out_type, out, c, 1, v);
        }
      }
    }
  }
}

using Forward = void (*)(LogprobArgs);
using Backward = void (*)(LogprobArgs, int);
template <bool TOP>
Forward forward_of(int type) {
  return type == MOC_BF16 ? logprob_forward_kernel<MOC_BF16, TOP> : type == MOC_F16 ? logprob_forward_kernel<MOC_F16, TOP> : logprob_forward_kernel<MOC_F32, TOP>;
}
template <bool TOP>
Forward join_of(int type) {
  return type == MOC_BF16 ? logprob_join_kernel<MOC_BF16, TOP> : type == MOC_F16 ? logprob_join_kernel<MOC_F16, TOP> : logprob_join_kernel<MOC_F32, TOP>;
}

// Into how many parts a row is cut, and of how many columns: four workgroups for a unit, of whole steps.  `before`: how many
// columns before a row its first run may begin.
struct Parts {
  int parts, cols;
};
Parts parts_of(int64_t rows, int64_t vocab, int units, int before) {
  const int64_t steps = (vocab + before + kStep - 1) / kStep, wanted = std::min<int64_t>({(4 * (int64_t)units + rows - 1) / std::max<int64_t>(rows, 1), steps, kMostParts});
  const int64_t each = (steps + wanted - 1) / wanted;
  return Parts{(int)((steps + each - 1) / each), (int)(each * kStep)};
}
int64_t part_bytes(const Parts& p, int64_t rows, int top) { return p.parts > 1 ? rows * p.parts * (int64_t)(sizeof(Sums) + top * sizeof(Key)) : 0; }
template <bool ENTROPY>
Backward backward_of(int type) {
  return type == MOC_BF16 ? logprob_backward_kernel<MOC_BF16, ENTROPY> : type == MOC_F16 ? logprob_backward_kernel<MOC_F16, ENTROPY> : logprob_backward_kernel<MOC_F32, ENTROPY>;
}

float scale2_of(float scale) { return (float)((double)scale * 1.4426950408889634); }
bool scale_ok(float scale) { return scale > 0.0f && scale <= 0x1p64f && scale >= 0x1p-64f; }
bool tokens_ok(const void* tokens, int bytes) { return !tokens || ((bytes == 4 || bytes == 8) && aligned_to(tokens, bytes)); }

}  // namespace

extern "C" {

int64_t moc_logprob_forward_work(int64_t rows, int64_t vocab, int32_t top) {
  if (!sizes_ok(rows, vocab) || vocab < 1 || top < 0 || top > kMostTop || top > vocab) return MOC_EINVAL;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  return std::max(part_bytes(parts_of(rows, vocab, units, 0), rows, top), part_bytes(parts_of(rows, vocab, units, kRun - 1), rows, top));
}

int moc_logprob_forward(int64_t rows, int64_t vocab, const moc_matrix* logits, const void* tokens, int32_t token_bytes, float scale, int32_t top, float* logp, float* lse,
                        float* entropy, float* top_logp, int64_t* top_tokens, void* work, int64_t work_bytes, void* hip_stream) {
  if (!sizes_ok(rows, vocab) || vocab < 1 || top < 0 || top > kMostTop || top > vocab || !scale_ok(scale)) return MOC_EINVAL;
  if (!matrix_ok(logits, rows, vocab, true, false) || !tokens_ok(tokens, token_bytes)) return MOC_EINVAL;
  if (rows == 0) return MOC_OK;
  if ((tokens == nullptr) != (logp == nullptr) || !lse || !entropy || !aligned_to(logp, 4) || !aligned_to(lse, 4) || !aligned_to(entropy, 4)) return MOC_EINVAL;
  if (top > 0 && (!top_logp || !top_tokens || !aligned_to(top_logp, 4) || !aligned_to(top_tokens, 8))) return MOC_EINVAL;
  int units = 0;
  const int rc = moc_compute_units(&units);
  if (rc != MOC_OK) return rc;
  const bool aligned = aligned_to(logits->data, 16) && (rows == 1 || logits->stride * type_bytes(logits->type) % 16 == 0);
  const Parts p = parts_of(rows, vocab, units, aligned ? 0 : kRun - 1);
  if (p.parts > 1 && (!work || !aligned_to(work, 16) || work_bytes < part_bytes(p, rows, top))) return MOC_EINVAL;
  LogprobArgs g = {};
  g.parts = p.parts; g.part_cols = p.cols;
  if (p.parts > 1) {
    g.part_sums = static_cast<Sums*>(work);
    g.part_keys = reinterpret_cast<Key*>(g.part_sums + rows * p.parts);
  }
  g.logits = logits->data; g.stride = logits->stride;
  g.rows = rows; g.vocab = (int)vocab; g.top = top; g.token_bytes = token_bytes;
  g.scale = scale; g.scale2 = scale2_of(scale);
  g.tokens = tokens; g.logp = logp; g.lse = lse; g.entropy = entropy; g.top_logp = top_logp; g.top_tokens = top_tokens;
  hipLaunchKernelGGL(top > 0 ? forward_of<true>(logits->type) : forward_of<false>(logits->type), grid_of(rows * p.parts), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), g);
  MOC_HIP(hipGetLastError());
  if (p.parts > 1) {
    hipLaunchKernelGGL(top > 0 ? join_of<true>(logits->type) : join_of<false>(logits->type), grid_of(rows), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), g);
    MOC_HIP(hipGetLastError());
  }
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
  g.scale = scale; g.scale2 = scale2_of(scale);
  g.tokens = tokens; g.lse_of = lse; g.entropy_of = entropy; g.dlogp = dlogp; g.dentropy = dentropy;
  g.out = out->data; g.out_stride = out->stride; g.out_type = out->type;
  // a row's first run may begin up to seven columns before it
  const bool aligned = logits->type == MOC_F32 || out->type != logits->type || (aligned_to(out->data, 16) && (rows == 1 || out->stride * type_bytes(out->type) % 16 == 0));
  const int pieces = (int)((vocab + (aligned ? 0 : kRun - 1) + kAtOnce - 1) / kAtOnce);
  hipLaunchKernelGGL(dentropy ? backward_of<true>(logits->type) : backward_of<false>(logits->type), grid_of(rows * pieces), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), g,
                     pieces);
  MOC_HIP(hipGetLastError());
  return MOC_OK;
}

}  // extern "C"
