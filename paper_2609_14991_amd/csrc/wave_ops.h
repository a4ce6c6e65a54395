// Wave-wide reductions and row access shared by the scoring kernels
// (logprobs.hip, joint_logprobs.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <climits>
#include <cstdint>

namespace fusion {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// stands for -infinity in x - max: e^it is 0, and 0 times it is 0 and not NaN
constexpr float kFar = -1e4f;

// one step of a reduction: the neighbour's value under a DPP pattern
template <int CTRL, int ROWS>
__device__ __forceinline__ int wave_move(int ident, int v) {
  return __builtin_amdgcn_update_dpp(ident, v, CTRL, ROWS, 0xF, false);
}
// op over the 64 lanes, the result in every lane: quads, half rows and rows of 16
// lanes, then row 0 into 1 and 2 into 3, then the lower half into the upper
template <class F>
__device__ __forceinline__ int wave_reduce(int ident, int v, F op) {
  v = op(v, wave_move<0xB1, 0xF>(ident, v));
  v = op(v, wave_move<0x4E, 0xF>(ident, v));
  v = op(v, wave_move<0x141, 0xF>(ident, v));
  v = op(v, wave_move<0x140, 0xF>(ident, v));
  v = op(v, wave_move<0x142, 0xA>(ident, v));
  v = op(v, wave_move<0x143, 0xC>(ident, v));
  return __builtin_amdgcn_readlane(v, 63);
}
// Order-preserving image of a float that is not NaN, the zeros as one, and back.
// (Integer maxima and minima take their neighbour's value in the same instruction.)
__device__ __forceinline__ int order_of(float x) {
  const int b = __float_as_int(x + 0.0f);
  return b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float of_order(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7FFFFFFF)); }
__device__ __forceinline__ int wave_max(int x) {
  return wave_reduce(INT_MIN, x, [](int a, int b) { return max(a, b); });
}
__device__ __forceinline__ float wave_max(float x) { return of_order(wave_max(order_of(x))); }
__device__ __forceinline__ float wave_add(float x) {
  return __int_as_float(wave_reduce(0, __float_as_int(x), [](int a, int b) {
    return __float_as_int(__int_as_float(a) + __int_as_float(b));
  }));
}
__device__ __forceinline__ int wave_min(int x) {
  return wave_reduce(INT_MAX, x, [](int a, int b) { return min(a, b); });
}

// op over lanes l, l ^ 16, l ^ 32 and l ^ 48, the result in all four: exchanging a
// register with itself leaves the two sides' values in its two copies
template <class F>
__device__ __forceinline__ float across_rows(float x, F op) {
  auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Softmax statistics of a set of values: their maximum m, how many equal it, the
// sum of e^(x - m) over the others and the sum of (x - m) e^(x - m).  The ones are
// counted apart from the sum because where one value holds nearly all of the
// probability, its log probability is -log(1 + rest) and the entropy is of the
// size of the rest, which 1 + rest in fp32 would round off.
// A NaN or +infinity among the values makes `rest` NaN and stays there.
struct Stat {
  float m, ones, rest, u;
};
__device__ __forceinline__ Stat stat_none() { return Stat{-INFINITY, 0.0f, 0.0f, 0.0f}; }

// the same set's statistics relative to a maximum M >= s.m
__device__ __forceinline__ void stat_lift(Stat &s, float M) {
  const float base = M == -INFINITY ? 0.0f : M;
  const float d = fmaxf(s.m - base, kFar), f = exp_of(d), all = s.ones + s.rest;
  if (s.m != M) {
    s.u = f * (s.u + d * all);
    s.rest = f * all;
    s.ones = 0.0f;
    s.m = M;
  }
}

// `n` more values; lane_max is their maximum
template <int n>
__device__ __forceinline__ void stat_take(Stat &s, const float (&x)[n], float lane_max) {
  stat_lift(s, fmaxf(s.m, lane_max));
  const float base = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll
  for (int j = 0; j < n; ++j) {
    const float d = x[j] - base, e = exp_of(d);
    s.ones += d == 0.0f ? 1.0f : 0.0f;
    s.rest += d == 0.0f ? 0.0f : e;
    s.u = fmaf(fmaxf(d, kFar), e, s.u);
  }
}

// Statistics that a wave gathers over a row: relative to a maximum that its lanes
// share, the sums a lane's own; u in units of log2 e.  The maxima are among the rest
// as long as that is 1.25 or more, and counted as ones where it would be less.
struct WaveStat {
  float m, ones, rest, u;
};
__device__ __forceinline__ WaveStat wave_stat_none() { return WaveStat{-INFINITY, 0.0f, 0.0f, 0.0f}; }

// x - base in units of log2 e, kFar for -infinity (NaN stays)
__device__ __forceinline__ float log2_of(float x, float base) {
  return __builtin_elementwise_maximum((x - base) * kLog2e, kFar);
}

// `n` more values of every lane; top: the lane's largest, all_top: the wave's.  Six
// operations a value, the exponential among them.
template <int n>
__device__ __forceinline__ void wave_stat_take(WaveStat &s, const float (&x)[n], float top, float all_top) {
  if (all_top > s.m) {  // uniform
    const float d = fmaxf((s.m - all_top) * kLog2e, kFar), f = __builtin_amdgcn_exp2f(d), all = s.ones + s.rest;
    s.u = f * (s.u + d * all);
    s.rest = f * all;
    s.ones = 0.0f;
    s.m = all_top;
  }
  const float base = s.m == -INFINITY ? 0.0f : s.m;
  float sum[4] = {}, u[4] = {};
#pragma unroll
  for (int j = 0; j < n; ++j) {
    const float t = log2_of(x[j], base), e = __builtin_amdgcn_exp2f(t);
    sum[j % 4] += e;
    u[j % 4] = fmaf(t, e, u[j % 4]);
  }
  const float more = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  // the maximum is new, and next to nothing with it: its 1 apart
  if (all_top == s.m && all_top != -INFINITY && __ballot(top == s.m && more < 1.25f) && wave_add(more) < 1.25f) {
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float t = log2_of(x[j], base), e = x[j] == s.m ? 0.0f : __builtin_amdgcn_exp2f(t);
      s.ones += x[j] == s.m ? 1.0f : 0.0f;
      s.rest += e;
      s.u = fmaf(t, e, s.u);
    }
  } else {
    s.rest += more;
    s.u += (u[0] + u[1]) + (u[2] + u[3]);
  }
}

// the lanes' together, in every lane
__device__ __forceinline__ Stat wave_stat_done(const WaveStat &s) {
  return Stat{s.m, wave_add(s.ones), wave_add(s.rest), wave_add(s.u * kLn2)};
}

// two sets' statistics as one
__device__ __forceinline__ void stat_join(Stat &s, Stat o) {
  const float M = fmaxf(s.m, o.m);
  stat_lift(s, M);
  stat_lift(o, M);
  s.ones += o.ones;
  s.rest += o.rest;
  s.u += o.u;
}

// several sets' statistics as one
template <int n>
__device__ __forceinline__ Stat stat_of(const Stat (&v)[n]) {
  Stat s = stat_none();
#pragma unroll
  for (int q = 0; q < n; ++q) s.m = fmaxf(s.m, v[q].m);
  const float base = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll
  for (int q = 0; q < n; ++q) {
    const float d = fmaxf(v[q].m - base, kFar), f = exp_of(d), all = v[q].ones + v[q].rest;
    const bool top = v[q].m == s.m;
    s.ones += top ? v[q].ones : 0.0f;
    s.rest += top ? v[q].rest : f * all;
    s.u += f * (v[q].u + d * all);
  }
  return s;
}

// the 64 lanes' statistics as one, in every lane
__device__ __forceinline__ void stat_wave(Stat &s) {
  stat_lift(s, wave_max(s.m));
  s.ones = wave_add(s.ones);
  s.rest = wave_add(s.rest);
  s.u = wave_add(s.u);
}

// those of lanes l, l ^ 16, l ^ 32 and l ^ 48 as one, in all four
__device__ __forceinline__ Stat stat_across(Stat s) {
  const auto add = [](float a, float b) { return a + b; };
  stat_lift(s, across_rows(s.m, [](float a, float b) { return fmaxf(a, b); }));
  return Stat{s.m, across_rows(s.ones, add), across_rows(s.rest, add), across_rows(s.u, add)};
}

// what a finished set's statistics say
struct RowScore {
  float m, log_s, lse, entropy;
  bool empty, bad;  // nothing above -infinity; a NaN or +infinity in the row
};
__device__ __forceinline__ RowScore row_score(const Stat &s) {
  RowScore r;
  const float all = s.ones + s.rest;
  r.bad = !(all < INFINITY);
  r.empty = all == 0.0f;
  r.m = s.m;
  r.log_s = log1pf((s.ones - 1.0f) + s.rest);
  r.lse = s.m + r.log_s;
  r.entropy = r.log_s - s.u / all;
  if (r.empty) {
    r.log_s = 0.0f;
    r.lse = -INFINITY;
    r.entropy = 0.0f;
  }
  if (r.bad) r.log_s = r.lse = r.entropy = __int_as_float(0x7FC00000);
  return r;
}
// log probability of a value of the row
__device__ __forceinline__ float row_logp(const RowScore &r, float x) {
  return r.empty ? -INFINITY : (x - r.m) - r.log_s;
}

// Where the token of slot b of stream s at frame t was chosen: the row of its
// parent slot, or its own without parents; -1 for a dead slot, -2 for a parent
// outside the beam
__device__ __forceinline__ int64_t row_of_token(const int32_t *parents, int32_t m, int32_t B) {
  if (!parents) return m;
  const int32_t p = parents[m];
  if (p == -1) return -1;
  if (p < 0 || p >= B) return -2;
  return (int64_t)(m / B) * B + p;
}

}  // namespace fusion
