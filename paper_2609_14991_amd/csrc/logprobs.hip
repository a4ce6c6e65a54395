// Log probabilities of the tokens that a decode chose, with the entropy of the
// acoustic distribution they were chosen from and its best alternatives, and the
// gradient of both with respect to the logits.
//
// Per token (slot h of frame t), x the logits row it was chosen on:
//   m = max x, s = sum e^(x - m), u = sum (x - m) e^(x - m)
//   lse = m + log s,  logp = (x_tok - m) - log s,  entropy = log s - u / s
// and the k largest x - lse, ties to the lowest id.  Backward, p = e^(x - lse):
//   dx_y = sum over the row's tokens of  g_logp (1[y = tok] - p_y)
//                                      - g_entropy p_y (log p_y + entropy)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "fusion_internal.h"
#include "row_types.h"
#include "score_status.h"
#include "wave_ops.h"

namespace fusion {
namespace {

__device__ int32_t g_score_status;

typedef int Words __attribute__((ext_vector_type(4)));
typedef int UnalignedWords __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kPer = 16;           // values a lane holds of a wave's chunk
constexpr int kChunk = 64 * kPer;  // columns of a chunk
constexpr int kList = 128;         // candidates a wave keeps

// Column of value j of a lane's chunk
template <class T>
__device__ __forceinline__ int column(int base, int lane, int j) {
  constexpr int n = Pack<T>::n;
  return base + ((j / n) * 64 + lane) * n + j % n;
}

// Columns base .. base + 1023 of a row, -infinity past its end.  The pack that
// straddles the end is read whole, ending at the row's last element, and shifted.
template <class T>
__device__ __forceinline__ void load_chunk(const T *row, int V, int base, int lane, float (&x)[kPer]) {
  constexpr int n = Pack<T>::n;
  if (V < n) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int c = column<T>(base, lane, j);
      x[j] = c < V ? to_float(row[c]) : -INFINITY;
    }
    return;
  }
  Pack<T> p[kPer / n];
#pragma unroll
  for (int i = 0; i < kPer / n; ++i) __builtin_memcpy(&p[i], row + min(base + (i * 64 + lane) * n, V - n), 16);
#pragma unroll
  for (int j = 0; j < kPer; ++j) x[j] = to_float(p[j / n].v[j % n]);
  if (base + kChunk > V) {
#pragma unroll
    for (int i = 0; i < kPer / n; ++i) {
      if (base + (i + 1) * 64 * n <= V) continue;  // uniform
      const int shift = base + (i * 64 + lane) * n - (V - n);
#pragma unroll
      for (int b = 1; b < n; b *= 2)
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (shift > 0 && (shift & b)) x[i * n + e] = e + b < n ? x[i * n + e + b] : -INFINITY;
#pragma unroll
      for (int e = 0; e < n; ++e)
        if (shift >= n) x[i * n + e] = -INFINITY;
    }
  }
}

// Orders a wave's own LDS writes before its later LDS reads by other lanes
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

// The k best (value descending, id ascending) of two entries a lane, values by
// their order (none: kNone); lane r < k ends with the r-th, kNone where there is none
constexpr int kNone = INT_MIN;
__device__ __forceinline__ bool before(int va, int ia, int vb, int ib) { return va > vb || (va == vb && ia < ib); }
__device__ __forceinline__ void pick_best(int v0, int i0, int v1, int i1, int k, int lane, int &v, int &id) {
  v = kNone;
  id = -1;
  for (int r = 0; r < k; ++r) {
    const bool second = before(v1, i1, v0, i0);
    const int b = second ? v1 : v0;
    const int w = wave_max(b);
    if (w == kNone) break;
    const int bi = wave_min(b == w ? (second ? i1 : i0) : INT_MAX);
    if (lane == r) {
      v = w;
      id = bi;
    }
    if (v0 == w && i0 == bi) v0 = kNone;
    if (v1 == w && i1 == bi) v1 = kNone;
  }
}

// The candidates for the k best of the columns a wave has seen: a list in LDS that
// holds at least k (or all there are) which are no less than `floor`, and all that
// are greater; -infinity is none
struct Best {
  int *val, *id;  // (order, column)
  int count;      // uniform, as the floor
  float floor;
};

// keeps the k best of the list, in order
__device__ __forceinline__ void best_shrink(Best &b, int k, int lane) {
  wave_lds_sync();
  const bool h0 = lane < b.count, h1 = lane + 64 < b.count;
  const int v0 = h0 ? b.val[lane] : kNone, v1 = h1 ? b.val[lane + 64] : kNone;
  const int i0 = h0 ? b.id[lane] : INT_MAX, i1 = h1 ? b.id[lane + 64] : INT_MAX;
  int v, id;
  if (b.count <= 24) {
    // few: each counts those before it, a third of a round of pick_best a candidate
    int rank = 0;
    for (int c = 0; c < b.count; ++c)
      rank += before(__builtin_amdgcn_readlane(v0, c), __builtin_amdgcn_readlane(i0, c), v0, i0) ? 1 : 0;
    wave_lds_sync();
    if (h0) {
      b.val[rank] = v0;
      b.id[rank] = i0;
    }
    wave_lds_sync();
    v = b.val[lane];
    id = b.id[lane];
  } else {
    pick_best(v0, i0, v1, i1, k, lane, v, id);
  }
  wave_lds_sync();
  b.count = min(b.count, k);
  if (lane < b.count) {
    b.val[lane] = v;
    b.id[lane] = id;
  }
  if (b.count == k) b.floor = of_order(__builtin_amdgcn_readlane(v, k - 1));
  wave_lds_sync();
}

// the columns of one more chunk, which lie behind all seen before; top: of the lane's,
// chunk_top: of the chunk's; trim: candidates above which the list is cut to raise
// the floor
template <class T>
__device__ __forceinline__ void best_take(Best &b, const float (&x)[kPer], float top, float chunk_top, int base, int k,
                                          int trim, int lane, bool first) {
  float above = b.floor;  // a column behind the k that are no less than the floor has to exceed it
  if (first) {
    // the k-th largest of the lanes' maxima: at least k columns are no less
    int left = order_of(top), at = order_of(chunk_top);
    for (int r = 1; r < k; ++r) {
      if (lane == __builtin_ctzll(__ballot(left == at))) left = kNone;
      at = wave_max(left);
    }
    b.floor = of_order(at);
    above = of_order(at == 0 ? -2 : at - 1);  // the float below (-1 is -0)
    if (!(b.floor > -INFINITY)) b.floor = above = -INFINITY;  // fewer lanes than k hold any
  } else if (!(chunk_top > above)) {
    return;
  }
  // (the comparisons first, then the few that hold anything: 16 comparisons with a
  // branch each 173 -> 180 us for 76800 rows of 4096 in bf16, 4 alternatives)
  unsigned long long mask[kPer];
  int more = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    mask[j] = __ballot(x[j] > above);
    more += __popcll(mask[j]);
  }
  if (b.count + more <= kList) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (!mask[j]) continue;
      if (x[j] > above) {
        const int at = b.count + __builtin_amdgcn_mbcnt_hi(mask[j] >> 32, __builtin_amdgcn_mbcnt_lo((uint32_t)mask[j], 0));
        b.val[at] = order_of(x[j]);
        b.id[at] = column<T>(base, lane, j);
      }
      b.count += __popcll(mask[j]);
    }
    if (b.count > trim) best_shrink(b, k, lane);
    return;
  }
  // many candidates (long runs of equal or rising values): the k best so far, and the
  // chunk's k best one by one, each the best behind the one before
  if (b.count > k) best_shrink(b, k, lane);
  int last_v = INT_MAX, last_id = -1;
  for (int r = 0; r < k; ++r) {
    int v = kNone, id = INT_MAX;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int o = order_of(x[j]), c = column<T>(base, lane, j);
      if (x[j] > -INFINITY && before(last_v, last_id, o, c) && before(o, c, v, id)) {
        v = o;
        id = c;
      }
    }
    last_v = wave_max(v);
    if (last_v == kNone) break;
    last_id = wave_min(v == last_v ? id : INT_MAX);
    if (lane == 0) {
      b.val[b.count] = last_v;
      b.id[b.count] = last_id;
    }
    ++b.count;
  }
  best_shrink(b, k, lane);
}

struct ScoreArgs {
  const void *logits;
  const int32_t *tokens, *parents;
  float *logp, *entropy, *lse, *top_logp;
  int32_t *top_tokens;
  int64_t stride;
  int32_t M, B, V, k;
};

// W waves a row of logits: 4 rows a workgroup of 256 lanes with one wave each, else
// one.  A row is looked at once for all the tokens that were chosen on it (a beam's
// slots share parents: 300 frames of 64 x 4 slots with random parents are chosen on two
// thirds of the rows, 185 us token by token and 166 so); a row nothing was chosen on is not.
// Bound by memory in fp32 (25600 rows of 1024: 19 us without alternatives, 5.4 TB/s)
// and by the vector units where alternatives are asked for or values are 16 bits (busy
// 73 % of the time on the beam above, 85 % on 16000 x 8190 in bf16).
// (32 values a lane instead of 16: half the waves fit, 173 -> 204 us for 76800 rows
// of 4096 in bf16 with 4 alternatives.)
// beam: there are parents.
template <class T, int W, bool beam>
__global__ void __launch_bounds__(W == 1 ? 256 : 64 * W) score_kernel(ScoreArgs p) {
  constexpr int kWaves = W == 1 ? 4 : W;
  __shared__ int s_val[kWaves][kList];
  __shared__ int s_id[kWaves][kList];
  __shared__ Stat s_stat[kWaves];
  __shared__ int s_count[kWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row_at = W == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  if (row_at >= p.M) return;  // whole waves, and with W > 1 none
  const int r = (int)row_at;
  const float nan = __int_as_float(0x7FC00000);

  // The tokens chosen on this row: lane i looks at slot i of the row's stream
  const int slots = beam ? p.B : 1, first = beam ? r / p.B * p.B : r, m = first + lane;
  const T *row = static_cast<const T *>(p.logits) + r * p.stride;
  int par = lane, tok = -1;
  if (lane < slots) {
    if (beam) par = p.parents[m];
    if (p.tokens) tok = p.tokens[m];
  }
  const bool bad_token = tok < -1 || tok >= p.V;
  const bool mine = lane < slots && (!beam || par == r - first);
  const unsigned long long any = beam ? __ballot(mine) : 1;
  if (beam) {
    const bool bad_parent = par < -1 || par >= slots;
    if (wave % W == 0 && lane == r - first && (par == -1 || bad_parent)) {
      // the slot of the row's own number is dead: nobody else writes its outputs
      if (p.logp) p.logp[r] = bad_token || bad_parent ? nan : 0.0f;
      if (p.entropy) p.entropy[r] = bad_parent ? nan : 0.0f;
      if (p.lse) p.lse[r] = bad_parent ? nan : -INFINITY;
      for (int j = 0; j < p.k; ++j) {
        p.top_tokens[(int64_t)r * p.k + j] = -1;
        p.top_logp[(int64_t)r * p.k + j] = bad_parent ? nan : -INFINITY;
      }
      if (bad_token || bad_parent) atomicOr(&g_score_status, FUSION_STATUS_BAD_TOKEN);
    }
    if (!any) return;  // (the same in every wave of the row)
  }
  float x_tok = 0.0f;
  if (mine && wave % W == 0 && tok >= 0 && !bad_token) x_tok = to_float(row[tok]);
  WaveStat ws = wave_stat_none();
  Best b{s_val[wave], s_id[wave], 0, -INFINITY};
  const int start = (W == 1 ? 0 : wave) * kChunk;
  // Raising the floor now and then pays over 8 chunks or more with many alternatives
  // (us, 8 of them: 513 x 100003 53 -> 45, 16000 x 8190 82 -> 75, but 3000 x 8190
  // with 4 waves a row 27.1 -> 27.7), not where a row's own time counts (16 x 131072
  // with 16 waves 23.6 -> 25.6)
  const int trim = W <= 8 && p.k > 4 && p.V >= 8 * W * kChunk - kChunk / 2 ? 6 * p.k : kList;
  for (int base = start; base < p.V; base += W * kChunk) {
    float x[kPer];
    load_chunk(row, p.V, base, lane, x);
    float top = fmaxf(x[0], -INFINITY);
#pragma unroll
    for (int j = 1; j < kPer; ++j) top = fmaxf(top, x[j]);
    const float chunk_top = wave_max(top);
    if (p.k) best_take<T>(b, x, top, chunk_top, base, p.k, trim, lane, base == start);
    wave_stat_take(ws, x, top, chunk_top);
  }
  Stat s = wave_stat_done(ws);
  if (p.k && (b.count > 0 || W == 1)) best_shrink(b, p.k, lane);
  int v = kNone, id = -1;
  if (W > 1) {
    if (lane == 0) {
      s_stat[wave] = s;
      s_count[wave] = b.count;
    }
    __syncthreads();
    if (wave != 0) return;
    s = lane < W ? s_stat[lane] : stat_none();
    stat_wave(s);
    if (p.k) {
      int ev[2], ei[2];
      for (int q = 0; q < 2; ++q) {
        const int w = (lane + 64 * q) / FUSION_MAX_K, at = (lane + 64 * q) % FUSION_MAX_K;
        const bool has = w < W && at < s_count[w < W ? w : 0];
        ev[q] = has ? s_val[w][at] : kNone;
        ei[q] = has ? s_id[w][at] : INT_MAX;
      }
      pick_best(ev[0], ei[0], ev[1], ei[1], p.k, lane, v, id);
    }
  } else if (lane < b.count) {
    v = b.val[lane];
    id = b.id[lane];
  }
  const RowScore q = row_score(s);
  if (p.k) {
    const int top = q.bad ? -1 : id;
    const float top_logp = q.bad ? nan : id < 0 ? -INFINITY : row_logp(q, of_order(v));
    for (unsigned long long todo = any; todo; todo &= todo - 1) {
      const int64_t at = (int64_t)(first + (beam ? __builtin_ctzll(todo) : 0)) * p.k + lane;
      if (lane < p.k) {
        p.top_tokens[at] = top;
        p.top_logp[at] = top_logp;
      }
    }
  }
  if (mine) {
    if (p.logp) p.logp[m] = bad_token ? nan : tok < 0 ? 0.0f : row_logp(q, x_tok);
    if (p.entropy) p.entropy[m] = q.entropy;
    if (p.lse) p.lse[m] = q.lse;
    if (bad_token) atomicOr(&g_score_status, FUSION_STATUS_BAD_TOKEN);
  }
}

struct GradArgs {
  const void *logits;
  const int32_t *tokens, *parents;
  const float *logp, *entropy, *lse, *g_logp, *g_entropy;
  void *grad;
  int64_t stride, g_stride;
  int32_t M, B, V, parts;  // parts: waves a row
};

// A wave takes every parts-th chunk of 1024 columns of a row.  Bound by memory: 16000
// x 8190 in bf16 79 us, 262 MB in and as much out, 6.6 TB/s.  The stores are streaming
// ones (105 us without), and waves that stay for several chunks pay for their tokens'
// look-up once (1024 columns a wave: 140 us).
template <class T>
__global__ void __launch_bounds__(256) grad_kernel(GradArgs p) {
  constexpr int n = Pack<T>::n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t job = (int64_t)blockIdx.x * 4 + wave;
  if (job >= (int64_t)p.M * p.parts) return;
  const int r = (int)(job / p.parts), part = (int)(job % p.parts);
  int parts = p.parts;
  const T *row = static_cast<const T *>(p.logits) + r * p.stride;
  T *out = static_cast<T *>(p.grad) + r * p.g_stride;

  // The tokens chosen on this row: lane i looks at slot i of the row's stream
  const int slots = p.parents ? p.B : 1, first = p.parents ? r / p.B * p.B : r;
  const int at = first + lane;
  bool mine = lane < slots, bad = false;
  if (mine && p.parents) {
    const int par = p.parents[at];
    bad = par < -1 || par >= p.B;
    mine = par == r - first;
  }
  int tok = -1;
  float gl = 0.0f, ge = 0.0f, lp_tok = 0.0f, lse = 0.0f, H = 0.0f;
  const bool told = p.tokens && p.logp;
  if (lane < slots && told) tok = p.tokens[at];  // of dead slots too: one out of range is told of
  if (mine) {
    lse = p.lse[at];
    if (told) lp_tok = p.logp[at];
    if (p.g_logp) gl = p.g_logp[at];
    if (p.g_entropy) {
      ge = p.g_entropy[at];
      H = p.entropy[at];
    }
  }
  bad |= tok < -1 || tok >= p.V;
  if (!mine || tok < 0 || tok >= p.V) {
    tok = -1;
    gl = 0.0f;
  }
  const unsigned long long any = __ballot(mine);
  if (__ballot(bad) && lane == 0) atomicOr(&g_score_status, FUSION_STATUS_BAD_TOKEN);
  const int one = any ? __builtin_ctzll(any) : 0;  // the row's statistics are the same for all its tokens
  lse = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(lse), one));
  H = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(H), one));
  const float GL = wave_add(gl), GE = wave_add(ge);
  // What the rounding of lse left out: x - log p of a token is the same value in full,
  // and its logit x is the one of type T nearest to lse + log p (the logits themselves may
  // be overwritten already).  From the likeliest token, where its log p is short enough
  // to be the better one; else 0.
  const bool tells = tok >= 0 && 4.0f * fabsf(lp_tok) <= fabsf(lse);
  float fix = 0.0f;
  if (__ballot(tells)) {
    T x_tok;
    from_float(lse + lp_tok, x_tok);
    fix = (lse - to_float(x_tok)) + lp_tok;
    const int at_most = tells ? order_of(lp_tok) : INT_MIN, best = wave_max(at_most);
    fix = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(fix), __builtin_ctzll(__ballot(at_most == best))));
  } else if ((GL != 0.0f || GE != 0.0f) && fabsf(lse) >= 4096.0f && fabsf(lse) < INFINITY) {
    // no token tells, and p would be off by 2^-12 or more: m and log s once more.  One
    // wave takes the row, which in place no other may overwrite meanwhile.
    if (part != 0) return;
    parts = 1;
    WaveStat ws = wave_stat_none();
    for (int base = 0; base < p.V; base += kChunk) {
      float x[kPer];
      load_chunk(row, p.V, base, lane, x);
      float top = fmaxf(x[0], -INFINITY);
#pragma unroll
      for (int j = 1; j < kPer; ++j) top = fmaxf(top, x[j]);
      wave_stat_take(ws, x, top, wave_max(top));
    }
    const RowScore q = row_score(wave_stat_done(ws));
    fix = (lse - q.m) - q.log_s;
  }
  const float by = exp_of(fix), GLf = GL * by, GEf = GE * by, Hf = H + fix;
  const bool nothing = !any || lse == -INFINITY;  // an empty row's outputs are constant

  for (int base = part * kChunk; base < p.V; base += parts * kChunk) {
    const bool whole = base + kChunk <= p.V;
    float x[kPer];
    if (nothing) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) x[j] = 0.0f;
    } else {
      if (whole) {
        Pack<T> q[kPer / n];
#pragma unroll
        for (int i = 0; i < kPer / n; ++i) __builtin_memcpy(&q[i], row + base + (i * 64 + lane) * n, 16);
#pragma unroll
        for (int j = 0; j < kPer; ++j) x[j] = to_float(q[j / n].v[j % n]);
      } else {
        // (a lane reads its own columns alone: where the gradient is written in
        // place, others are already overwritten)
#pragma unroll
        for (int i = 0; i < kPer / n; ++i) {
          const int c = base + (i * 64 + lane) * n;
          if (c + n <= p.V) {
            Pack<T> q;
            __builtin_memcpy(&q, row + c, 16);
#pragma unroll
            for (int e = 0; e < n; ++e) x[i * n + e] = to_float(q.v[e]);
          } else {
#pragma unroll
            for (int e = 0; e < n; ++e) x[i * n + e] = c + e < p.V ? to_float(row[c + e]) : -INFINITY;
          }
        }
      }
      if (GE == 0.0f) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) x[j] = -exp_of(x[j] - lse) * GLf;
      } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const float lp = x[j] - lse;
          x[j] = -exp_of(lp) * (GLf + GEf * (fmaxf(lp, kFar) + Hf));
        }
      }
      // the tokens' own columns, from their log probabilities: 1 - p is lost in x - lse where p is near 1
      unsigned long long todo = __ballot(tok >= base && tok < base + kChunk);
      while (todo) {
        const int i = __builtin_ctzll(todo);
        const int y = __builtin_amdgcn_readlane(tok, i);
        const float lp = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(lp_tok), i));
        const bool same = tok == y;
        const float own = wave_add(same ? gl : 0.0f), others = wave_add(same ? 0.0f : gl);
        const float e = exp_of(lp), g = own * -expm1f(lp) - e * (others + GE * (fmaxf(lp, kFar) + H));
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (column<T>(base, lane, j) == y) x[j] = g;
        todo &= ~__ballot(same);
      }
    }
#pragma unroll
    for (int i = 0; i < kPer / n; ++i) {
      const int c = base + (i * 64 + lane) * n;
      if (whole || c + n <= p.V) {
        Pack<T> q;
#pragma unroll
        for (int e = 0; e < n; ++e) from_float(x[i * n + e], q.v[e]);
        // (streaming: nothing reads it back soon)
        __builtin_nontemporal_store(__builtin_bit_cast(Words, q), reinterpret_cast<UnalignedWords *>(out + c));
      } else {
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (c + e < p.V) from_float(x[i * n + e], out[c + e]);
      }
    }
  }
}

}  // namespace

int score_status_word(int32_t **word) {
  void *p = nullptr;
  const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(g_score_status));
  if (e != hipSuccess) return hip_error(e, "hipGetSymbolAddress");
  *word = static_cast<int32_t *>(p);
  return FUSION_OK;
}

namespace {
constexpr int64_t kMaxRows = (1 << 24) - 1;
constexpr int64_t kGradWaves = 1 << 16;  // enough to fill the chip several times
// the checks that scoring and its gradient share
int check_rows(int32_t dtype, int64_t stride, int32_t T, int32_t S, int32_t B, int32_t V, const void *parents) {
  if (dtype != FUSION_F32 && dtype != FUSION_BF16 && dtype != FUSION_F16) return set_error(FUSION_E_ARG, "unknown dtype");
  if (T < 0 || S < 0 || B < 1) return set_error(FUSION_E_ARG, "T, S or B out of range");
  if (parents && B > FUSION_MAX_BEAM) return set_error(FUSION_E_UNSUPPORTED, "parents of more than FUSION_MAX_BEAM slots");
  if (V < 1 || V > FUSION_MAX_SCORED_VOCAB) return set_error(FUSION_E_ARG, "V out of range");
  if (stride < V) return set_error(FUSION_E_ARG, "rows overlap: stride below V");
  const int64_t H = (int64_t)S * B;
  // (a launch holds fewer than 2^32 lanes)
  if (H > kMaxRows || (H > 0 && T > kMaxRows / H)) return set_error(FUSION_E_UNSUPPORTED, "more than 2^24 - 1 rows");
  // the last row's end within a 63-bit byte offset
  if (stride > (INT64_MAX >> 3) / (H > 0 && T > 0 ? T * H : 1)) return set_error(FUSION_E_ARG, "stride out of range");
  return FUSION_OK;
}
}  // namespace

}  // namespace fusion

using namespace fusion;

extern "C" int token_logprobs(const void *logits, int32_t dtype, int64_t stride, int32_t T, int32_t S, int32_t B,
                              int32_t V, const int32_t *tokens, const int32_t *parents, int32_t k, float *logp,
                              float *entropy, float *lse, int32_t *top_tokens, float *top_logp, hipStream_t stream) {
  const int rc = check_rows(dtype, stride, T, S, B, V, parents);
  if (rc != FUSION_OK) return rc;
  if (k < 0 || k > FUSION_MAX_K) return set_error(FUSION_E_ARG, "k out of range");
  const int64_t M = (int64_t)T * S * B;
  if (M == 0) return FUSION_OK;
  if (!logits) return set_error(FUSION_E_ARG, "NULL logits");
  if ((uintptr_t)logits % (dtype == FUSION_F32 ? 4 : 2) != 0) return set_error(FUSION_E_ARG, "misaligned logits");
  if (logp && !tokens) return set_error(FUSION_E_ARG, "log probabilities of NULL tokens");
  if (k > 0 && (!top_tokens || !top_logp)) return set_error(FUSION_E_ARG, "NULL buffer for the alternatives");
  if (!logp && !entropy && !lse && k == 0) return set_error(FUSION_E_ARG, "no output buffer");
  const ScoreArgs p{logits, logp ? tokens : nullptr, parents, logp, entropy, lse, top_logp, top_tokens, stride, (int32_t)M,
                    B, V, k};
  auto launch = [&](auto type, auto beam_) {
    using T_ = decltype(type);
    constexpr bool beam = decltype(beam_)::value;
    // Waves a row, enough rows or chunks to fill the chip (us; fp32, 4 alternatives):
    //                 1      4      8      16
    //    6000 x 2500  17.4   27.2                 (a wave alone joins nothing)
    //    3000 x 4096  13.7   17.8
    //    3000 x 8190  23.3   24.1                 (35.4 and 29.4 with 8 alternatives)
    //    1500 x 8190         12.9   16.4          (bf16)
    //    600 x 8190          9.4    9.5    14.5
    //    300 x 32000         19.9   15.4   18.0
    //    513 x 100003        54     40     50     (bf16)
    if (M >= 4096 || (M >= 2048 && V <= 4 * kChunk) || V <= kChunk)
      hipLaunchKernelGGL((score_kernel<T_, 1, beam>), dim3((unsigned)((M + 3) / 4)), dim3(256), 0, stream, p);
    else if (M >= 1024 || V <= 4 * kChunk)
      hipLaunchKernelGGL((score_kernel<T_, 4, beam>), dim3((unsigned)M), dim3(256), 0, stream, p);
    else if (M >= 256 || V <= 8 * kChunk)
      hipLaunchKernelGGL((score_kernel<T_, 8, beam>), dim3((unsigned)M), dim3(512), 0, stream, p);
    else
      hipLaunchKernelGGL((score_kernel<T_, 16, beam>), dim3((unsigned)M), dim3(1024), 0, stream, p);
  };
  auto go = [&](auto type) { parents ? launch(type, std::true_type{}) : launch(type, std::false_type{}); };
  if (dtype == FUSION_F32) go(float{});
  else if (dtype == FUSION_BF16) go(Brain{});
  else go(Half{});
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FUSION_OK : hip_error(e, "token scoring launch");
}

extern "C" int token_logprobs_backward(const void *logits, int32_t dtype, int64_t stride, int32_t T, int32_t S, int32_t B,
                                       int32_t V, const int32_t *tokens, const int32_t *parents, const float *logp,
                                       const float *entropy, const float *lse, const float *grad_logp,
                                       const float *grad_entropy, void *grad_logits, int64_t grad_stride,
                                       hipStream_t stream) {
  const int rc = check_rows(dtype, stride, T, S, B, V, parents);
  if (rc != FUSION_OK) return rc;
  if (check_rows(dtype, grad_stride, T, S, B, V, parents) != FUSION_OK)
    return set_error(FUSION_E_ARG, "gradient rows overlap or their stride is out of range");
  const int64_t M = (int64_t)T * S * B;
  if (M == 0) return FUSION_OK;
  if (!logits || !grad_logits || !lse) return set_error(FUSION_E_ARG, "NULL logits, gradient or lse");
  if (((uintptr_t)logits | (uintptr_t)grad_logits) % (dtype == FUSION_F32 ? 4 : 2) != 0)
    return set_error(FUSION_E_ARG, "misaligned logits or gradient");
  if (!grad_logp && !grad_entropy) return set_error(FUSION_E_ARG, "no incoming gradient");
  if (grad_logp && (!tokens || !logp)) return set_error(FUSION_E_ARG, "gradient of the log probabilities without tokens or logp");
  if (grad_entropy && !entropy) return set_error(FUSION_E_ARG, "gradient of the entropy without entropy");
  if (logits == grad_logits && stride != grad_stride) return set_error(FUSION_E_ARG, "in place with another stride");
  const int chunks = (V + kChunk - 1) / kChunk;
  const int parts = (int)std::min<int64_t>(chunks, std::max<int64_t>(1, kGradWaves / M));
  const int64_t blocks = (M * parts + 3) / 4;
  const GradArgs p{logits, tokens, parents, logp, entropy, lse, grad_logp, grad_entropy, grad_logits, stride, grad_stride,
                   (int32_t)M, B, V, parts};
  const dim3 grid((unsigned)blocks), block(256);
  if (dtype == FUSION_F32) hipLaunchKernelGGL(grad_kernel<float>, grid, block, 0, stream, p);
  else if (dtype == FUSION_BF16) hipLaunchKernelGGL(grad_kernel<Brain>, grid, block, 0, stream, p);
  else hipLaunchKernelGGL(grad_kernel<Half>, grid, block, 0, stream, p);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FUSION_OK : hip_error(e, "token scoring gradient launch");
}
