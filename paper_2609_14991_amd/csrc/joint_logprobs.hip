// Log probabilities of given tokens straight from the joint network's hidden
// states: the projection of joint_proj.hip whose logits are never stored.
//
// A tile of logits, x = bias + A W^T, leaves as the softmax statistics of its rows
// (wave_ops.h's Stat, 16 bytes a row instead of 4 a logit); a second kernel joins a
// token's row over the column tiles and computes the token's own logit again, by
// the same matrix instructions over the same steps of K, so that it is the value
// which the statistics contain, to the bit.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "fusion_internal.h"
#include "joint_tile.h"
#include "score_status.h"
#include "wave_ops.h"

namespace fusion {
namespace {

// Statistics of a row's 16 TN logits in four lanes (l, l ^ 16, l ^ 32, l ^ 48), in
// all of them.  Four operations a logit, the exponential among them: (x - m) log2 e is
// one fma of x, off by what the rounding of m log2 e left, the same for the whole row,
// and the sums are put right by it.  The maxima are counted as one, the sum less 1: the
// sum's roundings (24 halves of a last place at most) are 2.4e-5 or less of a rest of 1/16
// or more, whatever m is.  Where the rest is less (one logit far above the row's others),
// a logit is -infinity (0 times it leaves u NaN) or the largest is past 2800 (the
// shift past 4096, its rounding past 2^-12), once more with care.
template <int TN>
__device__ __forceinline__ Stat tile_row_stat(const f32x4 (&x)[TN]) {
  float top = x[0][0];
#pragma unroll
  for (int j = 1; j < 4 * TN; ++j) top = fmaxf(top, x[j / 4][j % 4]);
  Stat s{across_rows(top, [](float a, float b) { return fmaxf(a, b); }), 1.0f, 0.0f, 0.0f};
  const float shift = -s.m * kLog2e, off = fmaf(-s.m, kLog2e, -shift);
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < 4 * TN; ++j) {
    const float t = fmaf(x[j / 4][j % 4], kLog2e, shift), e = __builtin_amdgcn_exp2f(t);
    sum += e;
    s.u = fmaf(t, e, s.u);
  }
  const auto add = [](float a, float b) { return a + b; };
  sum = across_rows(sum, add);
  const float by = fmaf(off, kLn2, 1.0f);  // 2^off, to 2^-25 for an |off| up to 2^-12
  s.rest = fmaf(sum, by, -1.0f);
  s.u = fmaf(off, sum, across_rows(s.u, add)) * (by * kLn2);
  if (__ballot(s.u != s.u || !(s.rest >= 0.0625f && fabsf(shift) < 4096.0f))) {
    float v[4 * TN];
#pragma unroll
    for (int j = 0; j < 4 * TN; ++j) v[j] = x[j / 4][j % 4];
    Stat c = stat_none();
    stat_take(c, v, s.m);
    s = Stat{s.m, across_rows(c.ones, add), across_rows(c.rest, add), across_rows(c.u, add)};
  }
  return s;
}

struct StatArgs {
  const uint16_t *A, *W;
  const float *bias;
  float *part;  // [column tiles][4][M] (m, ones, rest, u)
  int M, N, K, n_col_tiles, map;
};

// A workgroup a tile, as joint_proj_kernel.  76800 x 4096 x 640: 377 us back to back
// (1.07 PFLOP/s; the logits' projection alone, with its stores, 456), of which the
// products take 290 and the statistics behind them the rest: with 128 KB of stages a
// CU holds one workgroup, and nothing runs beside its vector work.  What would overlap
// the two was slower: workgroups that go on from tile to tile with the next one's stages
// under way (438), two of 128 x 256 tiles a CU in stages of half the size (400).
template <class S>
__global__ void __launch_bounds__(64 * S::waves, 2) joint_stat_kernel(StatArgs p) {
  static_assert(S::lds >= S::BM * S::WN * 16, "LDS too small for the statistics");
  __shared__ __align__(1024) unsigned char smem[S::lds];
  int tr, tc;
  tile_place(p.map, p.n_col_tiles, tr, tc);
  const int bm = tr * S::BM, bn = tc * S::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fc = lane >> 4;
  const int wm = (wave / S::WN) * S::RM, wn = (wave % S::WN) * S::RN;
  // the sums start at the bias: lane l holds row l % 16 of each 16 x 16 tile, columns
  // 4 * (l / 16) .. + 3
  f32x4 acc[S::TM][S::TN];
  Bf16Op op;
  tile_product<S>(op, smem, p.A, p.W, p.M, p.N, p.K * 2, bm, bn, acc, [&](auto &c) {
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      f32x4 b;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = bn + wn + j * 16 + fc * 4 + r;
        b[r] = p.bias && n < p.N ? p.bias[n] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < S::TM; ++i) c[i][j] = b;
    }
  });
  // columns past N are -infinity (not from the start: their weights are zeros, and a
  // state that is not finite times 0 would make them NaN)
  if (bn + S::BN > p.N) {
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      if (bn + wn + j * 16 + 16 <= p.N) continue;  // uniform
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (bn + wn + j * 16 + fc * 4 + r >= p.N)
#pragma unroll
          for (int i = 0; i < S::TM; ++i) acc[i][j][r] = -INFINITY;
    }
  }

  wait_barrier<0>();  // every wave has read the last stage
  f32x4 *stat = reinterpret_cast<f32x4 *>(smem);
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
    const Stat s = tile_row_stat<S::TN>(acc[i]);
    if (fc == 0) stat[(wm + i * 16 + fr) * S::WN + wave % S::WN] = f32x4{s.m, s.ones, s.rest, s.u};
  }
  __syncthreads();
  for (int row = threadIdx.x; row < S::BM; row += 64 * S::waves) {
    if (bm + row >= p.M) break;
    Stat v[S::WN];
#pragma unroll
    for (int q = 0; q < S::WN; ++q) {
      const f32x4 w = stat[row * S::WN + q];
      v[q] = Stat{w[0], w[1], w[2], w[3]};
    }
    const Stat s = stat_of(v);
    float *o = p.part + (int64_t)tc * 4 * p.M + bm + row;
    o[0] = s.m;
    o[p.M] = s.ones;
    o[2 * (int64_t)p.M] = s.rest;
    o[3 * (int64_t)p.M] = s.u;
  }
}

struct JoinArgs {
  const uint16_t *A, *W;
  const float *bias, *part;
  const int32_t *tokens, *parents;
  float *logp, *entropy, *lse;
  int32_t *status;  // scoring's word: bit set when a token or parent is out of range
  int32_t M, N, K, B, n_col_tiles;
};

// A wave computes the logits of 16 tokens; `split` waves join the column tiles of
// their rows, four lanes a row each.  One wave a group for many tokens; four where
// there are few and each waits for its loads alone (256 tokens of 64 column tiles:
// 4.6 us, 12 with one wave and its loads one after the other).  76800 tokens 24 us, by
// their hidden states and weight rows (196 MB); picking the tokens' logits out of the
// tiles instead cost those 31 us.
template <int split>
__global__ void __launch_bounds__(256) joint_join_kernel(JoinArgs p) {
  static_assert(split == 1 || split == 4, "one wave a group of 16 tokens, or the workgroup");
  constexpr int groups = 4 / split;  // of 16 tokens a workgroup
  __shared__ f32x4 s_part[4][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fc = lane >> 4;
  const int64_t at = ((int64_t)blockIdx.x * groups + wave / split) * 16 + fr;
  const bool here = at < p.M;
  const int m = here ? (int)at : 0;
  const int64_t r = here ? row_of_token(p.parents, m, p.B) : -1;
  const int tok = here && p.tokens ? p.tokens[m] : -1;
  const bool bad_token = tok < -1 || tok >= p.N, scored = r >= 0 && tok >= 0 && !bad_token;

  Stat s = stat_none();
  if (r >= 0) {
    constexpr int kAhead = 4;
    for (int c = wave % split * 4 + fc; c < p.n_col_tiles; c += 4 * split * kAhead) {
      Stat v[kAhead];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        const float *o = p.part + (int64_t)min(c + 4 * split * q, p.n_col_tiles - 1) * 4 * p.M + r;
        v[q] = Stat{o[0], o[p.M], o[2 * (int64_t)p.M], o[3 * (int64_t)p.M]};
      }
#pragma unroll
      for (int q = 0; q < kAhead; ++q)
        if (c + 4 * split * q < p.n_col_tiles) stat_join(s, v[q]);
    }
  }
  s = stat_across(s);
  if (split > 1) {
    if (fc == 0) s_part[wave][fr] = f32x4{s.m, s.ones, s.rest, s.u};
    __syncthreads();
    if (wave != 0) return;
    const f32x4 v = s_part[fc][fr];
    s = stat_across(Stat{v[0], v[1], v[2], v[3]});
  }

  // the token's logit: of the 16 x 16 products of the wave's hidden states and
  // weight rows, those on the diagonal
  float x = 0.0f;
  if (p.logp) {
    const __amdgpu_buffer_rsrc_t ra = rsrc(p.A, (uint32_t)((int64_t)p.M * p.K * 2));
    const __amdgpu_buffer_rsrc_t rw = rsrc(p.W, (uint32_t)((int64_t)p.N * p.K * 2));
    const float b = scored && p.bias ? p.bias[tok] : 0.0f;
    f32x4 acc = {b, b, b, b};
    const uint32_t oa = scored ? (uint32_t)(r * p.K * 2) : kOutside, ow = scored ? (uint32_t)((int64_t)tok * p.K * 2) : kOutside;
    // the loads of 10 steps at a time: one step after the other they would be most of the time
    constexpr int kSteps = 10;
    for (int k = 0; k < p.K; k += 32 * kSteps) {
      i32x4 a[kSteps], w[kSteps];
#pragma unroll
      for (int q = 0; q < kSteps; ++q) {
        const int e = k + q * 32 + fc * 8;
        const bool in = e < p.K && scored;
        a[q] = __builtin_amdgcn_raw_buffer_load_b128(ra, in ? oa + e * 2 : kOutside, 0, 0);
        w[q] = __builtin_amdgcn_raw_buffer_load_b128(rw, in ? ow + e * 2 : kOutside, 0, 0);
      }
#pragma unroll
      for (int q = 0; q < kSteps; ++q)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[q]), __builtin_bit_cast(bf16x8, a[q]), acc, 0,
                                                      0, 0);
    }
    const float d = (fr & 3) == 0 ? acc[0] : (fr & 3) == 1 ? acc[1] : (fr & 3) == 2 ? acc[2] : acc[3];
    x = __shfl(d, fr + 16 * (fr >> 2));
  }
  if (fc != 0 || !here) return;
  const RowScore q = row_score(s);
  const float nan = __int_as_float(0x7FC00000);
  const bool bad = bad_token || r == -2;
  if (p.logp) p.logp[m] = bad ? nan : !scored ? 0.0f : row_logp(q, x);
  if (p.entropy) p.entropy[m] = r == -2 ? nan : q.entropy;
  if (p.lse) p.lse[m] = r == -2 ? nan : q.lse;
  if (bad) atomicOr(p.status, FUSION_STATUS_BAD_TOKEN);
}

constexpr TileShape<2, 4, 8, 4, 2> t256{};
constexpr TileShape<2, 2, 4, 4, 2> t128{};
constexpr TileShape<2, 2, 2, 4, 3> t64x128{};
constexpr TileShape<2, 2, 2, 2, 4> t64{};
constexpr TileShape<2, 2, 1, 2, 4> t32{};
constexpr int64_t kCus = 256;

template <class C>
int64_t tiles(C, int M, int N) {
  return (int64_t)((M + C::BM - 1) / C::BM) * ((N + C::BN - 1) / C::BN);
}

// The largest tile that fills the chip.  (Of joint_project's rules the plain ones; its
// finer ones follow its stores, and are not measured here.)
template <class F>
auto with_shape(int M, int N, F f) {
  if (tiles(t256, M, N) >= 1000 && N > 128) return f(t256);
  if (tiles(t128, M, N) > kCus) return f(t128);
  if (tiles(t64x128, M, N) > kCus) return f(t64x128);
  if (tiles(t64, M, N) > kCus) return f(t64);
  return f(t32);
}

// four statistics of each row and column tile
int64_t workspace(int M, int N) {
  return with_shape(M, N, [&](auto c) { return (int64_t)((N + decltype(c)::BN - 1) / decltype(c)::BN) * 4 * M; });
}

int check_sizes(int64_t M, int32_t N, int32_t K) {
  if (M < 0 || N < 1 || K < 8) return set_error(FUSION_E_ARG, "sizes out of range");
  if (K % 8 != 0) return set_error(FUSION_E_UNSUPPORTED, "K must be a multiple of 8");
  if (M > 0x7FFFFFF0ll / 2 / K || (int64_t)N * K * 2 > 0x7FFFFFF0ll)
    return set_error(FUSION_E_UNSUPPORTED, "operand larger than 2 GiB: split the call along T");
  return FUSION_OK;
}

}  // namespace

}  // namespace fusion

using namespace fusion;

extern "C" int joint_logprobs_workspace(int32_t M, int32_t V, int32_t K, int64_t *floats) {
  if (!floats) return set_error(FUSION_E_ARG, "NULL output");
  const int rc = check_sizes(M, V, K);
  if (rc != FUSION_OK) return rc;
  *floats = workspace(M, V);
  return FUSION_OK;
}

extern "C" int joint_logprobs(const uint16_t *A, const uint16_t *W, const float *bias, int32_t K, int32_t T, int32_t S,
                              int32_t B, int32_t V, const int32_t *tokens, const int32_t *parents, float *logp,
                              float *entropy, float *lse, float *workspace_, int64_t workspace_floats,
                              hipStream_t stream) {
  if (T < 0 || S < 0 || B < 1) return set_error(FUSION_E_ARG, "T, S or B out of range");
  if (parents && B > FUSION_MAX_BEAM) return set_error(FUSION_E_UNSUPPORTED, "parents of more than FUSION_MAX_BEAM slots");
  const int64_t H = (int64_t)S * B;
  if (H > INT32_MAX || (H > 0 && T > INT32_MAX / H)) return set_error(FUSION_E_UNSUPPORTED, "more than 2^31 - 1 rows");
  const int64_t M = T * H;
  const int rc = check_sizes(M, V, K);
  if (rc != FUSION_OK) return rc;
  if (M == 0) return FUSION_OK;
  if (!A || !W || !workspace_) return set_error(FUSION_E_ARG, "NULL operand or workspace");
  if (((uintptr_t)A | (uintptr_t)W) % 16 != 0) return set_error(FUSION_E_ARG, "A and W must be 16-byte aligned");
  if (logp && !tokens) return set_error(FUSION_E_ARG, "log probabilities of NULL tokens");
  if (!logp && !entropy && !lse) return set_error(FUSION_E_ARG, "no output buffer");
  if (workspace_floats < workspace((int)M, V)) return set_error(FUSION_E_ARG, "workspace too small");
  if (!logp) tokens = nullptr;
  int32_t *status = nullptr;
  const int no_word = score_status_word(&status);
  if (no_word != FUSION_OK) return no_word;
  const int nct = with_shape((int)M, V, [&](auto c) -> int {
    using C = decltype(c);
    const int cols = (V + C::BN - 1) / C::BN, rows = ((int)M + C::BM - 1) / C::BM;
    if ((int64_t)cols * rows >= (1 << 23)) return -1;  // a launch holds fewer than 2^32 lanes
    const int map = tile_map(rows, cols, tiles(t128, (int)M, V) > kCus, (int)M, V, (int64_t)V * K * 2);
    const StatArgs q{A, W, bias, workspace_, (int)M, V, K, cols, map};
    hipLaunchKernelGGL((joint_stat_kernel<C>), dim3(cols * rows), dim3(64 * C::waves), 0, stream, q);
    return cols;
  });
  if (nct < 0) return set_error(FUSION_E_UNSUPPORTED, "too many tiles: split the call along T");
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_error(e, "joint statistics launch");
  const JoinArgs p{A, W, bias, workspace_, tokens, parents, logp, entropy, lse, status, (int32_t)M, V, K, B, nct};
  if (M >= 64 * kCus) hipLaunchKernelGGL(joint_join_kernel<1>, dim3((unsigned)((M + 63) / 64)), dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(joint_join_kernel<4>, dim3((unsigned)((M + 15) / 16)), dim3(256), 0, stream, p);
  e = hipGetLastError();
  return e == hipSuccess ? FUSION_OK : hip_error(e, "joint scoring launch");
}
