// Output projection of the Transducer joint network on MFMA: the logits that
// the acoustic term of Eq. (1) (Sec. III-C) is computed from, for a batch of
// hypothesis-frames at once:
//
//   out[m, n] = sum_k A[m, k] * W[n, k] + bias[n]      (bf16 inputs, fp32 accumulate)
//
// A is [M, K] and W is [N, K], both row-major bf16 (W in the usual layout of a
// linear layer's weight), so both MFMA operands are contiguous along K.  The
// tiles are joint_tile.h's.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "fusion_internal.h"
#include "joint_tile.h"

namespace fusion {
namespace {

template <class S, int kAux>
__global__ void __launch_bounds__(64 * S::waves, 2) joint_proj_kernel(const uint16_t *__restrict__ A,
                                                                     const uint16_t *__restrict__ W,
                                                                     const float *__restrict__ bias, int M, int N,
                                                                     int K, int n_col_tiles, int map,
                                                                     float *__restrict__ out) {
  __shared__ __align__(1024) unsigned char smem[S::lds];
  int tr, tc;
  tile_place(map, n_col_tiles, tr, tc);
  f32x4 acc[S::TM][S::TN];
  Bf16Op op;
  tile_product<S>(op, smem, A, W, M, N, K * 2, tr * S::BM, tc * S::BN, acc, [](auto &c) { tile_zero<S>(c); });
  tile_store<S, kAux>(smem, bias, M, N, tr * S::BM, tc * S::BN, acc, out);
}

}  // namespace
}  // namespace fusion

using namespace fusion;

extern "C" int joint_project(const uint16_t *A, const uint16_t *W, const float *bias, int32_t M, int32_t N,
                             int32_t K, float *out, hipStream_t stream) {
  if (M < 0 || N < 1 || K < 8) return set_error(FUSION_E_ARG, "M, N or K out of range");
  if (K % 8 != 0) return set_error(FUSION_E_UNSUPPORTED, "K must be a multiple of 8");
  if ((int64_t)M * K * 2 > 0x7FFFFFF0ll || (int64_t)N * K * 2 > 0x7FFFFFF0ll)
    return set_error(FUSION_E_UNSUPPORTED, "operand larger than 2 GiB: split the call along M");
  if (M == 0) return FUSION_OK;
  if (!A || !W || !out) return set_error(FUSION_E_ARG, "NULL operand");
  if (((uintptr_t)A | (uintptr_t)W) % 16 != 0) return set_error(FUSION_E_ARG, "A and W must be 16-byte aligned");
  constexpr TileShape<2, 4, 8, 4, 2> t256{};
  constexpr TileShape<2, 2, 4, 4, 2> t128{};
  constexpr TileShape<2, 2, 2, 4, 2> t64x128_3a_cu{};
  constexpr TileShape<2, 2, 2, 4, 3> t64x128{};
  constexpr TileShape<2, 2, 2, 2, 4> t64{};
  constexpr TileShape<2, 2, 1, 2, 4> t32{};
  constexpr int64_t kCus = 256;
  auto tiles = [&](auto cfg) -> int64_t {
    using C = decltype(cfg);
    return (int64_t)((M + C::BM - 1) / C::BM) * ((N + C::BN - 1) / C::BN);
  };
  auto go = [&](auto cfg) -> int {
    using C = decltype(cfg);
    const int nct = (N + C::BN - 1) / C::BN, nrt = (M + C::BM - 1) / C::BM;
    if (tiles(cfg) > 0x7FFFFFFFll) return set_error(FUSION_E_UNSUPPORTED, "too many tiles");
    const int map = tile_map(nrt, nct, tiles(t128) > kCus, M, N, (int64_t)N * K * 2);
    // Rows of whole 128-byte lines leave as streaming stores (nt with sc1: 459 us
    // for 76800 x 4096 x 640, plain 535, launches back to back); rows that share lines with their
    // neighbours are left for the L2 to merge (76800 x 1001 x 136: 91 us plain,
    // over 100 streaming)
    const dim3 grid(nct * nrt), block(64 * C::waves);
    if (N % 32 == 0)
      hipLaunchKernelGGL((joint_proj_kernel<C, 18>), grid, block, 0, stream, A, W, bias,
                         M, N, K, nct, map, out);
    else
      hipLaunchKernelGGL((joint_proj_kernel<C, 0>), grid, block, 0, stream, A, W, bias,
                         M, N, K, nct, map, out);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FUSION_OK : hip_error(e, "joint projection launch");
  };
  // By the number of tiles, which decides how evenly a launch fills the 256 CUs: a
  // larger tile reads less LDS per multiply-accumulate, a smaller one fills the
  // chip.  Measured (us; tiles in brackets):
  //              256x256      128x128      64x128       64x64        32x64
  //   256x4096   19 [16]      9.6 [64]     7.5 [128]    6.2 [256]    6.1 [512]     K = 640
  //   777x2500   12 [40]      7.2 [140]    6.7 [260]    7.8 [520]    7.3 [1000]    K = 256
  //   1664x4096  21 [112]     13.3 [416]   16.7 [832]   20 [1664]    23 [3328]     K = 640
  //   3328x1001  13 [52]      8.3 [208]    7.4 [416]    8.6 [832]    9.2 [1664]    K = 136
  // 256 x 256 from a thousand tiles on, except where
  //   - half of each tile or more would lie past N: 512000 x 100 x 128 took 93 us
  //     with it, 69 with 128 x 128; x 64 x 640 188 and 151; x 200 x 640 237 and 300
  //   - K is over 640 and rows are whole lines, for fewer than 2000 tiles, where the two
  //     are level or 128 x 128 ahead (25600 x 4096: 191 and 177 at K = 704, 218 and 206
  //     at 832, 249 and 252 at 1024).  With more tiles: 76800 x 4096 508 and 545 us at
  //     704, 660 and 764 at 1024; 51200 x 4096 341 and 351, 456 and 498; 512000 x 256
  //     263 and 315, 347 and 397.  With rows that share lines, 1000 tiles do:
  //     25600 x 2500 117 and 136 at 704, 148 and 169 at 1024
  // and from 400 on where W is over 4 MB and 128 x 128 tiles cannot be dealt 4 x 2 (A
  // then goes to all XCDs, half as often): 7711 x 3968 x 648 59 us and 73, 8837 x 6784 x
  // 504 96 and 118, but 12594 x 4032 x 536 97 and 91.
  // A single column of them (N of 129 to 256) also pays as one full round, 129 to 256
  // tiles, and from 400 on: A is read once, not twice (61385 x 208 x 240 18.3 us and
  // 25.5, in runs 20.4; 188 tiles of 192 x 912 31 and 48, 35; 503 of 181 x 600 62 and 87,
  // 70; but 299 of 165 x 128 32 and 26).
  // 128 x 128 holds two workgroups a CU: 513 to 640 tiles of it leave a second
  // round nearly empty, and 64 x 128 with two stages in LDS (three a CU) is ahead:
  // 3323 x 2500 x 256 13.3 us and 17.0, 8315 x 1001 x 512 23.1 and 27.7, 3195 x 3072 x
  // 512 17.1 and 20.4; at 680 tiles the two are level.  Not for wide rows dealt 4 x 2
  // (2555 x 4096 x 640 24 and 22.8 us) or of a long K (1580 x 5635 x 560 33.8 and 31.1).
  const int64_t n256 = tiles(t256), n128 = tiles(t128);
  const bool even128 = (N + 127) / 128 % 2 == 0;
  const bool t128_4x2 = (M + 127) / 128 % 4 == 0 && even128, t64x128_4x2 = (M + 63) / 64 % 4 == 0 && even128;
  if (n256 >= 1000 && N > 128 && (K <= 640 || n256 >= 2000 || N % 32 != 0)) return go(t256);
  if (n256 >= 400 && (int64_t)N * K * 2 > 4 << 20 && !t128_4x2) return go(t256);
  if (N > 128 && N <= 256 && n256 > kCus / 2 && (n256 <= kCus || n256 >= 400)) return go(t256);
  if (n128 > 2 * kCus && n128 <= 5 * kCus / 2 && (N < 4096 || (!t64x128_4x2 && K <= 512))) return go(t64x128_3a_cu);
  if (n128 > kCus) return go(t128);
  // (the narrower tiles store 8 rows at once: their offsets need 8 rows under 2 GiB)
  if (tiles(t64x128) > kCus || N >= (1 << 25)) return go(t64x128);
  if (tiles(t64) > kCus) return go(t64);
  return go(t32);
}
