// Operands in microscaled 4-bit floating point, and the joint projection of two
// of them.
//
// A row's blocks of 32 values share a power of two, 2^e, kept as the byte e + 127;
// a value is held as sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (e2m1), two to a
// byte, the even one in the low half.  e puts the block's largest magnitude in
// [4, 8): e = max(floor(log2 amax) - 2, -127).  Elements are x / 2^e rounded to the
// nearest level, halfway to the even code, above 6 to 6.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>
#include <utility>

#include "fusion_internal.h"
#include "joint_tile.h"
#include "row_types.h"

namespace fusion {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 32;

// A lane takes 16 bytes of a row, so 8 (fp32) or 4 lanes share a block and find its
// largest magnitude among themselves.  Bound by memory: 76800 x 640 in bf16 21 us (98 MB
// in, 26 out, 5.9 TB/s), 38421 x 1184 in fp32 34 us (6.1 TB/s), 46 from rows not in
// any cache.
template <class T>
__global__ void __launch_bounds__(256) quantize_kernel(const T *__restrict__ x, int64_t stride, uint32_t packs, uint32_t per_row,
                                                       int K, uint8_t *__restrict__ q, uint8_t *__restrict__ scales) {
  constexpr int n = Pack<T>::n, lanes = kBlock / n;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  const bool here = i < packs;  // the lanes of a block agree: a row holds whole blocks
  const uint32_t row = here ? i / per_row : 0, col = here ? (i - row * per_row) * n : 0;
  Pack<T> p;
  __builtin_memcpy(&p, x + row * stride + col, 16);
  float v[n];
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < n; ++j) {
    v[j] = to_float(p.v[j]);
    top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  }
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, false));
  if (lanes == 8) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x141, 0xF, 0xF, false));
  if (!here) return;
  const bool bad = top >= 0x7F800000u;  // a NaN or an infinity: the block is NaN
  const int e = bad ? 255 : max((int)(top >> 23) - 2, 0);
  const float by = bad ? 0.0f : __uint_as_float((uint32_t)(254 - e) << 23);  // 2^(127 - e)
  uint32_t code = 0;
#pragma unroll
  for (int j = 0; j < n; ++j) v[j] = bad ? 0.0f : v[j] * by;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], 1.0f, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], 1.0f, 1);
  const int64_t at = (int64_t)row * (K / 2) + col / 2;
  if constexpr (n == 8) {
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], 1.0f, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], 1.0f, 3);
    *reinterpret_cast<uint32_t *>(q + at) = code;
  } else {
    *reinterpret_cast<uint16_t *>(q + at) = (uint16_t)code;
  }
  if (threadIdx.x % lanes == 0) {
    const int blocks = K / kBlock, b = col / kBlock, ss = FUSION_MX_SCALE_STRIDE(K);
    uint8_t *s = scales + (int64_t)row * ss;
    s[b] = (uint8_t)e;
    if (b == blocks - 1)
      for (int j = blocks; j < ss; ++j) s[j] = 0;
  }
}

// A lane writes 16 bytes of a row.  Bound by its stores: 38421 x 1184 in fp32 31 us,
// 182 MB out, 6.7 TB/s with what it reads.
template <class T>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t *__restrict__ q, const uint8_t *__restrict__ scales,
                                                         uint32_t packs, uint32_t per_row, int K, int64_t stride,
                                                         T *__restrict__ out) {
  constexpr int n = Pack<T>::n;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= packs) return;
  const uint32_t row = i / per_row, col = (i - row * per_row) * n;
  const uint8_t *src = q + (int64_t)row * (K / 2) + col / 2;
  const uint32_t code = n == 8 ? *reinterpret_cast<const uint32_t *>(src) : *reinterpret_cast<const uint16_t *>(src);
  const uint32_t e = scales[(int64_t)row * FUSION_MX_SCALE_STRIDE(K) + col / kBlock];
  const float by = __uint_as_float(e == 255 ? 0x7FC00000u : e == 0 ? 0x00400000u : e << 23);
  f32x2 v[4];
  v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0);
  v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1);
  v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2);
  v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3);
  Pack<T> p;
#pragma unroll
  for (int j = 0; j < n; ++j) from_float(v[j / 2][j % 2] * by, p.v[j]);
  __builtin_memcpy(out + row * stride + col, &p, 16);
}

// 16 x 16 outputs over 128 of K, both operands fp4: lane l holds row l % 16's block
// l / 16 of each, and that block's scale in byte bw or ba of its register
template <int bw, int ba>
__device__ __forceinline__ f32x4 mfma_mx(i32x4 w, i32x4 a, f32x4 c, int sw, int sa) {
  const i32x8 w8 = __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
  const i32x8 a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, a8, c, 4, 4, bw, sw, ba, sa);
}

// Operands of the product: a stage is 256 elements of K, 8 blocks a row, two steps
// of v_mfma_scale_f32_16x16x128_f8f6f4.  A lane of group g reads chunks (blocks) 2 g
// and 2 g + 1, one a step: any split of K over the groups gives the same sum, and
// so both scales of a row are one 16-bit load, a stage ahead.
template <int TM, int TN>
struct MxOp {
  const uint8_t *A_scales, *W_scales;
  int blocks, stride;  // of a row of scales
  __amdgpu_buffer_rsrc_t ra, rw;
  uint32_t oa[TM], ow[TN];
  int sa[TM], sw[TN], next_a[TM], next_w[TN];
  int group;
  __device__ __forceinline__ void load(int s) {
    const int b = s * 8 + 2 * group;
    const int valid = (b < blocks ? 0xFF : 0) | (b + 1 < blocks ? 0xFF00 : 0);  // bytes behind the last block are not read
#pragma unroll
    for (int i = 0; i < TM; ++i) next_a[i] = __builtin_amdgcn_raw_buffer_load_b16(ra, oa[i], s * 8, 0) & valid;
#pragma unroll
    for (int j = 0; j < TN; ++j) next_w[j] = __builtin_amdgcn_raw_buffer_load_b16(rw, ow[j], s * 8, 0) & valid;
  }
  __device__ __forceinline__ void begin(int M, int N, int row_a, int row_w, int fc) {
    group = fc;
    ra = rsrc(A_scales, (uint32_t)((int64_t)M * stride));
    rw = rsrc(W_scales, (uint32_t)((int64_t)N * stride));
#pragma unroll
    for (int i = 0; i < TM; ++i) oa[i] = row_a + 16 * i < M ? (uint32_t)((row_a + 16 * i) * (int64_t)stride + 2 * fc) : kOutside;
#pragma unroll
    for (int j = 0; j < TN; ++j) ow[j] = row_w + 16 * j < N ? (uint32_t)((row_w + 16 * j) * (int64_t)stride + 2 * fc) : kOutside;
    load(0);
  }
  __device__ __forceinline__ void stage(int s) {
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = next_a[i];
#pragma unroll
    for (int j = 0; j < TN; ++j) sw[j] = next_w[j];
    if ((s + 1) * 8 < blocks) load(s + 1);
  }
  static __device__ __forceinline__ int chunk(int ks, int fc) { return 2 * fc + ks; }
  template <int ks>
  __device__ __forceinline__ f32x4 mfma(i32x4 w, i32x4 a, f32x4 c, int j, int i) const {
    return mfma_mx<ks, ks>(w, a, c, sw[j], sa[i]);
  }
};

struct MxArgs {
  const uint8_t *A, *A_scales, *W, *W_scales;
  const float *bias;
  float *out;
  int M, N, K, n_col_tiles, map;
};

// Tile by tile, as joint_proj_kernel: for few tiles, where latency counts (256 x 4096
// x 640: 5.4 us), and for a K that mx_panel_kernel's registers do not hold.  A large
// output it writes at 4.3 TB/s (290 us for 76800 x 4096 x 640: operands 170, stores 190).
template <class S, int kAux>
__global__ void __launch_bounds__(64 * S::waves, 2) mx_proj_kernel(MxArgs p) {
  __shared__ __align__(1024) unsigned char smem[S::lds];
  int tr, tc;
  tile_place(p.map, p.n_col_tiles, tr, tc);
  f32x4 acc[S::TM][S::TN];
  MxOp<S::TM, S::TN> op;
  op.A_scales = p.A_scales;
  op.W_scales = p.W_scales;
  op.blocks = p.K / kBlock;
  op.stride = FUSION_MX_SCALE_STRIDE(p.K);
  tile_product<S>(op, smem, p.A, p.W, p.M, p.N, p.K / 2, tr * S::BM, tc * S::BN, acc, [](auto &c) { tile_zero<S>(c); });
  tile_store<S, kAux>(smem, p.bias, p.M, p.N, tr * S::BM, tc * S::BN, acc, p.out);
}

// The same product for launches that the output's stores bound.  Two things keep
// stores and products from overlapping in a tile kernel: a wave's loads and stores
// complete in one order, so that a wave which stores a tile and then waits for the
// next one's operands waits for its stores; and operands of 4 bits are used up so
// fast that bringing both takes longer than their product.  Here a workgroup keeps
// its 128 columns of W in registers, all of K, and goes down the rows of A, 64 at a
// time; two waves do all the loading, a tile each in turn, and the four that multiply
// and store wait for nothing but their barrier.  Two workgroups a CU, out of step.
// 76800 x 4096 x 640: 194 us back to back, 1.26 GB of output at 6.5 TB/s (a fill of that
// size: 6.9); the same without its stores 85.
// 64 rows x 128 columns, 32 x 64 a wave: it stores 256 bytes of a row at once (204 us
// for 76800 x 4096 x 640, 230 in 128 bytes).  From 6 steps of 128 along K on, W's
// registers allow 32 columns a wave only.
template <int steps>
using Panel = std::conditional_t<steps <= 5, TileShape<2, 2, 2, 4>, TileShape<1, 4, 4, 2>>;
constexpr int kPanelSteps = 6, kPanelRows = 64, kPanelCols = 128;

struct PanelArgs {
  MxArgs g;
  int slices, row_tiles;  // a workgroup takes a column tile and every slices-th row tile
};

template <class F, int... s>
__device__ __forceinline__ void each_step(F f, std::integer_sequence<int, s...>) {
  (f(std::integral_constant<int, s>{}), ...);
}

// steps: of 128 along K, each unrolled
template <int steps, int kAux>
__global__ void __launch_bounds__(64 * 6, 3) mx_panel_kernel(PanelArgs q) {
  typedef Panel<steps> S;
  static_assert(S::BM == kPanelRows && S::BN == kPanelCols, "as the launch takes them");
  const MxArgs &p = q.g;
  // a buffer: a tile of A, steps x 64 rows x 64 bytes, then its scales' rows
  constexpr int kScales = steps * S::BM * 64, kBuf = kScales + S::BM * FUSION_MX_SCALE_STRIDE(128 * steps);
  __shared__ __align__(1024) unsigned char s_buf[2][kBuf];
  __shared__ f32x4 s_slab[S::waves][4 * S::seg];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fc = lane >> 4;
  constexpr int stride = FUSION_MX_SCALE_STRIDE(128 * steps);  // (of K too: it goes by whole 256s)
  const int blocks = p.K / kBlock;
  // a run of consecutive workgroups, column-fastest, on each XCD: its L2 fetches a
  // slice's rows of A once, and merges the lines that neighbouring columns share
  const int x = blockIdx.x & 7, per = gridDim.x >> 3, more = gridDim.x & 7;
  const int unit = x * per + min(x, more) + (blockIdx.x >> 3);
  const int slice = __builtin_amdgcn_readfirstlane(unit / p.n_col_tiles), col = unit - slice * p.n_col_tiles;
  const int tiles = __builtin_amdgcn_readfirstlane((q.row_tiles - slice + q.slices - 1) / q.slices);

  if (wave >= S::waves) {
    const int who = wave - S::waves;
    const __amdgpu_buffer_rsrc_t ra = rsrc(p.A, (uint32_t)((int64_t)p.M * (p.K / 2)));
    const uint32_t scale_bytes = (uint32_t)((int64_t)p.M * stride);
    const __amdgpu_buffer_rsrc_t rs = rsrc(p.A_scales, scale_bytes);
    // a load brings 16 rows of a step, 4 chunks each; lane l's lands in row l / 4, slot l % 4
    const int row = lane >> 2, chunk = Slots64::of(row, lane & 3);
    auto issue = [&](int k) {
      const int tile = slice + k * q.slices;
      unsigned char *at = s_buf[who];
      uint32_t vo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = tile * S::BM + j * 16 + row;
        vo[j] = r < p.M ? (uint32_t)(r * (int64_t)(p.K / 2) + chunk * 16) : kOutside;
      }
#pragma unroll
      for (int s = 0; s < steps; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          load_lds(ra, at + (s * 4 + j) * 1024, s < steps - 1 || s * 4 + chunk < blocks ? vo[j] : kOutside, s * 64);
      // the scales of 64 rows lie together: 256 bytes a load, zeros past the operand (the
      // whole distance in the lane's offset: a scalar one is not range checked)
      const uint32_t so = (uint32_t)((int64_t)tile * S::BM * stride + lane * 4);
#pragma unroll
      for (int j = 0; j < stride / 4; ++j)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(at + kScales + j * 256), 4,
                                                 so + j * 256 < scale_bytes ? so + j * 256 : kOutside, 0, 0, 0);
    };
    // the workgroup's tiles `who`, `who` + 2 ..: each into this wave's buffer, once
    // the others are behind the barrier of the tile after the one that was there
    if (who == 0) issue(0);
    for (int k = 0; k < tiles; ++k) {
      if (k % 2 == who) wait_barrier<0>();
      else {
        asm volatile("s_barrier" ::: "memory");
        if (k + 1 < tiles) issue(k + 1);
      }
    }
    return;
  }

  const int bn = col * S::BN + wave % S::WN * S::RN, wm = wave / S::WN * S::RM;
  i32x4 w[steps][S::TN];
  int sw[(steps + 3) / 4][S::TN] = {};  // a byte a step
  const __amdgpu_buffer_rsrc_t rw = rsrc(p.W, (uint32_t)((int64_t)p.N * (p.K / 2)));
  const __amdgpu_buffer_rsrc_t rv = rsrc(p.W_scales, (uint32_t)((int64_t)p.N * stride));
#pragma unroll
  for (int s = 0; s < steps; ++s)
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int n = bn + j * 16 + fr, c = s * 4 + fc;
      const bool in = n < p.N && c < blocks;
      w[s][j] = __builtin_amdgcn_raw_buffer_load_b128(rw, in ? (uint32_t)(n * (int64_t)(p.K / 2) + c * 16) : kOutside, 0, 0);
      sw[s / 4][j] |= (int)__builtin_amdgcn_raw_buffer_load_b8(rv, in ? (uint32_t)(n * (int64_t)stride + c) : kOutside, 0, 0) << (s % 4 * 8);
    }
  constexpr int kLanes = S::seg / 4;
  static_assert(S::seg == S::RN, "one segment a row");
  float bv[1][4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int n = bn + lane % kLanes * 4 + r;
    bv[0][r] = p.bias && n < p.N ? p.bias[n] : 0.0f;
  }
  for (int k = 0; k < tiles; ++k) {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const unsigned char *at = s_buf[k & 1];
    f32x4 acc[S::TM][S::TN];
    tile_zero<S>(acc);
    auto step = [&](auto s_) {
      constexpr int s = decltype(s_)::value;
      i32x4 a[S::TM];
      int sa[S::TM];
#pragma unroll
      for (int i = 0; i < S::TM; ++i) {
        a[i] = *reinterpret_cast<const i32x4 *>(at + s * 4096 + (wm + i * 16 + fr) * 64 + Slots64::of(fr, fc) * 16);
        sa[i] = at[kScales + (wm + i * 16 + fr) * stride + s * 4 + fc];
      }
#pragma unroll
      for (int i = 0; i < S::TM; ++i) sa[i] &= s * 4 + fc < blocks ? 0xFF : 0;  // (bytes behind the last block mean nothing)
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[i][j] = mfma_mx<s % 4, 0>(w[s][j], a[i], acc[i][j], sw[s / 4][j], sa[i]);
    };
    each_step(step, std::make_integer_sequence<int, steps>{});
    slab_store<S, kAux>(s_slab[wave], bv, p.M, p.N, (slice + k * q.slices) * S::BM + wm, bn, acc, p.out);
  }
}

template <int... s>
void launch_panel(const PanelArgs &q, hipStream_t stream, std::integer_sequence<int, s...>) {
  const dim3 grid(q.slices * q.g.n_col_tiles), block(64 * 6);
  const int steps = (q.g.K + 127) / 128;
  // streaming stores for rows of whole 128-byte lines, as in joint_project
  auto go = [&](auto n) {
    if (steps != decltype(n)::value) return;
    if (q.g.N % 32 == 0) hipLaunchKernelGGL((mx_panel_kernel<decltype(n)::value, 18>), grid, block, 0, stream, q);
    else hipLaunchKernelGGL((mx_panel_kernel<decltype(n)::value, 0>), grid, block, 0, stream, q);
  };
  (go(std::integral_constant<int, s + 1>{}), ...);
}

int check_mx(int32_t dtype, int64_t stride, int32_t R, int32_t K) {
  if (dtype != FUSION_F32 && dtype != FUSION_BF16 && dtype != FUSION_F16) return set_error(FUSION_E_ARG, "unknown dtype");
  if (R < 0 || K < kBlock) return set_error(FUSION_E_ARG, "R or K out of range");
  if (K % kBlock != 0) return set_error(FUSION_E_UNSUPPORTED, "K must be a multiple of 32");
  if (stride < K) return set_error(FUSION_E_ARG, "rows overlap: stride below K");
  if (stride > (INT64_MAX >> 3) / (R > 0 ? R : 1)) return set_error(FUSION_E_ARG, "stride out of range");
  // (a launch holds fewer than 2^32 lanes)
  if ((int64_t)R * (K / (dtype == FUSION_F32 ? 4 : 8)) > 0xFFFFFF00ll)
    return set_error(FUSION_E_UNSUPPORTED, "too many elements: split the call along R");
  return FUSION_OK;
}

}  // namespace
}  // namespace fusion

using namespace fusion;

extern "C" int mx_quantize(const void *x, int32_t dtype, int64_t stride, int32_t R, int32_t K, uint8_t *q,
                           uint8_t *scales, hipStream_t stream) {
  const int rc = check_mx(dtype, stride, R, K);
  if (rc != FUSION_OK) return rc;
  if (R == 0) return FUSION_OK;
  if (!x || !q || !scales) return set_error(FUSION_E_ARG, "NULL operand");
  if ((uintptr_t)x % (dtype == FUSION_F32 ? 4 : 2) != 0 || (uintptr_t)q % 16 != 0 || (uintptr_t)scales % 8 != 0)
    return set_error(FUSION_E_ARG, "misaligned operand: q needs 16 bytes, scales 8");
  auto go = [&](auto type) {
    using T = decltype(type);
    const uint32_t per_row = K / Pack<T>::n, packs = (uint32_t)R * per_row;
    hipLaunchKernelGGL(quantize_kernel<T>, dim3(packs / 256 + (packs % 256 != 0)), dim3(256), 0, stream,
                       static_cast<const T *>(x), stride, packs, per_row, K, q, scales);
  };
  if (dtype == FUSION_F32) go(float{});
  else if (dtype == FUSION_BF16) go(Brain{});
  else go(Half{});
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FUSION_OK : hip_error(e, "quantisation launch");
}

extern "C" int mx_dequantize(const uint8_t *q, const uint8_t *scales, int32_t R, int32_t K, void *out, int32_t dtype,
                             int64_t stride, hipStream_t stream) {
  const int rc = check_mx(dtype, stride, R, K);
  if (rc != FUSION_OK) return rc;
  if (R == 0) return FUSION_OK;
  if (!out || !q || !scales) return set_error(FUSION_E_ARG, "NULL operand");
  if ((uintptr_t)out % (dtype == FUSION_F32 ? 4 : 2) != 0 || (uintptr_t)q % 16 != 0 || (uintptr_t)scales % 8 != 0)
    return set_error(FUSION_E_ARG, "misaligned operand: q needs 16 bytes, scales 8");
  auto go = [&](auto type) {
    using T = decltype(type);
    const uint32_t per_row = K / Pack<T>::n, packs = (uint32_t)R * per_row;
    hipLaunchKernelGGL(dequantize_kernel<T>, dim3(packs / 256 + (packs % 256 != 0)), dim3(256), 0, stream, q, scales,
                       packs, per_row, K, stride, static_cast<T *>(out));
  };
  if (dtype == FUSION_F32) go(float{});
  else if (dtype == FUSION_BF16) go(Brain{});
  else go(Half{});
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FUSION_OK : hip_error(e, "dequantisation launch");
}

extern "C" int joint_project_mx(const uint8_t *A, const uint8_t *A_scales, const uint8_t *W, const uint8_t *W_scales,
                                const float *bias, int32_t M, int32_t N, int32_t K, float *out, hipStream_t stream) {
  if (M < 0 || N < 1 || K < kBlock) return set_error(FUSION_E_ARG, "M, N or K out of range");
  if (K % kBlock != 0) return set_error(FUSION_E_UNSUPPORTED, "K must be a multiple of 32");
  if ((int64_t)M * (K / 2) > 0x7FFFFFF0ll || (int64_t)N * (K / 2) > 0x7FFFFFF0ll || N >= (1 << 25))
    return set_error(FUSION_E_UNSUPPORTED, "operand larger than 2 GiB: split the call");
  if (M == 0) return FUSION_OK;
  if (!A || !A_scales || !W || !W_scales || !out) return set_error(FUSION_E_ARG, "NULL operand");
  if (((uintptr_t)A | (uintptr_t)W) % 16 != 0 || ((uintptr_t)A_scales | (uintptr_t)W_scales) % 8 != 0 || (uintptr_t)out % 4 != 0)
    return set_error(FUSION_E_ARG, "misaligned operand: A and W need 16 bytes, scales 8");
  constexpr TileShape<2, 4, 8, 4, 2> t256{};
  constexpr TileShape<2, 2, 4, 4, 2> t128{};
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
    if (tiles(cfg) >= (1 << 23)) return set_error(FUSION_E_UNSUPPORTED, "too many tiles: split the call along M");
    const MxArgs p{A, A_scales, W, W_scales, bias, out, M, N, K, nct,
                   tile_map(nrt, nct, tiles(t128) > kCus, M, N, (int64_t)N * K / 2)};
    const dim3 grid(nct * nrt), block(64 * C::waves);
    // streaming stores for rows of whole 128-byte lines, as in joint_project
    if (N % 32 == 0) hipLaunchKernelGGL((mx_proj_kernel<C, 18>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((mx_proj_kernel<C, 0>), grid, block, 0, stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FUSION_OK : hip_error(e, "4-bit projection launch");
  };
  // By panels from 512 tiles of 128 x 128 on and up to the K that W's registers hold
  // (us, tiles and panels): 76800 x 4096 x 640 299 and 194, 3328 x 4096 x 640 18.9 and
  // 15.9, 30000 x 2500 x 640 88 and 84, 97585 x 401 x 64 35 and 29; below that the two
  // are level, and with few columns or a long K tiles ahead (1024 x 1024 x 512 4.9 and
  // 5.9).  Not for many rows that share lines with their neighbours and a short K: the
  // workgroups of neighbouring columns drift apart, and the L2 merges fewer of those
  // lines (52396 x 3209 x 32 134 and 173, 145915 x 1459 x 128 186 and 226; of 12 such
  // sizes two were better off: 26090 x 8441 x 96 269 and 218).
  const bool drifts = N % 32 != 0 && K <= 128 && tiles(t128) >= 4500;
  if (K <= 128 * kPanelSteps && tiles(t128) >= 512 && !drifts) {
    PanelArgs q{{A, A_scales, W, W_scales, bias, out, M, N, K, (N + kPanelCols - 1) / kPanelCols, 0}, 1,
                (M + kPanelRows - 1) / kPanelRows};
    q.slices = std::max<int>(1, std::min<int>(2 * kCus / q.g.n_col_tiles, q.row_tiles));
    launch_panel(q, stream, std::make_integer_sequence<int, kPanelSteps>{});
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FUSION_OK : hip_error(e, "4-bit projection launch");
  }
  // the largest tile that fills the chip
  if (tiles(t256) >= 1000 && N > 128) return go(t256);
  if (tiles(t128) > kCus) return go(t128);
  if (tiles(t64x128) > kCus) return go(t64x128);
  if (tiles(t64) > kCus) return go(t64);
  return go(t32);
}
