// Output tiles of products with both operands contiguous along K,
//   out[m, n] = sum_k A[m, k] * W[n, k],
// shared by the joint projection (joint_proj.hip), its 4-bit form (mx.hip) and
// the scoring straight from hidden states (joint_logprobs.hip).
//
// Tiling for gfx950: a workgroup of WM x WN waves computes a (16 TM WM) x
// (16 TN WN) output tile, each wave (16 TM) x (16 TN) as a TM x TN grid of
// 16 x 16 MFMA tiles.  K advances in stages of 128 bytes a row, NB of them in
// LDS; the operands go straight from global memory to LDS (16 bytes a lane, no
// registers, no LDS store instructions), NB - 1 stages ahead, with one barrier
// a stage that waits for the oldest stage's loads only.  A stage's rows are 128
// bytes, all LDS banks, so a fragment read (16 rows, one 16-byte chunk of each)
// would hit the same banks in every row: chunk c of row r is kept in slot
// c ^ (r % 8), which the loading lane arranges by the global chunk it picks
// SQ_LDS_BANK_CONFLICT reads 0 (rows padded by 16 bytes: 47 % of the LDS's
// active cycles).  The MFMA operands are swapped (W rows as the tile's rows),
// so a lane ends with 4 consecutive columns of one output row.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace fusion {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kMapNone = 0, kMap4x2 = 1, kMapRuns = 2;  // tiles to XCDs
constexpr uint32_t kOutside = 0x80000000u;    // an offset past every descriptor (operands are under 2 GiB)

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void *base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), (short)0, (int)bytes, 0x00020000);
}
// the same of values that are uniform without the compiler seeing it, which would
// otherwise go through the lanes' descriptors one by one at each access
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_uniform(const void *base, uint32_t bytes) {
  const uint64_t v = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
  return rsrc(reinterpret_cast<const void *>((uint64_t)hi << 32 | lo), (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes));
}
// 16 bytes per lane straight into LDS (lane l lands at lds + 16 l)
__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t r, unsigned char *lds, uint32_t voff, uint32_t soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)lds, 16, voff, soff, 0, 0);
}
// Barrier that also waits for this wave's LDS reads and for all but its N newest
// vector-memory operations (the loads into LDS count there, in order)
template <int N>
__device__ __forceinline__ void wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Slot in LDS of a 16-byte chunk of a row, rows of 128 or 64 bytes: 16 rows' reads
// of one chunk meet all banks
struct Slots128 {
  static __device__ __forceinline__ int of(int row, int chunk) { return chunk ^ (row & 7); }
};
struct Slots64 {
  static __device__ __forceinline__ int of(int row, int chunk) { return chunk ^ (row >> 2 & 3); }
};

// a launch shape: WM x WN waves of TM x TN tiles, NB stages
template <int WM_, int WN_, int TM_, int TN_, int NB_ = 1>
struct TileShape {
  static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, NB = NB_;
  static constexpr int SB = 128;  // bytes of a row in a stage
  static constexpr int RM = 16 * TM_, RN = 16 * TN_;  // rows and columns of a wave's tile
  static constexpr int BM = RM * WM_, BN = RN * WN_, waves = WM_ * WN_;
  static constexpr int stage = (BM + BN) * SB;
  static constexpr int lds = NB_ * stage;
  static constexpr int seg = RN < 64 ? RN : 64;  // columns of a stored row segment
};

// Tile of this workgroup, which runs on XCD x = blockIdx % 8 under the hardware's
// round-robin (see tile_map for the choice):
// kMap4x2 (row tiles a multiple of 4, column tiles even): XCD x takes the row
// tiles = x % 4 (mod 4) against column half x / 4, so a row band of A is fetched by
// two XCDs instead of eight and each XCD's L2 keeps half of W.
// kMapRuns: each XCD takes a run of consecutive tiles, column-fastest, so that a row
// band of A is fetched by one XCD (two at a run's end) and every L2 holds W.
// kMapNone: column-fastest over all XCDs
__device__ __forceinline__ void tile_place(int map, int n_col_tiles, int &tr, int &tc) {
  if (map == kMap4x2) {
    const int x = blockIdx.x & 7, i = blockIdx.x >> 3;
    const int half = n_col_tiles >> 1;
    tr = (i / half) * 4 + (x & 3);
    tc = (x >> 2) * half + i % half;
  } else {
    int t = blockIdx.x;
    if (map == kMapRuns) {
      const int x = t & 7, per = gridDim.x >> 3, more = gridDim.x & 7;  // the first `more` XCDs take one tile more
      t = x * per + min(x, more) + (t >> 3);
    }
    tr = t / n_col_tiles;
    tc = t % n_col_tiles;
  }
}

// Tiles to XCDs: 4 x 2 where the tiles divide so; else, in a launch of more than a
// round, in runs if W fits an L2 (up to 4 MB), has at most 32 column tiles and is
// the smaller operand.  Not dealt at all, 128 x 128 tiles of bf16 fetch every row band of A on
// all eight XCDs: 30343 x 1024 x 248 45 us, in runs 36; 48340 x 1024 x 768 117 and 88;
// over 190 random sizes that the rule takes 5 % (M < 2 N) to 14 % (M > 8 N) faster in
// runs, 256 x 256 tiles 4 to 5 %.  Against 4 x 2 runs gain 7 % to lose 19 %.
inline int tile_map(int row_tiles, int col_tiles, bool many, int M, int N, int64_t w_bytes) {
  if (row_tiles % 4 == 0 && col_tiles % 2 == 0) return kMap4x2;
  return many && M >= N && col_tiles <= 32 && w_bytes <= 4 << 20 ? kMapRuns : kMapNone;
}

// bf16 operands: a stage is 64 elements of K, two steps of v_mfma_f32_16x16x32_bf16
struct Bf16Op {
  __device__ __forceinline__ void begin(int, int, int, int, int) {}
  __device__ __forceinline__ void stage(int) {}
  // the 16-byte chunk that lanes of group fc (lane / 16) read at a step
  static __device__ __forceinline__ int chunk(int ks, int fc) { return ks * 4 + fc; }
  template <int ks>
  __device__ __forceinline__ f32x4 mfma(i32x4 w, i32x4 a, f32x4 c, int, int) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
  }
};

template <class S>
__device__ __forceinline__ void tile_zero(f32x4 (&acc)[S::TM][S::TN]) {
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
}

// The loads of a tile's stages into LDS.  row_bytes: of a row of A and W (a multiple of 16)
template <class S>
struct TileLoads {
  static constexpr int kChunks = S::SB / 16;      // 16-byte chunks per row and stage
  static constexpr int kRowsPer = 64 / kChunks;   // rows one wave-wide load brings (1 KiB)
  static constexpr int kLA = S::BM / kRowsPer / S::waves, kLW = S::BN / kRowsPer / S::waves, kL = kLA + kLW;  // loads per wave
  static_assert(kLA * kRowsPer * S::waves == S::BM && kLW * kRowsPer * S::waves == S::BN, "whole loads per wave");
  __amdgpu_buffer_rsrc_t ra, rw;
  int M, N, row_bytes, wave, lr, lc;
  uint32_t vo[kL];

  __device__ __forceinline__ TileLoads(const void *A, const void *W, int M_, int N_, int row_bytes_)
      : M(M_), N(N_), row_bytes(row_bytes_) {
    const int lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    ra = rsrc(A, (uint32_t)((int64_t)M * row_bytes));
    rw = rsrc(W, (uint32_t)((int64_t)N * row_bytes));
    lr = lane / kChunks;
    lc = Slots128::of(lr, lane % kChunks);  // (kRowsPer is 8: the row's low bits are lr)
  }
  // Load j of a stage brings rows (j * waves + wave) * kRowsPer .. of A (j < kLA)
  // or W to consecutive LDS: lane l lands 16 l bytes in, i.e. row l / kChunks, slot
  // l % kChunks, and fetches the chunk which that slot holds.  Rows past the operand
  // and, in a ragged last stage, chunks past K read as zeros (range check).
  __device__ __forceinline__ void tile(int bm, int bn) {
#pragma unroll
    for (int j = 0; j < kL; ++j) {
      const int row = (j < kLA ? bm + (j * S::waves + wave) * kRowsPer : bn + ((j - kLA) * S::waves + wave) * kRowsPer) + lr;
      vo[j] = row < (j < kLA ? M : N) ? (uint32_t)((int64_t)row * row_bytes + lc * 16) : kOutside;
    }
  }
  // stage s into the LDS of stage buffer `at`
  __device__ __forceinline__ void issue(int s, unsigned char *at) const {
    unsigned char *base = at + wave * 1024;
    const bool ragged = (s + 1) * S::SB > row_bytes && s * S::SB + lc * 16 >= row_bytes;
#pragma unroll
    for (int j = 0; j < kL; ++j)
      load_lds(j < kLA ? ra : rw, base + j * S::waves * 1024, ragged ? kOutside : vo[j], s * S::SB);
  }
};

// adds a stage in LDS to acc, for the wave whose tile is at row wm, column wn of the
// workgroup's.  Fragment of a 16-row operand tile: lane l holds row l % 16, the
// chunk of its group l / 16
template <class S, class Op>
__device__ __forceinline__ void tile_stage(const Op &op, const unsigned char *pa, int wm, int wn, f32x4 (&acc)[S::TM][S::TN]) {
  const int fr = threadIdx.x & 15, fc = (threadIdx.x & 63) >> 4;
  const unsigned char *pw = pa + S::BM * S::SB;
  auto step = [&](auto ks_) {
    constexpr int ks = decltype(ks_)::value;
    i32x4 fa[S::TM], fw[S::TN];
    const int at = Slots128::of(fr, op.chunk(ks, fc)) * 16;
#pragma unroll
    for (int j = 0; j < S::TN; ++j) fw[j] = *reinterpret_cast<const i32x4 *>(pw + (wn + j * 16 + fr) * S::SB + at);
#pragma unroll
    for (int i = 0; i < S::TM; ++i) fa[i] = *reinterpret_cast<const i32x4 *>(pa + (wm + i * 16 + fr) * S::SB + at);
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j) acc[i][j] = op.template mfma<ks>(fw[j], fa[i], acc[i][j], j, i);
  };
  step(std::integral_constant<int, 0>{});
  step(std::integral_constant<int, 1>{});
}

// The tile at row bm, column bn, added to what `start` puts into acc while the first
// stages are on their way
template <class S, class Op, class Start>
__device__ __forceinline__ void tile_product(Op &op, unsigned char *smem, const void *A, const void *W, int M, int N,
                                             int row_bytes, int bm, int bn, f32x4 (&acc)[S::TM][S::TN], Start start) {
  TileLoads<S> loads(A, W, M, N, row_bytes);
  constexpr int kL = TileLoads<S>::kL;
  const int lane = threadIdx.x & 63, wave = loads.wave;
  const int wm = (wave / S::WN) * S::RM, wn = (wave % S::WN) * S::RN;
  loads.tile(bm, bn);
  const int nk = (row_bytes + S::SB - 1) / S::SB;
  op.begin(M, N, bm + wm + (lane & 15), bn + wn + (lane & 15), lane >> 4);
#pragma unroll
  for (int s = 0; s < S::NB - 1; ++s)
    if (s < nk) loads.issue(s, smem + s * S::stage);
  start(acc);
  int buf = 0;
  for (int s = 0; s < nk; ++s) {
    // stage s has landed for every wave, and every wave is done reading the
    // buffer of stage s - 1, which stage s + NB - 1 is loaded into
    if (s + S::NB - 2 < nk) wait_barrier<(S::NB - 2) * kL>();
    else wait_barrier<0>();
    op.stage(s);
    if (s + S::NB - 1 < nk) loads.issue(s + S::NB - 1, smem + (buf == 0 ? S::NB - 1 : buf - 1) * S::stage);
    tile_stage<S>(op, smem + buf * S::stage, wm, wn, acc);
    buf = buf == S::NB - 1 ? 0 : buf + 1;
  }
}

// Stores a wave's tile, at row m0, column n0 of the output.  In the accumulator of
// a 16 x 16 tile lane l holds output row l % 16, columns 4 * (l / 16) .. + 3.  Each
// 16-row slab of the tile goes through the wave's own LDS area, chunks swizzled by
// the row as above, and leaves as whole row segments of S::seg columns, kRowsI rows
// a store, with the bias bv of the lane's columns of each segment added.
// kAux: cache policy of the output stores (see joint_project)
template <class S, int kAux>
__device__ __forceinline__ void slab_store(f32x4 *slab, const float (&bv)[S::RN / S::seg][4], int M, int N, int m0_, int n0,
                                           const f32x4 (&acc)[S::TM][S::TN], float *__restrict__ out) {
  constexpr int kSeg = S::seg, kLanes = kSeg / 4, kRowsI = 64 / kLanes;
  const int lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4;
  const int orow = lane / kLanes, ochunk = lane % kLanes;
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
#pragma unroll
    for (int sg = 0; sg < S::RN / kSeg; ++sg) {
#pragma unroll
      for (int j = 0; j < kSeg / 16; ++j)
        slab[fr * kLanes + ((j * 4 + fc) ^ (fr & (kLanes - 1)))] = acc[i][sg * (kSeg / 16) + j];
      __builtin_amdgcn_wave_barrier();
      const int n = n0 + sg * kSeg + ochunk * 4;
#pragma unroll
      for (int q = 0; q < 16 / kRowsI; ++q) {
        const int row = q * kRowsI + orow;
        const f32x4 x = slab[row * kLanes + (ochunk ^ (row & (kLanes - 1)))];
        i32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = __float_as_int(x[r] + bv[sg][r]);
        // a descriptor of this store's rows that exist; columns past N fall outside it
        const int m0 = m0_ + i * 16 + q * kRowsI;
        const int rows = min(max(M - m0, 0), kRowsI);
        const __amdgpu_buffer_rsrc_t ro = rsrc_uniform(out + (int64_t)m0 * N, (uint32_t)rows * (uint32_t)N * 4u);
        const uint32_t o = ((uint32_t)orow * (uint32_t)N + (uint32_t)n) * 4u;
        __builtin_amdgcn_raw_buffer_store_b128(v, ro, n + 3 < N ? o : kOutside, 0, kAux);
        if (N % 4 != 0) {  // uniform: the row's last columns, one at a time
#pragma unroll
          for (int r = 0; r < 3; ++r)
            __builtin_amdgcn_raw_buffer_store_b32(v[r], ro, (n + 3 >= N && n + r < N) ? o + 4 * r : kOutside, 0, kAux);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Stores the workgroup's tile: the slabs are the stages' LDS, free once every wave
// has read the last stage.  The bias is fetched before the first store: a load
// behind stores would wait for all of them.
template <class S, int kAux>
__device__ __forceinline__ void tile_store(unsigned char *smem, const float *__restrict__ bias, int M, int N, int bm,
                                           int bn, const f32x4 (&acc)[S::TM][S::TN], float *__restrict__ out) {
  constexpr int kSeg = S::seg, kLanes = kSeg / 4;
  static_assert(S::lds >= S::waves * 16 * kSeg * 4, "LDS too small for the epilogue");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave / S::WN) * S::RM, wn = (wave % S::WN) * S::RN;
  float bv[S::RN / kSeg][4];
#pragma unroll
  for (int sg = 0; sg < S::RN / kSeg; ++sg)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = bn + wn + sg * kSeg + (lane % kLanes) * 4 + r;
      bv[sg][r] = (bias && n < N) ? bias[n] : 0.0f;
    }
  wait_barrier<0>();
  slab_store<S, kAux>(reinterpret_cast<f32x4 *>(smem) + wave * 16 * kLanes, bv, M, N, bm + wm, bn + wn, acc, out);
}

}  // namespace fusion
