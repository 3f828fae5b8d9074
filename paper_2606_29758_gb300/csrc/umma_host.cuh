// Host side of the tensor-core products (umma_gemm.cuh): tensor maps, the choice of the tile's height, launches,
// and the epilogues that store the accumulator as it is.
#pragma once

#include "internal.h"
#include "umma_gemm.cuh"

namespace psk {

// The accumulator itself, f32, overwriting the output or adding to it, through TMA: a warp stages its
// 32 x 32 slices (4 KB) and one lane issues the tensor store or, to accumulate, the tensor reduction,
// which adds in L2 and so waits for no load. The store engine clips rows and columns past the output.
// The output is all this epilogue moves: a tile of a short K loop (dW over a few hundred rows) is
// bound by writing it. dW of 185 rows (3 k-blocks per tile) at d = 3584, V = 152064 takes 336 us, 6.5 TB/s
// of its 2.2 GB, against 860 us with 4 warps that stored 16 bytes per row and instruction from their
// registers.
struct StoreF32Epi {
  static constexpr int kEpiWarps = 8;
  static constexpr bool kTmaStore = true, kReadAhead = true;
  static constexpr int kStageBytes = 32 * 128;
  struct Params {
    int N;
    int accumulate;
  };
  struct State {};
  static __device__ __forceinline__ int cols(const Params& p) { return p.N; }
  static __device__ __forceinline__ void begin_unit(const Params&, State&, int, int) {}
  static __device__ __forceinline__ void chunk_to_smem(const Params&, State&, int, int, const uint32_t (&r)[32],
                                                       uint8_t* buf, int lane) {
    uint4* dst = reinterpret_cast<uint4*>(buf + lane * 128);
#pragma unroll
    for (int q = 0; q < 8; ++q) dst[q ^ (lane & 7)] = make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]);
  }
  static __device__ __forceinline__ void store(const Params& p, const CUtensorMap* map, const uint8_t* buf, int col,
                                               int row) {
    if (p.accumulate) tma_reduce_add_2d(map, buf, col, row);
    else tma_store_2d(map, buf, col, row);
  }
  static __device__ __forceinline__ void end_unit(const Params&, State&, int, int) {}
};

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's function of this name, nullptr if it has none.
static void* driver_fn(const char* name) {
  void* p = nullptr;
  cudaDriverEntryPointQueryResult q;
  return cudaGetDriverEntryPointByVersion(name, &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                 q == cudaDriverEntryPointSuccess
             ? p
             : nullptr;
}
static EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = reinterpret_cast<EncodeTiledFn>(driver_fn("cuTensorMapEncodeTiled"));
  return fn;
}

// 2-D tensor of bf16 elements (unless `type` says otherwise) [outer][inner] with row pitch
// `pitch_bytes`, 128-byte swizzled boxes unless `swizzle` says otherwise.
static bool make_map(CUtensorMap* m, const void* base, uint64_t inner, uint64_t outer, uint64_t pitch_bytes,
                     uint32_t box_inner, uint32_t box_outer,
                     CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B,
                     CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  if ((reinterpret_cast<uintptr_t>(base) & 15) || (pitch_bytes & 15)) return false;
  const cuuint64_t dims[2] = {inner, outer};
  const cuuint64_t strides[1] = {pitch_bytes};
  const cuuint32_t box[2] = {box_inner, box_outer};
  const cuuint32_t estr[2] = {1, 1};
  return enc(m, type, 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Operand maps. K-major [rows][K]: box 64 (K) x rows_box. MN-major [K][MN]: box 64 x 64.
static bool map_kmajor(CUtensorMap* m, const void* base, int64_t rows, int64_t K, int64_t pitch_elems,
                       uint32_t rows_box) {
  return make_map(m, base, K, rows, pitch_elems * 2, kBK, rows_box);
}
// Output map of StoreF32Epi: f32 [rows][cols], 32 x 32 boxes from 128-byte-swizzled staging.
static bool map_out_f32(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t pitch_elems) {
  return make_map(m, base, cols, rows, pitch_elems * 4, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_DATA_TYPE_FLOAT32);
}
// Output map of 2-byte elements [rows][cols]: 32 x 32 boxes from 64-byte-swizzled staging.
static bool map_out_16(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t pitch_elems,
                       CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16) {
  return make_map(m, base, cols, rows, pitch_elems * 2, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B, type);
}
// Output map of bf16 [rows][cols]: boxes of 32 rows x 64 columns from 128-byte-swizzled staging.
static bool map_out_bf16(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t pitch_elems) {
  return make_map(m, base, cols, rows, pitch_elems * 2, 64, 32);
}
static bool map_mnmajor(CUtensorMap* m, const void* base, int64_t K, int64_t MN, int64_t pitch_elems) {
  return make_map(m, base, MN, K, pitch_elems * 2, 64, kBK);
}

template <bool A_MN, bool B_MN, class Epi, int HALVES = 1>
static int launch_gemm_single(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc, int64_t M,
                              int64_t N, int64_t K, int splits, int band_m, const typename Epi::Params& ep,
                              uint32_t* status, cudaStream_t s, bool clear = false) {
  Sched sc;
  sc.clear = clear ? 1 : 0;
  sc.m_blocks = static_cast<int>((M + kBM * HALVES - 1) / (kBM * HALVES));
  sc.n_blocks = static_cast<int>((N + kBN - 1) / kBN);
  sc.splits = splits > 0 ? splits : sc.n_blocks;
  sc.band_m = band_m > 0 ? band_m : 1;
  sc.num_units = sc.m_blocks * sc.splits;
  sc.num_kb = static_cast<int>((K + kBK - 1) / kBK);
  if (sc.num_units == 0) return PS_OK;
  if (sc.num_kb == 0) return PS_ERR_INVALID_ARG;
  auto kern = umma_gemm_kernel<A_MN, B_MN, Epi, HALVES>;
  constexpr int EW = EpiWarps<Epi>::value;
  constexpr size_t smem = gemm_smem_bytes<HALVES, Epi>();
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) !=
      cudaSuccess)
    return PS_ERR_CUDA;
  const int grid = sc.num_units < num_sms_current() ? sc.num_units : num_sms_current();
  return launch_after(kern, dim3(static_cast<unsigned>(grid)), 64 + 32 * EW, smem, s, 1, 1, !clear, ta, tb, tc, sc, ep,
                      status, kDefaultTimeoutNs) == cudaSuccess
             ? PS_OK
             : PS_ERR_CUDA;
}

// The maps of a product with two B operands or several outputs; the unused ones repeat another.
struct TwoMaps {
  CUtensorMap a, b, c, b2, c2, c3;
};

// M x N outputs of each product.
template <bool A_MN, bool B_MN, class Epi, int HALVES, int PAIR>
static int launch_gemm_two(const TwoMaps& m, int64_t M, int64_t N, int64_t K, int band_m,
                           const typename Epi::Params& ep, uint32_t* status, cudaStream_t s, bool clear) {
  Sched sc;
  sc.clear = clear ? 1 : 0;
  constexpr int tn = PAIR == kTwoB ? kBN / 2 : kBN;
  sc.m_blocks = static_cast<int>((M + kBM * HALVES - 1) / (kBM * HALVES));
  sc.n_blocks = static_cast<int>((N + tn - 1) / tn);
  sc.splits = sc.n_blocks;
  sc.band_m = band_m > 0 ? band_m : 1;
  sc.num_units = sc.m_blocks * sc.splits;
  sc.num_kb = static_cast<int>((K + kBK - 1) / kBK);
  if (sc.num_units == 0) return PS_OK;
  if (sc.num_kb == 0) return PS_ERR_INVALID_ARG;
  auto kern = umma_gemm_two_kernel<A_MN, B_MN, Epi, HALVES, PAIR>;
  constexpr size_t smem = gemm_smem_bytes<HALVES, Epi>();
  static_assert(smem <= 232448, "shared memory of one CTA");
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess)
    return PS_ERR_CUDA;
  const int grid = sc.num_units < num_sms_current() ? sc.num_units : num_sms_current();
  return launch_after(kern, dim3(static_cast<unsigned>(grid)), 64 + 32 * EpiWarps<Epi>::value, smem, s, 1, 1, !clear,
                      m.a, m.b, m.c, m.b2, m.c2, m.c3, sc, ep, status, kDefaultTimeoutNs) == cudaSuccess
             ? PS_OK
             : PS_ERR_CUDA;
}

// The same on CTA pairs (A K-major, one 256 x TN tile a pair): the A map's boxes are of 128 rows, B's of 128 as well.
template <bool B_MN, class Epi, int PAIR>
static int launch_pair_own(const TwoMaps& m, int64_t M, int64_t N, int64_t K, int band_m, const typename Epi::Params& ep,
                           uint32_t* status, cudaStream_t s, bool clear) {
  const int pairs = clusters_at_once(0);
  if (pairs < 1) return PS_ERR_CUDA;
  Sched sc;
  sc.clear = clear ? 1 : 0;
  constexpr int tn = PAIR == kTwoB ? kBN / 2 : kBN;
  sc.m_blocks = static_cast<int>((M + 255) / 256);
  sc.n_blocks = static_cast<int>((N + tn - 1) / tn);
  sc.splits = sc.n_blocks;
  sc.band_m = band_m > 0 ? band_m : 1;
  sc.num_units = sc.m_blocks * sc.splits;
  sc.num_kb = static_cast<int>((K + kBK - 1) / kBK);
  auto kern = umma_pair_own_kernel<B_MN, Epi, PAIR>;
  constexpr size_t smem = sizeof(PairOwnSmem<Epi>) + 1024;
  static_assert(smem <= 232448, "shared memory of one CTA");
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess)
    return PS_ERR_CUDA;
  const int n = sc.num_units < pairs ? sc.num_units : pairs;
  if (launch_after(kern, dim3(static_cast<unsigned>(2 * n)), 320, smem, s, 2, 1, true, m.a, m.b, m.c, m.b2, m.c2, m.c3, sc,
                   ep, status, kDefaultTimeoutNs) == cudaSuccess)
    return PS_OK;
  cudaGetLastError();
  return PS_ERR_CUDA;
}

// Tile height in 128-row halves (see GemmCfg) of a GEMM whose units are M x N tiles. The wide tile moves a third
// fewer operand bytes per FLOP (about 0.8 vs 0.95 pJ per FLOP at the power cap) and takes 1.8-1.95 times as long as
// a 128 x 256 one, so it is the faster of the two unless the narrow one needs clearly fewer than twice its rounds
// over the SMs: when few rows leave its last row block half empty, or few tiles its last round. limit: the most
// narrow rounds per 10 wide ones. Measured, narrow / wide (us):
//   logits recomputed, limit 18: 60 rows, d = 3584, V = 152064 (4 rounds / 4) 174 / 198; 571 rows, d = 512, V =
//     151936 (20 / 12) 88 / 98; 571 rows, d = 392, V = 2000 (1 / 1) 14.2 / 17.2; 200 rows, d = 3584 (8 / 4) 224 / 203
//   forward, limit 18: 60 rows, d = 1536, V = 151936 (4 / 4) 95 / 108; 1200 rows, d = 1024, V = 32000 (9 / 5) 72 / 74;
//     20000 rows, d = 128, V = 9000 (38 / 19) 105 / 89; 3000 rows, d = 768, V = 32000 (20 / 10) 115 / 108
//   forward from d = 2048 on, limit 16: 571 rows, d = 3584 with a store (20 / 12) 495 / 490
//   dW, limit 17: 571 rows, d = 392, V = 2000 (1 / 1) 11.7 / 14.5; 20000 rows, d = 128, V = 9000 (1 / 1) 118 / 190; 1200
//     rows, d = 768, V = 32000 (5 / 3) 59 / 63; 8000 rows, d = 1024, V = 32000 (7 / 4) 338 / 325
static int tile_halves(int64_t M, int64_t N, int limit) {
  const int64_t sms = num_sms_current(), nb = (N + kBN - 1) / kBN;
  const int64_t narrow = ((M + kBM - 1) / kBM * nb + sms - 1) / sms;
  const int64_t wide = ((M + 2 * kBM - 1) / (2 * kBM) * nb + sms - 1) / sms;
  return narrow * 10 <= wide * limit ? 1 : 2;
}

}  // namespace psk
