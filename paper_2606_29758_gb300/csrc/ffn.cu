// The gated feed-forward block of a policy layer on the tcgen05 tensor cores (sm_103a), forward and backward.
//
//   G = X Wg^T, U = X Wu^T, A = s(G) U, Y = A Wd^T                 s: silu or gelu
//   dA = dY Wd, dU = dA s(G), dG = dA U s'(G)
//   dX = dG Wg + dU Wu, dWg = dG^T X, dWu = dU^T X, dWd = dY^T A
//
// Forward: one product whose tile holds 128 columns of G and the same columns of U, so that the epilogue has both and
// writes A; then A Wd^T. For a backward the first product also keeps P = U s'(G) and Q = s(G) (the store), and the
// backward's first product, dA, turns them into dG = dA P and dU = dA Q in its epilogue, in place. So a training
// step executes the 18 N d F FLOPs of its six products and no recomputation, and no f32 N x F value reaches memory.
// A, dG and dU are rounded to bf16, the operand type of the products that read them; P and Q are kept in f16 relative to
// a power of two per row and 32 columns (2^-11 of the value down to 2^-28 of the slice's largest, 2^-39 of the largest
// below that), which in bf16 would have been a third rounding of 2^-8 under dX and dW.
#include <cuda_runtime.h>
#include <stdint.h>

#include <climits>

#include "internal.h"
#include "ps_nvtx.h"
#include "umma_host.cuh"

namespace psk {

// ============================================================================= epilogues
// A slice of 32 rows x 32 2-byte values (this lane's row: pk) through one of the warp's two staging buffers.
static __device__ __forceinline__ void store_slice16(const uint32_t (&pk)[16], uint8_t* bufs, uint32_t& stored, int lane,
                                                     const CUtensorMap* map, int col0, int row_base) {
  uint8_t* buf = bufs + (stored++ & 1u) * (32 * 64);
  if (lane == 0) bulk_wait_group_read<1>();   // the store before the last one has read this buffer
  __syncwarp();
  uint4* dst = reinterpret_cast<uint4*>(buf + lane * 64);
  const int x = (lane >> 1) & 3;
#pragma unroll
  for (int q = 0; q < 4; ++q) dst[q ^ x] = make_uint4(pk[4 * q], pk[4 * q + 1], pk[4 * q + 2], pk[4 * q + 3]);
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    tma_store_2d(map, buf, col0, row_base);
    bulk_commit_group();
  }
}

// The exponent e (biased, as in f32) of the power of two that a slice is kept relative to: its largest value over 2^e
// lies in [2^14, 2^15), the top of f16's range (2^14: the exponent's clamp leaves 2^e and 2^-e exact f32 factors).
static __device__ __forceinline__ uint32_t slice_exponent(float largest) {
  const uint32_t e = (__float_as_uint(largest) >> 23) & 255u;
  return min(max(e, 15u), 254u) - 14u;
}

template <int ACT>
static __device__ __forceinline__ void act_and_slope(float g, float& q, float& slope) {
  if (ACT == PS_ACT_SILU) {
    const float sig = __fdividef(1.f, 1.f + ex2_ftz(-g * kLog2e));
    q = g * sig;
    slope = fmaf(q, 1.f - sig, sig);
  } else {
    const float cdf = 0.5f * erfcf(-0.70710678f * g);
    q = g * cdf;
    slope = fmaf(g, 0.39894228f * ex2_ftz(-0.5f * kLog2e * g * g), cdf);
  }
}

// Gate and up slices -> A, and for a backward P, Q and their exponents.
template <int ACT, bool KEEP>
struct FfnUpEpi {
  static constexpr int kEpiWarps = 8;
  static constexpr bool kTmaStore = true, kReadAhead = false, kOwnStore = true;
  static constexpr int kStageBytes = 2 * 32 * 64;
  struct Params {
    int M, F;
    uint32_t* scale;   // [ceil(F / 32)][M]
  };
  struct State {};
  struct Ahead {};
  static __device__ __forceinline__ int cols(const Params& p) { return p.F; }
  static __device__ __forceinline__ void begin_unit(const Params&, State&, int, int) {}
  static __device__ __forceinline__ void end_unit(const Params&, State&, int, int) {}
  static __device__ __forceinline__ void load_ahead(const Params&, int, int, Ahead&) {}
  static __device__ __forceinline__ void chunk_own(const Params& p, int row, int col0, const uint32_t (&rg)[32],
                                                   const uint32_t (&ru)[32], const Ahead&, uint8_t* bufs,
                                                   uint32_t& stored, int lane, int row_base, const CUtensorMap* mapA,
                                                   const CUtensorMap* mapP, const CUtensorMap* mapQ) {
    uint32_t pk[16];
    float q[32], s[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) act_and_slope<ACT>(__uint_as_float(rg[j]), q[j], s[j]);
#pragma unroll
    for (int j = 0; j < 16; ++j)
      pk[j] = pack_bf16x2(q[2 * j] * __uint_as_float(ru[2 * j]), q[2 * j + 1] * __uint_as_float(ru[2 * j + 1]));
    store_slice16(pk, bufs, stored, lane, mapA, col0, row_base);
    if (!KEEP) return;
    float mp = 0.f, mq = 0.f;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      s[j] *= __uint_as_float(ru[j]);
      mp = fmaxf(mp, fabsf(s[j]));
      mq = fmaxf(mq, fabsf(q[j]));
    }
    const uint32_t ep = slice_exponent(mp), eq = slice_exponent(mq);
    const float ip = __uint_as_float((254u - ep) << 23), iq = __uint_as_float((254u - eq) << 23);
#pragma unroll
    for (int j = 0; j < 16; ++j) pk[j] = pack_f16x2(s[2 * j] * ip, s[2 * j + 1] * ip);
    store_slice16(pk, bufs, stored, lane, mapP, col0, row_base);
#pragma unroll
    for (int j = 0; j < 16; ++j) pk[j] = pack_f16x2(q[2 * j] * iq, q[2 * j + 1] * iq);
    store_slice16(pk, bufs, stored, lane, mapQ, col0, row_base);
    if (row < p.M) p.scale[static_cast<int64_t>(col0 >> 5) * p.M + row] = ep | eq << 8;
  }
};

// A dA slice with the kept P and Q of the same place -> dG and dU over them.
struct FfnDaEpi {
  static constexpr int kEpiWarps = 8;
  static constexpr bool kTmaStore = true, kReadAhead = false, kOwnStore = true;
  static constexpr int kStageBytes = 2 * 32 * 64;
  struct Params {
    int M, F;
    const uint16_t *P, *Q;   // [M][F]
    const uint32_t* scale;
  };
  struct State {};
  struct Ahead {
    uint4 p[4], q[4];
    uint32_t scale;
  };
  static __device__ __forceinline__ int cols(const Params& p) { return p.F; }
  static __device__ __forceinline__ void begin_unit(const Params&, State&, int, int) {}
  static __device__ __forceinline__ void end_unit(const Params&, State&, int, int) {}
  static __device__ __forceinline__ void load_ahead(const Params& p, int row, int col0, Ahead& a) {
    const bool in = row < p.M;
    const int64_t at = static_cast<int64_t>(row) * p.F + col0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool here = in && col0 + 8 * i < p.F;   // F is a multiple of 8
      a.p[i] = here ? *reinterpret_cast<const uint4*>(p.P + at + 8 * i) : make_uint4(0, 0, 0, 0);
      a.q[i] = here ? *reinterpret_cast<const uint4*>(p.Q + at + 8 * i) : make_uint4(0, 0, 0, 0);
    }
    a.scale = in && col0 < p.F ? p.scale[static_cast<int64_t>(col0 >> 5) * p.M + row] : 0u;
  }
  static __device__ __forceinline__ void chunk_own(const Params&, int, int col0, const uint32_t (&r)[32],
                                                   const uint32_t (&)[1], const Ahead& a, uint8_t* bufs,
                                                   uint32_t& stored, int lane, int row_base, const CUtensorMap* mapG,
                                                   const CUtensorMap* mapU, const CUtensorMap*) {
    auto out = [&](const uint4 (&kept)[4], float factor, const CUtensorMap* map) {
      const uint32_t w[16] = {kept[0].x, kept[0].y, kept[0].z, kept[0].w, kept[1].x, kept[1].y, kept[1].z, kept[1].w,
                              kept[2].x, kept[2].y, kept[2].z, kept[2].w, kept[3].x, kept[3].y, kept[3].z, kept[3].w};
      uint32_t pk[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float2 v = unpack_f16x2(w[j]);
        pk[j] = pack_bf16x2(__uint_as_float(r[2 * j]) * v.x * factor, __uint_as_float(r[2 * j + 1]) * v.y * factor);
      }
      store_slice16(pk, bufs, stored, lane, map, col0, row_base);
    };
    out(a.p, __uint_as_float((a.scale & 255u) << 23), mapG);
    out(a.q, __uint_as_float((a.scale >> 8 & 255u) << 23), mapU);
  }
};

// ============================================================================= host side
struct FfnStore {
  uint16_t *A, *P, *Q;   // [N][F] each
  uint32_t* scale;       // [ceil(F / 32)][N]: the biased exponents of P (bits 0-7) and Q (8-15)
  size_t bytes;
};
static FfnStore ffn_store(void* base, int64_t N, int F) {
  const size_t plane = (static_cast<size_t>(N) * F * 2 + 255) / 256 * 256;
  uint8_t* b = static_cast<uint8_t*>(base);
  FfnStore f;
  f.A = reinterpret_cast<uint16_t*>(b);
  f.P = reinterpret_cast<uint16_t*>(b + plane);
  f.Q = reinterpret_cast<uint16_t*>(b + 2 * plane);
  f.scale = reinterpret_cast<uint32_t*>(b + 3 * plane);
  f.bytes = 3 * plane + (static_cast<size_t>(N) * ((F + 31) / 32) * 4 + 255) / 256 * 256;
  return f;
}

// Row blocks walked together: the X (or dY) rows of a band stay in a quarter of L2 while the weights stream by.
static int band_of_rows(int64_t K, int halves) {
  const int b = static_cast<int>(30e6 / (2.0 * K * kBM * halves));
  return b < 1 ? 1 : b;
}
constexpr int kBandLongK = 4;   // products with a long K loop: column tiles of 4 row blocks side by side

template <int ACT, bool KEEP>
static int ffn_up(int64_t N, int d, int F, const void* X, int64_t ldx, const void* Wg, const void* Wu,
                  const FfnStore& f, uint32_t* status, cudaStream_t s) {
  using Epi = FfnUpEpi<ACT, KEEP>;
  const int halves = tile_halves(N, 2 * static_cast<int64_t>(F), 18);
  TwoMaps m;
  if (!map_kmajor(&m.a, X, N, d, ldx, kBM * halves) || !map_kmajor(&m.b, Wg, F, d, d, kBN / 2) ||
      !map_kmajor(&m.b2, Wu, F, d, d, kBN / 2) || !map_out_16(&m.c, f.A, N, F, F))
    return PS_ERR_INVALID_ARG;
  m.a2 = m.a;
  m.c2 = m.c3 = m.c;
  if (KEEP && (!map_out_16(&m.c2, f.P, N, F, F, CU_TENSOR_MAP_DATA_TYPE_FLOAT16) ||
               !map_out_16(&m.c3, f.Q, N, F, F, CU_TENSOR_MAP_DATA_TYPE_FLOAT16)))
    return PS_ERR_INVALID_ARG;
  const typename Epi::Params ep{static_cast<int>(N), F, f.scale};
  const int band = band_of_rows(d, halves);
  return halves == 1 ? launch_gemm_two<false, false, Epi, 1, kTwoB>(m, N, F, d, band, ep, status, s, true)
                     : launch_gemm_two<false, false, Epi, 2, kTwoB>(m, N, F, d, band, ep, status, s, true);
}

static int ffn_down(int64_t N, int d, int F, const void* A, const void* Wd, void* Y, int64_t ldy, uint32_t* status,
                    cudaStream_t s) {
  const int halves = tile_halves(N, d, 18);
  CUtensorMap ta, tb, tc;
  if (!map_kmajor(&ta, A, N, F, F, kBM * halves) || !map_kmajor(&tb, Wd, d, F, F, kBN) || !map_out_16(&tc, Y, N, d, ldy))
    return PS_ERR_INVALID_ARG;
  const StoreBf16Epi::Params ep{d};
  return halves == 1
             ? launch_gemm_single<false, false, StoreBf16Epi, 1>(ta, tb, tc, N, d, F, 0, 2 * kBandLongK, ep, status, s)
             : launch_gemm_single<false, false, StoreBf16Epi, 2>(ta, tb, tc, N, d, F, 0, kBandLongK, ep, status, s);
}

// dA = dY Wd and, from the kept P and Q, dG and dU over them.
static int ffn_da(int64_t N, int d, int F, const void* dY, int64_t lddy, const void* Wd, const FfnStore& f,
                  uint32_t* status, cudaStream_t s) {
  const int halves = tile_halves(N, F, 18);
  TwoMaps m;
  if (!map_kmajor(&m.a, dY, N, d, lddy, kBM * halves) || !map_mnmajor(&m.b, Wd, d, F, F) ||
      !map_out_16(&m.c, f.P, N, F, F) || !map_out_16(&m.c2, f.Q, N, F, F))
    return PS_ERR_INVALID_ARG;
  m.a2 = m.a;
  m.b2 = m.b;
  m.c3 = m.c;
  const FfnDaEpi::Params ep{static_cast<int>(N), F, f.P, f.Q, f.scale};
  const int band = band_of_rows(d, halves);
  return halves == 1 ? launch_gemm_two<false, true, FfnDaEpi, 1, kNoPair>(m, N, F, d, band, ep, status, s, true)
                     : launch_gemm_two<false, true, FfnDaEpi, 2, kNoPair>(m, N, F, d, band, ep, status, s, true);
}

template <class Epi>
static typename Epi::Params store_params(int N, int accumulate);
template <>
StoreF32Epi::Params store_params<StoreF32Epi>(int N, int accumulate) {
  return {N, accumulate};
}
template <>
StoreBf16Epi::Params store_params<StoreBf16Epi>(int N, int) {
  return {N};
}
template <class Epi>
static bool map_out(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t pitch) {
  return std::is_same<Epi, StoreF32Epi>::value ? map_out_f32(m, base, rows, cols, pitch)
                                               : map_out_16(m, base, rows, cols, pitch);
}

// dX (+)= dG Wg + dU Wu
template <class Epi>
static int ffn_dx(int64_t N, int d, int F, const FfnStore& f, const void* Wg, const void* Wu, void* dX, int64_t lddx,
                  int accumulate, uint32_t* status, cudaStream_t s) {
  const int halves = tile_halves(N, d, 18);
  TwoMaps m;
  if (!map_kmajor(&m.a, f.P, N, F, F, kBM * halves) || !map_kmajor(&m.a2, f.Q, N, F, F, kBM * halves) ||
      !map_mnmajor(&m.b, Wg, F, d, d) || !map_mnmajor(&m.b2, Wu, F, d, d) || !map_out<Epi>(&m.c, dX, N, d, lddx))
    return PS_ERR_INVALID_ARG;
  m.c2 = m.c3 = m.c;
  const auto ep = store_params<Epi>(d, accumulate);
  return halves == 1 ? launch_gemm_two<false, true, Epi, 1, kSumK>(m, N, d, F, 2 * kBandLongK, ep, status, s, false)
                     : launch_gemm_two<false, true, Epi, 2, kSumK>(m, N, d, F, kBandLongK, ep, status, s, false);
}

// dWg (+)= dG^T X and dWu (+)= dU^T X, one below the other
template <class Epi>
static int ffn_dw_up(int64_t N, int d, int F, const FfnStore& f, const void* X, int64_t ldx, void* dWg, void* dWu,
                     int accumulate, uint32_t* status, cudaStream_t s) {
  TwoMaps m;
  if (!map_mnmajor(&m.a, f.P, N, F, F) || !map_mnmajor(&m.a2, f.Q, N, F, F) || !map_mnmajor(&m.b, X, N, d, ldx) ||
      !map_out<Epi>(&m.c, dWg, F, d, d) || !map_out<Epi>(&m.c2, dWu, F, d, d))
    return PS_ERR_INVALID_ARG;
  m.b2 = m.b;
  m.c3 = m.c;
  const auto ep = store_params<Epi>(d, accumulate);
  const int halves = tile_halves(2 * static_cast<int64_t>(F), d, 17);
  return halves == 1 ? launch_gemm_two<true, true, Epi, 1, kTwoM>(m, F, d, N, 2 * kBandLongK, ep, status, s, false)
                     : launch_gemm_two<true, true, Epi, 2, kTwoM>(m, F, d, N, kBandLongK, ep, status, s, false);
}

// dWd (+)= dY^T A
template <class Epi>
static int ffn_dw_down(int64_t N, int d, int F, const void* dY, int64_t lddy, const FfnStore& f, void* dWd,
                       int accumulate, uint32_t* status, cudaStream_t s) {
  CUtensorMap ta, tb, tc;
  if (!map_mnmajor(&ta, dY, N, d, lddy) || !map_mnmajor(&tb, f.A, N, F, F) || !map_out<Epi>(&tc, dWd, d, F, F))
    return PS_ERR_INVALID_ARG;
  const auto ep = store_params<Epi>(F, accumulate);
  const int halves = tile_halves(d, F, 17);
  return halves == 1 ? launch_gemm_single<true, true, Epi, 1>(ta, tb, tc, d, F, N, 0, 2 * kBandLongK, ep, status, s)
                     : launch_gemm_single<true, true, Epi, 2>(ta, tb, tc, d, F, N, 0, kBandLongK, ep, status, s);
}

static bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
static bool ld_ok(int64_t ld, int64_t cols, int64_t step) { return ld >= cols && ld % step == 0; }
// Rows whose tiles, and sizes whose k loops, the kernels count in 32 bits.
static bool sizes_ok(int64_t N, int d, int F) {
  return N >= 0 && d >= 8 && F >= 8 && d % 8 == 0 && F % 8 == 0;
}
static bool sizes_fit(int64_t N, int d, int F) {
  if (N > (1 << 30) || d > (1 << 24) || F > (1 << 24)) return false;
  const int64_t w = d > F ? d : F;
  return (N / kBM + 1) * (w / 128 + 2) <= INT32_MAX && (2 * (w / kBM) + 2) * (w / kBN + 1) <= INT32_MAX;
}

}  // namespace psk

using namespace psk;

extern "C" {

size_t ps_gated_ffn_store_size(int64_t N, int F) {
  if (N < 0 || F < 8 || F % 8) return 0;
  return ffn_store(nullptr, N, F).bytes;
}

size_t ps_gated_ffn_fwd_workspace_size(int64_t N, int F, int with_store) {
  if (N < 0 || F < 8 || F % 8) return 0;
  return kWsHeader + (with_store ? 0 : static_cast<size_t>(N) * F * 2);
}

int ps_gated_ffn_fwd(int64_t N, int d, int F, int dtype, int act, const void* X, int64_t ldx, const void* Wg,
                     const void* Wu, const void* Wd, void* Y, int64_t ldy, void* store, size_t store_bytes, void* ws,
                     size_t ws_bytes, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_gated_ffn_fwd");
  if (!sizes_ok(N, d, F) || (act != PS_ACT_SILU && act != PS_ACT_GELU)) return PS_ERR_INVALID_ARG;
  if (dtype != PS_DTYPE_BF16) return dtype == PS_DTYPE_F32 ? PS_ERR_UNSUPPORTED : PS_ERR_INVALID_ARG;
  if (!ld_ok(ldx, d, 8) || !ld_ok(ldy, d, 8)) return PS_ERR_INVALID_ARG;
  if (N > 0 && (!X || !Wg || !Wu || !Wd || !Y || !al16(X) || !al16(Wg) || !al16(Wu) || !al16(Wd) || !al16(Y)))
    return PS_ERR_INVALID_ARG;
  if (store && (!al16(store) || store_bytes < ffn_store(nullptr, N, F).bytes))
    return al16(store) ? PS_ERR_WORKSPACE : PS_ERR_INVALID_ARG;
  if (!sizes_fit(N, d, F) || !device_is_sm103()) return PS_ERR_UNSUPPORTED;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int rc = check_ws(ws, ws_bytes, ps_gated_ffn_fwd_workspace_size(N, F, store != nullptr));
  if (rc != PS_OK) return rc;
  if (N == 0) return refused(PS_OK, ws, s);
  uint32_t* status = static_cast<uint32_t*>(ws);
  FfnStore f = ffn_store(store, N, F);
  if (!store) f.A = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(ws) + kWsHeader);
  if (act == PS_ACT_SILU)
    rc = store ? ffn_up<PS_ACT_SILU, true>(N, d, F, X, ldx, Wg, Wu, f, status, s)
               : ffn_up<PS_ACT_SILU, false>(N, d, F, X, ldx, Wg, Wu, f, status, s);
  else
    rc = store ? ffn_up<PS_ACT_GELU, true>(N, d, F, X, ldx, Wg, Wu, f, status, s)
               : ffn_up<PS_ACT_GELU, false>(N, d, F, X, ldx, Wg, Wu, f, status, s);
  if (rc != PS_OK) return refused(rc, ws, s);
  return ffn_down(N, d, F, f.A, Wd, Y, ldy, status, s);
}

size_t ps_gated_ffn_bwd_workspace_size(void) { return kWsHeader; }

int ps_gated_ffn_bwd(int64_t N, int d, int F, int dtype, const void* dY, int64_t lddy, const void* X, int64_t ldx,
                     const void* Wg, const void* Wu, const void* Wd, void* store, size_t store_bytes, void* dX,
                     int64_t lddx, int dx_dtype, void* dWg, void* dWu, void* dWd, int dw_dtype, int flags, void* ws,
                     size_t ws_bytes, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_gated_ffn_bwd");
  if (!sizes_ok(N, d, F) || (flags & ~(PS_DW_ACCUMULATE | PS_DH_ACCUMULATE))) return PS_ERR_INVALID_ARG;
  if (dtype != PS_DTYPE_BF16) return dtype == PS_DTYPE_F32 ? PS_ERR_UNSUPPORTED : PS_ERR_INVALID_ARG;
  if ((dx_dtype != PS_DTYPE_BF16 && dx_dtype != PS_DTYPE_F32) || (dw_dtype != PS_DTYPE_BF16 && dw_dtype != PS_DTYPE_F32))
    return PS_ERR_INVALID_ARG;
  // sums over calls are kept in f32
  if ((flags & PS_DH_ACCUMULATE && dx_dtype != PS_DTYPE_F32) || (flags & PS_DW_ACCUMULATE && dw_dtype != PS_DTYPE_F32))
    return PS_ERR_UNSUPPORTED;
  if (!ld_ok(lddy, d, 8) || !ld_ok(ldx, d, 8) || (dX && !ld_ok(lddx, d, dx_dtype == PS_DTYPE_F32 ? 4 : 8)))
    return PS_ERR_INVALID_ARG;
  if ((dWg == nullptr) != (dWu == nullptr)) return PS_ERR_INVALID_ARG;
  if (!al16(dX) || !al16(dWg) || !al16(dWu) || !al16(dWd)) return PS_ERR_INVALID_ARG;
  if (N > 0 && (!dY || !X || !Wg || !Wu || !Wd || !store || !al16(dY) || !al16(X) || !al16(Wg) || !al16(Wu) ||
                !al16(Wd) || !al16(store)))
    return PS_ERR_INVALID_ARG;
  if (N > 0 && store_bytes < ffn_store(nullptr, N, F).bytes) return PS_ERR_WORKSPACE;
  if (!sizes_fit(N, d, F) || !device_is_sm103()) return PS_ERR_UNSUPPORTED;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int rc = check_ws(ws, ws_bytes, kWsHeader);
  if (rc != PS_OK) return rc;
  uint32_t* status = static_cast<uint32_t*>(ws);
  const int dw_acc = (flags & PS_DW_ACCUMULATE) ? 1 : 0, dx_acc = (flags & PS_DH_ACCUMULATE) ? 1 : 0;
  if (N == 0) {
    refused(PS_OK, ws, s);
    const size_t bytes = static_cast<size_t>(d) * F * (dw_dtype == PS_DTYPE_F32 ? 4 : 2);
    for (void* g : {dWg, dWu, dWd})
      if (g && !dw_acc && cudaMemsetAsync(g, 0, bytes, s) != cudaSuccess) return PS_ERR_CUDA;
    return PS_OK;
  }
  const FfnStore f = ffn_store(store, N, F);
  rc = ffn_da(N, d, F, dY, lddy, Wd, f, status, s);
  if (rc != PS_OK) return refused(rc, ws, s);
  if (dX) {
    rc = dx_dtype == PS_DTYPE_F32 ? ffn_dx<StoreF32Epi>(N, d, F, f, Wg, Wu, dX, lddx, dx_acc, status, s)
                                  : ffn_dx<StoreBf16Epi>(N, d, F, f, Wg, Wu, dX, lddx, 0, status, s);
    if (rc != PS_OK) return rc;
  }
  if (dWg) {
    rc = dw_dtype == PS_DTYPE_F32 ? ffn_dw_up<StoreF32Epi>(N, d, F, f, X, ldx, dWg, dWu, dw_acc, status, s)
                                  : ffn_dw_up<StoreBf16Epi>(N, d, F, f, X, ldx, dWg, dWu, 0, status, s);
    if (rc != PS_OK) return rc;
  }
  if (dWd) {
    rc = dw_dtype == PS_DTYPE_F32 ? ffn_dw_down<StoreF32Epi>(N, d, F, dY, lddy, f, dWd, dw_acc, status, s)
                                  : ffn_dw_down<StoreBf16Epi>(N, d, F, dY, lddy, f, dWd, 0, status, s);
    if (rc != PS_OK) return rc;
  }
  return PS_OK;
}

}  // extern "C"
