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
// A, dG and dU are rounded to bf16, the operand type of the products that read them (few rows of narrow blocks: in two
// parts, see kept_parts); P and Q are kept in f16 relative to a power of two per row and 32 columns (2^-11 of the value
// down to 2^-28 of the slice's largest, 2^-39 of the largest below that), which in bf16 would have been a third rounding
// of 2^-8 under dX and dW.
#include <cuda_runtime.h>
#include <stdint.h>

#include <climits>

#include "internal.h"
#include "ps_nvtx.h"
#include "psppo_diag.h"
#include "umma_group.cuh"
#include "umma_host.cuh"

namespace psk {

// ============================================================================= epilogues
// A slice of 32 rows x 32 2-byte values (this lane's row: pk) through one of the warp's BUFS staging buffers in turn.
template <int BUFS>
static __device__ __forceinline__ void store_slice16(const uint32_t (&pk)[16], uint8_t* bufs, uint32_t& stored, int lane,
                                                     const CUtensorMap* map, int col0, int row_base) {
  uint8_t* buf = bufs + (stored++ % BUFS) * (32 * 64);
  if (lane == 0) bulk_wait_group_read<BUFS - 1>();   // the store that last used this buffer has read it
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

static __device__ __forceinline__ float finite_size(float x) { return fabsf(x) <= 3.4028235e38f ? fabsf(x) : 0.f; }

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
template <int ACT, bool KEEP, int BUFS>
struct FfnUpEpi {
  static constexpr int kEpiWarps = 8;
  static constexpr bool kTmaStore = true, kReadAhead = false, kOwnStore = true;
  static constexpr int kLoadSets = 0;
  static constexpr int kStageBytes = BUFS * 32 * 64;
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
    store_slice16<BUFS>(pk, bufs, stored, lane, mapA, col0, row_base);
    if (!KEEP) return;
    float mp = 0.f, mq = 0.f;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      s[j] *= __uint_as_float(ru[j]);
      mp = fmaxf(mp, fabsf(s[j]));
      mq = fmaxf(mq, fabsf(q[j]));
    }
    if (fmaxf(mp, mq) > 3.4028235e38f) {   // beside an infinity the finite values keep their own scale
      mp = mq = 0.f;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        mp = fmaxf(mp, finite_size(s[j]));
        mq = fmaxf(mq, finite_size(q[j]));
      }
    }
    const uint32_t ep = slice_exponent(mp), eq = slice_exponent(mq);
    const float ip = __uint_as_float((254u - ep) << 23), iq = __uint_as_float((254u - eq) << 23);
#pragma unroll
    for (int j = 0; j < 16; ++j) pk[j] = pack_f16x2(s[2 * j] * ip, s[2 * j + 1] * ip);
    store_slice16<BUFS>(pk, bufs, stored, lane, mapP, col0, row_base);
#pragma unroll
    for (int j = 0; j < 16; ++j) pk[j] = pack_f16x2(q[2 * j] * iq, q[2 * j + 1] * iq);
    store_slice16<BUFS>(pk, bufs, stored, lane, mapQ, col0, row_base);
    if (row < p.M) p.scale[static_cast<int64_t>(col0 >> 5) * p.M + row] = ep | eq << 8;
  }
};

// A dA slice with the kept P and Q of the same place -> dG and dU over them, in place in the staging buffer too. P and Q
// by TMA: 571 rows at d = 392, F = 1048 13.0 us, 8000 rows at d = 392, F = 2000 33, 6030 at d = 1536, F = 8192 133; into registers
// a slice ahead 16.5, 46 and 121 (with a long K loop the 64-byte rows of the slices are in the operands' way).
struct FfnDaEpi {
  static constexpr int kEpiWarps = 8;
  static constexpr bool kTmaStore = true, kReadAhead = false, kOwnStore = true;
  static constexpr int kLoadSets = 2;
  static constexpr int kStageBytes = kLoadSets * 2 * 32 * 64;
  struct Params {
    int M, F;
    const uint32_t* scale;
  };
  struct State {};
  struct Ahead {
    uint32_t scale[4];   // of the lane's row, for the tile's slices
  };
  static __device__ __forceinline__ int cols(const Params& p) { return p.F; }
  static __device__ __forceinline__ void load_ahead(const Params& p, int row, int first, Ahead& a) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      a.scale[c] = row < p.M && first + 32 * c < p.F ? p.scale[static_cast<int64_t>((first >> 5) + c) * p.M + row] : 0u;
  }
  // One plane of the slice, the lane's own row.
  static __device__ __forceinline__ void plane(const uint32_t (&r)[32], float factor, uint8_t* buf, int lane) {
    uint4* own = reinterpret_cast<uint4*>(buf) + lane * 4;
    const int x = (lane >> 1) & 3;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint4 v = own[q ^ x];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = unpack_f16x2(w[j]);
        o[j] = pack_bf16x2(__uint_as_float(r[8 * q + 2 * j]) * f.x * factor,
                           __uint_as_float(r[8 * q + 2 * j + 1]) * f.y * factor);
      }
      own[q ^ x] = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
  static __device__ __forceinline__ void chunk_own(const Params&, int, int col0, const uint32_t (&r)[32],
                                                   const uint32_t (&)[1], const Ahead& a, uint8_t* bufs,
                                                   uint32_t& set, int lane, int row_base, const CUtensorMap* mapG,
                                                   const CUtensorMap* mapU, const CUtensorMap*) {
    bufs += set * (2 * 32 * 64);
    const int c = (col0 >> 5) & 3;   // (a column group's slices begin at a multiple of 128)
    const uint32_t scale = c == 0 ? a.scale[0] : c == 1 ? a.scale[1] : c == 2 ? a.scale[2] : a.scale[3];
    plane(r, __uint_as_float((scale & 255u) << 23), bufs, lane);
    plane(r, __uint_as_float((scale >> 8 & 255u) << 23), bufs + 32 * 64, lane);
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(mapG, bufs, col0, row_base);
      tma_store_2d(mapU, bufs + 32 * 64, col0, row_base);
      bulk_commit_group();
    }
  }
};

// ============================================================================= few rows
// Up to 128 rows (dA: 64): reading the weights is all that costs (one row at d = 3584, F = 16384: 352 MB), so the weights are the
// 128-row operand of the MMA and the rows its N side (NT = 16 to 128 columns), and every SM streams weights. A CTA takes
// 64 columns of F (their 64 gate and 64 up rows are one tile), or 128 outputs of Y or dA; where that gives too few CTAs a
// cluster shares the K loop, and the partial tiles are added in rank order through distributed shared memory. Two CTAs
// fit on an SM. The second product is launched while the first runs and loads its first weights before it waits for A.
// One row of d = 3584, F = 16384 57 us (6.1 TB/s of weights), 128 rows 73; d = 1536, F = 8192 21 and 33 (the general
// kernels, 128 rows to a tile and F or d / 256 CTAs: 145 and 138, 68 and 66).
constexpr int kFewThreads = 192;
constexpr uint32_t kFewWBytes = 128 * kBK * 2;
template <int NT>
struct FewCfg {
  static constexpr uint32_t kXBytes = NT * kBK * 2;
  static constexpr uint32_t kStage = kFewWBytes + kXBytes;
  static constexpr int kStages = (112 * 1024 - 1024 - 256) / kStage;
  static constexpr uint32_t kCols = NT < 32 ? 32 : NT;
  static_assert(kStages * kStage >= NT * 128 * 4, "the partial tile lies over the ring");
};
template <int NT>
struct FewSmem {
  uint8_t ring[FewCfg<NT>::kStages][FewCfg<NT>::kStage];   // weights, then rows (both 1024-byte aligned)
  uint64_t full[FewCfg<NT>::kStages];
  uint64_t empty[FewCfg<NT>::kStages];
  uint64_t tfull;
  uint32_t tmem_base;
  int abort;
};

static __device__ __forceinline__ float2 ld_cluster_v2(uint32_t cl_addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(cl_addr) : "memory");
  return v;
}

// What the first product keeps for a backward (KEEP), [N][C] and the exponents of each row and 32 columns; what dA turns
// into dG and dU.
struct FewKept {
  uint16_t *P, *Q;
  uint32_t* scale;
  int parts;   // of A, dG and dU: 1, or 2 (see kept_parts)
};
// Two values in bf16, and with two parts what their rounding leaves, `apart` elements further on.
static __device__ __forceinline__ void store_parts(uint16_t* to, int64_t apart, int parts, float x, float y) {
  const uint32_t v = pack_bf16x2(x, y);
  *reinterpret_cast<uint32_t*>(to) = v;
  if (parts == 2) {
    const float hx = __uint_as_float(v << 16), hy = __uint_as_float(v & 0xffff0000u);
    *reinterpret_cast<uint32_t*>(to + apart) =
        pack_bf16x2(fabsf(hx) <= 3.4028235e38f ? x - hx : 0.f, fabsf(hy) <= 3.4028235e38f ? y - hy : 0.f);
  }
}

// kFewUp: out[n][f] = s(x_n . Wg_f) (x_n . Wu_f), tmW and tmW2 the two weights in boxes of 64 rows; kFewDown: out[n][c] =
// x_n . W_c, tmW in boxes of 128 rows; kFewDa: dA[n][f] = sum_c x_n,c W_c,f (W as it lies, MN-major, in boxes of 64 x 64) and
// dG, dU over the kept P, Q. N rows, C output columns (a multiple of 8).
enum FewOp { kFewUp, kFewDown, kFewDa };
template <int NT, int OP, int ACT, bool KEEP>
__global__ void __launch_bounds__(kFewThreads, 2)
    ffn_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmW2,
                   const __grid_constant__ CUtensorMap tmX, int N, int C, int num_kb, uint16_t* out, int64_t ldo,
                   const FewKept kept, uint32_t* status, uint64_t timeout_ns) {
  using Cfg = FewCfg<NT>;
  constexpr int S = Cfg::kStages;
  constexpr bool UP = OP == kFewUp, DA = OP == kFewDa;
  extern __shared__ uint8_t smem_raw[];
  FewSmem<NT>& sm = *reinterpret_cast<FewSmem<NT>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int nranks = static_cast<int>(cluster_nctarank()), rank = static_cast<int>(cluster_ctarank());
  const int unit = blockIdx.x / nranks;
  const int kb0 = static_cast<int>(static_cast<long long>(num_kb) * rank / nranks);
  const int kb1 = static_cast<int>(static_cast<long long>(num_kb) * (rank + 1) / nranks);
  const int row0 = unit * (UP ? 64 : 128);
  const int operand_rows = N * (OP == kFewDown ? kept.parts : 1);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    mbar_init(&sm.tfull, 1);
    sm.abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, Cfg::kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (UP || DA) {   // a call's first kernel: what the calls before it wrote is there from here on
    wait_for_previous_kernel();
    let_next_kernel_in();
    if (blockIdx.x == 0 && threadIdx.x == 0) clear_status(status);   // (a bit is set only after seconds)
  }
  const uint32_t tmem_base = sm.tmem_base;
  volatile int* abort = &sm.abort;

  if (warp == 0) {
    if (lane == 0) {
      auto weights = [&](int kb, int s) {
        mbar_arrive_expect_tx(&sm.full[s], Cfg::kStage);
        if (DA) {
          tma_load_2d(sm.ring[s], &tmW, &sm.full[s], row0, kb * kBK);
          tma_load_2d(sm.ring[s] + kFewWBytes / 2, &tmW, &sm.full[s], row0 + 64, kb * kBK);
          return;
        }
        tma_load_2d(sm.ring[s], &tmW, &sm.full[s], kb * kBK, row0);
        if (UP) tma_load_2d(sm.ring[s] + kFewWBytes / 2, &tmW2, &sm.full[s], kb * kBK, row0);
      };
      auto rows = [&](int kb, int s) { tma_load_2d(sm.ring[s] + kFewWBytes, &tmX, &sm.full[s], kb * kBK, 0); };
      // the weights come from before the call: in its second kernel a ring of them before the rows' kernel is done
      const int ahead = min(S, kb1 - kb0);
      for (int i = 0; i < ahead; ++i) weights(kb0 + i, i);
      if (!UP && !DA) {
        wait_for_previous_kernel();
        let_next_kernel_in();
      }
      for (int i = 0; i < ahead; ++i) rows(kb0 + i, i);
      bool ok = true;
      int kc = ahead;
      for (int kb = kb0 + ahead; kb < kb1; ++kb, ++kc) {
        const int s = kc % S;
        if (!mbar_wait(&sm.empty[s], ((kc / S) & 1u) ^ 1u, timeout_ns, abort)) { ok = false; break; }
        weights(kb, s);
        rows(kb, s);
      }
      if (!ok) {
        *abort = 1;
        raise_status(status, PS_DEV_TIMEOUT);
      }
      // the ring is reused below: every load has landed
      for (int j = kc > S ? kc - S : 0; j < kc; ++j) mbar_wait(&sm.full[j % S], (j / S) & 1u, timeout_ns, nullptr);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_bf16_f32(128, NT, DA, false);
      constexpr uint32_t w_lbo = DA ? kBK * 128 : 16, w_step = DA ? 2048 : 32;
      int kc = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++kc) {
        const int s = kc % S;
        if (!mbar_wait(&sm.full[s], (kc / S) & 1u, timeout_ns, abort)) {
          *abort = 1;
          raise_status(status, PS_DEV_TIMEOUT);
          break;
        }
        tc_fence_after();
        const uint32_t w = smem_addr(sm.ring[s]);
#pragma unroll
        for (int k = 0; k < kBK / 16; ++k)
          umma_bf16(tmem_base, smem_desc_sw128(w + k * w_step, w_lbo, 1024),
                    smem_desc_sw128(w + kFewWBytes + k * 32, 16, 1024),
                    idesc, (kc | k) != 0 ? 1u : 0u);
        umma_commit(&sm.empty[s]);
      }
      umma_commit(&sm.tfull);   // also after an expired wait: the MMAs issued so far still finish
    }
  }
  __syncwarp();
  {
    int got = 0;
    if (lane == 0) got = mbar_wait(&sm.tfull, 0, timeout_ns, nullptr) ? 1 : 0;
    got = __shfl_sync(0xffffffffu, got, 0);
    if (!got && lane == 0) raise_status(status, PS_DEV_TIMEOUT);
  }
  tc_fence_after();
  __syncthreads();   // the loads have landed (warp 0), the MMAs are done: the ring is idle

  // this rank's partial tile, [row n][128 outputs] f32
  float* part = reinterpret_cast<float*>(sm.ring);
  if (warp >= 2) {
    const int r = (warp & 3) * 32 + lane;
    const uint32_t t_row = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
#pragma unroll 1
    for (int c = 0; c < NT && c < operand_rows; c += 32) {
      uint32_t v[32];
      tmem_ld32(t_row + c, v);
      tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (j < NT - c && c + j < operand_rows) part[(c + j) * 128 + r] = __uint_as_float(v[j]);
    }
  }
  tc_fence_before();
  if (nranks > 1) cluster_sync_all();
  else __syncthreads();

  // rows rank, rank + nranks, ...: the ranks' partials added in rank order
  const uint32_t base = smem_addr(part);
  constexpr int kPer = 32;   // threads of a row: two columns of F each, or four of Y
  for (int i = threadIdx.x; ; i += kFewThreads) {
    const int n = rank + (i / kPer) * nranks, j = i % kPer;
    if (n >= N) break;
    if (UP) {
      float2 g = make_float2(0.f, 0.f), u = g;
      for (int k = 0; k < nranks; ++k) {
        const float2 a = ld_cluster_v2(mapa_shared(base + (n * 128 + 2 * j) * 4, k));
        const float2 b = ld_cluster_v2(mapa_shared(base + (n * 128 + 64 + 2 * j) * 4, k));
        g.x += a.x;
        g.y += a.y;
        u.x += b.x;
        u.y += b.y;
      }
      float q0, q1, s0, s1;
      act_and_slope<ACT>(g.x, q0, s0);
      act_and_slope<ACT>(g.y, q1, s1);
      const int64_t at = static_cast<int64_t>(n) * ldo + row0 + 2 * j;
      const bool in = row0 + 2 * j < C;
      if (in) store_parts(out + at, static_cast<int64_t>(N) * ldo, kept.parts, q0 * u.x, q1 * u.y);
      if (KEEP) {   // a warp has the row's 64 columns, so half of it a slice of 32 (columns past C hold zeros)
        s0 *= u.x;
        s1 *= u.y;
        float mp = fmaxf(finite_size(s0), finite_size(s1)), mq = fmaxf(finite_size(q0), finite_size(q1));
#pragma unroll
        for (int o = 8; o >= 1; o >>= 1) {
          mp = fmaxf(mp, __shfl_xor_sync(0xffffffffu, mp, o));
          mq = fmaxf(mq, __shfl_xor_sync(0xffffffffu, mq, o));
        }
        const uint32_t ep = slice_exponent(mp), eq = slice_exponent(mq);
        const float ip = __uint_as_float((254u - ep) << 23), iq = __uint_as_float((254u - eq) << 23);
        if (in) {
          *reinterpret_cast<uint32_t*>(kept.P + at) = pack_f16x2(s0 * ip, s1 * ip);
          *reinterpret_cast<uint32_t*>(kept.Q + at) = pack_f16x2(q0 * iq, q1 * iq);
          if ((j & 15) == 0) kept.scale[static_cast<int64_t>((row0 + 2 * j) >> 5) * N + n] = ep | eq << 8;
        }
      }
    } else {
      const bool in = row0 + 4 * j < C;
      const int64_t at = static_cast<int64_t>(n) * ldo + row0 + 4 * j;
      uint2 p, q;
      uint32_t scale = 0;
      if (DA && in) {   // (under way beside the partials)
        p = *reinterpret_cast<const uint2*>(kept.P + at);
        q = *reinterpret_cast<const uint2*>(kept.Q + at);
        scale = kept.scale[static_cast<int64_t>((row0 + 4 * j) >> 5) * N + n];
      }
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < nranks; ++k) {
        const float4 a = ld_cluster_v4(mapa_shared(base + (n * 128 + 4 * j) * 4, k));
        y.x += a.x;
        y.y += a.y;
        y.z += a.z;
        y.w += a.w;
        if (OP == kFewDown && kept.parts == 2) {
          const float4 b = ld_cluster_v4(mapa_shared(base + ((N + n) * 128 + 4 * j) * 4, k));
          y.x += b.x;
          y.y += b.y;
          y.z += b.z;
          y.w += b.w;
        }
      }
      if (!in) continue;
      if (DA) {
        auto over = [&](uint16_t* plane, uint2 v, uint32_t exponent) {
          const float factor = __uint_as_float(exponent << 23);
          const float2 a = unpack_f16x2(v.x), b = unpack_f16x2(v.y);
          const int64_t apart = static_cast<int64_t>(N) * ldo;
          store_parts(plane + at, apart, kept.parts, y.x * a.x * factor, y.y * a.y * factor);
          store_parts(plane + at + 2, apart, kept.parts, y.z * b.x * factor, y.w * b.y * factor);
        };
        over(kept.P, p, scale & 255u);
        over(kept.Q, q, scale >> 8 & 255u);
      } else {
        *reinterpret_cast<uint2*>(out + at) = make_uint2(pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
      }
    }
  }
  __syncwarp();
  if (nranks > 1) cluster_sync_all();   // nobody reads this rank's partial any more
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, Cfg::kCols);
  }
}

// ============================================================================= host side
struct FfnStore {
  uint16_t *A, *P, *Q;   // [N][F] each
  uint32_t* scale;       // [ceil(F / 32)][N]: the biased exponents of P (bits 0-7) and Q (8-15)
  size_t bytes;
};
static size_t plane_bytes(int64_t N, int F) { return (static_cast<size_t>(N) * F * 2 + 255) / 256 * 256; }
// Few rows of a narrow block have A, dG and dU in two parts, each of N rows: the bf16 values, and in bf16 what their
// rounding left, which the products that read them add up. An element's error from one part is the same for any N and d
// (2^-8 of a term at most, over K = F terms of Y, 2 F of dX and N of dW); but outputs over few values do not average it
// out: in 2-norm they were up to 1.8 times as far off as their own rounding alone leaves them (d = 100, F = 300; 1.55 at 300,
// 1000; from d = 1000, F = 3000 on 1.41, the two roundings' mean). The rule's edges are what it costs: calls this small are
// launches rather than products. One part / two, forward and backward, us: 8 rows, d = 304, F = 1000 24.7 / 25.5; 16, 600, 2000
// 30.4 / 31.7; 64, 304, 1000 34 / 37; beyond: 32, 1000, 4000 37.8 / 41.8; 1, 3584, 16384 206 / 237. From 65 rows on the general
// kernels have no second plane to write.
constexpr int kPartsRows = 64, kPartsF = 2048;
static int kept_parts(int64_t N, int F) { return N <= kPartsRows && F <= kPartsF ? 2 : 1; }
static FfnStore ffn_store(void* base, int64_t N, int F) {
  const size_t plane = plane_bytes(N * kept_parts(N, F), F);
  uint8_t* b = static_cast<uint8_t*>(base);
  FfnStore f;
  f.A = reinterpret_cast<uint16_t*>(b);
  f.P = reinterpret_cast<uint16_t*>(b + plane);
  f.Q = reinterpret_cast<uint16_t*>(b + 2 * plane);
  f.scale = reinterpret_cast<uint32_t*>(b + 3 * plane);
  f.bytes = 3 * plane + (static_cast<size_t>(N) * ((F + 31) / 32) * 4 + 255) / 256 * 256;
  return f;
}

// Rows of a plane, and the store's bytes, that hold a call of N rows or of any fewer.
static int64_t kept_rows_up_to(int64_t N, int F) {
  const int64_t two = N < kPartsRows ? N : kPartsRows, rows = two * kept_parts(two, F);
  return N > rows ? N : rows;
}
static size_t store_bytes_up_to(int64_t N, int F) {
  return 3 * plane_bytes(kept_rows_up_to(N, F), F) + (static_cast<size_t>(N) * ((F + 31) / 32) * 4 + 255) / 256 * 256;
}

// Blocks of 256 rows walked together: the X (or dY) rows of a band stay in a quarter of L2 while the weights stream by.
static int band_of_rows(int64_t K) {
  const int b = static_cast<int>(30e6 / (2.0 * K * 2 * kBM));
  return b < 1 ? 1 : b;
}
constexpr int kBandRows = 1024;   // products with a long K loop: column tiles of these rows side by side

constexpr int kFewRows = 128;
constexpr int kPlanSms = 152;   // the SMs that sizes and rules go by

// CTAs that share a unit's K loop: as many as keep all units' CTAs resident at once (two per SM), with at least 8
// k blocks each.
static int few_ranks(int64_t units, int num_kb) {
  const int64_t slots = 2 * static_cast<int64_t>(num_sms_current());
  int r = 8;
  while (r > 1 && (units * r > slots || num_kb / r < 8)) r /= 2;
  return r;
}

template <int NT, int OP, int ACT, bool KEEP>
static int launch_few(int64_t N, int C, int64_t K, const void* X, int64_t ldx, const void* W, const void* W2, void* out,
                      int64_t ldo, const FewKept& kept, uint32_t* status, cudaStream_t s) {
  constexpr bool UP = OP == kFewUp;
  CUtensorMap tw, tw2, tx;
  auto map_w = [&](CUtensorMap* m, const void* w) {
    return OP == kFewDa ? map_mnmajor(m, w, K, C, C) : map_kmajor(m, w, C, K, K, UP ? 64 : 128);
  };
  if (!map_w(&tw, W) || !map_w(&tw2, W2) ||
      !map_kmajor(&tx, X, OP == kFewDown ? N * kept.parts : N, K, ldx, NT))
    return PS_ERR_INVALID_ARG;
  auto kern = ffn_few_kernel<NT, OP, ACT, KEEP>;
  constexpr size_t smem = sizeof(FewSmem<NT>) + 1024;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess)
    return PS_ERR_CUDA;
  const int64_t units = (C + (UP ? 63 : 127)) / (UP ? 64 : 128);
  static_assert(kPartsRows * 2 <= kFewRows, "both parts are the operand's rows");
  const int num_kb = static_cast<int>((K + kBK - 1) / kBK);
  int ranks = few_ranks(units, num_kb);
  for (;; ranks /= 2) {
    if (launch_after(kern, dim3(static_cast<unsigned>(units * ranks)), kFewThreads, smem, s, static_cast<unsigned>(ranks),
                     1, true, tw, tw2, tx, static_cast<int>(N), C, num_kb, static_cast<uint16_t*>(out), ldo, kept,
                     status, kDefaultTimeoutNs) == cudaSuccess)
      return PS_OK;
    cudaGetLastError();
    if (ranks == 1) return PS_ERR_CUDA;   // (else the context's SMs do not hold such a cluster)
  }
}
template <int OP, int ACT, bool KEEP>
static int ffn_few(int64_t N, int C, int64_t K, const void* X, int64_t ldx, const void* W, const void* W2, void* out,
                   int64_t ldo, const FewKept& kept, uint32_t* status, cudaStream_t s) {
  const int64_t rows = OP == kFewDown ? N * kept.parts : N;
  if (rows <= 16) return launch_few<16, OP, ACT, KEEP>(N, C, K, X, ldx, W, W2, out, ldo, kept, status, s);
  if (rows <= 32) return launch_few<32, OP, ACT, KEEP>(N, C, K, X, ldx, W, W2, out, ldo, kept, status, s);
  if (OP == kFewDa || rows <= 64) return launch_few<64, OP, ACT, KEEP>(N, C, K, X, ldx, W, W2, out, ldo, kept, status, s);
  if constexpr (OP != kFewDa) return launch_few<128, OP, ACT, KEEP>(N, C, K, X, ldx, W, W2, out, ldo, kept, status, s);
}

// Whether gate and up of these rows go by the kernel for few rows: always up to 64; from there to 128 unless the general
// kernel's CTA pairs come in one round that is enough to stream the weights, or the weights are small. Both products, nothing
// kept, us few / pairs at 65, 96 and 128 rows: d = 3584, F = 16384 68 / 75, 70 / 76, 72 / 78; 3584, 4096 22 / 32, 24 / 33, 27 / 35; 2048,
// 6144 22 / 25, 24 / 26, 27 / 28; 2048, 3000 18 / 23, 19 / 24, 21 / 25; 512, 16384 25 / 31, 26 / 31, 27 / 29; 3000, 9000 45 / 43, 49 / 44,
// 52 / 48; 1536, 8192 22.6 / 24.2, 24.4 / 25.1, 27.2 / 26.1; 1000, 3000 17.4 / 18.7, 18.8 / 19.8, 21.2 / 21.5; 768, 2048 14.9 / 15.5,
// 16.3 / 16.1, 18.4 / 16.9; 392, 1048 15.2 / 15.1, 16.8 / 16.1, 19.2 / 17.5 (kept: 23 / 19 at 128). Where the rule takes the slower one
// it is by 10% at most (1000, 3000 at 65 rows, kept: 18.4 / 20.2).
static bool few_up(int64_t N, int d, int F) {
  const int tiles = (F + 127) / 128;
  return N <= 64 || (N <= kFewRows && (tiles > kPlanSms / 2 || (tiles < kPlanSms / 3 && d >= 1024)));
}

template <int ACT, bool KEEP>
static int ffn_up(int64_t N, int d, int F, const void* X, int64_t ldx, const void* Wg, const void* Wu,
                  const FfnStore& f, uint32_t* status, cudaStream_t s) {
  const FewKept kept = {f.P, f.Q, f.scale, kept_parts(N, F)};
  if (few_up(N, d, F)) return ffn_few<kFewUp, ACT, KEEP>(N, F, d, X, ldx, Wg, Wu, f.A, F, kept, status, s);
  TwoMaps m;
  auto maps = [&](int rows) {
    if (!map_kmajor(&m.a, X, N, d, ldx, rows) || !map_kmajor(&m.b, Wg, F, d, d, kBN / 2) ||
        !map_kmajor(&m.b2, Wu, F, d, d, kBN / 2) || !map_out_16(&m.c, f.A, N, F, F))
      return false;
    m.c2 = m.c3 = m.c;
    return !KEEP || (map_out_16(&m.c2, f.P, N, F, F, CU_TENSOR_MAP_DATA_TYPE_FLOAT16) &&
                     map_out_16(&m.c3, f.Q, N, F, F, CU_TENSOR_MAP_DATA_TYPE_FLOAT16));
  };
  // On CTA pairs the epilogue runs beside the next tile's main loop, and a round over the SMs is half a wide tile. Alone
  // (a store to write, 5 KB a row and 1000 columns) they are the faster throughout; without one a wide tile per SM is 5%
  // faster where the rounds do not decide. Measured, us wide / pairs, kept: 6030 rows, d = 1536, F = 8192 207 / 193; 2000, 2000,
  // 8000 105 / 88; 1200, 3584, 16384 192 / 177; 7835, 3584, 16384 1011 / 1006; not kept: 173 / 173, 94 / 80, 178 / 169, 912 / 965.
  const int64_t tiles = (N + 255) / 256 * ((F + kBN / 2 - 1) / (kBN / 2)), sms = num_sms_current();
  const int64_t wide_rounds = (tiles + sms - 1) / sms, pair_rounds = (2 * tiles + sms - 1) / sms;
  if (!KEEP && wide_rounds * 2000 <= pair_rounds * 1055) {
    if (!maps(2 * kBM)) return PS_ERR_INVALID_ARG;
    using Epi = FfnUpEpi<ACT, false, 2>;
    return launch_gemm_two<false, false, Epi, 2, kTwoB>(m, N, F, d, band_of_rows(d), {static_cast<int>(N), F, f.scale},
                                                        status, s, true);
  }
  if (!maps(kBM)) return PS_ERR_INVALID_ARG;
  return launch_pair_own<false, FfnUpEpi<ACT, KEEP, 4>, kTwoB>(m, N, F, d, band_of_rows(d),
                                                               {static_cast<int>(N), F, f.scale}, status, s, true);
}

// dA = dY Wd and, from the kept P and Q, dG and dU over them. Few rows / CTA pairs, us: 1 row, d = 3584, F = 16384 21.6 / 40; 20,
// 1600, 6400 9.0 / 15.5; 64, 3000, 12000 19 / 23; 64, 1000, 3000 11.7 / 13.1; 100, 3000, 12000 26 / 23; 100, 600, 2000
// 18 / 11; 128, 1536, 8192 15.2 / 15.7 (each row is a turn of the join's loads).
constexpr int kFewDaRows = 64;   // (of the 16, 32 and 64 row kernels)
static int ffn_da(int64_t N, int d, int F, const void* dY, int64_t lddy, const void* Wd, const FfnStore& f,
                  uint32_t* status, cudaStream_t s) {
  const FewKept kept = {f.P, f.Q, f.scale, kept_parts(N, F)};
  if (N <= kFewDaRows) return ffn_few<kFewDa, PS_ACT_SILU, false>(N, F, d, dY, lddy, Wd, Wd, nullptr, F, kept, status, s);
  TwoMaps m;
  if (!map_kmajor(&m.a, dY, N, d, lddy, kBM) || !map_mnmajor(&m.b, Wd, d, F, F) || !map_out_16(&m.c, f.P, N, F, F) ||
      !map_out_16(&m.c2, f.Q, N, F, F))
    return PS_ERR_INVALID_ARG;
  m.b2 = m.b;
  m.c3 = m.c;
  return launch_pair_own<true, FfnDaEpi, kNoPair>(m, N, F, d, band_of_rows(d),
                                                  {static_cast<int>(N), F, f.scale}, status, s, true);
}

// ----------------------------------------------------------------------------- products in one launch
// The products of a group as the caller states them, and how they are cut (the same on every device: what the workspace
// holds depends on it).
struct Product {
  int64_t M, N, K;              // outputs and the K loop (of each operand set)
  bool two_sets;
  bool a_mn, b_mn;
  const void *A, *A2, *B, *B2;
  int64_t lda, ldb;
  void* out;
  int64_t ldo;
  int kind;                     // kOutBf16, kOutF32 or kOutF32Add
  bool fold = false;            // the second half of the M rows is added to the first
};
struct GroupTile {
  int halves, ctas;   // of the kernel
  int rows() const { return kBM * halves * ctas; }
  int workers() const { return kPlanSms / ctas; }
};
struct GroupPlan {
  GroupTile tile;
  int splits[kGroupMost];
  size_t part_off[kGroupMost], bytes;   // the partial tiles' places
};
constexpr int kLeastKb = 12;   // k blocks a share has at least: below that its partial tile costs more than it saves

static int64_t tiles_of(const Product& p, int rows) { return (p.M + rows - 1) / rows * ((p.N + kBN - 1) / kBN); }
static int kb_of(const Product& p) {
  const int64_t kb = (p.K + kBK - 1) / kBK;
  return static_cast<int>(p.two_sets ? 2 * kb : kb);
}
static bool partial(const Product& p, int splits) { return splits > 1 || p.fold; }
// What a unit costs, in hundredths of a 256 x 256 k block's MMAs on one SM (0.55 us): its k blocks at the rate that the tile
// sustains (or at the rate at which an SM gets its share of the weights from HBM, 43 GB/s, where few row blocks read them),
// its outputs at 43 GB/s, and its start and end. Loads and outputs share an SM's port to L2, so they add up.
static double unit_cost(const Product& p, GroupTile t, int splits) {
  double kb_cost = t.halves == 2 ? 100 : t.ctas == 2 ? 62 : 68;
  const double row_blocks = static_cast<double>((p.M + t.rows() - 1) / t.rows());
  const double hbm = kTileBBytes / t.ctas * (t.ctas == 2 && p.M <= kBM ? 5.5e-3 : 4.2e-3) / row_blocks;
  if (!p.a_mn && hbm > kb_cost) kb_cost = hbm;
  const double out = kBM * t.halves * kBN * (partial(p, splits) || p.kind != kOutBf16 ? 4 : 2) * 4.2e-3;
  return kb_cost * kb_of(p) / splits + out + (t.halves == 2 ? 200 : 120);
}

// CTAs (or pairs) with the same load, side by side.
struct LoadSeg {
  int cta0, cta1;
  double load;
};
struct Loads {
  LoadSeg seg[kGroupSegs];
  int n;
};
// n units of one cost dealt to the CTAs so that the highest load is lowest: what fits under the level that they would fill
// if they could be cut anywhere, then one more each for those that it leaves lowest. Splits one segment at most. Returns
// the highest load; out: what each segment takes.
static_assert(kGroupSegs > kGroupMost + 1, "a segment more with each product");
static double deal(Loads& L, int64_t n, double cost, GroupSeg* out, int* out_n) {
  int64_t take[kGroupSegs];
  bool more[kGroupSegs];
  double level = 0;
  for (int i = 0; i < L.n; ++i) more[i] = true;
  for (bool again = true; again;) {   // the level, without the segments that are above it already
    double sum = static_cast<double>(n) * cost, ctas = 0;
    for (int i = 0; i < L.n; ++i)
      if (more[i]) {
        sum += L.seg[i].load * (L.seg[i].cta1 - L.seg[i].cta0);
        ctas += L.seg[i].cta1 - L.seg[i].cta0;
      }
    level = sum / ctas;
    again = false;
    for (int i = 0; i < L.n; ++i)
      if (more[i] && L.seg[i].load > level) {
        more[i] = false;
        again = true;
      }
  }
  int64_t left = n;
  for (int i = 0; i < L.n; ++i) {
    const int len = L.seg[i].cta1 - L.seg[i].cta0;
    take[i] = more[i] ? static_cast<int64_t>((level - L.seg[i].load) / cost) : 0;
    if (take[i] * len > left) take[i] = left / len;   // (rounding)
    left -= take[i] * len;
  }
  while (left > 0) {
    int w = 0;
    for (int i = 1; i < L.n; ++i)
      if (L.seg[i].load + take[i] * cost < L.seg[w].load + take[w] * cost) w = i;
    const int len = L.seg[w].cta1 - L.seg[w].cta0;
    if (left < len) {
      for (int i = L.n; i > w + 1; --i) {
        L.seg[i] = L.seg[i - 1];
        take[i] = take[i - 1];
      }
      L.seg[w + 1] = L.seg[w];
      L.seg[w].cta1 = L.seg[w + 1].cta0 = L.seg[w].cta0 + static_cast<int>(left);
      take[w + 1] = take[w];
      ++L.n;
    }
    ++take[w];
    left -= L.seg[w].cta1 - L.seg[w].cta0;
  }
  double most = 0;
  int64_t unit = 0;
  *out_n = 0;
  for (int i = 0; i < L.n; ++i) {
    const int len = L.seg[i].cta1 - L.seg[i].cta0;
    if (take[i] > 0) {
      out[(*out_n)++] = {L.seg[i].cta0, L.seg[i].cta1, static_cast<int>(take[i]), static_cast<int>(unit)};
      unit += take[i] * len;
      L.seg[i].load += take[i] * cost;
    }
    if (L.seg[i].load > most) most = L.seg[i].load;
  }
  return most;
}

// The tile and each product's shares: a product whose tiles are fewer than the workers (CTAs or pairs) is split into shares of
// what one has to do anyway, or of kLeastKb; the tile is the one whose dealt units end first.
static GroupPlan plan_group(const Product* p, int count) {
  GroupPlan best;
  double best_cost = 0;
  for (const GroupTile tile : {GroupTile{2, 2}, GroupTile{1, 2}, GroupTile{1, 1}}) {
    GroupPlan g;
    g.tile = tile;
    const int workers = tile.workers();
    double work = 0, cost = 0;
    for (int t = 0; t < count; ++t) work += static_cast<double>(tiles_of(p[t], tile.rows())) * unit_cost(p[t], tile, 1);
    const double fair = work / workers * (count > 1 ? 0.66 : 1.0);
    Loads L;
    L.n = 1;
    L.seg[0] = {0, workers, 0.0};
    for (int t = 0; t < count; ++t) {
      const int kb = kb_of(p[t]);
      const int64_t tiles = tiles_of(p[t], tile.rows());
      const double fair_kb = fair / unit_cost(p[t], tile, 1) * kb, share = fair_kb > kLeastKb ? fair_kb : kLeastKb;
      int s = static_cast<int>(kb / share + 0.5);
      if (tiles >= workers) s = 1;
      if (s * tiles > 2 * workers) s = static_cast<int>(2 * workers / tiles);
      g.splits[t] = s < 2 ? 1 : s;
      GroupSeg seg[kGroupSegs];
      int n;
      const double end = deal(L, tiles * g.splits[t], unit_cost(p[t], tile, g.splits[t]), seg, &n);
      if (end > cost) cost = end;
    }
    for (int t = 0; t < count; ++t)
      if (g.splits[t] > 1) cost += 500 + 1.45e-4 * g.splits[t] * p[t].M * p[t].N;   // the shares' way through L2
    if (best_cost == 0 || cost < best_cost) {
      best = g;
      best_cost = cost;
    }
  }
  best.bytes = 0;
  for (int t = 0; t < count; ++t) {
    best.part_off[t] = best.bytes;
    if (!partial(p[t], best.splits[t])) continue;
    const size_t unit = best.tile.rows(), rows = (p[t].M + unit - 1) / unit * unit;
    best.bytes += (best.splits[t] * rows * p[t].N * 4 + 255) / 256 * 256;
  }
  return best;
}

// Bytes that hold the partial tiles of these products or of any some of them, and of as many with fewer rows: a share has
// at least kLeastKb k blocks, and a K loop is cut only into shares of at most two tiles of at most 256 x 256 per SM (or
// 512 x 256 per pair); outputs in two parts (fold) have a plane of every tile also where nothing is cut.
static size_t part_bytes(const Product* p, int count) {
  size_t sum = 0;
  for (int t = 0; t < count; ++t) {
    const size_t shares = static_cast<size_t>(kb_of(p[t])) / kLeastKb + 1;
    if (shares < 2 && !p[t].fold) continue;
    const size_t plane = static_cast<size_t>((p[t].M + 4 * kBM - 1) / (4 * kBM) * (4 * kBM)) * p[t].N * 4;
    const size_t most = static_cast<size_t>(2 * kPlanSms) * 2 * kBM * kBN * 4;
    size_t bytes = shares * plane < most ? shares * plane : most;
    if (p[t].fold && plane > bytes) bytes = plane;
    sum += (bytes + 255) / 256 * 256;
  }
  return sum;
}

template <int HALVES, int CTAS>
static int launch_group(const GroupArgs& g, uint32_t* status, cudaStream_t s) {
  auto kern = umma_group_kernel<HALVES, CTAS>;
  constexpr size_t smem = sizeof(GroupSmem<HALVES, CTAS>) + 1024;
  static_assert(smem <= 232448, "shared memory of one CTA");
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess)
    return PS_ERR_CUDA;
  int workers = 1;
  for (int t = 0; t < g.count; ++t)
    for (int i = 0; i < g.segs[t]; ++i) workers = g.seg[t][i].cta1 > workers ? g.seg[t][i].cta1 : workers;
  if (launch_after(kern, dim3(static_cast<unsigned>(workers * CTAS)), kGroupThreads, smem, s, CTAS, 1, true, g, status,
                   kDefaultTimeoutNs) == cudaSuccess)
    return PS_OK;
  cudaGetLastError();
  return PS_ERR_CUDA;
}

// The products p[0 .. count), cut as `plan` (plan_group's of them) says, its partial tiles at `part`.
static int run_group(const GroupPlan& plan, const Product* p, int count, void* part, uint32_t* status, cudaStream_t s) {
  GroupArgs g;
  SumArgs sums;
  sums.count = 0;
  g.count = count;
  Loads loads;
  loads.n = 1;
  const int rows = plan.tile.rows(), workers = plan.tile.ctas == 2 ? clusters_at_once(0) : num_sms_current();
  if (workers < 1) return PS_ERR_CUDA;
  loads.seg[0] = {0, workers, 0.0};
  for (int t = 0; t < count; ++t) {
    const Product& q = p[t];
    GroupProduct& o = g.p[t];
    o.m_blocks = static_cast<int>((q.M + rows - 1) / rows);
    o.n_blocks = static_cast<int>((q.N + kBN - 1) / kBN);
    o.splits = plan.splits[t];
    o.num_kb = kb_of(q);
    o.first_kb = q.two_sets ? o.num_kb / 2 : o.num_kb;
    o.band_m = kBandRows / rows;
    o.a_mn = q.a_mn;
    o.b_mn = q.b_mn;
    o.cols = static_cast<int>(q.N);
    o.part_rows = o.m_blocks * rows;
    o.out = partial(q, o.splits) ? kOutPartial : q.kind;
    deal(loads, static_cast<int64_t>(o.m_blocks) * o.n_blocks * o.splits, unit_cost(q, plan.tile, o.splits), g.seg[t],
         &g.segs[t]);
    auto map_a = [&](CUtensorMap* m, const void* at) {
      return q.a_mn ? map_mnmajor(m, at, q.K, q.M, q.lda) : map_kmajor(m, at, q.M, q.K, q.lda, kBM * plan.tile.halves);
    };
    auto map_b = [&](CUtensorMap* m, const void* at) {
      return q.b_mn ? map_mnmajor(m, at, q.K, q.N, q.ldb) : map_kmajor(m, at, q.N, q.K, q.ldb, kBN / plan.tile.ctas);
    };
    if (!map_a(&g.a[t], q.A) || !map_b(&g.b[t], q.B)) return PS_ERR_INVALID_ARG;
    if (q.two_sets && (!map_a(&g.a2[t], q.A2) || !map_b(&g.b2[t], q.B2))) return PS_ERR_INVALID_ARG;
    bool ok;
    if (partial(q, o.splits)) {
      float* planes = reinterpret_cast<float*>(static_cast<uint8_t*>(part) + plan.part_off[t]);
      ok = map_out_f32(&g.c[t], planes, static_cast<int64_t>(o.splits) * o.part_rows, q.N, q.N);
      SumItem& it = sums.item[sums.count];
      const int64_t rows_out = q.fold ? q.M / 2 : q.M;
      it = {planes, static_cast<int64_t>(o.part_rows) * q.N, o.splits, static_cast<int>(rows_out), static_cast<int>(q.N / 4),
            q.fold ? static_cast<int>(rows_out) : 0, q.out, q.ldo, q.kind};
      sums.end[sums.count] = rows_out * (q.N / 4) + (sums.count > 0 ? sums.end[sums.count - 1] : 0);
      ++sums.count;
    } else {
      ok = q.kind == kOutBf16 ? map_out_bf16(&g.c[t], q.out, q.M, q.N, q.ldo) : map_out_f32(&g.c[t], q.out, q.M, q.N, q.ldo);
    }
    if (!ok) return PS_ERR_INVALID_ARG;
  }
  const int rc = plan.tile.ctas == 1     ? launch_group<1, 1>(g, status, s)
                 : plan.tile.halves == 1 ? launch_group<1, 2>(g, status, s)
                                         : launch_group<2, 2>(g, status, s);
  if (rc != PS_OK || sums.count == 0) return rc;
  const int64_t blocks = (sums.end[sums.count - 1] + 255) / 256, most = 8 * static_cast<int64_t>(num_sms_current());
  return launch_after(sum_partials_kernel, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), 256, 0, s, 1, 1, true,
                      sums) == cudaSuccess
             ? PS_OK
             : PS_ERR_CUDA;
}

static Product down_product(int64_t N, int d, int F, const void* A, const void* Wd, void* Y, int64_t ldy) {
  return {N, d, F, false, false, false, A, nullptr, Wd, nullptr, F, F, Y, ldy, kOutBf16};
}
// rows that go by the grouped kernel: as `plan` cuts down_product()
static int ffn_down(int64_t N, int d, int F, const void* A, const void* Wd, void* Y, int64_t ldy, const GroupPlan& plan,
                    void* part, uint32_t* status, cudaStream_t s) {
  const FewKept kept = {nullptr, nullptr, nullptr, kept_parts(N, F)};
  if (N <= kFewRows) return ffn_few<kFewDown, PS_ACT_SILU, false>(N, d, F, A, F, Wd, Wd, Y, ldy, kept, status, s);
  const Product p = down_product(N, d, F, A, Wd, Y, ldy);
  return run_group(plan, &p, 1, part, status, s);
}
static size_t down_part_bytes(int64_t N, int d, int F) {
  const Product p = down_product(N, d, F, nullptr, nullptr, nullptr, d);
  return N <= kFewRows ? 0 : part_bytes(&p, 1);
}

// dX = dG Wg + dU Wu, dWg = dG^T X, dWu = dU^T X and dWd = dY^T A, the longest K loop first; those asked for.
static int grad_products(Product* p, int64_t N, int d, int F, const FfnStore& f, const void* dY, int64_t lddy,
                         const void* X, int64_t ldx, const void* Wg, const void* Wu, void* dX, int64_t lddx, int dx_kind,
                         void* dWg, void* dWu, void* dWd, int dw_kind) {
  // the second parts of A, dG and dU: further rows of dX, a second operand set of the others
  const bool two = kept_parts(N, F) == 2;
  auto rest = [&](uint16_t* plane) { return two ? plane + N * F : nullptr; };
  int n = 0;
  if (dX) p[n++] = {two ? 2 * N : N, d, F, true, false, true, f.P, f.Q, Wg, Wu, F, d, dX, lddx, dx_kind, two};
  if (dWg) {
    p[n++] = {F, d, N, two, true, true, f.P, rest(f.P), X, X, F, ldx, dWg, d, dw_kind};
    p[n++] = {F, d, N, two, true, true, f.Q, rest(f.Q), X, X, F, ldx, dWu, d, dw_kind};
  }
  if (dWd) p[n++] = {d, F, N, two, true, true, dY, dY, f.A, rest(f.A), lddy, F, dWd, F, dw_kind};
  return n;
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
  return store_bytes_up_to(N, F);
}

size_t ps_gated_ffn_fwd_workspace_size(int64_t N, int d, int F, int with_store) {
  if (!sizes_ok(N, d, F)) return 0;
  return kWsHeader + (with_store ? 0 : plane_bytes(kept_rows_up_to(N, F), F)) + down_part_bytes(N, d, F);
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
  int rc = check_ws(ws, ws_bytes, ps_gated_ffn_fwd_workspace_size(N, d, F, store != nullptr));
  if (rc != PS_OK) return rc;
  if (N == 0) return refused(PS_OK, ws, s);
  uint32_t* status = static_cast<uint32_t*>(ws);
  FfnStore f = ffn_store(store, N, F);
  uint8_t* scratch = static_cast<uint8_t*>(ws) + kWsHeader;
  size_t left = ws_bytes - kWsHeader;
  if (!store) {
    f.A = reinterpret_cast<uint16_t*>(scratch);
    scratch += plane_bytes(N * kept_parts(N, F), F);
    left -= plane_bytes(N * kept_parts(N, F), F);
  }
  GroupPlan plan = {};
  if (N > kFewRows) {
    const Product p = down_product(N, d, F, f.A, Wd, Y, ldy);
    plan = plan_group(&p, 1);
    if (plan.bytes > left) return refused(PS_ERR_WORKSPACE, ws, s);   // (the size function and the plan are two formulas)
  }
  if (act == PS_ACT_SILU)
    rc = store ? ffn_up<PS_ACT_SILU, true>(N, d, F, X, ldx, Wg, Wu, f, status, s)
               : ffn_up<PS_ACT_SILU, false>(N, d, F, X, ldx, Wg, Wu, f, status, s);
  else
    rc = store ? ffn_up<PS_ACT_GELU, true>(N, d, F, X, ldx, Wg, Wu, f, status, s)
               : ffn_up<PS_ACT_GELU, false>(N, d, F, X, ldx, Wg, Wu, f, status, s);
  if (rc != PS_OK) return refused(rc, ws, s);
  return ffn_down(N, d, F, f.A, Wd, Y, ldy, plan, scratch, status, s);
}

size_t ps_gated_ffn_bwd_workspace_size(int64_t N, int d, int F) {
  if (!sizes_ok(N, d, F)) return 0;
  auto parts = [&](int64_t rows) {
    Product p[kGroupMost];
    void* some = reinterpret_cast<void*>(16);   // (not read)
    const int n = grad_products(p, rows, d, F, ffn_store(nullptr, rows, F), nullptr, d, nullptr, d, nullptr, nullptr, some, d,
                                kOutF32, some, some, some, kOutF32);
    return part_bytes(p, n);
  };
  const size_t all = parts(N), few = parts(N < kPartsRows ? N : kPartsRows);   // (any fewer rows too)
  return kWsHeader + (all > few ? all : few);
}

size_t ps_diag_gated_ffn_partial_bytes(int64_t N, int d, int F, int products, int f32) {
  if (!sizes_ok(N, d, F) || !sizes_fit(N, d, F) || N == 0 || products < 0 || products > 7) return 0;
  void* some = reinterpret_cast<void*>(16);   // (not read)
  Product p[kGroupMost];
  int n = 1;
  if (products == 0) {
    if (N <= kFewRows) return 0;
    p[0] = down_product(N, d, F, nullptr, nullptr, nullptr, d);
  } else {
    void *dX = products & 1 ? some : nullptr, *dWgu = products & 2 ? some : nullptr, *dWd = products & 4 ? some : nullptr;
    const int kind = f32 ? kOutF32 : kOutBf16;
    n = grad_products(p, N, d, F, ffn_store(nullptr, N, F), nullptr, d, nullptr, d, nullptr, nullptr, dX, d, kind, dWgu, dWgu,
                      dWd, kind);
  }
  return plan_group(p, n).bytes;
}

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
  int rc = check_ws(ws, ws_bytes, N == 0 ? kWsHeader : ps_gated_ffn_bwd_workspace_size(N, d, F));
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
  auto kind = [](int dtype, int acc) { return dtype == PS_DTYPE_BF16 ? kOutBf16 : acc ? kOutF32Add : kOutF32; };
  Product p[kGroupMost];
  const int n = grad_products(p, N, d, F, f, dY, lddy, X, ldx, Wg, Wu, dX, lddx, kind(dx_dtype, dx_acc), dWg, dWu, dWd,
                              kind(dw_dtype, dw_acc));
  GroupPlan plan = {};
  if (n > 0) plan = plan_group(p, n);
  if (plan.bytes > ws_bytes - kWsHeader) return refused(PS_ERR_WORKSPACE, ws, s);   // (before the store is consumed)
  rc = ffn_da(N, d, F, dY, lddy, Wd, f, status, s);
  if (rc != PS_OK) return refused(rc, ws, s);
  return n == 0 ? PS_OK : run_group(plan, p, n, static_cast<uint8_t*>(ws) + kWsHeader, status, s);
}

}  // extern "C"
