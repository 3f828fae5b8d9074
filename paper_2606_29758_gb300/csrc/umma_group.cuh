// Several tensor-core products in one persistent launch, their K loops split where there are few tiles (sm_103a).
//
//   D_t[M_t, N_t] = sum_k A_t[m, k] B_t[n, k],  t = 0 .. count - 1;  a product may add up two operand sets over its K loop
//
// The kernel of umma_gemm.cuh (tiles, ring, roles, bounded waits), with a unit that is (product, tile, share of the k
// blocks): what a product's layouts are, where its operands lie and how its accumulator is stored is read per unit. So
// products that depend on nothing of each other fill each other's last rounds over the SMs (the host says which CTAs take
// how many units of which product, so that all end together), and a product of few tiles and a long K loop is shared by
// as many CTAs as there are: a share stores its f32 partial tile, and sum_partials_kernel adds the shares in order.
//
// CTAS = 2: a unit is a CTA pair's (cta_group::2): each CTA has 128 HALVES rows of A and half of the B tile, so that a k block
// of a 512 x 256 tile is 48 KB of loads per SM for 1024 cycles of MMAs. (A 256 x 256 tile on one SM is 64 KB, which is
// what an SM's port to L2 carries in that time, and the outputs come on top.) A backward's four products on 256 x 256 tiles of
// one SM / on pairs, us: 6030 rows, d = 1536, F = 8192 428 / 405; 2000, 2000, 8000 188 / 174; 400, 3000, 12000 151 / 138. Pairs
// of HALVES = 1, whose accumulators alternate, fill the SMs better with few tiles; single CTAs are for up to 128 rows of dX.
#pragma once

#include "umma_gemm.cuh"

namespace psk {

constexpr int kGroupMost = 4;
enum GroupOut { kOutBf16 = 0, kOutF32 = 1, kOutF32Add = 2, kOutPartial = 3 };

// CTAs (or pairs) [cta0, cta1) take `count` units each of a product, from unit0 on: neighbours side by side, round after round.
struct GroupSeg {
  int cta0, cta1, count, unit0;
};
constexpr int kGroupSegs = 12;

struct GroupProduct {
  int m_blocks, n_blocks, splits, num_kb;
  int first_kb;    // k blocks of the first operand set (num_kb without a second)
  int band_m;
  int a_mn, b_mn;  // MN-major operands
  int out, cols;
  int part_rows;   // rows from one share's partial to the next
};
struct GroupArgs {
  CUtensorMap a[kGroupMost], b[kGroupMost], c[kGroupMost], a2[kGroupMost], b2[kGroupMost];
  GroupProduct p[kGroupMost];
  GroupSeg seg[kGroupMost][kGroupSegs];
  int segs[kGroupMost];
  int count;
};

// This CTA's units, product after product.
struct GroupWalk {
  int t = -1, left = 0, unit = 0, step = 0;
  __device__ __forceinline__ bool next(const GroupArgs& g, int cta) {
    if (left > 0) {
      --left;
      unit += step;
      return true;
    }
    while (++t < g.count) {
      for (int i = 0; i < g.segs[t]; ++i) {
        const GroupSeg& s = g.seg[t][i];
        if (cta < s.cta0 || cta >= s.cta1 || s.count == 0) continue;
        left = s.count - 1;
        step = s.cta1 - s.cta0;
        unit = s.unit0 + cta - s.cta0;
        return true;
      }
    }
    return false;
  }
};
struct GroupUnit {
  int t, m_blk, n_blk, split, kb0, kb1;
};
static __device__ __forceinline__ GroupUnit group_unit(const GroupArgs& g, const GroupWalk& at) {
  GroupUnit r;
  r.t = at.t;
  const GroupProduct& p = g.p[r.t];
  int i = at.unit;
  const int tiles = p.m_blocks * p.n_blocks;
  r.split = i / tiles;
  i -= r.split * tiles;
  const int per_band = p.band_m * p.n_blocks;
  const int band = i / per_band;
  i -= band * per_band;
  const int m_first = band * p.band_m, this_band = min(p.band_m, p.m_blocks - m_first);
  r.n_blk = i / this_band;
  r.m_blk = m_first + (i - r.n_blk * this_band);
  r.kb0 = static_cast<int>(static_cast<long long>(p.num_kb) * r.split / p.splits);
  r.kb1 = static_cast<int>(static_cast<long long>(p.num_kb) * (r.split + 1) / p.splits);
  return r;
}

constexpr int kGroupEpiWarps = 8;
constexpr int kGroupThreads = 64 + 32 * kGroupEpiWarps;
template <int HALVES, int CTAS>
struct GroupCfg {
  static constexpr int kRows = kBM * HALVES * CTAS;   // rows of a tile
  static constexpr uint32_t kABytes = kTileABytes * HALVES, kBBytes = kTileBBytes / CTAS;   // of a CTA's stage
  static constexpr int kStages = 192 * 1024 / (kABytes + kBBytes);
  static constexpr int kAccBufs = HALVES == 1 ? 2 : 1;
};
template <int HALVES, int CTAS>
struct GroupSmem {
  using Cfg = GroupCfg<HALVES, CTAS>;
  uint8_t a[Cfg::kStages][Cfg::kABytes];
  uint8_t b[Cfg::kStages][Cfg::kBBytes];
  uint8_t stage[kGroupEpiWarps][32 * 128];
  uint64_t full[Cfg::kStages];    // (of the pair's even CTA: loads and arrivals of both)
  uint64_t empty[Cfg::kStages];
  uint64_t tfull[2];
  uint64_t tempty[2];             // (the even CTA's: the epilogue warps of both)
  uint64_t drain;
  uint32_t tmem_base;
  int abort;
};

template <int HALVES, int CTAS>
__global__ void __launch_bounds__(kGroupThreads, 1)
    umma_group_kernel(const __grid_constant__ GroupArgs g, uint32_t* status, uint64_t timeout_ns) {
  using Cfg = GroupCfg<HALVES, CTAS>;
  using Smem = GroupSmem<HALVES, CTAS>;
  constexpr int S = Cfg::kStages;
  constexpr int NB = Cfg::kAccBufs;
  constexpr int CPG = kBN / 32 / (kGroupEpiWarps / 4);   // 32-column chunks per column group
  constexpr bool PAIR = CTAS == 2;
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? static_cast<int>(cluster_ctarank()) : 0;
  const int worker = blockIdx.x / CTAS;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&sm.full[s], CTAS);
      mbar_init(&sm.empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&sm.tfull[a], 1);
      mbar_init(&sm.tempty[a], CTAS * kGroupEpiWarps);
    }
    mbar_init(&sm.drain, 1);
    sm.abort = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane < g.count) {
    tma_prefetch_desc(&g.a[lane]);
    tma_prefetch_desc(&g.b[lane]);
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      tmem_alloc_pair(&sm.tmem_base, kTmemCols);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(&sm.tmem_base, kTmemCols);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  if constexpr (PAIR) cluster_sync_all();   // barriers of both CTAs initialised before any remote arrival
  else __syncthreads();
  tc_fence_after();
  wait_for_previous_kernel();
  let_next_kernel_in();
  const uint32_t tmem_base = sm.tmem_base;
  volatile int* abort = &sm.abort;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t kc = 0;
      bool ok = true;
      for (GroupWalk at; ok && at.next(g, worker);) {
        const GroupUnit w = group_unit(g, at);
        const GroupProduct& p = g.p[w.t];
        const int m0 = w.m_blk * Cfg::kRows + rank * (kBM * HALVES), n0 = w.n_blk * kBN + rank * (kBN / CTAS);
        const int first = p.first_kb;
        const bool a_mn = p.a_mn != 0, b_mn = p.b_mn != 0;
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++kc) {
          const int s = kc % S;
          if (!mbar_wait(&sm.empty[s], ((kc / S) & 1u) ^ 1u, timeout_ns, abort)) { ok = false; break; }
          const uint32_t full = PAIR ? mapa_shared(smem_addr(&sm.full[s]), 0) : 0;
          if constexpr (PAIR) mbar_arrive_expect_tx_cluster(full, Cfg::kABytes + Cfg::kBBytes);
          else mbar_arrive_expect_tx(&sm.full[s], Cfg::kABytes + Cfg::kBBytes);
          auto load = [&](void* to, const CUtensorMap* map, int c0, int c1) {
            if constexpr (PAIR) tma_load_2d_pair(to, map, full, c0, c1);
            else tma_load_2d(to, map, &sm.full[s], c0, c1);
          };
          const bool second = kb >= first;
          const CUtensorMap* const ma = second ? &g.a2[w.t] : &g.a[w.t];
          const CUtensorMap* const mb = second ? &g.b2[w.t] : &g.b[w.t];
          const int k0 = (second ? kb - first : kb) * kBK;
          if (a_mn) {
            for (int i = 0; i < 2 * HALVES; ++i) load(sm.a[s] + i * (kBK * 128), ma, m0 + i * 64, k0);
          } else {
            load(sm.a[s], ma, k0, m0);
          }
          if (b_mn) {
            for (int i = 0; i < kBN / CTAS / 64; ++i) load(sm.b[s] + i * (kBK * 128), mb, n0 + i * 64, k0);
          } else {
            load(sm.b[s], mb, k0, n0);
          }
        }
      }
      if (!ok) {
        *abort = 1;
        raise_status(status, PS_DEV_TIMEOUT);
        // the loads already issued land before the CTA can exit: the even CTA can see that; the odd one, whose loads count
        // on the other's barriers, gives them a bounded time
        if (rank == 0) {
          const uint32_t first = kc > static_cast<uint32_t>(S) ? kc - S : 0;
          for (uint32_t j = first; j < kc; ++j) mbar_wait(&sm.full[j % S], (j / S) & 1u, timeout_ns, nullptr);
        } else {
          const uint64_t t0 = globaltimer_ns();
          while (globaltimer_ns() - t0 < 2000000ull) {
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      auto commit = [&](uint64_t* bar) {
        if constexpr (PAIR) umma_commit_pair_multicast(bar, 0x3);
        else umma_commit(bar);
      };
      uint32_t kc = 0, tile = 0;
      bool ok = true;
      for (GroupWalk at; ok && at.next(g, worker); ++tile) {
        const GroupUnit w = group_unit(g, at);
        const bool a_mn = g.p[w.t].a_mn != 0, b_mn = g.p[w.t].b_mn != 0;
        const uint32_t idesc = idesc_bf16_f32(kBM * CTAS, kBN, a_mn, b_mn);
        const uint32_t a_lbo = a_mn ? kBK * 128 : 16, a_step = a_mn ? 2048 : 32;
        const uint32_t b_lbo = b_mn ? kBK * 128 : 16, b_step = b_mn ? 2048 : 32;
        const uint32_t acc = tile % NB, aph = (tile / NB) & 1u;
        if (!mbar_wait(&sm.tempty[acc], aph ^ 1u, timeout_ns, abort)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + acc * kBN;   // NB = 1: halves at columns 0 and 256
        const int num_kb = w.kb1 - w.kb0;
        auto issue_half = [&](int h, int s, int kb) {
          const uint32_t a_base = smem_addr(sm.a[s]) + h * kTileABytes, b_base = smem_addr(sm.b[s]);
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k) {
            const uint64_t ad = smem_desc_sw128(a_base + k * a_step, a_lbo, 1024);
            const uint64_t bd = smem_desc_sw128(b_base + k * b_step, b_lbo, 1024);
            if constexpr (PAIR) umma_bf16_pair(d_tmem + h * kBN, ad, bd, idesc, (kb | k) != 0 ? 1u : 0u);
            else umma_bf16(d_tmem + h * kBN, ad, bd, idesc, (kb | k) != 0 ? 1u : 0u);
          }
        };
        if constexpr (HALVES == 1) {
          for (int kb = 0; kb < num_kb; ++kb, ++kc) {
            const int s = kc % S;
            if (!mbar_wait(&sm.full[s], (kc / S) & 1u, timeout_ns, abort)) { ok = false; break; }
            tc_fence_after();
            issue_half(0, s, kb);
            commit(&sm.empty[s]);
          }
        } else {
          // the halves are handed back one after the other; see umma_gemm.cuh
          bool h1_free = false;
          const uint32_t kc0 = kc;
          for (int kb = 0; kb < num_kb; ++kb, ++kc) {
            const int s = kc % S;
            if (!mbar_wait(&sm.full[s], (kc / S) & 1u, timeout_ns, abort)) { ok = false; break; }
            tc_fence_after();
            issue_half(0, s, kb);
            if (h1_free) {
              issue_half(1, s, kb);
              commit(&sm.empty[s]);
              continue;
            }
            if (!mbar_try_wait(&sm.tempty[1], aph ^ 1u)) {
              if (kb + 1 < S && kb + 1 < num_kb) continue;
              if (!mbar_wait(&sm.tempty[1], aph ^ 1u, timeout_ns, abort)) { ok = false; break; }
            }
            h1_free = true;
            tc_fence_after();
            for (int j = 0; j <= kb; ++j) {
              const int sj = (kc0 + j) % S;
              issue_half(1, sj, j);
              commit(&sm.empty[sj]);
            }
          }
        }
        if (ok) commit(&sm.tfull[acc]);
      }
      if (!ok) {
        *abort = 1;
        raise_status(status, PS_DEV_TIMEOUT);
        if constexpr (PAIR) umma_commit_pair_multicast(&sm.drain, 0x1);
        else umma_commit(&sm.drain);
        mbar_wait(&sm.drain, 0, timeout_ns, nullptr);
      }
    }
  } else {
    const int quad = warp & 3, ew = warp - 2, grp = ew >> 2;
    uint8_t* const stage = sm.stage[ew];
    uint4* const own = reinterpret_cast<uint4*>(stage + lane * 128);   // this lane's row of the staged slice
    uint32_t tile = 0;
    bool ok = true;
    auto hand_back = [&](int a) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (PAIR) mbar_arrive_cluster(mapa_shared(smem_addr(&sm.tempty[a]), 0));
        else mbar_arrive(&sm.tempty[a]);
      }
    };
    for (GroupWalk at; at.next(g, worker); ++tile) {
      const GroupUnit w = group_unit(g, at);
      const GroupProduct& p = g.p[w.t];
      const CUtensorMap* const map = &g.c[w.t];
      const int cols = p.cols, out = p.out;
      const int row0 = w.m_blk * Cfg::kRows + rank * (kBM * HALVES) + quad * 32 + (out == kOutPartial ? w.split * p.part_rows : 0);
      const int col0 = w.n_blk * kBN + grp * CPG * 32;
      const uint32_t acc = tile % NB, aph = (tile / NB) & 1u;
      int got = 0;
      if (lane == 0) got = mbar_wait(&sm.tfull[acc], aph, timeout_ns, abort) ? 1 : 0;
      got = __shfl_sync(0xffffffffu, got, 0);
      if (!got) { ok = false; break; }
      tc_fence_after();
      const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + acc * kBN + grp * CPG * 32;
      // 32 rows of 128 bytes through the staging buffer; one lane stores the box
      auto staged = [&](int col, int row, auto&& quarter) {
        if (col >= cols) return;
        if (lane == 0) bulk_wait_group_read<0>();
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 8; ++q) own[q ^ (lane & 7)] = quarter(q);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (out == kOutF32Add) tma_reduce_add_2d(map, stage, col, row);
          else tma_store_2d(map, stage, col, row);
          bulk_commit_group();
        }
      };
      auto pack = [](const uint32_t (&r)[32], uint32_t* pk) {
#pragma unroll
        for (int j = 0; j < 16; ++j) pk[j] = pack_bf16x2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
      };
      auto store_bf16 = [&](const uint32_t (&pk)[32], int col, int row) {   // 64 columns
        staged(col, row, [&](int q) { return make_uint4(pk[4 * q], pk[4 * q + 1], pk[4 * q + 2], pk[4 * q + 3]); });
      };
      auto store_f32 = [&](const uint32_t (&r)[32], int col, int row) {
        staged(col, row, [&](int q) { return make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]); });
      };
      if constexpr (HALVES == 2) {
        if (out == kOutBf16) {
          // The warp's share of both halves into registers, so that the MMA warp has them back before the stores are waited
          // for; the first slice goes to the staging buffer before the second half is read (for the registers).
          uint32_t pk[2][CPG / 2][32];
          auto read_half = [&](int h) {
#pragma unroll
            for (int c = 0; c < CPG; ++c) {
              uint32_t r[32];
              tmem_ld32(t_row + h * kBN + c * 32, r);
              tmem_ld_wait();
              pack(r, pk[h][c / 2] + (c % 2) * 16);
            }
            hand_back(h);
          };
          read_half(0);
          store_bf16(pk[0][0], col0, row0);
          read_half(1);
          store_bf16(pk[0][1], col0 + 64, row0);
          store_bf16(pk[1][0], col0, row0 + kBM);
          store_bf16(pk[1][1], col0 + 64, row0 + kBM);
          static_assert(CPG == 4, "two slices of 64 columns a half");
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[CPG][32];
#pragma unroll
            for (int c = 0; c < CPG; ++c) tmem_ld32(t_row + h * kBN + c * 32, r[c]);
            tmem_ld_wait();
            hand_back(h);
#pragma unroll
            for (int c = 0; c < CPG; ++c) store_f32(r[c], col0 + c * 32, row0 + h * kBM);
          }
        }
      } else {
#pragma unroll 1
        for (int c = 0; c < CPG; c += 2) {
          uint32_t r[2][32];
          tmem_ld32(t_row + c * 32, r[0]);
          tmem_ld32(t_row + c * 32 + 32, r[1]);
          tmem_ld_wait();
          if (c == CPG - 2) hand_back(acc);
          if (out == kOutBf16) {
            uint32_t pk[32];
            pack(r[0], pk);
            pack(r[1], pk + 16);
            store_bf16(pk, col0 + c * 32, row0);
          } else {
            store_f32(r[0], col0 + c * 32, row0);
            store_f32(r[1], col0 + c * 32 + 32, row0);
          }
        }
      }
    }
    if (!ok) {
      *abort = 1;
      raise_status(status, PS_DEV_TIMEOUT);
    }
    if (lane == 0) bulk_wait_group_all();
  }

  tc_fence_before();
  __syncwarp();
  if constexpr (PAIR) cluster_sync_all();   // no remote arrival or multicast commit can target an exited CTA
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    if constexpr (PAIR) tmem_dealloc_pair(tmem_base, kTmemCols);
    else tmem_dealloc(tmem_base, kTmemCols);
  }
}

// ----------------------------------------------------------------------------- joining the shares of split products
struct SumItem {
  const float* part;     // [splits][part_rows][cols] f32
  int64_t plane;         // part_rows * cols
  int splits, rows, quads;   // quads of columns a row
  int fold;              // rows whose outputs come in two parts: the second so many rows further down (0: in one)
  void* out;
  int64_t ld;
  int kind;              // kOutBf16, kOutF32 or kOutF32Add
};
struct SumArgs {
  SumItem item[kGroupMost];
  int64_t end[kGroupMost];   // quads up to and with each item
  int count;
};
static __global__ void __launch_bounds__(256) sum_partials_kernel(const __grid_constant__ SumArgs a) {
  wait_for_previous_kernel();
  let_next_kernel_in();
  const int64_t all = a.end[a.count - 1];
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * 256) {
    int t = 0;
    while (i >= a.end[t]) ++t;
    const SumItem& it = a.item[t];
    const int64_t j = i - (t > 0 ? a.end[t - 1] : 0);
    const int row = static_cast<int>(j / it.quads), col = static_cast<int>(j - static_cast<int64_t>(row) * it.quads) * 4;
    const float* p = it.part + static_cast<int64_t>(row) * it.quads * 4 + col;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int k = 0; k < it.splits; ++k, p += it.plane) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
      if (it.fold > 0) {
        const float4 u = __ldcg(reinterpret_cast<const float4*>(p + static_cast<int64_t>(it.fold) * it.quads * 4));
        s.x += u.x;
        s.y += u.y;
        s.z += u.z;
        s.w += u.w;
      }
    }
    const int64_t at = static_cast<int64_t>(row) * it.ld + col;
    if (it.kind == kOutBf16) {
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(it.out) + at) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
    } else {
      float4* o = reinterpret_cast<float4*>(static_cast<float*>(it.out) + at);
      if (it.kind == kOutF32Add) {
        const float4 v = *o;
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
      }
      *o = s;
    }
  }
}

}  // namespace psk
