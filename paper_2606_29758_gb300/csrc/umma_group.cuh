// Several tensor-core products in one persistent launch, their K loops split where there are few tiles (sm_103a).
//
//   D_t[M_t, N_t] = sum_k A_t[m, k] B_t[n, k],  t = 0 .. count - 1;  product 0 may add up two operand sets over its K loop
//
// The kernel of umma_gemm.cuh (tiles, ring, roles, bounded waits), with a unit that is (product, tile, share of the k
// blocks): what a product's layouts are, where its operands lie and how its accumulator is stored is read per unit. So
// products that depend on nothing of each other fill each other's last rounds over the SMs (the host says which CTAs take
// how many units of which product, so that all end together), and a product of few tiles and a long K loop is shared by
// as many CTAs as there are: a share stores its f32 partial tile, and sum_partials_kernel adds the shares in order.
#pragma once

#include "umma_gemm.cuh"

namespace psk {

constexpr int kGroupMost = 4;
enum GroupOut { kOutBf16 = 0, kOutF32 = 1, kOutF32Add = 2, kOutPartial = 3 };

// CTAs [cta0, cta1) take `count` units each of a product, from unit0 on: neighbours side by side, round after round.
struct GroupSeg {
  int cta0, cta1, count, unit0;
};
constexpr int kGroupSegs = 12;

struct GroupProduct {
  int m_blocks, n_blocks, splits, num_kb;
  int first_kb;    // k blocks of the first operand set (product 0; else num_kb)
  int band_m;
  int a_mn, b_mn;  // MN-major operands
  int out, cols;
  int part_rows;   // rows from one share's partial to the next
};
struct GroupArgs {
  CUtensorMap a[kGroupMost], b[kGroupMost], c[kGroupMost], a2, b2;
  GroupProduct p[kGroupMost];
  GroupSeg seg[kGroupMost][kGroupSegs];
  int segs[kGroupMost];
  int count, clear;
};

// This CTA's units, product after product.
struct GroupWalk {
  int t = -1, left = 0, unit = 0, step = 0;
  __device__ __forceinline__ bool next(const GroupArgs& g) {
    if (left > 0) {
      --left;
      unit += step;
      return true;
    }
    while (++t < g.count) {
      const int cta = blockIdx.x;
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
template <int HALVES>
using GroupSmem = GemmSmemT<HALVES, kGroupEpiWarps, 32 * 128>;

template <int HALVES>
__global__ void __launch_bounds__(kGroupThreads, 1)
    umma_group_kernel(const __grid_constant__ GroupArgs g, uint32_t* status, uint64_t timeout_ns) {
  using Cfg = GemmCfg<HALVES>;
  constexpr int S = Cfg::kStagesH;
  constexpr int NB = Cfg::kAccBufs;
  constexpr int CPG = kBN / 32 / (kGroupEpiWarps / 4);   // 32-column chunks per column group
  extern __shared__ uint8_t smem_raw[];
  GroupSmem<HALVES>& sm =
      *reinterpret_cast<GroupSmem<HALVES>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    if (g.clear && blockIdx.x == 0) clear_status(status);   // (a bit is set only after seconds)
    for (int s = 0; s < S; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&sm.tfull[a], 1);
      mbar_init(&sm.tempty[a], 32 * kGroupEpiWarps);
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
    tmem_alloc(&sm.tmem_base, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  wait_for_previous_kernel();
  const uint32_t tmem_base = sm.tmem_base;
  volatile int* abort = &sm.abort;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t kc = 0;
      bool ok = true;
      for (GroupWalk at; ok && at.next(g);) {
        const GroupUnit w = group_unit(g, at);
        const GroupProduct& p = g.p[w.t];
        const int m0 = w.m_blk * Cfg::kRows, n0 = w.n_blk * kBN, first = p.first_kb;
        const bool a_mn = p.a_mn != 0, b_mn = p.b_mn != 0;
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++kc) {
          const int s = kc % S;
          if (!mbar_wait(&sm.empty[s], ((kc / S) & 1u) ^ 1u, timeout_ns, abort)) { ok = false; break; }
          mbar_arrive_expect_tx(&sm.full[s], Cfg::kABytes + kTileBBytes);
          const bool second = kb >= first;
          const CUtensorMap* const ma = second ? &g.a2 : &g.a[w.t];
          const CUtensorMap* const mb = second ? &g.b2 : &g.b[w.t];
          const int k0 = (second ? kb - first : kb) * kBK;
          if (a_mn) {
            for (int i = 0; i < Cfg::kRows / 64; ++i)
              tma_load_2d(sm.a[s] + i * (kBK * 128), ma, &sm.full[s], m0 + i * 64, k0);
          } else {
            tma_load_2d(sm.a[s], ma, &sm.full[s], k0, m0);
          }
          if (b_mn) {
            for (int i = 0; i < kBN / 64; ++i)
              tma_load_2d(sm.b[s] + i * (kBK * 128), mb, &sm.full[s], n0 + i * 64, k0);
          } else {
            tma_load_2d(sm.b[s], mb, &sm.full[s], k0, n0);
          }
        }
      }
      if (!ok) {
        *abort = 1;
        raise_status(status, PS_DEV_TIMEOUT);
        // let the loads already issued land before the CTA can exit
        const uint32_t first = kc > static_cast<uint32_t>(S) ? kc - S : 0;
        for (uint32_t j = first; j < kc; ++j) mbar_wait(&sm.full[j % S], (j / S) & 1u, timeout_ns, nullptr);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t kc = 0, tile = 0;
      bool ok = true;
      for (GroupWalk at; ok && at.next(g); ++tile) {
        const GroupUnit w = group_unit(g, at);
        const bool a_mn = g.p[w.t].a_mn != 0, b_mn = g.p[w.t].b_mn != 0;
        const uint32_t idesc = idesc_bf16_f32(kBM, kBN, a_mn, b_mn);
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
          for (int k = 0; k < kBK / 16; ++k)
            umma_bf16(d_tmem + h * kBN, smem_desc_sw128(a_base + k * a_step, a_lbo, 1024),
                      smem_desc_sw128(b_base + k * b_step, b_lbo, 1024), idesc, (kb | k) != 0 ? 1u : 0u);
        };
        if constexpr (HALVES == 1) {
          for (int kb = 0; kb < num_kb; ++kb, ++kc) {
            const int s = kc % S;
            if (!mbar_wait(&sm.full[s], (kc / S) & 1u, timeout_ns, abort)) { ok = false; break; }
            tc_fence_after();
            issue_half(0, s, kb);
            umma_commit(&sm.empty[s]);
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
              umma_commit(&sm.empty[s]);
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
              umma_commit(&sm.empty[sj]);
            }
          }
        }
        if (ok) umma_commit(&sm.tfull[acc]);
      }
      if (!ok) {
        *abort = 1;
        raise_status(status, PS_DEV_TIMEOUT);
        umma_commit(&sm.drain);
        mbar_wait(&sm.drain, 0, timeout_ns, nullptr);
      }
    }
  } else {
    const int quad = warp & 3, ew = warp - 2, grp = ew >> 2;
    uint8_t* const stage = sm.stage[ew];
    uint32_t tile = 0, stored = 0;
    int out = -1;
    bool ok = true;
    for (GroupWalk at; at.next(g); ++tile) {
      const GroupUnit w = group_unit(g, at);
      const GroupProduct& p = g.p[w.t];
      const CUtensorMap* const map = &g.c[w.t];
      const int cols = p.cols;
      if (p.out != out) {   // (another kind of slice: the buffer is free again first)
        if (lane == 0) bulk_wait_group_read<0>();
        __syncwarp();
        out = p.out;
      }
      const int row0 = w.m_blk * Cfg::kRows + quad * 32 + (out == kOutPartial ? w.split * p.part_rows : 0);
      const uint32_t acc = tile % NB, aph = (tile / NB) & 1u;
      int got = 0;
      if (lane == 0) got = mbar_wait(&sm.tfull[acc], aph, timeout_ns, abort) ? 1 : 0;
      got = __shfl_sync(0xffffffffu, got, 0);
      if (!got) { ok = false; break; }
      tc_fence_after();
      // a 32 x 32 slice (this lane's row: r) into the staging buffer, then one lane stores the warp's box
      auto slice = [&](const uint32_t (&r)[32], int col0, int row) {
        if (col0 >= cols) return;
        // 2-byte slices take turns in the two halves of the buffer (the store before the last one has read its half)
        uint8_t* const buf = out == kOutBf16 ? stage + (stored++ & 1u) * (32 * 64) : stage;
        if (lane == 0) {
          if (out == kOutBf16) bulk_wait_group_read<1>();
          else bulk_wait_group_read<0>();
        }
        __syncwarp();
        if (out == kOutBf16) {
          uint4* dst = reinterpret_cast<uint4*>(buf + lane * 64);
          auto two = [&](int j) { return pack_bf16x2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])); };
#pragma unroll
          for (int q = 0; q < 4; ++q)
            dst[q ^ ((lane >> 1) & 3)] = make_uint4(two(8 * q), two(8 * q + 2), two(8 * q + 4), two(8 * q + 6));
        } else {
          uint4* dst = reinterpret_cast<uint4*>(buf + lane * 128);
#pragma unroll
          for (int q = 0; q < 8; ++q)
            dst[q ^ (lane & 7)] = make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (out == kOutF32Add) tma_reduce_add_2d(map, buf, col0, row);
          else tma_store_2d(map, buf, col0, row);
          bulk_commit_group();
        }
      };
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + (acc + h) * kBN;
        const int col0 = w.n_blk * kBN + grp * CPG * 32;
        if constexpr (HALVES == 2) {
          // the warp's share of the half into registers, so that the MMA warp has it back before it is staged
          uint32_t r[CPG][32];
#pragma unroll
          for (int c = 0; c < CPG; ++c) tmem_ld32(t_row + (grp * CPG + c) * 32, r[c]);
          tmem_ld_wait();
          tc_fence_before();
          mbar_arrive(&sm.tempty[h]);
#pragma unroll
          for (int c = 0; c < CPG; ++c) slice(r[c], col0 + c * 32, row0 + h * kBM);
        } else {
#pragma unroll 1
          for (int c = 0; c < CPG; ++c) {
            uint32_t r[32];
            tmem_ld32(t_row + (grp * CPG + c) * 32, r);
            tmem_ld_wait();
            if (c == CPG - 1) {
              tc_fence_before();
              mbar_arrive(&sm.tempty[acc]);
            }
            slice(r, col0 + c * 32, row0);
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
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kTmemCols);
  }
}

// ----------------------------------------------------------------------------- joining the shares of split products
struct SumItem {
  const float* part;     // [splits][part_rows][cols] f32
  int64_t plane;         // part_rows * cols
  int splits, rows, quads;   // quads of columns a row
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
