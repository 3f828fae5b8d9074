// Row-wise operators of a policy block over packed rows: norms of queries and keys per head with the rotary
// positions in the same pass (forward and backward), the rotation's table, and dropout of a branch's rows added to the
// residual rows, from a counter-based generator.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <climits>

#include "internal.h"
#include "ps_common.cuh"
#include "ps_nvtx.h"

namespace psk {

// ================================================================== elements
struct Bf16 {
  uint16_t v;
};
template <class T>
struct Elem;
template <>
struct Elem<Bf16> {
  static __device__ __forceinline__ float get(Bf16 x) { return __uint_as_float(static_cast<uint32_t>(x.v) << 16); }
  static __device__ __forceinline__ Bf16 put(float x) {
    return Bf16{static_cast<uint16_t>(pack_bf16x2(x, 0.f) & 0xffffu)};
  }
};
template <>
struct Elem<float> {
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};

// Eight consecutive elements at a 16-byte boundary, as they are loaded and as floats.
template <class T>
struct Raw8;
template <>
struct Raw8<Bf16> {
  uint4 v;
  __device__ __forceinline__ void load(const Bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float* f) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(Bf16* p, const float* f) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                              pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
    f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float* f) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// Two f32 in one register pair: an instruction for both.
struct F2 {
  unsigned long long v;
};
static __device__ __forceinline__ F2 pair2(float x, float y) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(x), "f"(y));
  return r;
}
static __device__ __forceinline__ void split2(F2 a, float& x, float& y) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(a.v));
}
static __device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
static __device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// The 16 values of a lane as eight pairs to be turned together: a[j] holds the first members of pairs 2 j and 2 j + 1, b[j]
// the second ones. Half: the pairs are (lo[i], hi[i]) of the lane's two runs of eight; even: (v[2 i], v[2 i + 1]).
template <bool EVEN>
static __device__ __forceinline__ void to_pairs(const Raw8<Bf16>& lo, const Raw8<Bf16>& hi, F2 (&a)[4], F2 (&b)[4]) {
  const uint32_t l[4] = {lo.v.x, lo.v.y, lo.v.z, lo.v.w}, h[4] = {hi.v.x, hi.v.y, hi.v.z, hi.v.w};
  auto low = [](uint32_t w) { return __uint_as_float(w << 16); };
  auto high = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (EVEN) {
      const uint32_t w0 = j < 2 ? l[2 * j] : h[2 * j - 4], w1 = j < 2 ? l[2 * j + 1] : h[2 * j - 3];
      a[j] = pair2(low(w0), low(w1));
      b[j] = pair2(high(w0), high(w1));
    } else {
      a[j] = pair2(low(l[j]), high(l[j]));
      b[j] = pair2(low(h[j]), high(h[j]));
    }
  }
}
template <bool EVEN>
static __device__ __forceinline__ void to_pairs(const Raw8<float>& lo, const Raw8<float>& hi, F2 (&a)[4], F2 (&b)[4]) {
  const float l[8] = {lo.a.x, lo.a.y, lo.a.z, lo.a.w, lo.b.x, lo.b.y, lo.b.z, lo.b.w};
  const float h[8] = {hi.a.x, hi.a.y, hi.a.z, hi.a.w, hi.b.x, hi.b.y, hi.b.z, hi.b.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (EVEN) {
      const float* v = j < 2 ? l + 4 * j : h + 4 * j - 8;
      a[j] = pair2(v[0], v[2]);
      b[j] = pair2(v[1], v[3]);
    } else {
      a[j] = pair2(l[2 * j], l[2 * j + 1]);
      b[j] = pair2(h[2 * j], h[2 * j + 1]);
    }
  }
}
template <bool EVEN, class T>
static __device__ __forceinline__ void store_pairs(T* lo, T* hi, const F2 (&a)[4], const F2 (&b)[4]) {
  float u[8], v[8], l[8], h[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    split2(a[j], u[2 * j], u[2 * j + 1]);
    split2(b[j], v[2 * j], v[2 * j + 1]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    l[i] = EVEN ? (i & 1 ? v[i / 2] : u[i / 2]) : u[i];
    h[i] = EVEN ? (i & 1 ? v[4 + i / 2] : u[4 + i / 2]) : v[i];
  }
  Raw8<T>::store(lo, l);
  Raw8<T>::store(hi, h);
}

// ================================================================== q/k norms and rotation
//   n = x r g, r = (mean x^2 + eps)^(-1/2) over a head's D values; y = rotation(position) of n's first R dims.
//   backward: dn = rotation^T dy, dg = sum dn x r, dx = r (g dn - x r^2 mean(g dn x)).
// HBM-bound (a read and a write of every element; the backward two reads and a write); short rows by the issue slots. A head
// lies on G lanes, 16 values each: eight pairs, so a lane rotates by itself and only the mean crosses lanes (log2 G
// shuffles). A warp takes 32 / G heads of one row at a time, keys after queries, and keeps its lanes' cosines and sines for
// the row and their gains for the side; the arithmetic is on pairs of f32 (two to an instruction). The heads come through a
// ring in shared memory of the warp's own, filled by its lanes' copies some steps ahead. us forward / backward, before from
// bulk copies (bf16, from 4 steps a row on) or registers a step ahead: bf16, 106k rows of 28 + 4 heads of 128 270 / 421 (6.4 and
// 6.2 TB/s; 282 / 452); 20k of 40 + 8 of 256, half of it rotated, 169 / 240 (182 / 237); 100k of 6 + 2 of 96, half rotated, 96 / 148
// (100 / 153), of 64 57 / 86 (68 / 103); 4000 of 28 + 4 18 / 31; f32, 50k of 28 + 4 253 / 366 (259 / 380), 100k of 6 + 2 of 64
// 78 / 124 (93 / 146).
constexpr int kQkThreads = 128;
constexpr int kQkWarps = kQkThreads / 32;
template <class T, bool BWD>
struct QkCfg {
  static constexpr int kArrays = BWD ? 2 : 1;                      // x, and dy
  static constexpr int kStages = sizeof(T) == 2 ? 4 : BWD ? 2 : 3;
  static constexpr int kSlot = 512 * sizeof(T);                    // a step's heads: at most 32 lanes of 16 values
  static constexpr int kWarp = kStages * kArrays * kSlot;          // a warp's ring, in the end its gain gradients [2][D]
  static constexpr int kBlocks = BWD ? 3 : 4;                      // per SM
  // Of long rows fewer at once, which HBM prefers. 3 / 2, us: f32, 50k rows of 28 + 4 heads of 128 285 / 253 (backward
  // 418 / 366), of 16 + 16 of 64 (8 KB) 144 / 138, of 12 + 2 of 128 (7 KB) 115 / 135; 4 / 3: bf16, 20k of 40 + 8 of 256
  // 178 / 160, 106k of 28 + 4 of 128 (8 KB) 270 / 300.
  static int blocks_of(int64_t row_bytes) {
    if (sizeof(T) == 4 && row_bytes >= 8 * 1024) return 2;
    return !BWD && sizeof(T) == 2 && row_bytes >= 16 * 1024 ? 3 : kBlocks;
  }
};
static_assert(QkCfg<uint16_t, true>::kWarp >= 2 * 512 * 4, "a warp's gain gradients lie over its ring");
// The status is cleared by a memset before the launch, as any block may set it early; of fewer rows the first block looks at
// every position and sets the word alone (a token's call takes one launch, 6.3 -> 4 us on the device).
constexpr int kQkCheckRows = 2048;

// 16 bytes global -> shared.
static __device__ __forceinline__ void lane_copy(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

struct QkArgs {
  int64_t N;
  int Hq, Hk, D, R, G;          // G: lanes per head, a power of two, at least D / 16
  int parts;                    // warps that share a row's heads
  const void *q, *k;            // rows of [heads][D], pitches in elements
  int64_t ldq, ldk;
  const void *gq, *gk;          // [D] gains, or nullptr: 1
  float eps;
  const int32_t* pos;
  int pos_base, T;
  const float2* table;          // [T][R / 2] (cos, sin)
  void *qo, *ko;                // forward: the outputs; backward: dq, dk
  int64_t ldqo, ldko;
  const void *dqy, *dky;        // backward: gradients of the forward's outputs
  int64_t lddqy, lddky;
  float* part;                  // backward: [blocks][2][D] partial gain gradients, nullptr without
  float *dgq, *dgk;             // their sums, or nullptr
  int accumulate;
  uint32_t* status;
};

static __device__ __forceinline__ float group_sum(float v, int G) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1)
    if (G > o) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ALL: every dim is rotated (R = D). Else the lanes of the others take their values as they are: by a cosine of 1 and a sine of
// 0 an infinity would reach the value beside it as 0 inf. (The selects cost 3-5% of many bf16 rows, 28 + 4 heads of 128, 64 of
// them rotated, 106k rows: 283 / 448 us instead of 270 / 432; a branch of the lanes 9% and every call.)
template <class T, bool EVEN, bool BWD, bool ALL>
__global__ void __launch_bounds__(kQkThreads, (QkCfg<T, BWD>::kBlocks)) qk_kernel(const QkArgs a) {
  using Cfg = QkCfg<T, BWD>;
  constexpr int ST = Cfg::kStages;
  extern __shared__ __align__(128) uint8_t qk_smem[];   // the warps' rings, gains [2][D]
  __shared__ float4 other[BWD ? kQkWarps : 1][4][32];   // gain gradients of the side that is not at work
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint8_t* const ring = qk_smem + warp * Cfg::kWarp;
  float* const all_gains = reinterpret_cast<float*>(qk_smem + kQkWarps * Cfg::kWarp);
  for (int i = threadIdx.x; i < 2 * a.D; i += kQkThreads) {
    const void* g = i < a.D ? a.gq : a.gk;
    all_gains[i] = g ? Elem<T>::get(static_cast<const T*>(g)[i < a.D ? i : i - a.D]) : 1.f;
  }
  if (BWD)
#pragma unroll
    for (int i = 0; i < 4; ++i) other[warp][i][lane] = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();

  const int c = lane & (a.G - 1), slot = lane / a.G, at_once = 32 / a.G;
  const bool here = 16 * c < a.D, rotated = 16 * c < a.R;
  const int lo = EVEN || !rotated ? 16 * c : 8 * c;
  const int hi = EVEN || !rotated ? 16 * c + 8 : a.R / 2 + 8 * c;
  const int apart = hi - lo, in_step = slot * a.D + lo;
  const int heads = a.Hq + a.Hk, steps = (heads + at_once - 1) / at_once;   // keys follow queries within a step
  const float inv_d = 1.f / static_cast<float>(a.D);

  // This warp's units: a row's steps, or a part of them.
  const int64_t units = a.N * a.parts, stride = static_cast<int64_t>(gridDim.x) * kQkWarps;
  auto row_of = [&](int64_t u) { return a.parts == 1 ? u : u / a.parts; };
  struct Run {
    int64_t u, row;
    int s, s1;        // steps of the unit still to come
  };
  auto open = [&](Run& r) {   // the next unit
    r.u += stride;
    if (r.u >= units) return;
    r.row = row_of(r.u);
    r.s = 0;
    r.s1 = steps;
    if (a.parts > 1) {   // (the divisions are a quarter of what a short row takes)
      const int part = static_cast<int>(r.u - r.row * a.parts);
      r.s = steps * part / a.parts;
      r.s1 = steps * (part + 1) / a.parts;
    }
  };
  // The copies of the next step's heads into stage st: P pieces of 16 bytes a lane, counted through the row's heads (queries,
  // then keys). A group of copies for each step, be it empty.
  constexpr int P = Cfg::kSlot / 512, E = 16 / sizeof(T);
  const int step_elems = at_once * a.D, row_elems = heads * a.D, first_k = a.Hq * a.D;
  const T *xq, *xk, *yq, *yk;   // the row's queries, and its keys less the queries' elements, at this lane's first piece
  auto sources = [&](const Run& r) {
    auto at = [&](const void* base, int64_t ld, int before) {
      return static_cast<const T*>(base) + (r.row * ld + lane * E - before);
    };
    xq = at(a.q, a.ldq, 0);
    xk = at(a.k, a.ldk, first_k);
    if (BWD) {
      yq = at(a.dqy, a.lddqy, 0);
      yk = at(a.dky, a.lddky, first_k);
    }
  };
  auto issue = [&](Run& r, int st) {
    if (r.u < units) {
      const uint32_t to = smem_addr(ring) + st * Cfg::kArrays * Cfg::kSlot + lane * 16;
      const int e0 = r.s * step_elems, end = min(e0 + step_elems, row_elems) - lane * E;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int e = e0 + i * 32 * E;
        if (e >= end) continue;
        const bool k = e + lane * E >= first_k;
        lane_copy(to + i * 512, (k ? xk : xq) + e);
        if (BWD) lane_copy(to + Cfg::kSlot + i * 512, (k ? yk : yq) + e);
      }
      if (++r.s >= r.s1) {
        open(r);
        if (r.u < units) sources(r);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // the table's row of unit u's position; the position is known a unit earlier
  auto position = [&](int64_t u) { return a.R > 0 && u < units ? __ldg(a.pos + row_of(u)) : 0; };
  auto in_table = [&](int pos) {
    const int64_t t = static_cast<int64_t>(pos) - a.pos_base;
    return t >= 0 && t < a.T;
  };

  Run t, n;
  t.u = static_cast<int64_t>(blockIdx.x) * kQkWarps + warp - stride;
  open(t);
  n = t;
  if (n.u < units) sources(n);
  int pos = position(t.u), pos_next = position(t.u + stride);
#pragma unroll
  for (int s = 0; s < ST; ++s) issue(n, s);
  const F2 zero2 = pair2(0.f, 0.f), one2 = pair2(1.f, 1.f), minus2 = pair2(-1.f, -1.f);
  F2 cs[4], sn[4], ga[4], gb[4];          // the row's cosines and sines; the side's gains
  F2 acca[4], accb[4];                    // backward: the side's gain gradients
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    cs[j] = one2;
    sn[j] = zero2;
    if (BWD) acca[j] = accb[j] = zero2;
  }
  auto load_gains = [&](bool keys) {
    const float* g = all_gains + (keys ? a.D : 0) + (here ? lo : 0);
    Raw8<float> l, h;
    l.load(g);
    h.load(g + apart);
    to_pairs<EVEN>(l, h, ga, gb);
  };
  bool keys = false;                      // the side that this lane's gains and gradients are of
  load_gains(false);
  auto turn_to = [&](bool side) {
    keys = side;
    load_gains(side);
    if (BWD)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 v = other[warp][j][lane];
        float4 w;
        split2(acca[j], w.x, w.y);
        split2(accb[j], w.z, w.w);
        other[warp][j][lane] = w;
        acca[j] = pair2(v.x, v.y);
        accb[j] = pair2(v.z, v.w);
      }
  };
  int st = 0;
  if (a.N <= kQkCheckRows && blockIdx.x == 0) {   // (the loads above are under way)
    int bad = 0;
    if (a.R > 0)
      for (int i = threadIdx.x; i < a.N; i += kQkThreads) bad |= !in_table(__ldg(a.pos + i));
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
      clear_status(a.status);
      if (bad) raise_status(a.status, PS_DEV_BAD_LENGTH);
    }
  }
  for (; t.u < units; open(t)) {
    if (a.R > 0) {
      const bool good = in_table(pos);
      if (!good && a.N > kQkCheckRows) raise_status(a.status, PS_DEV_BAD_LENGTH);
      if (rotated) {
        const int64_t row = good ? static_cast<int64_t>(pos) - a.pos_base : 0;
        const float4* at = reinterpret_cast<const float4*>(a.table + row * (a.R / 2) + 8 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float4 v = __ldg(at + i);
          if (!good) v.x = v.y = v.z = v.w = __int_as_float(0x7fffffff);   // outside the table: NaN
          cs[i] = pair2(v.x, v.z);
          sn[i] = pair2(v.y, v.w);
        }
      }
      pos = pos_next;
      pos_next = position(t.u + 2 * stride);
    }
    for (; t.s < t.s1; ++t.s) {
      const int head = t.s * at_once + slot;
      const bool mine = here && head < heads, side = min(head, heads - 1) >= a.Hq;   // (without a head: a side that the row has)
      if (side != keys) turn_to(side);
      asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
      __syncwarp();   // every lane's copies of the step
      F2 xa[4], xb[4], ya[4], yb[4];
      Raw8<T> va, vb, wa, wb;
      if (mine) {
        const T* from = reinterpret_cast<const T*>(ring + st * Cfg::kArrays * Cfg::kSlot) + in_step;
        va.load(from);
        vb.load(from + apart);
        if (BWD) {
          wa.load(from + 512);
          wb.load(from + 512 + apart);
        }
      } else {
        va.zero(), vb.zero();
        if (BWD) wa.zero(), wb.zero();
      }
      to_pairs<EVEN>(va, vb, xa, xb);
      if (BWD) to_pairs<EVEN>(wa, wb, ya, yb);
      __syncwarp();   // the stage has been read
      issue(n, st);
      st = st + 1 == ST ? 0 : st + 1;
      F2 sq = zero2;
#pragma unroll
      for (int j = 0; j < 4; ++j) sq = fma2(xb[j], xb[j], fma2(xa[j], xa[j], sq));
      float s0, s1;
      split2(sq, s0, s1);
      float sum = s0 + s1;
      if (!BWD) {
        sum = group_sum(sum, a.G);
        const float r = mine ? rsqrtf(fmaf(sum, inv_d, a.eps)) : 0.f;
        const F2 r2 = pair2(r, r);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const F2 na = mul2(mul2(xa[j], r2), ga[j]), nb = mul2(mul2(xb[j], r2), gb[j]);
          const F2 ta = fma2(minus2, mul2(nb, sn[j]), mul2(na, cs[j])), tb = fma2(na, sn[j], mul2(nb, cs[j]));
          ya[j] = ALL || rotated ? ta : na;
          yb[j] = ALL || rotated ? tb : nb;
        }
      } else {
        // With n = x r: dg += dn n, dx = r (g dn - n mean(g dn n)). bf16: the two sums over the head go side by side, the
        // second over x instead of n (106k rows of 28 + 4 heads of 128 463 us, one after the other 476); f32, whose loads
        // ahead take the registers that this needs, would be slower by 6%.
        constexpr bool kBoth = sizeof(T) == 2;
        auto inverse = [&]() { return mine ? rsqrtf(fmaf(sum, inv_d, a.eps)) : 0.f; };   // (no head here: gains get nothing)
        float r = 0.f;
        if (!kBoth) {
          sum = group_sum(sum, a.G);
          r = inverse();
        }
        F2 r2 = pair2(r, r), dot = zero2;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const F2 ta = fma2(yb[j], sn[j], mul2(ya[j], cs[j])), tb = fma2(minus2, mul2(ya[j], sn[j]), mul2(yb[j], cs[j]));
          const F2 da = ALL || rotated ? ta : ya[j], db = ALL || rotated ? tb : yb[j];
          if (kBoth) {
            ya[j] = da;
            yb[j] = db;
            dot = fma2(mul2(db, gb[j]), xb[j], fma2(mul2(da, ga[j]), xa[j], dot));
          } else {
            xa[j] = mul2(xa[j], r2);
            xb[j] = mul2(xb[j], r2);
            acca[j] = fma2(da, xa[j], acca[j]);
            accb[j] = fma2(db, xb[j], accb[j]);
            ya[j] = mul2(da, ga[j]);
            yb[j] = mul2(db, gb[j]);
            dot = fma2(yb[j], xb[j], fma2(ya[j], xa[j], dot));
          }
        }
        split2(dot, s0, s1);
        float m = s0 + s1;
        if (kBoth) {
#pragma unroll
          for (int o = 16; o >= 1; o >>= 1)
            if (a.G > o) {
              sum += __shfl_xor_sync(0xffffffffu, sum, o);
              m += __shfl_xor_sync(0xffffffffu, m, o);
            }
          r = inverse();
          r2 = pair2(r, r);
          m *= r;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            xa[j] = mul2(xa[j], r2);
            xb[j] = mul2(xb[j], r2);
            acca[j] = fma2(ya[j], xa[j], acca[j]);
            accb[j] = fma2(yb[j], xb[j], accb[j]);
            ya[j] = mul2(ya[j], ga[j]);
            yb[j] = mul2(yb[j], gb[j]);
          }
        } else {
          m = group_sum(m, a.G);
        }
        m *= -inv_d;
        const F2 m2 = pair2(m, m);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          ya[j] = mul2(r2, fma2(xa[j], m2, ya[j]));
          yb[j] = mul2(r2, fma2(xb[j], m2, yb[j]));
        }
      }
      if (mine) {
        T* out = static_cast<T*>(keys ? a.ko : a.qo) + t.row * (keys ? a.ldko : a.ldqo) +
                 static_cast<int64_t>(keys ? head - a.Hq : head) * a.D + lo;
        store_pairs<EVEN>(out, out + apart, ya, yb);
      }
    }
  }
  if (!BWD || a.part == nullptr) return;
  if (keys) turn_to(false);
  __syncwarp();

  // gain gradients: over the warp's heads, then the block's warps; qk_gain_sum_kernel adds the blocks'
  float* mineq = reinterpret_cast<float*>(ring);   // (every copy into it has been waited for)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float v[4], w[4];   // this side's a and b of two pairs, the other side's
    split2(acca[j], v[0], v[1]);
    split2(accb[j], v[2], v[3]);
    const float4 o = other[warp][j][lane];
    w[0] = o.x, w[1] = o.y, w[2] = o.z, w[3] = o.w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      for (int d = 16; d >= a.G; d >>= 1) {
        v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
        w[i] += __shfl_xor_sync(0xffffffffu, w[i], d);
      }
      if (here && slot == 0) {
        const int p = 2 * j + (i & 1);   // the pair
        const int at = EVEN ? lo + 2 * p + (i >> 1) : (i < 2 ? lo : hi) + p;
        mineq[at] = keys ? w[i] : v[i];
        mineq[a.D + at] = keys ? v[i] : w[i];
      }
    }
  }
  __syncthreads();
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.D;
  for (int i = threadIdx.x; i < 2 * a.D; i += kQkThreads) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kQkWarps; ++w) t += reinterpret_cast<const float*>(qk_smem + w * Cfg::kWarp)[i];
    part[i] = t;
  }
}

// The blocks' partial gain gradients [blocks][2][D], eight columns a block: a thread adds every 32nd block's, the shares are
// added in order, all in f64, so that reruns give the same bits. (The last block to finish did it before, alone: 456
// blocks of 256 columns took it 40 us.)
__global__ void __launch_bounds__(256) qk_gain_sum_kernel(int D, int blocks, const float* __restrict__ part, float* dgq,
                                                          float* dgk, int accumulate) {
  __shared__ double sums[32][8];
  wait_for_previous_kernel();
  const int j = threadIdx.x & 7, share = threadIdx.x >> 3, col = blockIdx.x * 8 + j;
  double t = 0.0;
#pragma unroll 8
  for (int b = share; b < blocks; b += 32) t += static_cast<double>(part[static_cast<int64_t>(b) * 2 * D + col]);
  sums[share][j] = t;
  __syncthreads();
  if (share != 0) return;
  t = 0.0;
  for (int k = 0; k < 32; ++k) t += sums[k][j];
  float* out = col < D ? dgq : dgk;
  if (!out) return;
  float& o = out[col < D ? col : col - D];
  o = static_cast<float>(accumulate ? t + o : t);
}

// cos and sin of t theta^(-2 i / R), in double and rounded once.
__global__ void rope_table_kernel(int T, int R, double theta, float2* table) {
  const int64_t n = static_cast<int64_t>(T) * (R / 2);
  for (int64_t j = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; j < n;
       j += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t t = j / (R / 2);
    const int i = static_cast<int>(j - t * (R / 2));
    double s, c;
    sincos(static_cast<double>(t) * pow(theta, -2.0 * i / R), &s, &c);
    table[j] = make_float2(static_cast<float>(c), static_cast<float>(s));
  }
}

// ================================================================== dropout
// Philox4x32-10 (Salmon et al., SC'11): 128 bits for eight columns of a row, 16 each.
static __device__ __forceinline__ uint4 philox4x32_10(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    uint32_t hi0, lo0, hi1, lo1;
    asm("{\n\t.reg .b64 p;\n\tmul.wide.u32 p, %2, %3;\n\tmov.b64 {%0, %1}, p;\n\t}" : "=r"(lo0), "=r"(hi0) : "r"(c.x), "r"(0xD2511F53u));
    asm("{\n\t.reg .b64 p;\n\tmul.wide.u32 p, %2, %3;\n\tmov.b64 {%0, %1}, p;\n\t}" : "=r"(lo1), "=r"(hi1) : "r"(c.z), "r"(0xCD9E8D57u));
    c = make_uint4(hi1 ^ c.y ^ k0, lo1, hi0 ^ c.w ^ k1, lo0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

struct DropArgs {
  int64_t N;
  int d, blocks;              // blocks of eight columns
  int G, parts;               // lanes per row (a power of two), warps that share a row
  const void *x, *res;
  void* y;
  int64_t ldx, ldr, ldy;
  const int32_t *traj, *pos;
  uint32_t traj_base, step, site, k0, k1, cut;
  float scale;
};

// The four words of a row's block b of eight columns; column 8 b + j is kept where the low (even j) or high half of word
// j / 2 is at least the cut. Halves are compared in the upper 16 bits of a word: cut is K 2^16, and what lies below the
// half does not change the comparison.
static __device__ __forceinline__ uint4 draw8(const DropArgs& a, uint32_t traj, uint32_t pos, int b) {
  return philox4x32_10(make_uint4((a.site << 16) + static_cast<uint32_t>(b), pos, traj, a.step), a.k0, a.k1);
}
static __device__ __forceinline__ bool kept(const uint4& w, int j, uint32_t cut) {
  const uint32_t v = j < 2 ? w.x : j < 4 ? w.y : j < 6 ? w.z : w.w;
  return ((j & 1) ? v : v << 16) >= cut;
}

static __device__ __forceinline__ uint32_t kept8(const DropArgs& a, uint32_t traj, uint32_t pos, int b) {
  const uint4 w = draw8(a, traj, pos, b);
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m |= kept(w, j, a.cut) ? 1u << j : 0u;
  return m;
}

// HBM-bound next to about a dozen integer operations an element.
//   kWhole    rows of whole blocks at 16-byte boundaries: a lane's eight columns in 16-byte accesses, two blocks under way
//   kShifted  rows that start anywhere, but x, res and y alike: a lane takes the eight columns at a 16-byte boundary, which
//             lie in two blocks; the mask of the other one comes from its neighbour (from the round before for the first
//             lane), and only a row's two ends go element by element
//   kAnyhow   otherwise: the lanes load G neighbouring elements of a row at a time, all of a round before its first is
//             used, and get each one's bit from the lane that drew it
enum DropRows { kWhole = 0, kShifted = 1, kAnyhow = 2 };
constexpr int kDropThreads = 256;

template <class T, bool RES, int ROWS>
__global__ void __launch_bounds__(kDropThreads, sizeof(T) == 4 || ROWS != kWhole ? 3 : 4) dropout_kernel(const DropArgs a) {
  const int lane = threadIdx.x & 31, c = lane & (a.G - 1), slot = lane / a.G, rows = 32 / a.G;
  const int64_t row_units = (a.N + rows - 1) / rows, units = row_units * a.parts;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * (kDropThreads / 32);
  wait_for_previous_kernel();   // (calls of one step follow each other: 6330 rows of 771 f32, both ways 20.8 us, 21.8 without)
  let_next_kernel_in();
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kDropThreads / 32) + (threadIdx.x >> 5); u < units; u += stride) {
    const int64_t ru = a.parts == 1 ? u : u / a.parts;
    const int part = static_cast<int>(u - ru * a.parts);
    const int64_t row = ru * rows + slot;
    const bool live = row < a.N;
    const uint32_t traj = live ? static_cast<uint32_t>(__ldg(a.traj + row)) + a.traj_base : 0u;
    const uint32_t pos = live ? static_cast<uint32_t>(__ldg(a.pos + row)) : 0u;
    const T* xs = static_cast<const T*>(a.x) + row * a.ldx;
    const T* rs = static_cast<const T*>(a.res) + (RES ? row * a.ldr : 0);
    T* ys = static_cast<T*>(a.y) + row * a.ldy;
    // this warp's share of the row's blocks, in whole rounds of G
    const int rounds = (a.blocks + a.G - 1) / a.G;
    const int t0 = static_cast<int>(static_cast<int64_t>(rounds) * part / a.parts);
    const int t1 = static_cast<int>(static_cast<int64_t>(rounds) * (part + 1) / a.parts);
    if (ROWS == kWhole) {
      for (int t = t0; t < t1; t += 2) {
        Raw8<T> rx[2], rr[2];
        bool in[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int b = (t + h) * a.G + c;
          in[h] = live && t + h < t1 && b < a.blocks;
          rx[h].zero();
          if (RES) rr[h].zero();
          if (!in[h]) continue;
          rx[h].load(xs + 8 * b);
          if (RES) rr[h].load(rs + 8 * b);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int b = (t + h) * a.G + c;
          const uint4 w = draw8(a, traj, pos, b);
          float x[8], y[8];
          rx[h].get(x);
          if (RES) rr[h].get(y);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float base = RES ? y[j] : 0.f;
            y[j] = kept(w, j, a.cut) ? fmaf(x[j], a.scale, base) : base;
          }
          if (in[h]) Raw8<T>::store(ys + 8 * b, y);
        }
      }
    } else if (ROWS == kShifted) {
      const int off = static_cast<int>((reinterpret_cast<uintptr_t>(xs) & 15) / sizeof(T));
      // the mask of the block before this share's first (there is none before column 0)
      uint32_t carry = t0 > 0 ? kept8(a, traj, pos, t0 * a.G - 1) : 0u;
      for (int t = t0; t < t1; t += 2) {
        Raw8<T> rx[2], rr[2];
        int c0[2];
        bool all[2], some[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          c0[h] = 8 * ((t + h) * a.G + c) - off;
          some[h] = live && t + h < t1 && c0[h] < a.d;
          all[h] = some[h] && c0[h] >= 0 && c0[h] + 8 <= a.d;
          rx[h].zero();
          if (RES) rr[h].zero();
          if (!all[h]) continue;
          rx[h].load(xs + c0[h]);
          if (RES) rr[h].load(rs + c0[h]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t m = kept8(a, traj, pos, (t + h) * a.G + c);
          const uint32_t before = __shfl_sync(0xffffffffu, m, slot * a.G + ((c + a.G - 1) & (a.G - 1)));
          const uint32_t k = ((c == 0 ? carry : before) | m << 8) >> (8 - off);   // bit j: column c0 + j
          carry = before;
          if (all[h]) {
            float x[8], y[8];
            rx[h].get(x);
            if (RES) rr[h].get(y);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float base = RES ? y[j] : 0.f;
              y[j] = (k >> j & 1u) ? fmaf(x[j], a.scale, base) : base;
            }
            Raw8<T>::store(ys + c0[h], y);
          } else if (some[h]) {
            for (int j = 0; j < 8; ++j) {
              const int col = c0[h] + j;
              if (col < 0 || col >= a.d) continue;
              const float base = RES ? Elem<T>::get(rs[col]) : 0.f;
              ys[col] = Elem<T>::put((k >> j & 1u) ? fmaf(Elem<T>::get(xs[col]), a.scale, base) : base);
            }
          }
        }
      }
    } else {
      for (int t = t0; t < t1; ++t) {
        const int b0 = t * a.G;
        float x[8], y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int col = b0 * 8 + j * a.G + c;
          const bool in = live && col < a.d;
          x[j] = in ? Elem<T>::get(xs[col]) : 0.f;
          y[j] = RES && in ? Elem<T>::get(rs[col]) : 0.f;
        }
        const uint32_t m = kept8(a, traj, pos, b0 + c);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int in_round = j * a.G + c, col = b0 * 8 + in_round;
          const uint32_t mm = __shfl_sync(0xffffffffu, m, slot * a.G + (in_round >> 3));
          if (live && col < a.d) ys[col] = Elem<T>::put((mm >> (in_round & 7) & 1u) ? fmaf(x[j], a.scale, y[j]) : y[j]);
        }
      }
    }
  }
}

// ================================================================== host side
static bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
static int elem_bytes(int dtype) { return dtype == PS_DTYPE_BF16 ? 2 : 4; }
static int lanes_for(int chunks) {
  int g = 1;
  while (g < chunks && g < 32) g *= 2;
  return g;
}
// Warps that share a row so that about `want` are at work, at most `steps`.
static int parts_for(int64_t rows, int64_t want, int steps) {
  if (rows >= want || rows < 1) return 1;
  const int64_t p = want / rows;
  return static_cast<int>(p < steps ? p : steps);
}
constexpr int64_t kQkMaxBlocks = 760;   // at most; the backward's workspace holds a partial sum of each

// A row of heads: its pitch, base and the rows' last element stay within what the kernel addresses.
static bool rows_ok(const void* p, int64_t ld, int64_t cols, int dtype) {
  return al16(p) && ld >= cols && ld * elem_bytes(dtype) % 16 == 0;
}
static bool qk_sizes_ok(int64_t N, int Hq, int Hk, int D, int R, int dtype, int layout) {
  if (N < 0 || Hq < 0 || Hk < 0 || Hq > 65536 || Hk > 65536 || D < 16 || D > 512 || D % 16 || R < 0 || R > D || R % 16)
    return false;
  return (dtype == PS_DTYPE_BF16 || dtype == PS_DTYPE_F32) && (layout == PS_ROPE_HALF || layout == PS_ROPE_EVEN);
}

template <class T, bool BWD, bool ALL>
static int launch_qk(const QkArgs& a, int layout, cudaStream_t s) {
  using Cfg = QkCfg<T, BWD>;
  // resident blocks take their units in turn
  const int64_t want = (a.N * a.parts + kQkWarps - 1) / kQkWarps;
  int64_t most = static_cast<int64_t>(num_sms_current()) *
                 Cfg::blocks_of(static_cast<int64_t>(a.Hq + a.Hk) * a.D * static_cast<int64_t>(sizeof(T)));
  if (most > kQkMaxBlocks) most = kQkMaxBlocks;
  const unsigned grid = static_cast<unsigned>(want < most ? want : most);
  const size_t smem = kQkWarps * Cfg::kWarp + 2 * sizeof(float) * a.D;
  auto kern = layout == PS_ROPE_EVEN ? qk_kernel<T, true, BWD, ALL> : qk_kernel<T, false, BWD, ALL>;
  if (smem > 32 * 1024 &&
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess)
    return refused(PS_ERR_CUDA, a.status, s);
  if (a.N > kQkCheckRows && cudaMemsetAsync(a.status, 0, kWsHeader, s) != cudaSuccess) return PS_ERR_CUDA;
  kern<<<grid, kQkThreads, smem, s>>>(a);
  if (cudaGetLastError() != cudaSuccess) return refused(PS_ERR_CUDA, a.status, s);
  if (!a.part) return PS_OK;
  return launch_after(qk_gain_sum_kernel, dim3(static_cast<unsigned>(2 * a.D / 8)), 256, 0, s, 1, 1, true, a.D,
                      static_cast<int>(grid), a.part, a.dgq, a.dgk, a.accumulate) == cudaSuccess
             ? PS_OK
             : PS_ERR_CUDA;
}
template <bool BWD>
static int run_qk(QkArgs a, int dtype, int layout, cudaStream_t s) {
  a.G = lanes_for(a.D / 16);
  const int at_once = 32 / a.G;
  a.parts = parts_for(a.N, static_cast<int64_t>(num_sms_current()) * 2 * kQkWarps, (a.Hq + a.Hk + at_once - 1) / at_once);
  if (a.R == a.D)
    return dtype == PS_DTYPE_F32 ? launch_qk<float, BWD, true>(a, layout, s) : launch_qk<Bf16, BWD, true>(a, layout, s);
  return dtype == PS_DTYPE_F32 ? launch_qk<float, BWD, false>(a, layout, s) : launch_qk<Bf16, BWD, false>(a, layout, s);
}

}  // namespace psk

using namespace psk;

extern "C" {

int ps_rope_table(int T, int R, double theta, float* table, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_rope_table");
  if (T < 1 || R < 16 || R > 512 || R % 16 || !(theta > 0.0) || isinf(theta) || !table || !al16(table))
    return PS_ERR_INVALID_ARG;
  rope_table_kernel<<<num_sms_current() * 4, 256, 0, reinterpret_cast<cudaStream_t>(stream)>>>(
      T, R, theta, reinterpret_cast<float2*>(table));
  return cudaGetLastError() == cudaSuccess ? PS_OK : PS_ERR_CUDA;
}

size_t ps_qk_norm_rope_workspace_size(int D) {
  if (D < 16 || D > 512 || D % 16) return 0;
  return kWsHeader + static_cast<size_t>(kQkMaxBlocks) * 2 * D * sizeof(float);
}

int ps_qk_norm_rope_fwd(int64_t N, int Hq, int Hk, int D, int R, int dtype, int layout, const void* q, int64_t ldq,
                        const void* k, int64_t ldk, const void* gq, const void* gk, double eps, const int32_t* pos,
                        int pos_base, int T, const float* table, void* q_out, int64_t ldqo, void* k_out, int64_t ldko,
                        void* ws, size_t ws_bytes, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_qk_norm_rope_fwd");
  if (!qk_sizes_ok(N, Hq, Hk, D, R, dtype, layout) || !(eps >= 0.0)) return PS_ERR_INVALID_ARG;
  if (N > 0 && R > 0 && (!pos || !table || T < 1 || !al16(table))) return PS_ERR_INVALID_ARG;
  if (N > 0 && Hq > 0 && (!q || !q_out || !rows_ok(q, ldq, static_cast<int64_t>(Hq) * D, dtype) ||
                          !rows_ok(q_out, ldqo, static_cast<int64_t>(Hq) * D, dtype)))
    return PS_ERR_INVALID_ARG;
  if (N > 0 && Hk > 0 && (!k || !k_out || !rows_ok(k, ldk, static_cast<int64_t>(Hk) * D, dtype) ||
                          !rows_ok(k_out, ldko, static_cast<int64_t>(Hk) * D, dtype)))
    return PS_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int rc = check_ws(ws, ws_bytes, kWsHeader);
  if (rc != PS_OK) return rc;
  if (N == 0 || Hq + Hk == 0) return refused(PS_OK, ws, s);
  QkArgs a = {};
  a.N = N, a.Hq = Hq, a.Hk = Hk, a.D = D, a.R = R;
  a.q = q, a.k = k, a.ldq = ldq, a.ldk = ldk, a.gq = gq, a.gk = gk, a.eps = static_cast<float>(eps);
  a.pos = pos, a.pos_base = pos_base, a.T = T, a.table = reinterpret_cast<const float2*>(table);
  a.qo = q_out, a.ko = k_out, a.ldqo = ldqo, a.ldko = ldko;
  a.status = static_cast<uint32_t*>(ws);
  return run_qk<false>(a, dtype, layout, s);
}

int ps_qk_norm_rope_bwd(int64_t N, int Hq, int Hk, int D, int R, int dtype, int layout, const void* dq_out,
                        int64_t lddqo, const void* dk_out, int64_t lddko, const void* q, int64_t ldq, const void* k,
                        int64_t ldk, const void* gq, const void* gk, double eps, const int32_t* pos, int pos_base,
                        int T, const float* table, void* dq, int64_t lddq, void* dk, int64_t lddk, float* dgq,
                        float* dgk, int flags, void* ws, size_t ws_bytes, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_qk_norm_rope_bwd");
  if (!qk_sizes_ok(N, Hq, Hk, D, R, dtype, layout) || !(eps >= 0.0) || (flags & ~PS_DW_ACCUMULATE))
    return PS_ERR_INVALID_ARG;
  if (N > 0 && R > 0 && (!pos || !table || T < 1 || !al16(table))) return PS_ERR_INVALID_ARG;
  const int64_t wq = static_cast<int64_t>(Hq) * D, wk = static_cast<int64_t>(Hk) * D;
  if (N > 0 && Hq > 0 && (!q || !dq_out || !dq || !rows_ok(q, ldq, wq, dtype) || !rows_ok(dq_out, lddqo, wq, dtype) ||
                          !rows_ok(dq, lddq, wq, dtype)))
    return PS_ERR_INVALID_ARG;
  if (N > 0 && Hk > 0 && (!k || !dk_out || !dk || !rows_ok(k, ldk, wk, dtype) || !rows_ok(dk_out, lddko, wk, dtype) ||
                          !rows_ok(dk, lddk, wk, dtype)))
    return PS_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const bool gains = dgq || dgk;
  const int rc = check_ws(ws, ws_bytes, gains ? ps_qk_norm_rope_workspace_size(D) : kWsHeader);
  if (rc != PS_OK) return rc;
  if (N == 0 || Hq + Hk == 0) {
    refused(PS_OK, ws, s);
    for (float* g : {dgq, dgk})
      if (g && !(flags & PS_DW_ACCUMULATE) && cudaMemsetAsync(g, 0, sizeof(float) * D, s) != cudaSuccess)
        return PS_ERR_CUDA;
    return PS_OK;
  }
  QkArgs a = {};
  a.N = N, a.Hq = Hq, a.Hk = Hk, a.D = D, a.R = R;
  a.q = q, a.k = k, a.ldq = ldq, a.ldk = ldk, a.gq = gq, a.gk = gk, a.eps = static_cast<float>(eps);
  a.pos = pos, a.pos_base = pos_base, a.T = T, a.table = reinterpret_cast<const float2*>(table);
  a.qo = dq, a.ko = dk, a.ldqo = lddq, a.ldko = lddk;
  a.dqy = dq_out, a.dky = dk_out, a.lddqy = lddqo, a.lddky = lddko;
  a.part = gains ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kWsHeader) : nullptr;
  a.dgq = dgq, a.dgk = dgk, a.accumulate = (flags & PS_DW_ACCUMULATE) ? 1 : 0;
  a.status = static_cast<uint32_t*>(ws);
  return run_qk<true>(a, dtype, layout, s);
}

int ps_dropout_rows(int64_t N, int d, int dtype, const void* x, int64_t ldx, const void* res, int64_t ldr,
                    const int32_t* row_traj, const int32_t* row_pos, int64_t traj_base, double p, uint64_t seed,
                    uint64_t step, int site, void* y, int64_t ldy, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_dropout_rows");
  if (N < 0 || d < 1 || d > 8 * 65536 || (dtype != PS_DTYPE_BF16 && dtype != PS_DTYPE_F32)) return PS_ERR_INVALID_ARG;
  if (!(p >= 0.0 && p < 1.0) || step > UINT32_MAX || site < 0 || site > 65535 || traj_base < 0 || traj_base > UINT32_MAX)
    return PS_ERR_INVALID_ARG;
  const double cut = floor(p * 65536.0 + 0.5);
  if (cut > 65535.0) return PS_ERR_INVALID_ARG;   // p rounds to 1: nothing would be kept
  if (ldx < d || ldy < d || (res && ldr < d)) return PS_ERR_INVALID_ARG;
  if (N == 0) return PS_OK;
  const int e = elem_bytes(dtype);
  auto aligned = [&](const void* v) { return reinterpret_cast<uintptr_t>(v) % e == 0; };
  if (!x || !y || !row_traj || !row_pos || !aligned(x) || !aligned(y) || !aligned(res)) return PS_ERR_INVALID_ARG;
  DropArgs a = {};
  a.N = N, a.d = d, a.blocks = (d + 7) / 8;
  a.x = x, a.res = res, a.y = y, a.ldx = ldx, a.ldr = ldr, a.ldy = ldy, a.traj = row_traj, a.pos = row_pos;
  a.traj_base = static_cast<uint32_t>(traj_base), a.step = static_cast<uint32_t>(step);
  a.site = static_cast<uint32_t>(site), a.k0 = static_cast<uint32_t>(seed), a.k1 = static_cast<uint32_t>(seed >> 32);
  a.cut = static_cast<uint32_t>(cut) << 16;
  a.scale = static_cast<float>(65536.0 / (65536.0 - cut));
  // rows whose starts lie alike to 16 bytes can be read and written 16 bytes at a time
  auto start = [&](const void* v, int64_t ld, int64_t row) {
    return (reinterpret_cast<uintptr_t>(v) + static_cast<uint64_t>(row) * static_cast<uint64_t>(ld) * e) % 16;
  };
  auto alike = [&](const void* v, int64_t ld) {   // the first two rows decide all
    return start(v, ld, 0) == start(x, ldx, 0) && (N == 1 || start(v, ld, 1) == start(x, ldx, 1));
  };
  int kind = alike(y, ldy) && (!res || alike(res, ldr)) ? kShifted : kAnyhow;
  if (kind == kShifted && d % 8 == 0 && start(x, ldx, 0) == 0 && (N == 1 || start(x, ldx, 1) == 0)) kind = kWhole;
  if (kind == kShifted) a.blocks = (d + 16 / e - 1 + 7) / 8;   // at the largest shift
  a.G = lanes_for(a.blocks);
  const int rows = 32 / a.G, sms = num_sms_current();
  const int64_t row_units = (N + rows - 1) / rows;
  a.parts = parts_for(row_units, static_cast<int64_t>(sms) * 32, (a.blocks + a.G - 1) / a.G);
  // Blocks are dealt out as others end, each with some eight rounds a warp: 60k rows of 771 f32 132 us with as many blocks as
  // are resident, 114 so; 60k of 1537 bf16 152 / 130; a million of 48 (one round a unit) 113 / 139 with a unit a warp.
  const int per_unit = ((a.blocks + a.G - 1) / a.G + a.parts - 1) / a.parts, units_a_warp = per_unit < 8 ? 8 / per_unit : 1;
  const int64_t a_block = static_cast<int64_t>(kDropThreads / 32) * units_a_warp, few = 4 * static_cast<int64_t>(sms);
  int64_t want = (row_units * a.parts + a_block - 1) / a_block;
  const int64_t single = (row_units * a.parts + kDropThreads / 32 - 1) / (kDropThreads / 32);
  if (want < few) want = single < few ? single : few;   // (first every SM has work)
  const unsigned grid = static_cast<unsigned>(want < INT32_MAX ? want : INT32_MAX);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto kern) {
    return launch_after(kern, dim3(grid), kDropThreads, 0, s, 1, 1, true, a) == cudaSuccess ? PS_OK : PS_ERR_CUDA;
  };
  if (dtype == PS_DTYPE_BF16) {
    if (kind == kWhole) return res ? go(dropout_kernel<Bf16, true, kWhole>) : go(dropout_kernel<Bf16, false, kWhole>);
    if (kind == kShifted) return res ? go(dropout_kernel<Bf16, true, kShifted>) : go(dropout_kernel<Bf16, false, kShifted>);
    return res ? go(dropout_kernel<Bf16, true, kAnyhow>) : go(dropout_kernel<Bf16, false, kAnyhow>);
  }
  if (kind == kWhole) return res ? go(dropout_kernel<float, true, kWhole>) : go(dropout_kernel<float, false, kWhole>);
  if (kind == kShifted) return res ? go(dropout_kernel<float, true, kShifted>) : go(dropout_kernel<float, false, kShifted>);
  return res ? go(dropout_kernel<float, true, kAnyhow>) : go(dropout_kernel<float, false, kAnyhow>);
}

}  // extern "C"
