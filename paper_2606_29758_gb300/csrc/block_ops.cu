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

// ================================================================== q/k norms and rotation
//   n = x r g, r = (mean x^2 + eps)^(-1/2) over a head's D values; y = rotation(position) of n's first R dims.
//   backward: dn = rotation^T dy, dg = sum dn x r, dx = r (g dn - x r^2 mean(g dn x)).
// HBM-bound (a read and a write of every element; the backward two reads and a write). A head lies on G lanes, 16
// values each: eight pairs, so a lane rotates by itself and only the mean crosses lanes (log2 G shuffles). A warp takes
// 32 / G heads of one row at a time, queries first, and keeps its lanes' cosines and sines for the row; the loads of
// the next heads are under way while it works on these.
constexpr int kQkThreads = 256;
constexpr int kQkWarps = kQkThreads / 32;

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
  uint32_t* status;             // status word and the count of finished blocks
};

// cos and sin of the lane's eight pairs at a row's position (1 and 0 where the lane's dims are not rotated).
static __device__ __forceinline__ void row_turn(const QkArgs& a, int64_t row, int c, bool rotated, float (&cs)[8],
                                                float (&sn)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = 1.f, sn[i] = 0.f;
  if (a.R == 0) return;
  const int64_t t = static_cast<int64_t>(__ldg(a.pos + row)) - a.pos_base;
  if (t < 0 || t >= a.T) {   // outside the table: NaN in the row's rotated dims
    raise_status(a.status, PS_DEV_BAD_LENGTH);
    if (rotated)
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[i] = sn[i] = __int_as_float(0x7fffffff);
    return;
  }
  if (!rotated) return;
  const float4* at = reinterpret_cast<const float4*>(a.table + t * (a.R / 2) + 8 * c);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = __ldg(at + i);
    cs[2 * i] = v.x, sn[2 * i] = v.y, cs[2 * i + 1] = v.z, sn[2 * i + 1] = v.w;
  }
}

// The lane's 16 values as eight pairs (half: (v[i], v[8 + i]); even: (v[2 i], v[2 i + 1])), turned by (cs, sign sn).
template <bool EVEN>
static __device__ __forceinline__ void turn16(float (&v)[16], const float (&cs)[8], const float (&sn)[8], float sign) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& x = v[EVEN ? 2 * i : i];
    float& y = v[EVEN ? 2 * i + 1 : 8 + i];
    const float s = sign * sn[i], x0 = x, y0 = y;
    x = x0 * cs[i] - y0 * s;
    y = x0 * s + y0 * cs[i];
  }
}

static __device__ __forceinline__ float group_sum(float v, int G) {
  for (int o = G >> 1; o >= 1; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <class T, bool EVEN, bool BWD>
__global__ void __launch_bounds__(kQkThreads) qk_kernel(const QkArgs a) {
  extern __shared__ float qk_smem[];          // gains [2][D]; backward: then a warp's gain gradients [warps][2][D]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (gridDim.x == 1 && threadIdx.x == 0) clear_status(a.status);   // (several blocks: a memset before the launch)
  for (int i = threadIdx.x; i < 2 * a.D; i += kQkThreads) {
    const void* g = i < a.D ? a.gq : a.gk;
    qk_smem[i] = g ? Elem<T>::get(static_cast<const T*>(g)[i < a.D ? i : i - a.D]) : 1.f;
  }
  __syncthreads();

  const int c = lane & (a.G - 1), slot = lane / a.G, at_once = 32 / a.G;
  const bool here = 16 * c < a.D, rotated = 16 * c < a.R;
  const int lo = EVEN || !rotated ? 16 * c : 8 * c;
  const int hi = EVEN || !rotated ? 16 * c + 8 : a.R / 2 + 8 * c;
  const int steps_q = (a.Hq + at_once - 1) / at_once, steps = steps_q + (a.Hk + at_once - 1) / at_once;
  const float inv_d = 1.f / static_cast<float>(a.D);
  float accq[16], acck[16];
  if (BWD) {
#pragma unroll
    for (int i = 0; i < 16; ++i) accq[i] = acck[i] = 0.f;
  }

  const int64_t units = a.N * a.parts, stride = static_cast<int64_t>(gridDim.x) * kQkWarps;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * kQkWarps + warp; u < units; u += stride) {
    const int64_t row = u / a.parts;
    const int part = static_cast<int>(u - row * a.parts);
    const int s0 = steps * part / a.parts, s1 = steps * (part + 1) / a.parts;
    Raw8<T> xa, xb, ya, yb;
    // the head of step s that lies on this lane's group; false where there is none
    auto place = [&](int s, bool& of_q, int& head) {
      of_q = s < steps_q;
      head = (of_q ? s : s - steps_q) * at_once + slot;
      return here && s < s1 && head < (of_q ? a.Hq : a.Hk);
    };
    auto fetch = [&](int s) {
      bool of_q;
      int head;
      xa.zero(), xb.zero();
      if (BWD) ya.zero(), yb.zero();
      if (!place(s, of_q, head)) return;
      const T* x = static_cast<const T*>(of_q ? a.q : a.k) + row * (of_q ? a.ldq : a.ldk) + static_cast<int64_t>(head) * a.D;
      xa.load(x + lo);
      xb.load(x + hi);
      if (BWD) {
        const T* y = static_cast<const T*>(of_q ? a.dqy : a.dky) + row * (of_q ? a.lddqy : a.lddky) +
                     static_cast<int64_t>(head) * a.D;
        ya.load(y + lo);
        yb.load(y + hi);
      }
    };
    fetch(s0);
    float cs[8], sn[8];
    row_turn(a, row, c, rotated, cs, sn);
    for (int s = s0; s < s1; ++s) {
      float x[16], y[16];
      xa.get(x);
      xb.get(x + 8);
      if (BWD) {
        ya.get(y);
        yb.get(y + 8);
      }
      bool of_q;
      int head;
      const bool mine = place(s, of_q, head);
      if (s + 1 < s1) fetch(s + 1);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
      const float r = rsqrtf(fmaf(group_sum(ss, a.G), inv_d, a.eps));
      const float* g = qk_smem + (of_q ? 0 : a.D);
      float gain[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        gain[i] = here ? g[lo + i] : 0.f;
        gain[8 + i] = here ? g[hi + i] : 0.f;
      }
      if (!BWD) {
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = x[i] * r * gain[i];
        turn16<EVEN>(y, cs, sn, 1.f);
      } else {
        turn16<EVEN>(y, cs, sn, -1.f);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float t = y[i] * (x[i] * r);
          if (mine) {
            if (of_q) accq[i] += t;
            else acck[i] += t;
          }
          y[i] *= gain[i];
          dot = fmaf(y[i], x[i], dot);
        }
        const float m = group_sum(dot, a.G) * inv_d * r * r;
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = r * (y[i] - x[i] * m);
      }
      if (mine) {
        T* out = static_cast<T*>(of_q ? a.qo : a.ko) + row * (of_q ? a.ldqo : a.ldko) + static_cast<int64_t>(head) * a.D;
        Raw8<T>::store(out + lo, y);
        Raw8<T>::store(out + hi, y + 8);
      }
    }
  }
  if (!BWD || a.part == nullptr) return;

  // gain gradients: over the warp's heads, the block's warps, then (the last block to finish) the blocks, in f64 and
  // in a fixed order, so that reruns give the same bits
  float* mineq = qk_smem + 2 * a.D + warp * 2 * a.D;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    for (int o = 16; o >= a.G; o >>= 1) {
      accq[i] += __shfl_xor_sync(0xffffffffu, accq[i], o);
      acck[i] += __shfl_xor_sync(0xffffffffu, acck[i], o);
    }
    if (here && slot == 0) {
      const int at = i < 8 ? lo + i : hi + i - 8;
      mineq[at] = accq[i];
      mineq[a.D + at] = acck[i];
    }
  }
  __syncthreads();
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.D;
  for (int i = threadIdx.x; i < 2 * a.D; i += kQkThreads) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kQkWarps; ++w) t += qk_smem[2 * a.D + w * 2 * a.D + i];
    part[i] = t;
  }
  __threadfence();
  __syncthreads();
  __shared__ bool last;
  if (threadIdx.x == 0) last = atomicAdd(a.status + 1, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  // a warp per 32 columns and share of the blocks: shares in shared memory, added up in order
  double* sums = reinterpret_cast<double*>(qk_smem);   // [warps][32]
  for (int col0 = 0; col0 < 2 * a.D; col0 += 32) {
    const int b0 = static_cast<int>(static_cast<int64_t>(gridDim.x) * warp / kQkWarps);
    const int b1 = static_cast<int>(static_cast<int64_t>(gridDim.x) * (warp + 1) / kQkWarps);
    double t = 0.0;
#pragma unroll 8
    for (int b = b0; b < b1; ++b) t += static_cast<double>(__ldcg(a.part + static_cast<int64_t>(b) * 2 * a.D + col0 + lane));
    __syncthreads();
    sums[warp * 32 + lane] = t;
    __syncthreads();
    if (warp == 0) {
      double v = 0.0;
      for (int w = 0; w < kQkWarps; ++w) v += sums[w * 32 + lane];
      const int col = col0 + lane;
      float* out = col < a.D ? a.dgq : a.dgk;
      if (out) {
        float& o = out[col < a.D ? col : col - a.D];
        o = static_cast<float>(a.accumulate ? v + o : v);
      }
    }
  }
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
    const uint32_t hi0 = __umulhi(0xD2511F53u, c.x), lo0 = 0xD2511F53u * c.x;
    const uint32_t hi1 = __umulhi(0xCD9E8D57u, c.z), lo1 = 0xCD9E8D57u * c.z;
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

// Bit j: column 8 b + j of the row is kept.
static __device__ __forceinline__ uint32_t keep8(const DropArgs& a, uint32_t traj, uint32_t pos, int b) {
  const uint4 w = philox4x32_10(make_uint4((a.site << 16) + static_cast<uint32_t>(b), pos, traj, a.step), a.k0, a.k1);
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m |= ((v[i] & 0xffffu) >= a.cut ? 1u << 2 * i : 0u) | ((v[i] >> 16) >= a.cut ? 2u << 2 * i : 0u);
  return m;
}

// HBM-bound next to about ten integer operations an element. VEC: rows of whole blocks at 16-byte boundaries, a
// lane's eight columns in 16-byte accesses. Otherwise the lanes of a warp load 32 neighbouring elements at a time and
// get each one's bit from the lane that drew it.
constexpr int kDropThreads = 256;

template <class T, bool RES, bool VEC>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropArgs a) {
  const int lane = threadIdx.x & 31, c = lane & (a.G - 1), slot = lane / a.G, rows = 32 / a.G;
  const int64_t row_units = (a.N + rows - 1) / rows, units = row_units * a.parts;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * (kDropThreads / 32);
  const T* xs = static_cast<const T*>(a.x);
  const T* rs = static_cast<const T*>(a.res);
  T* ys = static_cast<T*>(a.y);
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kDropThreads / 32) + (threadIdx.x >> 5); u < units; u += stride) {
    const int64_t ru = u / a.parts;
    const int part = static_cast<int>(u - ru * a.parts);
    const int64_t row = ru * rows + slot;
    const bool live = row < a.N;
    const uint32_t traj = live ? static_cast<uint32_t>(__ldg(a.traj + row)) + a.traj_base : 0u;
    const uint32_t pos = live ? static_cast<uint32_t>(__ldg(a.pos + row)) : 0u;
    // this warp's share of the row's blocks, in whole rounds of G
    const int rounds = (a.blocks + a.G - 1) / a.G;
    const int t0 = static_cast<int>(static_cast<int64_t>(rounds) * part / a.parts);
    const int t1 = static_cast<int>(static_cast<int64_t>(rounds) * (part + 1) / a.parts);
    if (VEC) {
#pragma unroll 2
      for (int t = t0; t < t1; ++t) {
        const int b = t * a.G + c;
        if (!live || b >= a.blocks) continue;
        Raw8<T> rx, rr;
        rx.load(xs + row * a.ldx + 8 * b);
        if (RES) rr.load(rs + row * a.ldr + 8 * b);
        const uint32_t m = keep8(a, traj, pos, b);
        float x[8], r[8], y[8];
        rx.get(x);
        if (RES) rr.get(r);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float base = RES ? r[j] : 0.f;
          y[j] = (m >> j & 1u) ? fmaf(x[j], a.scale, base) : base;
        }
        Raw8<T>::store(ys + row * a.ldy + 8 * b, y);
      }
    } else {
      for (int t = t0; t < t1; ++t) {
        const int b0 = t * a.G;
        const uint32_t m = b0 + c < a.blocks ? keep8(a, traj, pos, b0 + c) : 0u;
        // the round's 8 G columns of this lane's row, G at a time
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int in_round = j * a.G + c;
          const uint32_t mm = __shfl_sync(0xffffffffu, m, slot * a.G + (in_round >> 3));
          const int col = b0 * 8 + in_round;
          if (!live || col >= a.d) continue;
          const float base = RES ? Elem<T>::get(rs[row * a.ldr + col]) : 0.f;
          const float x = Elem<T>::get(xs[row * a.ldx + col]);
          ys[row * a.ldy + col] = Elem<T>::put((mm >> (in_round & 7) & 1u) ? fmaf(x, a.scale, base) : base);
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
constexpr int64_t kQkMaxBlocks = 608;   // four per SM; the backward's workspace holds this many partial sums

// A row of heads: its pitch, base and the rows' last element stay within what the kernel addresses.
static bool rows_ok(const void* p, int64_t ld, int64_t cols, int dtype) {
  return al16(p) && ld >= cols && ld * elem_bytes(dtype) % 16 == 0;
}
static bool qk_sizes_ok(int64_t N, int Hq, int Hk, int D, int R, int dtype, int layout) {
  if (N < 0 || Hq < 0 || Hk < 0 || Hq > 65536 || Hk > 65536 || D < 16 || D > 512 || D % 16 || R < 0 || R > D || R % 16)
    return false;
  return (dtype == PS_DTYPE_BF16 || dtype == PS_DTYPE_F32) && (layout == PS_ROPE_HALF || layout == PS_ROPE_EVEN);
}

template <bool BWD>
static int launch_qk(QkArgs a, int dtype, int layout, cudaStream_t s) {
  a.G = lanes_for(a.D / 16);
  const int at_once = 32 / a.G;
  const int steps = (a.Hq + at_once - 1) / at_once + (a.Hk + at_once - 1) / at_once;
  const int sms = num_sms_current();
  a.parts = parts_for(a.N, static_cast<int64_t>(sms) * kQkWarps, steps);
  const int64_t want = (a.N * a.parts + kQkWarps - 1) / kQkWarps;
  const unsigned grid = static_cast<unsigned>(want < kQkMaxBlocks ? want : kQkMaxBlocks);
  const size_t gains = 2 * sizeof(float) * a.D, least = sizeof(double) * kQkWarps * 32;
  const size_t all = BWD ? gains * (1 + kQkWarps) : gains;
  const size_t smem = all > least ? all : least;
  // a block sets its bit early, so one block of several cannot clear the status
  if (grid > 1 && cudaMemsetAsync(a.status, 0, kWsHeader, s) != cudaSuccess) return PS_ERR_CUDA;
  auto go = [&](auto kern) {
    kern<<<grid, kQkThreads, smem, s>>>(a);
    return cudaGetLastError() == cudaSuccess ? PS_OK : refused(PS_ERR_CUDA, a.status, s);
  };
  if (dtype == PS_DTYPE_BF16)
    return layout == PS_ROPE_EVEN ? go(qk_kernel<Bf16, true, BWD>) : go(qk_kernel<Bf16, false, BWD>);
  return layout == PS_ROPE_EVEN ? go(qk_kernel<float, true, BWD>) : go(qk_kernel<float, false, BWD>);
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
  return launch_qk<false>(a, dtype, layout, s);
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
  return launch_qk<true>(a, dtype, layout, s);
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
  a.cut = static_cast<uint32_t>(cut);
  a.scale = static_cast<float>(65536.0 / (65536.0 - cut));
  a.G = lanes_for(a.blocks);
  const int rows = 32 / a.G, sms = num_sms_current();
  const int64_t row_units = (N + rows - 1) / rows;
  a.parts = parts_for(row_units, static_cast<int64_t>(sms) * 32, (a.blocks + a.G - 1) / a.G);
  const int64_t want = (row_units * a.parts + kDropThreads / 32 - 1) / (kDropThreads / 32);
  const int64_t most = static_cast<int64_t>(sms) * 8;
  const unsigned grid = static_cast<unsigned>(want < most ? want : most);
  const bool vec = d % 8 == 0 && rows_ok(x, ldx, d, dtype) && rows_ok(y, ldy, d, dtype) &&
                   (!res || rows_ok(res, ldr, d, dtype));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto kern) {
    kern<<<grid, kDropThreads, 0, s>>>(a);
    return cudaGetLastError() == cudaSuccess ? PS_OK : PS_ERR_CUDA;
  };
  if (dtype == PS_DTYPE_BF16) {
    if (vec) return res ? go(dropout_kernel<Bf16, true, true>) : go(dropout_kernel<Bf16, false, true>);
    return res ? go(dropout_kernel<Bf16, true, false>) : go(dropout_kernel<Bf16, false, false>);
  }
  if (vec) return res ? go(dropout_kernel<float, true, true>) : go(dropout_kernel<float, false, true>);
  return res ? go(dropout_kernel<float, true, false>) : go(dropout_kernel<float, false, false>);
}

}  // extern "C"
