// The norms before and after a branch of a policy block with its gate and the scaled residual sum, in one pass over the
// rows, forward and backward.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "internal.h"
#include "ps_common.cuh"
#include "ps_nvtx.h"
#include "row_elems.cuh"

namespace psk {

//   n = y r_y gy (r_y = (mean y^2 + eps)^(-1/2); without the branch's norm y gy), h = a x + b gate n, o = h r_h go.
//   backward: dH = dh + r_h (go do - h r_h^2 mean(go do h)), dx = a dH, dn = b gate dH, dgy = sum dn y r_y,
//   dgo = sum do h r_h, dy = r_y (gy dn - y r_y^2 mean(gy dn y)), dgate = b sum dH n = b r_y sum gy dH y. That last sum, which
//   dy's mean and dgate share, is sum gy y dh + r_h (sum gy y go do - r_h^2 mean(go do h) sum gy y h), so that all of a
//   backward row's sums are one round of six. (The forward's are two: h's squares from sums over x and y would cancel.)
// HBM-bound: each input is read once and each output written once. A row lies on a team of threads (part of a warp, a
// warp, or some), CH chunks of 16 bytes each, the same columns of every row, so that the gains and their gradients stay
// in its registers over all rows. Rows come through a ring in shared memory that a thread's own copies fill some rows
// ahead: what a thread reads is what it copied, so only the sums cross threads; a row's first sums are taken beside the
// outputs of the row before it, so that their way through the team is hidden.
// Rows that do not start at 16-byte boundaries or have no whole chunks (SHIFT): a chunk is the columns from one
// 16-byte boundary to the next, so the first and last chunks reach over the row's ends; a thread keeps its columns as its rows are
// a multiple of eight apart, whose starts lie alike.
// EXACT (bf16 forwards with the branch's norm): h is the nearest f32 of the sum rounded to bf16,
// whatever the order of the row's sums: the sum of squares, the root and the scales are kept in two f32 each (to 2^-36), y gy is exact in
// f32, the sum over the streams is right up to an f32 and a half, and a value that lies so near to the middle of two bf16 values is
// settled by the roundings that it left. Otherwise some 2 of 10^5 values are rounded to the other neighbour, and one of
// those may show in dgo's sums over few rows as a hundred times f32's error.
// That takes a third of the time more (60000 rows of 3584 without a gate 280 -> 374 us, 6030 of 1536 13.4 -> 16.9).
// Forward and backward of 60000 rows of 3584 bf16 with both norms and a gate 382 and 510 us (4.5 and 5.1 TB/s), without branch norm and
// gate 258 and 500 (6.7 and 5.2); of 30000 f32 rows 275 and 386 (6.3 and 6.7). Both are bound by latency and issue at the 14 warps
// of an SM that the registers allow (forward 52 % of the issue slots, backward 61 %), the lighter ones by HBM. Rows of more than 1024
// chunks (four a thread): 30000 of 8192 bf16 415 and 545 us (4.7 and 5.4 TB/s), 13000 of 16384 400 and 690, 12000 of 8192 f32 283 and
// 570 (5.5 and 4.1); rows of odd widths: 100000 of 771 bf16 232 and 318 (2.7 and 2.9), f32 268 and 395 (4.6 and 4.7).
constexpr int kNormThreads = 512;   // at most
__host__ __device__ constexpr int norm_arrays(bool bwd) { return bwd ? 4 : 2; }   // h, y, do, dh; x, y
// Rows in shared memory: as many as fit beside what the registers allow of threads.
__host__ __device__ constexpr int norm_stages(int ch, bool bwd) { return ch <= 2 ? 3 : bwd ? 1 : 2; }

struct NormArgs {
  int64_t N;
  int d, chunks;                  // chunks of 16 bytes a row
  int team, teams;                // threads per row, and teams of a block
  const void *in[4];              // forward: x, y; backward: h, y, do, dh (nullptr: absent)
  int64_t ld[4];
  int copied;                     // bits of the arrays whose rows come by copies: those there are, but `apart`
  int apart;                      // SHIFT: bits of the arrays (inputs, then outputs from bit 4) whose rows lie otherwise
  const void* like;               // SHIFT: the array that the others lie like, and its pitch
  int64_t ld_like;
  int edge;                       // SHIFT: rows at either end whose chunks may reach over the whole tensor's ends
  const void *gy, *go;            // gains [d], nullptr: 1
  const float* gate;              // [N], nullptr: 1
  int post, pre;                  // a norm of the branch; a normed output (or its gradient)
  float a, b, eps, inv_d;
  float a_lo, b_lo, eps_lo, inv_d_lo;   // EXACT: what f32 leaves of them
  void *out0, *out1;              // forward: h, o; backward: dx, dy
  int64_t ldo0, ldo1;
  float* dgate;
  uint32_t* status;
  float* part;                    // backward: [blocks][2][d] partial gain gradients (dgy, dgo), nullptr without
};

// Two columns: in the forward the two f32 of one instruction (60000 rows of 3584 bf16, post norm and gate, sums in one f32, 306 -> 295 us), in the
// backward plain ones, whose registers the packed ones' pairs would overrun (515 / 537 us).
struct Plain2 {
  float x, y;
};
static __device__ __forceinline__ Plain2 mul2(Plain2 a, Plain2 b) { return {a.x * b.x, a.y * b.y}; }
static __device__ __forceinline__ Plain2 fma2(Plain2 a, Plain2 b, Plain2 c) { return {fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)}; }
static __device__ __forceinline__ void split2(Plain2 a, float& x, float& y) { x = a.x, y = a.y; }
static __device__ __forceinline__ Plain2 add2(Plain2 a, Plain2 b) { return {__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)}; }
static __device__ __forceinline__ F2 add2(F2 a, F2 b) {   // (a packed addition after a packed product would be taken as one fma)
  float x, y, u, v;
  split2(a, x, y);
  split2(b, u, v);
  return pair2(__fadd_rn(x, u), __fadd_rn(y, v));
}
template <bool PACKED>
struct PairOf;
template <>
struct PairOf<true> {
  using type = F2;
  static __device__ __forceinline__ F2 two(float x, float y) { return pair2(x, y); }
};
template <>
struct PairOf<false> {
  using type = Plain2;
  static __device__ __forceinline__ Plain2 two(float x, float y) { return {x, y}; }
};
template <int E, class P2>
struct Vals {   // a chunk's columns
  P2 p[E / 2];
};
template <class P2>
static __device__ __forceinline__ float sum2(P2 v) {
  float x, y;
  split2(v, x, y);
  return x + y;
}

// Bytes of a thread in a stage. (A piece's threads lie side by side: a warp's copies to places apart are fetched a piece at a
// time, half a sector each, 147 instead of 125 us for a backward of 12000 rows of 3584 bf16.)
__host__ __device__ constexpr int norm_thread_bytes(int ch, bool bwd) { return norm_arrays(bwd) * ch * 16; }   // (and 4 for the row's gate)

// The larger of the sizes of two pairs of bf16 (their signs are any).
static __device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// h + l of two f32: with h' + l' (the sums' lower parts added plainly).
static __device__ __forceinline__ void add_two(float& h, float& l, float h2, float l2) {
  const float s = h + h2, b = s - h;
  l = (l + l2) + ((h - (s - b)) + (h2 - b));
  h = s;
}
// a x + w n to the nearest f32: a and w of two parts each, the sum's and the products' roundings taken back.
static __device__ __forceinline__ float settled(float a, float a_lo, float x, float w, float w_lo, float n) {
  const float ax = __fmul_rn(a, x), p = __fmul_rn(w, n), s = __fadd_rn(ax, p), b = s - ax;
  const float left = ((ax - (s - b)) + (p - b)) + (fmaf(w, n, -p) + fmaf(a, x, -ax) + fmaf(w_lo, n, a_lo * x));
  return s + left;
}
// Whether v is the middle of two bf16 values or up to two f32 from it.
static __device__ __forceinline__ bool in_the_middle(float v) { return (__float_as_uint(v) << 16) + 0x80020000u < 0x50000u; }
// Smaller of l and the lower halves of u and v past two before the middle of two bf16 values, in 16 bits each.
static __device__ __forceinline__ uint32_t low_min2(uint32_t l, float u, float v) {
  uint32_t both;
  asm("prmt.b32 %0, %1, %2, 0x5410;" : "=r"(both) : "r"(__float_as_uint(u)), "r"(__float_as_uint(v)));
  asm("add.u16x2 %0, %0, %1;" : "+r"(both) : "r"(0x80028002u));
  asm("min.u16x2 %0, %0, %1;" : "+r"(l) : "r"(both));
  return l;
}
// The sum over a warp of h + l, h >= 0 and |l| of up to 32 roundings of h, the same bits in any order: in units of four roundings
// of the largest h (22 bits) and in 2^-18 of those, by integers. (Exchanges with a sum of two parts each took three times that; they
// are left where the largest h is below 2^-79, whose units f32 would not hold.)
static __device__ __forceinline__ void warp_sum_two(float& h, float& l) {
  const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(h));
  if (top >= 0x7f800000u) {   // infinite, or not a number
    h = __uint_as_float(top);
    l = 0.f;
    return;
  }
  const uint32_t e = top >> 23;
  if (e < 48u) {
#pragma unroll 1
    for (int o = 16; o >= 1; o >>= 1) add_two(h, l, __shfl_xor_sync(0xffffffffu, h, o), __shfl_xor_sync(0xffffffffu, l, o));
    return;
  }
  const float g = __uint_as_float((e - 21) << 23), inv_g = __uint_as_float((275 - e) << 23), magic = 12582912.f;   // 1.5 2^23
  const float big = fmaf(h, inv_g, magic);
  const float rest = fmaf(-(big - magic), g, h) + l, small = fmaf(rest, inv_g * 262144.f, magic);
  const int hs = __reduce_add_sync(0xffffffffu, __float_as_int(big) - 0x4b400000);
  const int ls = __reduce_add_sync(0xffffffffu, __float_as_int(small) - 0x4b400000);
  const float sum = static_cast<float>(hs & ~15) * g, left = static_cast<float>((hs & 15) * 262144 + ls) * (g * (1.f / 262144.f));
  h = sum + left;
  l = left - (h - sum);
}

template <class T, int CH, bool BWD, bool SHIFT, bool EXACT>
__global__ void __launch_bounds__(kNormThreads, 1) norm_kernel(const NormArgs a) {
  constexpr int A = norm_arrays(BWD), ST = norm_stages(CH, BWD), BYTES = norm_thread_bytes(CH, BWD);
  constexpr int E = 16 / static_cast<int>(sizeof(T));             // columns of a chunk
  using P2 = typename PairOf<!BWD>::type;
  using V8 = Vals<E, P2>;
  auto two = [](float x, float y) { return PairOf<!BWD>::two(x, y); };
  constexpr bool PIPE = ST > 1;   // the next row's first sums are taken beside a row's outputs
  constexpr bool kHeld = CH <= 2;                                          // gains in registers
  constexpr int K = BWD ? 6 : EXACT ? 2 : 1;                               // sums of a first round
  extern __shared__ __align__(128) uint8_t norm_smem[];
  __shared__ __align__(16) float red[2][2][kNormThreads / 32 * 8];
  const int threads = blockDim.x, tid = threadIdx.x, lane = tid & 31;
  const int unit_threads = a.team > 32 ? a.team : 32;             // what goes through the rows together
  const int unit_in = tid / unit_threads, units_here = threads / unit_threads;
  const int t = tid % a.team, sub = a.team < 32 ? lane / a.team : 0;
  const int rows_a_unit = a.team < 32 ? 32 / a.team : 1;
  const int64_t units = (a.N + rows_a_unit - 1) / rows_a_unit, stride = static_cast<int64_t>(gridDim.x) * units_here;
  const int64_t u0 = static_cast<int64_t>(blockIdx.x) * units_here + unit_in;
  // from one of a thread's pieces to the next (the forward's in places that the compiler knows)
  const int step = (BWD ? threads : kNormThreads) * 16, stage_bytes = step / 16 * BYTES;
  uint8_t* const mine = norm_smem + tid * 16;
  const P2 zero2 = two(0.f, 0.f);
  auto row_of = [&](int64_t u) { return u * rows_a_unit + sub; };

  // this thread's columns: chunk j begins at col(j)
  int shift = 0;
  if (SHIFT)
    shift = static_cast<int>((reinterpret_cast<uintptr_t>(a.like) + static_cast<uint64_t>(row_of(u0)) * a.ld_like * sizeof(T)) & 15) /
            static_cast<int>(sizeof(T));
  auto col = [&](int j) { return E * (j * a.team + t) - shift; };
  auto some = [&](int j) { return SHIFT ? col(j) < a.d : j * a.team + t < a.chunks; };
  auto all = [&](int j) { return SHIFT ? col(j) >= 0 && col(j) + E <= a.d : some(j); };
  const int apart_j = E * a.team;   // columns from a chunk to the next

  // A round of sums over a team, the same bits in each of its threads: publish() by all, sync(), then totals(). Two rounds that
  // follow each other have different places (which, parity). Six sums: a warp's lanes first share the values out among them,
  // four lanes a value, which takes 9 exchanges instead of 30.
  const int warps = a.team / 32, w0 = unit_in * (a.team > 256 ? 16 : 8);
  auto publish = [&](float (&v)[K], int which, int parity) {
    if (EXACT && which == 0) {
      if (a.team < 32) {
#pragma unroll
        for (int o = 8; o >= 1; o >>= 1)
          if (a.team > o) add_two(v[0], v[K - 1], __shfl_xor_sync(0xffffffffu, v[0], o), __shfl_xor_sync(0xffffffffu, v[K - 1], o));
      } else {
        warp_sum_two(v[0], v[K - 1]);
      }
      if (a.team > 32 && lane == 0) {
        red[which][parity][2 * (w0 + t / 32)] = v[0];
        red[which][parity][2 * (w0 + t / 32) + 1] = v[K - 1];
      }
    } else if (BWD && a.team >= 32) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i < K ? v[i < K ? i : 0] : 0.f;
#pragma unroll
      for (int o = 4; o >= 1; o >>= 1) {
        const bool up = lane & (4 * o);
#pragma unroll
        for (int i = 0; i < o; ++i) x[i] = (up ? x[i + o] : x[i]) + __shfl_xor_sync(0xffffffffu, up ? x[i] : x[i + o], 4 * o);
      }
      x[0] += __shfl_xor_sync(0xffffffffu, x[0], 2);
      x[0] += __shfl_xor_sync(0xffffffffu, x[0], 1);
      v[0] = x[0];   // of value lane / 4
      if (a.team > 32 && (lane & 3) == 0) red[which][parity][(unit_in * warps + t / 32) * 8 + lane / 4] = x[0];
    } else if (!BWD && a.team >= 32) {
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
      if (a.team > 32 && lane == 0) red[which][parity][w0 + t / 32] = v[0];
    } else {
#pragma unroll
      for (int o = 8; o >= 1; o >>= 1)
        if (a.team > o)
#pragma unroll
          for (int i = 0; i < (BWD ? K : 1); ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
  };
  auto sync = [&]() {
    if (a.team > 32) asm volatile("bar.sync %0, %1;" ::"r"(unit_in + 1), "r"(a.team) : "memory");
  };
  auto totals = [&](float (&v)[K], int which, int parity) {
    if (EXACT && which == 0) {
      if (a.team <= 32) return;
      const float2 x = lane < warps ? *reinterpret_cast<const float2*>(red[which][parity] + 2 * (w0 + lane)) : make_float2(0.f, 0.f);
      v[0] = x.x, v[K - 1] = x.y;
      warp_sum_two(v[0], v[K - 1]);
    } else if (BWD) {
      if (a.team < 32) return;
      float x = v[0];
      int at = 4;                                 // lanes from a value to the next
      if (a.team > 32) {
        const int w = lane >> 3;
        const float* from = red[which][parity] + (unit_in * warps + w) * 8 + (lane & 7);
        x = w < warps ? from[0] : 0.f;
#pragma unroll
        for (int k = 1; k < 4; ++k)
          if (4 * k < warps) x += w + 4 * k < warps ? from[32 * k] : 0.f;
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        x += __shfl_xor_sync(0xffffffffu, x, 16);
        at = 1;
      }
#pragma unroll
      for (int i = 0; i < K; ++i) v[i] = __shfl_sync(0xffffffffu, x, i * at);
    } else if (a.team > 32) {
      const float4* from = reinterpret_cast<const float4*>(red[which][parity] + w0);   // (zeros behind the last warp)
      const float4 x = from[0], y = from[1];
      v[0] = ((x.x + x.y) + (x.z + x.w)) + ((y.x + y.y) + (y.z + y.w));
      if (a.team > 256) {
        const float4 z = from[2], w = from[3];
        v[0] += ((z.x + z.y) + (z.z + z.w)) + ((w.x + w.y) + (w.z + w.w));
      }
    }
  };

  // chunk j of an array's row in a stage
  auto slot = [&](int st, int arr, int j) { return mine + st * stage_bytes + (arr * CH + j) * step; };
  auto get = [&](int st, int arr, int j) {
    V8 v;
    const uint4 w = *reinterpret_cast<const uint4*>(slot(st, arr, j));
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < E / 2; ++i)
      v.p[i] = E == 8 ? two(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u))
                      : two(__uint_as_float(x[2 * i & 3]), __uint_as_float(x[(2 * i + 1) & 3]));
    return v;
  };
  // what no copy reaches (absent arrays, chunks behind the row) reads as zeros
  auto clear_row = [&](int st) {
#pragma unroll 1
    for (int i = 0; i < A * CH; ++i) *reinterpret_cast<uint4*>(mine + st * stage_bytes + i * step) = make_uint4(0, 0, 0, 0);
  };
  // the row's gate, beside its pieces (loaded ahead into a register it is waited for where the loop hands it on: 346 instead of
  // 271 us for a forward of 60000 rows of 3584 bf16, sums in one f32)
  float* const gates = reinterpret_cast<float*>(norm_smem + ST * stage_bytes) + tid;
  for (int s = 0; s < ST; ++s) {
    clear_row(s);
    gates[s * threads] = 1.f;
  }
  if (!BWD) {
    for (int i = tid; i < 4 * kNormThreads / 32 * 8; i += threads) (&red[0][0][0])[i] = 0.f;
    __syncthreads();
  }
  // The copies of a unit's row into a stage; a group for each, be it empty.
  auto issue = [&](int64_t u, int st) {
    const int64_t row = row_of(u);
    if (row < a.N) {
      if (a.gate)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_addr(gates + st * threads)), "l"(a.gate + row) : "memory");
#pragma unroll
      for (int arr = 0; arr < A; ++arr) {
        const T* from = static_cast<const T*>(a.in[arr]) + row * a.ld[arr] + (E * t - shift);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          const int c = col(j);
          // a chunk with some of the row; beyond the first row's start and the last one's end it goes element by element
          if (SHIFT ? c + E <= 0 || c >= a.d || (c < 0 && row < a.edge) || (c + E > a.d && row >= a.N - a.edge) : !some(j)) continue;
          if (a.copied >> arr & 1) lane_copy(smem_addr(slot(st, arr, j)), from + j * apart_j);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // chunk j of a row, element by element: what its copies left out
  auto load_plainly = [&](int64_t row, int st, int j) {
#pragma unroll 1
    for (int arr = 0; arr < A; ++arr) {
      if (!a.in[arr] || ((a.copied >> arr & 1) && all(j))) continue;
      const T* at = static_cast<const T*>(a.in[arr]) + row * a.ld[arr];
#pragma unroll 1
      for (int i = 0; i < E; ++i)
        if (col(j) + i >= 0 && col(j) + i < a.d) reinterpret_cast<T*>(slot(st, arr, j))[i] = at[col(j) + i];
    }
  };
  // a unit's row in its stage: the stages after it may still be under way
  auto arrive = [&](int64_t row, int st, bool first) {
    if (first || !PIPE)
      asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
    else
      asm volatile("cp.async.wait_group %0;" ::"n"(PIPE ? ST - 2 : 0) : "memory");
    if (row >= a.N) clear_row(st);
    if (SHIFT && row < a.N) {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        if (some(j) && ((a.apart & 15) || ((row < a.edge || row >= a.N - a.edge) && !all(j)))) load_plainly(row, st, j);
        if (!some(j) || all(j)) continue;
        uint32_t keep[4];   // of the row's end only its columns
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int c = col(j) + w * E / 4;
          keep[w] = E == 8 ? (c >= 0 && c < a.d ? 0xffffu : 0u) | (c + 1 >= 0 && c + 1 < a.d ? 0xffff0000u : 0u)
                           : c >= 0 && c < a.d ? 0xffffffffu : 0u;
        }
#pragma unroll
        for (int arr = 0; arr < A; ++arr) {
          uint4& v = *reinterpret_cast<uint4*>(slot(st, arr, j));
          v = make_uint4(v.x & keep[0], v.y & keep[1], v.z & keep[2], v.w & keep[3]);
        }
      }
    }
  };
  auto gains_at = [&](const void* g, int j) {
    const T* at = static_cast<const T*>(g);
    float f[8];
    if (!SHIFT && g && E == 8 && all(j)) {
      Raw8<T> r;
      r.load(at + col(j));
      r.get(f);
    } else
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = g && col(j) + i >= 0 && col(j) + i < a.d ? Elem<T>::get(at[col(j) + i]) : 1.f;
    V8 v;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) v.p[i] = two(f[2 * i], f[2 * i + 1]);
    return v;
  };
  auto put = [&](int which, int64_t row, int j, const V8& v) {
    T* at = static_cast<T*>(which ? a.out1 : a.out0) + row * (which ? a.ldo1 : a.ldo0) + col(j);
    float f[8];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) split2(v.p[i], f[2 * i], f[2 * i + 1]);
    if (all(j) && !(SHIFT && (a.apart >> (4 + which) & 1))) {
      *reinterpret_cast<uint4*>(at) =
          E == 8 ? make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4 % E], f[5 % E]),
                              pack_bf16x2(f[6 % E], f[7 % E]))
                 : make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    } else if (SHIFT && some(j)) {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (col(j) + i >= 0 && col(j) + i < a.d) at[i] = Elem<T>::put(f[i]);
    }
  };

  wait_for_previous_kernel();
  let_next_kernel_in();
  if (BWD && a.status && blockIdx.x == 0 && tid == 0) clear_status(a.status);
#pragma unroll
  for (int s = 0; s < ST; ++s) issue(u0 + s * stride, s);

  V8 gy_r[kHeld ? CH : 1], go_r[kHeld ? CH : 1];
  if (kHeld)
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      gy_r[j] = gains_at(a.gy, j);
      go_r[j] = gains_at(a.go, j);
    }
  auto gain_y = [&](int j) { return kHeld ? gy_r[kHeld ? j : 0] : gains_at(a.gy, j); };
  auto gain_o = [&](int j) { return kHeld ? go_r[kHeld ? j : 0] : gains_at(a.go, j); };
  V8 accy[BWD ? CH : 1], acco[BWD ? CH : 1];
  if (BWD)
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
      for (int i = 0; i < E / 2; ++i) accy[j].p[i] = acco[j].p[i] = zero2;

  // the sums over a row as it comes in
  auto first_sums = [&](int st, float (&s)[K]) {
    if (BWD) {
      P2 q2[6] = {zero2, zero2, zero2, zero2, zero2, zero2};
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const V8 h = get(st, 0, j), y = get(st, 1, j), q = get(st, BWD ? 2 : 0, j), dh = get(st, BWD ? 3 : 0, j);
        const V8 gy = gain_y(j), go = gain_o(j);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          const P2 gq = mul2(go.p[i], q.p[i]), yg = mul2(gy.p[i], y.p[i]);
          q2[0] = fma2(h.p[i], h.p[i], q2[0]);
          q2[1] = fma2(gq, h.p[i], q2[1]);
          q2[2] = fma2(y.p[i], y.p[i], q2[2]);
          q2[3] = fma2(yg, dh.p[i], q2[3]);
          q2[4] = fma2(yg, gq, q2[4]);
          q2[5] = fma2(yg, h.p[i], q2[5]);
        }
      }
#pragma unroll
      for (int i = 0; i < K; ++i) s[i] = sum2(q2[i]);
    } else {
      P2 q2 = zero2;
      if (EXACT) {
        // A square of eight bits is exact. From the largest one on each sum is at most doubled, so that its difference to the sum
        // before it is exact, and so is what it left out (four packed operations for two squares).
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          const uint4 w = *reinterpret_cast<const uint4*>(slot(st, 1, j));
          m = max_abs2(max_abs2(m, w.x), max_abs2(w.y, max_abs2(w.z, w.w)));
        }
        const float most = fmaxf(__uint_as_float(m << 16 & 0x7fffffffu), __uint_as_float(m & 0x7fff0000u));
        const float from = most < 1e18f ? most * most : 0.f;   // (a sum near f32's range from 0 on)
        const P2 minus = two(-1.f, -1.f), one = two(1.f, 1.f);
        P2 hi = two(from, from), lo = zero2;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          const V8 y = get(st, 1, j);
#pragma unroll
          for (int i = 0; i < E / 2; ++i) {
            const P2 sum = fma2(y.p[i], y.p[i], hi);
            lo = fma2(fma2(y.p[i], y.p[i], fma2(sum, minus, hi)), one, lo);
            hi = sum;
          }
        }
        float h2, l2;
        split2(hi, s[0], h2);
        split2(lo, s[K - 1], l2);
        add_two(s[0], s[K - 1], h2, l2);
        if (s[0] < INFINITY) add_two(s[0], s[K - 1], -2.f * from, 0.f);
        return;
      }
      if (a.post)
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          const V8 y = get(st, 1, j);
#pragma unroll
          for (int i = 0; i < E / 2; ++i) q2 = fma2(y.p[i], y.p[i], q2);
        }
      s[0] = sum2(q2);
    }
  };

  float s[K];
  int st = 0, parity = 0;
  if (u0 < units) {
    arrive(row_of(u0), 0, true);
    first_sums(0, s);
    publish(s, 0, 0);
    sync();
    totals(s, 0, 0);
  }
  for (int64_t u = u0; u < units; u += stride) {
    const int64_t row = row_of(u);
    const bool live = row < a.N, more = u + stride < units;
    const float gate = gates[st * threads];
    const bool open = live && a.in[1] && gate != 0.f;   // (a closed gate leaves the branch out whatever it holds)
    const int st_next = st + 1 == ST ? 0 : st + 1;
    float s_next[K];
    parity ^= 1;
    if (PIPE && more) {
      arrive(row_of(u + stride), st_next, false);
      first_sums(st_next, s_next);
      publish(s_next, 0, parity);
    }
    if (!BWD) {
      float ry = 1.f, w = a.b * gate, w_lo = 0.f;
      if (!EXACT) {
        ry = a.post ? rsqrtf(fmaf(s[0], a.inv_d, a.eps)) : 1.f;
        w *= ry;
      } else {
        w_lo = fmaf(a.b, gate, -w) + a.b_lo * gate;
        if (a.post) {
          // the mean and eps, the inverse root by a step from its approximation r (1 - v r^2 without cancelling), times the scales
          float v = s[0] * a.inv_d, v_lo = fmaf(s[0], a.inv_d, -v) + (s[0] * a.inv_d_lo + s[K - 1] * a.inv_d);
          add_two(v, v_lo, a.eps, a.eps_lo);
          ry = rsqrtf(v);
          const float q = ry * ry;
          const float left = fmaf(-v, q, 1.f) - fmaf(v, fmaf(ry, ry, -q), v_lo * q);
          // (no step from a root of 0, or from one whose square is beyond f32: v below 3e-39)
          const float r_lo = fabsf(left) < 1.f ? 0.5f * ry * left : 0.f, wr = w * ry;
          w_lo = fmaf(w, ry, -wr) + fmaf(w, r_lo, w_lo * ry);
          w = wr;
        }
      }
      const P2 w2 = two(w, w), a2 = two(a.a, a.a), wl2 = two(w_lo, w_lo), al2 = two(a.a_lo, a.a_lo), minus = two(-1.f, -1.f);
      const P2 minus_a = mul2(a2, minus), minus_w = mul2(w2, minus);
      const bool unit = a.a == 1.f && a.a_lo < 1e-30f;
      V8 h[CH];
      P2 q = zero2;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const V8 x = get(st, 0, j);
        if (EXACT && open) {
          const V8 y = get(st, 1, j), g = gain_y(j);
          V8 n;
          uint32_t lowest = 0xffffffffu;
#pragma unroll
          for (int i = 0; i < E / 2; ++i) {
            n.p[i] = mul2(y.p[i], g.p[i]);   // (exact)
            // a x + w n up to one f32 and a half: negated, and what its first parts left
            if (unit) {
              h[j].p[i] = fma2(wl2, n.p[i], fma2(w2, n.p[i], x.p[i]));
            } else {
              const P2 wn = mul2(n.p[i], minus_w);   // (of a x an infinity stays one in both parts)
              const P2 left = fma2(x.p[i], al2, fma2(wl2, n.p[i], fma2(w2, n.p[i], wn)));
              h[j].p[i] = fma2(fma2(x.p[i], minus_a, wn), minus, left);
            }
            float u, v;
            split2(h[j].p[i], u, v);
            lowest = low_min2(lowest, u, v);
          }
          if ((lowest & 0xffffu) <= 4u || lowest <= 0x4ffffu) {   // (as in_the_middle, for all at once)
            float hv[E], xv[E], nv[E];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
              split2(h[j].p[i], hv[2 * i], hv[2 * i + 1]);
              split2(x.p[i], xv[2 * i], xv[2 * i + 1]);
              split2(n.p[i], nv[2 * i], nv[2 * i + 1]);
#pragma unroll
              for (int k = 2 * i; k < 2 * i + 2; ++k)
                if (in_the_middle(hv[k])) hv[k] = settled(a.a, a.a_lo, xv[k], w, w_lo, nv[k]);
              h[j].p[i] = two(hv[2 * i], hv[2 * i + 1]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < E / 2; ++i) h[j].p[i] = EXACT ? fma2(x.p[i], a2, mul2(x.p[i], al2)) : mul2(x.p[i], a2);
          if (open) {
            const V8 y = get(st, 1, j), g = gain_y(j);
#pragma unroll
            // (the product rounded before the sum: scales like 0.7 then give sums of few bits what they give in decimals)
            for (int i = 0; i < E / 2; ++i) h[j].p[i] = add2(h[j].p[i], mul2(mul2(y.p[i], g.p[i]), w2));
          }
        }
        if (live && a.in[1]) put(0, row, j, h[j]);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) q = fma2(h[j].p[i], h[j].p[i], q);
      }
      float sh[K] = {sum2(q)};
      publish(sh, 1, parity);
      issue(u + ST * stride, st);   // (the stage has been read: its values went into what was published)
      sync();
      if (a.pre) {
        totals(sh, 1, parity);
        const float rh = rsqrtf(fmaf(sh[0], a.inv_d, a.eps));
        const P2 r2 = two(rh, rh);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          const V8 g = gain_o(j);
          V8 o;
#pragma unroll
          for (int i = 0; i < E / 2; ++i) o.p[i] = mul2(mul2(h[j].p[i], r2), g.p[i]);
          if (live) put(1, row, j, o);
        }
      }
    } else {
      // (0 for rows that are not there: dgo's sums go over them)
      const float rh = a.pre && live ? rsqrtf(fmaf(s[0], a.inv_d, a.eps)) : 0.f, m = -s[K > 1 ? 1 : 0] * a.inv_d * rh * rh;
      const float ry = a.post ? rsqrtf(fmaf(s[K > 2 ? 2 : 0], a.inv_d, a.eps)) : 1.f;
      const float dot = s[K > 3 ? 3 : 0] + rh * fmaf(m, s[K > 5 ? 5 : 0], s[K > 4 ? 4 : 0]);   // of gy dH y
      const float w = a.b * gate * ry, k = a.post ? -dot * a.inv_d * ry * ry * w : 0.f;
      const P2 r2 = two(rh, rh), m2 = two(m, m), a2 = two(a.a, a.a), w2 = two(w, w), k2 = two(k, k);
      if (a.dgate && live && t == 0) a.dgate[row] = a.b * ry * dot;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        V8 dH = get(st, BWD ? 3 : 0, j);
        {
          const V8 h = get(st, 0, j), q = get(st, BWD ? 2 : 0, j), g = gain_o(j);
#pragma unroll
          for (int i = 0; i < E / 2; ++i) {
            dH.p[i] = fma2(r2, fma2(h.p[i], m2, mul2(g.p[i], q.p[i])), dH.p[i]);
            acco[BWD ? j : 0].p[i] = fma2(q.p[i], mul2(h.p[i], r2), acco[BWD ? j : 0].p[i]);
          }
        }
        V8 v;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) v.p[i] = mul2(a2, dH.p[i]);
        if (live) put(0, row, j, v);
        if (open) {
          const V8 y = get(st, 1, j), g = gain_y(j);
#pragma unroll
          for (int i = 0; i < E / 2; ++i) {
            const P2 dn = mul2(w2, dH.p[i]);
            accy[BWD ? j : 0].p[i] = fma2(dn, y.p[i], accy[BWD ? j : 0].p[i]);
            v.p[i] = fma2(k2, y.p[i], mul2(g.p[i], dn));
          }
          put(1, row, j, v);
        } else if (live && a.in[1]) {
#pragma unroll
          for (int i = 0; i < E / 2; ++i) v.p[i] = zero2;
          put(1, row, j, v);
        }
      }
      issue(u + ST * stride, st);   // (the stage has been read: its values went into what was stored)
      if (PIPE) sync();
    }
    if (more) {
      if (!PIPE) {
        arrive(row_of(u + stride), st_next, false);
        first_sums(st_next, s_next);
        publish(s_next, 0, parity);
        sync();
      }
      totals(s_next, 0, parity);
#pragma unroll
      for (int i = 0; i < K; ++i) s[i] = s_next[i];
    }
    st = st_next;
  }
  if (!BWD || a.part == nullptr) return;

  // gain gradients: over a warp's rows, then the block's units in order; norm_gain_sum_kernel adds the blocks'
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  float* sums = reinterpret_cast<float*>(norm_smem) + static_cast<size_t>(unit_in) * 2 * a.d;
  if (SHIFT) {   // (a warp's rows may have different columns; those without a row have none)
    for (int c = tid % unit_threads; c < 2 * a.d; c += unit_threads) sums[c] = 0.f;
    __syncthreads();
  }
  for (int k = 0; k < (SHIFT ? rows_a_unit : 1); ++k) {
    if (!SHIFT || sub == k)
#pragma unroll
      for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int i = 0; i < E; ++i) {
          float v[2], w[2];
          split2(accy[BWD ? j : 0].p[i / 2], v[0], v[1]);
          split2(acco[BWD ? j : 0].p[i / 2], w[0], w[1]);
          const int c = col(j) + i;
          if (SHIFT) {
            if (c >= 0 && c < a.d) {
              sums[c] += v[i & 1];
              sums[a.d + c] += w[i & 1];
            }
          } else {
            for (int o = 16; o >= a.team; o >>= 1) {
              v[i & 1] += __shfl_xor_sync(0xffffffffu, v[i & 1], o);
              w[i & 1] += __shfl_xor_sync(0xffffffffu, w[i & 1], o);
            }
            if (sub == 0 && c < a.d) {
              sums[c] = v[i & 1];
              sums[a.d + c] = w[i & 1];
            }
          }
        }
    if (SHIFT) __syncwarp();
  }
  __syncthreads();
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.d;
  for (int c = tid; c < 2 * a.d; c += threads) {
    float v = 0.f;
    for (int k = 0; k < units_here; ++k) v += reinterpret_cast<const float*>(norm_smem)[static_cast<size_t>(k) * 2 * a.d + c];
    part[c] = v;
  }
}

// The blocks' partial gain gradients [blocks][2][d], 32 columns a block: a thread adds every 32nd block's of four columns, the
// shares are added in order in f64, so that reruns give the same bits.
__global__ void __launch_bounds__(256) norm_gain_sum_kernel(int d, int blocks, const float* __restrict__ part, float* dgy,
                                                            float* dgo, int accumulate) {
  __shared__ float sums[32][33];
  wait_for_previous_kernel();
  const int g = threadIdx.x & 7, share = threadIdx.x >> 3, col = blockIdx.x * 32 + 4 * g;
  float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 5
  for (int b = share; b < blocks; b += 32)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < 2 * d) t[i] += part[static_cast<int64_t>(b) * 2 * d + col + i];
#pragma unroll
  for (int i = 0; i < 4; ++i) sums[share][4 * g + i] = t[i];
  __syncthreads();
  // eight threads a column, four shares each
  const int c = threadIdx.x >> 3, at = blockIdx.x * 32 + c;
  double v = 0.0;
#pragma unroll
  for (int k = 0; k < 4; ++k) v += static_cast<double>(sums[4 * g + k][c]);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (g != 0 || at >= 2 * d) return;
  float* out = at < d ? dgy : dgo;
  if (!out) return;
  float& o = out[at < d ? at : at - d];
  o = static_cast<float>(accumulate ? v + o : v);
}

// ================================================================== host side
constexpr int kNormMaxBytes = 32768;        // of a row: bf16 16384 columns, f32 8192
constexpr size_t kSmemOfSm = 227 * 1024;
constexpr int64_t kNormMaxBlocks = 304;    // of a backward at most; its workspace holds a partial sum of each

struct NormPlan {
  int ch, team, teams, threads, blocks_a_sm;
  size_t smem;
};
// Threads of two chunks of a row each, up to 512 to a row, then four each. (One chunk each: 183750 rows of 128 bf16 47 and 62 us
// instead of 36 and 56; four: 100000 of 1536 321 instead of 234 forward.)
static NormPlan norm_plan(int chunks, int d, bool bwd) {
  NormPlan p;
  p.ch = 2;
  while ((chunks + p.ch - 1) / p.ch > kNormThreads) p.ch *= 2;
  const int need = (chunks + p.ch - 1) / p.ch;
  if (need <= 32) {
    p.team = 1;
    while (p.team < need) p.team *= 2;
  } else {
    p.team = (need + 31) / 32 * 32;
  }
  const int unit_threads = p.team > 32 ? p.team : 32;
  // blocks of about 256 threads, or of as many teams as fill an SM better (6030 rows of 1536 bf16, five teams of 96 instead of
  // four: backward 45 -> 40 us)
  auto filled = [&](int teams) { return kNormThreads / (teams * unit_threads) * teams; };
  p.teams = 256 / unit_threads > 1 ? 256 / unit_threads : 1;
  for (int t = p.teams + 1; t * unit_threads <= kNormThreads; ++t)
    if (filled(t) > filled(p.teams)) p.teams = t;
  p.threads = p.teams * unit_threads;
  p.smem = static_cast<size_t>(norm_stages(p.ch, bwd)) * (norm_thread_bytes(p.ch, bwd) + 4) * (bwd ? p.threads : kNormThreads);
  const size_t sums = bwd ? static_cast<size_t>(p.teams) * 2 * d * sizeof(float) : 0;
  if (p.smem < sums) p.smem = sums;
  p.blocks_a_sm = 512 / p.threads;
  const int fit = static_cast<int>(kSmemOfSm / (p.smem + 2048));
  if (p.blocks_a_sm > fit) p.blocks_a_sm = fit;
  if (p.blocks_a_sm < 1) p.blocks_a_sm = 1;
  return p;
}

template <class T, int CH, bool BWD, bool SHIFT, bool EXACT>
static int launch_as(NormArgs& a, const NormPlan& p, int& grid, cudaStream_t s) {
  auto kern = norm_kernel<T, CH, BWD, SHIFT, EXACT>;
  if (p.smem > 40 * 1024 &&   // (beside the block's own)
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(p.smem)) != cudaSuccess)
    return PS_ERR_CUDA;
  const int rows_a_unit = a.team < 32 ? 32 / a.team : 1;
  const int64_t units = (a.N + rows_a_unit - 1) / rows_a_unit;
  int64_t want = (units + p.teams - 1) / p.teams, most = static_cast<int64_t>(num_sms_current()) * p.blocks_a_sm;
  if (BWD && most > kNormMaxBlocks) most = kNormMaxBlocks;
  if (SHIFT) {   // units a multiple of eight, so that a thread's rows start alike
    want = (want + 7) / 8 * 8;
    most = most > 8 ? most / 8 * 8 : 8;
  }
  grid = static_cast<int>(want < most ? want : most);
  a.copied = 0;
  for (int i = 0; i < 4; ++i)
    if (a.in[i] && !(SHIFT && (a.apart >> i & 1))) a.copied |= 1 << i;
  return launch_after(kern, dim3(static_cast<unsigned>(grid)), static_cast<unsigned>(p.threads), p.smem, s, 1, 1, true, a) ==
                 cudaSuccess
             ? PS_OK
             : PS_ERR_CUDA;
}
template <class T, int CH, bool BWD, bool SHIFT>
static int launch_norm(NormArgs& a, const NormPlan& p, int& grid, cudaStream_t s) {
  if constexpr (!BWD && sizeof(T) == 2)
    if (a.in[1] && a.post) return launch_as<T, CH, BWD, SHIFT, true>(a, p, grid, s);
  return launch_as<T, CH, BWD, SHIFT, false>(a, p, grid, s);
}
template <class T, bool BWD>
static int run_norm(NormArgs a, bool shift, int& grid, cudaStream_t s) {
  constexpr int E = 16 / static_cast<int>(sizeof(T));
  a.chunks = shift ? (a.d + 2 * E - 2) / E : a.d / E;   // at the largest shift
  if (a.chunks > 4 * kNormThreads) return PS_ERR_UNSUPPORTED;
  const NormPlan p = norm_plan(a.chunks, a.d, BWD);
  a.team = p.team, a.teams = p.teams;
  a.edge = (E + a.d - 2) / a.d;                           // (a chunk reaches E - 1 columns over a row's end at most)
  a.inv_d = static_cast<float>(1.0 / a.d);
  a.inv_d_lo = static_cast<float>(1.0 / a.d - a.inv_d);
  switch (p.ch) {
    case 2: return shift ? launch_norm<T, 2, BWD, true>(a, p, grid, s) : launch_norm<T, 2, BWD, false>(a, p, grid, s);
    default: return shift ? launch_norm<T, 4, BWD, true>(a, p, grid, s) : launch_norm<T, 4, BWD, false>(a, p, grid, s);
  }
}

}  // namespace psk

using namespace psk;

namespace {

bool norm_sizes_ok(int64_t N, int d, int dtype, int norms, double a, double b, double eps) {
  auto isfinite = [](double v) { return ::isfinite(static_cast<float>(v)) != 0; };   // (as the kernels have them)
  return N >= 0 && d >= 1 && (dtype == PS_DTYPE_BF16 || dtype == PS_DTYPE_F32) && d <= kNormMaxBytes / elem_bytes(dtype) &&
         !(norms & ~(PS_NORM_BRANCH | PS_NORM_OUT)) && isfinite(a) && isfinite(b) && eps >= 0.0 && isfinite(eps);
}
// The tensors of a call: on their elements' boundaries, and whether all rows lie on 16-byte boundaries, or like each other.
struct NormRows {
  const int64_t N;
  const int e, d;
  bool ok = true, whole;
  const void* like = nullptr;
  int64_t ld_like = 0;
  int apart = 0;
  NormRows(int64_t N_, int d_, int dtype) : N(N_), e(elem_bytes(dtype)), d(d_), whole(d_ * e % 16 == 0) {}
  void rows(const void* p, int64_t ld, int bit) {
    ok = ok && p && ld >= d && reinterpret_cast<uintptr_t>(p) % e == 0;
    whole = whole && al16(p) && (N == 1 || ld * e % 16 == 0);
    if (!like) like = p, ld_like = ld;
    auto start = [&](const void* v, int64_t l, int64_t row) {
      return (reinterpret_cast<uintptr_t>(v) + static_cast<uint64_t>(row) * static_cast<uint64_t>(l) * e) % 16;
    };
    // the first two rows decide all
    if (start(p, ld, 0) != start(like, ld_like, 0) || (N > 1 && start(p, ld, 1) != start(like, ld_like, 1))) apart |= 1 << bit;
  }
  void gains(const void* p) {
    ok = ok && reinterpret_cast<uintptr_t>(p) % e == 0;
    whole = whole && al16(p);
  }
  void into(NormArgs& a) const { a.apart = apart, a.like = like, a.ld_like = ld_like; }
};

}  // namespace

extern "C" {

int ps_residual_norm_fwd(int64_t N, int d, int dtype, int norms, const void* x, int64_t ldx, const void* y, int64_t ldy,
                         const void* gy, const void* go, const float* gate, double res_scale, double branch_scale, double eps,
                         void* h, int64_t ldh, void* o, int64_t ldo, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_residual_norm_fwd");
  if (!norm_sizes_ok(N, d, dtype, norms, res_scale, branch_scale, eps)) return PS_ERR_INVALID_ARG;
  if (N == 0) return PS_OK;
  const bool out = norms & PS_NORM_OUT;
  if (!y && ((norms & PS_NORM_BRANCH) || gate || !out)) return PS_ERR_INVALID_ARG;   // a branch's norm or gate without one
  NormRows r(N, d, dtype);
  r.rows(x, ldx, 0);
  if (y) {
    r.rows(y, ldy, 1);
    r.rows(h, ldh, 4);
    r.gains(gy);
  }
  if (out) {
    r.rows(o, ldo, 5);
    r.gains(go);
  }
  if (!r.ok || reinterpret_cast<uintptr_t>(gate) % 4) return PS_ERR_INVALID_ARG;
  NormArgs a = {};
  a.N = N, a.d = d;
  a.in[0] = x, a.in[1] = y, a.ld[0] = ldx, a.ld[1] = ldy;
  a.gy = gy, a.go = go, a.gate = gate;
  a.post = (norms & PS_NORM_BRANCH) ? 1 : 0, a.pre = out ? 1 : 0;
  r.into(a);
  a.a = y ? static_cast<float>(res_scale) : 1.f, a.b = static_cast<float>(branch_scale), a.eps = static_cast<float>(eps);
  a.a_lo = y ? static_cast<float>(res_scale - a.a) : 0.f;
  a.b_lo = static_cast<float>(branch_scale - a.b), a.eps_lo = static_cast<float>(eps - a.eps);
  if (y && dtype == PS_DTYPE_BF16 && (norms & PS_NORM_BRANCH) && fabsf(a.a) > 1e-30f) {
    // EXACT: both parts of one sign and neither 0, so that the two products of an infinity add up to it.
    if (fabs(static_cast<double>(a.a)) > fabs(res_scale)) a.a = nextafterf(a.a, 0.f);
    a.a_lo = static_cast<float>(res_scale - a.a);
    if (a.a_lo == 0.f) a.a_lo = copysignf(1e-45f, a.a);
  }
  a.out0 = h, a.out1 = o, a.ldo0 = ldh, a.ldo1 = ldo;
  int grid;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return dtype == PS_DTYPE_F32 ? run_norm<float, false>(a, !r.whole, grid, s) : run_norm<Bf16, false>(a, !r.whole, grid, s);
}

size_t ps_residual_norm_workspace_size(int d) {
  if (d < 1 || d > kNormMaxBytes / 2) return 0;
  return kWsHeader + static_cast<size_t>(kNormMaxBlocks) * 2 * d * sizeof(float);
}

int ps_residual_norm_bwd(int64_t N, int d, int dtype, int norms, const void* dout, int64_t lddo, const void* dh, int64_t lddh,
                         const void* h, int64_t ldh, const void* y, int64_t ldy, const void* gy, const void* go,
                         const float* gate, double res_scale, double branch_scale, double eps, void* dx, int64_t lddx, void* dy,
                         int64_t lddy, float* dgy, float* dgo, float* dgate, int flags, void* ws, size_t ws_bytes,
                         ps_stream_t stream) {
  NvtxRange nvtx_range("ps_residual_norm_bwd");
  if (!norm_sizes_ok(N, d, dtype, norms, res_scale, branch_scale, eps) || (flags & ~PS_DW_ACCUMULATE)) return PS_ERR_INVALID_ARG;
  const bool out = norms & PS_NORM_OUT;
  if (N > 0 && ((!y && ((norms & PS_NORM_BRANCH) || gate || dgy || !out)) || (dgate && !gate))) return PS_ERR_INVALID_ARG;
  if (dgo && !out) return PS_ERR_INVALID_ARG;
  const bool gains = dgy || dgo;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  auto aligned4 = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; };
  if (!aligned4(gate) || !aligned4(dgate) || !aligned4(dgy) || !aligned4(dgo)) return PS_ERR_INVALID_ARG;
  NormRows r(N, d, dtype);
  if (N > 0) {
    if (!out && !dh) return PS_ERR_INVALID_ARG;   // no gradient comes in
    r.rows(dx, lddx, 4);
    if (out) {
      r.rows(dout, lddo, 2);
      r.rows(h, ldh, 0);
      r.gains(go);
    }
    if (dh) r.rows(dh, lddh, 3);
    if (y) {
      r.rows(y, ldy, 1);
      r.rows(dy, lddy, 5);
      r.gains(gy);
    }
    if (!r.ok) return PS_ERR_INVALID_ARG;
  }
  int rc = check_ws(ws, ws_bytes, gains ? ps_residual_norm_workspace_size(d) : kWsHeader);
  if (rc != PS_OK) return rc;
  if (N == 0) {
    refused(PS_OK, ws, s);
    for (float* g : {dgy, dgo})
      if (g && !(flags & PS_DW_ACCUMULATE) && cudaMemsetAsync(g, 0, sizeof(float) * d, s) != cudaSuccess) return PS_ERR_CUDA;
    return PS_OK;
  }
  NormArgs a = {};
  a.N = N, a.d = d;
  a.in[0] = out ? h : nullptr, a.in[1] = y, a.in[2] = out ? dout : nullptr, a.in[3] = dh;
  a.ld[0] = ldh, a.ld[1] = ldy, a.ld[2] = lddo, a.ld[3] = lddh;
  a.gy = gy, a.go = go, a.gate = gate;
  a.post = (norms & PS_NORM_BRANCH) ? 1 : 0, a.pre = out ? 1 : 0;
  // without a branch the stream is x itself, whatever the scales
  r.into(a);
  a.a = y ? static_cast<float>(res_scale) : 1.f, a.b = static_cast<float>(branch_scale), a.eps = static_cast<float>(eps);
  a.out0 = dx, a.out1 = dy, a.ldo0 = lddx, a.ldo1 = lddy;
  a.dgate = dgate;
  a.status = static_cast<uint32_t*>(ws);
  a.part = gains ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kWsHeader) : nullptr;
  int grid = 0;
  rc = dtype == PS_DTYPE_F32 ? run_norm<float, true>(a, !r.whole, grid, s) : run_norm<Bf16, true>(a, !r.whole, grid, s);
  if (rc != PS_OK) return refused(rc, ws, s);
  if (!gains) return PS_OK;
  return launch_after(norm_gain_sum_kernel, dim3(static_cast<unsigned>((2 * d + 31) / 32)), 256, 0, s, 1, 1, true, d, grid, a.part,
                      dgy, dgo, (flags & PS_DW_ACCUMULATE) ? 1 : 0) == cudaSuccess
             ? PS_OK
             : PS_ERR_CUDA;
}

}  // extern "C"
