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
//   dgo = sum do h r_h, dy = r_y (gy dn - y r_y^2 mean(gy dn y)), dgate = b sum dH n = b r_y sum gy dH y: the
//   row's sums are two rounds, three sums (h^2, go do h, y^2) and then one (gy dH y), which dy's mean and dgate share.
// HBM-bound: each input is read once and each output written once. A row lies on a team of threads (part of a warp, a
// warp, or some), CH chunks of eight values each, the same columns of every row, so that the gains' gradients stay in its
// registers over all rows. Rows come through a ring in shared memory that a thread's own copies fill ST rows ahead: what a
// thread reads is what it copied, so only the sums cross threads.
constexpr int kNormThreads = 512;   // at most
__host__ __device__ constexpr int norm_arrays(bool bwd) { return bwd ? 4 : 2; }   // h, y, do, dh; x, y
// Rows ahead: as many as lie in shared memory beside what the registers allow of threads.
__host__ __device__ constexpr int norm_stages(int e, int ch, bool bwd, bool vec) { return !vec ? 1 : ch * e <= 4 ? 3 : bwd ? 1 : 2; }

struct NormArgs {
  int64_t N;
  int d, chunks;                  // chunks of eight columns
  int team, teams;                // threads per row, and teams of a block
  const void *in[4];              // forward: x, y; backward: h, y, do, dh (nullptr: absent)
  int64_t ld[4];
  const void *gy, *go;            // gains [d], nullptr: 1
  const float* gate;              // [N], nullptr: 1
  int post, pre;                  // a norm of the branch; a normed output (or its gradient)
  float a, b, eps, inv_d;
  void *out0, *out1;              // forward: h, o; backward: dx, dy
  int64_t ldo0, ldo1;
  float* dgate;
  uint32_t* status;
  float* part;                    // backward: [blocks][2][d] partial gain gradients (dgy, dgo), nullptr without
};

template <class T, int CH, bool BWD, bool VEC>
__global__ void __launch_bounds__(kNormThreads, BWD ? 1 : 2) norm_kernel(const NormArgs a) {
  constexpr int A = norm_arrays(BWD), ST = norm_stages(sizeof(T), CH, BWD, VEC);
  constexpr int P = VEC ? sizeof(T) / 2 : 1;      // 16-byte pieces of a chunk
  extern __shared__ __align__(128) uint8_t norm_smem[];
  __shared__ float4 red[2][kNormThreads / 32];
  const int threads = blockDim.x, tid = threadIdx.x;
  const int unit_threads = a.team > 32 ? a.team : 32;             // what goes through the rows together
  const int unit_in = tid / unit_threads, units_here = threads / unit_threads;
  const int t = tid % a.team, sub = a.team < 32 ? (tid & 31) / a.team : 0;
  const int rows_a_unit = a.team < 32 ? 32 / a.team : 1;
  const int64_t units = (a.N + rows_a_unit - 1) / rows_a_unit, stride = static_cast<int64_t>(gridDim.x) * units_here;
  int parity = 0;

  // the sums of K values over a team, the same bits in each of its threads
  auto team_sum = [&](auto& v) {
    constexpr int K = sizeof(v) / sizeof(float);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1)
      if (a.team > o)
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (a.team > 32) {
      const int w0 = unit_in * (a.team / 32);
      if ((tid & 31) == 0) red[parity][tid >> 5] = make_float4(v[0], K > 1 ? v[K > 1 ? 1 : 0] : 0.f, K > 2 ? v[K > 2 ? 2 : 0] : 0.f, 0.f);
      asm volatile("bar.sync %0, %1;" ::"r"(unit_in + 1), "r"(a.team) : "memory");
      float s[3] = {0.f, 0.f, 0.f};
      for (int w = 0; w < a.team / 32; ++w) {
        const float4 r = red[parity][w0 + w];
        s[0] += r.x, s[1] += r.y, s[2] += r.z;
      }
#pragma unroll
      for (int i = 0; i < K; ++i) v[i] = s[i];
      parity ^= 1;   // (the next sum's barrier lies between this one's reads and the sum after it)
    }
  };

  auto slot = [&](int st, int arr, int j, int p) {   // VEC: this thread's piece
    return norm_smem + ((((st * A + arr) * CH + j) * P + p) * threads + tid) * 16;
  };
  auto cell = [&](int arr, int e) {                  // else: its element e = 8 j + i of the row
    return reinterpret_cast<T*>(norm_smem) + (arr * CH * 8 + e) * threads + tid;
  };
  auto column = [&](int j, int i) { return VEC ? (j * a.team + t) * 8 + i : (j * 8 + i) * a.team + t; };
  auto in_chunk = [&](int j) { return VEC ? j * a.team + t < a.chunks : true; };
  // the copies of a unit's row into a stage; a group for each, be it empty
  auto issue = [&](int64_t u, int st) {
    const int64_t row = u * rows_a_unit + sub;
    if (VEC) {
      if (u < units && row < a.N) {
#pragma unroll
        for (int arr = 0; arr < A; ++arr) {
          if (!a.in[arr]) continue;
          const T* from = static_cast<const T*>(a.in[arr]) + row * a.ld[arr];
#pragma unroll
          for (int j = 0; j < CH; ++j) {
            if (!in_chunk(j)) continue;
#pragma unroll
            for (int p = 0; p < P; ++p) lane_copy(smem_addr(slot(st, arr, j, p)), from + column(j, 0) + p * (16 / sizeof(T)));
          }
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  };
  auto arrive = [&](int64_t row, bool live) {
    if (VEC) {
      asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
    } else if (live) {
      T v[A][CH * 8];
#pragma unroll
      for (int arr = 0; arr < A; ++arr) {
        const T* from = static_cast<const T*>(a.in[arr]) + row * a.ld[arr];
#pragma unroll
        for (int e = 0; e < CH * 8; ++e)
          if (a.in[arr] && e * a.team + t < a.d) v[arr][e] = from[e * a.team + t];
      }
#pragma unroll
      for (int arr = 0; arr < A; ++arr)
#pragma unroll
        for (int e = 0; e < CH * 8; ++e)
          if (a.in[arr] && e * a.team + t < a.d) *cell(arr, e) = v[arr][e];
    }
  };
  // eight values of an array's row, zeros where there is none
  auto get = [&](int st, int arr, int j, bool live, float (&f)[8]) {
    if (VEC) {
      if (live && a.in[arr] && in_chunk(j)) {
        if (sizeof(T) == 2) {
          Raw8<Bf16> r;
          r.load(reinterpret_cast<const Bf16*>(slot(st, arr, j, 0)));
          r.get(f);
        } else {
          const float4 u = *reinterpret_cast<const float4*>(slot(st, arr, j, 0));
          const float4 v = *reinterpret_cast<const float4*>(slot(st, arr, j, P - 1));
          f[0] = u.x, f[1] = u.y, f[2] = u.z, f[3] = u.w;
          f[4] = v.x, f[5] = v.y, f[6] = v.z, f[7] = v.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = live && a.in[arr] && column(j, i) < a.d ? Elem<T>::get(*cell(arr, j * 8 + i)) : 0.f;
    }
  };
  auto gains = [&](const void* g, int j, float (&f)[8]) {
    const T* from = static_cast<const T*>(g);
    if (VEC && g && in_chunk(j)) {
      Raw8<T> r;
      r.load(from + column(j, 0));
      r.get(f);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = !VEC && g && column(j, i) < a.d ? Elem<T>::get(from[column(j, i)]) : 1.f;
    }
  };
  auto put = [&](void* base, int64_t ld, int64_t row, int j, const float (&f)[8]) {
    T* to = static_cast<T*>(base) + row * ld;
    if (VEC) {
      if (in_chunk(j)) Raw8<T>::store(to + column(j, 0), f);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (column(j, i) < a.d) to[column(j, i)] = Elem<T>::put(f[i]);
    }
  };

  float accy[BWD ? CH : 1][8], acco[BWD ? CH : 1][8];
  if (BWD)
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) accy[j][i] = acco[j][i] = 0.f;

  wait_for_previous_kernel();
  let_next_kernel_in();
  if (BWD && a.status && blockIdx.x == 0 && tid == 0) clear_status(a.status);
  const int64_t u0 = static_cast<int64_t>(blockIdx.x) * units_here + unit_in;
#pragma unroll
  for (int s = 0; s < ST; ++s) issue(u0 + s * stride, s);
  int st = 0;
  for (int64_t u = u0; u < units; u += stride) {
    const int64_t row = u * rows_a_unit + sub;
    const bool live = row < a.N;
    const float gate = live && a.gate ? __ldg(a.gate + row) : 1.f;
    const bool open = live && a.in[1] && gate != 0.f;   // (a closed gate leaves the branch out whatever it holds)
    arrive(row, live);
    if (!BWD) {
      float ry = 1.f;
      if (a.post) {
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          float y[8];
          get(st, 1, j, live, y);
#pragma unroll
          for (int i = 0; i < 8; ++i) s[0] = fmaf(y[i], y[i], s[0]);
        }
        team_sum(s);
        ry = rsqrtf(fmaf(s[0], a.inv_d, a.eps));
      }
      const float w = a.b * gate * ry;
      float h[CH][8], s[1] = {0.f};
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        get(st, 0, j, live, h[j]);
        if (a.in[1]) {
          float y[8], g[8];
          get(st, 1, j, open, y);
          gains(a.gy, j, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) h[j][i] = fmaf(a.a, h[j][i], open ? w * (y[i] * g[i]) : 0.f);
          if (live) put(a.out0, a.ldo0, row, j, h[j]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fmaf(h[j][i], h[j][i], s[0]);
      }
      if (a.pre) {
        team_sum(s);
        const float rh = rsqrtf(fmaf(s[0], a.inv_d, a.eps));
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          float g[8];
          gains(a.go, j, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) g[i] *= h[j][i] * rh;
          if (live) put(a.out1, a.ldo1, row, j, g);
        }
      }
    } else {
      float s[3] = {0.f, 0.f, 0.f};
      if (a.pre || a.post) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          float h[8], y[8], q[8], g[8];
          get(st, 0, j, live, h);
          get(st, 1, j, live, y);
          get(st, 2, j, live, q);
          gains(a.go, j, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            s[0] = fmaf(h[i], h[i], s[0]);
            s[1] = fmaf(g[i] * q[i], h[i], s[1]);
            s[2] = fmaf(y[i], y[i], s[2]);
          }
        }
        team_sum(s);
      }
      const float rh = a.pre ? rsqrtf(fmaf(s[0], a.inv_d, a.eps)) : 0.f, m = s[1] * a.inv_d * rh * rh;
      const float ry = a.post ? rsqrtf(fmaf(s[2], a.inv_d, a.eps)) : 1.f;
      float dH[CH][8], dot[1] = {0.f};
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        get(st, 3, j, live, dH[j]);
        if (a.pre) {
          float h[8], q[8], g[8];
          get(st, 0, j, live, h);
          get(st, 2, j, live, q);
          gains(a.go, j, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dH[j][i] = fmaf(rh, fmaf(h[i], -m, g[i] * q[i]), dH[j][i]);
            acco[j][i] += live ? q[i] * (h[i] * rh) : 0.f;
          }
        }
        if (a.dgate || a.post) {
          float y[8], g[8];
          get(st, 1, j, live, y);
          gains(a.gy, j, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) dot[0] = fmaf(g[i] * dH[j][i], y[i], dot[0]);
        }
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = a.a * dH[j][i];
        if (live) put(a.out0, a.ldo0, row, j, v);
      }
      if (a.in[1]) {
        if (a.dgate || a.post) team_sum(dot);
        if (a.dgate && live && t == 0) a.dgate[row] = a.b * ry * dot[0];
        const float w = a.b * gate * ry, k = a.post ? dot[0] * a.inv_d * ry * ry : 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          float y[8], g[8];
          get(st, 1, j, open, y);
          gains(a.gy, j, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            accy[j][i] += open ? w * dH[j][i] * y[i] : 0.f;
            y[i] = open ? w * fmaf(y[i], -k, g[i] * dH[j][i]) : 0.f;
          }
          if (live) put(a.out1, a.ldo1, row, j, y);
        }
      }
    }
    issue(u + ST * stride, st);   // (the stage has been read: its values went into what was stored)
    st = st + 1 == ST ? 0 : st + 1;
  }
  if (!BWD || a.part == nullptr) return;

  // gain gradients: over a warp's rows, then the block's units in order; norm_gain_sum_kernel adds the blocks'
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  float* mine = reinterpret_cast<float*>(norm_smem) + static_cast<size_t>(unit_in) * 2 * a.d;
#pragma unroll
  for (int j = 0; j < CH; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v = accy[BWD ? j : 0][i], w = acco[BWD ? j : 0][i];
      for (int o = 16; o >= a.team; o >>= 1) {
        v += __shfl_xor_sync(0xffffffffu, v, o);
        w += __shfl_xor_sync(0xffffffffu, w, o);
      }
      const int c = column(j, i);
      if (sub == 0 && c < a.d) {
        mine[c] = v;
        mine[a.d + c] = w;
      }
    }
  __syncthreads();
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.d;
  for (int c = tid; c < 2 * a.d; c += threads) {
    float v = 0.f;
    for (int k = 0; k < units_here; ++k) v += reinterpret_cast<const float*>(norm_smem)[static_cast<size_t>(k) * 2 * a.d + c];
    part[c] = v;
  }
}

// The blocks' partial gain gradients [blocks][2][d], eight columns a block: a thread adds every 32nd block's, the shares are
// added in order, all in f64, so that reruns give the same bits.
__global__ void __launch_bounds__(256) norm_gain_sum_kernel(int d, int blocks, const float* __restrict__ part, float* dgy,
                                                            float* dgo, int accumulate) {
  __shared__ double sums[32][8];
  wait_for_previous_kernel();
  const int j = threadIdx.x & 7, share = threadIdx.x >> 3, col = blockIdx.x * 8 + j;
  double t = 0.0;
  if (col < 2 * d)
#pragma unroll 8
    for (int b = share; b < blocks; b += 32) t += static_cast<double>(part[static_cast<int64_t>(b) * 2 * d + col]);
  sums[share][j] = t;
  __syncthreads();
  if (share != 0 || col >= 2 * d) return;
  t = 0.0;
  for (int k = 0; k < 32; ++k) t += sums[k][j];
  float* out = col < d ? dgy : dgo;
  if (!out) return;
  float& o = out[col < d ? col : col - d];
  o = static_cast<float>(accumulate ? t + o : t);
}

// ================================================================== host side
constexpr int kNormMaxBytes = 32768;        // of a row: bf16 16384 columns, f32 8192
constexpr size_t kSmemOfSm = 227 * 1024;
constexpr int64_t kNormMaxBlocks = 304;    // of a backward at most; its workspace holds a partial sum of each

struct NormPlan {
  int ch, team, teams, threads, blocks_a_sm;
  size_t smem;
};
// Threads of 32 bytes of a row each, up to 512 to a row, then more bytes each.
static NormPlan norm_plan(int d, int e, bool bwd, bool vec) {
  NormPlan p;
  const int chunks = (d + 7) / 8, unit = 32 / (8 * e) > 0 ? 32 / (8 * e) : 1;   // bf16 2, f32 1
  p.ch = chunks <= 32 ? 1 : unit;
  while ((chunks + p.ch - 1) / p.ch > kNormThreads) p.ch *= 2;
  const int need = (chunks + p.ch - 1) / p.ch;
  if (need <= 32) {
    p.team = 1;
    while (p.team < need) p.team *= 2;
  } else {
    p.team = (need + 31) / 32 * 32;
  }
  const int unit_threads = p.team > 32 ? p.team : 32;
  p.teams = 256 / unit_threads > 1 ? 256 / unit_threads : 1;
  p.threads = p.teams * unit_threads;
  p.smem = static_cast<size_t>(norm_stages(e, p.ch, bwd, vec)) * norm_arrays(bwd) * p.ch * 8 * e * p.threads;
  const size_t sums = bwd ? static_cast<size_t>(p.teams) * 2 * d * sizeof(float) : 0;
  if (p.smem < sums) p.smem = sums;
  p.blocks_a_sm = (bwd ? 512 : 1024) / p.threads;
  const int fit = static_cast<int>(kSmemOfSm / (p.smem + 2048));
  if (p.blocks_a_sm > fit) p.blocks_a_sm = fit;
  if (p.blocks_a_sm < 1) p.blocks_a_sm = 1;
  return p;
}

template <class T, int CH, bool BWD, bool VEC>
static int launch_norm(NormArgs& a, const NormPlan& p, int& grid, cudaStream_t s) {
  auto kern = norm_kernel<T, CH, BWD, VEC>;
  if (p.smem > 40 * 1024 &&   // (beside the block's own)
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(p.smem)) != cudaSuccess)
    return PS_ERR_CUDA;
  const int rows_a_unit = a.team < 32 ? 32 / a.team : 1;
  const int64_t units = (a.N + rows_a_unit - 1) / rows_a_unit, want = (units + p.teams - 1) / p.teams;
  int64_t most = static_cast<int64_t>(num_sms_current()) * p.blocks_a_sm;
  if (BWD && most > kNormMaxBlocks) most = kNormMaxBlocks;
  grid = static_cast<int>(want < most ? want : most);
  return launch_after(kern, dim3(static_cast<unsigned>(grid)), static_cast<unsigned>(p.threads), p.smem, s, 1, 1, true, a) ==
                 cudaSuccess
             ? PS_OK
             : PS_ERR_CUDA;
}
template <class T, bool BWD>
static int run_norm(NormArgs a, bool vec, int& grid, cudaStream_t s) {
  const NormPlan p = norm_plan(a.d, sizeof(T), BWD, vec);
  a.chunks = (a.d + 7) / 8, a.team = p.team, a.teams = p.teams;
  a.inv_d = 1.f / static_cast<float>(a.d);
  switch (p.ch) {
    case 1: return vec ? launch_norm<T, 1, BWD, true>(a, p, grid, s) : launch_norm<T, 1, BWD, false>(a, p, grid, s);
    case 2: return vec ? launch_norm<T, 2, BWD, true>(a, p, grid, s) : launch_norm<T, 2, BWD, false>(a, p, grid, s);
    default: break;
  }
  if constexpr (sizeof(T) == 2)   // (f32 rows of 8192 columns take two chunks)
    return vec ? launch_norm<T, 4, BWD, true>(a, p, grid, s) : launch_norm<T, 4, BWD, false>(a, p, grid, s);
  return PS_ERR_UNSUPPORTED;
}

}  // namespace psk

using namespace psk;

namespace {

bool norm_sizes_ok(int64_t N, int d, int dtype, int norms, double a, double b, double eps) {
  return N >= 0 && d >= 1 && (dtype == PS_DTYPE_BF16 || dtype == PS_DTYPE_F32) && d <= kNormMaxBytes / elem_bytes(dtype) &&
         !(norms & ~(PS_NORM_BRANCH | PS_NORM_OUT)) && isfinite(a) && isfinite(b) && eps >= 0.0 && isfinite(eps);
}
struct NormRows {   // the tensors of a call: placed on their elements, and all rows on 16-byte boundaries or not
  int e, d;
  bool ok = true, vec;
  NormRows(int d_, int dtype) : e(elem_bytes(dtype)), d(d_), vec(d_ % 8 == 0) {}
  void rows(const void* p, int64_t ld) {
    ok = ok && p && ld >= d && reinterpret_cast<uintptr_t>(p) % e == 0;
    vec = vec && al16(p) && ld * e % 16 == 0;
  }
  void gains(const void* p) {
    ok = ok && reinterpret_cast<uintptr_t>(p) % e == 0;
    vec = vec && al16(p);
  }
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
  NormRows r(d, dtype);
  r.rows(x, ldx);
  if (y) {
    r.rows(y, ldy);
    r.rows(h, ldh);
    r.gains(gy);
  }
  if (out) {
    r.rows(o, ldo);
    r.gains(go);
  }
  if (!r.ok || reinterpret_cast<uintptr_t>(gate) % 4) return PS_ERR_INVALID_ARG;
  NormArgs a = {};
  a.N = N, a.d = d;
  a.in[0] = x, a.in[1] = y, a.ld[0] = ldx, a.ld[1] = ldy;
  a.gy = gy, a.go = go, a.gate = gate;
  a.post = (norms & PS_NORM_BRANCH) ? 1 : 0, a.pre = out ? 1 : 0;
  a.a = static_cast<float>(res_scale), a.b = static_cast<float>(branch_scale), a.eps = static_cast<float>(eps);
  a.out0 = h, a.out1 = o, a.ldo0 = ldh, a.ldo1 = ldo;
  int grid;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return dtype == PS_DTYPE_F32 ? run_norm<float, false>(a, r.vec, grid, s) : run_norm<Bf16, false>(a, r.vec, grid, s);
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
  NormRows r(d, dtype);
  if (N > 0) {
    if (!out && !dh) return PS_ERR_INVALID_ARG;   // no gradient comes in
    r.rows(dx, lddx);
    if (out) {
      r.rows(dout, lddo);
      r.rows(h, ldh);
      r.gains(go);
    }
    if (dh) r.rows(dh, lddh);
    if (y) {
      r.rows(y, ldy);
      r.rows(dy, lddy);
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
  a.a = y ? static_cast<float>(res_scale) : 1.f, a.b = static_cast<float>(branch_scale), a.eps = static_cast<float>(eps);
  a.out0 = dx, a.out1 = dy, a.ldo0 = lddx, a.ldo1 = lddy;
  a.dgate = dgate;
  a.status = static_cast<uint32_t*>(ws);
  a.part = gains ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kWsHeader) : nullptr;
  int grid = 0;
  rc = dtype == PS_DTYPE_F32 ? run_norm<float, true>(a, r.vec, grid, s) : run_norm<Bf16, true>(a, r.vec, grid, s);
  if (rc != PS_OK) return refused(rc, ws, s);
  if (!gains) return PS_OK;
  return launch_after(norm_gain_sum_kernel, dim3(static_cast<unsigned>((2 * d + 7) / 8)), 256, 0, s, 1, 1, true, d, grid, a.part,
                      dgy, dgo, (flags & PS_DW_ACCUMULATE) ? 1 : 0) == cudaSuccess
             ? PS_OK
             : PS_ERR_CUDA;
}

}  // extern "C"
