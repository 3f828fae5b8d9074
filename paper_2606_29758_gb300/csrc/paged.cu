// A paged cache of keys and values in sampling: new tokens' rows written into their pages, and attention of one new token
// a sequence over the pages, split over all keys and joined.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <climits>
#include <type_traits>

#include "internal.h"
#include "ps_common.cuh"
#include "ps_nvtx.h"
#include "row_elems.cuh"
#include "umma_host.cuh"

namespace psk {

// The cache of one layer: keys and values [pages][Hk][page][D]; the table [seqs][ldt] names the pages of a sequence in order.
struct PagesOf {
  const int32_t* table;
  int64_t ldt;                // pages a row of the table holds
  int pages, page_log2, page;
  int Hk, D;
};

// ================================================================== append
struct AppendArgs {
  int64_t N;
  PagesOf c;
  int seqs;
  const void *k, *v;
  int64_t ldk, ldv;
  const int32_t *seq, *pos;
  int pos_base;
  void *kc, *vc;
  int pieces, head_pieces;    // 16-byte pieces of a row, of a head
  int parts;                  // warps that share a row
  int checked;                // the first block looks at every row and writes the status alone
  uint32_t* status;
};
constexpr int kAppendThreads = 128;
// Up to so many rows the first block looks at all of them and writes the status; beyond, the status is cleared by an operation of its
// own before (512 rows of 4 heads of 128: 3.4 against 6.2 us, 2000 rows: 8.1 against 6.2).
constexpr int kAppendCheckRows = 1024;

// Where row i goes, or what is wrong with it: 0 and its page and slot, -1 for a row without a sequence, else status bits.
static __device__ __forceinline__ int append_place(const AppendArgs& a, int64_t row, int& page_id, int& in_page) {
  const int seq = __ldg(a.seq + row);
  if (seq == -1) return -1;
  const int64_t p = static_cast<int64_t>(__ldg(a.pos + row)) - a.pos_base;
  if (seq < 0 || seq >= a.seqs || p < 0 || (p >> a.c.page_log2) >= a.c.ldt) return PS_DEV_BAD_LENGTH;
  page_id = __ldg(a.c.table + seq * a.c.ldt + (p >> a.c.page_log2));
  in_page = static_cast<int>(p & (a.c.page - 1));
  return page_id < 0 || page_id >= a.c.pages ? PS_DEV_BAD_PAGE : 0;
}

// Each row is read once and written once: HBM, or the latency of three dependent loads (sequence and position, page, row). A warp
// a row, or several where there are few; its 64 pieces of 16 bytes are under way while its place is looked up. (72600 rows of 4
// heads of 128 bf16: 52 us, 5.8 TB/s; 128 rows: 2.6 us, of which a launch is 2.)
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t units = a.N * a.parts, stride = static_cast<int64_t>(gridDim.x) * (kAppendThreads / 32);
  wait_for_previous_kernel();
  let_next_kernel_in();
  if (a.checked && blockIdx.x == 0) {
    int bad = 0, id, at;
    for (int i = threadIdx.x; i < static_cast<int>(a.N); i += kAppendThreads) bad |= max(0, append_place(a, i, id, at));
    const int len = __syncthreads_or(bad & PS_DEV_BAD_LENGTH), page = __syncthreads_or(bad & PS_DEV_BAD_PAGE);
    if (threadIdx.x == 0) {
      a.status[1] = 0u;
      a.status[0] = (len ? PS_DEV_BAD_LENGTH : 0) | (page ? PS_DEV_BAD_PAGE : 0);
    }
  }
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kAppendThreads / 32) + (threadIdx.x >> 5); u < units; u += stride) {
    const int64_t row = a.parts == 1 ? u : u / a.parts;
    const int part = static_cast<int>(u - row * a.parts);
    const uint4* ks = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.k) + row * a.ldk);
    const uint4* vs = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.v) + row * a.ldv);
    const int p1 = static_cast<int>(static_cast<int64_t>(a.pieces) * (part + 1) / a.parts);
    int p0 = static_cast<int>(static_cast<int64_t>(a.pieces) * part / a.parts);
    uint4 kv[2], vv[2];
    auto read = [&]() {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int p = p0 + h * 32 + lane;
        if (p < p1) kv[h] = __ldg(ks + p), vv[h] = __ldg(vs + p);
      }
    };
    read();   // (the row is on its way while its place is looked up)
    int id = 0, slot = 0;
    const int bad = append_place(a, row, id, slot);
    if (bad) {
      if (bad > 0 && !a.checked && lane == 0) raise_status(a.status, bad);
      continue;
    }
    const int64_t first = static_cast<int64_t>(id) * a.c.Hk;
    while (true) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int p = p0 + h * 32 + lane;
        if (p >= p1) continue;
        const int head = p / a.head_pieces;
        const int64_t to = (((first + head) << a.c.page_log2) + slot) * a.head_pieces + (p - head * a.head_pieces);
        static_cast<uint4*>(a.kc)[to] = kv[h];
        static_cast<uint4*>(a.vc)[to] = vv[h];
      }
      p0 += 64;
      if (p0 >= p1) break;
      read();
    }
  }
}

// ================================================================== decode
//   x_j = c q.k_j (c = scale log2 e) over a sequence's keys j, m = max x_j, l = sum 2^(x_j - m), o = sum 2^(x_j - m) v_j / l;
//   parts of a sequence join by m = max m_i, l = sum l_i 2^(m_i - m), o likewise.
// HBM-bound: every key and value is read once for the query heads of a unit, which share it: up to 16 of a key head, in f32 and above
// 128 dims up to 8 (a key head with more has several units, each of which reads its keys: 32 on one key head, 64 sequences of 2300 keys
// of 128, bf16 38 us where its bytes take 11, f32 128 and 22). The work is a list of tiles of 64 keys of a unit; each CTA takes an
// equal run of the list, whatever the lengths are. Its four warps take 16 keys of a tile each, through rings of their own in shared
// memory that their lanes' copies fill some tiles ahead, across units; within a unit nothing crosses warps. What a CTA has of a unit that it does not hold whole goes to the workspace (two slots a CTA), and decode_join_kernel adds those up.
// bf16: products by mma.sync with the keys (S^T = K Q^T, 16 keys x 8 heads) and the values' dims (O^T = V^T P^T, 16 dims x 8
// heads) as rows, so that eight heads fill a product's columns; P in three bf16 parts, which hold all 24 bits of a weight, and a
// chunk's products in a sum of their own that an f32 addition joins to o, as the tensor cores cut what they add to a large
// sum off at its last bit instead of rounding it. (Two parts, 2^-17 of a weight, and sums by the tensor cores over all chunks left
// 0.15 to 0.34 % of the outputs at another bf16 than the nearest, f32 sums of the plain form 0.04 to 0.13 %, these 0.02 to 0.06 %; 128
// sequences of 12400 keys 482 -> 489 us, one of 16384 keys 13.6 -> 14.5.) The rows of tcgen05 products would be 64 or more of one
// operand in shared memory and accumulators in TMEM, whose round trips a chunk of 16 keys would wait for, and these
// products are a few per cent of what mma.sync does. More than eight heads a key head: sixteen a unit (16 on one key head, 128
// sequences of 12400 keys 139 us, eight a unit 251; 64 of 2300 27.5 and 26.2, 16 of 1000 11.5 and 10.2; 7 heads, 64 of 2300 55.4 and 57.6).
// 128 sequences of about 2300 keys, 28 / 4 heads of 128: 103 us, 5.9 TB/s; of 12400 keys 489 us, 6.7 TB/s; one of 16384 keys 14.5
// us, of which the two launches, the lists and the join are 10: latency. 256 sequences of 3 to 16 keys 14.5 us, f32 22 to 24: a chunk's
// work for one warp of four, then the unit's join, in turn.
constexpr int kDecWarps = 4;
constexpr int kDecThreads = 32 * kDecWarps;
constexpr int kChunk = 16;                        // keys of a warp's share of a tile
constexpr int kTile = kChunk * kDecWarps;
constexpr int kBoxBytes = kChunk * 128;

struct DecodeArgs {
  int B, Hq, group, blocks;     // sequences, query heads, query heads a key head, units a key head
  PagesOf c;
  const int32_t* lens;
  int window;                   // 0: all keys
  float scale2;                 // scale log2 e
  const void* q;
  int64_t ldq;
  const void *kc, *vc;
  void* o;
  int64_t ldo;
  float* lse;                   // [B][Hq] or nullptr
  uint32_t* status;
  int4* seg;                    // [CTAs] status bits, the unit that begins here and goes on (sequence or -1, block), the CTA where it ends
  int2* unit;                   // [units] the CTAs where it begins and ends (-1: in one, or nothing of it), nullptr: by seg
  float2* ml;                   // [2 CTAs][heads of a unit] (m, l)
  float* part;                  // [2 CTAs][heads of a unit][DP]
};

static __device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
static __device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
static __device__ __forceinline__ uint32_t transposed(uint32_t x) {   // an 8 x 8 matrix of 16-bit elements over the warp
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
static __device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// A product of its own: c = a b.
static __device__ __forceinline__ void mma_bf16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// 16 bytes global -> shared, or zeros.
static __device__ __forceinline__ void lane_copy_or_zero(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}

// A warp's part of a unit: m, l and o of its query heads over the keys that it has seen.
//   load    the unit's queries
//   chunk   keys and values lo to nv of 16 in shared memory (the others' values are zeros). bf16: boxes of 64 dims, 128 bytes a
//           row, 16-byte piece p of row r at p ^ (r & 7) (TMA's 128-byte swizzle); f32: whole rows, pieces likewise
//   put_ml  m and l to shared memory
//   add_o   o times a head's factor, to or added to what shared memory [heads][DP + 4] holds
template <class T, int DP, int NB>
struct DecodeMath;

template <int DP, int NB>
struct DecodeMath<Bf16, DP, NB> {
  static constexpr int kHeads = 8 * NB;
  uint32_t q[NB][DP / 16][2];
  float o[NB][DP / 16][4];      // o[dim lane / 4 (+ 8)][head 2 (lane % 4) (+ 1)]
  float m[NB][2], l[NB][2];     // of heads 2 (lane % 4) and the next; l of this lane's keys

  __device__ __forceinline__ void load(const Bf16* qs, int heads, int D, int lane) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int head = n * 8 + lane / 4;
#pragma unroll
      for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = k * 16 + i * 8 + 2 * (lane & 3);
          q[n][k][i] = head < heads && at < D ? *reinterpret_cast<const uint32_t*>(qs + head * D + at) : 0u;
        }
#pragma unroll
      for (int t = 0; t < DP / 16; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][t][i] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
    }
  }
  __device__ __forceinline__ void poison() {
#pragma unroll
    for (int n = 0; n < NB; ++n) l[n][0] = l[n][1] = __int_as_float(0x7fffffff);
  }
  __device__ __forceinline__ void chunk(uint32_t ks, uint32_t vs, int lo, int nv, float scale2, float*, int lane) {
    const int r = lane & 15, hi = lane >> 4;
    float s[NB][4];
#pragma unroll
    for (int n = 0; n < NB; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
    // rows: keys 0-7 and 8-15 by the lanes' first 16 addresses, then the next eight dims
    const uint32_t ka = ks + r * 128 + ((hi ^ (r & 7)) << 4);
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
      uint32_t a[4];
      ldsm4(a, (ka ^ ((k & 3) * 32)) + (k >> 2) * kBoxBytes);
#pragma unroll
      for (int n = 0; n < NB; ++n) mma_bf16(s[n], a, q[n][k][0], q[n][k][1]);
    }
    const int key = lane / 4;
    uint32_t w[3][NB][2];   // the weights' parts, the largest last
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      float x[4], top[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = key + (i & 2 ? 8 : 0);
        x[i] = at >= lo && at < nv ? s[n][i] * scale2 : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float v = fmaxf(x[i], x[i + 2]);
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
        top[i] = fmaxf(m[n][i], v);
      }
      if (__any_sync(0xffffffffu, top[0] != m[n][0] || top[1] != m[n][1])) {
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f[i] = m[n][i] == top[i] ? 1.f : ex2_ftz(m[n][i] - top[i]);
          m[n][i] = top[i];
          l[n][i] *= f[i];
        }
#pragma unroll
        for (int t = 0; t < DP / 16; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][t][i] *= f[i & 1];
      }
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = ex2_ftz(x[i] - (m[n][i & 1] == -INFINITY ? 0.f : m[n][i & 1]));
        l[n][i & 1] += p[i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float u = p[2 * i], v = p[2 * i + 1];
#pragma unroll
        for (int k = 2; k >= 0; --k) {
          const uint32_t part = pack_bf16x2(u, v);
          u -= __uint_as_float(part << 16);
          v -= __uint_as_float(part & 0xffff0000u);
          w[k][n][i] = transposed(part);
        }
      }
    }
    const int row = (lane & 7) + (hi << 3);
    const uint32_t va = vs + row * 128 + ((((lane >> 3) & 1) ^ (row & 7)) << 4);
#pragma unroll
    for (int t = 0; t < DP / 16; ++t) {
      uint32_t a[4];   // dims 0-7 and 8-15 of keys 0-7, then of keys 8-15
      ldsm4_t(a, (va ^ ((t & 3) * 32)) + (t >> 2) * kBoxBytes);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float c[4];
        mma_bf16_first(c, a, w[0][n][0], w[0][n][1]);
        mma_bf16(c, a, w[1][n][0], w[1][n][1]);
        mma_bf16(c, a, w[2][n][0], w[2][n][1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][t][i] += c[i];
      }
    }
  }
  __device__ __forceinline__ void put_ml(float2* ml, int lane) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float v = l[n][i];
        v += __shfl_xor_sync(0xffffffffu, v, 4);
        v += __shfl_xor_sync(0xffffffffu, v, 8);
        v += __shfl_xor_sync(0xffffffffu, v, 16);
        if (lane < 4) ml[n * 8 + 2 * lane + i] = make_float2(m[n][i], v);
      }
  }
  template <class F>
  __device__ __forceinline__ void add_o(float* to, F&& factor, bool first, int lane) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int head = n * 8 + 2 * (lane & 3) + i;
        const float f = factor(head);
        float* at = to + head * (DP + 4) + lane / 4;
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) {
          const float v = f == 0.f ? 0.f : o[n][t][i] * f, w = f == 0.f ? 0.f : o[n][t][i + 2] * f;
          at[t * 16] = first ? v : at[t * 16] + v;
          at[t * 16 + 8] = first ? w : at[t * 16 + 8] + w;
        }
      }
  }
};

// NB heads on the f32 pipe, two f32 an instruction. Scores: eight lanes (sixteen of 256 dims) a key, each with its share of the dims
// of all heads' queries in registers; the lanes' sums are handed out so that a lane ends with one head's score (seven exchanges for
// eight heads), and has that head's m and l. Outputs: a lane has four dims (or eight) of all heads, of every key or every second.
// (With the queries in shared memory, half a key's dims a lane, a load came with every four products: 64 sequences of 2300 keys,
// 28 query heads on 4 of 128 dims, 212 us instead of 131, 4.6 TB/s; 5 on one of 64 62 instead of 24.)
template <int DP, int NB>
struct DecodeMath<float, DP, NB> {
  static constexpr int kHeads = NB, kRow = DP * 4;
  static constexpr int kLanes = DP > 128 ? 16 : 8, kKeys = 32 / kLanes, kRounds = kChunk / kKeys;   // lanes a key, keys at a time
  static constexpr int kPieces = DP / 4 / kLanes;               // of four dims, a lane's of a key
  static constexpr int kTurns = DP < 128 ? 2 : 1, kOwn = DP < 128 ? 1 : DP / 128;   // lanes that share dims of the outputs; pieces of those a lane
  F2 q[kHeads][kPieces][2];
  F2 o[kHeads][kOwn][2];
  float m, l;                                                   // of this lane's head; l of its keys

  static __device__ __forceinline__ int head_of(int lane) { return (lane & (kLanes - 1)) / (kLanes / kHeads); }
  static __device__ __forceinline__ int piece(int w, int lane) { return kTurns == 2 ? lane & 15 : w * 32 + lane; }

  __device__ __forceinline__ void load(const float* qs, int heads, int D, int lane) {
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int at = 4 * ((lane & (kLanes - 1)) + kLanes * i);
        const float4 v = h < heads && at < D ? *reinterpret_cast<const float4*>(qs + h * D + at) : make_float4(0.f, 0.f, 0.f, 0.f);
        q[h][i][0] = pair2(v.x, v.y);
        q[h][i][1] = pair2(v.z, v.w);
      }
#pragma unroll
      for (int w = 0; w < kOwn; ++w) o[h][w][0] = o[h][w][1] = pair2(0.f, 0.f);
    }
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void poison() { l = __int_as_float(0x7fffffff); }
  // piece p of row r
  static __device__ __forceinline__ void at(uint32_t base, int r, int p, F2& a, F2& b) {
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(a.v), "=l"(b.v) : "r"(base + r * kRow + ((p ^ (r & 7)) << 4)) : "memory");
  }
  __device__ __forceinline__ void chunk(uint32_t ks, uint32_t vs, int lo, int nv, float scale2, float* ps, int lane) {
    const int g = lane & (kLanes - 1), sub = lane / kLanes;
    float x[kRounds];   // of keys sub, kKeys + sub, ...
#pragma unroll
    for (int n = 0; n < kRounds; ++n) {
      F2 s[kHeads];
#pragma unroll
      for (int h = 0; h < kHeads; ++h) s[h] = pair2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        F2 a, b;
        at(ks, n * kKeys + sub, g + kLanes * i, a, b);
#pragma unroll
        for (int h = 0; h < kHeads; ++h) s[h] = fma2(b, q[h][i][1], fma2(a, q[h][i][0], s[h]));
      }
      float v[kHeads];
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        float b;
        split2(s[h], v[h], b);
        v[h] += b;
      }
#pragma unroll
      for (int d = kLanes / 2; d >= 1; d >>= 1) {   // lane distance d: half of the values each, while there are several
        const int left = kHeads * 2 * d / kLanes;
        const bool up = lane & d;
        if (left > 1) {
#pragma unroll
          for (int k = 0; k < left / 2; ++k)
            v[k] = (up ? v[k + left / 2] : v[k]) + __shfl_xor_sync(0xffffffffu, up ? v[k] : v[k + left / 2], d);
        } else {
          v[0] += __shfl_xor_sync(0xffffffffu, v[0], d);
        }
      }
      x[n] = v[0];
    }
    float top = m;
#pragma unroll
    for (int n = 0; n < kRounds; ++n)
      if (n * kKeys + sub >= lo && n * kKeys + sub < nv) top = fmaxf(top, x[n] * scale2);
    if (kLanes == 8) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
    if (__any_sync(0xffffffffu, top != m)) {
      const float f = top == m ? 1.f : ex2_ftz(m - top);
      m = top;
      l *= f;
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        const float fh = __shfl_sync(0xffffffffu, f, h * (kLanes / kHeads));
        const F2 f2 = pair2(fh, fh);
#pragma unroll
        for (int w = 0; w < kOwn; ++w) {
          o[h][w][0] = mul2(o[h][w][0], f2);
          o[h][w][1] = mul2(o[h][w][1], f2);
        }
      }
    }
#pragma unroll
    for (int n = 0; n < kRounds; ++n) {
      const int key = n * kKeys + sub;
      const float scaled = key >= lo && key < nv ? x[n] * scale2 : -INFINITY;
      // (the scaled score is rounded with the difference only)
      const float p = scaled == -INFINITY ? 0.f : ex2_ftz(fmaf(x[n], scale2, m == -INFINITY ? 0.f : -m));
      l += p;
      ps[head_of(lane) * kChunk + key % kTurns * (kChunk / kTurns) + key / kTurns] = p;
    }
    __syncwarp();
    const int turn = kTurns == 2 ? lane >> 4 : 0;
#pragma unroll
    for (int r = 0; r < kChunk; r += 4 * kTurns) {
      if (r >= nv) break;
      F2 v[kOwn][4][2];
#pragma unroll
      for (int w = 0; w < kOwn; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) at(vs, r + i * kTurns + turn, piece(w, lane), v[w][i][0], v[w][i][1]);
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        const float4 p = *reinterpret_cast<const float4*>(ps + h * kChunk + turn * (kChunk / kTurns) + r / kTurns);
        const float pv[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const F2 p2 = pair2(pv[i], pv[i]);
#pragma unroll
          for (int w = 0; w < kOwn; ++w) {
            o[h][w][0] = fma2(p2, v[w][i][0], o[h][w][0]);
            o[h][w][1] = fma2(p2, v[w][i][1], o[h][w][1]);
          }
        }
      }
    }
    __syncwarp();
  }
  __device__ __forceinline__ void put_ml(float2* ml, int lane) {
    if (kLanes == 8) l += __shfl_xor_sync(0xffffffffu, l, 8);
    l += __shfl_xor_sync(0xffffffffu, l, 16);
    if (lane < kLanes) ml[head_of(lane)] = make_float2(m, l);   // (lanes of the same head have the same)
  }
  template <class F>
  __device__ __forceinline__ void add_o(float* to, F&& factor, bool first, int lane) {
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const float f = factor(h);
#pragma unroll
      for (int w = 0; w < kOwn; ++w) {
        float x[4];
        split2(o[h][w][0], x[0], x[1]);
        split2(o[h][w][1], x[2], x[3]);
        if (kTurns == 2) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], 16);
          if (lane >= 16) continue;
        }
        float4& at = *reinterpret_cast<float4*>(to + h * (DP + 4) + piece(w, lane) * 4);
        float4 v = first ? make_float4(0.f, 0.f, 0.f, 0.f) : at;
        if (f != 0.f) {
          v.x += x[0] * f;
          v.y += x[1] * f;
          v.z += x[2] * f;
          v.w += x[3] * f;
        }
        at = v;
      }
    }
  }
};

template <class T, int DP, int NB>
struct DecodeCfg {
  using Math = DecodeMath<T, DP, NB>;
  static constexpr int kChunkBytes = kChunk * DP * static_cast<int>(sizeof(T));   // of keys, and of values
  // rows of 512 bytes: one stage and two blocks an SM rather than three and one (64 sequences of 2300 keys: f32, 28 / 4 heads of 128,
  // 163 -> 131 us; bf16, 4 / 4 of 256, 100 -> 97). Of f32 rows of 1024 bytes no more than one stage and one block fit (28 / 4 heads of
  // 256 441 us, 4 / 4 241, where the bytes take 178).
  static constexpr int kStages = kChunkBytes >= 8192 ? 1 : kChunkBytes >= 4096 ? 3 : 4;
  static constexpr int kRing = kStages * 2 * kChunkBytes;
  static constexpr int kPs = sizeof(T) == 4 ? Math::kHeads * kChunk * 4 : 0;
  static constexpr int kWarp = kRing + kPs;
  static constexpr int kOuts = sizeof(T) == 4 || NB == 1 ? 2 : 1;                 // where the warps' o are added up
  static constexpr int kOut = Math::kHeads * (DP + 4) * 4;
  static constexpr int kSmem = kDecWarps * kWarp + kOuts * kOut;
  static constexpr int kBlocks = kSmem <= 112 * 1024 ? 2 : 1;                     // per SM
  static_assert(kSmem <= 226 * 1024, "an SM's shared memory");
};

// A sequence's keys: the last `window` of its length, or all; in chunks, of TMA from a multiple of 16 on.
struct Keys {
  int first, base, end;
  bool bad;
  __device__ __forceinline__ int tiles() const { return (end - base + kTile - 1) / kTile; }
};
template <bool TMA>
static __device__ __forceinline__ Keys keys_of(const DecodeArgs& a, int b) {
  const int len = __ldg(a.lens + b);
  if (len < 0 || len > (a.c.ldt << a.c.page_log2)) return {0, 0, 0, true};
  const int first = a.window > 0 && len > a.window ? len - a.window : 0;
  return {first, TMA ? first & ~(kChunk - 1) : first, len, false};
}

// TMA (bf16, pages of 16 positions and more: a chunk lies in one page): one lane has a chunk's boxes copied, four instructions
// of D = 128 in the place of 16 copies a lane with their addresses; an mbarrier a stage. Values behind a sequence's end, or
// before its window, may be anything: they are zeroed in shared memory. Else the lanes copy, rows of any pages.
template <class T, int DP, int NB, bool TMA>
__global__ void __launch_bounds__(kDecThreads, (DecodeCfg<T, DP, NB>::kBlocks))
    decode_kernel(const DecodeArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using Cfg = DecodeCfg<T, DP, NB>;
  using Math = typename Cfg::Math;
  constexpr int ST = Cfg::kStages, E = 16 / static_cast<int>(sizeof(T)), PR = DP / E, H = Math::kHeads;
  extern __shared__ __align__(1024) uint8_t dec_smem[];
  __shared__ __align__(8) uint64_t full[kDecWarps][ST];
  __shared__ float2 ml_s[kDecWarps][H];
  __shared__ int64_t scan_s[kDecWarps], start_s;
  __shared__ int b_s, bad_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint8_t* const mine = dec_smem + warp * Cfg::kWarp;
  const uint32_t ring = smem_addr(mine);
  float* const out_s = reinterpret_cast<float*>(dec_smem + kDecWarps * Cfg::kWarp);
  float* const p_s = reinterpret_cast<float*>(mine + Cfg::kRing);
  const int per_head = a.blocks, HM = a.c.Hk * per_head;    // units a sequence

  // dims behind D stay zeros in every stage (TMA fills its last box itself)
  if (a.c.D < DP && (!TMA || a.c.D <= DP - 64)) {
    for (int i = lane; i < ST * 2 * kChunk * PR; i += 32) *reinterpret_cast<uint4*>(mine + i * 16) = make_uint4(0, 0, 0, 0);
    if (TMA) fence_proxy_async_smem();
  }
  if (TMA && lane == 0) {
    for (int s = 0; s < ST; ++s) mbar_init(&full[warp][s], 1);
    fence_mbar_init();
  }
  if (tid == 0) bad_s = 0, b_s = a.B;
  __syncthreads();
  wait_for_previous_kernel();
  let_next_kernel_in();

  // the list's length, and the sequence in which this CTA's run begins
  const int per = (a.B + kDecThreads - 1) / kDecThreads, b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
  const int tiles0 = b0 < b1 ? keys_of<TMA>(a, b0).tiles() : 0;
  int64_t sum = tiles0;
  for (int b = b0 + 1; b < b1; ++b) sum += keys_of<TMA>(a, b).tiles();
  int64_t upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) scan_s[warp] = upto;
  __syncthreads();
  int64_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) {
    if (w < warp) before += scan_s[w];
    total += scan_s[w];
  }
  upto += before;
  const int64_t list = total * HM;
  // (of a list with fewer tiles than CTAs the first ones have one each, so that a unit's parts are its CTAs' in a row)
  const int64_t takers = min(static_cast<int64_t>(gridDim.x), list), me = min(static_cast<int64_t>(blockIdx.x), takers);
  const int64_t t0 = me < takers ? list * me / takers : list, t1 = me < takers ? list * (me + 1) / takers : list;
  if (t0 < t1 && (upto - sum) * HM <= t0 && t0 < upto * HM) {
    int64_t at = upto - sum;
    int b = b0;
    for (int n = tiles0; t0 >= (at + n) * HM; n = keys_of<TMA>(a, b).tiles()) {
      at += n;
      ++b;
    }
    b_s = b;
    start_s = at * HM;
  }
  __syncthreads();

  // A place in the list: tile `tile` of `tiles` of unit hm of sequence b.
  struct Place {
    int64_t t;
    int b, hm, tile, tiles, first, base, end;
  };
  auto enter = [&](Place& p) {   // the sequence's keys
    const Keys k = keys_of<TMA>(a, p.b);
    p.first = k.first;
    p.base = k.base;
    p.end = k.end;
    p.tiles = k.tiles();
  };
  auto next = [&](Place& p) {
    if (++p.t >= t1) return;
    if (++p.tile < p.tiles) return;
    p.tile = 0;
    if (++p.hm < HM) return;
    p.hm = 0;
    do {
      ++p.b;
      enter(p);
    } while (p.tiles == 0);
  };
  // The page of the warp's chunk at a place, or (lanes) of this lane's key, row lane % 16: -1 where there is no key.
  auto page_at = [&](const Place& p) {
    const int key = p.base + p.tile * kTile + warp * kChunk + (TMA ? 0 : lane & 15);
    return p.t < t1 && key < p.end && (TMA || key >= p.first) ? __ldg(a.c.table + p.b * a.c.ldt + (key >> a.c.page_log2)) : -1;
  };
  uint32_t bad_stages = 0, phases = 0;
  bool stuck = false;
  auto issue = [&](const Place& p, int id, int st) {
    const int k0 = p.base + p.tile * kTile + warp * kChunk;
    bad_stages &= ~(1u << st);
    if (p.t < t1 && k0 < p.end && !stuck) {
      const int hk = per_head == 1 ? p.hm : p.hm / per_head;
      const uint32_t to = ring + st * 2 * Cfg::kChunkBytes;
      if (TMA) {
        if (id < 0 || id >= a.c.pages) bad_stages |= 1u << st;
        if (lane == 0) {
          const int64_t row = ((static_cast<int64_t>(id < 0 || id >= a.c.pages ? 0 : id) * a.c.Hk + hk) << a.c.page_log2) + (k0 & (a.c.page - 1));
          uint8_t* at = mine + st * 2 * Cfg::kChunkBytes;
          const int boxes = (a.c.D + 63) / 64;
          mbar_arrive_expect_tx(&full[warp][st], boxes * 2 * kBoxBytes);
#pragma unroll
          for (int x = 0; x < DP / 64; ++x) {
            if (x >= boxes) break;
            tma_load_2d(at + x * kBoxBytes, &k_map, &full[warp][st], x * 64, static_cast<int>(row));
            tma_load_2d(at + Cfg::kChunkBytes + x * kBoxBytes, &v_map, &full[warp][st], x * 64, static_cast<int>(row));
          }
        }
      } else {
        const int key = k0 + (lane & 15);
        const bool in = key >= p.first && key < p.end, good = in && id >= 0 && id < a.c.pages;
        if (__any_sync(0xffffffffu, in && !good)) bad_stages |= 1u << st;
        const int valid_id = good ? id : -1;
#pragma unroll
        for (int i = 0; i < kChunk * PR / 32; ++i) {
          const int idx = i * 32 + lane, r = idx / PR, pc = idx % PR;
          const int pid = __shfl_sync(0xffffffffu, valid_id, r);
          const int64_t row = ((static_cast<int64_t>(max(pid, 0)) * a.c.Hk + hk) << a.c.page_log2) + ((k0 + r) & (a.c.page - 1));
          const int64_t off = row * a.c.D + pc * E;
          const uint32_t at = to + (sizeof(T) == 2 ? (pc >> 3) * kBoxBytes + r * 128 + (((pc & 7) ^ (r & 7)) << 4)
                                                   : (r * PR + (pc ^ (r & 7))) * 16);
          if (pc * E < a.c.D) {
            lane_copy_or_zero(at, static_cast<const T*>(a.kc) + off, pid >= 0);
            lane_copy_or_zero(at + Cfg::kChunkBytes, static_cast<const T*>(a.vc) + off, pid >= 0);
          }
        }
      }
    }
    if (!TMA) asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // The warp's keys lo to nv of a tile in their stage: false where it has none.
  auto arrive = [&](const Place& p, int tile, int st, int& lo, int& nv) {
    const int k0 = p.base + tile * kTile + warp * kChunk;
    lo = max(0, p.first - k0);
    nv = min(kChunk, p.end - k0);
    if (!TMA) {
      asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
      __syncwarp();
      return nv > 0;
    }
    if (nv <= 0) return false;
    if (stuck || !mbar_wait(&full[warp][st], phases >> st & 1u, kDefaultTimeoutNs, nullptr)) stuck = true;
    stuck = __any_sync(0xffffffffu, stuck);
    phases ^= 1u << st;
    if (lo > 0 || nv < kChunk) {
      uint8_t* v = mine + st * 2 * Cfg::kChunkBytes + Cfg::kChunkBytes;
      for (int i = lane; i < kChunk * DP / 8; i += 32)
        if (i / 8 % kChunk < lo || i / 8 % kChunk >= nv) reinterpret_cast<uint4*>(v)[i] = make_uint4(0, 0, 0, 0);
      fence_proxy_async_smem();   // (before the stage's next copies)
      __syncwarp();
    }
    return true;
  };

  int4 seg = make_int4(0, -1, 0, 0);
  if (t0 < t1) {
    Place t, n;
    t.b = b_s;
    t.t = t0;
    enter(t);
    const int64_t in_seq = t0 - start_s;
    t.hm = static_cast<int>(in_seq / t.tiles);
    t.tile = static_cast<int>(in_seq - static_cast<int64_t>(t.hm) * t.tiles);
    n = t;
    Place ahead[ST];   // (their pages are looked up side by side)
    int ids[ST];
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      ahead[s] = n;
      ids[s] = page_at(n);
      next(n);
    }
    int id = page_at(n);
#pragma unroll
    for (int s = 0; s < ST; ++s) issue(ahead[s], ids[s], s);
    int st = 0, bad = 0;
    Math math;
    while (t.t < t1) {
      const int b = t.b, hm = t.hm, tile0 = t.tile;
      const int hk = per_head == 1 ? hm : hm / per_head, h0 = hk * a.group + (hm - hk * per_head) * H;
      const int heads = min(H, (hk + 1) * a.group - h0);
      const int tile1 = static_cast<int>(min(static_cast<int64_t>(t.tiles), tile0 + (t1 - t.t)));
      const bool whole = tile0 == 0 && tile1 == t.tiles;
      const int64_t end_tile = t.t - tile0 + t.tiles - 1;   // of the list
      math.load(static_cast<const T*>(a.q) + b * a.ldq + static_cast<int64_t>(h0) * a.c.D, heads, a.c.D, lane);
      for (int tile = tile0; tile < tile1; ++tile) {
        int lo, nv;
        const uint32_t from = ring + st * 2 * Cfg::kChunkBytes;
        if (arrive(t, tile, st, lo, nv)) math.chunk(from, from + Cfg::kChunkBytes, lo, nv, a.scale2, p_s, lane);
        if ((bad_stages >> st & 1u) || stuck) {
          math.poison();
          bad |= stuck ? PS_DEV_TIMEOUT : PS_DEV_BAD_PAGE;
        }
        __syncwarp();   // the stage has been read
        const Place now = n;
        const int now_id = id;
        next(n);
        id = page_at(n);
        issue(now, now_id, st);
        st = st + 1 == ST ? 0 : st + 1;
        next(t);
      }
      // the warps' parts together
      math.put_ml(ml_s[warp], lane);
      __syncthreads();
      auto top_of = [&](int h) {
        float top = ml_s[0][h].x;
#pragma unroll
        for (int w = 1; w < kDecWarps; ++w) top = fmaxf(top, ml_s[w][h].x);
        return top;
      };
      constexpr int OUTS = Cfg::kOuts, OUT = Cfg::kOut / 4;
#pragma unroll
      for (int k = 0; k < kDecWarps / OUTS; ++k) {
        if (warp / OUTS == k)
          math.add_o(out_s + warp % OUTS * OUT, [&](int h) {
            const float top = top_of(h);
            return top == -INFINITY ? 1.f : ex2_ftz(ml_s[warp][h].x - top);   // (0 where this warp had no keys)
          }, k == 0, lane);
        __syncthreads();
      }
      const int slot = 2 * blockIdx.x + (tile0 == 0 ? 1 : 0);
      for (int i = tid; i < heads * (DP / 8); i += kDecThreads) {   // eight dims of a head
        const int h = i / (DP / 8), c = i % (DP / 8) * 8;
        const float top = top_of(h);
        float l = 0.f, v[8];
#pragma unroll
        for (int w = 0; w < kDecWarps; ++w) l += ml_s[w][h].x == top ? ml_s[w][h].y : ml_s[w][h].y * ex2_ftz(ml_s[w][h].x - top);
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          float4 x = *reinterpret_cast<const float4*>(out_s + h * (DP + 4) + c + j);
          if (OUTS == 2) {
            const float4 y = *reinterpret_cast<const float4*>(out_s + OUT + h * (DP + 4) + c + j);
            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
          }
          v[j] = x.x, v[j + 1] = x.y, v[j + 2] = x.z, v[j + 3] = x.w;
        }
        if (whole) {
          const float r = 1.f / l;
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= r;
          if (c < a.c.D) Raw8<T>::store(static_cast<T*>(a.o) + b * a.ldo + static_cast<int64_t>(h0 + h) * a.c.D + c, v);
          if (c == 0 && a.lse) a.lse[static_cast<int64_t>(b) * a.Hq + h0 + h] = (top + log2f(l)) * kLn2;
        } else {
          Raw8<float>::store(a.part + (static_cast<int64_t>(slot) * H + h) * DP + c, v);
          if (c == 0) a.ml[slot * H + h] = make_float2(top, l);
        }
      }
      if (!whole) {
        if (tile0 == 0) seg = make_int4(0, b, hm, static_cast<int>(((end_tile + 1) * takers - 1) / list));
      }
      if (a.unit && tile0 == 0 && tid == 0) a.unit[b * HM + hm] = whole ? make_int2(-1, -1) : make_int2(blockIdx.x, seg.w);
      __syncthreads();
    }
    if (bad) atomicOr(&bad_s, bad);
    if (TMA && stuck)   // copies that may still come
      for (int s = 0; s < ST; ++s) mbar_wait(&full[warp][s], phases >> s & 1u, kDefaultTimeoutNs, nullptr);
  }
  // sequences without keys
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    const Keys k = keys_of<TMA>(a, b);
    if (k.end > 0) continue;
    if (k.bad && tid == 0) atomicOr(&bad_s, PS_DEV_BAD_LENGTH);
    for (int i = tid; i < a.Hq * a.c.D; i += kDecThreads)
      static_cast<T*>(a.o)[b * a.ldo + i] = Elem<T>::put(k.bad ? __int_as_float(0x7fffffff) : 0.f);
    if (a.unit)
      for (int i = tid; i < HM; i += kDecThreads) a.unit[b * HM + i] = make_int2(-1, -1);
    if (a.lse)
      for (int i = tid; i < a.Hq; i += kDecThreads) a.lse[static_cast<int64_t>(b) * a.Hq + i] = k.bad ? __int_as_float(0x7fffffff) : -INFINITY;
  }
  __syncthreads();
  if (tid == 0) {
    seg.x = bad_s;
    a.seg[blockIdx.x] = seg;
  }
}

// The units that several CTAs had parts of, and the call's status. BY_UNIT (few units, so long ones): a block for each head of
// each unit, whose warps share the parts; else a block for each CTA, which joins the unit that begins there and goes on, a warp a
// head where the parts are few. What a block needs it finds by one load, then the parts and their m and l come eight at a time. (A block for each head of each CTA that looks for its parts took 9 us, a third of it to start them.)
constexpr int kJoinThreads = 256;
template <class T, int DP, int H, bool BY_UNIT>
__global__ void __launch_bounds__(kJoinThreads) decode_join_kernel(const DecodeArgs a, int ctas) {
  constexpr int W = kJoinThreads / 32, C = (DP + 127) / 128, LD = 8 / C;
  __shared__ float2 ml_s[W];
  __shared__ float o_s[W][DP];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  wait_for_previous_kernel();
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    int bits = 0;
    for (int j = tid; j < ctas; j += kJoinThreads) bits |= a.seg[j].x;
    const int len = __syncthreads_or(bits & PS_DEV_BAD_LENGTH), page = __syncthreads_or(bits & PS_DEV_BAD_PAGE);
    const int time = __syncthreads_or(bits & PS_DEV_TIMEOUT);
    if (tid == 0) {
      a.status[1] = 0u;
      a.status[0] = (len ? PS_DEV_BAD_LENGTH : 0) | (page ? PS_DEV_BAD_PAGE : 0) | (time ? PS_DEV_TIMEOUT : 0);
    }
  }
  int i, last, b, hm;
  if (BY_UNIT) {
    const int2 at = a.unit[blockIdx.x];
    i = at.x, last = at.y;
    b = blockIdx.x / (a.c.Hk * a.blocks), hm = blockIdx.x - b * (a.c.Hk * a.blocks);
    if (i < 0) return;
  } else {
    const int4 at = a.seg[blockIdx.x];
    i = blockIdx.x, b = at.y, hm = at.z, last = at.w;
    if (b < 0) return;
  }
  const int hk = hm / a.blocks, h0 = hk * a.group + (hm - hk * a.blocks) * H, heads = min(H, (hk + 1) * a.group - h0);
  if (BY_UNIT && static_cast<int>(blockIdx.y) >= heads) return;
  const int parts = last - i + 1;
  auto slot = [&](int k, int h) { return (k == 0 ? 2 * i + 1 : 2 * (i + k)) * H + h; };
  // parts first, first + every, ... of head h: m and l, in every lane, and this lane's dims of o
  auto gather = [&](int h, int first, int every, float4 (&v)[C]) {
    float top = -INFINITY, l = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = first; k0 < parts; k0 += LD * every) {
      float2 ml[LD];
      float4 p[LD][C];
#pragma unroll
      for (int n = 0; n < LD; ++n) {
        const int k = k0 + n * every;
        ml[n] = make_float2(-INFINITY, 0.f);
        if (k < parts) ml[n] = a.ml[slot(k, h)];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          p[n][c] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (k < parts && (c * 32 + lane) * 4 < DP)
            p[n][c] = *reinterpret_cast<const float4*>(a.part + static_cast<int64_t>(slot(k, h)) * DP + (c * 32 + lane) * 4);
        }
      }
      float up = top;
#pragma unroll
      for (int n = 0; n < LD; ++n) up = fmaxf(up, ml[n].x);
      auto add = [&](float m, float lk, const float4 (&q)[C]) {
        const float f = m == up ? 1.f : ex2_ftz(m - up);
        l = fmaf(lk, f, l);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          v[c].x += f == 0.f ? 0.f : q[c].x * f;
          v[c].y += f == 0.f ? 0.f : q[c].y * f;
          v[c].z += f == 0.f ? 0.f : q[c].z * f;
          v[c].w += f == 0.f ? 0.f : q[c].w * f;
        }
      };
      if (up != top) {
        float4 had[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          had[c] = v[c];
          v[c] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        const float had_l = l;
        l = 0.f;
        add(top, had_l, had);
        top = up;
      }
#pragma unroll
      for (int n = 0; n < LD; ++n)
        if (k0 + n * every < parts) add(ml[n].x, ml[n].y, p[n]);
    }
    return make_float2(top, l);
  };
  auto put = [&](int h, int c, float v, float2 ml) {
    static_cast<T*>(a.o)[b * a.ldo + static_cast<int64_t>(h0 + h) * a.c.D + c] = Elem<T>::put(v / ml.y);
    if (c == 0 && a.lse) a.lse[static_cast<int64_t>(b) * a.Hq + h0 + h] = (ml.x + log2f(ml.y)) * kLn2;
  };
  float4 v[C];
  if (!BY_UNIT && parts <= 2 * W) {
    for (int h = warp; h < heads; h += W) {
      const float2 ml = gather(h, 0, 1, v);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int at = (c * 32 + lane) * 4;
        if (at >= a.c.D) continue;
        put(h, at, v[c].x, ml);
        put(h, at + 1, v[c].y, ml);
        put(h, at + 2, v[c].z, ml);
        put(h, at + 3, v[c].w, ml);
      }
    }
    return;
  }
  for (int h = BY_UNIT ? blockIdx.y : 0; h < (BY_UNIT ? static_cast<int>(blockIdx.y) + 1 : heads); ++h) {
    const float2 mine = gather(h, warp, W, v);
    if (lane == 0) ml_s[warp] = mine;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if ((c * 32 + lane) * 4 < DP) *reinterpret_cast<float4*>(&o_s[warp][(c * 32 + lane) * 4]) = v[c];
    __syncthreads();
    float top = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, ml_s[w].x);
    float f[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      f[w] = ml_s[w].x == top ? 1.f : ex2_ftz(ml_s[w].x - top);
      l = fmaf(ml_s[w].y, f[w], l);
    }
    for (int c = tid; c < a.c.D; c += kJoinThreads) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += f[w] == 0.f ? 0.f : o_s[w][c] * f[w];
      put(h, c, s, make_float2(top, l));
    }
    __syncthreads();
  }
}

// ================================================================== host side
constexpr int kDecMaxCtas = 304;
constexpr int kDecMaxHeads = 16, kDecMaxDim = 256;
constexpr size_t kDecSeg = (sizeof(int4) + sizeof(int2)) * kDecMaxCtas, kDecMl = sizeof(float2) * 2 * kDecMaxCtas * kDecMaxHeads;

static bool pages_ok(int seqs, int Hk, int D, int dtype, int pages, int page, int64_t ldt) {
  return seqs >= 0 && Hk >= 1 && Hk <= 65536 && D >= 16 && D <= kDecMaxDim && D % 16 == 0 &&
         (dtype == PS_DTYPE_BF16 || dtype == PS_DTYPE_F32) && pages >= 1 && page >= 1 && page <= 65536 && !(page & (page - 1)) &&
         ldt >= 1 && ldt <= INT32_MAX / page - 64;
}
static int log2_of(int v) {
  int n = 0;
  while ((1 << n) < v) ++n;
  return n;
}
static PagesOf pages_of(const int32_t* table, int64_t ldt, int pages, int page, int Hk, int D) {
  PagesOf c;
  c.table = table, c.ldt = ldt, c.pages = pages, c.page = page, c.page_log2 = log2_of(page), c.Hk = Hk, c.D = D;
  return c;
}

template <class T, int DP, int NB, bool TMA>
static int launch_decode(DecodeArgs a, cudaStream_t s) {
  using Cfg = DecodeCfg<T, DP, NB>;
  auto kern = decode_kernel<T, DP, NB, TMA>;
  CUtensorMap maps[2] = {};
  if (TMA)
    for (int i = 0; i < 2; ++i)
      if (!make_map(&maps[i], i ? a.vc : a.kc, a.c.D, static_cast<uint64_t>(a.c.pages) * a.c.Hk * a.c.page, a.c.D * 2, 64, kChunk))
        return PS_ERR_CUDA;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem) != cudaSuccess) return PS_ERR_CUDA;
  constexpr int H = Cfg::Math::kHeads;
  a.blocks = (a.group + H - 1) / H;
  int ctas = num_sms_current() * Cfg::kBlocks;
  if (ctas > kDecMaxCtas) ctas = kDecMaxCtas;
  // no more than the tiles that the table can name
  const int64_t most = static_cast<int64_t>(a.B) * a.c.Hk * a.blocks * (((a.c.ldt << a.c.page_log2) + kTile - 1) / kTile);
  if (ctas > most) ctas = static_cast<int>(most);
  const int64_t units = static_cast<int64_t>(a.B) * a.c.Hk * a.blocks;
  // Units of more than four CTAs' runs are joined by unit, a block a head, else by CTA (one sequence of 16384 keys, 4 key heads:
  // 14.2 us by unit, 27.3 by CTA; 8 of 4096 17.1 and 17.9; 32 of 2300 34.2 and 32.6; 64 of 2300 60.7 and 55.4).
  if (units * 4 > ctas) a.unit = nullptr;
  if (launch_after(kern, dim3(static_cast<unsigned>(ctas)), kDecThreads, Cfg::kSmem, s, 1, 1, true, a, maps[0], maps[1]) != cudaSuccess)
    return PS_ERR_CUDA;
  const cudaError_t e = a.unit ? launch_after(decode_join_kernel<T, DP, H, true>, dim3(static_cast<unsigned>(units), H), kJoinThreads, 0,
                                                    s, 1, 1, true, a, ctas)
                                     : launch_after(decode_join_kernel<T, DP, H, false>, dim3(static_cast<unsigned>(ctas)), kJoinThreads, 0,
                                                    s, 1, 1, true, a, ctas);
  return e == cudaSuccess ? PS_OK : PS_ERR_CUDA;
}

}  // namespace psk

using namespace psk;

extern "C" {

int ps_paged_append(int64_t N, int seqs, int Hk, int D, int dtype, const void* k, int64_t ldk, const void* v, int64_t ldv,
                    const int32_t* row_seq, const int32_t* row_pos, int pos_base, const int32_t* table, int64_t ldt, int pages,
                    int page, void* k_cache, void* v_cache, void* ws, size_t ws_bytes, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_paged_append");
  if (N < 0 || !pages_ok(seqs, Hk, D, dtype, pages, page, ldt)) return PS_ERR_INVALID_ARG;
  const int e = elem_bytes(dtype);
  const int64_t cols = static_cast<int64_t>(Hk) * D;
  auto rows_ok = [&](const void* p, int64_t ld) { return p && al16(p) && ld >= cols && ld * e % 16 == 0; };
  if (N > 0 && (!rows_ok(k, ldk) || !rows_ok(v, ldv) || !row_seq || !row_pos || !table || !k_cache || !v_cache || !al16(k_cache) ||
                !al16(v_cache)))
    return PS_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int rc = check_ws(ws, ws_bytes, kWsHeader);
  if (rc != PS_OK) return rc;
  if (N == 0) return refused(PS_OK, ws, s);
  AppendArgs a = {};
  a.N = N, a.seqs = seqs, a.c = pages_of(table, ldt, pages, page, Hk, D);
  a.k = k, a.v = v, a.ldk = ldk * e, a.ldv = ldv * e, a.seq = row_seq, a.pos = row_pos, a.pos_base = pos_base;
  a.kc = k_cache, a.vc = v_cache;
  a.pieces = static_cast<int>(cols * e / 16), a.head_pieces = D * e / 16;
  const int64_t want = static_cast<int64_t>(num_sms_current()) * 16;
  const int steps = (a.pieces + 63) / 64;
  a.parts = N >= want ? 1 : static_cast<int>(want / N < steps ? want / N : steps);
  a.checked = N <= kAppendCheckRows;
  a.status = static_cast<uint32_t*>(ws);
  if (!a.checked && cudaMemsetAsync(ws, 0, kWsHeader, s) != cudaSuccess) return PS_ERR_CUDA;
  const int64_t blocks = (N * a.parts + kAppendThreads / 32 - 1) / (kAppendThreads / 32), most = want;
  const int rc2 = launch_after(append_kernel, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), kAppendThreads, 0, s, 1, 1,
                               true, a) == cudaSuccess
                      ? PS_OK
                      : PS_ERR_CUDA;
  return rc2 == PS_OK ? rc2 : refused(rc2, ws, s);
}

size_t ps_paged_decode_workspace_size(int D) {
  if (D < 16 || D > kDecMaxDim || D % 16) return 0;
  const int DP = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  return kWsHeader + kDecSeg + kDecMl + sizeof(float) * 2 * kDecMaxCtas * kDecMaxHeads * DP;
}

int ps_paged_decode(int seqs, int Hq, int Hk, int D, int dtype, const void* q, int64_t ldq, const void* k_cache,
                    const void* v_cache, int pages, int page, const int32_t* table, int64_t ldt, const int32_t* lengths, int window,
                    double scale, void* o, int64_t ldo, float* lse, void* ws, size_t ws_bytes, ps_stream_t stream) {
  NvtxRange nvtx_range("ps_paged_decode");
  if (!pages_ok(seqs, Hk, D, dtype, pages, page, ldt) || Hq < Hk || Hq > 65536 || Hq % Hk || window < 0 ||
      !isfinite(static_cast<float>(scale * 1.4426950408889634)))
    return PS_ERR_INVALID_ARG;
  const int e = elem_bytes(dtype);
  const int64_t cols = static_cast<int64_t>(Hq) * D;
  auto rows_ok = [&](const void* p, int64_t ld) { return p && al16(p) && ld >= cols && ld * e % 16 == 0; };
  if (seqs > 0 && (!rows_ok(q, ldq) || !rows_ok(o, ldo) || !k_cache || !v_cache || !al16(k_cache) || !al16(v_cache) || !table ||
                   !lengths))
    return PS_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int rc = check_ws(ws, ws_bytes, ps_paged_decode_workspace_size(D));
  if (rc != PS_OK) return rc;
  if (seqs == 0) return refused(PS_OK, ws, s);
  DecodeArgs a = {};
  a.B = seqs, a.Hq = Hq, a.group = Hq / Hk, a.c = pages_of(table, ldt, pages, page, Hk, D);
  a.lens = lengths, a.window = window, a.scale2 = static_cast<float>(scale * 1.4426950408889634);
  a.q = q, a.ldq = ldq, a.kc = k_cache, a.vc = v_cache, a.o = o, a.ldo = ldo, a.lse = lse;
  uint8_t* w = static_cast<uint8_t*>(ws);
  a.status = reinterpret_cast<uint32_t*>(w);
  a.seg = reinterpret_cast<int4*>(w + kWsHeader);
  a.unit = reinterpret_cast<int2*>(a.seg + kDecMaxCtas);
  a.ml = reinterpret_cast<float2*>(w + kWsHeader + kDecSeg);
  a.part = reinterpret_cast<float*>(w + kWsHeader + kDecSeg + kDecMl);
  const bool tma = page >= kChunk && static_cast<int64_t>(pages) * Hk * page <= INT32_MAX - kChunk;   // (rows are counted in 32 bits)
  auto bf16 = [&](auto DP, auto NB) {
    return tma ? launch_decode<Bf16, decltype(DP)::value, decltype(NB)::value, true>(a, s)
               : launch_decode<Bf16, decltype(DP)::value, decltype(NB)::value, false>(a, s);
  };
  auto f32 = [&](auto DP) {
    constexpr int D_ = decltype(DP)::value;
    // (64 sequences of 2300 keys, 4 key heads of 128: one head each 97 us, by units of four 109; two 107, by units of one 182; four 106,
    // of eight 130; five 130, of four 206. Of 64 and 256 dims likewise.)
    if (a.group == 1) return launch_decode<float, D_, 1, false>(a, s);
    return a.group > 4 ? launch_decode<float, D_, 8, false>(a, s) : launch_decode<float, D_, 4, false>(a, s);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 128> d128;
  const std::integral_constant<int, 256> d256;
  int out;
  if (dtype == PS_DTYPE_F32)
    out = D <= 64 ? f32(d64) : D <= 128 ? f32(d128) : f32(d256);
  else if (D <= 64)
    out = a.group <= 8 ? bf16(d64, one) : bf16(d64, two);
  else if (D <= 128)
    out = a.group <= 8 ? bf16(d128, one) : bf16(d128, two);
  else
    out = bf16(d256, one);
  return out == PS_OK ? out : refused(out, ws, s);
}

}  // extern "C"
