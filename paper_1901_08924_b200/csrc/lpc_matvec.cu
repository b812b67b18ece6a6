// Products with a matrix held as packed 4-bit rows, W[r][k] = delta[r][k / group] (code - 8), as lpc_quantize_pack writes them:
//   packed_matvec     Y[m][r] = sum_k X[m][k] W[r][k]
//   packed_matvec_t   dX[m][k] = sum_r dY[m][r] W[r][k], the gradient of the first one for X
// for a few vectors at a time.
//
// What bounds them is reading the codes, and next to it the instructions that unpack them: at 6.5 TB/s an SM gets 46 codes a clock, and 128
// lanes can spend less than three instructions on each, at half that rate where they shift and mask.  So the multiplications go to the
// matrix instruction with 16-bit operands and fp32 sums, and two codes at a time become a pair of 16-bit floats by a mask that also sets
// the exponent of a power of two and one subtraction of that power and 8, all exact.  m16n8k16 takes 16 rows of codes and 8 vectors;
// mma.sync and not tcgen05, because the codes are unpacked in registers and are used straight from there, with no trip to shared memory, and 8
// columns are all there is.  Vectors are split into 16-bit pieces that add up to them, each piece a column of its own.
#include "lpc_matvec.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/lpc.h"
#include "lpc_device.cuh"

namespace cg = cooperative_groups;

namespace lpc {
namespace {

constexpr int MT = 256, MWARPS = MT / 32;
constexpr int SLAB = 128;  // columns of codes that a quad takes at a time: 16 words

__device__ __forceinline__ float half_value(uint32_t h, int type) {
  return type == LPC_BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half((unsigned short)h));
}
__device__ __forceinline__ void store_value(void* p, int64_t i, int type, float v) {
  if (type == LPC_F32) static_cast<float*>(p)[i] = v;
  else if (type == LPC_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[i] = __float2half_rn(v);
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// Asynchronous copies of single words to shared memory.
__device__ __forceinline__ void copy_word(float* to, const float* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Of two words, and in groups of which all but the last LEFT are waited for.
__device__ __forceinline__ void copy_words2(uint32_t* to, const uint32_t* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait_but() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Codes are read once: they take no room in L1.  The kernel before this one in the stream may have written them, and may still be running when this one
// starts: volatile, so that the load stays behind wait_for_launch_before, and coherent, as all loads here are (a non-coherent one is for what nobody writes
// while a kernel lives).
__device__ __forceinline__ void load_codes(uint32_t* w, const uint32_t* p) {  // 16 bytes
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
}

__device__ __forceinline__ uint32_t mask_or(uint32_t w, uint32_t mask, uint32_t set) {  // (w & mask) | set in one instruction
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(set));
  return r;
}

// The 8 codes of a word, less 8, as four fp16 pairs: codes (0, 4), (1, 5), (2, 6), (3, 7).  1024 + c and 1024 + 16 c are fp16 numbers, and
// so are the differences; the second form spares a shift.
__device__ __forceinline__ void unpack_fp16(uint32_t w, uint32_t* a) {
  const uint32_t v = w >> 8;
  const uint32_t p0 = mask_or(w, 0x000F000Fu, 0x64006400u), p1 = mask_or(w, 0x00F000F0u, 0x64006400u);
  const uint32_t p2 = mask_or(v, 0x000F000Fu, 0x64006400u), p3 = mask_or(v, 0x00F000F0u, 0x64006400u);
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(a[0]) : "r"(p0), "r"(0x64086408u));
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(a[1]) : "r"(p1), "r"(0x2C002C00u), "r"(0xD480D480u));  // / 16 - 72
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(a[2]) : "r"(p2), "r"(0x64086408u));
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(a[3]) : "r"(p3), "r"(0x2C002C00u), "r"(0xD480D480u));
}

// c = a b, and c += a b.
__device__ __forceinline__ void mma_fp16_first(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_fp16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The codes in the low 4 bits of both halves of w, less 8, as bfloat16: 128 + code is a bfloat16 number, and so is the difference.
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
  uint32_t r = mask_or(w, 0x000F000Fu, 0x43004300u);
  asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(0x43084308u));
  return r;
}

__device__ __forceinline__ void mma_bf16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The sum of a number's P pieces, `step` apart, in the shared memory of all CTAs of a cluster (8 at most), in the CTAs' order.  All are asked for before
// any is added.
template <int P>
__device__ __forceinline__ float sum_of_cluster(cg::cluster_group& cluster, float* sums, int at, int step) {
  const int ranks = (int)cluster.num_blocks();
  float v[8][P];
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < ranks) {
      const float* from = ranks > 1 ? cluster.map_shared_rank(sums, k) : sums;
#pragma unroll
      for (int p = 0; p < P; ++p) v[k][p] = from[at + p * step];
    }
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < ranks) {
#pragma unroll
      for (int p = 0; p < P; ++p) s = add_rn(s, v[k][p]);
    }
  return s;
}

struct MatvecPlan {
  int vectors;  // vectors of a pass
  int span;     // slabs (steps of 16 rows in the transposed product) of a CTA of the cluster
  int chunk;    // turns of a warp for which the vectors are brought in together
  int parts_log2;  // parts of a row whose scales are brought in together, at most 16
};

// ---- Y = X W^T ----------------------------------------------------------------------------------------------------------------
// A warp takes 16 RT rows and a slab of 128 columns at a time: lane (g, t) of it has 32 codes each of rows g and g + 8, which are the
// operands of 8 RT matrix instructions; which of the slab's columns sit at which place of the instruction's contraction is free as long as
// the vectors, laid out in shared memory, follow the same order.  LW: consecutive words a lane takes of a row, chosen so that an
// instruction never mixes groups of columns with different scales: 32 LW columns make up a group or a part of one.  WK warps share the rows'
// columns, and CTAs of a cluster do (through distributed shared memory at the end, without a workspace), so that some thousand rows fill the
// chip (eight CTAs at most share theirs: 128 rows leave 140 SMs idle); 8 / WK have rows of their own, so that the vectors, which every CTA lays out for itself, are not laid out too often.  Codes
// go from memory to the registers they are used in, AHEAD slabs before (copies to shared memory and more slabs ahead were no gain).
//
// The vectors are fp16 pieces.  An fp16 vector is its own piece.  128 columns of another are multiplied by the power of two that brings their
// largest magnitude to 2^14 .. 2^15, which the sums are divided by again; a bfloat16 vector (8 significant bits) is then one piece, an fp32
// vector two (11 bits each and the sign of the second: of 24 bits the last may be lost, 2^-23 of a value at most).  What falls out of fp16's
// range at the lower end is below 2^-39 of the largest of the 128.  Where one of the 128 is not finite, every product with them is
// infinite or NaN whatever the others are: those are taken as zeros, so that none of them overflows.
// Small vectors are multiplied by much, and a sum of 128 products, up to 2^25 then, times a large scale could leave the floats though the result does not:
// the factor f that undoes the power is taken in two parts, f1 = f but 2^-26 at least and 1 at most before the scale, f2 = f / f1 behind it.  Where f is below
// 1 the first product is below the scale and the second one smaller still; where it is not, what overflows does so rightly.
//
// 16384 x 16384, groups of 128: 33 us for one vector (4.3 TB/s; 24 us with nothing to read, 28 us with a quarter of the arithmetic: both sides
// overlap, but not fully with the 16 warps an SM that the registers allow), 44 us for 8, 58 us for 16 (a third of the instructions unpack, 0.4 of 3.5 a code scale), 119 us
// for 16 in fp32; groups of 32, one vector: 64 us (floors 21.8 to 25.6).  4096 x 4096, one vector: 6.1 us, of which a launch is 3.
template <int NT, int LW> constexpr int AHEAD = LW == 4 && NT < 4 ? 2 : 1;  // slabs of codes on their way
// Eights of columns that a thread brings in at a time: those of AHEAD turns of all the vectors of a pass, or more.
template <int NT, int WK, int LW, int NW> constexpr int TASKS_OF = (AHEAD<NT, LW> * WK * 16 * 8 * NT + NW * 32 - 1) / (NW * 32);

template <int NT, int RT, int WK, int LW, int TYPE, int NW>  // NW warps a CTA
__global__ void __launch_bounds__(NW * 32, 16 / NW) packed_matvec_kernel(MatvecArgs a, MatvecPlan plan) {
  constexpr int FT = NW * 32, WR = NW / WK, ROWS = 16 * RT * WR, NG = 4 / LW, P = TYPE == LPC_F32 ? 2 : 1, PD = AHEAD<NT, LW>;
  launch_dependents();
  wait_for_launch_before();
  extern __shared__ __align__(16) unsigned char smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp = threadIdx.x >> 5;
  const int wk = warp % WK, wr = warp / WK;
  const int m0 = blockIdx.y * plan.vectors, M = min(plan.vectors, a.M - m0);
  const int NC = M * P;  // column p * M + m: piece p of vector m
  const int64_t row0 = (int64_t)(blockIdx.x / ranks) * ROWS;
  const int slabs = (a.cols + SLAB - 1) / SLAB;
  const int s0 = rank * plan.span, s1 = min(slabs, s0 + plan.span);
  const int per_group = a.group / (32 * LW), parts = (a.cols + 32 * LW - 1) / (32 * LW);
  const int chunk_slabs = plan.chunk * WK;

  // shared memory: two buffers of vectors, their factors
  uint4* sx = reinterpret_cast<uint4*>(smem);
  const int sx_size = chunk_slabs * 16 * NC;
  float2* factor = reinterpret_cast<float2*>(sx + 2 * sx_size);  // f1 and f2
  float* red = reinterpret_cast<float*>(smem);

  // ---- codes, PD slabs ahead.  Behind the last row the last one is read again (its result is not kept); what is behind a row's last word stays
  // what it was (any codes will do there: the vectors have zeros)
  const uint32_t* row[RT][2];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t r = min(row0 + (wr * RT + i) * 16 + h * 8 + g, (int64_t)a.rows - 1);
      row[i][h] = a.codes + r * a.stride_words + (int64_t)(s0 + wk) * 16 + LW * t;
    }
  const int words = (int)a.stride_words - (s0 + wk) * 16 - LW * t;  // of a row, from this lane's first on
  uint32_t w[PD][RT][2][4];
#pragma unroll
  for (int u = 0; u < PD; ++u)
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 4; ++q) w[u][i][h][q] = 0u;
  auto fetch = [&](int turn, int u, uint32_t (&ww)[RT][2][4]) {  // `row` is at turn - u
    const int s = s0 + wk + turn * WK;
    if (s >= s1) return;
#pragma unroll
    for (int q = 0; q < 4; q += LW) {
      if (turn * WK * 16 + 4 * q < words) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t* at = row[i][h] + u * WK * 16 + 4 * q;
            if constexpr (LW == 4) {
              load_codes(ww[i][h], at);
            } else if constexpr (LW == 2) {
              const uint2 x = *reinterpret_cast<const uint2*>(at);
              ww[i][h][q] = x.x; ww[i][h][q + 1] = x.y;
            } else {
              ww[i][h][q] = *at;
            }
          }
      }
    }
  };
#pragma unroll
  for (int u = 0; u < PD; ++u) fetch(u, u, w[u]);

  // ---- scales: those of 16 parts of 32 LW columns at a time, a row's next to each other in memory and the rows' next to each other in shared memory
  constexpr int PARTS = 16, SROW = ROWS + 1, SCALE_TURNS = PARTS / NG / WK;
  float* sd = reinterpret_cast<float*>(factor + (TYPE == LPC_F16 ? 0 : 2 * chunk_slabs * M));
  auto bring_scales = [&](int stretch) {
    const int part = threadIdx.x & ((1 << plan.parts_log2) - 1), p = s0 * NG + stretch * PARTS + part;  // as many threads to a row as there are parts
    if (p >= min(parts, s1 * NG)) return;
    const float* from = a.delta + (per_group == 1 ? p : p / per_group);
    float* to = sd + ((stretch & 1) * PARTS + part) * SROW;
    for (int r = threadIdx.x >> plan.parts_log2; r < ROWS; r += FT >> plan.parts_log2) copy_word(to + r, from + min(row0 + r, (int64_t)a.rows - 1) * a.groups);
  };
  bring_scales(0);

  // ---- vectors: a task is 8 columns of one; 16 consecutive threads have a slab of it
  const int tasks = chunk_slabs * 16 * M, word = threadIdx.x & 15;
  const int lt = LW == 4 ? word >> 2 : LW == 2 ? (word >> 1) & 3 : word & 3;
  const int lq = LW == 4 ? word & 3 : LW == 2 ? (word >> 3) * 2 + (word & 1) : word >> 2;
  constexpr int RAW = TYPE == LPC_F32 ? 8 : 4, ELEM = TYPE == LPC_F32 ? 4 : 2;
  constexpr int TASKS = TASKS_OF<NT, WK, LW, NW>;
  const int s_first = (threadIdx.x >> 4) / M, m_first = (threadIdx.x >> 4) % M, s_next = FT / 16 / M, m_next = FT / 16 % M;
  uint32_t raw[TASKS][RAW];
  auto bring = [&](int chunk) {
    int s = s_first, m = m_first;
#pragma unroll
    for (int k = 0; k < TASKS; ++k) {
#pragma unroll
      for (int e = 0; e < RAW; ++e) raw[k][e] = 0u;
      const int slab = s0 + chunk * chunk_slabs + s;
      const int64_t col = (int64_t)slab * SLAB + word * 8;
      if (s < chunk_slabs && slab < s1 && col < a.cols) {
        const unsigned char* p = static_cast<const unsigned char*>(a.x) + ((int64_t)(m0 + m) * a.ldx + col) * ELEM;
        if (col + 8 <= a.cols && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
          const uint4 q0 = *reinterpret_cast<const uint4*>(p);
          raw[k][0] = q0.x; raw[k][1] = q0.y; raw[k][2] = q0.z; raw[k][3] = q0.w;
          if constexpr (TYPE == LPC_F32) {
            const uint4 q1 = reinterpret_cast<const uint4*>(p)[1];
            raw[k][4] = q1.x; raw[k][5] = q1.y; raw[k][6] = q1.z; raw[k][7] = q1.w;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e < a.cols) {
              if constexpr (TYPE == LPC_F32) raw[k][e] = reinterpret_cast<const uint32_t*>(p)[e];
              else raw[k][e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
            }
        }
      }
      m += m_next; s += s_next;
      if (m >= M) { m -= M; ++s; }
    }
  };
  auto lay_out = [&](int chunk) {
    uint4* to = sx + (chunk & 1) * sx_size;
    float2* fto = factor + (chunk & 1) * chunk_slabs * M;
    int s = s_first, m = m_first;
#pragma unroll
    for (int k = 0; k < TASKS; ++k) {
      if ((int)(threadIdx.x & ~31u) + k * FT < tasks) {  // the whole warp
        const bool mine = s < chunk_slabs;
        if constexpr (TYPE == LPC_F16) {
          if (mine) {
            const uint32_t* v = raw[k];
            to[((s * 4 + lq) * NC + m) * 4 + lt] = make_uint4(__byte_perm(v[0], v[2], 0x5410u), __byte_perm(v[0], v[2], 0x7632u),
                                                              __byte_perm(v[1], v[3], 0x5410u), __byte_perm(v[1], v[3], 0x7632u));
          }
        } else {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x[e] = TYPE == LPC_F32 ? __uint_as_float(raw[k][e & (RAW - 1)]) : __uint_as_float((e & 1) ? raw[k][e >> 1] & 0xFFFF0000u : raw[k][e >> 1] << 16);
          uint32_t top = 0;
          if constexpr (TYPE == LPC_BF16) {
#pragma unroll
            for (int e = 0; e < 4; ++e) top = __vmaxu2(top, raw[k][e] & 0x7FFF7FFFu);
            top = max(top & 0xFFFF0000u, top << 16);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
          }
          top = __reduce_max_sync(0xFFFFu << (threadIdx.x & 16), top);
          const bool all_finite = top < 0x7F800000u;
          const int ex = max((int)(top >> 23), 15);  // 2^(127 + 14 - ex) is a float from there on
          const float up = all_finite ? __uint_as_float((uint32_t)(268 - ex) << 23) : 1.f;
          __half2 hi[4], lo[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float u = mul_rn(x[e], up), v = mul_rn(x[e + 4], up);
            if (!all_finite) { u = finite(u) ? 0.f : u; v = finite(v) ? 0.f : v; }
            hi[e] = __floats2half2_rn(u, v);
            if constexpr (P == 2) {
              const float ul = __fsub_rn(u, __low2float(hi[e])), vl = __fsub_rn(v, __high2float(hi[e]));
              lo[e] = all_finite ? __floats2half2_rn(ul, vl) : __half2();
            }
          }
          if (mine) {
            to[((s * 4 + lq) * NC + m) * 4 + lt] = *reinterpret_cast<uint4*>(hi);
            if constexpr (P == 2) to[((s * 4 + lq) * NC + M + m) * 4 + lt] = *reinterpret_cast<uint4*>(lo);
            if (word == 0) {
              const int down = all_finite ? ex - 14 : 127, first = min(max(down, 127 - 26), 127);  // exponent fields of f and f1
              fto[s * M + m] = make_float2(__uint_as_float((uint32_t)first << 23), __uint_as_float((uint32_t)(127 + down - first) << 23));
            }
          }
        }
      }
      m += m_next; s += s_next;
      if (m >= M) { m -= M; ++s; }
    }
  };

  float tot[RT][NT][4];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) tot[i][n][e] = 0.f;
  int vec[NT][2];  // the vectors of this lane's two columns of a result
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) vec[n][e] = min(n * 8 + t * 2 + e, NC - 1) % M;

  int column[NT];  // where this lane's columns of the vectors are; a column behind the last is the last again, and its result is not kept
#pragma unroll
  for (int n = 0; n < NT; ++n) column[n] = min(n * 8 + g, NC - 1) * 4;
  bring(0);
  const int turns = (plan.span + WK - 1) / WK;  // the same for all warps of the cluster
  for (int turn0 = 0; turn0 < turns; turn0 += plan.chunk) {
    const int chunk = turn0 / plan.chunk, stretch = turn0 / SCALE_TURNS;
    lay_out(chunk);
    if (turn0 % SCALE_TURNS == 0) copies_wait();
    __syncthreads();  // scales are there; the other buffers' readers are through, too: they have been since the last one
    if (turn0 % SCALE_TURNS == 0) bring_scales(stretch + 1);
    bring(chunk + 1);  // behind the last chunk: zeros, nothing is read
    const float* ds = sd + ((stretch & 1) * PARTS + (turn0 % SCALE_TURNS * WK + wk) * NG) * SROW + wr * RT * 16 + g;
    const uint4* xs = sx + (chunk & 1) * sx_size + (size_t)wk * 16 * NC + t;
    const float2* fs = factor + (chunk & 1) * chunk_slabs * M + wk * M;
    for (int turn1 = turn0; turn1 < min(turn0 + plan.chunk, turns); turn1 += PD) {
#pragma unroll
      for (int u = 0; u < PD; ++u) {
        const int s = s0 + wk + (turn1 + u) * WK;
        if (s < s1) {
          float sum[RT][NT][4];
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            if (k > 0 && s * NG + k >= parts) break;  // behind the last column
            float acc[RT][NT][4];
#pragma unroll
            for (int q = k * LW; q < (k + 1) * LW; ++q) {
              uint4 b[NT];
#pragma unroll
              for (int n = 0; n < NT; ++n) b[n] = xs[q * NC * 4 + column[n]];
              uint32_t lo[RT][4], hi[RT][4];
#pragma unroll
              for (int i = 0; i < RT; ++i) {
                unpack_fp16(w[u][i][0][q], lo[i]);
                unpack_fp16(w[u][i][1][q], hi[i]);
              }
#pragma unroll
              for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  if (q == k * LW) mma_fp16_first(acc[i][n], lo[i][0], hi[i][0], lo[i][1], hi[i][1], b[n].x, b[n].y);
                  else mma_fp16(acc[i][n], lo[i][0], hi[i][0], lo[i][1], hi[i][1], b[n].x, b[n].y);
                }
#pragma unroll
              for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) mma_fp16(acc[i][n], lo[i][2], hi[i][2], lo[i][3], hi[i][3], b[n].z, b[n].w);
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
              const float d0 = ds[k * SROW + i * 16], d1 = ds[k * SROW + i * 16 + 8];
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float part = TYPE == LPC_F16 ? acc[i][n][e] : mul_rn(fs[vec[n][e & 1]].x, acc[i][n][e]);
                  sum[i][n][e] = k == 0 ? mul_rn(e < 2 ? d0 : d1, part) : __fmaf_rn(e < 2 ? d0 : d1, part, sum[i][n][e]);
                }
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float f = TYPE == LPC_F16 ? 1.f : fs[vec[n][e]].y;
#pragma unroll
              for (int i = 0; i < RT; ++i) {
                tot[i][n][e] = __fmaf_rn(f, sum[i][n][e], tot[i][n][e]);
                tot[i][n][e + 2] = __fmaf_rn(f, sum[i][n][e + 2], tot[i][n][e + 2]);
              }
            }
        }
        xs += WK * 16 * NC;
        fs += WK * M;
        ds += WK * NG * SROW;
        fetch(turn1 + u + PD, u + PD, w[u]);
      }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) row[i][h] += PD * WK * 16;
    }
  }

  // add up the warps that share rows, then the CTAs of the cluster, in a fixed order
  constexpr int COLS = 8 * NT;
  copies_wait();
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        red[(wk * COLS + n * 8 + t * 2 + (e & 1)) * ROWS + (wr * RT + i) * 16 + (e >> 1) * 8 + g] = tot[i][n][e];
  __syncthreads();
  for (int i = threadIdx.x; i < NC * ROWS; i += FT) {
    float s = red[i];
#pragma unroll
    for (int k = 1; k < WK; ++k) s = add_rn(s, red[k * COLS * ROWS + i]);
    red[i] = s;
  }
  if (ranks > 1) cluster.sync();
  else __syncthreads();
  const int share = (M * ROWS + ranks - 1) / ranks;
  for (int i = rank * share + threadIdx.x; i < min(M * ROWS, (rank + 1) * share); i += FT) {
    const int m = i / ROWS, r = i % ROWS;
    const float s = sum_of_cluster<P>(cluster, red, m * ROWS + r, M * ROWS);
    if (row0 + r < a.rows) store_value(a.y, (int64_t)(m0 + m) * a.ldy + row0 + r, TYPE, s);
  }
  if (ranks > 1) cluster.sync();  // nobody leaves while its sums are read
}

// ---- dX = dY W --------------------------------------------------------------------------------------------------------------------
// The contraction runs over rows, so a scale belongs to an operand: dY delta, a float, in bfloat16 pieces (fp16 has not the range), for each
// group of columns.  A warp takes 128 columns of 16 rows at a time; lane (g, t) has the codes of rows 4t .. 4t + 3 at 16 columns (CW = 16: two
// consecutive words; 8: a word of each of two groups; 4: half a word of each of four), and codes of two rows are paired by byte permutes.
// P pieces of MP vectors, piece by piece, are the instruction's columns, so that a lane that has a vector forms its pieces together.  With
// two pieces, for outputs of 8 or 11 significant bits, 2^-18 of a factor is lost; three hold all of it.
// WC blocks of 128 columns make up a CTA, and 8 / WC warps share a block's rows.  Scales of 512 rows at a time are copied to shared memory: a row's are
// next to each other and far from the next row's, so that every lane fetching its own kept the memory pipe busy with single words (16384 x 8192, groups of
// 64, 8 vectors: 53 us, 35 us of them with no scales to fetch).  At 16384 x 16384 one vector takes 55 us, 16 take 103 and 16 fp32 ones 178; with 256 rows,
// through registers, 59, 129 and 228; with 1024 rows groups of 32 took 80 us instead of 74 (now 71).
// 16384 x 8192, groups of 64, 8 vectors: 36 us (floor 11.6); 16384 x 16384, groups of 128, one vector: 55 us (floor 21.8), of which some 40 pass with the
// codes at hand: the operands' instructions, 3.5 a code, bound it.  4096 x 4096, one vector: 8.3 us, of which a launch is 3.
constexpr int SCALE_ROWS = 512;
// Codes are copied to shared memory RING - 1 steps ahead, a lane's words 2g and 2g + 1 of its four rows (groups of 32, where a lane has half words of
// its rows to fetch: 95 us -> 74 us for one vector at 16384 x 16384; 8 slots took 2 % longer than 4).  TROW and the place of a quad's rows keep banks
// apart for all three ways of reading.
constexpr int RING = 4, TROW = 72, SLOT = 4 * TROW;

template <int TYPE> constexpr int PIECES = TYPE == LPC_F32 ? 3 : 2;

// The P pieces of two floats, as pairs.
template <int P>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t* out) {
  if constexpr (P == 2) {
    // A finite x may round to infinity: the first piece stops at the largest bfloat16 instead, and the second one has the rest.  An infinite x has an
    // infinite rest.
    uint32_t h;
    asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(y), "f"(x));
    const float fx = __uint_as_float(h << 16), fy = __uint_as_float(h & 0xFFFF0000u);
    const __nv_bfloat162 lo = __floats2bfloat162_rn(__fsub_rn(x, fx), __fsub_rn(y, fy));
    out[0] = h;
    out[1] = *reinterpret_cast<const uint32_t*>(&lo);
  } else {  // cut off, not rounded: exact, and nothing overflows
    float v[2] = {x, y};
    uint32_t p[3][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool ok = finite(v[i]);
      const float hi = __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u), r = ok ? __fsub_rn(v[i], hi) : 0.f;
      const float mid = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
      p[0][i] = v[i] != v[i] ? 0x7FC00000u : __float_as_uint(hi);
      p[1][i] = __float_as_uint(mid);
      p[2][i] = __float_as_uint(__fsub_rn(r, mid));
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) out[i] = __byte_perm(p[i][0], p[i][1], 0x7632u);
  }
}

template <int TYPE, int MP, int CW, int WC>
__global__ void __launch_bounds__(MT, PIECES<TYPE> * MP <= 16 ? 2 : 1) packed_matvec_t_kernel(MatvecArgs a, MatvecPlan plan) {
  constexpr int P = PIECES<TYPE>;
  constexpr int NT = (P * MP + 7) / 8, NG = 16 / CW, PD = 2, NV = MP > 8 ? 2 : 1;
  constexpr int TWC = WC, TWR = MWARPS / WC, CHUNK = SCALE_ROWS / (16 * TWR);  // turns of a warp for so many rows
  static_assert(CHUNK % PD == 0 && CHUNK >= RING, "whole rounds of the vectors' registers; a chunk's scales arrive during the one before");
  launch_dependents();
  wait_for_launch_before();
  extern __shared__ __align__(16) unsigned char smem[];
  float* red = reinterpret_cast<float*>(smem);
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp = threadIdx.x >> 5;
  const int wc = warp % TWC, wr = warp / TWC;
  const int m0 = blockIdx.y * plan.vectors, M = min(plan.vectors, a.M - m0);
  const int64_t col0 = (int64_t)(blockIdx.x / ranks) * (TWC * 128) + wc * 128;
  const int steps = (a.rows + 15) / 16;
  const int first = rank * plan.span, last = min(steps, first + plan.span);
  const int64_t word0 = col0 / 8;
  const int per_group = a.group / (CW * 8);
  constexpr int ELEM = P == 3 ? 4 : 2;

  // scales: parts of 8 CW columns, rows next to each other; zeros behind the last row (of this CTA, too) and the last group
  constexpr int NGC = NG * TWC, SROW = SCALE_ROWS + 4;
  const int part = threadIdx.x % NGC, group = ((int)((int64_t)(blockIdx.x / ranks) * (TWC * NG)) + part) / per_group;
  float* scales = reinterpret_cast<float*>(smem);
  auto bring_scales = [&](int chunk) {  // part of the next group of copies
    const int row0 = (first + chunk * CHUNK * TWR) * 16, end = min(a.rows, last * 16) - row0;
    const float* from = a.delta + (int64_t)row0 * a.groups + group;
    float* to = scales + ((chunk & 1) * NGC + part) * SROW;
#pragma unroll
    for (int i = 0; i < SCALE_ROWS * NGC / MT; ++i) {
      const int r = (int)threadIdx.x / NGC + i * (MT / NGC);
      if (r < end && group < a.groups) copy_word(to + r, from + (int64_t)r * a.groups);
      else to[r] = 0.f;
    }
  };
  bring_scales(0);
  // codes, a ring of slots for every warp.  Behind the last row the last one again, behind a row's last word what was there before: results that are not kept
  uint32_t* ring = reinterpret_cast<uint32_t*>(scales + 2 * NGC * SROW) + warp * RING * SLOT;
  const int place = t * 16 + (t >> 1) * 8;
  const bool in_row = word0 + 2 * g < a.stride_words;
  const uint32_t* lane_codes = a.codes + (in_row ? word0 + 2 * g : 0);
  int next = first + wr;  // the step whose codes are fetched next, and its first row of this lane
  const uint32_t* next_codes = lane_codes + ((int64_t)next * 16 + t * 4) * a.stride_words;
  auto fetch = [&](int slot) {
    if (next < last && in_row) {
      uint32_t* to = ring + slot * SLOT + place + 2 * g;
      if (next * 16 + 16 <= a.rows) {
        const uint32_t* from = next_codes;
#pragma unroll
        for (int i = 0; i < 4; ++i, from += a.stride_words) copy_words2(to + i * TROW, from);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) copy_words2(to + i * TROW, lane_codes + (int64_t)min(next * 16 + t * 4 + i, a.rows - 1) * a.stride_words);
      }
    }
    next += TWR;
    next_codes += (int64_t)(16 * TWR) * a.stride_words;
    copies_commit();
  };
  // this lane's vectors: token g of 8, or two of 16, or one of few with the piece that its column is
  const int piece = MP < 8 ? g / MP : 0;
  const unsigned char* ys[NV];
  bool has[NV], fast[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int m = (MP < 8 ? g % MP : g) + 8 * i;
    has[i] = m < M && (NT > 1 || piece < P);
    ys[i] = static_cast<const unsigned char*>(a.x) + (has[i] ? (int64_t)(m0 + m) * a.ldx * ELEM : 0);
    fast[i] = (reinterpret_cast<uintptr_t>(ys[i]) & (4 * ELEM - 1)) == 0;
  }
  auto fetch_vectors = [&](int turn, uint32_t (&y)[NV][ELEM]) {  // four values of each vector as they are
    const int step = first + turn * TWR + wr;
    const int64_t r0 = (int64_t)step * 16 + t * 4;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int e = 0; e < ELEM; ++e) y[v][e] = 0u;
      if (has[v] && step < last) {
        const unsigned char* p = ys[v] + r0 * ELEM;
        if (fast[v] && r0 + 4 <= a.rows) {
          if constexpr (P == 3) {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            y[v][0] = q.x; y[v][1] = q.y; y[v][2] = q.z; y[v][3] = q.w;
          } else {
            const uint2 q = *reinterpret_cast<const uint2*>(p);
            y[v][0] = q.x; y[v][1] = q.y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (r0 + e < a.rows) {
              if constexpr (P == 3) y[v][e] = reinterpret_cast<const uint32_t*>(p)[e];
              else y[v][e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
            }
        }
      }
    }
  };

  float acc[8][NT][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][n][e] = 0.f;
#pragma unroll
  for (int u = 0; u < RING - 1; ++u) fetch(u);
  uint32_t y[PD][NV][ELEM];
#pragma unroll
  for (int u = 0; u < PD; ++u) {
    fetch_vectors(u, y[u]);
  }
  const int chunks = ((plan.span + TWR - 1) / TWR + CHUNK - 1) / CHUNK;  // the same for all warps of the cluster
  for (int chunk = 0; chunk < chunks; ++chunk) {
    // this chunk's scales came with the group of copies of the last chunk's first turn, at least RING - 1 groups ago, or less in a warp without more turns
    if (first + (chunk * CHUNK - 1) * TWR + wr < last) copies_wait_but<RING - 2>();
    else copies_wait();
    __syncthreads();  // and the other buffer's readers are through
    if (chunk + 1 < chunks) bring_scales(chunk + 1);
    const float* sd = scales + ((chunk & 1) * NGC + wc * NG) * SROW + wr * 16 + 4 * t;
#pragma unroll 1
    for (int turn0 = chunk * CHUNK; turn0 < (chunk + 1) * CHUNK; turn0 += PD) {
#pragma unroll
      for (int u = 0; u < PD; ++u) {
        if (first + (turn0 + u) * TWR + wr >= last) break;
        copies_wait_but<RING - 2>();
        __syncwarp();  // the other lanes' copies are there, and all lanes have read the slot that is filled next
        fetch((turn0 + u + RING - 1) % RING);
        const uint32_t* from = ring + (turn0 + u) % RING * SLOT + place;
        float x[NV][4];
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (P == 3) x[v][i] = __uint_as_float(y[u][v][i]);
            else x[v][i] = half_value((i & 1) ? y[u][v][i >> 1] >> 16 : y[u][v][i >> 1] & 0xFFFFu, TYPE);
          }
#pragma unroll
        for (int k = 0; k < NG; ++k) {
          uint32_t b[NT][2];
          const float4 dk = *reinterpret_cast<const float4*>(sd + k * SROW + (turn0 + u - chunk * CHUNK) * TWR * 16);
          const float d[4] = {dk.x, dk.y, dk.z, dk.w};
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t p[P];
              split_pair<P>(mul_rn(d[2 * h], x[v][2 * h]), mul_rn(d[2 * h + 1], x[v][2 * h + 1]), p);
              if constexpr (MP < 8) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {  // column 8 n + g has piece (8 n + g) / MP
                  const int q = 8 / MP * n + piece;
                  b[n][h] = q == 0 ? p[0] : q == 1 ? p[1] : NT > 1 && q >= P ? 0u : p[P - 1];
                }
              } else {
#pragma unroll
                for (int q = 0; q < P; ++q) b[q * NV + v][h] = p[q];
              }
            }
          if constexpr (CW >= 8) {
            uint2 both[4];
#pragma unroll
            for (int q = (CW == 16 ? 0 : k); q <= (CW == 16 ? 1 : k); ++q) {
              uint32_t w0, w1, w2, w3;
              if constexpr (CW == 16) {
                const uint2* at = reinterpret_cast<const uint2*>(from + 2 * g);
                if (q == 0) {
#pragma unroll
                  for (int i = 0; i < 4; ++i) both[i] = at[i * (TROW / 2)];
                }
                w0 = q ? both[0].y : both[0].x; w1 = q ? both[1].y : both[1].x; w2 = q ? both[2].y : both[2].x; w3 = q ? both[3].y : both[3].x;
              } else {
                const uint32_t* at = from + 8 * k + g;
                w0 = at[0]; w1 = at[TROW]; w2 = at[2 * TROW]; w3 = at[3 * TROW];
              }
              const uint32_t l01 = __byte_perm(w0, w1, 0x5410u), h01 = __byte_perm(w0, w1, 0x7632u);
              const uint32_t l23 = __byte_perm(w2, w3, 0x5410u), h23 = __byte_perm(w2, w3, 0x7632u);
#pragma unroll
              for (int i = 0; i < 4; ++i) {  // columns i and i + 4 of the word
                const uint32_t a0 = code_pair(l01 >> (4 * i)), a1 = code_pair(h01 >> (4 * i)), a2 = code_pair(l23 >> (4 * i)), a3 = code_pair(h23 >> (4 * i));
#pragma unroll
                for (int n = 0; n < NT; ++n) mma_bf16(acc[q * 4 + i][n], a0, a1, a2, a3, b[n][0], b[n][1]);
              }
            }
          } else {
            const uint32_t half = (g & 1) ? 0x7632u : 0x5410u;
            const uint32_t* at = from + 4 * k + (g >> 1);
            const uint32_t p01 = __byte_perm(at[0], at[TROW], half), p23 = __byte_perm(at[2 * TROW], at[3 * TROW], half);
#pragma unroll
            for (int i = 0; i < 2; ++i) {  // columns i and i + 2 of the half
              const uint32_t a0 = code_pair(p01 >> (4 * i)), a1 = code_pair(p01 >> (4 * i + 8)), a2 = code_pair(p23 >> (4 * i)), a3 = code_pair(p23 >> (4 * i + 8));
#pragma unroll
              for (int n = 0; n < NT; ++n) mma_bf16(acc[k * 2 + i][n], a0, a1, a2, a3, b[n][0], b[n][1]);
            }
          }
        }
        fetch_vectors(turn0 + u + PD, y[u]);
      }
    }
  }

  copies_wait();
  // add up the warps that share columns (the upper half of them hand their sums to the lower half), then the CTAs of the cluster
  for (int half = TWR / 2; half >= 1; half /= 2) {
    float* at = red + (size_t)((wr % half) * TWC + wc) * (32 * NT) * 32 + lane;
    __syncthreads();
    if (wr >= half && wr < 2 * half)
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) at[((i * NT + n) * 4 + e) * 32] = acc[i][n][e];
    __syncthreads();
    if (wr < half)
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][n][e] = add_rn(acc[i][n][e], at[((i * NT + n) * 4 + e) * 32]);
  }
  __syncthreads();
  constexpr int WIDTH = TWC * 128;
  if (wr == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          int col;  // of instruction i, row g or g + 8 of its result
          if constexpr (CW == 16) col = g * 16 + (i >> 2) * 8 + (i & 3) + 4 * (e >> 1);
          else if constexpr (CW == 8) col = (i >> 2) * 64 + g * 8 + (i & 3) + 4 * (e >> 1);
          else col = (i >> 1) * 32 + g * 4 + (i & 1) + 2 * (e >> 1);
          red[(n * 8 + t * 2 + (e & 1)) * WIDTH + wc * 128 + col] = acc[i][n][e];
        }
  }
  if (ranks > 1) cluster.sync();
  else __syncthreads();
  const int64_t base = (int64_t)(blockIdx.x / ranks) * WIDTH;
  const int share = (M * WIDTH + ranks - 1) / ranks;
  for (int i = rank * share + threadIdx.x; i < min(M * WIDTH, (rank + 1) * share); i += MT) {
    const int m = i / WIDTH, c = i % WIDTH;
    const float s = sum_of_cluster<P>(cluster, red, m * WIDTH + c, MP * WIDTH);
    if (base + c < a.cols) store_value(a.y, (int64_t)(m0 + m) * a.ldy + base + c, TYPE, s);
  }
  if (ranks > 1) cluster.sync();
}

template <class Kernel>
cudaError_t launch(Kernel kernel, int threads, unsigned groups, int ranks, unsigned passes, size_t smem, cudaStream_t st, const MatvecArgs& a, const MatvecPlan& plan) {
  if (smem > 48 * 1024) {  // always up to all there is: another host thread, whose call takes less, must not lower it before this launch
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(groups * (unsigned)ranks, passes);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ranks;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a, plan);
}

// How many CTAs of a cluster share a contraction of `turns` turns of a CTA's warps, for `groups` clusters: the number that takes the fewest turns
// when an SM holds `per_sm` CTAs, where filling a CTA's registers and adding up its sums take as long as OVERHEAD turns.  Returns those turns.
// With one CTA an SM, clusters of more than four do not find room on all SMs (transposed, 16 fp32 vectors, 16384 x 16384: eight 225 us, two 178), and of
// two numbers that are nearly equal the larger one is faster, whose CTAs even out (the same: one 210 us).
constexpr int OVERHEAD = 4;
int64_t split(int64_t groups, int64_t turns, int per_sm, int sm_count, int* ranks) {
  int64_t best = INT64_MAX;
  for (int r = 1; r <= 8; ++r) {
    const int64_t slots = per_sm > 1 ? per_sm * sm_count : r <= 4 ? sm_count : sm_count * 3 / 4;
    const int64_t t = (groups * r + slots - 1) / slots * ((turns + r - 1) / r + OVERHEAD);
    if (t < best || (per_sm == 1 && t <= best + best / 64)) { best = t; *ranks = r; }
    if (r >= turns) break;
  }
  return best;
}

// Turns of the CTAs where `warps` of them a CTA have 32 rows each, or WK of them share theirs.
int64_t forward_turns(const MatvecArgs& a, int64_t passes, int warps, int WK, int* ranks) {
  const int rows = 32 * warps / WK, slabs = (a.cols + SLAB - 1) / SLAB;
  return split(((int64_t)a.rows + rows - 1) / rows * passes, (slabs + WK - 1) / WK, 16 / warps, a.sm_count, ranks);
}

template <int NT, int RT, int WK, int LW, int TYPE, int NW>
cudaError_t launch_forward(const MatvecArgs& a, int vectors, cudaStream_t st) {
  constexpr int FT = NW * 32, ROWS = 16 * RT * (NW / WK), P = TYPE == LPC_F32 ? 2 : 1, PD = AHEAD<NT, LW>;
  MatvecPlan plan = {};
  plan.vectors = vectors;
  const int slabs = (a.cols + SLAB - 1) / SLAB, M = std::min(vectors, a.M);
  const int64_t groups = ((int64_t)a.rows + ROWS - 1) / ROWS, passes = (a.M + vectors - 1) / vectors;
  int ranks = 1;
  split(groups * passes, (slabs + WK - 1) / WK, 16 / NW, a.sm_count, &ranks);
  plan.span = ((slabs + WK - 1) / WK + ranks - 1) / ranks * WK;
  // as many turns as the threads' tasks cover, a power of two that divides the turns of a stretch of scales
  const int cover = std::min(TASKS_OF<NT, WK, LW, NW> * FT / (WK * 16 * M), LW * 4 / WK);
  plan.chunk = PD;
  while (plan.chunk * 2 <= cover && plan.chunk < (plan.span + WK - 1) / WK) plan.chunk *= 2;
  while (plan.parts_log2 < 4 && (1 << plan.parts_log2) < plan.span * (4 / LW)) ++plan.parts_log2;
  const size_t size = 2 * (size_t)plan.chunk * WK * M * (16 * P * 16 + (TYPE == LPC_F16 ? 0 : 8)) + 2 * 16 * (ROWS + 1) * 4;
  const size_t smem = std::max(size, (size_t)WK * 8 * NT * ROWS * 4);
  return launch(packed_matvec_kernel<NT, RT, WK, LW, TYPE, NW>, FT, (unsigned)groups, ranks, (unsigned)passes, smem, st, a, plan);
}

template <int LW, int TYPE>
cudaError_t launch_forward_of(const MatvecArgs& a, cudaStream_t st) {
  constexpr int P = TYPE == LPC_F32 ? 2 : 1;
  const int vectors = 32 / P, columns = std::min(vectors, a.M) * P;
  const int64_t passes = (a.M + vectors - 1) / vectors;
  int ranks = 1;
  if (columns <= 8) {  // two warps share rows where that takes fewer turns: few rows
    return forward_turns(a, passes, 8, 2, &ranks) < forward_turns(a, passes, 8, 1, &ranks) ? launch_forward<1, 2, 2, LW, TYPE, 8>(a, vectors, st)
                                                                                          : launch_forward<1, 2, 1, LW, TYPE, 8>(a, vectors, st);
  }
  if (columns <= 16) {
    // One CTA of 16 warps an SM lays the vectors out once where two of 8 do it twice (16384 x 16384, 16 vectors: 57 us against 60), two are better
    // where there is little to do (10007 x 1001, 5 fp32 vectors: 9.1 us against 9.9)
    return forward_turns(a, passes, 16, 1, &ranks) >= 16 ? launch_forward<2, 2, 1, LW, TYPE, 16>(a, vectors, st)
                                                         : launch_forward<2, 2, 1, LW, TYPE, 8>(a, vectors, st);
  }
  return launch_forward<4, 1, 1, LW, TYPE, 16>(a, vectors, st);
}

template <int LW>
cudaError_t launch_forward_type(const MatvecArgs& a, cudaStream_t st) {
  if (a.type == LPC_F32) return launch_forward_of<LW, LPC_F32>(a, st);
  if (a.type == LPC_BF16) return launch_forward_of<LW, LPC_BF16>(a, st);
  return launch_forward_of<LW, LPC_F16>(a, st);
}

// CTAs' turns where a CTA takes WC blocks of 128 columns, for `columns` pieces of vectors in a pass.  With more than 16 the registers leave room for one CTA
// an SM (12 fp32 vectors, 4096 x 4096: 14 us; counting on two 27).
int64_t transposed_turns(const MatvecArgs& a, int64_t passes, int columns, int WC, int* ranks) {
  const int64_t groups = ((int64_t)a.cols + WC * 128 - 1) / (WC * 128);
  const int steps = (a.rows + 15) / 16, TWR = MWARPS / WC;
  return split(groups * passes, (steps + TWR - 1) / TWR, columns <= 16 ? 2 : 1, a.sm_count, ranks);
}

template <int TYPE, int MP, int CW, int WC>
cudaError_t launch_transposed_wc(const MatvecArgs& a, cudaStream_t st) {
  constexpr int P = PIECES<TYPE>;
  constexpr int NT = (P * MP + 7) / 8, TWR = MWARPS / WC;
  MatvecPlan plan = {};
  plan.vectors = MP;
  const int64_t groups = ((int64_t)a.cols + WC * 128 - 1) / (WC * 128), passes = (a.M + MP - 1) / MP;
  const int steps = (a.rows + 15) / 16;
  int ranks = 1;
  transposed_turns(a, passes, P * MP, WC, &ranks);
  plan.span = ((steps + TWR - 1) / TWR + ranks - 1) / ranks * TWR;
  const size_t sums = (size_t)(TWR / 2) * WC * 32 * NT * 32 * 4;  // 32 NT sums of every lane of half the warps; more than the CTA's 8 NT columns
  const size_t scales = ((size_t)2 * (16 / CW) * WC * (SCALE_ROWS + 4) + MWARPS * RING * SLOT) * 4;
  return launch(packed_matvec_t_kernel<TYPE, MP, CW, WC>, MT, (unsigned)groups, ranks, (unsigned)passes, std::max(sums, scales), st, a, plan);
}

template <int TYPE, int MP, int CW>
cudaError_t launch_transposed(const MatvecArgs& a, cudaStream_t st) {
  // two blocks of columns share a row's scales; one fills the chip where columns are few.  With one CTA an SM, turns that differ by a sixteenth are equal
  // (16 fp32 vectors, 16384 x 16384: two blocks 178 us, one 210)
  constexpr int COLUMNS = PIECES<TYPE> * MP;
  const int64_t passes = (a.M + MP - 1) / MP;
  int ranks = 1;
  const int64_t two = transposed_turns(a, passes, COLUMNS, 2, &ranks), one = transposed_turns(a, passes, COLUMNS, 1, &ranks);
  return two <= one + (COLUMNS > 16 ? one / 16 : 0) ? launch_transposed_wc<TYPE, MP, CW, 2>(a, st) : launch_transposed_wc<TYPE, MP, CW, 1>(a, st);
}

template <int CW>
cudaError_t launch_transposed_of(const MatvecArgs& a, cudaStream_t st) {
  if (a.type == LPC_F32)
    return a.M <= 2 ? launch_transposed<LPC_F32, 2, CW>(a, st) : a.M <= 4 ? launch_transposed<LPC_F32, 4, CW>(a, st) : launch_transposed<LPC_F32, 8, CW>(a, st);
  if (a.type == LPC_BF16)
    return a.M <= 4 ? launch_transposed<LPC_BF16, 4, CW>(a, st) : a.M <= 8 ? launch_transposed<LPC_BF16, 8, CW>(a, st) : launch_transposed<LPC_BF16, 16, CW>(a, st);
  return a.M <= 4 ? launch_transposed<LPC_F16, 4, CW>(a, st) : a.M <= 8 ? launch_transposed<LPC_F16, 8, CW>(a, st) : launch_transposed<LPC_F16, 16, CW>(a, st);
}

}  // namespace

cudaError_t launch_packed_matvec(const MatvecArgs& a, cudaStream_t st) {
  if (a.group % 128 == 0) return launch_forward_type<4>(a, st);
  if (a.group % 64 == 0) return launch_forward_type<2>(a, st);
  return launch_forward_type<1>(a, st);
}

cudaError_t launch_packed_matvec_t(const MatvecArgs& a, cudaStream_t st) {
  if (a.group % 128 == 0) return launch_transposed_of<16>(a, st);
  if (a.group % 64 == 0) return launch_transposed_of<8>(a, st);
  return launch_transposed_of<4>(a, st);
}

}  // namespace lpc
