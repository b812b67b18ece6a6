// AdamW over the tensors of one vector, with moments in 32 or in 8 bits, from a dense gradient or from the workers' packed messages:
//   g' = g grad_scale            (packed: g = (sum_i delta_i k_i) (1 / N) + mu, the sum in worker order by fused multiply-adds)
//   m' = beta1 m + (1 - beta1) g'        v' = beta2 v + (1 - beta2) g'^2
//   p' = p (1 - lr wd) - lr / (1 - beta1^t) m' / (sqrt(v') / sqrt(1 - beta2^t) + eps)
// every other operation a separate fp32 round-to-nearest one.
//
// Moments in 8 bits.  A warp owns a block of 256 consecutive coordinates of a tensor and keeps, for each moment, the exponent e of
// the block's largest magnitude.  A value is scaled by 2^-e and by a constant that puts it where a float's own exponent field is the
// code's: the largest power of two at field 14 of the 4-bit field of m, at 30 of the 5-bit field of v (one field above is left for what
// rounding lifts over a power of two), and what is below field 1 among the floats without a leading one, whose even grid is the
// code's too.  Then the top bits of the float are the code, and stochastic rounding is one integer addition below them:
// code = (bits + 16 r + 8) >> 20 with r the 16-bit random lane.  Round to nearest would not do: at beta2 = 0.999 a step moves v by less than half
// a code and v would stand still.  A v above zero keeps a code above zero, so that m / sqrt(v) stays bounded.
//
// What bounds it.  One pass, eight consecutive coordinates a thread, everything asked for before anything is waited for.  2^26 weights: with 32-bit
// moments and an fp32 gradient (28 bytes a coordinate) 273 us, 6.9 TB/s, memory.  8-bit moments (16 bytes): 196 us, 5.5 TB/s; 72 instructions a coordinate
// take two thirds of the issue slots.  From 8 workers' 4-bit messages (24 or 12 bytes and 4 of codes): 328 us, 5.7 TB/s, with 32-bit moments, where 80
// registers leave 24 warps an SM to cover 86 instructions and the loads; 300 us, 3.6 TB/s, with 8-bit ones, 109 instructions in two thirds of the
// issue slots.  Values of 8-bit moments: 64 us, 6.3 TB/s.  62 tensors of 64 to 2.4 million weights, 11.7 million in all, 32 bits: 54 us (at the copy rate 50).
// Tensors that start anywhere, 2^25 weights: 152 us (32 bits), 124 us (8 bits).  Slower: five CTAs an SM for 8-bit moments (more spills), two chunks a CTA, a loop
// over chunks that loads the next one while it works on this one.  2^24 weights from 8 workers' messages: 84 to 94 us for 1, 2, 3, 4 and 8 bits (32-bit moments) and 73 to
// 94 (8-bit); widths known at run time 151 (16 bits) to 241 us (12 bits), 142 to 199.  All instances spill, those of 8 bits and run-time widths 400 to 580 bytes a thread.
#include "lpc_adamw.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "../../include/lpc.h"
#include "lpc_device.cuh"
#include "lpc_kernels.h"
#include "lpc_unpack.cuh"

namespace lpc {
namespace {

constexpr int ST = 256;
static_assert(STEP_CHUNK == ST * 8 && STEP_BLOCK == 32 * 8, "a thread owns 8 coordinates, a warp a block");
constexpr uint32_t TAG_MOMENT1 = 5, TAG_MOMENT2 = 6;
constexpr int TOP_M = 14, TOP_V = 30;         // exponent field of a block's largest power of two
constexpr uint32_t MOMENT_LIMIT = 253u << 23;  // 2^126, as bits: moments from here on have no 8-bit code, and are taken as not finite

// The root of the second moment and the quotient of the update.  With 32-bit moments, where memory is what bounds the step, correctly rounded; with 8-bit
// moments the instructions do, and the hardware's approximations (root: 2^-23 of the value; quotient: 2 units in the last place) take
// 3 of them where correct rounding takes some 20.  The root's takes a second moment below 2^-126 as zero, where that is less than half a unit of eps in the
// divisor: the moment's factor 1 / sqrt(1 - beta2^t) may lift it above that in the first steps of a beta2 next to 1, and those take roots of all
// floats (3 instructions more, 3 % of the step).  The quotient takes a first moment and a result below 2^-126 as zeros: the divisor is eps, 1e-10, at least, so
// that they are an update of less than 2^-92 of the step size.
template <bool APPROXIMATE>
__device__ __forceinline__ float root(float x) {
  if constexpr (!APPROXIMATE) return __fsqrt_rn(x);
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float root_of_any(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <bool APPROXIMATE>
__device__ __forceinline__ float quotient(float x, float y) {
  if constexpr (!APPROXIMATE) return __fdiv_rn(x, y);
  float r;
  asm("div.approx.ftz.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}

// 2^k as a float, -126 <= k <= 127
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// A warp's place in a tensor, and how its 256 values lie in its lanes: eight consecutive ones each, where an array's tensor starts on 16 bytes, or every
// 32nd, so that memory sees whole lines wherever it starts.  Arrays of one step may differ; `turn` takes a lane's values from one order to the
// other, through 1 KB of shared memory of the warp's own.
struct Place {
  int lane, n, count;  // consecutive values of this lane, values of the warp
  bool fast;           // known when the code is made: all 256 are there, and every array's tensor starts on 16 bytes
  uint32_t* buf;
};
__device__ __forceinline__ uint32_t word_of(const float* v, int e) { return __float_as_uint(v[e]); }
__device__ __forceinline__ uint32_t word_of(const uint16_t* v, int e) { return (uint32_t)v[2 * e] | (uint32_t)v[2 * e + 1] << 16; }
__device__ __forceinline__ void take_word(uint32_t w, float* v, int e) { v[e] = __uint_as_float(w); }
__device__ __forceinline__ void take_word(uint32_t w, uint16_t* v, int e) { v[2 * e] = (uint16_t)w; v[2 * e + 1] = (uint16_t)(w >> 16); }
// p: the lane's first value in the consecutive order.
template <class T>
__device__ __forceinline__ void load8(const T* p, const Place& at, bool consecutive, T* v) {
  if (at.fast || consecutive) {
    if (at.fast || at.n == 8) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint4 q = reinterpret_cast<const uint4*>(p)[i];
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) take_word(w[e], v, i * 4 + e);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < at.n ? p[e] : (T)0;
    }
  } else {
    const T* first = p - at.lane * 7;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = at.lane + 32 * k < at.count ? first[32 * k] : (T)0;
  }
}
template <class T>
__device__ __forceinline__ void store8(T* p, const Place& at, bool consecutive, const T* v) {
  if (at.fast || consecutive) {
    if (at.fast || at.n == 8) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = word_of(v, i * 4 + e);
        reinterpret_cast<uint4*>(p)[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < at.n) p[e] = v[e];
    }
  } else {
    T* first = p - at.lane * 7;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (at.lane + 32 * k < at.count) first[32 * k] = v[k];
  }
}
template <class T>
__device__ __forceinline__ void turn(const Place& at, bool to_consecutive, T* v) {
  T* buf = reinterpret_cast<T*>(at.buf);
  __syncwarp();
#pragma unroll
  for (int e = 0; e < 8; ++e) buf[to_consecutive ? at.lane + 32 * e : at.lane * 8 + e] = v[e];
  __syncwarp();
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = buf[to_consecutive ? at.lane * 8 + e : at.lane + 32 * e];
}
template <class T>
__device__ __forceinline__ bool starts_on_16(const T* p, const Place& at) { return aligned16(p - at.lane * 8); }

template <int TYPE>
__device__ __forceinline__ float of_half(uint16_t h) {
  if constexpr (TYPE == LPC_BF16) return __uint_as_float((uint32_t)h << 16);
  else return __half2float(__ushort_as_half(h));
}
__device__ __forceinline__ uint16_t to_half(float x, int type) {
  return type == LPC_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __half_as_ushort(__float2half_rn(x));
}

// The values of 8 codes of a block with this exponent.  A code's byte goes to the top of a word and from there to where a float has its exponent's lower
// bits (m: four and the sign, v: five) and three of its mantissa; what is left is a power of two, one factor unless it is too large for a float.
template <bool SIGNED>
__device__ __forceinline__ void decode_moment(uint2 c, uint32_t exponent, float* x) {
  constexpr int TOP = SIGNED ? TOP_M : TOP_V;
  const bool one = exponent <= 127 + TOP;
  const float scale = __uint_as_float(one && exponent ? (exponent + 127 - TOP) << 23 : exponent << 23);  // an exponent of 0: zeros
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t top = __byte_perm(e < 4 ? c.x : c.y, 0u, 0x0444u | (uint32_t)(e & 3) << 12);
    x[e] = __uint_as_float(SIGNED ? (uint32_t)((int32_t)top >> 4) & 0x87FFFFFFu : top >> 4);
  }
  if (!one) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = mul_rn(x[e], power_of_two(127 - TOP));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = mul_rn(x[e], scale);
}

// The codes of 8 values of a block with this exponent: the value where decode_moment starts from, (bits + 16 r + 8) >> 20, formed 4 bits higher
// so that the code is a byte of the sum.  v: a value above zero counts as a whole step of the grid at least.
template <bool SIGNED>
__device__ __forceinline__ uint2 encode_moment(const float* x, const U4& r, uint32_t exponent) {
  constexpr int TOP = SIGNED ? TOP_M : TOP_V;
  const bool one = exponent < 127 + TOP;
  const float scale = __uint_as_float((one ? 127 + TOP - exponent : 254u - exponent) << 23);
  const uint32_t rw[4] = {r.x, r.y, r.z, r.w};
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = mul_rn(SIGNED ? fabsf(x[e]) : x[e], scale);
  if (!one) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = mul_rn(s[e], power_of_two(TOP - 127));
  }
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (!SIGNED) s[e] = fmaxf(s[e], fminf(mul_rn(x[e], 1048576.f), __uint_as_float(1u << 20)));
    const uint32_t lane = __byte_perm(rw[e >> 1], 0x80u, (e & 1) ? 0x5324u : 0x5104u);  // 256 r + 128
    w[e] = (__float_as_uint(s[e]) << 4) + lane;
    if (SIGNED) w[e] |= __float_as_uint(x[e]) & 0x80000000u;
  }
  const uint32_t a = __byte_perm(w[0], w[1], 0x0073u), b = __byte_perm(w[2], w[3], 0x0073u), c = __byte_perm(w[4], w[5], 0x0073u),
                 d = __byte_perm(w[6], w[7], 0x0073u);
  return make_uint2(__byte_perm(a, b, 0x5410u), __byte_perm(c, d, 0x5410u));
}

__device__ __forceinline__ StepChunk chunk_of(const AdamwArgs& a) {
  StepChunk c;
  if (a.chunks) {
    const uint4* q = reinterpret_cast<const uint4*>(a.chunks + blockIdx.x);
    uint4* d = reinterpret_cast<uint4*>(&c);
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = q[i];
  } else {
    c = a.only;
    c.chunk = (int32_t)blockIdx.x;
  }
  return c;
}

// GRAD: LPC_F32, LPC_BF16, LPC_F16, or PACKED + the code width (0: from the arguments).
constexpr int PACKED = 64;

// acc + delta k at a group of 8 coordinates of one worker.
template <int BITS, class Word>
__device__ __forceinline__ void add_worker(f32x2* acc, float delta, Word lo, Word hi, int b) {
  f32x2 k[4];
  if constexpr (BITS == 0) {
    uint64_t x = lo, y = hi;
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = index_as_float(take_code(x, y, b), b);
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = pack2(f[2 * e], f[2 * e + 1]);
  } else {
    decode_pairs<BITS, 8>(lo, k);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = fma2_rn(pack2(delta, delta), k[e], acc[e]);
}

// A step's scalars, the same for a whole tensor.
struct StepScalars {
  float decay, step, second, gs;
  uint64_t t;
  bool small_roots;  // 8-bit moments: the root of a second moment below 2^-126 counts next to eps
};

template <int GRAD, bool BITS8, bool FAST>
__device__ __forceinline__ void adamw_chunk(const AdamwArgs& a, const StepChunk& c, StepScalars sc, const float* sdelta, uint32_t* buf) {
  const int tid = threadIdx.x;
  const int64_t j = (int64_t)c.chunk * STEP_CHUNK + tid * 8;
  Place at;
  at.fast = FAST;
  at.lane = tid & 31;
  at.count = FAST ? STEP_BLOCK : (int)max((int64_t)0, min((int64_t)STEP_BLOCK, c.len - (j - at.lane * 8)));
  at.n = FAST ? 8 : max(0, min(8, at.count - at.lane * 8));
  at.buf = buf;
  if (at.count == 0) return;  // the whole warp

  // everything that comes from memory is asked for before anything is waited for
  float p[8], g[8], m[8], v[8], mu[8];
  uint16_t gh[8];
  const int64_t block = c.block0 + (j >> 8);
  uint8_t* m8 = static_cast<uint8_t*>(a.m) + c.block0 * STEP_BLOCK + j;
  uint8_t* v8 = static_cast<uint8_t*>(a.v) + c.block0 * STEP_BLOCK + j;
  float* m32 = static_cast<float*>(a.m) + c.off + j;
  float* v32 = static_cast<float*>(a.v) + c.off + j;
  float* pj = a.p + c.off + j;
  const float* gj = static_cast<const float*>(a.g) + c.off + j;
  const uint16_t* ghj = static_cast<const uint16_t*>(a.g) + c.off + j;
  uint16_t* copyj = static_cast<uint16_t*>(a.copy) + c.off + j;
  const float* muj = a.mu + c.off + j;
  // codes, of moments or gradients, are in consecutive order; without them any order will do, and one that suits all arrays is taken
  constexpr bool CODES = BITS8 || GRAD >= PACKED;
  bool p_at = starts_on_16(pj, at), m_at = starts_on_16(m32, at), v_at = starts_on_16(v32, at);
  bool g_at = GRAD == LPC_F32 ? starts_on_16(gj, at) : starts_on_16(ghj, at), copy_at = !a.copy || starts_on_16(copyj, at);
  const bool mu_at = FAST || starts_on_16(muj, at);
  if constexpr (FAST) p_at = m_at = v_at = g_at = copy_at = true;
  else if constexpr (!CODES) p_at = m_at = v_at = g_at = copy_at = p_at && m_at && v_at && g_at && copy_at;
  uint2 cm = make_uint2(0u, 0u), cv = make_uint2(0u, 0u);
  uint32_t exps = 0;
  constexpr int BITS = GRAD >= PACKED ? GRAD - PACKED : 1;
  constexpr int WORKERS = BITS == 0 ? 4 : 8;  // workers whose codes a thread has on their way at a time
  using Word = std::conditional_t<(BITS >= 1 && BITS <= 4), uint32_t, uint64_t>;
  Word lo[WORKERS], hi[WORKERS];
  const int b = BITS == 0 ? a.b : BITS;
  const uint32_t* w = a.codes + c.word_off;
  auto fetch = [&](int worker, Word& l, Word& h) {
    uint64_t x, y;
    load_chunk<BITS>(w + (int64_t)worker * a.stride_words, j >> 3, b, c.pad_words, x, y);
    l = (Word)x; h = (Word)y;
  };
  auto fetch_group = [&](int first, Word (&l)[WORKERS], Word (&h)[WORKERS]) {  // those of WORKERS workers that there are
    if (first + WORKERS <= a.N) {
#pragma unroll
      for (int i = 0; i < WORKERS; ++i) fetch(first + i, l[i], h[i]);
    } else {
#pragma unroll
      for (int i = 0; i < WORKERS; ++i)
        if (first + i < a.N) fetch(first + i, l[i], h[i]);
    }
  };
  load8(pj, at, p_at, p);
  if constexpr (BITS8) {
    if (at.n > 0) {
      cm = *reinterpret_cast<const uint2*>(m8);
      cv = *reinterpret_cast<const uint2*>(v8);
    }
    exps = reinterpret_cast<const uint16_t*>(a.exps)[block];
  } else {
    load8(m32, at, m_at, m);
    load8(v32, at, v_at, v);
  }
  if constexpr (GRAD == LPC_F32) load8(gj, at, g_at, g);
  else if constexpr (GRAD < PACKED) load8(ghj, at, g_at, gh);
  else {
    if constexpr (BITS != 32) {
      if (at.n > 0) fetch_group(0, lo, hi);
    }
    if (a.mu) load8(muj, at, mu_at, mu);
  }
  if constexpr (CODES) {
    if (!p_at) turn(at, true, p);
    if constexpr (!BITS8) {
      if (!m_at) turn(at, true, m);
      if (!v_at) turn(at, true, v);
    }
    if constexpr (GRAD == LPC_F32) {
      if (!g_at) turn(at, true, g);
    } else if constexpr (GRAD < PACKED) {
      if (!g_at) turn(at, true, gh);
    } else {
      if (a.mu && !mu_at) turn(at, true, mu);
    }
  }

  if constexpr (GRAD == LPC_BF16 || GRAD == LPC_F16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = of_half<GRAD>(gh[e]);
  } else if constexpr (GRAD >= PACKED) {
    f32x2 acc[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = pack2(0.f, 0.f);
    if (at.n > 0) {
      if constexpr (BITS == 32) {
#pragma unroll 4
        for (int i = 0; i < a.N; ++i) {
          float k[8];
          load8f(reinterpret_cast<const float*>(w + (int64_t)i * a.stride_words), j, c.len, true, k);
          const float di = sdelta[i];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = fma2_rn(pack2(di, di), pack2(k[2 * e], k[2 * e + 1]), acc[e]);
        }
      } else {
        int i0 = 0;
#pragma unroll 1
        for (; i0 + WORKERS <= a.N; i0 += WORKERS) {  // the next eight workers' codes are asked for before these are added
          Word lo2[WORKERS], hi2[WORKERS];
          if (i0 + WORKERS < a.N) fetch_group(i0 + WORKERS, lo2, hi2);
#pragma unroll
          for (int i = 0; i < WORKERS; ++i) add_worker<BITS>(acc, sdelta[i0 + i], lo[i], hi[i], b);
#pragma unroll
          for (int i = 0; i < WORKERS; ++i) { lo[i] = lo2[i]; hi[i] = hi2[i]; }
        }
        if (i0 < a.N) {
#pragma unroll
          for (int i = 0; i < WORKERS; ++i)
            if (i0 + i < a.N) add_worker<BITS>(acc, sdelta[i0 + i], lo[i], hi[i], b);
        }
      }
    }
    const float invN = __fdiv_rn(1.0f, (float)a.divisor);
#pragma unroll
    for (int e = 0; e < 4; ++e) unpack2(mul2_rn(acc[e], pack2(invN, invN)), g[2 * e], g[2 * e + 1]);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = FAST || e < at.n ? add_rn(g[e], a.mu ? mu[e] : 0.f) : 0.f;  // behind the tensor there are codes, but no gradient
  }

  if constexpr (BITS8) {
    decode_moment<true>(cm, exps & 0xFFu, m);
    decode_moment<false>(cv, exps >> 8, v);
  }
  auto mul2 = [](float x, float y, float k0, float k1, float& u, float& w2) { unpack2(mul2_rn(pack2(x, y), pack2(k0, k1)), u, w2); };
  float m1[8], v1[8], p1[8];
  uint32_t top_m = 0, top_v = 0;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float x[2], q[2], y[2], z[2], d[2], o[2], r[2];
    mul2(g[e], g[e + 1], sc.gs, sc.gs, x[0], x[1]);
    mul2(x[0], x[1], x[0], x[1], q[0], q[1]);
    mul2(m[e], m[e + 1], a.b1, a.b1, y[0], y[1]);
    mul2(x[0], x[1], a.c1, a.c1, z[0], z[1]);
    m1[e] = add_rn(y[0], z[0]); m1[e + 1] = add_rn(y[1], z[1]);
    mul2(v[e], v[e + 1], a.b2, a.b2, y[0], y[1]);
    mul2(q[0], q[1], a.c2, a.c2, z[0], z[1]);
    v1[e] = add_rn(y[0], z[0]); v1[e + 1] = add_rn(y[1], z[1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      top_m = max(top_m, __float_as_uint(m1[e + h]) & 0x7FFFFFFFu);
      top_v = max(top_v, __float_as_uint(v1[e + h]));  // not negative, or NaN
      o[h] = root<BITS8>(v1[e + h]);
    }
    mul2(o[0], o[1], sc.second, sc.second, d[0], d[1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) r[h] = quotient<BITS8>(m1[e + h], add_rn(d[h], a.eps));
    mul2(r[0], r[1], sc.step, sc.step, r[0], r[1]);
    mul2(p[e], p[e + 1], sc.decay, sc.decay, y[0], y[1]);
    p1[e] = __fsub_rn(y[0], r[0]); p1[e + 1] = __fsub_rn(y[1], r[1]);
  }
  const bool beyond = warp_max_u32(max(top_m, top_v)) >= MOMENT_LIMIT;
  if (beyond || (BITS8 && sc.small_roots)) {  // some coordinates stay as they are, or all weights need another root: what they were is read again
    load8(pj, at, p_at, p);
    if (CODES && !p_at) turn(at, true, p);
    if constexpr (BITS8) {
      decode_moment<true>(cm, exps & 0xFFu, m);
      decode_moment<false>(cv, exps >> 8, v);
    } else {
      load8(m32, at, m_at, m);
      load8(v32, at, v_at, v);
      if (CODES && !m_at) turn(at, true, m);
      if (CODES && !v_at) turn(at, true, v);
    }
    top_m = top_v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool ok = fabsf(m1[e]) < __uint_as_float(MOMENT_LIMIT) && v1[e] < __uint_as_float(MOMENT_LIMIT);
      if (BITS8 && sc.small_roots)
        p1[e] = __fsub_rn(mul_rn(p[e], sc.decay), mul_rn(quotient<BITS8>(m1[e], add_rn(mul_rn(root_of_any(v1[e]), sc.second), a.eps)), sc.step));
      m1[e] = ok ? m1[e] : m[e];
      v1[e] = ok ? v1[e] : v[e];
      p1[e] = ok ? p1[e] : p[e];
      top_m = max(top_m, __float_as_uint(m1[e]) & 0x7FFFFFFFu);
      top_v = max(top_v, __float_as_uint(v1[e]) & 0x7FFFFFFFu);
    }
    if (beyond && at.lane == 0) atomicOr(a.dev_status, DEV_NONFINITE);
  }

  uint16_t h[8];
  if (a.copy) {
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = to_half(p1[e], a.copy_type);
    if (CODES && !copy_at) turn(at, false, h);
    store8(copyj, at, copy_at, h);
  }
  if (CODES && !p_at) turn(at, false, p1);
  store8(pj, at, p_at, p1);
  if constexpr (BITS8) {
    const uint32_t group = (uint32_t)((c.block0 * STEP_BLOCK + j) >> 3);
    const uint32_t em = min(max(warp_max_u32(top_m) >> 23, 1u), 253u), ev = min(max(warp_max_u32(top_v) >> 23, 1u), 253u);
    cm = encode_moment<true>(m1, stream_block(a.seed, TAG_MOMENT1, 0u, sc.t, group), em);
    cv = encode_moment<false>(v1, stream_block(a.seed, TAG_MOMENT2, 0u, sc.t, group), ev);
    if (at.n > 0) {
      *reinterpret_cast<uint2*>(m8) = cm;
      *reinterpret_cast<uint2*>(v8) = cv;
    }
    if (at.lane == 0) reinterpret_cast<uint16_t*>(a.exps)[block] = (uint16_t)(em | ev << 8);
  } else {
    if (CODES && !m_at) turn(at, false, m1);
    if (CODES && !v_at) turn(at, false, v1);
    store8(m32, at, m_at, m1);
    store8(v32, at, v_at, v1);
  }
}

template <int GRAD, bool BITS8>
__global__ void __launch_bounds__(ST, GRAD >= PACKED && !BITS8 ? 3 : 4) adamw_kernel(AdamwArgs a) {
  launch_dependents();
  wait_for_launch_before();
  extern __shared__ float sdelta[];
  __shared__ float sbias[2];
  __shared__ __align__(16) uint32_t sbuf[ST / 32][256];
  const StepChunk c = chunk_of(a);
  const int tid = threadIdx.x;
  BiasCorrection bc = a.bc;
  uint64_t t = a.t;
  if constexpr (GRAD >= PACKED)
    for (int i = tid; i < a.N; i += ST) sdelta[i] = a.delta[(int64_t)i * a.tensors + c.tensor];
  if (a.t_dev) {
    t += *a.t_dev;
    t = t ? t : 1;
    if (tid == 0) sbias[0] = __double2float_rn(__ddiv_rn(1.0, __dsub_rn(1.0, power_u64(a.beta1, t))));
    if (tid == 32) sbias[1] = __double2float_rn(__ddiv_rn(1.0, __dsqrt_rn(__dsub_rn(1.0, power_u64(a.beta2, t)))));
  }
  if (GRAD >= PACKED || a.t_dev) __syncthreads();
  if (a.t_dev) { bc.first = sbias[0]; bc.second = sbias[1]; }
  StepScalars sc;
  const float lr = mul_rn(a.lr_dev ? *a.lr_dev : a.lr, c.lr_scale);
  sc.decay = __fsub_rn(1.f, mul_rn(lr, c.weight_decay)); sc.step = mul_rn(lr, bc.first); sc.second = bc.second;
  sc.gs = a.grad_scale ? *a.grad_scale : 1.f;
  sc.t = t;
  sc.small_roots = mul_rn(sc.second, power_of_two(25 - 63)) > a.eps;  // a root below 2^-63 is more than 2^-25 of eps
  // a whole chunk of a tensor that starts on 16 bytes in every array takes code without a thought for anything else
  const int64_t at = c.off + (int64_t)c.chunk * STEP_CHUNK;
  bool fast = (int64_t)(c.chunk + 1) * STEP_CHUNK <= c.len && aligned16(a.p + at) && (!a.copy || aligned16(static_cast<const uint16_t*>(a.copy) + at));
  if constexpr (!BITS8) fast = fast && aligned16(static_cast<const float*>(a.m) + at) && aligned16(static_cast<const float*>(a.v) + at);
  if constexpr (GRAD == LPC_F32) fast = fast && aligned16(static_cast<const float*>(a.g) + at);
  else if constexpr (GRAD < PACKED) fast = fast && aligned16(static_cast<const uint16_t*>(a.g) + at);
  else fast = fast && (!a.mu || aligned16(a.mu + at));
  if (fast) adamw_chunk<GRAD, BITS8, true>(a, c, sc, sdelta, sbuf[tid >> 5]);
  else adamw_chunk<GRAD, BITS8, false>(a, c, sc, sdelta, sbuf[tid >> 5]);
}

// Three mantissa bits: what bfloat16 holds is the upper half of the float.  A block with a small exponent may have steps below 2^-133, where bfloat16 ends; its
// values, all below 2^-99, are rounded to the nearest multiple of that by a sum whose last place it is.  (By conversions, for all blocks: 65.8 us for 2^26 weights.)
template <bool SIGNED>
__device__ __forceinline__ void to_bf16(float* x, uint32_t exponent, uint16_t* h) {
  if (__builtin_expect(exponent < (SIGNED ? TOP_M : TOP_V) + 2 - 133 + 127, 0)) {
    const float c = mul_rn(1.5f, power_of_two(23 - 133));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __fsub_rn(add_rn(x[i], c), c);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = (uint16_t)(__float_as_uint(x[i]) >> 16);
}

template <bool FAST>
__device__ __forceinline__ void values_chunk(const AdamwArgs& a, const StepChunk& c, uint16_t* mo, uint16_t* vo, uint32_t* buf) {
  const int64_t j = (int64_t)c.chunk * STEP_CHUNK + threadIdx.x * 8;
  Place at;
  at.fast = FAST;
  at.lane = threadIdx.x & 31;
  at.count = FAST ? STEP_BLOCK : (int)max((int64_t)0, min((int64_t)STEP_BLOCK, c.len - (j - at.lane * 8)));
  at.n = FAST ? 8 : max(0, min(8, at.count - at.lane * 8));
  at.buf = buf;
  if (at.count == 0) return;
  uint2 cm = make_uint2(0u, 0u), cv = make_uint2(0u, 0u);
  if (at.n > 0) {
    cm = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.m) + c.block0 * STEP_BLOCK + j);
    cv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.v) + c.block0 * STEP_BLOCK + j);
  }
  const uint32_t e = reinterpret_cast<const uint16_t*>(a.exps)[c.block0 + (j >> 8)];
  mo += c.off + j;
  vo += c.off + j;
  const bool m_at = FAST || starts_on_16(mo, at), v_at = FAST || starts_on_16(vo, at);
  float x[8];
  uint16_t h[8];
  decode_moment<true>(cm, e & 0xFFu, x);
  to_bf16<true>(x, e & 0xFFu, h);
  if (!m_at) turn(at, false, h);
  store8(mo, at, m_at, h);
  decode_moment<false>(cv, e >> 8, x);
  to_bf16<false>(x, e >> 8, h);
  if (!v_at) turn(at, false, h);
  store8(vo, at, v_at, h);
}

__global__ void __launch_bounds__(ST) adamw_values_kernel(AdamwArgs a, uint16_t* m_out, uint16_t* v_out) {
  launch_dependents();
  wait_for_launch_before();
  __shared__ __align__(16) uint32_t sbuf[ST / 32][256];
  const StepChunk c = chunk_of(a);
  const int64_t at = c.off + (int64_t)c.chunk * STEP_CHUNK;
  const bool fast = (int64_t)(c.chunk + 1) * STEP_CHUNK <= c.len && aligned16(m_out + at) && aligned16(v_out + at);
  if (fast) values_chunk<true>(a, c, m_out, v_out, sbuf[threadIdx.x >> 5]);
  else values_chunk<false>(a, c, m_out, v_out, sbuf[threadIdx.x >> 5]);
}

template <int GRAD>
cudaError_t launch_of(const AdamwArgs& a, int state_bits, cudaStream_t st) {
  const size_t smem = GRAD >= PACKED ? (size_t)a.N * 4 : 0;
  return state_bits == 8 ? launch_overlapped(adamw_kernel<GRAD, true>, dim3((unsigned)a.nchunks), dim3(ST), smem, st, a)
                         : launch_overlapped(adamw_kernel<GRAD, false>, dim3((unsigned)a.nchunks), dim3(ST), smem, st, a);
}

}  // namespace

cudaError_t launch_adamw(const AdamwArgs& a, int state_bits, cudaStream_t st) {
  if (a.nchunks == 0) return cudaSuccess;
  if (a.g) {
    switch (a.g_type) {
      case LPC_F32: return launch_of<LPC_F32>(a, state_bits, st);
      case LPC_BF16: return launch_of<LPC_BF16>(a, state_bits, st);
      default: return launch_of<LPC_F16>(a, state_bits, st);
    }
  }
  switch (a.b) {
    case 1: return launch_of<PACKED + 1>(a, state_bits, st);
    case 2: return launch_of<PACKED + 2>(a, state_bits, st);
    case 3: return launch_of<PACKED + 3>(a, state_bits, st);
    case 4: return launch_of<PACKED + 4>(a, state_bits, st);
    case 8: return launch_of<PACKED + 8>(a, state_bits, st);
    case 32: return launch_of<PACKED + 32>(a, state_bits, st);
    default: return launch_of<PACKED>(a, state_bits, st);
  }
}

cudaError_t launch_adamw_values(const AdamwArgs& a, void* m_out, void* v_out, cudaStream_t st) {
  if (a.nchunks == 0) return cudaSuccess;
  return launch_overlapped(adamw_values_kernel, dim3((unsigned)a.nchunks), dim3(ST), 0, st, a, static_cast<uint16_t*>(m_out), static_cast<uint16_t*>(v_out));
}

}  // namespace lpc
