// Launch interface of the AdamW step over the tensors of one vector (lpc_adamw.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace lpc {

constexpr int STEP_CHUNK = 2048;  // coordinates per CTA: 256 threads with 8 consecutive ones each
constexpr int STEP_BLOCK = 256;   // coordinates of a tensor that share the exponents of their 8-bit moments: a warp's

// A chunk of a tensor, and the tensor.
struct __align__(16) StepChunk {
  int64_t off;        // first element of the tensor in the vector
  int64_t len;        // its elements
  int64_t word_off;   // first word of its packed stream inside a worker's stream
  int64_t pad_words;  // words reserved for it
  int64_t block0;     // first block of its 8-bit moments
  int32_t chunk;      // this is the tensor's chunk of that number
  int32_t tensor;
  float lr_scale, weight_decay;
  int64_t pad_;
};
static_assert(sizeof(StepChunk) == 64, "read as four 16-byte words");

// Bias corrections 1 / (1 - beta1^t) and 1 / sqrt(1 - beta2^t), formed in doubles: the power by repeated squaring, so that the host and a
// kernel get the same bits.
struct BiasCorrection { float first, second; };
__host__ __device__ inline double power_u64(double base, uint64_t t) {
  double r = 1.0;
  for (; t; t >>= 1) {
    if (t & 1) r *= base;
    base *= base;
  }
  return r;
}

struct AdamwArgs {
  const StepChunk* chunks;  // null for a vector of one tensor: `only`, with the CTA's number as the chunk
  StepChunk only;
  int nchunks;
  int tensors;
  float* p;
  const void* g;            // dense gradient (LPC_F32, LPC_BF16, LPC_F16); null: the packed messages below
  int g_type;
  void *m, *v;              // fp32, or codes
  uint8_t* exps;            // 8-bit moments: two bytes a block
  void* copy;               // nullable: 16-bit copy of the new weights
  int copy_type;
  double beta1, beta2;
  float b1, c1, b2, c2, eps;  // beta and 1 - beta in single precision
  float lr;
  BiasCorrection bc;
  uint64_t t;
  const float* lr_dev;      // nullable: takes the place of lr
  const uint64_t* t_dev;    // nullable: added to t
  const float* grad_scale;  // nullable
  uint64_t seed;
  // gradient from packed messages: their average, plus mu
  const uint32_t* codes;
  int64_t stride_words;
  const float* delta;
  int N, b, divisor;
  const float* mu;          // nullable
  unsigned int* dev_status;
};
cudaError_t launch_adamw(const AdamwArgs& a, int state_bits, cudaStream_t st);
// The values of 8-bit moments, in bfloat16 (three mantissa bits: exact where that is a normal number).
cudaError_t launch_adamw_values(const AdamwArgs& a, void* m_out, void* v_out, cudaStream_t st);

}  // namespace lpc
