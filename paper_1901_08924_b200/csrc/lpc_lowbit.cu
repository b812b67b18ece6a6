// C entry points (include/lpc.h) of the AdamW step over many tensors and of the products with packed 4-bit rows: argument checks, the
// table of a step's chunks, launches.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "../../include/lpc.h"
#include "lpc_adamw.h"
#include "lpc_ctx_view.h"
#include "lpc_kernels.h"
#include "lpc_matvec.h"

using namespace lpc;

struct lpc_adamw {
  lpc_ctx* ctx = nullptr;
  int device = 0;
  int64_t len = 0;
  int state_bits = 32;
  int64_t stride_words = 0;  // words of a worker's packed message, for the context's code width
  AdamwArgs args = {};       // what does not change from step to step
  StepChunk* chunks = nullptr;
};

namespace {

bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
size_t type_size(int type) { return type == LPC_F32 ? 4 : 2; }
bool valid_type(int type) { return type == LPC_F32 || type == LPC_BF16 || type == LPC_F16; }

bool valid_offsets(int64_t len, const int64_t* offs, int nseg) {
  if (len < 0 || nseg < 1) return false;
  if (!offs) return nseg == 1;
  if (offs[0] != 0 || offs[nseg] != len) return false;
  for (int s = 0; s < nseg; ++s)
    if (offs[s + 1] < offs[s]) return false;
  return true;
}

struct Profile {
  lpc_ctx* c;
  Profile(lpc_ctx* ctx, int kind) : c(ctx) { ctx_profile(c, kind, 1); }
  ~Profile() { ctx_profile(c, 0, 0); }
};

int cuda_status(lpc_ctx* c, cudaError_t e) { return e == cudaSuccess ? LPC_OK : ctx_fail(c, LPC_ERR_CUDA, cudaGetErrorString(e)); }

// The moments, the weights and the scalars of a step; fills what a launch needs of them.
int step_args(const lpc_adamw* h, AdamwArgs& a, float* p, void* m, void* v, uint8_t* exps, uint64_t t, float lr, const float* lr_dev,
              const uint64_t* t_dev, const float* grad_scale, void* copy_out, int copy_type) {
  lpc_ctx* c = h->ctx;
  if (h->len > 0 && (!p || !m || !v || (h->state_bits == 8 && !exps))) return ctx_fail(c, LPC_ERR_INVALID_ARG, "null weights or moments");
  if (!aligned_to(p, 4) || !aligned_to(m, h->state_bits == 8 ? 16 : 4) || !aligned_to(v, h->state_bits == 8 ? 16 : 4) || !aligned_to(exps, 2))
    return ctx_fail(c, LPC_ERR_INVALID_ARG, "alignment of weights or moments");
  if (t < 1 && !t_dev) return ctx_fail(c, LPC_ERR_INVALID_ARG, "steps count from 1");
  if (!lr_dev && !(lr >= 0.f && std::isfinite(lr))) return ctx_fail(c, LPC_ERR_INVALID_ARG, "lr");
  if (!aligned_to(lr_dev, 4) || !aligned_to(t_dev, 8) || !aligned_to(grad_scale, 4)) return ctx_fail(c, LPC_ERR_INVALID_ARG, "alignment of a device scalar");
  if (copy_out && copy_type != LPC_BF16 && copy_type != LPC_F16) return ctx_fail(c, LPC_ERR_INVALID_ARG, "the copy is LPC_BF16 or LPC_F16");
  if (!aligned_to(copy_out, 2)) return ctx_fail(c, LPC_ERR_INVALID_ARG, "alignment of the copy");
  a = h->args;
  a.p = p; a.m = m; a.v = v; a.exps = exps;
  a.t = t; a.lr = lr; a.lr_dev = lr_dev; a.t_dev = t_dev; a.grad_scale = grad_scale;
  a.copy = copy_out; a.copy_type = copy_type;
  if (!t_dev) {
    a.bc.first = (float)(1.0 / (1.0 - power_u64(a.beta1, t)));
    a.bc.second = (float)(1.0 / std::sqrt(1.0 - power_u64(a.beta2, t)));
  }
  const CtxView view = ctx_view(c);
  a.seed = view.seed; a.dev_status = view.dev_status;
  return LPC_OK;
}

int matvec_args(lpc_ctx* c, MatvecArgs& a, const uint32_t* codes, const float* delta, int64_t rows, int64_t cols, int64_t group, const void* x,
                int type, int64_t M, int64_t ldx, void* y, int64_t ldy, bool transposed) {
  const CtxView view = ctx_view(c);
  if (view.b != 4) return ctx_fail(c, LPC_ERR_UNSUPPORTED, "products with packed rows need 4-bit codes");
  if (rows < 0 || cols < 0 || M < 0) return ctx_fail(c, LPC_ERR_INVALID_ARG, "sizes");
  if (rows > (1 << 30) || cols > (1 << 25) || M > 65535)
    return ctx_fail(c, LPC_ERR_UNSUPPORTED, "more than 2^30 rows, 2^25 columns or 65,535 vectors");
  if (group < 0 || group % 32 != 0) return ctx_fail(c, LPC_ERR_INVALID_ARG, "a group is a multiple of 32 columns, or 0 for a whole row");
  if (!valid_type(type)) return ctx_fail(c, LPC_ERR_INVALID_ARG, "type");
  const int64_t in = transposed ? rows : cols, out = transposed ? cols : rows;
  if (ldx < in || ldy < out) return ctx_fail(c, LPC_ERR_INVALID_ARG, "row stride of a vector");
  if ((rows > 0 && cols > 0 && (!codes || !delta)) || (M > 0 && ((in > 0 && !x) || (out > 0 && !y)))) return ctx_fail(c, LPC_ERR_INVALID_ARG, "null matrix or vector");
  if (!aligned_to(codes, 16) || !aligned_to(delta, 4)) return ctx_fail(c, LPC_ERR_INVALID_ARG, "codes must be 16-byte aligned");
  if (!aligned_to(x, type_size(type)) || !aligned_to(y, type_size(type))) return ctx_fail(c, LPC_ERR_INVALID_ARG, "alignment of a vector");
  a.codes = codes; a.delta = delta;
  a.rows = (int)rows; a.cols = (int)cols;
  a.stride_words = ((cols + 7) / 8 + 3) / 4 * 4;
  // one scale per row: any group that covers the row says so, and whole blocks of 128 columns are the fast ones
  a.group = (int)(group > 0 && group < cols ? group : std::max<int64_t>((cols + 127) / 128 * 128, 128));
  a.groups = (int)((cols + a.group - 1) / a.group);
  a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy; a.M = (int)M; a.type = type; a.sm_count = view.sm_count;
  return LPC_OK;
}

}  // namespace

extern "C" {

int lpc_adamw_state_size(int64_t len, const int64_t* seg_offsets, int32_t nseg, int32_t state_bits, int64_t* values_out, int64_t* exps_out) {
  if (!values_out || !exps_out || !valid_offsets(len, seg_offsets, nseg)) return LPC_ERR_INVALID_ARG;
  if (state_bits != 8 && state_bits != 32) return LPC_ERR_INVALID_ARG;
  if (state_bits == 32) {
    *values_out = len;
    *exps_out = 0;
    return LPC_OK;
  }
  int64_t blocks = 0;
  for (int s = 0; s < nseg; ++s) blocks += ((seg_offsets ? seg_offsets[s + 1] - seg_offsets[s] : len) + STEP_BLOCK - 1) / STEP_BLOCK;
  *values_out = blocks * STEP_BLOCK;
  *exps_out = blocks * 2;
  return LPC_OK;
}

int lpc_adamw_create(lpc_adamw** out, lpc_ctx* ctx, int64_t len, const int64_t* seg_offsets, int32_t nseg, int32_t state_bits, double beta1,
                     double beta2, float eps, const float* weight_decay, const float* lr_scale) {
  if (!out) return LPC_ERR_INVALID_ARG;
  *out = nullptr;
  if (!ctx) return LPC_ERR_INVALID_ARG;
  if (!valid_offsets(len, seg_offsets, nseg)) return ctx_fail(ctx, LPC_ERR_INVALID_ARG, "offsets of the tensors");
  if (state_bits != 8 && state_bits != 32) return ctx_fail(ctx, LPC_ERR_INVALID_ARG, "moments have 8 or 32 bits");
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return ctx_fail(ctx, LPC_ERR_INVALID_ARG, "beta1 and beta2 are in [0, 1)");
  if (!((float)beta1 < 1.f) || !((float)beta2 < 1.f)) return ctx_fail(ctx, LPC_ERR_INVALID_ARG, "beta1 or beta2 rounds to 1");
  // with 8-bit moments the quotient's approximation gives 0 for divisors above 2^126
  if (!(eps > 0.f) || !std::isfinite(eps) || (state_bits == 8 && !(eps >= 1e-10f && eps <= 0x1p125f)))
    return ctx_fail(ctx, LPC_ERR_INVALID_ARG, "eps is above 0, with 8-bit moments from 1e-10 to 2^125");
  for (int s = 0; s < nseg; ++s) {
    if (weight_decay && !(weight_decay[s] >= 0.f && std::isfinite(weight_decay[s]))) return ctx_fail(ctx, LPC_ERR_INVALID_ARG, "weight decay");
    if (lr_scale && !(lr_scale[s] >= 0.f && std::isfinite(lr_scale[s]))) return ctx_fail(ctx, LPC_ERR_INVALID_ARG, "lr scale");
  }
  const CtxView view = ctx_view(ctx);
  const DeviceScope on(view.device);
  lpc_adamw* h = nullptr;
  try {
    std::vector<int64_t> words((size_t)nseg + 1);
    int64_t stride = 0;
    if (lpc_packed_layout(len, view.b, seg_offsets, nseg, words.data(), &stride) != LPC_OK) return ctx_fail(ctx, LPC_ERR_UNSUPPORTED, "vector too long");
    int64_t nchunks = 0, block = 0;
    for (int s = 0; s < nseg; ++s) nchunks += ((seg_offsets ? seg_offsets[s + 1] - seg_offsets[s] : len) + STEP_CHUNK - 1) / STEP_CHUNK;
    if (nchunks > INT32_MAX) return ctx_fail(ctx, LPC_ERR_UNSUPPORTED, "vector too long");
    std::vector<StepChunk> table;
    if (nseg > 1) table.reserve((size_t)nchunks);
    h = new lpc_adamw();
    for (int s = 0; s < nseg; ++s) {
      StepChunk k = {};
      k.off = seg_offsets ? seg_offsets[s] : 0;
      k.len = (seg_offsets ? seg_offsets[s + 1] : len) - k.off;
      k.word_off = words[s];
      k.pad_words = words[s + 1] - words[s];
      k.block0 = block;
      k.tensor = s;
      k.lr_scale = lr_scale ? lr_scale[s] : 1.f;
      k.weight_decay = weight_decay ? weight_decay[s] : 0.f;
      block += (k.len + STEP_BLOCK - 1) / STEP_BLOCK;
      if (nseg == 1) { h->args.only = k; continue; }
      for (int64_t i = 0; i * STEP_CHUNK < k.len; ++i) {
        k.chunk = (int32_t)i;
        table.push_back(k);
      }
    }
    if (block * STEP_BLOCK / 8 > 0xFFFFFFFFll) {  // the rounding streams count 8 coordinates a block, in 32 bits
      delete h;
      return ctx_fail(ctx, LPC_ERR_UNSUPPORTED, "vector too long");
    }
    h->ctx = ctx; h->device = view.device; h->len = len; h->state_bits = state_bits; h->stride_words = stride;
    h->args.nchunks = (int)nchunks; h->args.tensors = nseg;
    h->args.beta1 = beta1; h->args.beta2 = beta2; h->args.eps = eps;
    h->args.b1 = (float)beta1; h->args.c1 = (float)(1.0 - beta1); h->args.b2 = (float)beta2; h->args.c2 = (float)(1.0 - beta2);
    if (!table.empty()) {
      cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
      cudaError_t e = cudaStreamIsCapturing(view.stream, &cs);
      if (e == cudaSuccess && cs != cudaStreamCaptureStatusNone) {
        delete h;
        return ctx_fail(ctx, LPC_ERR_UNSUPPORTED, "make the step's handle outside a capture");
      }
      const size_t bytes = table.size() * sizeof(StepChunk);
      if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&h->chunks), bytes);
      if (e == cudaSuccess) e = cudaMemcpyAsync(h->chunks, table.data(), bytes, cudaMemcpyHostToDevice, view.stream);
      if (e == cudaSuccess) e = cudaStreamSynchronize(view.stream);  // the table is gone after this call
      if (e != cudaSuccess) {
        cudaGetLastError();
        if (h->chunks) cudaFree(h->chunks);
        delete h;
        return cuda_status(ctx, e);
      }
      h->args.chunks = h->chunks;
    }
  } catch (...) {
    delete h;
    return ctx_fail(ctx, LPC_ERR_UNSUPPORTED, "out of host memory");
  }
  *out = h;
  return LPC_OK;
}

int lpc_adamw_destroy(lpc_adamw* h) {
  if (!h) return LPC_OK;
  const DeviceScope on(h->device);
  if (h->chunks) cudaFree(h->chunks);  // waits for the device
  delete h;
  return LPC_OK;
}

int lpc_adamw_step(lpc_adamw* h, float* p, const void* g, int g_type, void* m, void* v, uint8_t* exps, uint64_t t, float lr,
                   const float* lr_dev, const uint64_t* t_dev, const float* grad_scale, void* copy_out, int copy_type) {
  if (!h) return LPC_ERR_INVALID_ARG;
  AdamwArgs a;
  const int rc = step_args(h, a, p, m, v, exps, t, lr, lr_dev, t_dev, grad_scale, copy_out, copy_type);
  if (rc != LPC_OK) return rc;
  if (!valid_type(g_type)) return ctx_fail(h->ctx, LPC_ERR_INVALID_ARG, "type of the gradient");
  if (h->len > 0 && !g) return ctx_fail(h->ctx, LPC_ERR_INVALID_ARG, "null gradient");
  if (!aligned_to(g, type_size(g_type))) return ctx_fail(h->ctx, LPC_ERR_INVALID_ARG, "alignment of the gradient");
  if (h->len == 0) return LPC_OK;
  a.g = g; a.g_type = g_type;
  const CtxView view = ctx_view(h->ctx);
  const DeviceScope on(view.device);
  Profile scope(h->ctx, LPC_KERNEL_OTHER);
  return cuda_status(h->ctx, launch_adamw(a, h->state_bits, view.stream));
}

int lpc_unpack_average_adamw(lpc_adamw* h, const uint32_t* codes, const float* delta, const float* mu, float* p, void* m, void* v, uint8_t* exps,
                             uint64_t t, float lr, const float* lr_dev, const uint64_t* t_dev, const float* grad_scale, void* copy_out,
                             int copy_type) {
  if (!h) return LPC_ERR_INVALID_ARG;
  AdamwArgs a;
  const int rc = step_args(h, a, p, m, v, exps, t, lr, lr_dev, t_dev, grad_scale, copy_out, copy_type);
  if (rc != LPC_OK) return rc;
  if (h->len > 0 && (!codes || !delta)) return ctx_fail(h->ctx, LPC_ERR_INVALID_ARG, "null messages");
  if (!aligned_to(codes, 16) || !aligned_to(delta, 4)) return ctx_fail(h->ctx, LPC_ERR_INVALID_ARG, "codes must be 16-byte aligned");
  if (!aligned_to(mu, 4)) return ctx_fail(h->ctx, LPC_ERR_INVALID_ARG, "alignment of mu");
  if (h->len == 0) return LPC_OK;
  const CtxView view = ctx_view(h->ctx);
  a.g = nullptr;
  a.codes = codes; a.stride_words = h->stride_words; a.delta = delta; a.mu = mu;
  a.N = view.N; a.b = view.b; a.divisor = view.divisor;
  const DeviceScope on(view.device);
  Profile scope(h->ctx, LPC_KERNEL_AGGREGATE);
  return cuda_status(h->ctx, launch_adamw(a, h->state_bits, view.stream));
}

int lpc_adamw_state_values(lpc_adamw* h, const void* m, const void* v, const uint8_t* exps, void* m_out, void* v_out) {
  if (!h) return LPC_ERR_INVALID_ARG;
  if (h->state_bits != 8) return ctx_fail(h->ctx, LPC_ERR_UNSUPPORTED, "moments in 32 bits are their own values");
  if (h->len == 0) return LPC_OK;
  if (!m || !v || !exps || !m_out || !v_out) return ctx_fail(h->ctx, LPC_ERR_INVALID_ARG, "null moments or output");
  if (!aligned_to(m, 16) || !aligned_to(v, 16) || !aligned_to(exps, 2) || !aligned_to(m_out, 2) || !aligned_to(v_out, 2))
    return ctx_fail(h->ctx, LPC_ERR_INVALID_ARG, "alignment of moments or output");
  AdamwArgs a = h->args;
  a.m = const_cast<void*>(m); a.v = const_cast<void*>(v); a.exps = const_cast<uint8_t*>(exps);
  const CtxView view = ctx_view(h->ctx);
  const DeviceScope on(view.device);
  Profile scope(h->ctx, LPC_KERNEL_OTHER);
  return cuda_status(h->ctx, launch_adamw_values(a, m_out, v_out, view.stream));
}

int lpc_packed_matvec(lpc_ctx* c, const uint32_t* codes, const float* delta, int64_t rows, int64_t cols, int64_t group, const void* X, int type,
                      int64_t M, int64_t ldx, void* Y, int64_t ldy) {
  if (!c) return LPC_ERR_INVALID_ARG;
  MatvecArgs a;
  const int rc = matvec_args(c, a, codes, delta, rows, cols, group, X, type, M, ldx, Y, ldy, false);
  if (rc != LPC_OK) return rc;
  if (M == 0 || rows == 0) return LPC_OK;
  const CtxView view = ctx_view(c);
  const DeviceScope on(view.device);
  Profile scope(c, LPC_KERNEL_OTHER);
  return cuda_status(c, launch_packed_matvec(a, view.stream));
}

int lpc_packed_matvec_t(lpc_ctx* c, const uint32_t* codes, const float* delta, int64_t rows, int64_t cols, int64_t group, const void* dY, int type,
                        int64_t M, int64_t ldy, void* dX, int64_t ldx) {
  if (!c) return LPC_ERR_INVALID_ARG;
  MatvecArgs a;
  const int rc = matvec_args(c, a, codes, delta, rows, cols, group, dY, type, M, ldy, dX, ldx, true);
  if (rc != LPC_OK) return rc;
  if (M == 0 || cols == 0) return LPC_OK;
  const CtxView view = ctx_view(c);
  const DeviceScope on(view.device);
  Profile scope(c, LPC_KERNEL_OTHER);
  return cuda_status(c, launch_packed_matvec_t(a, view.stream));
}

}  // extern "C"
