// Host side of the dense operators declared in include/sjd.h: argument
// checks and launches.

#include <cmath>

#include "sjd_dense.h"
#include "sjd_kv.h"

using namespace sjd_dense_ops;

namespace {

constexpr size_t kAlign = 256;

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool floating(int dtype) { return dtype == SJD_F32 || dtype == SJD_BF16; }
size_t size_of(int dtype) { return dtype == SJD_BF16 ? 2 : 4; }

bool count_sms(int* sms) {  // of the current device
  int device = 0;
  return cudaGetDevice(&device) == cudaSuccess && cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device) == cudaSuccess;
}
int launched(cudaError_t e) { return e == cudaSuccess ? SJD_OK : SJD_ERR_CUDA; }

// Rows of `size` bytes an element that a call cannot do without, or may.
bool there(const sjd_rows* r, size_t size) { return r && r->data_dev && aligned(r->data_dev, size); }
bool absent_or_there(const sjd_rows* r, size_t size) { return !r || there(r, size); }
Rows rows_of(const sjd_rows* r) { return r ? Rows{r->data_dev, r->row_stride} : Rows{nullptr, 0}; }

bool valid(int rows, int dim) { return rows >= 1 && dim >= 1 && dim <= kMaxFeatures; }
bool valid_weight(int out, int in) { return out >= 1 && out <= (1 << 24) && in >= 1 && in <= kMaxInput; }

}  // namespace

extern "C" {

size_t sjd_weight_size(int32_t out, int32_t in) { return valid_weight(out, in) ? packed_layout(out, in, nullptr, nullptr) : 0; }

int sjd_weight_pack(const int8_t* w, int64_t row_stride, const float* scale, int32_t out, int32_t in, void* packed, size_t bytes, void* stream) {
  if (!w || !scale || !packed || !valid_weight(out, in) || !aligned(scale, 4) || !aligned(packed, kAlign)) return SJD_ERR_ARG;
  Packed to;
  if (bytes < packed_layout(out, in, packed, &to)) return SJD_ERR_CAPACITY;
  return launched(launch_pack(w, row_stride, scale, to, static_cast<cudaStream_t>(stream)));
}

int sjd_weight_sync(void* packed, void* stream) {
  if (!packed || !aligned(packed, kAlign)) return SJD_ERR_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint32_t bits = 0;
  cudaError_t e = cudaMemcpyAsync(&bits, packed, sizeof bits, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && bits) {
    e = cudaMemsetAsync(packed, 0, sizeof bits, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  }
  if (e != cudaSuccess) return SJD_ERR_CUDA;
  if (bits & sjd_kv_ops::status_bit(SJD_ERR_TIMEOUT)) return SJD_ERR_TIMEOUT;
  return bits ? SJD_ERR_BOUNDS : SJD_OK;
}

size_t sjd_product_workspace_size(int32_t rows, int32_t out, int32_t in) {
  int sms = 0;
  if (rows < 1 || !valid_weight(out, in) || !count_sms(&sms)) return 0;
  return product_scratch_bytes(rows, out, in, sms);
}

int sjd_product(const void* packed, int32_t out, int32_t in, const sjd_rows* codes, const float* scale, int32_t rows, const float* bias,
                const sjd_rows* residual, int32_t dtype, const sjd_rows* y, void* workspace, size_t ws_bytes, void* stream) {
  if (!packed || !aligned(packed, kAlign) || !valid_weight(out, in) || rows < 1 || !floating(dtype)) return SJD_ERR_ARG;
  if (!there(codes, 1) || !scale || !aligned(scale, 4) || !aligned(bias, 4) || !absent_or_there(residual, size_of(dtype)) ||
      !there(y, size_of(dtype)) || !aligned(workspace, kAlign))
    return SJD_ERR_ARG;
  int sms = 0;
  if (!count_sms(&sms)) return SJD_ERR_CUDA;
  const size_t needed = product_scratch_bytes(rows, out, in, sms);
  if (needed && !workspace) return SJD_ERR_ARG;
  if (ws_bytes < needed) return SJD_ERR_CAPACITY;
  ProductParams p{};
  packed_layout(out, in, const_cast<void*>(packed), &p.w);
  p.codes = static_cast<const int8_t*>(codes->data_dev);
  p.codes_stride = codes->row_stride;
  p.scale = scale;
  p.bias = bias;
  p.residual = rows_of(residual);
  p.y = rows_of(y);
  p.rows = rows;
  return launched(launch_product(p, dtype, sms, static_cast<unsigned char*>(workspace), static_cast<cudaStream_t>(stream)));
}

int sjd_quantise(const sjd_rows* x, int32_t rows, int32_t dim, int32_t dtype, int8_t* codes, float* scale, void* stream) {
  if (!valid(rows, dim) || !floating(dtype) || !there(x, size_of(dtype)) || !codes || !scale || !aligned(scale, 4)) return SJD_ERR_ARG;
  NormParams p{};
  p.x = rows_of(x);
  p.codes = codes;
  p.scale = scale;
  p.rows = rows;
  p.dim = dim;
  int sms = 0;
  if (!count_sms(&sms)) return SJD_ERR_CUDA;
  return launched(launch_norm(p, kCodes, dtype, sms, static_cast<cudaStream_t>(stream)));
}

int sjd_norm(const sjd_rows* x, const sjd_rows* residual, const float* gain, const float* bias, float eps, int32_t centre, int32_t rows, int32_t dim,
             int32_t dtype, const sjd_rows* h, const sjd_rows* y, int8_t* codes, float* scale, void* stream) {
  const size_t size = floating(dtype) ? size_of(dtype) : 0;
  if (!valid(rows, dim) || !size || !there(x, size) || !absent_or_there(residual, size) || !aligned(gain, 4) || !aligned(bias, 4)) return SJD_ERR_ARG;
  if (!(eps >= 0.0f && eps < INFINITY) || (centre != 0 && centre != 1)) return SJD_ERR_ARG;
  if ((residual != nullptr) != (h != nullptr) || !absent_or_there(h, size)) return SJD_ERR_ARG;
  // a norm, or its codes and scales
  if ((codes != nullptr) != (scale != nullptr) || (codes != nullptr) == (y != nullptr) || !absent_or_there(y, size) || !aligned(scale, 4))
    return SJD_ERR_ARG;
  const NormParams p{rows_of(x), rows_of(residual), rows_of(y), rows_of(h), gain, bias, codes, scale, eps, rows, dim, centre};
  int sms = 0;
  if (!count_sms(&sms)) return SJD_ERR_CUDA;
  return launched(launch_norm(p, codes ? kNormCodes : kNorm, dtype, sms, static_cast<cudaStream_t>(stream)));
}

size_t sjd_norm_gradient_workspace_size(int32_t rows, int32_t dim, int32_t dtype) {
  int sms = 0;
  if (!valid(rows, dim) || !floating(dtype) || !count_sms(&sms)) return 0;
  return 2 * sizeof(float) * dim * static_cast<size_t>(norm_gradient_blocks(rows, dim, dtype, sms));
}

int sjd_norm_gradient(const sjd_rows* dy, const sjd_rows* x, const float* gain, float eps, int32_t centre, const sjd_rows* dh, int32_t rows,
                      int32_t dim, int32_t dtype, const sjd_rows* dx, float* dgain, float* dbias, void* workspace, size_t ws_bytes, void* stream) {
  const size_t size = floating(dtype) ? size_of(dtype) : 0;
  if (!valid(rows, dim) || !size || !there(dy, size) || !there(x, size) || !there(dx, size) || !absent_or_there(dh, size)) return SJD_ERR_ARG;
  if (!(eps >= 0.0f && eps < INFINITY) || (centre != 0 && centre != 1)) return SJD_ERR_ARG;
  if (!aligned(gain, 4) || !dgain || !aligned(dgain, 4) || !aligned(dbias, 4) || !workspace || !aligned(workspace, kAlign)) return SJD_ERR_ARG;
  int sms = 0;
  if (!count_sms(&sms)) return SJD_ERR_CUDA;
  const int blocks = norm_gradient_blocks(rows, dim, dtype, sms);
  if (ws_bytes < 2 * sizeof(float) * dim * static_cast<size_t>(blocks)) return SJD_ERR_CAPACITY;
  const NormGradientParams p{rows_of(dy), rows_of(x), rows_of(dh), rows_of(dx), gain, dgain, dbias, static_cast<float*>(workspace), eps, rows, dim, centre, blocks};
  return launched(launch_norm_gradient(p, dtype, static_cast<cudaStream_t>(stream)));
}

int sjd_embed(const sjd_rows* table, int32_t vocab, int32_t table_dtype, const int32_t* tokens, int32_t rows, int32_t dim, float scale, int32_t dtype,
              const sjd_rows* y, void* stream) {
  if (rows < 1 || vocab < 1 || dim < 1 || dim > kMaxInput || !floating(dtype) || !floating(table_dtype)) return SJD_ERR_ARG;
  if (!there(table, size_of(table_dtype)) || !there(y, size_of(dtype)) || !tokens || !aligned(tokens, 4)) return SJD_ERR_ARG;
  const EmbedParams p{rows_of(table), rows_of(y), tokens, scale, rows, dim, vocab};
  return launched(launch_embed(p, table_dtype, dtype, static_cast<cudaStream_t>(stream)));
}

size_t sjd_embed_gradient_workspace_size(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1) return 0;
  return sizeof(int4) * embed_gradient_lists(vocab) * (1 + kListIds) + sizeof(int32_t) * (static_cast<size_t>(vocab) + 1 + static_cast<size_t>(rows));
}

int sjd_embed_gradient(const sjd_rows* dy, const int32_t* tokens, int32_t rows, int32_t dim, int32_t vocab, float scale, int32_t dtype, float* grad,
                       void* workspace, size_t ws_bytes, void* stream) {
  if (rows < 1 || vocab < 1 || dim < 1 || dim > kMaxInput || !floating(dtype)) return SJD_ERR_ARG;
  if (!there(dy, size_of(dtype)) || !tokens || !aligned(tokens, 4) || !grad || !aligned(grad, 4) || !workspace || !aligned(workspace, kAlign))
    return SJD_ERR_ARG;
  if (ws_bytes < sjd_embed_gradient_workspace_size(rows, vocab)) return SJD_ERR_CAPACITY;
  int4* many = static_cast<int4*>(workspace);
  int32_t* first = reinterpret_cast<int32_t*>(many + static_cast<size_t>(embed_gradient_lists(vocab)) * (1 + kListIds));
  const EmbedGradientParams p{rows_of(dy), tokens, grad, first, first + vocab + 1ll, many, scale, rows, dim, vocab, rows <= 32 ? 32 : 8};
  int sms = 0;
  if (!count_sms(&sms)) return SJD_ERR_CUDA;
  return launched(launch_embed_gradient(p, dtype, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
