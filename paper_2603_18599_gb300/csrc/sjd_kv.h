// Shared by the window forward's operators: what a call gives the kernels
// (sjd_kv.cu, sjd_attend.cu) and their launch entry points.
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

#include "sjd.h"

namespace sjd_kv_ops {

constexpr int kMaxAxes = 8;
constexpr int kMaxDim = 128;      // head size of a cache
constexpr int kMaxRotateDim = 256;
constexpr int kMaxAttendBlocks = 160;  // blocks of the attention kernel, one per SM

// Error bits of the handle's status word: bit (code - 1).
__host__ __device__ constexpr uint32_t status_bit(int code) { return 1u << (code - 1); }

struct View {
  void* p;
  long long sb, st, sh;  // strides of sequence, token and head, in elements
};

// The cache and the spans of one call.
struct Cache {
  int B, Hq, Hkv, D, ps, n_pages, max_pages;
  void* k;
  void* v;
  float* ks;
  float* vs;
  const int32_t* table;
  const int32_t* start;
  const int32_t* count;
  int n;
  uint32_t* status;
  int group;                     // query heads of a key head
  uint32_t ps_mul, group_mul;    // x / ps = x * ps_mul >> (31 + ps_shift) below 2^31, and so for group
  int ps_shift, group_shift;
};

struct Rope {
  const uint64_t* turns;
  const int32_t* axis;
  const int32_t* positions;
  int pairs, axes, interleaved, inverse;
  uint32_t* status;  // NULL: a call without a handle
};

struct RotateParams {
  Rope rope;
  View x, y;
  int B, n, H, D;
};

struct WriteParams {
  Cache c;
  View k, v, q, q_out;  // q.p NULL: no queries
  Rope rope;            // turns NULL: no rotation
};

struct ReadParams {
  Cache c;
  void* k_out;
  void* v_out;
};

struct AttendParams {
  Cache c;
  View q;
  int mask_kind;
  const uint8_t* mask;
  long long mask_b, mask_r;
  float scale;
  void* o;
  float* lse;
};

// x / d = x * mul >> (31 + shift) for x < 2^31: shift = ceil(log2 d), mul =
// ceil(2^(31 + shift) / d) is above the true factor by less than 2^-31 of it.
struct Divisor {
  uint32_t mul;
  int shift;
};
inline Divisor divisor(int d) {
  int shift = 0;
  while ((1ll << shift) < d) ++shift;
  return {static_cast<uint32_t>(((1ull << (31 + shift)) + d - 1) / d), shift};
}

// Launches a kernel that may start while the one before it on the stream
// drains (it calls wait_for_previous).
template <typename... Args, typename... Given>
cudaError_t launch_early(void (*kernel)(Args...), dim3 grid, int threads, size_t shared, cudaStream_t s, Given&&... given) {
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t at = {};
  at.gridDim = grid;
  at.blockDim = dim3(threads);
  at.dynamicSmemBytes = shared;
  at.stream = s;
  at.attrs = &early;
  at.numAttrs = 1;
  return cudaLaunchKernelEx(&at, kernel, static_cast<Args>(given)...);
}

// kv_dtype of the cache: SJD_BF16, SJD_E4M3, SJD_S8; dtype of the caller's tensors: SJD_F32, SJD_BF16.
cudaError_t launch_rotate(const RotateParams& p, int dtype, int sms, cudaStream_t s);
cudaError_t launch_write(const WriteParams& p, int dtype, int kv_dtype, int sms, cudaStream_t s);
cudaError_t launch_read(const ReadParams& p, int dtype, int kv_dtype, int sms, cudaStream_t s);
// scratch: attend_scratch_bytes(head_dim, max_new * heads / kv_heads), 256-byte aligned.
cudaError_t launch_attend(const AttendParams& p, int kv_dtype, int sms, unsigned char* scratch, cudaStream_t s);
// Sets the kernels' limits on the current device, once for a handle.
cudaError_t prepare_attend(int kv_dtype, int head_dim);
size_t attend_scratch_bytes(int head_dim, long long rows);
size_t attend_counter_bytes();  // the scratch's beginning, which is to be 0 before the first call

}  // namespace sjd_kv_ops
