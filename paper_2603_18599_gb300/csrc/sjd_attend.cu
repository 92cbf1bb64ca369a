// Attention of a chunk of new tokens over the paged cache.
//
// One warp takes one query row. It goes through the keys 32 at a time, one
// key to a lane for the scores, keeps the running maximum and sum, and then
// gathers the 32 weighted values with the head's elements spread over the
// lanes.

#include <cfloat>

#include "sjd_kv_device.cuh"

namespace sjd_kv_ops {

namespace {

constexpr int kRows = 4;  // query rows (warps) of a block

template <int KV>
__device__ __forceinline__ float value_at(const void* p, long long i) {
  if constexpr (KV == SJD_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  else if constexpr (KV == SJD_S8) return static_cast<float>(static_cast<const int8_t*>(p)[i]);
  else return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<const uint8_t*>(p)[i], __NV_E4M3)));
}

template <int KV>
__global__ void __launch_bounds__(32 * kRows) attend_kernel(const AttendParams p) {
  __shared__ float qs[kRows][kMaxDim];
  const Cache& c = p.c;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * kRows + warp;
  if (row >= static_cast<long long>(c.B) * c.n * c.Hq) return;
  const int h = static_cast<int>(row % c.Hq), t = static_cast<int>(row / c.Hq % c.n), b = static_cast<int>(row / c.Hq / c.n);
  const int kvh = h / (c.Hq / c.Hkv);
  const int2 span = span_of(c, b);
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q.p) + b * p.q.sb + t * p.q.st + h * p.q.sh;
  for (int i = lane; i < c.D; i += 32) qs[warp][i] = __bfloat162float(q[i]);
  __syncwarp();
  float acc[kMaxDim / 32] = {};
  float top = -INFINITY, sum = 0.0f;
  const int last = t >= span.y ? 0 : p.mask_kind == SJD_MASK_CAUSAL ? span.x + t + 1 : span.x + span.y;
  for (int k0 = 0; k0 < last; k0 += 32) {
    const int key = k0 + lane;
    bool seen = key < last;
    if (seen && p.mask_kind == SJD_MASK_GIVEN && key >= span.x)
      seen = p.mask[p.mask_b * b + p.mask_r * t + (key - span.x)] != 0;
    const long long slot = seen ? slot_of(c, b, key) : -1;
    const long long at = slot < 0 ? -1 : slot + static_cast<long long>(kvh) * c.ps;
    float s = -INFINITY;
    if (seen) {
      s = 0.0f;
      for (int i = 0; at >= 0 && i < c.D; ++i) s += qs[warp][i] * value_at<KV>(c.k, at * c.D + i);
      if (KV != SJD_BF16 && at >= 0) s *= c.ks[at];
      s *= p.scale;
    }
    float m = s;
    for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = fmaxf(m, top);
    const float base = m == -INFINITY ? 0.0f : m, old = expf(top - base);
    float w = seen ? expf(s - base) : 0.0f, total = w;
    for (int o = 16; o > 0; o /= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
    sum = sum * old + total;
    top = m;
#pragma unroll
    for (int i = 0; i < kMaxDim / 32; ++i) acc[i] *= old;
    const unsigned some = __ballot_sync(0xffffffffu, seen && at >= 0);
    if (KV != SJD_BF16 && seen && at >= 0) w *= c.vs[at];
    for (unsigned left = some; left; left &= left - 1) {
      const int j = __ffs(left) - 1;
      const float wj = __shfl_sync(0xffffffffu, w, j);
      const long long aj = __shfl_sync(0xffffffffu, at, j);
      for (int i = 0; i < kMaxDim / 32; ++i)
        if (lane + 32 * i < c.D) acc[i] += wj * value_at<KV>(c.v, aj * c.D + lane + 32 * i);
    }
  }
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.o) + row * c.D;
  for (int i = 0; i < kMaxDim / 32; ++i)
    if (lane + 32 * i < c.D) o[lane + 32 * i] = __float2bfloat16_rn(sum > 0.0f || sum != sum ? acc[i] / sum : 0.0f);
  if (p.lse && lane == 0) p.lse[row] = top + logf(sum);
}

}  // namespace

cudaError_t launch_attend(const AttendParams& p, int kv_dtype, cudaStream_t s) {
  const long long rows = static_cast<long long>(p.c.B) * p.c.n * p.c.Hq;
  const unsigned blocks = static_cast<unsigned>((rows + kRows - 1) / kRows);
  if (kv_dtype == SJD_BF16) attend_kernel<SJD_BF16><<<blocks, 32 * kRows, 0, s>>>(p);
  else if (kv_dtype == SJD_E4M3) attend_kernel<SJD_E4M3><<<blocks, 32 * kRows, 0, s>>>(p);
  else attend_kernel<SJD_S8><<<blocks, 32 * kRows, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace sjd_kv_ops
