// Matrix products of 8-bit integers with scales per token and per channel:
// y[t][n] = sx[t] sw[n] sum_k x[t][k] w[n][k] + bias[n] + residual[t][n], the
// sum exact.

#include "sjd_dense.h"
#include "sjd_kv_device.cuh"

namespace sjd_dense_ops {

using sjd_kv_ops::launch_early;
using sjd_kv_ops::let_next_start;
using sjd_kv_ops::wait_for_previous;

namespace {

// A block packs one channel's codes: a tile's 128 at a time.
__global__ void __launch_bounds__(128) pack_kernel(const int8_t* w, long long stride, const float* scale, const Packed to) {
  __shared__ uint32_t words[4];
  wait_for_previous();
  let_next_start();
  const int channel = blockIdx.x, r = channel % kTileOut;
  unsigned char* tile = to.codes + static_cast<long long>(channel / kTileOut) * to.tiles_in * kTileBytes + r * kTileIn;
  uint32_t squares = 0;
  for (int k = threadIdx.x; k < to.tiles_in * kTileIn; k += 128) {
    const int c = channel < to.out && k < to.in ? w[channel * stride + k] : 0;
    squares += c * c;
    const int piece = (k % kTileIn) / 16 ^ (r % 8);
    tile[static_cast<long long>(k / kTileIn) * kTileBytes + piece * 16 + k % 16] = static_cast<unsigned char>(c + 128);
  }
  squares = __reduce_add_sync(0xffffffffu, squares);
  if (threadIdx.x % 32 == 0) words[threadIdx.x / 32] = squares;
  __syncthreads();
  if (threadIdx.x == 0) {
    to.squares[channel] = words[0] + words[1] + words[2] + words[3];
    to.scale[channel] = channel < to.out ? scale[channel] : 0.0f;
    if (channel == 0) *to.header = PackedHeader{0u, to.out, to.in, {}};
  }
}

// 64 channels x 64 tokens to a block, 4 x 4 to a thread.
template <typename T>
__global__ void __launch_bounds__(256) product_kernel(const ProductParams p) {
  __shared__ uint32_t ws[64][17], xs[64][17];
  wait_for_previous();
  let_next_start();
  const int n0 = blockIdx.x * 64, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const long long t0 = static_cast<long long>(blockIdx.y) * 64;
  int sum[4][4] = {};
  for (int k0 = 0; k0 < p.w.in; k0 += 64) {
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * 16; i += 256) {
      const int r = i / 16, word = i % 16, k = k0 + 4 * word;
      const unsigned char* tile = p.w.codes + (static_cast<long long>((n0 + r) / kTileOut) * p.w.tiles_in + k / kTileIn) * kTileBytes;
      const int c = (n0 + r) % kTileOut;
      ws[r][word] = *reinterpret_cast<const uint32_t*>(tile + c * kTileIn + ((k % kTileIn / 16) ^ (c % 8)) * 16 + k % 16) ^ 0x80808080u;
      uint32_t x = 0;
      if (t0 + r < p.rows) {
        const int8_t* row = p.codes + (t0 + r) * p.codes_stride;
        for (int j = 0; j < 4; ++j) {
          if (k + j < p.w.in) x |= static_cast<uint32_t>(row[k + j] & 0xff) << 8 * j;
        }
      }
      xs[r][word] = x;
    }
    __syncthreads();
    for (int word = 0; word < 16; ++word) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i][j] = __dp4a(static_cast<int>(ws[tx + 16 * i][word]), static_cast<int>(xs[ty + 16 * j][word]), sum[i][j]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const long long t = t0 + ty + 16 * j;
    if (t >= p.rows) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + tx + 16 * i;
      if (n >= p.w.out) continue;
      // (each step rounded by itself: the result is the same whichever way the sum was taken)
      float y = __fmul_rn(__fmul_rn(static_cast<float>(sum[i][j]), p.scale[t]), p.w.scale[n]);
      if (p.bias) y = __fadd_rn(y, p.bias[n]);
      if (p.residual.p) y = __fadd_rn(y, static_cast<float>(static_cast<const T*>(p.residual.p)[t * p.residual.stride + n]));
      static_cast<T*>(p.y.p)[t * p.y.stride + n] = static_cast<T>(y);
    }
  }
}

}  // namespace

cudaError_t launch_pack(const int8_t* w, long long stride, const float* scale, const Packed& to, cudaStream_t s) {
  return launch_early(pack_kernel, static_cast<unsigned>(to.tiles_out) * kTileOut, 128, 0, s, w, stride, scale, to);
}

size_t product_scratch_bytes(int rows, int out, int in, int sms) { return 256; }

cudaError_t launch_product(const ProductParams& p, int dtype, int sms, unsigned char* scratch, cudaStream_t s) {
  const dim3 grid((p.w.out + 63) / 64, (p.rows + 63) / 64);
  if (dtype == SJD_BF16) return launch_early(product_kernel<__nv_bfloat16>, grid, 256, 0, s, p);
  return launch_early(product_kernel<float>, grid, 256, 0, s, p);
}

}  // namespace sjd_dense_ops
