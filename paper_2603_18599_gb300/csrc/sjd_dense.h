// Shared by the window forward's dense operators: what a call gives the
// kernels (sjd_dense.cu, sjd_product.cu) and their launch entry points.
#pragma once

#include <atomic>
#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

#include "sjd.h"

namespace sjd_dense_ops {

constexpr int kMaxFeatures = 16384;  // of a row that is normed or quantised
constexpr int kMaxInput = 65536;     // of a product: |sum| <= 2^14 * 2^16 stays in an int32

// Rows of T elements apart by `stride` of them.
struct Rows {
  void* p;
  long long stride;
};

struct NormParams {
  Rows x, residual, y, h;   // residual.p NULL: none (nor h)
  const float* gain;        // NULL: 1
  const float* bias;        // NULL: 0
  int8_t* codes;
  float* scale;
  float eps;
  int rows, dim, centre;
};

enum NormMode { kNorm, kNormCodes, kCodes };

struct NormGradientParams {
  Rows dy, x, dh, dx;       // dh.p NULL: none
  const float* gain;
  float* dgain;
  float* dbias;             // NULL: not wanted
  float* parts;             // [blocks][1 or 2][dim]
  float eps;
  int rows, dim, centre, blocks;
};

struct EmbedParams {
  Rows table, y;
  const int32_t* tokens;
  float scale;
  int rows, dim, vocab;
};

struct EmbedGradientParams {
  Rows dy;
  const int32_t* tokens;
  float* grad;              // [vocab][dim]
  int32_t* first;           // [vocab + 1]: where each id's places begin in `places`
  int32_t* places;          // [rows]: the rows of each id, ascending
  int4* many;               // [lists][1 + ids of a list]: how many ids have many rows; of each the id, where its places begin, how many
  float scale;
  int rows, dim, vocab;
  int few;                  // an id with more rows is one of many
};

// A packed weight: a header, the channels' scales and the codes in tiles of
// kTileOut channels x kTileIn features, one after another along the features.
// In a tile a channel's kTileIn codes are neighbours, in pieces of 16 that
// stand in the order piece ^ (channel / 2 % 4), so that eight channels' pieces
// of one number lie in different banks; a code c is held as c + 128.
// Channels and features that fill up the last tiles are codes of 0.
constexpr int kTileOut = 128, kTileIn = 64;
constexpr int kTileBytes = kTileOut * kTileIn;
struct PackedHeader {
  uint32_t status;
  int32_t out, in;
  uint32_t reserved[61];
};
static_assert(sizeof(PackedHeader) == 256, "the codes begin on a 256-byte boundary");

struct Packed {
  PackedHeader* header;
  float* scale;        // [out]
  uint32_t* squares;   // [out, filled up to whole pairs of tiles]: the sum of the squares of a channel's codes
  unsigned char* codes;
  int out, in, tiles_out, tiles_in;  // (tiles of channels are a multiple of two)
};
inline size_t packed_layout(int out, int in, void* base, Packed* p) {
  const size_t pairs = (static_cast<size_t>(out) + 2 * kTileOut - 1) / (2 * kTileOut), tiles_in = (static_cast<size_t>(in) + kTileIn - 1) / kTileIn;
  const size_t channels = pairs * 2 * kTileOut, at_scale = sizeof(PackedHeader), at_squares = at_scale + channels * sizeof(float),
               at_codes = at_squares + channels * sizeof(uint32_t);
  unsigned char* b = static_cast<unsigned char*>(base);
  if (p) *p = {reinterpret_cast<PackedHeader*>(b), reinterpret_cast<float*>(b + at_scale), reinterpret_cast<uint32_t*>(b + at_squares), b + at_codes,
               out, in, static_cast<int>(pairs * 2), static_cast<int>(tiles_in)};
  return at_codes + channels * tiles_in * kTileIn;
}

struct ProductParams {
  Packed w;
  const int8_t* codes;
  long long codes_stride;
  const float* scale;
  const float* bias;
  Rows residual;   // p NULL: none
  Rows y;
  int rows;
};

// Lets a kernel's launches on the current device take up to `most` bytes of dynamic shared
// memory, whatever one of them asks for. The limit is the kernel's on the device, not the call's:
// were it set to what each call needs, another host thread could lower it between a call's setting and
// its launch. So it is the same for all calls of a kernel, and set once a device (it costs as much as a launch).
template <auto Kernel>
cudaError_t allow_shared(int most) {
  static std::atomic<uint64_t> allowed{0};
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess || (device < 64 && (allowed.load(std::memory_order_acquire) >> device & 1))) return e;
  e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  if (e == cudaSuccess && device < 64) allowed.fetch_or(1ull << device, std::memory_order_release);
  return e;
}

cudaError_t launch_norm(const NormParams& p, int mode, int dtype, int sms, cudaStream_t s);
int norm_gradient_blocks(int rows, int dim, int dtype, int sms);
cudaError_t launch_norm_gradient(const NormGradientParams& p, int dtype, cudaStream_t s);
cudaError_t launch_embed(const EmbedParams& p, int table_dtype, int dtype, cudaStream_t s);
constexpr int kListIds = 256;  // ids of a list
int embed_gradient_lists(int vocab);
cudaError_t launch_embed_gradient(const EmbedGradientParams& p, int dtype, int sms, cudaStream_t s);
cudaError_t launch_pack(const int8_t* w, long long stride, const float* scale, const Packed& to, cudaStream_t s);
size_t product_scratch_bytes(int rows, int out, int in, int sms);
cudaError_t launch_product(const ProductParams& p, int dtype, int sms, unsigned char* scratch, cudaStream_t s);

}  // namespace sjd_dense_ops
