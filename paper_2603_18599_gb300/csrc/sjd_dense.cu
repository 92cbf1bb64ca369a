// The window forward's operators on rows of features: norms with a residual,
// their codes of 8 bits and their gradient, the embedding of tokens and its
// gradient. All of them move rows through once and are bound by HBM in long
// calls and by one chain of loads and sums in short ones.
//
// A row is taken by a group of G threads, C pieces of 8 features to a thread,
// and stays in their registers from its load to its store: its mean, the mean
// of the squares around it (both as sums of the differences themselves, so
// that nothing cancels) and its largest magnitude are sums over the group.

#include <cfloat>

#include "sjd_dense.h"
#include "sjd_kv_device.cuh"

namespace sjd_dense_ops {

using sjd_kv_ops::launch_early;
using sjd_kv_ops::let_next_start;
using sjd_kv_ops::pack_bf16;
using sjd_kv_ops::unpack_bf16;
using sjd_kv_ops::wait_for_previous;

namespace {

// Feature j of piece i of a thread: neighbours where a row can be accessed 16
// bytes at a time (`W`), else every G-th, so that a warp's accesses of single
// elements lie side by side.
template <bool W>
__device__ __forceinline__ int feature(int i, int j, int lane, int G) {
  return W ? (i * G + lane) * 8 + j : (i * 8 + j) * G + lane;
}

template <bool W, typename T>
__device__ __forceinline__ void load8(const T* row, int i, int lane, int G, int D, float (&v)[8]) {
  if constexpr (W) {
    const int e = (i * G + lane) * 8;
    if (e >= D) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.0f;
    } else if constexpr (sizeof(T) == 2) {
      const uint4 u = *reinterpret_cast<const uint4*>(row + e);
      const float2 a = unpack_bf16(u.x), b = unpack_bf16(u.y), c = unpack_bf16(u.z), d = unpack_bf16(u.w);
      v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
    } else {
      const float4 a = *reinterpret_cast<const float4*>(row + e), b = *reinterpret_cast<const float4*>(row + e + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = feature<false>(i, j, lane, G);
      v[j] = e < D ? static_cast<float>(row[e]) : 0.0f;
    }
  }
}

template <bool W, typename T>
__device__ __forceinline__ void store8(T* row, int i, int lane, int G, int D, const float (&v)[8]) {
  if constexpr (W) {
    const int e = (i * G + lane) * 8;
    if (e >= D) return;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(row + e) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
      *reinterpret_cast<float4*>(row + e) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(row + e + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = feature<false>(i, j, lane, G);
      if (e < D) row[e] = static_cast<T>(v[j]);
    }
  }
}

// Vectors of one float a feature (gains), which are 16-byte aligned where rows are.
template <bool W>
__device__ __forceinline__ void load_vector(const float* p, float otherwise, int i, int lane, int G, int D, float (&v)[8]) {
  if (p) {
    load8<W>(p, i, lane, G, D, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = otherwise;
  }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Sums over the group of G threads: a warp, or the whole block. `turn`
// numbers the sums of a block: two neighbours take different words of `words`
// [2][N][32], so that one barrier a sum is enough.
template <int N>
__device__ __forceinline__ void group_sum(float (&x)[N], int G, float* words, int& turn) {
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = warp_sum(x[k]);
  if (G == 32) return;
  float* w = words + (turn & 1) * 64;
  ++turn;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) w[32 * k + threadIdx.x / 32] = x[k];
  }
  __syncthreads();
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = warp_sum(lane < G / 32 ? w[32 * k + lane] : 0.0f);
}
__device__ __forceinline__ uint32_t group_max(uint32_t x, int G, float* words, int& turn) {
  x = __reduce_max_sync(0xffffffffu, x);
  if (G == 32) return x;
  uint32_t* w = reinterpret_cast<uint32_t*>(words) + (turn & 1) * 64;
  ++turn;
  if ((threadIdx.x & 31) == 0) w[threadIdx.x / 32] = x;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  return __reduce_max_sync(0xffffffffu, lane < G / 32 ? w[lane] : 0u);
}

// y = (h - m) r gain + bias, h = x + residual rounded to the rows' type, m the
// mean (0 without centring), r = 1 / sqrt(mean of (h - m)^2 + eps); or y's
// codes and scale, or (MODE kCodes) those of x itself.
template <typename T, bool W, int C, int MODE>
__global__ void __launch_bounds__(512) norm_kernel(const NormParams p, int G) {
  __shared__ float words[2 * 64];
  wait_for_previous();
  let_next_start();
  const int per = blockDim.x / G, lane = threadIdx.x % G;
  const long long row = static_cast<long long>(blockIdx.x) * per + threadIdx.x / G;
  if (row >= p.rows) return;   // (whole warps: a group of more than a warp is a block)
  int turn = 0;
  const int D = p.dim;
  float v[C][8];
  const T* x = static_cast<const T*>(p.x.p) + row * p.x.stride;
#pragma unroll
  for (int i = 0; i < C; ++i) load8<W>(x, i, lane, G, D, v[i]);
  if (MODE != kCodes && p.residual.p) {
    const T* r = static_cast<const T*>(p.residual.p) + row * p.residual.stride;
    T* h = static_cast<T*>(p.h.p) + row * p.h.stride;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float w[8];
      load8<W>(r, i, lane, G, D, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = static_cast<float>(static_cast<T>(v[i][j] + w[j]));
      store8<W>(h, i, lane, G, D, v[i]);
    }
  }
  if constexpr (MODE != kCodes) {
    if (p.centre) {
      float sum[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < C; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[0] += v[i][j];
      }
      group_sum(sum, G, words, turn);
      const float mean = sum[0] / static_cast<float>(D);
#pragma unroll
      for (int i = 0; i < C; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (feature<W>(i, j, lane, G) < D) v[i][j] -= mean;
        }
      }
    }
    float squares[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < C; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) squares[0] = fmaf(v[i][j], v[i][j], squares[0]);
    }
    group_sum(squares, G, words, turn);
    const float r = 1.0f / sqrtf(squares[0] / static_cast<float>(D) + p.eps);
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float g[8], b[8];
      load_vector<W>(p.gain, 1.0f, i, lane, G, D, g);
      load_vector<W>(p.bias, 0.0f, i, lane, G, D, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * r * g[j] + b[j];
    }
  }
  if constexpr (MODE == kNorm) {
    T* y = static_cast<T*>(p.y.p) + row * p.y.stride;
#pragma unroll
    for (int i = 0; i < C; ++i) store8<W>(y, i, lane, G, D, v[i]);
  } else {
    // the largest magnitude, by its bits: an infinity or a NaN is above all others
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < C; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (what fills up the row may be a NaN here: 0 times an infinite factor)
        if (feature<W>(i, j, lane, G) < D) bits = max(bits, __float_as_uint(v[i][j]) & 0x7fffffffu);
      }
    }
    const float top = __uint_as_float(group_max(bits, G, words, turn)), scale = __fdiv_rn(top, 127.0f);
    const bool some = top <= FLT_MAX && scale > 0.0f;
    int8_t* codes = p.codes + row * D;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      uint32_t q[2] = {0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (a subnormal scale has few bits: quotients by it may pass 127)
        const int c = some ? __float2int_rn(fminf(fmaxf(__fdiv_rn(v[i][j], scale), -127.0f), 127.0f)) : 0;
        if constexpr (W) q[j / 4] |= static_cast<uint32_t>(c & 0xff) << 8 * (j % 4);
        else if (feature<false>(i, j, lane, G) < D) codes[feature<false>(i, j, lane, G)] = static_cast<int8_t>(c);
      }
      if constexpr (W) {
        if (feature<true>(i, 0, lane, G) < D) *reinterpret_cast<uint2*>(codes + feature<true>(i, 0, lane, G)) = make_uint2(q[0], q[1]);
      }
    }
    if (lane == 0) p.scale[row] = top <= FLT_MAX ? scale : NAN;
  }
}

bool aligned16(const void* p, long long stride, size_t size) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(stride) * size) & 15) == 0;
}
// (the stride of a single row is not looked at)
bool wide(const Rows& r, int rows, size_t size) { return !r.p || aligned16(r.p, rows > 1 ? r.stride : 0, size); }
bool wide(const float* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int threads_of(int dim, int pieces) { return ((dim + 8 * pieces - 1) / (8 * pieces) + 31) / 32 * 32; }

template <typename T, bool W, int MODE>
cudaError_t norm_by(const NormParams& p, cudaStream_t s) {
  const int C = p.dim <= 256 ? 1 : p.dim <= 8192 ? 2 : 4, G = threads_of(p.dim, C), threads = G == 32 ? 128 : G;
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(p.rows) * G + threads - 1) / threads);
  if (C == 1) return launch_early(norm_kernel<T, W, 1, MODE>, blocks, threads, 0, s, p, G);
  if (C == 2) return launch_early(norm_kernel<T, W, 2, MODE>, blocks, threads, 0, s, p, G);
  return launch_early(norm_kernel<T, W, 4, MODE>, blocks, threads, 0, s, p, G);
}

template <typename T>
cudaError_t norm_of(const NormParams& p, int mode, cudaStream_t s) {
  const bool w = p.dim % 8 == 0 && wide(p.x, p.rows, sizeof(T)) && wide(p.residual, p.rows, sizeof(T)) && wide(p.y, p.rows, sizeof(T)) &&
                 wide(p.h, p.rows, sizeof(T)) && wide(p.gain) && wide(p.bias) && reinterpret_cast<uintptr_t>(p.codes) % 8 == 0;
  if (mode == kNorm) return w ? norm_by<T, true, kNorm>(p, s) : norm_by<T, false, kNorm>(p, s);
  if (mode == kNormCodes) return w ? norm_by<T, true, kNormCodes>(p, s) : norm_by<T, false, kNormCodes>(p, s);
  return w ? norm_by<T, true, kCodes>(p, s) : norm_by<T, false, kCodes>(p, s);
}

// With u = (x - m) r and g = dy gain: dx = r (g - mean(g) - u mean(g u)) + dh
// (mean(g) where centred), dgain = sum of dy u over the rows, dbias = sum of dy.
// The sums over a row are those of x and g, then of (x - m)^2 and g (x - m). A
// block takes every blocks-th row and keeps the sums over its rows of its
// columns in registers (C 1), or, of rows of more than 8192 features, in shared
// memory; they are added up by a second kernel in the blocks' order.
template <typename T, bool W, int C, bool SHARED>
__global__ void __launch_bounds__(SHARED ? 1024 : 512) norm_gradient_kernel(const NormGradientParams p, int G) {
  __shared__ float words[2 * 64];
  extern __shared__ float sums[];   // SHARED: [2][D]
  wait_for_previous();
  let_next_start();
  const int lane = threadIdx.x, D = p.dim;
  const float over = 1.0f / static_cast<float>(D);
  int turn = 0;
  float dgain[SHARED ? 1 : C][8] = {}, dbias[SHARED ? 1 : C][8] = {};
  if constexpr (SHARED) {
    for (int i = lane; i < 2 * D; i += G) sums[i] = 0.0f;
    __syncthreads();
  }
  for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
    float x[C][8], g[C][8];
    const T* xs = static_cast<const T*>(p.x.p) + row * p.x.stride;
    const T* dys = static_cast<const T*>(p.dy.p) + row * p.dy.stride;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      load8<W>(xs, i, lane, G, D, x[i]);
      load8<W>(dys, i, lane, G, D, g[i]);
    }
    float mean = 0.0f, mean_g = 0.0f;
    if (p.centre) {
      float sum[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < C; ++i) {
        float gain[8];
        load_vector<W>(p.gain, 1.0f, i, lane, G, D, gain);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[0] += x[i][j], sum[1] = fmaf(g[i][j], gain[j], sum[1]);
      }
      group_sum(sum, G, words, turn);
      mean = sum[0] / static_cast<float>(D), mean_g = sum[1] * over;
    }
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float gain[8];
      load_vector<W>(p.gain, 1.0f, i, lane, G, D, gain);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = feature<W>(i, j, lane, G) < D ? x[i][j] - mean : 0.0f;
        x[i][j] = u;
        sum[0] = fmaf(u, u, sum[0]), sum[1] = fmaf(g[i][j] * gain[j], u, sum[1]);
      }
    }
    group_sum(sum, G, words, turn);
    const float r = 1.0f / sqrtf(sum[0] / static_cast<float>(D) + p.eps), along = sum[1] * over * r;
    T* dxs = static_cast<T*>(p.dx.p) + row * p.dx.stride;
    const T* dhs = static_cast<const T*>(p.dh.p) + row * p.dh.stride;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float gain[8], dh[8], dx[8];
      load_vector<W>(p.gain, 1.0f, i, lane, G, D, gain);
      if (p.dh.p) load8<W>(dhs, i, lane, G, D, dh);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = x[i][j] * r, dy = g[i][j];
        dx[j] = (dy * gain[j] - mean_g - u * along) * r;
        if (p.dh.p) dx[j] += dh[j];
        if constexpr (SHARED) {
          const int e = feature<W>(i, j, lane, G);
          if (e < D) sums[e] = fmaf(dy, u, sums[e]), sums[D + e] += dy;
        } else {
          dgain[i][j] = fmaf(dy, u, dgain[i][j]);
          dbias[i][j] += dy;
        }
      }
      store8<W>(dxs, i, lane, G, D, dx);
    }
  }
  const int kinds = p.dbias ? 2 : 1;
  float* part = p.parts + static_cast<long long>(blockIdx.x) * kinds * D;
#pragma unroll
  for (int i = 0; i < C; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = feature<W>(i, j, lane, G);
      if (e >= D) continue;
      part[e] = SHARED ? sums[e] : dgain[SHARED ? 0 : i][j];
      if (p.dbias) part[D + e] = SHARED ? sums[D + e] : dbias[SHARED ? 0 : i][j];
    }
  }
}

// Columns of [blocks][columns], added up by 32 threads each in a fixed order.
constexpr int kSumRows = 32;
__global__ void __launch_bounds__(32 * kSumRows) add_parts_kernel(const NormGradientParams p, int columns) {
  __shared__ float words[kSumRows][33];
  wait_for_previous();
  let_next_start();
  const int lane = threadIdx.x & 31, group = threadIdx.x / 32, column = blockIdx.x * 32 + lane;
  float sum = 0.0f;
  if (column < columns) {
#pragma unroll 4
    for (int b = group; b < p.blocks; b += kSumRows) sum += p.parts[static_cast<long long>(b) * columns + column];
  }
  words[group][lane] = sum;
  __syncthreads();
  sum = warp_sum(words[lane][group]);
  const int of = blockIdx.x * 32 + group;
  if (lane == 0 && of < p.dim) p.dgain[of] = sum;
  if (lane == 0 && of >= p.dim && of < columns) p.dbias[of - p.dim] = sum;
}

template <typename T, bool W>
cudaError_t norm_gradient_by(const NormGradientParams& p, cudaStream_t s) {
  const int G = threads_of(p.dim, 2);
  cudaError_t e;
  if (p.dim <= 8192) {
    e = launch_early(norm_gradient_kernel<T, W, 2, false>, p.blocks, G, 0, s, p, G);
  } else {
    const size_t shared = 2 * sizeof(float) * p.dim;
    e = cudaFuncSetAttribute(norm_gradient_kernel<T, W, 2, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(shared));
    if (e == cudaSuccess) e = launch_early(norm_gradient_kernel<T, W, 2, true>, p.blocks, G, shared, s, p, G);
  }
  if (e != cudaSuccess) return e;
  const int columns = p.dim * (p.dbias ? 2 : 1);
  return launch_early(add_parts_kernel, (columns + 31) / 32, 32 * kSumRows, 0, s, p, columns);
}

// --- embedding -----------------------------------------------------------------

// y[t] = scale table[tokens[t]], zeros where the token is no row of the table.
template <typename E, typename T, bool W>
__global__ void embed_kernel(const EmbedParams p) {
  wait_for_previous();
  let_next_start();
  for (long long row = blockIdx.y; row < p.rows; row += gridDim.y) {
    const int token = p.tokens[row], D = p.dim;
    const bool inside = token >= 0 && token < p.vocab;
    const E* x = static_cast<const E*>(p.table.p) + (inside ? token : 0) * p.table.stride;
    T* y = static_cast<T*>(p.y.p) + row * p.y.stride;
    float v[8] = {};
    if (inside) {
      load8<W>(x, blockIdx.x, threadIdx.x, blockDim.x, D, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= p.scale;
    }
    store8<W>(y, blockIdx.x, threadIdx.x, blockDim.x, D, v);
  }
}

template <typename E, typename T>
cudaError_t embed_of(const EmbedParams& p, cudaStream_t s) {
  const bool w = p.dim % 8 == 0 && wide(p.table, p.vocab, sizeof(E)) && wide(p.y, p.rows, sizeof(T));
  const int threads = min(128, threads_of(p.dim, 1));
  const dim3 grid((p.dim + 8 * threads - 1) / (8 * threads), min(p.rows, 65535));
  return w ? launch_early(embed_kernel<E, T, true>, grid, threads, 0, s, p) : launch_early(embed_kernel<E, T, false>, grid, threads, 0, s, p);
}

// The rows of each id, ascending. A block takes kIds ids and looks through all
// tokens (they stay in L2): it counts those of its ids and those before them,
// which is where its part of `places` begins, and then puts the rows of its ids
// there. Warp w looks through the w-th part of the tokens both times, so that
// its rows of an id stand behind those of the warps before it.
constexpr int kIds = 256, kIndexWarps = 32;
__global__ void __launch_bounds__(32 * kIndexWarps) index_kernel(const EmbedGradientParams p) {
  __shared__ int at[kIndexWarps][kIds];
  __shared__ int before[kIndexWarps], sums[kIds / 32];
  wait_for_previous();
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, low = blockIdx.x * kIds;
  for (int i = lane; i < kIds; i += 32) at[warp][i] = 0;
  __syncwarp();
  const long long per = (static_cast<long long>(p.rows) + 32 * kIndexWarps - 1) / (32 * kIndexWarps) * 32;
  const long long begin = warp * per, end = min(static_cast<long long>(p.rows), begin + per);
  const int here = min(kIds, p.vocab - low);
  int less = 0;
  for (long long t = begin + lane; t < end; t += 32) {
    const int token = p.tokens[t], id = token - low;
    if (token >= 0 && id < 0) ++less;
    if (token >= low && id < here) atomicAdd(&at[warp][id], 1);
  }
  less = __reduce_add_sync(0xffffffffu, less);
  if (lane == 0) before[warp] = less;
  __syncthreads();
  // where each warp's rows of each id begin
  int first = 0, count = 0;
  if (threadIdx.x < kIds) {
    for (int w = 0; w < kIndexWarps; ++w) count += at[w][threadIdx.x];
    first = count;
    for (int o = 1; o < 32; o *= 2) {
      const int x = __shfl_up_sync(0xffffffffu, first, o);
      if (lane >= o) first += x;
    }
    if (lane == 31) sums[warp] = first;
  }
  __syncthreads();
  if (threadIdx.x < kIds) {
    int base = first - count;
    for (int w = 0; w < kIndexWarps; ++w) base += before[w];
    for (int w = 0; w < warp; ++w) base += sums[w];
    if (static_cast<int>(threadIdx.x) < here) p.first[low + threadIdx.x] = base;
    if (low + static_cast<int>(threadIdx.x) == p.vocab - 1) p.first[p.vocab] = base + count;
    for (int w = 0; w < kIndexWarps; ++w) {
      const int n = at[w][threadIdx.x];
      at[w][threadIdx.x] = base;
      base += n;
    }
  }
  __syncthreads();
  for (long long t0 = begin; t0 < end; t0 += 32) {
    const long long t = t0 + lane;
    const int token = t < end ? p.tokens[t] : -1, id = token - low;
    const bool mine = token >= low && id < here;
    const unsigned which = __ballot_sync(0xffffffffu, mine);
    if (!which) continue;
    if (mine) {
      const unsigned same = __match_any_sync(which, id);
      p.places[at[warp][id] + __popc(same & ((1u << lane) - 1))] = static_cast<int>(t);
      __syncwarp(which);
      if (lane == 31 - __clz(same)) at[warp][id] += __popc(same);
    }
    __syncwarp();
  }
}

// grad[v] = scale sum of dy over the rows of v, in their order. A block takes
// kSumIds ids and kSumColumns columns of them; a thread 4 columns of every
// kSumGroups-th id.
constexpr int kSumIds = 16, kSumGroups = 4, kSumColumns = 256;
template <typename T, bool W>
__global__ void __launch_bounds__(kSumGroups * kSumColumns / 4) embed_gradient_kernel(const EmbedGradientParams p, int slices, long long items) {
  __shared__ int first[kSumIds + 1];
  wait_for_previous();
  let_next_start();
  const int group = threadIdx.x / (kSumColumns / 4), lane = threadIdx.x % (kSumColumns / 4), D = p.dim;
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int slice = static_cast<int>(item % slices), v0 = static_cast<int>(item / slices) * kSumIds;
    __syncthreads();
    if (threadIdx.x <= kSumIds) first[threadIdx.x] = p.first[min(p.vocab, v0 + static_cast<int>(threadIdx.x))];
    __syncthreads();
    auto column = [&](int j) { return slice * kSumColumns + (W ? 4 * lane + j : j * (kSumColumns / 4) + lane); };
    for (int k = group; k < kSumIds; k += kSumGroups) {
      if (v0 + k >= p.vocab) break;
      float sum[4] = {};
#pragma unroll 4
      for (int i = first[k]; i < first[k + 1]; ++i) {
        const T* dy = static_cast<const T*>(p.dy.p) + p.places[i] * p.dy.stride;
        float x[4] = {};
        if constexpr (W) {
          if (column(0) < D) sjd_kv_ops::load4(dy + column(0), true, x);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (column(j) < D) x[j] = static_cast<float>(dy[column(j)]);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] += x[j];
      }
      float* out = p.grad + static_cast<long long>(v0 + k) * D;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] *= p.scale;
      if constexpr (W) {
        if (column(0) < D) sjd_kv_ops::store4(out + column(0), true, sum);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (column(j) < D) out[column(j)] = sum[j];
        }
      }
    }
  }
}

template <typename T>
cudaError_t embed_gradient_of(const EmbedGradientParams& p, int sms, cudaStream_t s) {
  cudaError_t e = launch_early(index_kernel, static_cast<unsigned>((p.vocab + kIds - 1) / kIds), 32 * kIndexWarps, 0, s, p);
  if (e != cudaSuccess) return e;
  const bool w = p.dim % 4 == 0 && reinterpret_cast<uintptr_t>(p.grad) % 16 == 0 && reinterpret_cast<uintptr_t>(p.dy.p) % (4 * sizeof(T)) == 0 &&
                 (p.rows < 2 || p.dy.stride % 4 == 0);
  const int slices = (p.dim + kSumColumns - 1) / kSumColumns;
  const long long items = static_cast<long long>((p.vocab + kSumIds - 1) / kSumIds) * slices;
  const unsigned blocks = static_cast<unsigned>(min(items, 8ll * sms));
  const int threads = kSumGroups * kSumColumns / 4;
  return w ? launch_early(embed_gradient_kernel<T, true>, blocks, threads, 0, s, p, slices, items)
           : launch_early(embed_gradient_kernel<T, false>, blocks, threads, 0, s, p, slices, items);
}

}  // namespace

cudaError_t launch_norm(const NormParams& p, int mode, int dtype, cudaStream_t s) {
  return dtype == SJD_BF16 ? norm_of<__nv_bfloat16>(p, mode, s) : norm_of<float>(p, mode, s);
}

// Blocks of 512 threads and more an SM, each with several rows to sum up.
int norm_gradient_blocks(int rows, int dim, int sms) { return min(rows, sms * max(2, 512 / threads_of(dim, 2))); }

cudaError_t launch_norm_gradient(const NormGradientParams& p, int dtype, cudaStream_t s) {
  const size_t size = dtype == SJD_BF16 ? 2 : 4;
  const bool w = p.dim % 8 == 0 && wide(p.dy, p.rows, size) && wide(p.x, p.rows, size) && wide(p.dh, p.rows, size) && wide(p.dx, p.rows, size) &&
                 wide(p.gain);
  if (dtype == SJD_BF16) return w ? norm_gradient_by<__nv_bfloat16, true>(p, s) : norm_gradient_by<__nv_bfloat16, false>(p, s);
  return w ? norm_gradient_by<float, true>(p, s) : norm_gradient_by<float, false>(p, s);
}

cudaError_t launch_embed(const EmbedParams& p, int table_dtype, int dtype, int sms, cudaStream_t s) {
  if (table_dtype == SJD_BF16) return dtype == SJD_BF16 ? embed_of<__nv_bfloat16, __nv_bfloat16>(p, s) : embed_of<__nv_bfloat16, float>(p, s);
  return dtype == SJD_BF16 ? embed_of<float, __nv_bfloat16>(p, s) : embed_of<float, float>(p, s);
}

cudaError_t launch_embed_gradient(const EmbedGradientParams& p, int dtype, int sms, cudaStream_t s) {
  return dtype == SJD_BF16 ? embed_gradient_of<__nv_bfloat16>(p, sms, s) : embed_gradient_of<float>(p, sms, s);
}

}  // namespace sjd_dense_ops
