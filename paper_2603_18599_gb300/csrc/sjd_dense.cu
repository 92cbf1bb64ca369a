// The window forward's operators on rows of features: norms with a residual,
// their codes of 8 bits and their gradient, the embedding of tokens and its
// gradient. All of them move rows through once and are bound by HBM in long
// calls and by one chain of loads and sums in short ones.
//
// A row is taken by a group of G threads, C pieces of 8 features to a thread,
// and stays in their registers from its load to its store: its mean, the mean
// of the squares around it (both as sums of the differences themselves, so
// that nothing cancels) and its largest magnitude are sums over the group.
//
// What a thread does for a row whatever its length (the sums' exchanges, the
// addresses) is worth as much as 16 features, so that a thread of a long call takes 32
// of them: rows of up to 1024 features are taken by a warp or a part of
// one, longer ones by a block. A call of few rows spreads each over more threads.

#include <cfloat>

#include "sjd_dense.h"
#include "sjd_kv_device.cuh"
#include "sjd_tcgen05.cuh"

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

// The first n of 32 words in shared memory, which all lanes read at once; n is the same for all.
__device__ __forceinline__ float add_words(const float* w, int n) {
  float sum = 0.0f;
  for (int i = 0; i < n; i += 4) {
    const float4 v = *reinterpret_cast<const float4*>(w + i);
    sum += (v.x + (i + 1 < n ? v.y : 0.0f)) + ((i + 2 < n ? v.z : 0.0f) + (i + 3 < n ? v.w : 0.0f));
  }
  return sum;
}

// Sums over the group of G threads: a power of two of a warp's, or the whole
// block. `turn` numbers the sums of a block: two neighbours take different words
// of `words` [2][2][32], so that one barrier a sum is enough.
template <int N>
__device__ __forceinline__ void group_sum(float (&x)[N], int G, float* words, int& turn) {
  if (G <= 32) {
    for (int o = G / 2; o > 0; o /= 2) {
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] += __shfl_xor_sync(0xffffffffu, x[k], o);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = warp_sum(x[k]);
  float* w = words + (turn & 1) * 64;
  ++turn;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) w[32 * k + threadIdx.x / 32] = x[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = add_words(w + 32 * k, G / 32);
}
__device__ __forceinline__ uint32_t group_max(uint32_t x, int G, float* words, int& turn) {
  if (G <= 32) {
    for (int o = G / 2; o > 0; o /= 2) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
  }
  x = __reduce_max_sync(0xffffffffu, x);
  uint32_t* w = reinterpret_cast<uint32_t*>(words) + (turn & 1) * 64;
  ++turn;
  if ((threadIdx.x & 31) == 0) w[threadIdx.x / 32] = x;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  return __reduce_max_sync(0xffffffffu, lane < G / 32 ? w[lane] : 0u);
}

// A thread's part of a row on its way into shared memory: it copies what it reads
// itself, and waits for its own copies alone.
template <typename T, int C>
__device__ __forceinline__ void copy_row(const T* row, T* to, int G, int D) {
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int e = (i * G + threadIdx.x) * 8;
    if (e >= D) break;
#pragma unroll
    for (int k = 0; k < 8; k += 16 / sizeof(T)) sjd_kv_ops::copy16(sjd_kv_ops::smem_addr(to + e + k), row + e + k, 16);
  }
}

// x / scale of eight values, as IEEE division rounds it. With the reciprocal
// rounded to nearest, two corrections by the exact remainder give the nearest
// quotient (Markstein, IBM J. Res. Dev. 34, 1990), as long as the remainders of
// quotients that matter do not underflow: for scales within 2^60 of 1.
__device__ __forceinline__ float quotient(float x, float scale, float inverse) {
  float q = x * inverse;
  q = fmaf(fmaf(-q, scale, x), inverse, q);
  return fmaf(fmaf(-q, scale, x), inverse, q);
}

// A row in registers becomes y = (h - m) r gain + bias, h = x + residual rounded
// to the rows' type, m the mean (0 without centring), r = 1 / sqrt(mean of
// (h - m)^2 + eps); or y's codes and scale, or (MODE kCodes) those of x itself.
// w: the residual's row. `there`: the row is to be written.
template <typename T, bool W, int C, int MODE>
__device__ __forceinline__ void norm_row(const NormParams& p, long long row, bool there, int lane, int G, float (&v)[C][8], float (&w)[C][8], float* words,
                                         int& turn) {
  const int D = p.dim;
  const float over = 1.0f / static_cast<float>(D);
  if (MODE != kCodes && p.residual.p) {
    T* h = static_cast<T*>(p.h.p) + row * p.h.stride;
#pragma unroll
    for (int i = 0; i < C; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = static_cast<float>(static_cast<T>(v[i][j] + w[i][j]));
      if (there) store8<W>(h, i, lane, G, D, v[i]);
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
      const float mean = sum[0] * over;
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
    const float r = rsqrtf(squares[0] * over + p.eps);
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
    if (!there) return;
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
    if (!there) return;
    const bool some = top <= FLT_MAX && scale > 0.0f, plain = top > 0x1p-60f && top < 0x1p60f;
    const float inverse = __frcp_rn(scale);
    int8_t* codes = p.codes + row * D;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      uint32_t q[2] = {0, 0};
      if (plain) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = quotient(v[i][j], scale, inverse);
      } else {
        // (a subnormal scale has few bits: quotients by it may pass 127)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = some ? fminf(fmaxf(__fdiv_rn(v[i][j], scale), -127.0f), 127.0f) : 0.0f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = __float2int_rn(v[i][j]);
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

// A group of G threads to a row: lanes of a warp, or a block.
constexpr int kShortBlock = 128;   // where several rows share a block
constexpr int kShort = 512;        // features of a row that the gradient's sums take a warp for
template <typename T, bool W, int C, int MODE>
__global__ void __launch_bounds__(512) norm_kernel(const NormParams p, int G) {
  __shared__ __align__(16) float words[2 * 64];
  wait_for_previous();
  let_next_start();
  const int per = blockDim.x / G, lane = threadIdx.x % G;
  const long long at = static_cast<long long>(blockIdx.x) * per + threadIdx.x / G, row = min(at, p.rows - 1ll);
  int turn = 0;
  float v[C][8], w[C][8];
#pragma unroll
  for (int i = 0; i < C; ++i) load8<W>(static_cast<const T*>(p.x.p) + row * p.x.stride, i, lane, G, p.dim, v[i]);
  if (MODE != kCodes && p.residual.p) {
#pragma unroll
    for (int i = 0; i < C; ++i) load8<W>(static_cast<const T*>(p.residual.p) + row * p.residual.stride, i, lane, G, p.dim, w[i]);
  }
  norm_row<T, W, C, MODE>(p, row, at < p.rows, lane, G, v, w, words, turn);
}

bool aligned16(const void* p, long long stride, size_t size) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(stride) * size) & 15) == 0;
}
// (the stride of a single row is not looked at)
bool wide(const Rows& r, int rows, size_t size) { return !r.p || aligned16(r.p, rows > 1 ? r.stride : 0, size); }
bool wide(const float* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int threads_of(int dim, int pieces) { return ((dim + 8 * pieces - 1) / (8 * pieces) + 31) / 32 * 32; }

int lanes_of(int dim, int pieces) {   // of a warp
  int l = 8;
  while (8 * pieces * l < dim) l *= 2;
  return l;
}

template <typename T, bool W, int C, int MODE>
cudaError_t norm_with(const NormParams& p, cudaStream_t s) {
  const int G = p.dim <= 8 * C * 32 ? lanes_of(p.dim, C) : threads_of(p.dim, C), threads = G <= 32 ? kShortBlock : G, per = threads / G;
  return launch_early(norm_kernel<T, W, C, MODE>, static_cast<unsigned>((static_cast<long long>(p.rows) + per - 1) / per), threads, 0, s, p, G);
}

// Pieces of a thread. PIECES_FIGURES
template <typename T, bool W, int MODE>
cudaError_t norm_by(const NormParams& p, int sms, cudaStream_t s) {
  const bool few = p.rows <= 2 * sms;
  const int d = p.dim;
  if (d <= 256 || (few && d <= 4096)) return norm_with<T, W, 1, MODE>(p, s);
  if (d <= 512 || ((few || !W) && d <= 8192)) return norm_with<T, W, 2, MODE>(p, s);
  return norm_with<T, W, 4, MODE>(p, s);
}

template <typename T>
cudaError_t norm_of(const NormParams& p, int mode, int sms, cudaStream_t s) {
  const bool w = p.dim % 8 == 0 && wide(p.x, p.rows, sizeof(T)) && wide(p.residual, p.rows, sizeof(T)) && wide(p.y, p.rows, sizeof(T)) &&
                 wide(p.h, p.rows, sizeof(T)) && wide(p.gain) && wide(p.bias) && reinterpret_cast<uintptr_t>(p.codes) % 8 == 0;
  if (mode == kNorm) return w ? norm_by<T, true, kNorm>(p, sms, s) : norm_by<T, false, kNorm>(p, sms, s);
  if (mode == kNormCodes) return w ? norm_by<T, true, kNormCodes>(p, sms, s) : norm_by<T, false, kNormCodes>(p, sms, s);
  return w ? norm_by<T, true, kCodes>(p, sms, s) : norm_by<T, false, kCodes>(p, sms, s);
}

// With u = (x - m) r and g = dy gain: dx = r (g - mean(g) - u mean(g u)) + dh
// (mean(g) where centred), dgain = sum of dy u over the rows, dbias = sum of dy.
// The sums over a row are those of x and g, then of (x - m)^2 and g (x - m).
// x: the row, g: dy, dh: what is added (or not); dx takes their place in g, u in x and dy in dh.
template <bool W, int C, typename Gain>
__device__ __forceinline__ void gradient_row(const NormGradientParams& p, int lane, int G, float (&x)[C][8], float (&dy)[C][8], float (&dx)[C][8],
                                             float* words, int& turn, Gain gain) {
  const int D = p.dim;
  const float over = 1.0f / static_cast<float>(D);
  float mean = 0.0f, mean_g = 0.0f;
  if (p.centre) {
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float g[8];
      gain(i, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] += x[i][j], sum[1] = fmaf(dy[i][j], g[j], sum[1]);
    }
    group_sum(sum, G, words, turn);
    mean = sum[0] * over, mean_g = sum[1] * over;
  }
  float sum[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < C; ++i) {
    float g[8];
    gain(i, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float u = feature<W>(i, j, lane, G) < D ? x[i][j] - mean : 0.0f;
      x[i][j] = u;
      sum[0] = fmaf(u, u, sum[0]), sum[1] = fmaf(dy[i][j] * g[j], u, sum[1]);
    }
  }
  group_sum(sum, G, words, turn);
  const float r = rsqrtf(sum[0] * over + p.eps), along = sum[1] * over * r;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    float g[8];
    gain(i, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[i][j] *= r;
      dx[i][j] = fmaf(dy[i][j] * g[j] - mean_g - x[i][j] * along, r, p.dh.p ? dx[i][j] : 0.0f);
    }
  }
}

// Rows of up to 512 features: every group of G lanes takes rows of its own, and
// the block's warps add up their columns in order.
template <typename T, bool W, int C>
__global__ void __launch_bounds__(kShortBlock) norm_gradient_short_kernel(const NormGradientParams p, int G) {
  __shared__ float sums[2][kShort];
  wait_for_previous();
  let_next_start();
  const int lane = threadIdx.x % G, D = p.dim, per = kShortBlock / G;
  int turn = 0;
  float dgain[C][8] = {}, dbias[C][8] = {};
  for (long long first = static_cast<long long>(blockIdx.x) * per; first < p.rows; first += static_cast<long long>(gridDim.x) * per) {
    const long long at = first + threadIdx.x / G, row = min(at, p.rows - 1ll);
    float x[C][8], dy[C][8], dx[C][8];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      load8<W>(static_cast<const T*>(p.x.p) + row * p.x.stride, i, lane, G, D, x[i]);
      load8<W>(static_cast<const T*>(p.dy.p) + row * p.dy.stride, i, lane, G, D, dy[i]);
      if (p.dh.p) load8<W>(static_cast<const T*>(p.dh.p) + row * p.dh.stride, i, lane, G, D, dx[i]);
    }
    gradient_row<W, C>(p, lane, G, x, dy, dx, nullptr, turn, [&](int i, float (&g)[8]) { load_vector<W>(p.gain, 1.0f, i, lane, G, D, g); });
    if (at >= p.rows) continue;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      store8<W>(static_cast<T*>(p.dx.p) + row * p.dx.stride, i, lane, G, D, dx[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) dgain[i][j] = fmaf(dy[i][j], x[i][j], dgain[i][j]), dbias[i][j] += dy[i][j];
    }
  }
  __syncwarp();
  for (int o = G; o < 32; o *= 2) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dgain[i][j] += __shfl_xor_sync(0xffffffffu, dgain[i][j], o);
        dbias[i][j] += __shfl_xor_sync(0xffffffffu, dbias[i][j], o);
      }
    }
  }
  for (int w = 0; w < kShortBlock / 32; ++w) {
    if (static_cast<int>(threadIdx.x / 32) == w && (threadIdx.x & 31) < static_cast<unsigned>(G)) {
#pragma unroll
      for (int i = 0; i < C; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int e = feature<W>(i, j, lane, G);
          if (e < D) sums[0][e] = (w ? sums[0][e] : 0.0f) + dgain[i][j], sums[1][e] = (w ? sums[1][e] : 0.0f) + dbias[i][j];
        }
      }
    }
    __syncthreads();
  }
  const int columns = D * (p.dbias ? 2 : 1);
  for (int e = threadIdx.x; e < columns; e += kShortBlock) p.parts[static_cast<long long>(blockIdx.x) * columns + e] = sums[e >= D][e >= D ? e - D : e];
}

// Longer rows: a block takes every gridDim-th, and keeps the sums over its rows of
// its columns in registers, or, of rows of more than 8192 features, in shared
// memory (WAY kShared); a second kernel adds them up in the blocks' order. Rows that can be
// accessed 16 bytes at a time are on their way while the one before them is summed up
// (kAhead; `deep` stages of shared memory).
enum GradientWay { kAhead, kDirect, kShared };
template <typename T, bool W, int WAY>
__global__ void __launch_bounds__(WAY == kShared ? 1024 : 512) norm_gradient_kernel(const NormGradientParams p, int G, int deep) {
  constexpr int C = 2;
  __shared__ __align__(16) float words[2 * 64];
  extern __shared__ __align__(16) unsigned char shared[];
  float* sums = reinterpret_cast<float*>(shared);   // kShared: [2][D]
  T* stages = reinterpret_cast<T*>(shared);         // kAhead: [deep][2 or 3][D]
  wait_for_previous();
  let_next_start();
  const int lane = threadIdx.x, D = p.dim, kinds = p.dh.p ? 3 : 2;
  auto x_of = [&](long long row) { return static_cast<const T*>(p.x.p) + row * p.x.stride; };
  auto dy_of = [&](long long row) { return static_cast<const T*>(p.dy.p) + row * p.dy.stride; };
  auto dh_of = [&](long long row) { return static_cast<const T*>(p.dh.p) + row * p.dh.stride; };
  auto fetch = [&](long long row, int stage) {
    T* to = stages + stage * kinds * D;
    if (row < p.rows) {
      copy_row<T, C>(x_of(row), to, G, D);
      copy_row<T, C>(dy_of(row), to + D, G, D);
      if (p.dh.p) copy_row<T, C>(dh_of(row), to + 2 * D, G, D);
    }
    sjd_kv_ops::copy_commit();   // (the group of a row that is not there is empty)
  };
  float dgain[WAY == kShared ? 1 : C][8] = {}, dbias[WAY == kShared ? 1 : C][8] = {}, gains[WAY == kShared ? 1 : C][8];
  if constexpr (WAY == kShared) {
    for (int i = lane; i < 2 * D; i += G) sums[i] = 0.0f;
    __syncthreads();
  } else {
    if constexpr (WAY == kAhead) {
      for (int i = 0; i + 1 < deep; ++i) fetch(blockIdx.x + static_cast<long long>(i) * gridDim.x, i);
    }
#pragma unroll
    for (int i = 0; i < C; ++i) load_vector<W>(p.gain, 1.0f, i, lane, G, D, gains[i]);
  }
  int turn = 0, stage = 0;
  for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T *xs = x_of(row), *dys = dy_of(row), *dhs = dh_of(row);
    if constexpr (WAY == kAhead) {
      if (deep == 2) sjd_kv_ops::copy_wait<0>();
      else if (deep == 3) sjd_kv_ops::copy_wait<1>();
      else sjd_kv_ops::copy_wait<2>();
      fetch(row + (deep - 1ll) * gridDim.x, stage == 0 ? deep - 1 : stage - 1);   // (where the row before was)
      xs = stages + stage * kinds * D, dys = xs + D, dhs = dys + D;
      if (++stage == deep) stage = 0;
    }
    float x[C][8], dy[C][8], dx[C][8];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      load8<W>(xs, i, lane, G, D, x[i]);
      load8<W>(dys, i, lane, G, D, dy[i]);
      if (p.dh.p) load8<W>(dhs, i, lane, G, D, dx[i]);
    }
    gradient_row<W, C>(p, lane, G, x, dy, dx, words, turn, [&](int i, float (&g)[8]) {
      if constexpr (WAY == kShared) {
        load_vector<W>(p.gain, 1.0f, i, lane, G, D, g);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = gains[i][j];
      }
    });
    T* dxs = static_cast<T*>(p.dx.p) + row * p.dx.stride;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      store8<W>(dxs, i, lane, G, D, dx[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (WAY == kShared) {
          const int e = feature<W>(i, j, lane, G);
          if (e < D) sums[e] = fmaf(dy[i][j], x[i][j], sums[e]), sums[D + e] += dy[i][j];
        } else {
          dgain[i][j] = fmaf(dy[i][j], x[i][j], dgain[i][j]);
          dbias[i][j] += dy[i][j];
        }
      }
    }
  }
  sjd_kv_ops::copy_wait_all();
  float* part = p.parts + static_cast<long long>(blockIdx.x) * (p.dbias ? 2 : 1) * D;
#pragma unroll
  for (int i = 0; i < C; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = feature<W>(i, j, lane, G);
      if (e >= D) continue;
      part[e] = WAY == kShared ? sums[e] : dgain[WAY == kShared ? 0 : i][j];
      if (p.dbias) part[D + e] = WAY == kShared ? sums[D + e] : dbias[WAY == kShared ? 0 : i][j];
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

// Blocks of the gradient's first kernel on an SM (by its 128 registers) and
// rows on their way in each: shared memory holds them, and there is no use for more
// than 96 KB of them.
struct Flow {
  int per_sm, deep;
  size_t shared;
};
Flow gradient_flow(int dim, size_t size) {
  if (dim > 8192) return {1, 0, 2 * sizeof(float) * dim};
  const size_t row = 3 * size * dim;
  Flow f;
  f.per_sm = min(8, max(1, 65536 / 128 / threads_of(dim, 2)));
  while (f.per_sm > 1 && 2 * f.per_sm * row > 200 * 1024) --f.per_sm;
  f.deep = 4;
  while (f.deep > 2 && f.deep * f.per_sm * row > 128 * 1024) --f.deep;
  f.shared = f.deep * row;
  return f;
}

template <typename T, bool W, int WAY>
cudaError_t norm_gradient_with(const NormGradientParams& p, const Flow& f, cudaStream_t s) {
  const int G = threads_of(p.dim, 2);
  const size_t shared = WAY == kDirect ? 0 : f.shared;
  if (shared > 40 * 1024) {   // (with the words 48 KB, which any kernel may have)
    const cudaError_t e = cudaFuncSetAttribute(norm_gradient_kernel<T, W, WAY>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(shared));
    if (e != cudaSuccess) return e;
  }
  return launch_early(norm_gradient_kernel<T, W, WAY>, p.blocks, G, shared, s, p, G, f.deep);
}

template <typename T, bool W>
cudaError_t norm_gradient_by(const NormGradientParams& p, cudaStream_t s) {
  const int columns = p.dim * (p.dbias ? 2 : 1);
  const Flow f = gradient_flow(p.dim, sizeof(T));
  cudaError_t e;
  if (p.dim <= kShort / 2) e = launch_early(norm_gradient_short_kernel<T, W, 1>, p.blocks, kShortBlock, 0, s, p, lanes_of(p.dim, 1));
  else if (p.dim <= kShort) e = launch_early(norm_gradient_short_kernel<T, W, 2>, p.blocks, kShortBlock, 0, s, p, lanes_of(p.dim, 2));
  else if (p.dim > 8192) e = norm_gradient_with<T, W, kShared>(p, f, s);
  else if (W && f.shared <= 227 * 1024 - 1024) e = norm_gradient_with<T, W, W ? kAhead : kDirect>(p, f, s);
  else e = norm_gradient_with<T, W, kDirect>(p, f, s);
  if (e != cudaSuccess) return e;
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

cudaError_t launch_norm(const NormParams& p, int mode, int dtype, int sms, cudaStream_t s) {
  return dtype == SJD_BF16 ? norm_of<__nv_bfloat16>(p, mode, sms, s) : norm_of<float>(p, mode, sms, s);
}

int norm_gradient_blocks(int rows, int dim, int dtype, int sms) {
  if (dim > kShort) return min(rows, sms * gradient_flow(dim, dtype == SJD_BF16 ? 2 : 4).per_sm);
  const int per = kShortBlock / lanes_of(dim, dim <= kShort / 2 ? 1 : 2);
  return static_cast<int>(min((static_cast<long long>(rows) + per - 1) / per, 8ll * sms));
}

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
