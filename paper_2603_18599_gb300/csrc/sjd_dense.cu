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
#include "sjd_dense_rows.cuh"
#include "sjd_kv_device.cuh"
#include "sjd_tcgen05.cuh"

namespace sjd_dense_ops {

#ifdef SJD_CHECKS
using sjd_kv_ops::checked_index;
#endif
using sjd_kv_ops::add2;
using sjd_kv_ops::fma2;
using sjd_kv_ops::halves;
using sjd_kv_ops::launch_early;
using sjd_kv_ops::let_next_start;
using sjd_kv_ops::mul2;
using sjd_kv_ops::pack_bf16;
using sjd_kv_ops::Pair;
using sjd_kv_ops::pair;
using sjd_kv_ops::unpack_bf16;
using sjd_kv_ops::wait_for_previous;

namespace {

// (Wide loads behind the row's end take its last piece instead, and `FILL` puts zeros in its
// place: a select costs less than a branch around the load. `OWN`: the thread's first piece,
// which every thread has in rows of more than 512 features where it has two.)
template <bool W, bool FILL = true, bool OWN = false, typename T>
__device__ __forceinline__ void load8(const T* row, int i, Place at, int D, float (&v)[8]) {
  if constexpr (W) {
    const int e = feature<true>(i, 0, at), here = OWN ? (e < D ? e : at.first) : min(e, D - 8);
    if constexpr (sizeof(T) == 2) {
      uint4 u = *reinterpret_cast<const uint4*>(row + here);
      if (FILL) u.x = e < D ? u.x : 0, u.y = e < D ? u.y : 0, u.z = e < D ? u.z : 0, u.w = e < D ? u.w : 0;
      const float2 a = unpack_bf16(u.x), b = unpack_bf16(u.y), c = unpack_bf16(u.z), d = unpack_bf16(u.w);
      v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
    } else {
      const float4 a = *reinterpret_cast<const float4*>(row + here), b = *reinterpret_cast<const float4*>(row + here + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
      if (FILL) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e < D ? v[j] : 0.0f;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = is_there<false>(i, j, at, D) ? static_cast<float>(row[feature<false>(i, j, at)]) : 0.0f;
    }
  }
}

template <bool W, typename T>
__device__ __forceinline__ void store8(T* row, int i, Place at, int D, const float (&v)[8]) {
  if constexpr (W) {
    const int e = feature<true>(i, 0, at);
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
      if (is_there<false>(i, j, at, D)) row[feature<false>(i, j, at)] = static_cast<T>(v[j]);
    }
  }
}

// The same in pairs of neighbours, which are added and multiplied two at a time.
template <bool W, bool FILL = true, bool OWN = false, typename T>
__device__ __forceinline__ void load8(const T* row, int i, Place at, int D, Pair (&v)[4]) {
  float f[8];
  load8<W, FILL, OWN>(row, i, at, D, f);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = pair(f[2 * j], f[2 * j + 1]);
}
// Of a row that copy_row brought: the thread's own pieces alone are looked at, as the others'
// may be on their way.
template <typename T>
__device__ __forceinline__ void load_own8(const T* row, int i, Place at, int D, Pair (&v)[4]) {
  load8<true, true, true>(row, i, at, D, v);
}
template <bool W, typename T>
__device__ __forceinline__ void store8(T* row, int i, Place at, int D, const Pair (&v)[4]) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 x = halves(v[j]);
    f[2 * j] = x.x, f[2 * j + 1] = x.y;
  }
  store8<W>(row, i, at, D, f);
}
// x for the features that are there, 0 for those that fill up the last piece.
template <bool W>
__device__ __forceinline__ Pair where_there(float x, int i, int j, Place at, int D) {
  if constexpr (W) {
    const float y = is_there<true>(i, 0, at, D) ? x : 0.0f;
    return pair(y, y);
  } else {
    return pair(is_there<false>(i, 2 * j, at, D) ? x : 0.0f, is_there<false>(i, 2 * j + 1, at, D) ? x : 0.0f);
  }
}

// Vectors of one float a feature (gains), which are 16-byte aligned where rows are.
template <bool W>
__device__ __forceinline__ void load_vector(const float* p, float otherwise, int i, Place at, int D, Pair (&v)[4]) {
  if (p) {
    load8<W, false>(p, i, at, D, v);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pair(otherwise, otherwise);
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
template <int N>
__device__ __forceinline__ void group_max(uint32_t (&x)[N], int G, float* words, int& turn) {
  if (G <= 32) {
    for (int o = G / 2; o > 0; o /= 2) {
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = max(x[k], __shfl_xor_sync(0xffffffffu, x[k], o));
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = __reduce_max_sync(0xffffffffu, x[k]);
  uint32_t* w = reinterpret_cast<uint32_t*>(words) + (turn & 1) * 64;
  ++turn;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) w[32 * k + threadIdx.x / 32] = x[k];
  }
  __syncthreads();
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = __reduce_max_sync(0xffffffffu, lane < G / 32 ? w[32 * k + lane] : 0u);
}

// A thread's part of a row on its way into shared memory: it copies what it reads
// itself, and waits for its own copies alone.
template <typename T, int C>
__device__ __forceinline__ void copy_row(const T* row, T* to, int G, int D) {
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int e = (i * G + threadIdx.x) * 8;
    if (e < D) {
#pragma unroll
      for (int k = 0; k < 8; k += 16 / sizeof(T)) sjd_kv_ops::copy16(sjd_kv_ops::smem_addr(to + e + k), row + e + k, 16);
    }
  }
}

// x / scale, as IEEE division rounds it. With the reciprocal rounded to nearest,
// two corrections by the exact remainder give the nearest quotient (Markstein,
// IBM J. Res. Dev. 34, 1990), as long as the remainders of quotients that matter
// do not underflow: for scales within 2^60 of 1.
__device__ __forceinline__ Pair quotients(Pair x, Pair less, Pair inverse) {   // less: -scale
  Pair q = mul2(x, inverse);
  q = fma2(fma2(q, less, x), inverse, q);
  return fma2(fma2(q, less, x), inverse, q);
}
// The larger of m and |x|; a NaN, once met, stays.
__device__ __forceinline__ float larger(float m, float x) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(x)));
  return r;
}

// R rows in registers become y = (h - m) r gain + bias, h = x + residual rounded
// to the rows' type, m the mean (0 without centring), r = 1 / sqrt(mean of
// (h - m)^2 + eps); or y's codes and scale, or (MODE kCodes) those of x itself.
// w: the residuals' rows. `there`: the row is to be written.
template <typename T, bool W, int C, int MODE, int R, typename GainsOf>
__device__ __forceinline__ void norm_rows(const NormParams& p, const long long (&row)[R], const bool (&there)[R], int lane, int G, Place at, Pair (&v)[R][C][4],
                                          Pair (&w)[R][C][4], float* words, int& turn, const GainsOf& gains) {
  const int D = p.dim;
  const float over = 1.0f / static_cast<float>(D);
  if (MODE != kCodes && p.residual.p) {
#pragma unroll
    for (int q = 0; q < R; ++q) {
      T* h = static_cast<T*>(p.h.p) + row[q] * p.h.stride;
#pragma unroll
      for (int i = 0; i < C; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = halves(add2(v[q][i][j], w[q][i][j]));
          v[q][i][j] = pair(static_cast<float>(static_cast<T>(x.x)), static_cast<float>(static_cast<T>(x.y)));
        }
        if (there[q]) store8<W>(h, i, at, D, v[q][i]);
      }
    }
  }
  if constexpr (MODE != kCodes) {
    float sum[R];
    if (p.centre) {
#pragma unroll
      for (int q = 0; q < R; ++q) {
        Pair sums[2] = {pair(0.0f, 0.0f), pair(0.0f, 0.0f)};
#pragma unroll
        for (int i = 0; i < C; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) sums[j & 1] = add2(sums[j & 1], v[q][i][j]);
        }
        const float2 two = halves(add2(sums[0], sums[1]));
        sum[q] = two.x + two.y;
      }
      group_sum(sum, G, words, turn);
#pragma unroll
      for (int q = 0; q < R; ++q) {
        const float less = -(sum[q] * over);
#pragma unroll
        for (int i = 0; i < C; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[q][i][j] = add2(v[q][i][j], where_there<W>(less, i, j, at, D));
        }
      }
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      Pair sums[2] = {pair(0.0f, 0.0f), pair(0.0f, 0.0f)};
#pragma unroll
      for (int i = 0; i < C; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[j & 1] = fma2(v[q][i][j], v[q][i][j], sums[j & 1]);
      }
      const float2 two = halves(add2(sums[0], sums[1]));
      sum[q] = two.x + two.y;
    }
    group_sum(sum, G, words, turn);
    Pair r[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const float x = rsqrtf(sum[q] * over + p.eps);
      r[q] = pair(x, x);
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
      Pair g[4], b[4];
      gains.take(i, g, b);
#pragma unroll
      for (int q = 0; q < R; ++q) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[q][i][j] = fma2(mul2(v[q][i][j], r[q]), g[j], b[j]);
      }
    }
  }
  if constexpr (MODE == kNorm) {
#pragma unroll
    for (int q = 0; q < R; ++q) {
      T* y = static_cast<T*>(p.y.p) + row[q] * p.y.stride;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        if (there[q]) store8<W>(y, i, at, D, v[q][i]);
      }
    }
  } else {
    uint32_t tops[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      float most = 0.0f;
#pragma unroll
      for (int i = 0; i < C; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          // (what fills up the row may be a NaN here: 0 times an infinite factor)
          const float2 x = halves(v[q][i][j]);
          if (is_there<W>(i, 2 * j, at, D)) most = larger(most, x.x);
          if (is_there<W>(i, 2 * j + 1, at, D)) most = larger(most, x.y);
        }
      }
      tops[q] = __float_as_uint(most);
    }
    group_max(tops, G, words, turn);   // (by the bits, in which an infinity or a NaN is above all others)
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const float top = __uint_as_float(tops[q]), scale = __fdiv_rn(top, 127.0f);
      if (!there[q]) continue;
      const bool some = top <= FLT_MAX && scale > 0.0f;
      int8_t* codes = p.codes + row[q] * D;
      if (top > 0x1p-60f && top < 0x1p60f) {
        const float inverse = __frcp_rn(scale);
#pragma unroll
        for (int i = 0; i < C; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[q][i][j] = quotients(v[q][i][j], pair(-scale, -scale), pair(inverse, inverse));
        }
      } else {
        // (a subnormal scale has few bits: quotients by it may pass 127)
        auto held = [&](float x) { return some ? fminf(fmaxf(__fdiv_rn(x, scale), -127.0f), 127.0f) : 0.0f; };
#pragma unroll 1
        for (int i = 0; i < C; ++i) {
#pragma unroll
          for (int k = 0; k < C; ++k) {
            if (k != i) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 x = halves(v[q][k][j]);
              v[q][k][j] = pair(held(x.x), held(x.y));
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < C; ++i) {
        // rounded to nearest even by the sum with 1.5 * 2^23, whose last byte is the code
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = halves(add2(v[q][i][j], pair(0x1.8p23f, 0x1.8p23f)));
          c[2 * j] = __float_as_uint(x.x), c[2 * j + 1] = __float_as_uint(x.y);
        }
        if constexpr (W) {
          if (is_there<true>(i, 0, at, D))
            *reinterpret_cast<uint2*>(codes + feature<true>(i, 0, at)) =
                make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                           __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (is_there<false>(i, j, at, D)) codes[feature<false>(i, j, at)] = static_cast<int8_t>(c[j] & 0xff);
          }
        }
      }
      if (lane == 0) p.scale[row[q]] = top <= FLT_MAX ? scale : NAN;
    }
  }
}

// Gains as they lie in memory, or in registers.
template <bool W>
struct Gains {
  const NormParams& p;
  Place at;
  __device__ __forceinline__ void take(int i, Pair (&gain)[4], Pair (&bias)[4]) const {
    load_vector<W>(p.gain, 1.0f, i, at, p.dim, gain);
    load_vector<W>(p.bias, -0.0f, i, at, p.dim, bias);   // (adding -0 changes nothing)
  }
};

template <int C>
struct Kept {
  Pair g[C][4], b[C][4];
  __device__ __forceinline__ Kept(const NormParams& p, Place at) {
#pragma unroll
    for (int i = 0; i < C; ++i) load_vector<true>(p.gain, 1.0f, i, at, p.dim, g[i]), load_vector<true>(p.bias, -0.0f, i, at, p.dim, b[i]);
  }
  __device__ __forceinline__ void take(int i, Pair (&gain)[4], Pair (&bias)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) gain[j] = g[i][j], bias[j] = b[i][j];
  }
};

// Calls of many rows: a block takes two rows at a time, every gridDim-th, which share
// the sums' barriers, and `deep` - 1 pairs of them are on their way into shared memory
// meanwhile. The gains stay in registers (from the first-level cache they would be four times the
// bytes of a bf16 row).
template <typename T, int MODE>
__global__ void __launch_bounds__(512) norm_ahead_kernel(const NormParams p, int G, int deep) {
  constexpr int C = 2, R = 2;
  __shared__ __align__(16) float words[2 * 64];
  extern __shared__ __align__(16) unsigned char shared[];
  T* stages = reinterpret_cast<T*>(shared);
  wait_for_previous();
  let_next_start();
  const int lane = threadIdx.x, D = p.dim;
  const Place at = place_of<true>(lane, G, C);
  const bool added = MODE != kCodes && p.residual.p;
  const int row_size = added ? 2 * D : D;
  auto fetch = [&](long long first, int stage) {
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const long long row = first + q * static_cast<long long>(gridDim.x);
      T* to = stages + (stage * R + q) * row_size;
      if (row < p.rows) {
        copy_row<T, C>(static_cast<const T*>(p.x.p) + row * p.x.stride, to, G, D);
        if (added) copy_row<T, C>(static_cast<const T*>(p.residual.p) + row * p.residual.stride, to + D, G, D);
      }
    }
    sjd_kv_ops::copy_commit();   // (the group of rows that are not there is empty)
  };
  const long long step = static_cast<long long>(R) * gridDim.x;
  for (int i = 0; i + 1 < deep; ++i) fetch(blockIdx.x + i * step, i);
  const Kept<C> gains(p, at);
  int turn = 0, stage = 0;
  for (long long first = blockIdx.x; first < p.rows; first += step) {
    if (deep == 2) sjd_kv_ops::copy_wait<0>();
    else if (deep == 3) sjd_kv_ops::copy_wait<1>();
    else sjd_kv_ops::copy_wait<2>();
    fetch(first + (deep - 1) * step, stage == 0 ? deep - 1 : stage - 1);   // (where the rows before were)
    const T* from = stages + stage * R * row_size;
    if (++stage == deep) stage = 0;
    const long long row[R] = {first, first + gridDim.x};
    const bool there[R] = {true, row[1] < p.rows};   // (else what is left from another row, to no effect)
    Pair v[R][C][4], w[R][C][4];
#pragma unroll
    for (int q = 0; q < R; ++q) {
#pragma unroll
      for (int i = 0; i < C; ++i) {
        load_own8(from + q * row_size, i, at, D, v[q][i]);
        if (added) load_own8(from + q * row_size + D, i, at, D, w[q][i]);
      }
    }
    norm_rows<T, true, C, MODE, R>(p, row, there, lane, G, at, v, w, words, turn, gains);
  }
  sjd_kv_ops::copy_wait_all();
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
  const Place at = place_of<W>(lane, G, C);
  const long long mine = static_cast<long long>(blockIdx.x) * per + threadIdx.x / G, row[1] = {min(mine, p.rows - 1ll)};
  const bool there[1] = {mine < p.rows};
  int turn = 0;
  Pair v[1][C][4], w[1][C][4];
#pragma unroll
  for (int i = 0; i < C; ++i) load8<W>(static_cast<const T*>(p.x.p) + row[0] * p.x.stride, i, at, p.dim, v[0][i]);
  if (MODE != kCodes && p.residual.p) {
#pragma unroll
    for (int i = 0; i < C; ++i) load8<W>(static_cast<const T*>(p.residual.p) + row[0] * p.residual.stride, i, at, p.dim, w[0][i]);
  }
  norm_rows<T, W, C, MODE, 1>(p, row, there, lane, G, at, v, w, words, turn, Gains<W>{p, at});
}

bool aligned16(const void* p, long long stride, size_t size) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(stride) * size) & 15) == 0;
}
// (the stride of a single row is not looked at)
bool wide(const Rows& r, int rows, size_t size) { return !r.p || aligned16(r.p, rows > 1 ? r.stride : 0, size); }
bool wide(const float* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int threads_of(int dim, int pieces) { return ((dim + 8 * pieces - 1) / (8 * pieces) + 31) / 32 * 32; }

int lanes_of(int dim, int pieces, bool w) {   // of a warp
  int l = w ? 8 : 32;
  while (8 * pieces * l < dim) l *= 2;
  return l;
}

template <typename T, bool W, int C, int MODE>
cudaError_t norm_with(const NormParams& p, cudaStream_t s) {
  const int G = p.dim <= 8 * C * 32 ? lanes_of(p.dim, C, W) : threads_of(p.dim, C), threads = G <= 32 ? kShortBlock : G, per = threads / G;
  return launch_early(norm_kernel<T, W, C, MODE>, static_cast<unsigned>((static_cast<long long>(p.rows) + per - 1) / per), threads, 0, s, p, G);
}

constexpr int ahead_registers(int mode) { return mode == kCodes ? 64 : 128; }   // of norm_ahead_kernel, at most

// Blocks on an SM and rows on their way in each.
struct Flow {
  int per_sm, deep;
  size_t shared;
};
Flow flow_of(int threads, int registers, size_t row) {
  Flow f;
  f.per_sm = min(8, max(1, 65536 / registers / threads));
  while (f.per_sm > 1 && 2 * f.per_sm * row > 200 * 1024) --f.per_sm;
  f.deep = 4;
  while (f.deep > 2 && f.deep * f.per_sm * row > 128 * 1024) --f.deep;
  f.shared = f.deep * row;
  return f;
}
constexpr int kMostShared = 200 * 1024;   // dynamic shared memory of any call's block
static_assert(2 * sizeof(float) * kMaxFeatures <= kMostShared, "the columns' sums of the longest rows");

template <typename T, int MODE>
cudaError_t norm_ahead(const NormParams& p, int sms, const Flow& f, cudaStream_t s) {
  const cudaError_t e = allow_shared<norm_ahead_kernel<T, MODE>>(kMostShared);
  if (e != cudaSuccess) return e;
  return launch_early(norm_ahead_kernel<T, MODE>, static_cast<unsigned>(min(p.rows, sms * f.per_sm)), threads_of(p.dim, 2), f.shared, s, p,
                      threads_of(p.dim, 2), f.deep);
}

// 16200 rows of 1600, bf16, centred, with gain and bias: 27 us, 3.8 TB/s (a row at a time, 32
// features a thread: 33); issue slots and the sums' barriers bound it. 8100 rows of 4096: 30 us, and 23 with
// a gain alone, where a copy of them takes 21.6. 32 rows of 4096: 2.7 us. 8000 rows of 4097 with a
// residual, which cannot be accessed 16 bytes at a time: 77 us (147 with four pieces a thread).
// Codes of rows, without a norm: 7.3 us for 2048 rows of 4096, 1.9 for 32; a norm's codes of
// 2048 rows with a residual: 15.
template <typename T, bool W, int MODE>
cudaError_t norm_by(const NormParams& p, int sms, cudaStream_t s) {
  const bool few = p.rows <= 2 * sms;
  const int d = p.dim;
  if (d <= 256 || (few && d <= 4096)) return norm_with<T, W, 1, MODE>(p, s);
  if (W && !few && d > 512 && d <= 8192) {
    const Flow f = flow_of(threads_of(d, 2), ahead_registers(MODE), 2 * sizeof(T) * d * (MODE != kCodes && p.residual.p ? 2 : 1));
    if (f.shared <= kMostShared) return norm_ahead<T, MODE>(p, sms, f, s);
  }
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
// x: the row, which becomes u; dx: dh, where there is one, which becomes dx.
template <bool W, int C, typename Gain>
__device__ __forceinline__ void gradient_row(const NormGradientParams& p, int G, Place at, Pair (&x)[C][4], Pair (&dy)[C][4], Pair (&dx)[C][4],
                                             float* words, int& turn, Gain gain) {
  const int D = p.dim;
  const float over = 1.0f / static_cast<float>(D);
  const Pair zero = pair(0.0f, 0.0f);
  float less_mean_g = 0.0f;
  if (p.centre) {
    Pair sx = zero, sg = zero;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      Pair g[4];
      gain(i, g);
#pragma unroll
      for (int j = 0; j < 4; ++j) sx = add2(sx, x[i][j]), sg = fma2(dy[i][j], g[j], sg);
    }
    const float2 a = halves(sx), b = halves(sg);
    float sum[2] = {a.x + a.y, b.x + b.y};
    group_sum(sum, G, words, turn);
    const float less = -(sum[0] * over);
    less_mean_g = -(sum[1] * over);
#pragma unroll
    for (int i = 0; i < C; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i][j] = add2(x[i][j], where_there<W>(less, i, j, at, D));
    }
  }
  Pair sx = zero, sg = zero;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    Pair g[4];
    gain(i, g);
#pragma unroll
    for (int j = 0; j < 4; ++j) sx = fma2(x[i][j], x[i][j], sx), sg = fma2(mul2(dy[i][j], g[j]), x[i][j], sg);
  }
  const float2 a = halves(sx), b = halves(sg);
  float sum[2] = {a.x + a.y, b.x + b.y};
  group_sum(sum, G, words, turn);
  const float r = rsqrtf(sum[0] * over + p.eps), less_along = -(sum[1] * over * r);
  const Pair rr = pair(r, r), lg = pair(less_mean_g, less_mean_g), la = pair(less_along, less_along);
#pragma unroll
  for (int i = 0; i < C; ++i) {
    Pair g[4];
    gain(i, g);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[i][j] = mul2(x[i][j], rr);
      dx[i][j] = fma2(fma2(x[i][j], la, fma2(dy[i][j], g[j], lg)), rr, p.dh.p ? dx[i][j] : zero);
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
  const Place at = place_of<W>(lane, G, C);
  int turn = 0;
  Pair dgain[C][4] = {}, dbias[C][4] = {};
  for (long long first = static_cast<long long>(blockIdx.x) * per; first < p.rows; first += static_cast<long long>(gridDim.x) * per) {
    const long long mine = first + threadIdx.x / G, row = min(mine, p.rows - 1ll);
    Pair x[C][4], dy[C][4], dx[C][4];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      load8<W>(static_cast<const T*>(p.x.p) + row * p.x.stride, i, at, D, x[i]);
      load8<W>(static_cast<const T*>(p.dy.p) + row * p.dy.stride, i, at, D, dy[i]);
      if (p.dh.p) load8<W>(static_cast<const T*>(p.dh.p) + row * p.dh.stride, i, at, D, dx[i]);
    }
    gradient_row<W, C>(p, G, at, x, dy, dx, nullptr, turn, [&](int i, Pair (&g)[4]) { load_vector<W>(p.gain, 1.0f, i, at, D, g); });
    if (mine >= p.rows) continue;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      store8<W>(static_cast<T*>(p.dx.p) + row * p.dx.stride, i, at, D, dx[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) dgain[i][j] = fma2(dy[i][j], x[i][j], dgain[i][j]), dbias[i][j] = add2(dbias[i][j], dy[i][j]);
    }
  }
  __syncwarp();
  for (int o = G; o < 32; o *= 2) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        dgain[i][j] = add2(dgain[i][j], Pair{__shfl_xor_sync(0xffffffffu, dgain[i][j].v, o)});
        dbias[i][j] = add2(dbias[i][j], Pair{__shfl_xor_sync(0xffffffffu, dbias[i][j].v, o)});
      }
    }
  }
  for (int w = 0; w < kShortBlock / 32; ++w) {
    if (static_cast<int>(threadIdx.x / 32) == w && (threadIdx.x & 31) < static_cast<unsigned>(G)) {
#pragma unroll
      for (int i = 0; i < C; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int e = feature<W>(i, j, at);
          const float2 dg = halves(dgain[i][j / 2]), db = halves(dbias[i][j / 2]);
          if (e < D) sums[0][e] = (w ? sums[0][e] : 0.0f) + (j & 1 ? dg.y : dg.x), sums[1][e] = (w ? sums[1][e] : 0.0f) + (j & 1 ? db.y : db.x);
        }
      }
    }
    __syncthreads();
  }
  const int columns = D * (p.dbias ? 2 : 1);
  for (int e = threadIdx.x; e < columns; e += kShortBlock) p.parts[static_cast<long long>(blockIdx.x) * columns + e] = sums[e >= D][e >= D ? e - D : e];
}

// Longer rows (8100 of 4096, bf16, with what is added: 50 us, 5.3 TB/s, 102 without rows on
// their way; 12291 of 1600, f32, centred: 53 us, 4.5 TB/s; 4000 of 16384 in shared memory 259 us,
// which its reads and writes bound): a block takes every gridDim-th, and keeps the sums over its rows of
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
  const Place at = place_of<W>(lane, G, C);
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
  Pair dgain[WAY == kShared ? 1 : C][4] = {}, dbias[WAY == kShared ? 1 : C][4] = {}, gains[WAY == kShared ? 1 : C][4];
  if constexpr (WAY == kShared) {
    for (int i = lane; i < 2 * D; i += G) sums[i] = 0.0f;
    __syncthreads();
  } else {
    if constexpr (WAY == kAhead) {
      for (int i = 0; i + 1 < deep; ++i) fetch(blockIdx.x + static_cast<long long>(i) * gridDim.x, i);
    }
#pragma unroll
    for (int i = 0; i < C; ++i) load_vector<W>(p.gain, 1.0f, i, at, D, gains[i]);
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
    Pair x[C][4], dy[C][4], dx[C][4];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      if constexpr (WAY == kAhead) {
        load_own8(xs, i, at, D, x[i]);
        load_own8(dys, i, at, D, dy[i]);
        if (p.dh.p) load_own8(dhs, i, at, D, dx[i]);
      } else {
        load8<W>(xs, i, at, D, x[i]);
        load8<W>(dys, i, at, D, dy[i]);
        if (p.dh.p) load8<W>(dhs, i, at, D, dx[i]);
      }
    }
    gradient_row<W, C>(p, G, at, x, dy, dx, words, turn, [&](int i, Pair (&g)[4]) {
      if constexpr (WAY == kShared) {
        load_vector<W>(p.gain, 1.0f, i, at, D, g);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) g[j] = gains[i][j];
      }
    });
    T* dxs = static_cast<T*>(p.dx.p) + row * p.dx.stride;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      store8<W>(dxs, i, at, D, dx[i]);
      if constexpr (WAY == kShared) {
        // (a thread's own columns, four of them at a time where they are neighbours)
        if constexpr (W) {
          const int e = feature<true>(i, 0, at);
          if (e < D) {
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
              ulonglong2* a = reinterpret_cast<ulonglong2*>(sums + e + 2 * j);
              ulonglong2* b = reinterpret_cast<ulonglong2*>(sums + D + e + 2 * j);
              const ulonglong2 u = *a, v = *b;
              *a = make_ulonglong2(fma2(dy[i][j], x[i][j], Pair{u.x}).v, fma2(dy[i][j + 1], x[i][j + 1], Pair{u.y}).v);
              *b = make_ulonglong2(add2(dy[i][j], Pair{v.x}).v, add2(dy[i][j + 1], Pair{v.y}).v);
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int e = feature<false>(i, j, at);
            const float2 u = halves(x[i][j / 2]), d = halves(dy[i][j / 2]);
            if (e < D) sums[e] = fmaf(j & 1 ? d.y : d.x, j & 1 ? u.y : u.x, sums[e]), sums[D + e] += j & 1 ? d.y : d.x;
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) dgain[i][j] = fma2(dy[i][j], x[i][j], dgain[i][j]), dbias[i][j] = add2(dbias[i][j], dy[i][j]);
      }
    }
  }
  sjd_kv_ops::copy_wait_all();
  float* part = p.parts + static_cast<long long>(blockIdx.x) * (p.dbias ? 2 : 1) * D;
#pragma unroll
  for (int i = 0; i < C; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = feature<W>(i, j, at);
      if (e >= D) continue;
      const float2 dg = halves(dgain[WAY == kShared ? 0 : i][j / 2]), db = halves(dbias[WAY == kShared ? 0 : i][j / 2]);
      part[e] = WAY == kShared ? sums[e] : j & 1 ? dg.y : dg.x;
      if (p.dbias) part[D + e] = WAY == kShared ? sums[D + e] : j & 1 ? db.y : db.x;
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

// Blocks of the gradient's first kernel (of 128 registers a thread).
Flow gradient_flow(int dim, size_t size) {
  if (dim > 8192) return {1, 0, 2 * sizeof(float) * dim};
  return flow_of(threads_of(dim, 2), 128, 3 * size * dim);
}

template <typename T, bool W, int WAY>
cudaError_t norm_gradient_with(const NormGradientParams& p, const Flow& f, cudaStream_t s) {
  const int G = threads_of(p.dim, 2);
  const size_t shared = WAY == kDirect ? 0 : f.shared;
  const cudaError_t e = WAY == kDirect ? cudaSuccess : allow_shared<norm_gradient_kernel<T, W, WAY>>(kMostShared);
  if (e != cudaSuccess) return e;
  return launch_early(norm_gradient_kernel<T, W, WAY>, p.blocks, G, shared, s, p, G, f.deep);
}

template <typename T, bool W>
cudaError_t norm_gradient_by(const NormGradientParams& p, cudaStream_t s) {
  const int columns = p.dim * (p.dbias ? 2 : 1);
  const Flow f = gradient_flow(p.dim, sizeof(T));
  cudaError_t e;
  if (p.dim <= kShort / 2) e = launch_early(norm_gradient_short_kernel<T, W, 1>, p.blocks, kShortBlock, 0, s, p, lanes_of(p.dim, 1, W));
  else if (p.dim <= kShort) e = launch_early(norm_gradient_short_kernel<T, W, 2>, p.blocks, kShortBlock, 0, s, p, lanes_of(p.dim, 2, W));
  else if (p.dim > 8192) e = norm_gradient_with<T, W, kShared>(p, f, s);
  else if (W && f.shared <= kMostShared) e = norm_gradient_with<T, W, W ? kAhead : kDirect>(p, f, s);
  else e = norm_gradient_with<T, W, kDirect>(p, f, s);
  if (e != cudaSuccess) return e;
  return launch_early(add_parts_kernel, (columns + 31) / 32, 32 * kSumRows, 0, s, p, columns);
}

// --- embedding -----------------------------------------------------------------

// y[t] = scale table[tokens[t]], zeros where the token is no row of the table. A
// group of G threads to a row, four pieces of a thread on their way at a time (16200
// rows of 4096, bf16: 36 us).
constexpr int kEmbedBlock = 128;
template <typename E, typename T, bool W>
__global__ void __launch_bounds__(kEmbedBlock) embed_kernel(const EmbedParams p, int G) {
  constexpr int kDeep = 4;
  wait_for_previous();
  let_next_start();
  const long long row = static_cast<long long>(blockIdx.x) * (kEmbedBlock / G) + threadIdx.x / G;
  if (row >= p.rows) return;
  const int token = p.tokens[row], D = p.dim, lane = threadIdx.x % G;
  const bool inside = token >= 0 && token < p.vocab;
  const E* x = static_cast<const E*>(p.table.p) + (inside ? token : 0) * p.table.stride;
  T* y = static_cast<T*>(p.y.p) + row * p.y.stride;
  const int pieces = pieces_of(D, G);
  const Place at = place_of<W>(lane, G, pieces);
  for (int i0 = 0; i0 < pieces; i0 += kDeep) {
    float v[kDeep][8] = {};
    if (inside) {
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        if (is_mine<W>(i0 + i, pieces)) load8<W>(x, i0 + i, at, D, v[i]);
      }
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= p.scale;
      }
    }
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      if (is_mine<W>(i0 + i, pieces)) store8<W>(y, i0 + i, at, D, v[i]);
    }
  }
}

template <typename E, typename T>
cudaError_t embed_of(const EmbedParams& p, cudaStream_t s) {
  const bool w = p.dim % 8 == 0 && wide(p.table, p.vocab, sizeof(E)) && wide(p.y, p.rows, sizeof(T));
  const int G = p.dim <= 1024 ? lanes_of(p.dim, 4, w) : kEmbedBlock, per = kEmbedBlock / G;
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(p.rows) + per - 1) / per);
  return w ? launch_early(embed_kernel<E, T, true>, blocks, kEmbedBlock, 0, s, p, G) : launch_early(embed_kernel<E, T, false>, blocks, kEmbedBlock, 0, s, p, G);
}

// The rows of each id, ascending. A block takes kIds ids and looks through all
// tokens (they stay in L2; 12 us for 16200 of them): it counts those of its ids and those before them,
// which is where its part of `places` begins, and then puts the rows of its ids
// there. Warp w looks through the w-th part of the tokens both times, so that
// its rows of an id stand behind those of the warps before it. The ids that have
// more than p.few rows are listed.
constexpr int kIds = kListIds, kIndexWarps = 32;
__device__ __forceinline__ int4* many_of(const EmbedGradientParams& p, int list) { return p.many + static_cast<long long>(list) * (kIds + 1); }
__global__ void __launch_bounds__(32 * kIndexWarps) index_kernel(const EmbedGradientParams p) {
  constexpr int kDeep = 8;   // loads of a thread on their way
  __shared__ int at[kIndexWarps][kIds];
  __shared__ int before[kIndexWarps], sums[kIds / 32], n_many;
  wait_for_previous();
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, low = blockIdx.x * kIds;
  for (int i = lane; i < kIds; i += 32) at[warp][i] = 0;
  if (threadIdx.x == 0) n_many = 0;
  __syncwarp();
  const long long per = (static_cast<long long>(p.rows) + 32 * kIndexWarps - 1) / (32 * kIndexWarps) * 32;
  const long long begin = warp * per, end = min(static_cast<long long>(p.rows), begin + per);
  const int here = min(kIds, p.vocab - low);
  auto load = [&](long long t0, int (&token)[kDeep]) {
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const long long t = t0 + 32 * i + lane;
      token[i] = t < end ? p.tokens[t] : -1;
    }
  };
  int less = 0;
  for (long long t0 = begin; t0 < end; t0 += 32 * kDeep) {
    int token[kDeep];
    load(t0, token);
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const int id = token[i] - low;
      if (token[i] >= 0 && id < 0) ++less;
      if (token[i] >= low && id < here) atomicAdd(&at[warp][id], 1);
    }
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
    if (count > p.few) many_of(p, blockIdx.x)[1 + atomicAdd(&n_many, 1)] = make_int4(low + threadIdx.x, base, count, 0);
    if (low + static_cast<int>(threadIdx.x) == p.vocab - 1) p.first[p.vocab] = base + count;
    for (int w = 0; w < kIndexWarps; ++w) {
      const int n = at[w][threadIdx.x];
      at[w][threadIdx.x] = base;
      base += n;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) many_of(p, blockIdx.x)[0].x = n_many;
  for (long long t0 = begin; t0 < end; t0 += 32 * kDeep) {
    int token[kDeep];
    load(t0, token);
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const int id = token[i] - low;
      const bool mine = token[i] >= low && id < here;
      const unsigned which = __ballot_sync(0xffffffffu, mine);
      if (!which) continue;
      if (mine) {
        const unsigned same = __match_any_sync(which, id);
        p.places[SJD_KV_IDX(nullptr, at[warp][id] + __popc(same & ((1u << lane) - 1)), p.rows)] = static_cast<int>(t0 + 32 * i + lane);
        __syncwarp(which);
        if (lane == 31 - __clz(same)) at[warp][id] += __popc(same);
      }
      __syncwarp();
    }
  }
}

// (The bounds-checked build tests the index's places, rows and ids, and takes the nearest one.)
template <typename T>
__device__ __forceinline__ const T* row_of(const EmbedGradientParams& p, int row) {
  return static_cast<const T*>(p.dy.p) + SJD_KV_IDX(nullptr, row, p.rows) * p.dy.stride;
}
template <bool W, typename T>
__device__ __forceinline__ void load_columns(const T* p, float (&x)[W ? 4 : 1]) {
  if constexpr (W) sjd_kv_ops::load4(p, true, x);
  else x[0] = static_cast<float>(*p);
}
// The same past the first-level cache.
template <bool W, typename T>
__device__ __forceinline__ void load_columns_l2(const T* p, float (&x)[W ? 4 : 1]) {
  if constexpr (!W) {
    x[0] = static_cast<float>(__ldcg(p));
  } else if constexpr (sizeof(T) == 2) {
    const uint2 v = __ldcg(reinterpret_cast<const uint2*>(p));
    const float2 a = unpack_bf16(v.x), b = unpack_bf16(v.y);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  } else {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  }
}

// grad[v] = scale sum of dy over the rows of v, in their order (16000 rows of 4096 for 512 ids: 92 to 96
// us, of which the most frequent id's 2000 rows are most).
//
// The ids that have more than p.few rows are what most is read of. A block takes 128
// columns of its share of some lists: a warp an id, but for those of more than
// kMost rows, which are shared out to the block's warps, and their sums added up
// in order.
constexpr int kSumBlock = 256, kSumColumns = 128, kGroups = 8, kMost = 64, kPlaces = 512;
template <typename T, bool W>
__global__ void __launch_bounds__(kSumBlock, 2) embed_gradient_many_kernel(const EmbedGradientParams p, int slices, int shares, int groups, int lists) {
  constexpr int V = W ? 4 : 1, kDeep = W ? 16 : 8, kWarps = kSumBlock / 32, kPieces = kSumColumns / 32 / V;   // (pieces of a lane)
  __shared__ float sums[kWarps][kSumColumns];
  wait_for_previous();
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, D = p.dim;
  const int slice = blockIdx.x % slices, share = blockIdx.x / slices % shares, group = blockIdx.x / (slices * shares);
  auto column = [&](int c) { return slice * kSumColumns + (c * 32 + lane) * V; };
  auto add_rows = [&](int begin, int end, float (&sum)[kPieces][V]) {
    for (int r0 = begin; r0 < end; r0 += 32) {
      const int place = r0 + lane < end ? p.places[SJD_KV_IDX(nullptr, r0 + lane, p.rows)] : 0, rows = min(32, end - r0);
      for (int r = 0; r < rows; r += kDeep) {
        float x[kDeep][kPieces][V] = {};
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
          const int row = __shfl_sync(0xffffffffu, place, (r + u) & 31);
#pragma unroll
          for (int c = 0; c < kPieces; ++c) {
            if (r + u < rows && column(c) < D) load_columns<W>(row_of<T>(p, row) + column(c), x[u][c]);
          }
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
#pragma unroll
          for (int c = 0; c < kPieces; ++c) {
#pragma unroll
            for (int j = 0; j < V; ++j) sum[c][j] += x[u][c][j];   // (0 for those that are not there)
          }
        }
      }
    }
  };
  for (long long list0 = group; list0 < lists; list0 += 32ll * groups) {
    const long long of_lane = list0 + static_cast<long long>(lane) * groups;
    const int n_of_lane = of_lane < lists ? many_of(p, static_cast<int>(of_lane))[0].x : 0;
    for (unsigned some = __ballot_sync(0xffffffffu, n_of_lane > 0); some; some &= some - 1) {
      const int from_lane = __ffs(some) - 1, n = __shfl_sync(0xffffffffu, n_of_lane, from_lane);
      const int4* many = many_of(p, static_cast<int>(list0 + static_cast<long long>(from_lane) * groups)) + 1;
      for (int k = share * kWarps + warp; k < n; k += shares * kWarps) {
        const int4 id = many[k];   // the id, where its places begin, how many
        if (id.z > kMost) continue;
        float sum[kPieces][V] = {};
        add_rows(id.y, id.y + id.z, sum);
        float* out = p.grad + static_cast<long long>(SJD_KV_IDX(nullptr, id.x, p.vocab)) * D;
#pragma unroll
        for (int c = 0; c < kPieces; ++c) {
#pragma unroll
          for (int j = 0; j < V; ++j) sum[c][j] *= p.scale;
          if (column(c) >= D) continue;
          if constexpr (W) sjd_kv_ops::store4(out + column(c), true, sum[c]);
          else out[column(c)] = sum[c][0];
        }
      }
      for (int k0 = 0; k0 < n; k0 += 32) {
        const bool most = k0 + lane < n && many[k0 + lane].z > kMost;
        for (unsigned of = __ballot_sync(0xffffffffu, most); of; of &= of - 1) {
          const int k = k0 + __ffs(of) - 1;
          if (k % shares != share) continue;
          const int4 id = many[k];
          const int per = (id.z + kWarps - 1) / kWarps, begin = id.y + warp * per;
          float sum[kPieces][V] = {};
          add_rows(begin, min(begin + per, id.y + id.z), sum);
#pragma unroll
          for (int c = 0; c < kPieces; ++c) {
#pragma unroll
            for (int j = 0; j < V; ++j) sums[warp][(c * 32 + lane) * V + j] = sum[c][j];
          }
          __syncthreads();
          for (int i = threadIdx.x; i < kSumColumns; i += kSumBlock) {
            float all = 0.0f;
            for (int w = 0; w < kWarps; ++w) all += sums[w][i];
            if (slice * kSumColumns + i < D) p.grad[static_cast<long long>(SJD_KV_IDX(nullptr, id.x, p.vocab)) * D + slice * kSumColumns + i] = all * p.scale;
          }
          __syncthreads();
        }
      }
    }
  }
}

// The other ids (with the index and the kernel above 16200 rows of 4096 for 65536 ids: 209 to 214 us,
// 5.7 TB/s): what bounds it is the writing, so that a block writes
// neighbours, 64 KB of them (512-byte pieces of rows that lie apart: a third of the
// rate), and has few registers (32 warps' loads hide one another; half of them: 1.5
// times the time). A thread takes four columns at a time (one, where rows cannot be accessed
// four elements at a time).
//
// `early`: the kernel before this one on the stream is the one above, which writes other
// rows, and let this one in after the index was done: this one waits for it at its end, not
// at its beginning, so that the two run together. Its own wait has then not yet made
// what the index and the caller's kernels wrote visible to it, but the wait of the kernel
// above, which every block of that one has passed before the first block of this one starts, comes
// after those kernels' ends, when their writes stand in global memory. What this
// one must not do is find older values of those addresses in the first-level cache, which
// the other kernels' blocks on the SM share: it loads all of them (index, places and
// rows) past it, from L2.
template <typename T, bool W>
__global__ void __launch_bounds__(kSumBlock, 8) embed_gradient_kernel(const EmbedGradientParams p, int ids, int lanes, bool early) {
  constexpr int V = W ? 4 : 1;
  __shared__ int first[257], places[kPlaces];
  if (!early) {
    wait_for_previous();
    let_next_start();
  }
  const int D = p.dim, v0 = blockIdx.x * ids, here = min(ids, p.vocab - v0);
  for (int i = threadIdx.x; i <= here; i += kSumBlock) first[i] = __ldcg(p.first + v0 + i);
  __syncthreads();
  const int base = first[0], lane = threadIdx.x & (lanes - 1);
  if (first[here] > base) {
    for (int i = threadIdx.x; i < min(kPlaces, first[here] - base); i += kSumBlock) places[i] = __ldcg(p.places + SJD_KV_IDX(nullptr, base + i, p.rows));
    __syncthreads();
  }
  // `lanes` threads (a power of two) to an id
  for (int k = threadIdx.x / lanes; k < here; k += kSumBlock / lanes) {
    const int from = first[k] - base, count = first[k + 1] - base - from;
    if (count > p.few) continue;
    float* out = p.grad + SJD_KV_IDX(nullptr, static_cast<long long>(v0) + k, p.vocab) * D;
    for (int column = lane * V; column < D; column += lanes * V) {
      float sum[V] = {};
      for (int r = 0; r < count; ++r) {
        const int at = from + r;
        float x[V];
        load_columns_l2<W>(row_of<T>(p, at < kPlaces ? places[at] : __ldcg(p.places + SJD_KV_IDX(nullptr, base + at, p.rows))) + column, x);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += x[j];
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] *= p.scale;
      if constexpr (W) sjd_kv_ops::store4(out + column, true, sum);
      else out[column] = sum[0];
    }
  }
  if (early) {
    wait_for_previous();
    let_next_start();
  }
}

template <typename T>
cudaError_t embed_gradient_of(const EmbedGradientParams& p, int sms, cudaStream_t s) {
  const int lists = embed_gradient_lists(p.vocab);
  cudaError_t e = launch_early(index_kernel, static_cast<unsigned>(lists), 32 * kIndexWarps, 0, s, p);
  if (e != cudaSuccess) return e;
  const bool w = p.dim % 4 == 0 && reinterpret_cast<uintptr_t>(p.grad) % 16 == 0 && reinterpret_cast<uintptr_t>(p.dy.p) % (4 * sizeof(T)) == 0 &&
                 (p.rows < 2 || p.dy.stride % 4 == 0);
  int lanes = 8;
  while (lanes < kSumBlock && lanes * (w ? 4 : 1) < p.dim) lanes *= 2;
  // (64 KB to a block, or less where that leaves fewer than eight blocks to an SM)
  const int ids = max(kSumBlock / lanes, min(min(256, 16384 / p.dim), p.vocab / (8 * sms))), slices = (p.dim + kSumColumns - 1) / kSumColumns,
            groups = min(lists, kGroups), shares = max(1, min(min(64, 1024 / (slices * groups)), p.rows / (p.few * kSumBlock / 32 * groups) + 1));
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(p.vocab) + ids - 1) / ids);
  const bool many = p.rows > p.few;   // (some id may have so many)
  if (many) {
    const unsigned n = static_cast<unsigned>(slices) * shares * groups;
    e = w ? launch_early(embed_gradient_many_kernel<T, true>, n, kSumBlock, 0, s, p, slices, shares, groups, lists)
          : launch_early(embed_gradient_many_kernel<T, false>, n, kSumBlock, 0, s, p, slices, shares, groups, lists);
    if (e != cudaSuccess) return e;
  }
  return w ? launch_early(embed_gradient_kernel<T, true>, blocks, kSumBlock, 0, s, p, ids, lanes, many)
           : launch_early(embed_gradient_kernel<T, false>, blocks, kSumBlock, 0, s, p, ids, lanes, many);
}

}  // namespace

int embed_gradient_lists(int vocab) { return static_cast<int>((static_cast<long long>(vocab) + kIds - 1) / kIds); }

cudaError_t launch_norm(const NormParams& p, int mode, int dtype, int sms, cudaStream_t s) {
  return dtype == SJD_BF16 ? norm_of<__nv_bfloat16>(p, mode, sms, s) : norm_of<float>(p, mode, sms, s);
}

int norm_gradient_blocks(int rows, int dim, int dtype, int sms) {
  if (dim > kShort) return min(rows, sms * gradient_flow(dim, dtype == SJD_BF16 ? 2 : 4).per_sm);
  const int per = kShortBlock / lanes_of(dim, dim <= kShort / 2 ? 1 : 2, true);
  return static_cast<int>(min((static_cast<long long>(rows) + per - 1) / per, 8ll * sms));
}

cudaError_t launch_norm_gradient(const NormGradientParams& p, int dtype, cudaStream_t s) {
  const size_t size = dtype == SJD_BF16 ? 2 : 4;
  const bool w = p.dim % 8 == 0 && wide(p.dy, p.rows, size) && wide(p.x, p.rows, size) && wide(p.dh, p.rows, size) && wide(p.dx, p.rows, size) &&
                 wide(p.gain);
  if (dtype == SJD_BF16) return w ? norm_gradient_by<__nv_bfloat16, true>(p, s) : norm_gradient_by<__nv_bfloat16, false>(p, s);
  return w ? norm_gradient_by<float, true>(p, s) : norm_gradient_by<float, false>(p, s);
}

cudaError_t launch_embed(const EmbedParams& p, int table_dtype, int dtype, cudaStream_t s) {
  if (table_dtype == SJD_BF16) return dtype == SJD_BF16 ? embed_of<__nv_bfloat16, __nv_bfloat16>(p, s) : embed_of<__nv_bfloat16, float>(p, s);
  return dtype == SJD_BF16 ? embed_of<float, __nv_bfloat16>(p, s) : embed_of<float, float>(p, s);
}

cudaError_t launch_embed_gradient(const EmbedGradientParams& p, int dtype, int sms, cudaStream_t s) {
  return dtype == SJD_BF16 ? embed_gradient_of<__nv_bfloat16>(p, sms, s) : embed_gradient_of<float>(p, sms, s);
}

}  // namespace sjd_dense_ops
