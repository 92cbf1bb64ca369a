// Rotary positions with several axes, and the paged cache's write (rotating,
// quantising) and read.
//
// A block takes one token. Its threads first take the angles of the token's
// pairs, once for all heads, into shared memory; then each group of L threads
// (the power of two from D / 8 on) takes vectors of D elements, a chunk of 8
// elements to a thread, so that a pair's two elements meet in one thread and
// a vector's largest magnitude is log2 L shuffles away. Each vector is read
// and written once: the bound is HBM bandwidth, and for a few tokens the
// latency of one load, one angle and one store.

#include <cfloat>

#include "sjd_kv_device.cuh"

namespace sjd_kv_ops {

namespace {

constexpr int kBlock = 256;

__host__ __device__ int lanes_of(int chunks) {
  int l = 1;
  while (l < chunks) l *= 2;
  return l;
}

// Wide accesses of 4 elements: base and strides are multiples of their size.
__device__ __forceinline__ bool wide4(const View& v, int esize) {
  return ((reinterpret_cast<uintptr_t>(v.p) | static_cast<uintptr_t>(v.sb * esize) | static_cast<uintptr_t>(v.st * esize) |
           static_cast<uintptr_t>(v.sh * esize)) & (4 * esize - 1)) == 0;
}

__device__ __forceinline__ void angles(const Rope& r, long long token, float2* cs) {
  for (int i = threadIdx.x; i < r.pairs; i += kBlock) cs[i] = turn_of(r, r.positions + token * r.axes, i);
  __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kBlock) rotate_kernel(const RotateParams p) {
  let_next_start();
  wait_for_previous();
  __shared__ float2 cs[kMaxRotateDim / 2];
  const long long token = blockIdx.x;
  const int b = static_cast<int>(token / p.n), t = static_cast<int>(token % p.n);
  const int L = lanes_of(p.D / 8), c = threadIdx.x & (L - 1), groups = kBlock / L;
  const Chunk ch = chunk_at(c, p.rope.pairs, p.rope.interleaved);
  const bool wx = wide4(p.x, sizeof(T)), wy = wide4(p.y, sizeof(T));
  const T* x = static_cast<const T*>(p.x.p) + b * p.x.sb + t * p.x.st;
  T* y = static_cast<T*>(p.y.p) + b * p.y.sb + t * p.y.st;
  angles(p.rope, token, cs);
  if (8 * c >= p.D) return;
  float2 turn[4];
  if (ch.pair >= 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) turn[i] = cs[ch.pair + i];
  }
  for (int h = threadIdx.x / L; h < p.H; h += groups) {
    float u[4], w[4];
    load4(x + h * p.x.sh + ch.e0, wx, u);
    load4(x + h * p.x.sh + ch.e1, wx, w);
    if (ch.pair >= 0) turn_chunk(u, w, turn, p.rope.interleaved);
    store4(y + h * p.y.sh + ch.e0, wy, u);
    store4(y + h * p.y.sh + ch.e1, wy, w);
  }
}

template <typename T, int KV>
__global__ void __launch_bounds__(kBlock) write_kernel(const WriteParams p) {
  let_next_start();
  wait_for_previous();
  __shared__ float2 cs[kMaxDim / 2];
  const Cache& c = p.c;
  const long long token = blockIdx.x;
  const int b = static_cast<int>(token / c.n), t = static_cast<int>(token % c.n);
  const int2 span = span_of(c, b);
  if (t >= span.y) return;
  const uint32_t slot = vector_in(c, page_of(c, b, span.x + t), span.x + t, 0);  // head 0's
  const int L = lanes_of(c.D / 8), lane = threadIdx.x & (L - 1), groups = kBlock / L;
  const bool turned = p.rope.turns != nullptr, in = 8 * lane < c.D;
  const int n_q = p.q.p ? c.Hq : 0, n_vec = n_q + 2 * c.Hkv;
  if (turned) angles(p.rope, token, cs);
  const Chunk rot = turned ? chunk_at(lane, p.rope.pairs, p.rope.interleaved) : Chunk{8 * lane, 8 * lane + 4, -1};
  float2 turn[4];
  if (rot.pair >= 0 && in) {
#pragma unroll
    for (int i = 0; i < 4; ++i) turn[i] = cs[rot.pair + i];
  }
  // (the groups' rounds are the same for all, so that every thread takes part in the shuffles)
  for (int v0 = 0; v0 < n_vec; v0 += groups) {
    const int vec = v0 + threadIdx.x / L;
    const bool here = in && vec < n_vec, is_q = vec < n_q, is_k = !is_q && vec < n_q + c.Hkv;
    const View& src = is_q ? p.q : is_k ? p.k : p.v;
    const int h = is_q ? vec : is_k ? vec - n_q : vec - n_q - c.Hkv;
    const Chunk ch = is_q || is_k ? rot : Chunk{8 * lane, 8 * lane + 4, -1};
    float u[4] = {}, w[4] = {};
    if (here) {
      const T* x = static_cast<const T*>(src.p) + b * src.sb + t * src.st + h * src.sh;
      const bool wide = wide4(src, sizeof(T));
      load4(x + ch.e0, wide, u);
      load4(x + ch.e1, wide, w);
      if (ch.pair >= 0) turn_chunk(u, w, turn, p.rope.interleaved);
    }
    if (is_q) {
      if (here) {
        T* y = static_cast<T*>(p.q_out.p) + b * p.q_out.sb + t * p.q_out.st + h * p.q_out.sh;
        const bool wide = wide4(p.q_out, sizeof(T));
        store4(y + ch.e0, wide, u);
        store4(y + ch.e1, wide, w);
      }
      if constexpr (KV == SJD_BF16) continue;
    }
    using Code = typename Codes<KV>::type;
    const long long at = slot + static_cast<uint32_t>(h * c.ps);
    Code* out = static_cast<Code*>(is_k ? c.k : c.v) + at * c.D;
    if constexpr (KV == SJD_BF16) {
      if (here && slot != kNoVector) {
        store4(out + ch.e0, true, u);
        store4(out + ch.e1, true, w);
      }
    } else {
      // the vector's largest magnitude; infinite if a value is not finite
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = fabsf(u[i]), d = fabsf(w[i]);
        top = fmaxf(top, fmaxf(a <= FLT_MAX ? a : INFINITY, d <= FLT_MAX ? d : INFINITY));
      }
      for (int o = L / 2; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float scale = __fdiv_rn(top, Codes<KV>::kMost);
      const bool some = top <= FLT_MAX && scale > 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u[i] = some ? __fdiv_rn(u[i], scale) : 0.0f;
        w[i] = some ? __fdiv_rn(w[i], scale) : 0.0f;
      }
      if (here && !is_q && slot != kNoVector) {
        *reinterpret_cast<uint32_t*>(out + ch.e0) = codes4<KV>(u);
        *reinterpret_cast<uint32_t*>(out + ch.e1) = codes4<KV>(w);
        if (lane == 0) (is_k ? c.ks : c.vs)[at] = top <= FLT_MAX ? scale : NAN;
      }
    }
  }
}

template <typename T, int KV>
__global__ void __launch_bounds__(kBlock) read_kernel(const ReadParams p) {
  let_next_start();
  wait_for_previous();
  const Cache& c = p.c;
  const long long token = blockIdx.x;
  const int b = static_cast<int>(token / c.n), t = static_cast<int>(token % c.n);
  const int2 span = span_of(c, b);
  const uint32_t slot = t < span.y ? vector_in(c, page_of(c, b, span.x + t), span.x + t, 0) : kNoVector;
  const int L = lanes_of(c.D / 8), lane = threadIdx.x & (L - 1), groups = kBlock / L;
  if (8 * lane >= c.D) return;
  using Code = typename Codes<KV>::type;
  for (int vec = threadIdx.x / L; vec < 2 * c.Hkv; vec += groups) {
    const bool is_k = vec < c.Hkv;
    const int h = is_k ? vec : vec - c.Hkv;
    float u[4] = {}, w[4] = {};
    if (slot != kNoVector) {
      const long long at = slot + static_cast<uint32_t>(h * c.ps);
      const Code* x = static_cast<const Code*>(is_k ? c.k : c.v) + at * c.D + 8 * lane;
      if constexpr (KV == SJD_BF16) {
        load4(x, true, u);
        load4(x + 4, true, w);
      } else {
        const uint2 q = *reinterpret_cast<const uint2*>(x);
        const float scale = (is_k ? c.ks : c.vs)[at];
        values4<KV>(q.x, u);
        values4<KV>(q.y, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] *= scale, w[i] *= scale;
      }
    }
    T* y = static_cast<T*>(is_k ? p.k_out : p.v_out) + (token * c.Hkv + h) * c.D + 8 * lane;
    store4(y, true, u);
    store4(y + 4, true, w);
  }
}

template <typename T>
cudaError_t write_of(const WriteParams& p, int kv_dtype, cudaStream_t s) {
  const unsigned blocks = static_cast<unsigned>(p.c.B) * p.c.n;
  if (kv_dtype == SJD_BF16) return launch_early(write_kernel<T, SJD_BF16>, blocks, kBlock, 0, s, p);
  if (kv_dtype == SJD_E4M3) return launch_early(write_kernel<T, SJD_E4M3>, blocks, kBlock, 0, s, p);
  return launch_early(write_kernel<T, SJD_S8>, blocks, kBlock, 0, s, p);
}

template <typename T>
cudaError_t read_of(const ReadParams& p, int kv_dtype, cudaStream_t s) {
  const unsigned blocks = static_cast<unsigned>(p.c.B) * p.c.n;
  if (kv_dtype == SJD_BF16) return launch_early(read_kernel<T, SJD_BF16>, blocks, kBlock, 0, s, p);
  if (kv_dtype == SJD_E4M3) return launch_early(read_kernel<T, SJD_E4M3>, blocks, kBlock, 0, s, p);
  return launch_early(read_kernel<T, SJD_S8>, blocks, kBlock, 0, s, p);
}

}  // namespace

cudaError_t launch_rotate(const RotateParams& p, int dtype, cudaStream_t s) {
  const unsigned blocks = static_cast<unsigned>(p.B) * p.n;
  if (dtype == SJD_BF16) return launch_early(rotate_kernel<__nv_bfloat16>, blocks, kBlock, 0, s, p);
  return launch_early(rotate_kernel<float>, blocks, kBlock, 0, s, p);
}

cudaError_t launch_write(const WriteParams& p, int dtype, int kv_dtype, cudaStream_t s) {
  return dtype == SJD_BF16 ? write_of<__nv_bfloat16>(p, kv_dtype, s) : write_of<float>(p, kv_dtype, s);
}

cudaError_t launch_read(const ReadParams& p, int dtype, int kv_dtype, cudaStream_t s) {
  return dtype == SJD_BF16 ? read_of<__nv_bfloat16>(p, kv_dtype, s) : read_of<float>(p, kv_dtype, s);
}

}  // namespace sjd_kv_ops
