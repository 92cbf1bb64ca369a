// Rotary positions with several axes, and the paged cache's write (rotating,
// quantising) and read.
//
// All three move data through once, so HBM bandwidth bounds the long calls and
// one chain of loads the short ones. A block takes a few tokens (one of a
// short call, eight of a long one). Some of its threads find the tokens' places
// in the cache and take the angles of their pairs, once for all heads, into
// shared memory, while the loads of the first vectors are on their way. Then a
// thread takes chunks of 8 elements, such that a pair's two elements meet in
// one thread. A vector that is quantised is taken by a group of L threads, a
// power of two, two or three chunks to a thread, and its largest magnitude is
// found in log2 L shuffles.

#include <cfloat>

#include "sjd_kv_device.cuh"

namespace sjd_kv_ops {

namespace {

constexpr int kBlock = 256;
constexpr int kTokens = 8;   // most tokens of a block

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

// A call's tokens (B * n, below 2^31) shared out to the blocks, with what
// divides by the numbers that the kernels divide by.
struct Share {
  int per, n, chunks, lanes; // tokens of a block, of a sequence; chunks of a vector; threads of a vector that is quantised
  Divisor by_n, by_chunks, by_vectors;  // (vectors of a token)
};
struct Tokens {
  int first, count;
};
__device__ __forceinline__ Tokens tokens_of_block(const Share& s, int B) {
  const int first = static_cast<int>(blockIdx.x) * s.per;
  return {first, min(s.per, B * s.n - first)};
}
__device__ __forceinline__ int over(int x, const Divisor& d) { return divide(x, d.mul, d.shift); }

__device__ __forceinline__ void angles(const Rope& r, const Tokens& at, float2* cs) {
  for (int i = threadIdx.x; i < at.count * r.pairs; i += kBlock)
    cs[i] = turn_of(r, r.positions + static_cast<long long>(at.first + i / r.pairs) * r.axes, i % r.pairs);
}

// Three sequences of 4097 tokens, 20 heads of 80, f32: 28 us, 5.6 TB/s
// (83 % of the copy rate; half of the issue slots), 47 us with one token to a
// block. 32 tokens: 11 us a call, the host's.
template <typename T>
__global__ void __launch_bounds__(kBlock) rotate_kernel(const RotateParams p, const Share share) {
  __shared__ float2 cs[kTokens * kMaxRotateDim / 2];
  wait_for_previous();
  let_next_start();
  const Tokens at = tokens_of_block(share, p.B);
  const bool wx = wide4(p.x, sizeof(T)), wy = wide4(p.y, sizeof(T));
  const int items = at.count * p.H * share.chunks;
  float u[4], w[4];
  struct Place {
    int token, h, c;
  };
  auto place = [&](int i) {
    const int vec = over(i, share.by_chunks), token = over(vec, share.by_vectors);
    return Place{token, vec - token * p.H, i - vec * share.chunks};
  };
  auto address = [&](const View& v, const Place& q) {
    const int token = at.first + q.token, b = over(token, share.by_n), t = token - b * p.n;
    return static_cast<T*>(v.p) + b * v.sb + t * v.st + q.h * v.sh;
  };
  auto fetch = [&](int i) {
    const Place q = place(i);
    const Chunk ch = chunk_at(q.c, p.rope.pairs, p.rope.interleaved);
    const T* x = address(p.x, q);
    load4(x + ch.e0, wx, u);
    load4(x + ch.e1, wx, w);
  };
  if (threadIdx.x < items) fetch(threadIdx.x);
  angles(p.rope, at, cs);
  __syncthreads();
  for (int i = threadIdx.x; i < items; i += kBlock) {
    if (i != threadIdx.x) fetch(i);
    const Place q = place(i);
    const Chunk ch = chunk_at(q.c, p.rope.pairs, p.rope.interleaved);
    if (ch.pair >= 0) turn_chunk(u, w, cs + q.token * p.rope.pairs + ch.pair, p.rope.interleaved);
    T* y = address(p.y, q);
    store4(y + ch.e0, wy, u);
    store4(y + ch.e1, wy, w);
  }
}

// x / scale of four values, as IEEE division rounds it. With the reciprocal
// rounded to nearest, two corrections by the exact remainder give the nearest
// quotient (Markstein, IBM J. Res. Dev. 34, 1990), as long as the remainders of
// quotients that matter do not underflow: for scales within 2^60 of 1.
__device__ __forceinline__ void quotients(float (&x)[4], float scale, float inverse) {
  const Pair less = pair(-scale, -scale), inv = pair(inverse, inverse);
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const Pair v = pair(x[i], x[i + 1]);
    Pair q = mul2(v, inv);
    q = fma2(fma2(q, less, v), inv, q);
    const float2 r = halves(fma2(fma2(q, less, v), inv, q));
    x[i] = r.x, x[i + 1] = r.y;
  }
}

// A subnormal scale has few bits, and a quotient by it may pass the largest code (100 / 127
// of the least number is that number: quotients up to 190).
__device__ __forceinline__ float held(float x, float most) { return fminf(fmaxf(x, -most), most); }

// CP chunks of a vector to a thread: chunk i * L + lane. Four sequences of
// 8100 tokens, 16 heads of 96, f32 to s8, not rotated: 86 us, 5.8 TB/s (86 %
// of the copy rate); 410 with one token to a block, one chunk to a thread and
// plain divisions. 32 windows of 64, keys and queries rotated, bf16 to e4m3: 18 us.
//
// With queries (Q) a warp whose vectors are all queries leaves out the codes: 18
// us instead of 20.5 in the windows above. The vote for it costs the images 11 us
// (86 against 97), so that calls without queries have a kernel without it.
template <typename T, int KV, int CP, bool Q>
__global__ void __launch_bounds__(kBlock) write_kernel(const WriteParams p, const Share share) {
  __shared__ float2 cs[kTokens * kMaxDim / 2];
  __shared__ uint32_t slots[kTokens];   // the tokens' places for head 0
  __shared__ int there[kTokens];        // whether the token is in its sequence's span
  const Cache& c = p.c;
  wait_for_previous();
  let_next_start();
  const Tokens at = tokens_of_block(share, c.B);
  const int L = share.lanes, lane = threadIdx.x & (L - 1), groups = kBlock / L;
  const bool turned = p.rope.turns != nullptr;
  const int n_q = Q ? c.Hq : 0, n_vec = n_q + 2 * c.Hkv, items = at.count * n_vec;
  const bool wq = wide4(p.q, sizeof(T)), wk = wide4(p.k, sizeof(T)), wv = wide4(p.v, sizeof(T)), wo = wide4(p.q_out, sizeof(T));
  struct Place {
    int token, vec, b, t;
  };
  auto chunk_of = [&](int i, bool turn) {
    const int at = i * L + lane;
    return turn ? chunk_at(at, p.rope.pairs, p.rope.interleaved) : Chunk{8 * at, 8 * at + 4, -1};
  };
  float u[CP][4], w[CP][4];
  Place q;
  auto fetch = [&](int item) {
    const int token = over(item, share.by_vectors), of_call = at.first + token, b = over(of_call, share.by_n);
    q = {token, item - token * n_vec, b, of_call - b * c.n};
    const bool is_q = q.vec < n_q, is_k = !is_q && q.vec < n_q + c.Hkv;
    const View& src = is_q ? p.q : is_k ? p.k : p.v;
    const int h = is_q ? q.vec : is_k ? q.vec - n_q : q.vec - n_q - c.Hkv;
    const T* x = static_cast<const T*>(src.p) + q.b * src.sb + q.t * src.st + h * src.sh;
    const bool wide = is_q ? wq : is_k ? wk : wv;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const Chunk ch = chunk_of(i, turned && (is_q || is_k));
#pragma unroll
      for (int j = 0; j < 4; ++j) u[i][j] = w[i][j] = 0.0f;
      if (8 * (i * L + lane) < c.D) {
        load4(x + ch.e0, wide, u[i]);
        load4(x + ch.e1, wide, w[i]);
      }
    }
  };
  // (a group past the last vector takes the first again and stores nothing, so
  // that every thread takes part in the shuffles)
  int item = threadIdx.x / L;
  fetch(item < items ? item : 0);
  if (threadIdx.x < at.count) {
    const int of_call = at.first + threadIdx.x, b = over(of_call, share.by_n), t = of_call - b * c.n;
    const int2 span = span_of(c, b);
    there[threadIdx.x] = t < span.y;
    slots[threadIdx.x] = t < span.y ? vector_in(c, page_of(c, b, span.x + t), span.x + t, 0) : kNoVector;
  }
  if (turned) angles(p.rope, at, cs);
  __syncthreads();
  for (int i0 = 0; i0 < items; i0 += groups, item += groups) {
    if (i0 != 0) fetch(item < items ? item : 0);
    const bool is_q = q.vec < n_q, is_k = !is_q && q.vec < n_q + c.Hkv, turn = turned && (is_q || is_k);
    const int h = is_q ? q.vec : is_k ? q.vec - n_q : q.vec - n_q - c.Hkv;
    if (turn) {
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const Chunk ch = chunk_of(i, true);
        if (ch.pair >= 0) turn_chunk(u[i], w[i], cs + q.token * p.rope.pairs + ch.pair, p.rope.interleaved);
      }
    }
    if (is_q && item < items && there[q.token]) {
      T* y = static_cast<T*>(p.q_out.p) + q.b * p.q_out.sb + q.t * p.q_out.st + h * p.q_out.sh;
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const Chunk ch = chunk_of(i, turn);
        if (8 * (i * L + lane) < c.D) {
          store4(y + ch.e0, wo, u[i]);
          store4(y + ch.e1, wo, w[i]);
        }
      }
    }
    if (Q && __all_sync(0xffffffffu, is_q || item >= items)) continue;
    using Code = typename Codes<KV>::type;
    const uint32_t slot = slots[q.token];
    const bool store = item < items && !is_q && slot != kNoVector;
    const long long vector = slot + static_cast<uint32_t>(h * c.ps);
    Code* out = static_cast<Code*>(is_k ? c.k : c.v) + vector * c.D;
    if constexpr (KV != SJD_BF16) {
      // the vector's largest magnitude, by its bits: an infinity or a NaN is above all others
      uint32_t bits = 0;
#pragma unroll
      for (int i = 0; i < CP; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) bits = max(bits, max(__float_as_uint(u[i][j]) & 0x7fffffffu, __float_as_uint(w[i][j]) & 0x7fffffffu));
      }
      for (int o = L / 2; o > 0; o /= 2) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, o));
      const float top = __uint_as_float(bits), scale = __fdiv_rn(top, Codes<KV>::kMost);
      if (top > 0x1p-60f && top < 0x1p60f) {
        const float inverse = __frcp_rn(scale);
#pragma unroll
        for (int i = 0; i < CP; ++i) {
          quotients(u[i], scale, inverse);
          quotients(w[i], scale, inverse);
        }
      } else {
        const bool some = top <= FLT_MAX && scale > 0.0f;
#pragma unroll
        for (int i = 0; i < CP; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            u[i][j] = some ? held(__fdiv_rn(u[i][j], scale), Codes<KV>::kMost) : 0.0f;
            w[i][j] = some ? held(__fdiv_rn(w[i][j], scale), Codes<KV>::kMost) : 0.0f;
          }
        }
      }
      if (store && lane == 0) (is_k ? c.ks : c.vs)[vector] = top <= FLT_MAX ? scale : NAN;
    }
    if (store) {
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const Chunk ch = chunk_of(i, turn);
        if (8 * (i * L + lane) >= c.D) continue;
        if constexpr (KV == SJD_BF16) {
          store4(out + ch.e0, true, u[i]);
          store4(out + ch.e1, true, w[i]);
        } else {
          *reinterpret_cast<uint32_t*>(out + ch.e0) = codes4<KV>(u[i]);
          *reinterpret_cast<uint32_t*>(out + ch.e1) = codes4<KV>(w[i]);
        }
      }
    }
  }
}

// Up to 8100 tokens of 16 sequences, 8 heads of 128, e4m3 to bf16: 120 us,
// 5.2 TB/s (77 % of the copy rate, three quarters of the issue slots: conversion);
// 4 x 8100 tokens of 16 heads of 96, s8 to bf16: 53 us, 5.7 TB/s.
template <typename T, int KV>
__global__ void __launch_bounds__(kBlock) read_kernel(const ReadParams p, const Share share) {
  __shared__ uint32_t slots[kTokens];
  const Cache& c = p.c;
  wait_for_previous();
  let_next_start();
  const Tokens at = tokens_of_block(share, c.B);
  if (threadIdx.x < at.count) {
    const int of_call = at.first + threadIdx.x, b = over(of_call, share.by_n), t = of_call - b * c.n;
    const int2 span = span_of(c, b);
    slots[threadIdx.x] = t < span.y ? vector_in(c, page_of(c, b, span.x + t), span.x + t, 0) : kNoVector;
  }
  __syncthreads();
  using Code = typename Codes<KV>::type;
  constexpr int kDeep = 4;   // chunks of a thread on their way
  const int chunks = share.chunks, items = at.count * 2 * c.Hkv * chunks;
  for (int i0 = threadIdx.x; i0 < items; i0 += kDeep * kBlock) {
    uint4 codes[kDeep];        // (8 codes take half of it)
    float scale[kDeep];
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      codes[k] = make_uint4(0, 0, 0, 0);
      scale[k] = 0.0f;
      const int i = i0 + k * kBlock;
      if (i >= items) continue;
      const int vec = over(i, share.by_chunks), token = over(vec, share.by_vectors), of = vec - token * 2 * c.Hkv;
      const bool is_k = of < c.Hkv;
      const uint32_t slot = slots[token];
      if (slot == kNoVector) continue;
      const long long vector = slot + static_cast<uint32_t>((is_k ? of : of - c.Hkv) * c.ps);
      const Code* x = static_cast<const Code*>(is_k ? c.k : c.v) + vector * c.D + 8 * (i - vec * chunks);
      if constexpr (KV == SJD_BF16) {
        codes[k] = *reinterpret_cast<const uint4*>(x);
      } else {
        const uint2 q = *reinterpret_cast<const uint2*>(x);
        codes[k].x = q.x, codes[k].y = q.y;
        scale[k] = (is_k ? c.ks : c.vs)[vector];
      }
    }
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      const int i = i0 + k * kBlock;
      if (i >= items) continue;
      const int vec = over(i, share.by_chunks), token = over(vec, share.by_vectors), of = vec - token * 2 * c.Hkv;
      const bool is_k = of < c.Hkv;
      float u[4], w[4];
      if constexpr (KV == SJD_BF16) {
        const float2 a = unpack_bf16(codes[k].x), b = unpack_bf16(codes[k].y), d = unpack_bf16(codes[k].z), e = unpack_bf16(codes[k].w);
        u[0] = a.x, u[1] = a.y, u[2] = b.x, u[3] = b.y, w[0] = d.x, w[1] = d.y, w[2] = e.x, w[3] = e.y;
      } else {
        values4<KV>(codes[k].x, u);
        values4<KV>(codes[k].y, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] *= scale[k], w[j] *= scale[k];
      }
      T* y = static_cast<T*>(is_k ? p.k_out : p.v_out) + (static_cast<long long>(at.first + token) * c.Hkv + (is_k ? of : of - c.Hkv)) * c.D + 8 * (i - vec * chunks);
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(y) = make_uint4(pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]));
      } else {
        store4(y, true, u);
        store4(y + 4, true, w);
      }
    }
  }
}

// Tokens of a block: as many as leave each of `sms` SMs four blocks, at most kTokens (32 windows of
// 64 rotated and written: 18.1 us; 19.6 where eight or sixteen are left).
Share share_of(int B, int n, int dim, int vectors, int sms) {
  const long long tokens = static_cast<long long>(B) * n, fair = tokens / (4 * sms);
  const int per = static_cast<int>(fair < 1 ? 1 : fair < kTokens ? fair : kTokens);
  return {per, n, dim / 8, 0, divisor(n), divisor(dim / 8), divisor(vectors)};
}
unsigned blocks_of(const Share& s, int B) { return static_cast<unsigned>((static_cast<long long>(B) * s.n + s.per - 1) / s.per); }

template <typename T, int CP, bool Q>
cudaError_t write_by(const WriteParams& p, const Share& share, int kv_dtype, cudaStream_t s) {
  const unsigned blocks = blocks_of(share, p.c.B);
  if (kv_dtype == SJD_BF16) return launch_early(write_kernel<T, SJD_BF16, CP, Q>, blocks, kBlock, 0, s, p, share);
  if (kv_dtype == SJD_E4M3) return launch_early(write_kernel<T, SJD_E4M3, CP, Q>, blocks, kBlock, 0, s, p, share);
  return launch_early(write_kernel<T, SJD_S8, CP, Q>, blocks, kBlock, 0, s, p, share);
}

// Two chunks to a thread, or three where that leaves fewer threads of the
// group without one (9 to 12 chunks: heads of 72 to 96. The images above: 86
// us with three, 118 with two).
template <typename T>
cudaError_t write_of(const WriteParams& p, int kv_dtype, int sms, cudaStream_t s) {
  Share share = share_of(p.c.B, p.c.n, p.c.D, (p.q.p ? p.c.Hq : 0) + 2 * p.c.Hkv, sms);
  const int two = lanes_of((share.chunks + 1) / 2), three = lanes_of((share.chunks + 2) / 3);
  if (3 * three < 2 * two) {
    share.lanes = three;
    return p.q.p ? write_by<T, 3, true>(p, share, kv_dtype, s) : write_by<T, 3, false>(p, share, kv_dtype, s);
  }
  share.lanes = two;
  return p.q.p ? write_by<T, 2, true>(p, share, kv_dtype, s) : write_by<T, 2, false>(p, share, kv_dtype, s);
}

template <typename T>
cudaError_t read_of(const ReadParams& p, int kv_dtype, int sms, cudaStream_t s) {
  const Share share = share_of(p.c.B, p.c.n, p.c.D, 2 * p.c.Hkv, sms);
  const unsigned blocks = blocks_of(share, p.c.B);
  if (kv_dtype == SJD_BF16) return launch_early(read_kernel<T, SJD_BF16>, blocks, kBlock, 0, s, p, share);
  if (kv_dtype == SJD_E4M3) return launch_early(read_kernel<T, SJD_E4M3>, blocks, kBlock, 0, s, p, share);
  return launch_early(read_kernel<T, SJD_S8>, blocks, kBlock, 0, s, p, share);
}

}  // namespace

cudaError_t launch_rotate(const RotateParams& p, int dtype, int sms, cudaStream_t s) {
  const Share share = share_of(p.B, p.n, p.D, p.H, sms);
  const unsigned blocks = blocks_of(share, p.B);
  if (dtype == SJD_BF16) return launch_early(rotate_kernel<__nv_bfloat16>, blocks, kBlock, 0, s, p, share);
  return launch_early(rotate_kernel<float>, blocks, kBlock, 0, s, p, share);
}

cudaError_t launch_write(const WriteParams& p, int dtype, int kv_dtype, int sms, cudaStream_t s) {
  return dtype == SJD_BF16 ? write_of<__nv_bfloat16>(p, kv_dtype, sms, s) : write_of<float>(p, kv_dtype, sms, s);
}

cudaError_t launch_read(const ReadParams& p, int dtype, int kv_dtype, int sms, cudaStream_t s) {
  return dtype == SJD_BF16 ? read_of<__nv_bfloat16>(p, kv_dtype, sms, s) : read_of<float>(p, kv_dtype, sms, s);
}

}  // namespace sjd_kv_ops
