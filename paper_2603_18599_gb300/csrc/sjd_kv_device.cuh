// Device helpers of the window forward's operators: spans and pages, elements
// of the tensors' and the cache's types, rotary angles.
#pragma once

#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "sjd_kv.h"

namespace sjd_kv_ops {

// The kernels are launched while the one before them on the stream drains:
// this waits until it is done. Nothing is read or written before, and the next
// kernel is let in only then, so that what is done before a call on the stream
// is done when anything after the call starts.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Bounds-checked build (compiled with SJD_CHECKS): an index of a page table, of
// the cache's vectors, of the rotary axes, of the rows of a call and of the parts that blocks
// leave for one another is tested against its array's length; one outside latches
// SJD_ERR_BOUNDS in the status word (where there is one) and is clamped. Without
// SJD_CHECKS the macro is the index itself.
#ifdef SJD_CHECKS
__device__ __forceinline__ long long checked_index(uint32_t* status, long long i, long long n) {
  if (i >= 0 && i < n) return i;
  if (status) atomicOr(status, status_bit(SJD_ERR_BOUNDS));
  return i < 0 ? 0 : n - 1;
}
#define SJD_KV_IDX(status, i, n) checked_index((status), (i), (n))
#else
#define SJD_KV_IDX(status, i, n) (i)
#endif

// Sequence b's span of the call, {0, 0} where it does not fit its table.
__device__ __forceinline__ int2 span_of(const Cache& c, int b) {
  const int start = c.start[b], count = c.count ? c.count[b] : c.n;
  const long long room = static_cast<long long>(c.max_pages) * c.ps;
  if (start < 0 || count < 0 || count > c.n || start + static_cast<long long>(count) > room) {
    atomicOr(c.status, status_bit(SJD_ERR_PAGE));
    return make_int2(0, 0);
  }
  return make_int2(start, count);
}

// Vectors (of head_dim elements) of the cache are counted in 32 bits.
constexpr uint32_t kNoVector = 0xffffffffu;
constexpr int kNoPage = -0x7fffffff - 1;  // a token that is not there

__host__ __device__ __forceinline__ int divide(int x, uint32_t mul, int shift) {
  return static_cast<int>(static_cast<unsigned long long>(static_cast<uint32_t>(x)) * mul >> (31 + shift));
}
__device__ __forceinline__ int entry_of(const Cache& c, int pos) { return divide(pos, c.ps_mul, c.ps_shift); }
__host__ __device__ __forceinline__ int by_group(const Cache& c, int x) { return divide(x, c.group_mul, c.group_shift); }

// The table's entry of token pos of sequence b, as it stands there.
__device__ __forceinline__ int page_of(const Cache& c, int b, int pos) {
  return c.table[static_cast<long long>(b) * c.max_pages + SJD_KV_IDX(c.status, entry_of(c, pos), c.max_pages)];
}
// Token pos's vector of head h, or none where the page is no page of the cache.
__device__ __forceinline__ uint32_t vector_in(const Cache& c, int page, int pos, int h) {
  if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(c.n_pages)) {
    if (page != kNoPage) atomicOr(c.status, status_bit(SJD_ERR_PAGE));
    return kNoVector;
  }
  return static_cast<uint32_t>(SJD_KV_IDX(c.status, (static_cast<uint32_t>(page) * c.Hkv + h) * c.ps + (pos - entry_of(c, pos) * c.ps),
                                          static_cast<long long>(c.n_pages) * c.Hkv * c.ps));
}

constexpr int kTile = 128;              // rows of an attention's product, and keys of a tile

// The keys that some row of item mt (128 NM rows) of a span sees: 0 .. keys - 1.
template <int NM>
__host__ __device__ __forceinline__ int keys_of(const AttendParams& p, int start, int count, int mt) {
  if (p.mask_kind != SJD_MASK_CAUSAL) return start + count;
  return start + by_group(p.c, min((mt + 1) * (kTile * NM), count * p.c.group) - 1) + 1;
}

// Key tiles of one key head of a sequence, all its items.
template <int NM>
__host__ __device__ long long tiles_of(const AttendParams& p, int2 span) {
  const int items = (span.y * p.c.group + kTile * NM - 1) / (kTile * NM);
  long long sum = 0;  // (a long prompt of many heads has more than 2^31)
  for (int mt = 0; mt < items; ++mt) sum += (keys_of<NM>(p, span.x, span.y, mt) + kTile - 1) / kTile;
  return sum;
}

// Four neighbouring elements as fp32, in one access where the address allows
// it (`wide`).
__device__ __forceinline__ void load4(const float* p, bool wide, float (&x)[4]) {
  if (wide) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = p[i];
  }
}
__device__ __forceinline__ float2 unpack_bf16(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, bool wide, float (&x)[4]) {
  if (wide) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    const float2 a = unpack_bf16(v.x), b = unpack_bf16(v.y);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __bfloat162float(p[i]);
  }
}
__device__ __forceinline__ void store4(float* p, bool wide, const float (&x)[4]) {
  if (wide) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = x[i];
  }
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, bool wide, const float (&x)[4]) {
  if (wide) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __float2bfloat16_rn(x[i]);
  }
}

// Cosine and sine of pair i at a position. The product of a position and a
// fraction of a turn in units of 2^-64, modulo 2^64, is the angle's fraction
// of a turn: the product is reduced exactly at any position. (The table holds a
// frequency to 53 bits, so that the angle is off by up to 2^-52 of position times
// frequency: 5e-7 turns at position 2^31 and a turn a position.) Its top 32 bits, as a signed fraction f of half turns in [-1,
// 1), go to sincospi: the rounding to fp32 keeps 24 bits of f.
__device__ __forceinline__ float2 turn_of(const Rope& r, const int32_t* positions, int i) {
  const unsigned long long t = static_cast<unsigned long long>(static_cast<long long>(positions[SJD_KV_IDX(r.status, r.axis[i], r.axes)])) * r.turns[i];
  const float f = static_cast<float>(static_cast<int32_t>(t >> 32)) * 4.656612873077393e-10f;  // 2^-31
  float sn, cs;
  sincospif(f, &sn, &cs);
  return make_float2(cs, r.inverse ? -sn : sn);
}

// Where the two quads of a vector's 8-element chunk lie, and the pair its
// rotation starts at (-1: it is not turned).
struct Chunk {
  int e0, e1, pair;
};
__device__ __forceinline__ Chunk chunk_at(int c, int pairs, int interleaved) {
  if (4 * c >= pairs) return {8 * c, 8 * c + 4, -1};
  if (interleaved) return {8 * c, 8 * c + 4, 4 * c};
  return {4 * c, pairs + 4 * c, 4 * c};
}

// Turns the four pairs of a chunk.
__device__ __forceinline__ void turn_chunk(float (&a)[4], float (&b)[4], const float2* cs, int interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float u = a[2 * i], w = b[2 * i];
      a[2 * i] = u * cs[i].x - a[2 * i + 1] * cs[i].y;
      a[2 * i + 1] = u * cs[i].y + a[2 * i + 1] * cs[i].x;
      b[2 * i] = w * cs[2 + i].x - b[2 * i + 1] * cs[2 + i].y;
      b[2 * i + 1] = w * cs[2 + i].y + b[2 * i + 1] * cs[2 + i].x;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = a[i];
      a[i] = u * cs[i].x - b[i] * cs[i].y;
      b[i] = u * cs[i].y + b[i] * cs[i].x;
    }
  }
}

// Pairs of fp32.
struct Pair {
  unsigned long long v;
};
__device__ __forceinline__ Pair pair(float x, float y) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(x), "f"(y));
  return p;
}
__device__ __forceinline__ float2 halves(Pair p) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p.v));
  return f;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return d;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}

template <int KV>
struct Codes;  // one element of a cache of type KV
template <>
struct Codes<SJD_BF16> {
  using type = __nv_bfloat16;
};
template <>
struct Codes<SJD_E4M3> {
  using type = uint8_t;
  static constexpr float kMost = 448.0f;
};
template <>
struct Codes<SJD_S8> {
  using type = int8_t;
  static constexpr float kMost = 127.0f;
};

// Four codes of the quotients y, in one word.
template <int KV>
__device__ __forceinline__ uint32_t codes4(const float (&y)[4]) {
  if constexpr (KV == SJD_E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(y[0], y[1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(y[2], y[3]), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
  } else {
    // 1.5 * 2^23 + y, rounded to nearest even, ends in y's integer as a byte (|y| <= 127)
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(y[i] + 12582912.0f);
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  }
}

// The values of four codes in a word, fp32.
template <int KV>
__device__ __forceinline__ void values4(uint32_t w, float (&x)[4]) {
  if constexpr (KV == SJD_E4M3) {
    const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w), __NV_E4M3);
    const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> 16), __NV_E4M3);
    const float2 a = __half22float2(__half2(lo)), b = __half22float2(__half2(hi));
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = static_cast<float>(static_cast<int8_t>(w >> 8 * i));
  }
}

}  // namespace sjd_kv_ops
