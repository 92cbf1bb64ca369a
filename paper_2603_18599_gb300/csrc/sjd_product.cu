// Matrix products of 8-bit integers with scales per token and per channel:
// y[t][n] = sx[t] sw[n] sum_k x[t][k] w[n][k] + bias[n] + residual[t][n], the
// sum exact.
//
// sm_103a's tensor cores have no rate to speak of for 8-bit integers; fp16 holds
// them exactly, and so do its fp32 accumulators as long as every partial sum
// stays within 2^24. By Cauchy and Schwarz a sum over any part of the features is
// at most |x[t]| |w[n]|, the roots of the sums of squares, which the packing and
// the spreading of the codes leave behind: where their product is at most 2^24 (weights
// and activations of a bell shape, up to about 14000 features) a tile is summed
// up in one go, else in parts of 1024 features, 2^14 * 2^10 at most, that are
// added up as integers.
//
// The weight stays in 8 bits on its way: two blocks (a cluster) take 256 channels
// x up to 256 tokens together. Each copies its 128 channels' codes, tile by tile,
// into shared memory; eight warps turn them into fp16 in tensor memory, from
// where the product takes them as its A; the tokens' codes, spread to fp16 by a
// small kernel before, are its B, half of them in each block. So the weight is read
// once in bytes, which bounds calls of few tokens, and its conversion, four
// instructions for four codes, goes on beside the products, which bound those of many. Up to
// 192 tokens have two accumulators: a tile's results are given while the next one is summed
// up (8100 tokens x 16384 channels of 4096: 551 to 560 us in short runs, 1.97 PFLOP/s, and 614 to 629 in a long
// loop under the power cap, 1.75: a library product of bf16 reaches 1.90 and 1.71; 844 with one
// accumulator of 256 tokens). 128 tokens x 65536 channels, f32: 62 us, 300 MB; a copy of the kernel without
// conversion and products took 58 where this one took 64.

#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "sjd_dense.h"
#include "sjd_kv_device.cuh"
#include "sjd_tcgen05.cuh"

namespace sjd_dense_ops {

using namespace sjd_kv_ops;

namespace {

// 16 codes from k on, zeros behind the row's end; 16 bytes at a time where the row allows it.
__device__ __forceinline__ void load_codes(const int8_t* row, int k, int end, uint32_t (&c)[4]) {
  if (k + 16 <= end && reinterpret_cast<uintptr_t>(row + k) % 16 == 0) {
    const uint4 u = *reinterpret_cast<const uint4*>(row + k);
    c[0] = u.x, c[1] = u.y, c[2] = u.z, c[3] = u.w;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if (k + j < end) c[j / 4] |= static_cast<uint32_t>(row[k + j] & 0xff) << 8 * (j % 4);
    }
  }
}

// A block packs one channel's codes.
__global__ void __launch_bounds__(128) pack_kernel(const int8_t* w, long long stride, const float* scale, const Packed to) {
  __shared__ uint32_t words[4];
  wait_for_previous();
  let_next_start();
  const int channel = blockIdx.x, r = channel % kTileOut;
  unsigned char* tile = to.codes + static_cast<long long>(channel / kTileOut) * to.tiles_in * kTileBytes + r * kTileIn;
  uint32_t squares = 0;
#pragma unroll 2
  for (int k = threadIdx.x * 16; k < to.tiles_in * kTileIn; k += 128 * 16) {
    uint32_t c[4];
    load_codes(w + channel * stride, k, channel < to.out ? to.in : 0, c);
#pragma unroll
    for (int j = 0; j < 4; ++j) squares = __dp4a(static_cast<int>(c[j]), static_cast<int>(c[j]), static_cast<int>(squares)), c[j] ^= 0x80808080u;
    const int piece = (k % kTileIn) / 16 ^ (r / 2 % 4);
    *reinterpret_cast<uint4*>(tile + static_cast<long long>(k / kTileIn) * kTileBytes + piece * 16) = make_uint4(c[0], c[1], c[2], c[3]);
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

constexpr int kPart = 1024 / kTileIn;           // feature tiles of a part that cannot pass 2^24
constexpr int kMostTokens = 256, kTwoSums = 192; // of a tile; of one that has two accumulators
constexpr int kStageColumns = kTileIn / 2;      // a tile's features in tensor memory, two to a column
constexpr int kTmemColumns = 512;
constexpr int kMostCodes = 24, kStages = 8;     // most tiles on their way: codes, tokens and codes in fp16
constexpr uint32_t kRings = 222 * 1024;         // bytes of shared memory for them; in a call of few tokens less, which lets a block of
constexpr uint32_t kRingsBeside = 216 * 1024;   // the spreading kernel stay on the SM while this kernel's starts
constexpr int kMaxPairs = 80;
constexpr int kConvert = 4, kResults = 12;       // the first warps that convert codes, that give results: eight each
constexpr int kThreads = 640;
constexpr long long kWaitClocks = 4000000000ll; // about two seconds
constexpr uint32_t kAsleep = 100000;            // (0.1 ms: warps that wait leave the others the issue slots)

// How a call is shared out. The first `whole` tiles go round the pairs of blocks; the
// feature tiles of the others, `units`, are cut into equal runs, so that no
// pair waits for a last round, and a tile's parts are added up as integers.
struct Plan {
  int pairs, channel_tiles, token_tiles, per_tile;  // pairs of blocks; tiles of 256 channels; of tokens; feature tiles
  int tokens, codes_ring, x_ring, stages;           // tokens of a tile; tiles in shared memory, of codes in tensor memory
  int accumulators, sum_columns;                    // columns from one accumulator to the next
  int whole, shares, units;                         // shares: pairs that the rest is cut up for
  int share, longer;                                // units of a share; shares that have one more
  int block_slots, sum_slot;                        // what a block may leave: of up to two tiles that others have a part in, where tiles are
                                                    // cut up; the sum so far of a tile's parts, where there may be such
  const unsigned char* x;                           // the tokens' codes in fp16
  const uint32_t* squares;                          // of each token's codes
  int32_t* slots;
  int32_t* counters;
};

__device__ __forceinline__ int share_begin(const Plan& g, int share) { return share * g.share + min(share, g.longer); }
__device__ __forceinline__ int share_of(const Plan& g, int unit) {
  const int of_longer = g.longer * (g.share + 1);
  return unit < of_longer ? unit / (g.share + 1) : g.longer + (unit - of_longer) / g.share;
}

// What the bounds-checked build latches an index outside its array in (SJD_KV_IDX).
[[maybe_unused]] __device__ __forceinline__ uint32_t* status_of(const ProductParams& p) { return &p.w.header->status; }
// Part `slot` of what block `rank` of pair `of` may leave, and the counter of a shared tile.
__device__ __forceinline__ int32_t* slot_at(const ProductParams& p, const Plan& g, int of, int rank, int slot, long long slot_size) {
  return g.slots + SJD_KV_IDX(status_of(p), (2ll * of + rank) * g.block_slots + slot, 2ll * g.pairs * g.block_slots) * slot_size;
}
__device__ __forceinline__ int32_t* counter_at(const ProductParams& p, const Plan& g, int tile, int rank) {
  return g.counters + SJD_KV_IDX(status_of(p), 2 * (tile - g.whole) + rank, 4 * kMaxPairs);
}

// One piece of work: feature tiles k0 .. k1 - 1 of a tile.
struct Piece {
  int tile, channel, token, k0, k1;   // (channel, token: numbers of tiles)
};
struct Walk {
  int tile, at, end;
  __device__ __forceinline__ Walk(const Plan& g, int pair) : tile(pair), at(0), end(0) {
    if (pair < g.shares) at = share_begin(g, pair), end = share_begin(g, pair + 1);
  }
  __device__ __forceinline__ bool next(const Plan& g, Piece& p) {
    if (tile < g.whole) {
      p.tile = tile, p.k0 = 0, p.k1 = g.per_tile;
      tile += g.pairs;
    } else if (at < end) {
      const int t = at / g.per_tile;
      p.tile = g.whole + t;
      p.k0 = at - t * g.per_tile;
      p.k1 = min(g.per_tile, p.k0 + end - at);
      at += p.k1 - p.k0;
    } else {
      return false;
    }
    // eight tiles of tokens side by side: the pairs at work share what they read in L2
    const int band = p.tile / (8 * g.channel_tiles), in = p.tile - band * 8 * g.channel_tiles, across = min(8, g.token_tiles - 8 * band);
    p.channel = in / across;
    p.token = 8 * band + in - p.channel * across;
    return true;
  }
};

// What a piece's products and results need to know of its tokens.
struct Ready {
  alignas(16) float scale[kMostTokens];  // (0 behind the last)
  int parts;                             // its sums can pass 2^24
};

struct Misc {
  unsigned long long codes_full[kMostCodes], codes_empty[kMostCodes];  // a tile of codes is there; has been turned into fp16
  unsigned long long x_full[kStages], x_empty[kStages];                // the tokens' tile is there; has been used
  unsigned long long full[kStages], empty[kStages];                    // (block 0's) both operands of both blocks are there; A has been used
  unsigned long long sum_full[2], sum_empty[2];                        // an accumulator is done; (block 0's) has been read
  unsigned long long ready_full[2], ready_empty[2];
  unsigned long long drained;
  uint32_t tmem;
  int abort;
  int others[2], last;   // whether the others' parts are there (by the shared piece's number modulo 2), all are
  Ready ready[2];
};
constexpr uint32_t kAtRings = (sizeof(Misc) + 1023) / 1024 * 1024;

__device__ __forceinline__ void wait(Misc* m, unsigned long long* bar, uint32_t parity) {
  const uint32_t at = smem_addr(bar);
  if (mbar_try(at, parity)) return;
  const long long begun = clock64();
  while (!mbar_try_for(at, parity, kAsleep)) {
    // once a wait has run out, none waits any more: the block goes on to its
    // end over results that do not count
    if (*const_cast<volatile int*>(&m->abort)) return;
    if (clock64() - begun > kWaitClocks) {
      *const_cast<volatile int*>(&m->abort) = 1;
      return;
    }
  }
}
__device__ __forceinline__ bool aborted(Misc* m) { return *const_cast<volatile int*>(&m->abort) != 0; }

// The next stage of a ring, and the parity of its barriers' phase.
struct Ring {
  int i = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step(int n) {
    if (++i == n) i = 0, phase ^= 1;
  }
};

// Copies of this block's tiles into a ring of `n` stages of `bytes` (one lane).
// What is in flight lands before the block ends.
template <typename Source>
__device__ __forceinline__ void copy_tiles(Misc* m, const Plan& g, int pair, uint32_t ring_at, int n, uint32_t bytes, unsigned long long* full,
                                           unsigned long long* empty, Source source) {
  Ring r;
  int sent = 0;
  Walk walk(g, pair);
  Piece q;
  while (walk.next(g, q)) {
    const unsigned char* from = source(q);
    for (int k = q.k0; k < q.k1; ++k) {
      wait(m, &empty[r.i], r.phase ^ 1);
      if (aborted(m)) goto done;
      mbar_expect(smem_addr(&full[r.i]), bytes);
      copy_bulk(ring_at + r.i * bytes, from + static_cast<long long>(k) * bytes, bytes, smem_addr(&full[r.i]));
      r.step(n);
      sent = min(sent + 1, n);
    }
  }
done:
  for (; sent > 0; --sent) {
    if (--r.i < 0) r.i = n - 1, r.phase ^= 1;
    const long long begun = clock64();
    while (!mbar_try(smem_addr(&full[r.i]), r.phase) && clock64() - begun <= kWaitClocks) {}
  }
}

// The tokens' scales and whether a piece's sums can pass 2^24 (a warp, a piece
// or two ahead: two round trips to memory that nothing else waits for).
__device__ __forceinline__ void prepare(const ProductParams& p, Misc* m, const Plan& g, int pair) {
  const int lane = threadIdx.x & 31;
  Ring r;
  Walk walk(g, pair);
  Piece q;
  while (walk.next(g, q)) {
    const long long t0 = static_cast<long long>(q.token) * g.tokens;
    uint32_t w[2 * kTileOut / 32], x[kMostTokens / 32];
    float scale[kMostTokens / 32];
#pragma unroll
    for (int i = 0; i < 2 * kTileOut / 32; ++i) w[i] = __ldg(p.w.squares + q.channel * (2 * kTileOut) + 32 * i + lane);
#pragma unroll
    for (int i = 0; i < kMostTokens / 32; ++i) {
      const bool is = 32 * i + lane < g.tokens && t0 + 32 * i + lane < p.rows;
      x[i] = is ? g.squares[t0 + 32 * i + lane] : 0;
      scale[i] = is ? __ldg(p.scale + t0 + 32 * i + lane) : 0.0f;
    }
#pragma unroll
    for (int i = 1; i < 2 * kTileOut / 32; ++i) w[0] = max(w[0], w[i]);
#pragma unroll
    for (int i = 1; i < kMostTokens / 32; ++i) x[0] = max(x[0], x[i]);
    const uint32_t most_w = __reduce_max_sync(0xffffffffu, w[0]), most_x = __reduce_max_sync(0xffffffffu, x[0]);
    wait(m, &m->ready_empty[r.i], r.phase ^ 1);
#pragma unroll
    for (int i = 0; i < kMostTokens / 32; ++i) m->ready[r.i].scale[32 * i + lane] = scale[i];
    if (lane == 0) m->ready[r.i].parts = q.k1 - q.k0 > kPart && static_cast<unsigned long long>(most_w) * most_x > 1ull << 48;
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_addr(&m->ready_full[r.i]));
    r.step(2);
  }
}

// Codes (c + 128) of four neighbouring features as fp16: the byte behind 0x64 is
// 1024 + 128 + c.
__device__ __forceinline__ void halves_of(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  const __half2 less = __half2half2(__ushort_as_half(0x6480));   // 1152
  const uint32_t a = __byte_perm(codes, 0x64646464u, 0x4140), b = __byte_perm(codes, 0x64646464u, 0x4342);
  const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), less), y = __hsub2(*reinterpret_cast<const __half2*>(&b), less);
  lo = *reinterpret_cast<const uint32_t*>(&x), hi = *reinterpret_cast<const uint32_t*>(&y);
}

// Warps 0 to 3 take every other tile, warps 4 to 7 those between; a lane a
// channel. A tile's fp16 is on its way into tensor memory while the next one's codes are
// loaded and converted, and is announced after that (or at once, where the next
// codes are not there yet).
__device__ __forceinline__ void convert(Misc* m, const Plan& g, int pair, int warp, uint32_t codes_at, uint32_t tmem) {
  const int lane = threadIdx.x & 31, channel = (warp & 3) * 32 + lane, turn = warp / 4;
  const uint32_t full0 = cluster_addr(smem_addr(&m->full[0]), 0), stages_at = tmem + g.accumulators * g.sum_columns + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  const uint32_t row = codes_at + channel * kTileIn, swap = (channel / 2 & 3) << 4;
  int left = 0;   // tiles of all pieces
  {
    Walk walk(g, pair);
    Piece q;
    while (walk.next(g, q)) left += q.k1 - q.k0;
  }
  left -= turn;
  if (left <= 0) return;
  Ring c, s, x;
  if (turn) c.step(g.codes_ring), s.step(g.stages), x.step(g.x_ring);
  uint4 u[4];
  auto load = [&]() {
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = shared_load16(row + c.i * kTileBytes + ((i << 4) ^ swap));
  };
  int stage = -1;   // that is to be announced
  auto announce = [&]() {
    tmem_wait_store();
    // (one warp's arrival tells of this block's tokens too)
    if ((warp & 3) == 0) wait(m, &m->x_full[x.i], x.phase);
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive_cluster(full0 + stage * 8);
    stage = -1;
    x.step(g.x_ring), x.step(g.x_ring);
  };
  wait(m, &m->codes_full[c.i], c.phase);
  load();
  for (;;) {
    uint32_t v[32];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      halves_of(u[i].x, v[8 * i], v[8 * i + 1]), halves_of(u[i].y, v[8 * i + 2], v[8 * i + 3]);
      halves_of(u[i].z, v[8 * i + 4], v[8 * i + 5]), halves_of(u[i].w, v[8 * i + 6], v[8 * i + 7]);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_addr(&m->codes_empty[c.i]));
    if (stage >= 0) announce();
    wait(m, &m->empty[s.i], s.phase ^ 1);
    tc_fence_after();
    __syncwarp();
    tmem_store32(stages_at + s.i * kStageColumns, v);
    stage = s.i;
    left -= 2;
    if (left <= 0) break;
    s.step(g.stages), s.step(g.stages);
    c.step(g.codes_ring), c.step(g.codes_ring);
    if (!__all_sync(0xffffffffu, mbar_test(smem_addr(&m->codes_full[c.i]), c.phase))) {
      announce();
      wait(m, &m->codes_full[c.i], c.phase);
    }
    load();
    __syncwarp();
  }
  announce();
}

// The products of both blocks (one warp of block 0).
__device__ __forceinline__ void issue(Misc* m, const Plan& g, int pair, uint32_t x_at, uint32_t tmem) {
  const bool lead = elect_lane();
  const uint32_t kind = product_kind(2 * kTileOut, g.tokens, false, true), x_bytes = g.tokens * kTileIn;
  const uint32_t stages_at = tmem + g.accumulators * g.sum_columns;
  Ring s, x, d, r;
  Walk walk(g, pair);
  Piece q;
  while (walk.next(g, q)) {
    wait(m, &m->ready_full[r.i], r.phase);
    const bool parts = *const_cast<volatile int*>(&m->ready[r.i].parts) != 0;
    __syncwarp();
    if (lead) mbar_arrive(smem_addr(&m->ready_empty[r.i]));
    r.step(2);
    for (int k = q.k0; k < q.k1; ++k) {
      const bool first = k == q.k0 || (parts && (k - q.k0) % kPart == 0);
      const bool end = k + 1 == q.k1 || (parts && (k + 1 - q.k0) % kPart == 0);
      if (first) wait(m, &m->sum_empty[d.i], d.phase ^ 1);
      wait(m, &m->full[s.i], s.phase);
      tc_fence_after();
      const uint32_t a = stages_at + s.i * kStageColumns, sum = tmem + d.i * g.sum_columns;
      const uint64_t b = operand_k(x_at + x.i * x_bytes);
      if (lead) {
#pragma unroll
        for (int i = 0; i < kTileIn / 16; ++i) mma_ts_pair(sum, a + i * 8, b + i * 2, kind, !first || i > 0);
        mma_commit_pair(smem_addr(&m->empty[s.i]));
        mma_commit_pair(smem_addr(&m->x_empty[x.i]));
        if (end) mma_commit_pair(smem_addr(&m->sum_full[d.i]));
      }
      __syncwarp();
      s.step(g.stages);
      x.step(g.x_ring);
      if (end) d.step(g.accumulators);
    }
  }
  if (lead) mma_commit_pair(smem_addr(&m->drained));
  __syncwarp();
}

// A result from an exact sum. (Each step is rounded by itself: it is the same
// whichever way the sum was taken. Without a bias, -0 is added, which changes nothing.)
__device__ __forceinline__ float result(float sum, float token_scale, float channel_scale, float bias) {
  return __fadd_rn(__fmul_rn(__fmul_rn(sum, token_scale), channel_scale), bias);
}

constexpr int kColumns = 16;   // of an accumulator that are read at once

// Results of a lane's channel and kColumns tokens from t0 on, of which `count` are there.
template <typename T>
__device__ __forceinline__ void finish(const ProductParams& p, int n, long long t0, int count, const float* token_scale, float scale, float bias,
                                       float (&v)[kColumns]) {
  if (count <= 0 || n >= p.w.out) return;
#pragma unroll
  for (int j = 0; j < kColumns; j += 4) {
    const float4 sx = *reinterpret_cast<const float4*>(token_scale + j);
    v[j] = result(v[j], sx.x, scale, bias), v[j + 1] = result(v[j + 1], sx.y, scale, bias);
    v[j + 2] = result(v[j + 2], sx.z, scale, bias), v[j + 3] = result(v[j + 3], sx.w, scale, bias);
  }
  if (p.residual.p) {
    // (rows behind the last one: the last one's)
    const T* r = static_cast<const T*>(p.residual.p) + t0 * p.residual.stride + n;
    T x[kColumns];
#pragma unroll
    for (int j = 0; j < kColumns; ++j) x[j] = r[min(j, count - 1) * p.residual.stride];
#pragma unroll
    for (int j = 0; j < kColumns; ++j) v[j] = __fadd_rn(v[j], static_cast<float>(x[j]));
  }
  T* y = static_cast<T*>(p.y.p) + t0 * p.y.stride + n;
#pragma unroll
  for (int j = 0; j < kColumns; ++j) {
    if (j < count) *y = static_cast<T>(v[j]);
    y += p.y.stride;
  }
}

// Adds up the parts of a shared tile, whose first unit is `begin`, that the pairs from
// `first` to before `after` left, and gives the results. A lane takes four
// neighbouring channels, a warp every eighth token.
template <typename T>
__device__ __forceinline__ void join(const ProductParams& p, const Plan& g, const float* token_scale, int begin, int first, int after, int rank, int n0,
                                     long long t0, int tokens, int warp, long long slot_size) {
  constexpr int kDeep = 4;
  const int lane = threadIdx.x & 31, n = n0 + 4 * lane;
  if (n >= p.w.out) return;
  const float4 scale = __ldg(reinterpret_cast<const float4*>(p.w.scale + n));
  float bias[4] = {-0.0f, -0.0f, -0.0f, -0.0f};
  if (p.bias) {
#pragma unroll
    for (int i = 0; i < 4; ++i) bias[i] = n + i < p.w.out ? __ldg(p.bias + n + i) : 0.0f;
  }
  for (int c0 = warp; c0 < tokens; c0 += 8 * kDeep) {
    int4 sum[kDeep];
#pragma unroll
    for (int j = 0; j < kDeep; ++j) sum[j] = make_int4(0, 0, 0, 0);
#pragma unroll 2
    for (int other = first; other < after; ++other) {
      const int slot = share_begin(g, other) >= begin ? 0 : 1;
      const int32_t* from = slot_at(p, g, other, rank, slot, slot_size) + 4 * lane;
      int4 v[kDeep];
#pragma unroll
      for (int j = 0; j < kDeep; ++j) v[j] = __ldcg(reinterpret_cast<const int4*>(from + min(c0 + 8 * j, tokens - 1) * kTileOut));
#pragma unroll
      for (int j = 0; j < kDeep; ++j) sum[j].x += v[j].x, sum[j].y += v[j].y, sum[j].z += v[j].z, sum[j].w += v[j].w;
    }
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      const int c = c0 + 8 * j;
      if (c >= tokens) continue;
      const float sx = token_scale[c];
      float v[4] = {result(__int2float_rn(sum[j].x), sx, scale.x, bias[0]), result(__int2float_rn(sum[j].y), sx, scale.y, bias[1]),
                    result(__int2float_rn(sum[j].z), sx, scale.z, bias[2]), result(__int2float_rn(sum[j].w), sx, scale.w, bias[3])};
      T* y = static_cast<T*>(p.y.p) + (t0 + c) * p.y.stride + n;
      if (p.residual.p) {
        const T* r = static_cast<const T*>(p.residual.p) + (t0 + c) * p.residual.stride + n;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (n + i < p.w.out) v[i] = __fadd_rn(v[i], static_cast<float>(r[i]));
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (n + i < p.w.out) y[i] = static_cast<T>(v[i]);
      }
    }
  }
}

__device__ __forceinline__ int count_one(int32_t* at) {
  int old;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(old) : "l"(at) : "memory");
  return old;
}
__device__ __forceinline__ int counted(const int32_t* at) {
  int now;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(now) : "l"(at) : "memory");
  return now;
}

// Eight warps read the accumulators, a lane a channel, warps 0 to 3 every other
// 16 columns, warps 4 to 7 those between.
//
// Of a shared tile's pairs of blocks the last to be done gives the results. Most
// often the others' parts are there when it comes to its own (a run of
// units begins in one tile early and ends in the next one late): then it adds them to its
// accumulator's columns on the way. Else it leaves its part too, and whichever
// pair turns out to be the last adds them all up.
template <typename T>
__device__ __forceinline__ void results(const ProductParams& p, Misc* m, const Plan& g, int pair, int rank, int warp, uint32_t tmem) {
  const int lane = threadIdx.x & 31, row = (warp & 3) * 32 + lane;
  const uint32_t empty0 = cluster_addr(smem_addr(&m->sum_empty[0]), 0), sums_at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  const long long slot_size = static_cast<long long>(g.sum_columns) * kTileOut;
  auto slot_of = [&](int of, int slot) { return slot_at(p, g, of, rank, slot, slot_size); };
  int shared = 0;
  Ring d, r;
  Walk walk(g, pair);
  Piece q;
  while (walk.next(g, q)) {
    const bool whole = q.k1 - q.k0 == g.per_tile;
    const int n0 = (q.channel * 2 + rank) * kTileOut, n = n0 + row, begin = (q.tile - g.whole) * g.per_tile;
    const long long t0 = static_cast<long long>(q.token) * g.tokens;
    const int tokens = static_cast<int>(min(static_cast<long long>(g.tokens), p.rows - t0));
    const float scale = __ldg(p.w.scale + n), bias = p.bias && n < p.w.out ? __ldg(p.bias + n) : -0.0f;
    int first = 0, after = 0;   // the pairs with a part in the tile
    if (!whole) first = share_of(g, begin), after = share_of(g, begin + g.per_tile - 1) + 1;
    bool leave = false;
    wait(m, &m->ready_full[r.i], r.phase);
    const Ready& ready = m->ready[r.i];
    const int turns = ready.parts ? (q.k1 - q.k0 + kPart - 1) / kPart : 1;
    for (int turn = 0; turn < turns; ++turn) {
      const bool last = turn + 1 == turns;
      wait(m, &m->sum_full[d.i], d.phase);
      tc_fence_after();
      __syncwarp();
      if (!whole && last) {
        if (warp == 0 && lane == 0) m->others[shared & 1] = counted(counter_at(p, g, q.tile, rank)) == after - first - 1;
        named_barrier(1, 256);
        leave = *const_cast<volatile int*>(&m->others[shared & 1]) == 0;
        ++shared;
      }
      // (the sum of the parts so far; what is left for the pair that joins the tile)
      int32_t* const sum = turns > 1 ? slot_of(pair, g.sum_slot) + row : nullptr;
      int32_t* const to = !last ? sum : leave ? slot_of(pair, share_begin(g, pair) >= begin ? 0 : 1) + row : nullptr;
      const int c0 = warp / 4 * kColumns;
      uint32_t u[kColumns];
      if (c0 < g.tokens) tmem_load16(sums_at + d.i * g.sum_columns + c0, u);
#pragma unroll 1
      for (int c = c0; c < g.tokens; c += 2 * kColumns) {
        tmem_wait_load(u);
        float f[kColumns];
#pragma unroll
        for (int j = 0; j < kColumns; ++j) f[j] = __uint_as_float(u[j]);
        __syncwarp();
        if (c + 2 * kColumns < g.tokens) tmem_load16(sums_at + d.i * g.sum_columns + c + 2 * kColumns, u);
        if (turns > 1 || !whole) {
          int v[kColumns];
#pragma unroll
          for (int j = 0; j < kColumns; ++j) v[j] = __float2int_rn(f[j]);
          if (turn > 0) {
#pragma unroll
            for (int j = 0; j < kColumns; ++j) v[j] += sum[(c + j) * kTileOut];
          }
          if (!last || leave) {
#pragma unroll
            for (int j = 0; j < kColumns; ++j) to[(c + j) * kTileOut] = v[j];
            continue;
          }
          for (int other = first; other < after; ++other) {
            if (other == pair) continue;
            const int32_t* from = slot_of(other, share_begin(g, other) >= begin ? 0 : 1) + row + c * kTileOut;
            int w[kColumns];
#pragma unroll
            for (int j = 0; j < kColumns; ++j) w[j] = __ldcg(from + j * kTileOut);
#pragma unroll
            for (int j = 0; j < kColumns; ++j) v[j] += w[j];
          }
#pragma unroll
          for (int j = 0; j < kColumns; ++j) f[j] = __int2float_rn(v[j]);
        }
        finish<T>(p, n, t0 + c, tokens - c, ready.scale + c, scale, bias, f);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(empty0 + d.i * 8);
      d.step(g.accumulators);
    }
    if (leave) {
      named_barrier(1, 256);
      if (warp == 0 && lane == 0) m->last = count_one(counter_at(p, g, q.tile, rank)) == after - first - 1;
      named_barrier(1, 256);
      if (*const_cast<volatile int*>(&m->last)) join<T>(p, g, ready.scale, begin, first, after, rank, n0, t0, tokens, warp, slot_size);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_addr(&m->ready_empty[r.i]));
    r.step(2);
  }
}

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) product_kernel(const ProductParams p, const Plan g) {
  extern __shared__ __align__(1024) unsigned char raw[];
  Misc* m = reinterpret_cast<Misc*>(raw);
  const uint32_t smem = smem_addr(raw) + kAtRings, x_at = smem + g.codes_ring * kTileBytes;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), rank = static_cast<int>(cluster_rank()), pair = blockIdx.x / 2;
  if (warp == 3) tmem_alloc_pair(smem_addr(&m->tmem), kTmemColumns);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kMostCodes; ++i) mbar_init(smem_addr(&m->codes_full[i]), 1), mbar_init(smem_addr(&m->codes_empty[i]), 4);
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_addr(&m->x_full[i]), 1), mbar_init(smem_addr(&m->x_empty[i]), 1);
      mbar_init(smem_addr(&m->full[i]), 8), mbar_init(smem_addr(&m->empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&m->sum_full[i]), 1), mbar_init(smem_addr(&m->sum_empty[i]), 16);
      mbar_init(smem_addr(&m->ready_full[i]), 1), mbar_init(smem_addr(&m->ready_empty[i]), rank == 0 ? 9 : 8);
    }
    mbar_init(smem_addr(&m->drained), 1);
    m->abort = 0;
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = m->tmem;
  // The weight's codes are read at once: the kernel before this one, which spreads
  // the tokens' codes, has let it in after all before that was done and stood in global
  // memory, from where (through L2) bulk copies read, past the first-level cache. All else waits for it.
  if (warp != 0) wait_for_previous();
  if (warp == 0) {
    if (elect_lane()) {
      copy_tiles(m, g, pair, smem, g.codes_ring, kTileBytes, m->codes_full, m->codes_empty, [&](const Piece& q) {
        return p.w.codes + static_cast<long long>(SJD_KV_IDX(status_of(p), q.channel * 2 + rank, p.w.tiles_out)) * p.w.tiles_in * kTileBytes;
      });
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t bytes = static_cast<uint32_t>(g.tokens) * kTileIn;
    if (elect_lane()) {
      copy_tiles(m, g, pair, x_at, g.x_ring, bytes, m->x_full, m->x_empty,
                 [&](const Piece& q) { return g.x + static_cast<long long>(SJD_KV_IDX(status_of(p), q.token * 2 + rank, 2ll * g.token_tiles)) * g.per_tile * bytes; });
    }
    __syncwarp();
  } else if (warp == 2) {
    if (rank == 0) issue(m, g, pair, x_at, tmem);
  } else if (warp == 3) {
    let_next_start();
    prepare(p, m, g, pair);
  } else if (warp < kResults) {
    convert(m, g, pair, warp - kConvert, smem, tmem);
  } else {
    results<T>(p, m, g, pair, rank, warp - kResults, tmem);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 2) {
    // (no product is in flight, and no arrival at the other block's barriers, when the blocks end)
    const long long begun = clock64();
    while (!mbar_try(smem_addr(&m->drained), 0) && clock64() - begun <= kWaitClocks) {}
    __syncwarp();
  }
  cluster_sync();
  if (warp == 3) {
    tc_fence_after();
    tmem_free_pair(tmem, kTmemColumns);
  }
  if (threadIdx.x == 0 && m->abort) atomicOr(&p.w.header->status, status_bit(SJD_ERR_TIMEOUT));
}

// The tokens' codes in fp16, in the order in which the product's tiles lie in
// shared memory (rows of 128 bytes, the 128-byte swizzle), the sum of each token's
// squares, and the counters of shared tiles. A block takes a token.
constexpr int kSpreadBlock = 128;   // (with at most 32 registers a thread there is room for it beside a block of the product)
__global__ void __launch_bounds__(kSpreadBlock, 16) spread_kernel(const ProductParams p, const Plan g, unsigned char* x, uint32_t* squares) {
  __shared__ uint32_t words[kSpreadBlock / 32];
  wait_for_previous();
  let_next_start();
  const int t = blockIdx.x, lane = threadIdx.x & 31, half = g.tokens / 2;
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < 4 * kMaxPairs; i += kSpreadBlock) g.counters[i] = 0;
  }
  const int8_t* from = p.codes + t * p.codes_stride;
  const int tile = static_cast<int>(SJD_KV_IDX(status_of(p), t / g.tokens, g.token_tiles)), r = t - tile * g.tokens, of_half = r / half, row = r - of_half * half;
  unsigned char* to = x + static_cast<long long>(tile * 2 + of_half) * g.per_tile * half * 128 + row * 128;
  uint32_t sum = 0;
#pragma unroll 2
  for (int k = threadIdx.x * 16; k < g.per_tile * kTileIn; k += kSpreadBlock * 16) {
    uint32_t c[4], h[8];
    load_codes(from, k, p.w.in, c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum = __dp4a(static_cast<int>(c[i]), static_cast<int>(c[i]), static_cast<int>(sum));
      halves_of(c[i] ^ 0x80808080u, h[2 * i], h[2 * i + 1]);
    }
    unsigned char* at = to + static_cast<long long>(k / kTileIn) * half * 128;
    const int piece = (k % kTileIn) / 8;
    *reinterpret_cast<uint4*>(at + ((piece ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4*>(at + (((piece + 1) ^ (row & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
  }
  sum = __reduce_add_sync(0xffffffffu, sum);
  if (lane == 0) words[threadIdx.x / 32] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kSpreadBlock / 32; ++i) sum += words[i];
    squares[t] = sum;
  }
}

// --- a few tokens ---------------------------------------------------------------
// Up to kFewTokens tokens need nothing but the weight's bytes: integer dot
// products of four codes take less time than reading them, and the one launch
// has neither fp16 nor shared tiles to wait for. A block takes 32 channels, a warp
// every eighth tile of 64 features of them (2 KB side by side), kAhead of them in its
// registers at a time; a lane reads piece l % 4 of channels l / 4, 8 + l / 4, ... and adds to
// their sums with all tokens, whose codes lie in shared memory. One
// token x 65536 channels of 4096: 41 us, 6.5 TB/s; two x 6144: 6.0 us (14.4 the other way) where the
// weight's 25 MB are in L2, 7.6 where they come from HBM, as in a step that reads each weight once.
constexpr int kFewTokens = 8, kFewWarps = 8, kFewChannels = 32;

template <typename T, int N>   // N: at least the call's tokens
__global__ void __launch_bounds__(32 * kFewWarps, 2) few_kernel(const ProductParams p) {
  constexpr int kAhead = 4, kChunk = kFewWarps * kAhead * kTileIn;
  __shared__ __align__(16) unsigned char x[N][kChunk];
  __shared__ int sums[kFewWarps][N][kFewChannels];
  wait_for_previous();
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, n0 = blockIdx.x * kFewChannels;
  const unsigned char* from = p.w.codes + static_cast<long long>(n0 / kTileOut) * p.w.tiles_in * kTileBytes + n0 % kTileOut * kTileIn + lane * 16;
  const int piece = ((lane & 3) ^ (lane / 8 & 3)) * 16;   // that the lane's codes are
  int sum[4][N] = {};
  for (int k0 = 0; k0 < p.w.in; k0 += kChunk) {
    uint4 w[kAhead][4];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int tile = min(k0 / kTileIn + a * kFewWarps + warp, p.w.tiles_in - 1);   // (behind the last: with codes of 0 for the tokens)
#pragma unroll
      for (int i = 0; i < 4; ++i) w[a][i] = __ldg(reinterpret_cast<const uint4*>(from + static_cast<long long>(tile) * kTileBytes + i * 512));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < N * (kChunk / 16); i += 32 * kFewWarps) {
      const int t = i / (kChunk / 16), k = i % (kChunk / 16) * 16;
      uint32_t c[4];
      load_codes(p.codes + (t < p.rows ? t : 0) * p.codes_stride, k0 + k, t < p.rows ? p.w.in : 0, c);
      *reinterpret_cast<uint4*>(&x[t][k]) = make_uint4(c[0], c[1], c[2], c[3]);
    }
    __syncthreads();
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[a][i].x ^= 0x80808080u, w[a][i].y ^= 0x80808080u, w[a][i].z ^= 0x80808080u, w[a][i].w ^= 0x80808080u;
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const uint4 v = *reinterpret_cast<const uint4*>(&x[t][(a * kFewWarps + warp) * kTileIn + piece]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          int s = __dp4a(static_cast<int>(w[a][i].x), static_cast<int>(v.x), sum[i][t]);
          s = __dp4a(static_cast<int>(w[a][i].y), static_cast<int>(v.y), s);
          s = __dp4a(static_cast<int>(w[a][i].z), static_cast<int>(v.z), s);
          sum[i][t] = __dp4a(static_cast<int>(w[a][i].w), static_cast<int>(v.w), s);
        }
      }
    }
  }
  // the four lanes of a channel, then the warps
#pragma unroll
  for (int t = 0; t < N; ++t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[i][t] += __shfl_xor_sync(0xffffffffu, sum[i][t], 1);
      sum[i][t] += __shfl_xor_sync(0xffffffffu, sum[i][t], 2);
      if ((lane & 3) == i) sums[warp][t][8 * i + lane / 4] = sum[i][t];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < N * kFewChannels; i += 32 * kFewWarps) {
    const int t = i / kFewChannels, c = i % kFewChannels, n = n0 + c;
    if (t >= p.rows || n >= p.w.out) continue;
    int all = 0;
#pragma unroll
    for (int k = 0; k < kFewWarps; ++k) all += sums[k][t][c];
    float y = result(__int2float_rn(all), p.scale[t], p.w.scale[n], p.bias ? p.bias[n] : -0.0f);
    if (p.residual.p) y = __fadd_rn(y, static_cast<float>(static_cast<const T*>(p.residual.p)[t * p.residual.stride + n]));
    static_cast<T*>(p.y.p)[t * p.y.stride + n] = static_cast<T>(y);
  }
}

// Whether a call goes that way: its dot products take as long as the reading from
// about six tokens on, which large weights feel. (Eight tokens x 4096 channels of
// 4096: 9.6 us, 14.3 the other way, and 12.6 with the weight from HBM; x 65536 channels 79, and 55.)
bool is_few(int rows, int out, int in) { return rows <= 4 || (rows <= kFewTokens && static_cast<long long>(out) * in <= 1ll << 26); }

template <typename T>
cudaError_t few_of(const ProductParams& p, cudaStream_t s) {
  const unsigned blocks = static_cast<unsigned>((p.w.out + kFewChannels - 1) / kFewChannels);
  constexpr int kBlock = 32 * kFewWarps;
  if (p.rows == 1) return launch_early(few_kernel<T, 1>, blocks, kBlock, 0, s, p);
  if (p.rows == 2) return launch_early(few_kernel<T, 2>, blocks, kBlock, 0, s, p);
  if (p.rows <= 4) return launch_early(few_kernel<T, 4>, blocks, kBlock, 0, s, p);
  return launch_early(few_kernel<T, 8>, blocks, kBlock, 0, s, p);
}

struct Scratch {
  size_t squares, x, slots, bytes;   // (the counters are at the beginning)
};

// How a call is shared out is chosen by the time that it is expected to take, in
// ns. A feature tile takes as long as its products and their share of the rest, 1.22 a token,
// or its conversion, 225; all tiles no less than the weight takes from memory
// (6.5 bytes) or, once for each tile of tokens, from L2 (10); a tile's results 12 a token; leaving
// parts 15 a token, joining them 15 a token and part, and 2000.
// - Tiles of tokens: the fewest, or smaller ones, whose whole tiles fill the pairs
//   (1337 tokens x 512 channels of 4096: 24 us, 27 in tiles of 192; 408 x 32 of 8192: 30, 39).
// - Whole tiles go round the pairs. Or one round and what is left over are cut into equal runs (256 tokens x
//   16384 channels of 4096, 64 tiles: 30 us whole, 42 cut up). Or, of fewer tiles than half the pairs, each
//   into as many parts as their joining is worth (32 tokens x 4096 channels of 4096, 16 tiles: 13.5 us; 15.4
//   in 76 equal runs that cross the tiles; 408 x 32 of 8192: 39 us, 87 in 25 parts each).
struct Way {
  double ns;
  int token_tiles, tokens;
  bool cut;
  int parts;   // of a tile, or 0: equal runs
};
Way way_of(int rows, const Packed& w, int pairs) {
  Way best{};
  const double weight = static_cast<double>(w.tiles_out) * w.tiles_in * kTileBytes;
  const int most = rows <= kMostTokens ? kMostTokens : kTwoSums;
  long long n = (static_cast<long long>(rows) + most - 1) / most;
  for (;;) {
    const int tokens = static_cast<int>((rows + n - 1) / n + 15) / 16 * 16;
    n = (static_cast<long long>(rows) + tokens - 1) / tokens;
    const long long tiles = n * (w.tiles_out / 2), rounds = (tiles + pairs - 1) / pairs;
    const double stage = std::fmax(1.22 * tokens, 225.0), flow = std::fmax(weight / 6500.0, n * weight / 10000.0), results = 12.0 * tokens;
    auto offer = [&](double ns, bool cut, int parts) {
      if (best.token_tiles == 0 || ns < best.ns) best = {ns, static_cast<int>(n), tokens, cut, parts};
    };
    offer(std::fmax(rounds * w.tiles_in * stage, flow) + (tokens > kTwoSums ? rounds : 1) * results, false, 0);
    if (2 * tiles <= pairs) {
      const int worth = static_cast<int>(std::lround(std::sqrt(w.tiles_in * stage / (15.0 * tokens))));
      const int parts = std::min({worth, pairs / static_cast<int>(tiles), w.tiles_in / 4});
      if (parts > 1) offer(std::fmax(w.tiles_in * stage / parts, flow) + 15.0 * (parts + 1) * tokens + 2000.0 + results, true, parts);
    } else if (tiles % pairs && w.tiles_in >= 8) {
      offer(std::fmax(tiles * w.tiles_in * stage / pairs, flow) + 30.0 * tokens + 2000.0 + results, true, 0);
    }
    if (tokens <= 16 || tiles > 4ll * pairs) return best;
    n = (static_cast<long long>(rows) + tokens - 17) / (tokens - 16);
  }
}

Plan plan_of(int rows, const Packed& w, int sms, Scratch* at) {
  Plan g{};
  g.pairs = min(sms / 2, kMaxPairs);
  g.channel_tiles = w.tiles_out / 2;
  g.per_tile = w.tiles_in;
  const Way way = way_of(rows, w, g.pairs);
  g.token_tiles = way.token_tiles;
  g.tokens = way.tokens;
  g.accumulators = g.tokens <= kTwoSums ? 2 : 1;
  g.sum_columns = (g.tokens + 31) / 32 * 32;
  g.stages = min(kStages, (kTmemColumns - g.accumulators * g.sum_columns) / kStageColumns);
  g.x_ring = kStages;
  g.codes_ring = min(kMostCodes, static_cast<int>(((rows <= 2 * g.pairs ? kRingsBeside : kRings) - g.x_ring * g.tokens * kTileIn) / kTileBytes));
  const long long tiles = static_cast<long long>(g.channel_tiles) * g.token_tiles;
  const long long rounds = way.cut ? max(0ll, tiles / g.pairs - 1) : (tiles + g.pairs - 1) / g.pairs;
  g.whole = static_cast<int>(min(tiles, rounds * g.pairs));
  g.units = static_cast<int>(tiles - g.whole) * g.per_tile;
  g.shares = way.parts ? static_cast<int>(tiles) * way.parts : min(g.pairs, max(1, g.units / 4));
  g.sum_slot = g.units ? 2 : 0;
  g.block_slots = g.sum_slot + (g.per_tile > kPart ? 1 : 0);
  g.share = g.units / g.shares;
  g.longer = g.units % g.shares;
  at->squares = 4096;
  static_assert(4 * kMaxPairs * sizeof(int32_t) <= 4096, "counters");
  at->x = at->squares + (static_cast<size_t>(rows) * sizeof(uint32_t) + 255) / 256 * 256;
  at->slots = at->x + static_cast<size_t>(g.token_tiles) * g.tokens * g.per_tile * kTileIn * sizeof(__half);
  at->bytes = at->slots + 2 * static_cast<size_t>(g.pairs) * g.block_slots * g.sum_columns * kTileOut * sizeof(int32_t);
  return g;
}

template <typename T>
cudaError_t product_of(const ProductParams& p, const Plan& g, unsigned char* x, uint32_t* squares, cudaStream_t s) {
  constexpr int kShared = kAtRings + kRings;
  static_assert(kShared <= 227 * 1024, "shared memory");
  const int shared = kAtRings + g.codes_ring * kTileBytes + g.x_ring * g.tokens * kTileIn;
  cudaError_t e = allow_shared<product_kernel<T>>(kShared);
  if (e == cudaSuccess) e = launch_early(spread_kernel, p.rows, kSpreadBlock, 0, s, p, g, x, squares);
  if (e != cudaSuccess) return e;
  return launch_early(product_kernel<T>, 2 * g.pairs, kThreads, shared, s, p, g);
}

}  // namespace

cudaError_t launch_pack(const int8_t* w, long long stride, const float* scale, const Packed& to, cudaStream_t s) {
  return launch_early(pack_kernel, static_cast<unsigned>(to.tiles_out) * kTileOut, 128, 0, s, w, stride, scale, to);
}

size_t product_scratch_bytes(int rows, int out, int in, int sms) {
  if (is_few(rows, out, in)) return 0;
  Packed w;
  packed_layout(out, in, nullptr, &w);
  Scratch at;
  plan_of(rows, w, sms, &at);
  return at.bytes;
}

cudaError_t launch_product(const ProductParams& p, int dtype, int sms, unsigned char* scratch, cudaStream_t s) {
  if (is_few(p.rows, p.w.out, p.w.in)) return dtype == SJD_BF16 ? few_of<__nv_bfloat16>(p, s) : few_of<float>(p, s);
  Scratch at;
  Plan g = plan_of(p.rows, p.w, sms, &at);
  g.counters = reinterpret_cast<int32_t*>(scratch);
  g.squares = reinterpret_cast<uint32_t*>(scratch + at.squares);
  g.x = scratch + at.x;
  g.slots = reinterpret_cast<int32_t*>(scratch + at.slots);
  if (dtype == SJD_BF16) return product_of<__nv_bfloat16>(p, g, scratch + at.x, reinterpret_cast<uint32_t*>(scratch + at.squares), s);
  return product_of<float>(p, g, scratch + at.x, reinterpret_cast<uint32_t*>(scratch + at.squares), s);
}

}  // namespace sjd_dense_ops
