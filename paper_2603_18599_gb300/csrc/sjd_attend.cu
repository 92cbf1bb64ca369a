// Attention of a chunk of new tokens over the paged cache, on the tensor
// cores.
//
// The query heads that share a key head are stacked: row r = t * G + g of
// (sequence, key head) is chunk token t's g-th head of the group, so that one
// token of G heads, a window of W tokens or a prompt all are rows against
// the same keys. An item is 128 NM such rows of one (sequence, key head); its
// keys come in tiles of 128:
//
//   S = Q K^T (128 x 128, fp32 in tensor memory)
//   P = 2^(c S - m)                    one thread to a row, m the running maximum
//   O = 2^(m_old - m) O + P V          (fp32 in tensor memory)
//
// All key tiles of all items, in a row, are cut into equal parts, one for each
// block of a grid of one block per SM, from the sequences' lengths on the
// device: neither their number nor how ragged they are leaves an SM idle. An
// item that a cut went through is left as unnormalised parts with their
// maxima and sums, which a second kernel joins in the order of the parts.
//
// A block has four kinds of warps. 0-3 and 4-7 take the softmax, each group a
// slot: with NM = 1 the even and the odd tiles of the same 128 rows (each with
// an accumulator of its own, joined at the end), with NM = 2 the two halves
// of 256 rows. 8-11 load keys, 12-15 the queries and values, and warp 19
// issues the products: those of one slot run while the other's softmax does.
// A slot's weights are handed over in two halves of 64 keys, the second made
// while the first is multiplied.
//
// With at most 64 or 32 rows (a short window, one token) the rows lie in the
// tile two or four times (SP), so that the warps of a slot all have work:
// each copy takes the softmax over its own half or quarter of a tile's keys,
// with a maximum and a sum of its own and weights of 0 for the other keys, and
// the copies' accumulators are joined at the end like the slots'.
//
// What bounds it (one GB300): over a 16-bit cache few rows are bound by HBM (16
// tokens of 64 heads over up to 32768 tokens, 8 key heads: 253 us, 97 % of the
// copy rate); the same over e4m3 by what the loaders do for a tile (212 us, 60 %;
// of 214 in a loop of this call alone 199 stay without products and
// exponentials). A prompt of 4000 behind 4100 takes 380 us, 1050 TFLOP/s or 54 %
// of a dense product's rate: a tile of 256 rows takes 4400 cycles where its products
// take 2048 and both slots' softmax, measured alone, 1811. A slot's softmax, its
// products and the hand-overs between them follow one another, and the two slots
// that tensor memory has room for overlap little. 32 windows of 64 over 8100 in e4m3
// take 354 us (30 %): the keys' and values' factors make that softmax 2799 cycles
// (measured alone, without the upkeep of the values' unit; more where the values'
// factors lie far apart: Unit). One token over 300: 13 to 20 us a call, which is
// the host's part.

#include <cfloat>

#include "sjd_kv_device.cuh"
#include "sjd_tcgen05.cuh"

namespace sjd_kv_ops {

namespace {

constexpr int kHalf = kTile / 2;        // keys whose weights are handed over at a time
constexpr int kAttendThreads = 20 * 32;
constexpr int kMmaWarp = 19;            // (on another scheduler than the first rows' softmax)
constexpr uint32_t kTmemColumns = 512;  // S of the two slots (P over them), then O of the two
constexpr uint32_t kOColumn = 2 * kTile;
constexpr long long kWaitClocks = 4000000000ll;  // about two seconds
constexpr float kLeast = 1e-30f;        // least factor of the scores
constexpr int kRoom = 10;               // weights of an 8-bit cache are times 2^10: at most 2^(4 + 10), in fp16
constexpr float kNear = 64.0f;          // values' factors that share a unit lie within 2^6 of each other, and of 1
constexpr float kUnits = 0x1p40f;       // within 2^40: see Unit
constexpr float kFar = 0x1p20f;         // from here on a score's product with c is rounded too coarsely (2^-4)
template <int KV>
constexpr float kRise = KV == SJD_BF16 ? 8.0f : 4.0f;  // a row's reference maximum moves when it is behind by more than 2^kRise

__host__ __device__ constexpr uint32_t tile_bytes(int dp) { return static_cast<uint32_t>(kTile) * dp * 2; }

// Shared memory: queries, rings of key and value tiles (1024-byte aligned),
// for an 8-bit cache rings of the codes as they come, then the small things.
//
// Key and value tiles, and codes under way, as fit 227 KB. At a head of 128 and
// 8 bits deeper rings of codes beat more tiles with few rows (16 tokens over 32768:
// 212 us with one tile of each and four of codes, 231 with two tiles and two);
// with 256 rows two key tiles let the next scores start (32 windows
// of 64 over 8100: 357 us; 361 with two value tiles instead, 357 with one of
// each and three of codes).
template <int KV, int DP, int NM>
struct Plan {
  static constexpr bool kCodes = KV != SJD_BF16;
  static constexpr uint32_t kQ = NM * tile_bytes(DP);
  static constexpr int kK = kCodes ? (DP == 64 ? 3 : NM == 1 ? 1 : 2) : (DP == 128 ? 3 : 5);          // key tiles
  static constexpr int kV = kCodes ? (DP == 64 ? 3 : 1) : (DP == 128 ? (NM == 1 ? 3 : 2) : 5);        // value tiles
  static constexpr int kRaw = !kCodes ? 0 : DP == 64 || NM == 1 ? 4 : 2;  // of keys, and of values
  static constexpr uint32_t kAtK = kQ, kAtV = kAtK + kK * tile_bytes(DP), kAtRawK = kAtV + kV * tile_bytes(DP),
                            kAtRawV = kAtRawK + kRaw * kTile * DP, kAtMisc = kAtRawV + kRaw * kTile * DP;
};

struct Start {
  int kvh, b, mt, k;     // the block's first item: key head, sequence, row tile, key tile
  int start, count;      // the sequence's span
  long long tile, tiles, per;  // the block's part of all key tiles; a block's fair share
};

// Weights are powers of two: 2^(c (q . k)), c = |scale| log2 e. (Not 0, so that
// a score of -inf gives a weight of 0 at any scale.)
__device__ __forceinline__ float power_factor(const AttendParams& p) { return fmaxf(fabsf(p.scale) * 1.4426950408889634f, kLeast); }
// What a sum of weights against the reference score `from` is worth against `to`.
__device__ __forceinline__ float worth(float from, float to, float c) {
  return from == -INFINITY ? 0.0f : from == to ? 1.0f : exp2_fast((from - to) * c);
}
__device__ __forceinline__ float log_of_sum(const AttendParams& p, float ref, float sum) {
  return sum > 0.0f || sum != sum ? fmaf(log2f(sum), 0.69314718055994531f, ref * fabsf(p.scale)) : -INFINITY;
}

// What a block leaves for the joining kernel: the item of which it has the
// first part, if other blocks have the rest.
struct Shared {
  int parts, kvh, b, mt;
  int done;  // of an item that its blocks join themselves: parts that are there (0 between calls)
};

// A row of the call's result (token, head); and a row of a block's part of an item.
__device__ __forceinline__ long long row_index(const AttendParams& p, long long row) {
  return SJD_KV_IDX(p.c.status, row, static_cast<long long>(p.c.B) * p.c.n * p.c.Hq);
}
template <int NM>
__device__ __forceinline__ long long part_index(const AttendParams& p, long long part, int row) {
  return SJD_KV_IDX(p.c.status, part * (kTile * NM) + row, 2ll * gridDim.x * (kTile * NM));
}

// An item's position and its keys.
struct Item {
  int kvh, b, mt;       // key head, sequence, tile of 128 NM rows
  int start, count;     // the sequence's span
  int rows;             // rows of the sequence (count * G)
  int keys;             // keys that some row of the item sees: 0 .. keys - 1
  int tiles;            // of 128 keys
};

template <int NM>
__device__ __forceinline__ void fill(const AttendParams& p, Item& it) {
  it.rows = it.count * p.c.group;
  it.keys = keys_of<NM>(p, it.start, it.count, it.mt);
  it.tiles = (it.keys + kTile - 1) / kTile;
}

// A block's way through its part: one piece (tiles k0 .. k1 - 1 of an item)
// after the other.
template <int NM>
struct Walk {
  Item it;
  long long left;     // tiles of the block's part from this piece on
  int k0, k1;
  int piece;          // number of the piece

  __device__ __forceinline__ bool begin(const AttendParams& p, const Start& s) {
    left = s.tiles;
    piece = 0;
    if (left <= 0) return false;
    it.kvh = s.kvh, it.b = s.b, it.mt = s.mt, it.start = s.start, it.count = s.count;
    fill<NM>(p, it);
    k0 = s.k;
    k1 = static_cast<int>(min(static_cast<long long>(it.tiles), k0 + left));
    return true;
  }
  __device__ __forceinline__ bool next(const AttendParams& p) {
    left -= k1 - k0;
    if (left <= 0) return false;
    ++piece;
    if (++it.mt * (kTile * NM) >= it.rows) {
      it.mt = 0;
      do {
        if (++it.b == p.c.B) {
          it.b = 0;
          if (++it.kvh == p.c.Hkv) return false;  // (the spans changed during the call)
        }
        const int2 span = span_of(p.c, it.b);
        it.start = span.x, it.count = span.y;
      } while (it.count == 0);
    }
    fill<NM>(p, it);
    k0 = 0;
    k1 = static_cast<int>(min(static_cast<long long>(it.tiles), left));
    return true;
  }
};

template <int NM>
struct Misc {
  unsigned long long k_full[5], k_empty[5], v_full[5], v_empty[5], q_full, q_empty, o_full,
      s_full[2], p_full[2][2],  // by slot (and half)
      drained;                  // after a wait that ran out: no product is in flight
  uint32_t tmem;
  int abort;
  int last;                // whether the block joins the item's parts
  int bad_values[4];       // number of the piece (modulo 4) in which a value that some rows do not see is not finite
  Start start;
  Walk<NM> walk[2];        // the softmax groups' ways
  uint32_t poison[2][4];   // per slot: keys of the tile whose factor is no number
  signed char exponents[2][NM * kTile];  // of the queries' rows (8-bit cache), by the piece's number modulo 2
  ushort2 range[2][4];     // per slot and warp: the smallest and the largest of the tile's value factors, the upper halves of their bits
  alignas(16) float row[2][2][kTile];  // per slot: factors of the tile's keys and values; at the end the rows' maxima and sums
};

template <int KV, int DP, int NM>
constexpr uint32_t shared_bytes() {
  static_assert(Plan<KV, DP, NM>::kAtMisc + sizeof(Misc<NM>) <= 227 * 1024, "shared memory");
  return Plan<KV, DP, NM>::kAtMisc + static_cast<uint32_t>(sizeof(Misc<NM>));
}

template <int NM>
__device__ __forceinline__ void wait(Misc<NM>* m, unsigned long long* bar, uint32_t parity) {
  const uint32_t at = smem_addr(bar);
  if (mbar_try(at, parity)) return;
  const long long begun = clock64();
  while (!mbar_try(at, parity)) {
    // once a wait has run out, none waits any more: the block goes on to its
    // end over results that do not count
    if (*const_cast<volatile int*>(&m->abort)) return;
    if (clock64() - begun > kWaitClocks) {
      *const_cast<volatile int*>(&m->abort) = 1;
      return;
    }
  }
}

// Where the block's part begins (warp 0).
template <int NM>
__device__ void locate(const AttendParams& p, Start* s) {
  const int lane = threadIdx.x & 31;
  const int2 none = make_int2(0, 0);
  auto span_at = [&](int b) { return b < p.c.B ? span_of(p.c, b) : none; };
  int2 span = span_at(lane);
  long long x = tiles_of<NM>(p, span), per_head = x;
  for (int b = 32 + lane; b - lane < p.c.B; b += 32) per_head += tiles_of<NM>(p, span_at(b));
  for (int o = 16; o > 0; o /= 2) per_head += __shfl_xor_sync(0xffffffffu, per_head, o);
  const long long all = per_head * p.c.Hkv, per = (all + gridDim.x - 1) / gridDim.x, from = blockIdx.x * per;
  const long long mine = max(0ll, min(per, all - from));
  if (lane == 0) s->tile = from, s->tiles = mine, s->per = per;
  if (mine == 0) return;
  const int kvh = static_cast<int>(from / per_head);
  long long rest = from - kvh * per_head;
  for (int b0 = 0; b0 < p.c.B; b0 += 32) {
    if (b0 > 0) span = span_at(b0 + lane), x = tiles_of<NM>(p, span);
    long long upto = x;
    for (int o = 1; o < 32; o *= 2) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, upto > rest);
    if (past) {
      if (lane == __ffs(past) - 1) {
        rest -= upto - x;
        int mt = 0, t;
        while (rest >= (t = (keys_of<NM>(p, span.x, span.y, mt) + kTile - 1) / kTile)) rest -= t, ++mt;
        *s = {kvh, b0 + lane, mt, static_cast<int>(rest), span.x, span.y, from, mine, per};
      }
      return;
    }
    rest -= __shfl_sync(0xffffffffu, upto, 31);
  }
}

// The first key that not every row of the item sees (mask kinds).
template <int NM>
__device__ __forceinline__ int common_keys(const AttendParams& p, const Item& it) {
  if (p.mask_kind == SJD_MASK_ALL) return it.keys;
  if (p.mask_kind == SJD_MASK_GIVEN) return it.start;
  return it.start + by_group(p.c, it.mt * (kTile * NM)) + 1;
}

// Byte offset of a 16-byte piece (8 bf16 columns) of a row in a tile.
__device__ __forceinline__ uint32_t piece_at(int row, int piece) {
  return static_cast<uint32_t>((piece >> 3) * (kTile * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
}

// The fp16 values of 8 codes, exactly.
template <int KV>
__device__ __forceinline__ uint4 eight_values(uint2 w) {
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = i < 2 ? w.x : w.y;
    if constexpr (KV == SJD_E4M3) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(i & 1 ? x >> 16 : x), __NV_E4M3);
      v[i] = *reinterpret_cast<const uint32_t*>(&h);
    } else {
      // code + 128 in the last byte of 1024 + that, less 1152
      const uint32_t u = __byte_perm(x ^ 0x80808080u, 0x64646464u, i & 1 ? 0x4342 : 0x4140), less = 0x64806480u;
      const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&u), *reinterpret_cast<const __half2*>(&less));
      v[i] = *reinterpret_cast<const uint32_t*>(&d);
    }
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// --- loading --------------------------------------------------------------------

// The page of key `key` of the item's sequence.
__device__ __forceinline__ int key_page(const Cache& c, const Item& it, int key) {
  return key < it.keys ? page_of(c, it.b, key) : kNoPage;
}

// Queries of the item: rows of 16-byte pieces, zeros beyond.
template <int DP, int NM, int SP>
__device__ __forceinline__ void load_queries(const AttendParams& p, const Item& it, uint32_t smem, int tid) {
  constexpr int kPieces = DP / 8;
  const int G = p.c.group, pieces = p.c.D / 8;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q.p) + it.b * p.q.sb + static_cast<long long>(it.kvh) * G * p.q.sh;
  const int piece = tid % kPieces;
#pragma unroll 8
  for (int row = tid / kPieces; row < kTile * NM; row += 128 / kPieces) {
    const int r = it.mt * (kTile * NM) + row % (kTile * NM / SP), t = by_group(p.c, r), g = r - t * G;
    const bool in = r < it.rows && piece < pieces;
    copy16(smem + (row / kTile) * tile_bytes(DP) + piece_at(row % kTile, piece),
           in ? q + t * p.q.st + g * p.q.sh + 8 * piece : static_cast<const __nv_bfloat16*>(p.q.p), in ? 16 : 0);
  }
  copy_commit();
  copy_wait<0>();
  if (p.scale < 0.0f) {  // the kernel's factor is |scale|
    for (int row = tid / kPieces; row < kTile * NM; row += 128 / kPieces) {
      uint4* w = reinterpret_cast<uint4*>(__cvta_shared_to_generic(smem + (row / kTile) * tile_bytes(DP) + piece_at(row % kTile, piece)));
      const uint4 v = *w;
      *w = make_uint4(v.x ^ 0x80008000u, v.y ^ 0x80008000u, v.z ^ 0x80008000u, v.w ^ 0x80008000u);
    }
  }
}

// Queries for an 8-bit cache, whose codes are fp16 in the products: a row is
// divided by the power of two of its largest magnitude (bf16's 8 bits then fit
// fp16 but for elements below 2^-15 of it), which is kept for its scores.
template <int DP, int NM, int SP>
__device__ __forceinline__ void load_half_queries(const AttendParams& p, const Item& it, uint32_t smem, int tid, signed char* exponents) {
  constexpr int kPieces = DP / 8;
  const int G = p.c.group, pieces = p.c.D / 8;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q.p) + it.b * p.q.sb + static_cast<long long>(it.kvh) * G * p.q.sh;
  const int piece = tid % kPieces;
  const uint32_t flip = p.scale < 0.0f ? 0x80000000u : 0u;  // the kernel's factor is |scale|
#pragma unroll 4
  for (int row = tid / kPieces; row < kTile * NM; row += 128 / kPieces) {
    const int r = it.mt * (kTile * NM) + row % (kTile * NM / SP), t = by_group(p.c, r), g = r - t * G;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < it.rows && piece < pieces) v = *reinterpret_cast<const uint4*>(q + t * p.q.st + g * p.q.sh + 8 * piece);
    uint32_t w[4] = {v.x, v.y, v.z, v.w}, most = 0;
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack_bf16(w[i]);
      x[2 * i] = f.x, x[2 * i + 1] = f.y;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t bits = __float_as_uint(x[2 * i + e]) & 0x7fffffffu;
        most = max(most, bits < 0x7f800000u ? bits : 0u);
      }
    }
#pragma unroll
    for (int o = kPieces / 2; o > 0; o /= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    // (-120 to 120: the factor and its inverse are normal numbers)
    const int e = most == 0 ? 0 : max(-120, min(120, static_cast<int>(most >> 23) - 127));
    const float f = __uint_as_float(static_cast<uint32_t>(127 - e) << 23 | flip);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(x[2 * i] * f, x[2 * i + 1] * f);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    shared_store16(smem + (row / kTile) * tile_bytes(DP) + piece_at(row % kTile, piece), make_uint4(w[0], w[1], w[2], w[3]));
    if (piece == 0) exponents[row] = static_cast<signed char>(e);
  }
}

// Values that are not finite, in a tile of which some rows do not see every
// key, would reach those rows as 0 * inf: they are taken out of the tile
// here and given to the rows that see them at the end (add_bad_values).
__device__ __forceinline__ bool take_out(uint32_t& w) {
  uint32_t out = 0;
  if ((w & 0x7f800000u) == 0x7f800000u) out |= 0xffff0000u;
  if ((w & 0x00007f80u) == 0x00007f80u) out |= 0x0000ffffu;
  w &= ~out;
  return out != 0;
}

// The same for four codes of e4m3 (0x7f and 0xff stand for NaN).
__device__ __forceinline__ bool take_out_codes(uint32_t& w) {
  const uint32_t out = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  w &= ~((out >> 7) * 0xffu);
  return out != 0;
}
// (a call: it is for the tiles at the end of an item alone)
__device__ __noinline__ bool take_out_of_codes(uint32_t at, int rounds, int step) {
  bool any = false;
#pragma unroll 1
  for (int i = 0; i < rounds; ++i, at += step) {
    uint2 v = shared_load8(at);
    const bool x = take_out_codes(v.x), y = take_out_codes(v.y);
    if (x || y) shared_store8(at, v), any = true;
  }
  return any;
}

// The four warps of one operand, keys (IS_V false) or values, go through the
// block's tiles. A thread has the piece tid % (DP / 8) of every 128 / (DP /
// 8)-th row; a lane finds the vector of row (warp * 32 + lane) and the others
// ask it by shuffles. The page of the next tile's row is loaded while this
// tile's copies are issued.
template <int KV, int DP, int NM, int SP, bool IS_V>
__device__ __forceinline__ void load_operand(const AttendParams& p, Misc<NM>* m, uint32_t smem) {
  using P = Plan<KV, DP, NM>;
  using Code = typename Codes<KV>::type;
  constexpr int kPieces = DP / 8, kStep = 32 / kPieces, kRounds = 32 / kStep;  // rows of a warp at a time; rounds
  constexpr int kStages = IS_V ? P::kV : P::kK;
  const int tid = threadIdx.x & 127, warp = tid / 32, lane = tid & 31, piece = lane % kPieces, first = lane / kPieces;
  const uint32_t ring = smem + (IS_V ? P::kAtV : P::kAtK);
  unsigned long long* full = IS_V ? m->v_full : m->k_full;
  unsigned long long* empty = IS_V ? m->v_empty : m->k_empty;
  const uint32_t vector_bytes = p.c.D * sizeof(Code);
  // (a thread beyond the head's elements asks for nothing, at the vector's start)
  const unsigned char* own = static_cast<const unsigned char*>(IS_V ? p.c.v : p.c.k) + (8 * piece < p.c.D ? 8 * piece * sizeof(Code) : 0);
  const uint32_t in = 8 * piece < p.c.D ? 8 * sizeof(Code) : 0;  // bytes of the thread's pieces
  auto queries = [&](int number) {
    wait(m, &m->q_empty, (number & 1) ^ 1);
  };
  auto queries_there = [&]() {
    fence_async_shared();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_addr(&m->q_full));
  };
  Walk<NM> w;
  if (!w.begin(p, m->start)) return;
  int stage = 0;              // of the tile being loaded
  uint32_t round = 1;         // parity of the empty barriers' phase before it
  int page = key_page(p.c, w.it, w.k0 * kTile + tid);
  if constexpr (KV == SJD_BF16) {
    bool more = true;
    while (more) {
      if constexpr (IS_V) {
        queries(w.piece);
        load_queries<DP, NM, SP>(p, w.it, smem, tid);
        queries_there();
      }
      const int common = IS_V ? common_keys<NM>(p, w.it) : 0, k1 = w.k1, number = w.piece;
      for (int k = w.k0; k < k1; ++k) {
        const uint32_t mine = vector_in(p.c, page, k * kTile + tid, w.it.kvh);
        if (k + 1 < k1) {
          page = key_page(p.c, w.it, (k + 1) * kTile + tid);
        } else {
          more = w.next(p);
          if (more) page = key_page(p.c, w.it, w.k0 * kTile + tid);
        }
        wait(m, &empty[stage], round);
        const uint32_t to = ring + stage * tile_bytes(DP);
        uint32_t at[kRounds];
#pragma unroll
        for (int i = 0; i < kRounds; ++i) at[i] = __shfl_sync(0xffffffffu, mine, i * kStep + first);
#pragma unroll
        for (int i = 0; i < kRounds; ++i)
          copy16(to + piece_at(warp * 32 + i * kStep + first, piece), own + static_cast<size_t>(at[i] != kNoVector ? at[i] : 0) * vector_bytes,
                 at[i] != kNoVector ? in : 0);
        if (IS_V && (k + 1) * kTile > common) {  // some row does not see every key (take_out)
          copy_commit();
          copy_wait<0>();
          bool bad = false;
#pragma unroll 1
          for (int i = 0; i < kRounds; ++i) {
            const uint32_t at = to + piece_at(warp * 32 + i * kStep + first, piece);
            uint4 v = shared_load16(at);
            const bool a = take_out(v.x), b = take_out(v.y), c = take_out(v.z), d = take_out(v.w);
            if (a || b || c || d) shared_store16(at, v), bad = true;
          }
          if (bad) m->bad_values[number & 3] = number + 1;
          mbar_arrive(smem_addr(&full[stage]));
        } else {
          copy_arrive(smem_addr(&full[stage]));
        }
        if (++stage == kStages) stage = 0, round ^= 1;
      }
    }
  } else {
    // The codes come into a ring of their own, up to kRaw tiles ahead, 16 to a
    // copy where a vector's length is a multiple of that (past the L1 cache)
    // and else 8; a warp turns its 32 rows into fp16, 8 codes to a thread. (Into bf16
    // it takes three times the instructions: 1280 of the 1395 cycles that HBM
    // leaves a tile.)
    constexpr int kWide = DP / 16, kWideStep = 32 / kWide;
    const bool wide = p.c.D % 16 == 0;
    const uint32_t raw = smem + (IS_V ? P::kAtRawV : P::kAtRawK) + warp * 32 * DP;
    const uint32_t from = raw + first * DP + 8 * piece;
    const unsigned char* data = static_cast<const unsigned char*>(IS_V ? p.c.v : p.c.k);
    Walk<NM> a = w;           // the tile to be asked for
    int ka = a.k0, slot = 0;
    bool ahead = true;
    auto ask = [&](int to) {
      if (ahead) {
        const uint32_t mine = vector_in(p.c, page, ka * kTile + tid, a.it.kvh);
        if (wide) {
          const int part = 16 * (lane % kWide), row = lane / kWide, bytes = part < p.c.D ? 16 : 0;
          uint32_t at[32 / kWideStep];
#pragma unroll
          for (int i = 0; i < 32 / kWideStep; ++i) at[i] = __shfl_sync(0xffffffffu, mine, i * kWideStep + row);
#pragma unroll
          for (int i = 0; i < 32 / kWideStep; ++i)
            copy16(raw + to * (kTile * DP) + (i * kWideStep + row) * DP + part,
                   data + static_cast<size_t>(at[i] != kNoVector ? at[i] : 0) * vector_bytes + (bytes ? part : 0), at[i] != kNoVector ? bytes : 0);
        } else {
          uint32_t at[kRounds];
#pragma unroll
          for (int i = 0; i < kRounds; ++i) at[i] = __shfl_sync(0xffffffffu, mine, i * kStep + first);
#pragma unroll
          for (int i = 0; i < kRounds; ++i)
            copy8(from + to * (kTile * DP) + i * kStep * DP, own + static_cast<size_t>(at[i] != kNoVector ? at[i] : 0) * vector_bytes,
                  at[i] != kNoVector ? in : 0);
        }
        if (++ka == a.k1) {
          ahead = a.next(p);
          ka = a.k0;
        }
        if (ahead) page = key_page(p.c, a.it, ka * kTile + tid);
      }
      copy_commit();
    };
#pragma unroll 1
    for (int i = 0; i < P::kRaw; ++i) ask(i);
    do {
      if constexpr (IS_V) {
        queries(w.piece);
        load_half_queries<DP, NM, SP>(p, w.it, smem, tid, m->exponents[w.piece & 1]);
        queries_there();
      }
      const int common = IS_V && KV == SJD_E4M3 ? common_keys<NM>(p, w.it) : 0x7fffffff;
      for (int k = w.k0; k < w.k1; ++k) {
        wait(m, &empty[stage], round);
        copy_wait<P::kRaw - 1>();
        __syncwarp();
        if (IS_V && KV == SJD_E4M3 && (k + 1) * kTile > common) {  // some row does not see every key (take_out)
          if (take_out_of_codes(from + slot * (kTile * DP), kRounds, kStep * DP)) m->bad_values[w.piece & 3] = w.piece + 1;
        }
        const uint32_t to = ring + stage * tile_bytes(DP);
        // (unrolled, the batches crowd the instruction cache: 363 us instead of 353 for 32
        // windows of 64 over 8100, 215 instead of 208 for 16 tokens over 32768)
#pragma unroll 1
        for (int i0 = 0; i0 < kRounds; i0 += 8) {
          uint2 codes[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) codes[i] = shared_load8(from + slot * (kTile * DP) + (i0 + i) * kStep * DP);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            shared_store16(to + piece_at(warp * 32 + (i0 + i) * kStep + first, piece), eight_values<KV>(codes[i]));
        }
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&full[stage]));
        if (++stage == kStages) stage = 0, round ^= 1;
        ask(slot);
        if (++slot == P::kRaw) slot = 0;
      }
    } while (w.next(p));
  }
}

// --- products -------------------------------------------------------------------

// The same for a whole warp, which stays together.
template <int NM>
__device__ __forceinline__ void wait_together(Misc<NM>* m, unsigned long long* bar, uint32_t parity) {
  const uint32_t at = smem_addr(bar);
  if (__all_sync(0xffffffffu, mbar_try(at, parity))) return;
  const long long begun = clock64();
  while (!__all_sync(0xffffffffu, mbar_try(at, parity))) {
    const bool late = clock64() - begun > kWaitClocks;
    if (__any_sync(0xffffffffu, late || *const_cast<volatile int*>(&m->abort))) {
      *const_cast<volatile int*>(&m->abort) = 1;
      return;
    }
  }
}
// A value that is the same in all lanes, in a register that the warp shares.
__device__ __forceinline__ int shared_value(int x) { return __reduce_max_sync(0xffffffffu, x); }

// One warp issues the products of both slots, the slots in turn. What it
// counts and addresses with is kept in the warp's shared registers: else a
// product costs 110 cycles to issue, and this warp is what all others wait for.
template <int KV, int DP, int NM>
__device__ __forceinline__ void issue_products(const AttendParams& p, Misc<NM>* m, uint32_t smem, uint32_t tmem_) {
  using P = Plan<KV, DP, NM>;
  constexpr uint32_t kScores = product_kind(kTile, kTile, false, KV != SJD_BF16), kValues = product_kind(kTile, DP, true, KV != SJD_BF16);
  const bool lead = elect_lane();
  const uint32_t tmem = shared_value(tmem_);
  Walk<NM> w;
  if (!w.begin(p, m->start)) return;
  uint32_t ks = 0, kp = 0, vs = 0, vp = 0;  // the rings' stages and their parities
  uint32_t pp = 0;            // bit 2 * slot + h: parity of p_full[slot][h]
  uint32_t piece = 0;
  bool more = true;
  while (more) {
    const int tiles = shared_value(w.k1 - w.k0), turns = NM * tiles;   // of a slot and a tile, the slots in turn
    const int last_halves = shared_value(w.it.keys - (w.k1 - 1) * kTile <= kHalf ? 1 : 2);  // of the piece's last tile
    more = shared_value(w.next(p));
    // S of a slot = Q K^T
    auto scores = [&](int turn) {
      const uint32_t slot = turn & 1;
      if (NM == 1 || slot == 0) {
        wait_together(m, &m->k_full[ks], kp);
        if (KV == SJD_BF16) fence_async_shared();  // (of the copies, which the barrier has made this warp see)
      }
      tc_fence_after();
      const uint64_t q = operand_k(smem + (NM == 2 ? slot * tile_bytes(DP) : 0)), k = operand_k(smem + P::kAtK + ks * tile_bytes(DP));
      const uint32_t s = tmem + slot * kTile;
      if (lead) {
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
          constexpr uint32_t kAtom = kTile * 128 / 16;
          const uint64_t at = (i / 4) * kAtom + (i % 4) * 2;
          mma_ss(s, q + at, k + at, kScores, i > 0);
        }
        mma_commit(smem_addr(&m->s_full[slot]));
        if (NM == 1 || slot == 1) mma_commit(smem_addr(&m->k_empty[ks]));
        if (turn + 1 == turns) mma_commit(smem_addr(&m->q_empty));
      }
      __syncwarp();
      if (NM == 1 || slot == 1) {
        if (++ks == P::kK) ks = 0, kp ^= 1;
      }
    };
    wait_together(m, &m->q_full, piece & 1);
    scores(0);
    if (turns > 1) scores(1);
    for (int turn = 0; turn < turns; ++turn) {
      const uint32_t slot = turn & 1;
      const int halves = turn / NM + 1 == tiles ? last_halves : 2;
      if (NM == 1 || slot == 0) {
        wait_together(m, &m->v_full[vs], vp);
        if (KV == SJD_BF16) fence_async_shared();
      }
      const uint64_t v = operand_n(smem + P::kAtV + vs * tile_bytes(DP), kTile * 128);
      const uint32_t o = tmem + kOColumn + slot * DP, from = tmem + slot * kTile;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (h >= halves) continue;
        wait_together(m, &m->p_full[slot][h], pp >> (2 * slot + h) & 1);
        pp ^= 1u << (2 * slot + h);
        tc_fence_after();
        // O of a slot += P V; P lies over S, two weights to a column
        if (lead) {
#pragma unroll
          for (int i = 0; i < kHalf / 16; ++i)
            mma_ts(o, from + h * (kHalf / 2) + i * 8, v + (h * (kHalf * 128) + i * 2048) / 16, kValues, turn >= 2 || h > 0 || i > 0);
        }
        __syncwarp();
      }
      if (lead && (NM == 1 || slot == 1)) mma_commit(smem_addr(&m->v_empty[vs]));
      __syncwarp();
      if (NM == 1 || slot == 1) {
        if (++vs == P::kV) vs = 0, vp ^= 1;
      }
      if (turn + 2 < turns) scores(turn + 2);
    }
    if (lead) mma_commit(smem_addr(&m->o_full));
    __syncwarp();
    ++piece;
  }
  // (nothing is in flight when the block ends)
  wait_together(m, &m->o_full, (piece - 1) & 1);
  if (*const_cast<volatile int*>(&m->abort)) {
    if (lead) mma_commit(smem_addr(&m->drained));
    __syncwarp();
    const long long begun = clock64();
    while (!mbar_try(smem_addr(&m->drained), 0) && clock64() - begun <= kWaitClocks) {}
  }
}

// --- softmax --------------------------------------------------------------------

template <int KV>
__device__ __forceinline__ float value_of(typename Codes<KV>::type code) {
  if constexpr (KV == SJD_E4M3) return __half2float(__half(__nv_cvt_fp8_to_halfraw(code, __NV_E4M3)));
  else return static_cast<float>(code);
}

// Values that were taken out of the tiles (take_out, take_out_codes) or whose
// factor was set aside, for the rows that see them.
template <int KV, int N>
__device__ __noinline__ void add_bad_values(const AttendParams& p, const Item& it, int begin, int end, int t, int column, float (&o)[N]) {
  for (int key = begin; key < end; ++key) {
    const bool seen = key < it.start || p.mask_kind == SJD_MASK_ALL ||
                      (p.mask_kind == SJD_MASK_CAUSAL ? key <= it.start + t : p.mask[p.mask_b * it.b + p.mask_r * t + (key - it.start)] != 0);
    const uint32_t at = seen ? vector_in(p.c, key_page(p.c, it, key), key, it.kvh) : kNoVector;
    if (at == kNoVector) continue;
    if constexpr (KV == SJD_BF16) {
      const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.c.v) + static_cast<size_t>(at) * p.c.D;
      for (int i = 0; i < N && column + i < p.c.D; ++i) {
        const float x = __bfloat162float(v[column + i]);
        if (!(fabsf(x) <= FLT_MAX)) o[i] += x;
      }
    } else {
      const float f = p.c.vs[at];
      const typename Codes<KV>::type* v = static_cast<const typename Codes<KV>::type*>(p.c.v) + static_cast<size_t>(at) * p.c.D;
      for (int i = 0; i < N && column + i < p.c.D; ++i) {
        const float x = value_of<KV>(v[column + i]);
        if (!(f < INFINITY) || x != x) o[i] += x * f;
      }
    }
  }
}

// The keys of a piece's tiles that were looked over: those with a key that some row does not see.
template <int NM>
__device__ __forceinline__ int first_looked_over(const AttendParams& p, const Item& it, int k0) {
  return max(k0, common_keys<NM>(p, it) / kTile) * kTile;
}

// Scores of keys that the row does not see become -inf; of those that it
// sees and whose factor is no number (poison), NaN.
__device__ __forceinline__ void mask_scores(uint32_t s_at, const uint32_t (&seen)[4], const uint32_t* poison) {
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    uint32_t s[32];
    tmem_load32(s_at + 32 * i, s);
    tmem_wait_load(s);
    const uint32_t bits = i == 0 ? seen[0] : i == 1 ? seen[1] : i == 2 ? seen[2] : seen[3], bad = bits & poison[i];
#pragma unroll
    for (int j = 0; j < 32; ++j) s[j] = bits >> j & 1 ? (bad >> j & 1 ? 0x7fc00000u : s[j]) : 0xff800000u;
    tmem_store32(s_at + 32 * i, s);
  }
  tmem_wait_store();
}

// 32 scores times their keys' factors (an 8-bit cache).
__device__ __forceinline__ void times_factors(uint32_t (&s)[32], const float* factors) {
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    const float4 f = *reinterpret_cast<const float4*>(factors + j);
    const float2 u = halves(mul2(pair(__uint_as_float(s[j]), __uint_as_float(s[j + 1])), pair(f.x, f.y)));
    const float2 v = halves(mul2(pair(__uint_as_float(s[j + 2]), __uint_as_float(s[j + 3])), pair(f.z, f.w)));
    s[j] = __float_as_uint(u.x), s[j + 1] = __float_as_uint(u.y), s[j + 2] = __float_as_uint(v.x), s[j + 3] = __float_as_uint(v.y);
  }
}
__device__ __forceinline__ float largest_of(const uint32_t (&s)[32], float t) {
  float top[4] = {t, t, t, t};
#pragma unroll
  for (int j = 0; j < 32; j += 8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) top[e] = max3(top[e], __uint_as_float(s[j + 2 * e]), __uint_as_float(s[j + 2 * e + 1]));
  }
  return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}
// Scores so large that rounding their product with c would change weights by
// powers of two are taken less the reference first, in tensor memory.
template <int KEYS>
__device__ __noinline__ void less_reference(uint32_t s_at, float ref, float& base) {
  const float from = ref == -INFINITY ? 0.0f : ref;
  base = 0.0f;
#pragma unroll 1
  for (int i = 0; i < KEYS / 32; ++i) {
    uint32_t s[32];
    tmem_load32(s_at + 32 * i, s);
    tmem_wait_load(s);
#pragma unroll
    for (int j = 0; j < 32; ++j) s[j] = __float_as_uint(__uint_as_float(s[j]) - from);
    tmem_store32(s_at + 32 * i, s);
  }
  tmem_wait_store();
}
// The weights of 32 scores, 2^(c s - base), packed to 16 bits, in an 8-bit
// cache times the values' factors; and their sum.
template <int KV>
__device__ __forceinline__ void weights_of(const uint32_t (&s)[32], const float* factors, float c, float base, uint32_t (&out)[16], Pair (&sum)[2]) {
  const Pair c2 = pair(c, c), less = pair(-base, -base);
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    float4 f;
    if constexpr (KV != SJD_BF16) f = *reinterpret_cast<const float4*>(factors + j);
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      const float2 d = halves(fma2(pair(__uint_as_float(s[j + e]), __uint_as_float(s[j + e + 1])), c2, less));
      const Pair w = pair(exp2_fast(d.x), exp2_fast(d.y));
      sum[e / 2] = add2(sum[e / 2], w);
      if constexpr (KV == SJD_BF16) {
        const float2 v = halves(w);
        out[(j + e) / 2] = pack_bf16(v.x, v.y);
      } else {
        const float2 v = halves(mul2(w, e ? pair(f.z, f.w) : pair(f.x, f.y)));
        const __half2 h = __floats2half2_rn(v.x, v.y);
        out[(j + e) / 2] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
  }
}

// An 8-bit cache's weights go into the product in fp16, p v / unit 2^kRoom with
// the values' factors v, and O is kept in units. As long as all keys of the tiles
// so far, whether seen or not, have factors that lie near each other, they share a
// unit, a power of two above them all: the key with a row's largest score has a
// weight of 1 at least, and so the row's largest product is 1 / kNear of the unit
// or more. Else (`wide`: a key's factor could be large, small or 0 where the
// row's weight is not) each row has a unit of its own, near the largest product
// p v among the keys that it sees. Either way the row's largest is 2^4 to 2^14
// as fp16, and a product below 2^-29 of it is lost: less than the codes of the
// largest resolve (2^-10 of its factor for e4m3, 2^-1 for s8; times codes of
// up to 448 it is 2^-20).
struct Unit {
  bool wide = false;
  float of = 0.0f;        // the unit; 0: no key yet. wide: its logarithm
  float low = FLT_MAX;    // the smallest factor so far. wide: the logarithm of the row's largest p v so far, or less
  __device__ __forceinline__ void widen(bool some) {  // some: the row has seen keys
    low = some && of > 0.0f ? log2f(low) : -INFINITY;
    of = some && of > 0.0f ? log2f(of) : 0.0f;
    wide = true;
  }
  // What O is to be times. (Apart from what its reference is worth: the product of the two may underflow.)
  __device__ __forceinline__ float back() const { return wide ? exp2_fast(of - kRoom) : of * (1.0f / (1 << kRoom)); }
};

// What is kept of a value's factor for the weights.
__device__ __forceinline__ float value_factor(float v, bool wide) { return wide ? log2f(v) : v; }
// The smallest and the largest of the factors of a warp's keys, where there is a key and
// its factor a number: the upper halves of their bits, the largest's rounded up.
__device__ __forceinline__ ushort2 range_of_factors(float v, bool there) {
  const bool counts = there && v < INFINITY;
  const uint32_t bits = v > 0.0f ? __float_as_uint(v) : 0u;
  const uint32_t least = __reduce_min_sync(0xffffffffu, counts ? bits : 0x7f7fffffu), most = __reduce_max_sync(0xffffffffu, counts ? bits : 0u);
  return make_ushort2(static_cast<unsigned short>(least >> 16), static_cast<unsigned short>((most + 0xffffu) >> 16));
}
__device__ __forceinline__ ushort2 joint(ushort2 a, ushort2 b) { return make_ushort2(min(a.x, b.x), max(a.y, b.y)); }
// Another tile's factors: makes the unit wide, or returns the old unit over the
// new one. some: the row has seen keys.
__device__ __forceinline__ float take_factors(Unit& unit, ushort2 range, bool some) {
  const float least = __uint_as_float(static_cast<uint32_t>(range.x) << 16), most = __uint_as_float(static_cast<uint32_t>(range.y) << 16);
  if (least >= unit.low && most <= unit.of) return 1.0f;
  // (the power of two from the largest on)
  const float now = fmaxf(unit.of, __uint_as_float((__float_as_uint(most) + 0x7fffffu) & 0x7f800000u)), low = fminf(unit.low, least);
  float grown = 1.0f;
  if (now <= kUnits && now >= 1.0f / kUnits && low * kNear >= now) {
    if (now != unit.of && unit.of > 0.0f) grown = unit.of / now;
    unit.of = now, unit.low = low;
  } else {
    unit.widen(some);
  }
  return grown;
}

// The steps of a row with a unit of its own (of, most: Unit), whose factors come
// as logarithms.
// The reference moves to the tile's largest score, if that is far above it; returns by how much it was behind, as a power.
__device__ __forceinline__ float wide_move(float top, float c, float& ref, float& sum, float& most) {
  float behind = 0.0f;
  if ((top - ref) * c > kRise<SJD_E4M3> || (ref == -INFINITY && top != -INFINITY)) {
    if (ref != -INFINITY) behind = (ref - top) * c, sum *= exp2_fast(behind), most += behind;
    ref = top;
  }
  return behind;
}
// 32 scores become powers of two; their largest product p v.
__device__ __forceinline__ float wide_largest(uint32_t (&s)[32], const float* logs, float from, float c, float most) {
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const float t = (__uint_as_float(s[j]) - from) * c, u = t + logs[j];
    s[j] = __float_as_uint(t);
    most = fmaxf(most, u < INFINITY ? u : most);   // (an infinite factor has no part in it)
  }
  return most;
}
// The unit moves where the largest product has left 2^-4 to 2^4 of it. (-116 to 133: O's factor,
// 2^(of - kRoom), is a normal number, and no weight overflows at scales up to the largest number.)
__device__ __forceinline__ float wide_unit(float of, float most) {
  const bool turn = most > of + 4.0f || (most < of - 4.0f && most != -INFINITY);
  return turn ? fminf(133.0f, fmaxf(-116.0f, ceilf(most))) : of;
}
// The weights of 32 such powers, packed to 16 bits, and their sum.
__device__ __forceinline__ float wide_weights_of(const uint32_t (&t)[32], const float* logs, float of, uint32_t (&out)[16]) {
  const float up = kRoom - of;
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const float a = __uint_as_float(t[j]), b = __uint_as_float(t[j + 1]);
    sum += exp2_fast(a) + exp2_fast(b);
    const __half2 h = __floats2half2_rn(exp2_fast(a + (logs[j] + up)), exp2_fast(b + (logs[j + 1] + up)));
    out[j / 2] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return sum;
}

// The weights of a tile's keys (32 `chunks` of them) that way, from the scores
// at s_at to the 16-bit weights at w_at. Returns ref, sum, of and most. Two
// exponentials a score and a pass more over the scores: 32 windows of 64 over 8100 in
// e4m3 take 488 us where every tile comes this way, 354 where none does; 16 tokens
// over 32768 (the same steps in place) 241 and 212.
template <int DP>
__device__ __noinline__ float4 wide_weights(uint32_t s_at, uint32_t w_at, uint32_t o_at, int chunks, const float* logs, float c, float top,
                                            bool some_o, float ref, float sum, float of, float most) {
  const float behind = wide_move(top, c, ref, sum, most);
  __syncwarp();
  const float from = ref == -INFINITY ? 0.0f : ref;
  uint32_t s[32];
#pragma unroll 1
  for (int i = 0; i < chunks; ++i) {
    tmem_load32(s_at + 32 * i, s);
    tmem_wait_load(s);
    most = wide_largest(s, logs + 32 * i, from, c, most);
    tmem_store32(s_at + 32 * i, s);
  }
  tmem_wait_store();
  const float now = wide_unit(of, most);
  if (some_o && __any_sync(0xffffffffu, behind != 0.0f || now != of)) {
    const float f = exp2_fast(behind + (of - now));
#pragma unroll 1
    for (int i = 0; i < DP / 32; ++i) {
      tmem_load32(o_at + 32 * i, s);
      tmem_wait_load(s);
#pragma unroll
      for (int j = 0; j < 32; ++j) s[j] = __float_as_uint(__uint_as_float(s[j]) * f);
      tmem_store32(o_at + 32 * i, s);
    }
  }
#pragma unroll 1
  for (int i = 0; i < chunks; ++i) {
    uint32_t out[16];
    tmem_load32(s_at + 32 * i, s);
    tmem_wait_load(s);
    sum += wide_weights_of(s, logs + 32 * i, now, out);
    tmem_store16(w_at + 16 * i, out);
  }
  tmem_wait_store();
  return make_float4(ref, sum, now, most);
}

template <int KV, int DP, int NM>
__device__ __forceinline__ void softmax_rows(const AttendParams& p, Misc<NM>* m, uint32_t tmem, float* parts, float2* part_rows, Shared* shared) {
  const int slot = threadIdx.x / 128, row = threadIdx.x & 127, warp_row = row & ~31;
  const uint32_t lanes = static_cast<uint32_t>(warp_row) << 16;
  const uint32_t s_at = tmem + lanes + slot * kTile, o_at = tmem + lanes + kOColumn;
  const int G = p.c.group;
  const float c = power_factor(p);
  // (the group's way is kept in shared memory: its registers are for the scores)
  Walk<NM>& w = m->walk[slot];
  const Item& it = w.it;
  if (m->start.tiles <= 0) return;
  if (row == 0) w.begin(p, m->start);
  named_barrier(2 + slot, 128);
  uint32_t sp = 0;
  for (;;) {
    const int r0 = it.mt * (kTile * NM) + (NM == 2 ? slot * kTile : 0);
    const bool valid = r0 + row < it.rows, active = r0 + warp_row < it.rows;
    const int t = by_group(p.c, r0 + row);
    const int units = NM == 2 ? w.k1 - w.k0 : (w.k1 - w.k0 + 1 - slot) / 2;  // tiles of the slot
    constexpr int stride = NM == 2 ? 1 : 2;
    const int k_first = w.k0 + (NM == 2 ? 0 : slot);
    // keys below `whole` are seen, those from `limit` on are not (a given mask tells between)
    const int limit = !valid ? 0x7fffffff : p.mask_kind == SJD_MASK_CAUSAL ? it.start + t + 1 : it.keys;
    const int whole = !valid ? 0x7fffffff : p.mask_kind == SJD_MASK_GIVEN ? it.start : limit;
    const int common = common_keys<NM>(p, it);
    float ref = -INFINITY, sum = 0.0f, c_row = c, row_unit = 1.0f;
    Unit unit;
    // an 8-bit cache's factors of key `row` of the tiles: the next tile's are on their way while
    // one is worked on, and the page of the one after that
    float next_k = 0.0f, next_v = 0.0f;
    int page = kNoPage;
    auto factors = [&](int u) {
      const int key = (k_first + u * stride) * kTile + row;
      const uint32_t at = vector_in(p.c, page, key, it.kvh);
      next_k = next_v = 0.0f;
      if (at != kNoVector) next_k = p.c.ks[at], next_v = p.c.vs[at];
      page = u + 1 < units ? key_page(p.c, it, key + stride * kTile) : kNoPage;
    };
    if (KV != SJD_BF16 && units > 0) {
      page = key_page(p.c, it, k_first * kTile + row);
      factors(0);
    }
#pragma unroll 1
    for (int u = 0; u < units; ++u) {
      const int key0 = (k_first + u * stride) * kTile;
      const bool two = it.keys - key0 > kHalf;  // halves of the tile
      float grown = 1.0f;   // the unit: old over new
      if constexpr (KV != SJD_BF16) {
        // a factor that is no number would reach rows that do not see its key (and so would an
        // infinite one of a value, times a weight of 0): it is set aside in tiles where there
        // can be such rows (the values' are given to the others at the end)
        const bool apart = key0 + kTile > common;
        const bool bad_k = apart && next_k != next_k, bad_v = apart && !(next_v < INFINITY);
        named_barrier(2 + slot, 128);  // all have used the factors of the tile before
        m->row[slot][0][row] = bad_k ? kLeast : fmaxf(next_k, next_k == next_k ? kLeast : next_k);
        m->row[slot][1][row] = value_factor(bad_v ? 0.0f : next_v, unit.wide);
        const unsigned poison = __ballot_sync(0xffffffffu, bad_k);
        if (bad_v) m->bad_values[w.piece & 3] = w.piece + 1;
        const ushort2 range = range_of_factors(next_v, key0 + row < it.keys);
        if ((threadIdx.x & 31) == 0) m->poison[slot][row / 32] = poison, m->range[slot][row / 32] = range;
        named_barrier(2 + slot, 128);
        if (u + 1 < units) factors(u + 1);
        if (!unit.wide) {
          const ushort2* of = m->range[slot];
          grown = take_factors(unit, joint(joint(of[0], of[1]), joint(of[2], of[3])), ref != -INFINITY);
          if (unit.wide) {  // (the same for the slot)
            m->row[slot][1][row] = log2f(m->row[slot][1][row]);
            named_barrier(2 + slot, 128);
          }
        }
      }
      wait(m, &m->s_full[slot], sp);
      sp ^= 1;
      tc_fence_after();
      if (active) {
        const uint32_t* poison = m->poison[slot];
        const bool mixed = !__all_sync(0xffffffffu, key0 + kTile <= whole) || (KV != SJD_BF16 && (poison[0] | poison[1] | poison[2] | poison[3]));
        if (mixed) {
          uint32_t seen[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int n = limit - (key0 + 32 * i);
            seen[i] = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
          }
          if (p.mask_kind == SJD_MASK_GIVEN && valid) {
            const uint8_t* mask = p.mask + p.mask_b * it.b + p.mask_r * t - it.start;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int a = max(key0 + 32 * i, it.start), e = min(key0 + 32 * i + 32, it.keys);
#pragma unroll 8
              for (int key = a; key < e; ++key)
                if (!mask[key]) seen[i] &= ~(1u << (key - key0 - 32 * i));
            }
          }
          __syncwarp();
          mask_scores(s_at, seen, poison);
        }
        // The row's scores, 32 at a time (times their keys' factors in an 8-bit
        // cache): first the largest, then the weights.
        const float* fk = m->row[slot][0];
        const float* fv = m->row[slot][1];
        float top = -INFINITY;
        if (KV != SJD_BF16 && u == 0) {
          row_unit = __uint_as_float(static_cast<uint32_t>(127 + m->exponents[w.piece & 1][(NM == 2 ? slot * kTile : 0) + row]) << 23);
          c_row = fminf(fmaxf(c * row_unit, 1e-37f), FLT_MAX);
        }
        uint32_t s[2][32];
        tmem_load32(s_at, s[0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i < 2 || two) {
            tmem_wait_load(s[i & 1]);
            if (i < 3) tmem_load32(s_at + 32 * (i + 1), s[(i + 1) & 1]);
            if (KV != SJD_BF16) {
              times_factors(s[i & 1], fk + 32 * i);
              tmem_store32(s_at + 32 * i, s[i & 1]);
            }
            top = largest_of(s[i & 1], top);
          }
        }
        if (!two) tmem_wait_load(s[0]);
        if (KV != SJD_BF16) tmem_wait_store();
        if (KV != SJD_BF16 && unit.wide) {
          __syncwarp();
          const float4 r = wide_weights<DP>(s_at, s_at, o_at + slot * DP, two ? 4 : 2, fv, c_row, top, u > 0, ref, sum, unit.of, unit.low);
          ref = r.x, sum = r.y, unit.of = r.z, unit.low = r.w;
          tc_fence_before();
          __syncwarp();
          if ((threadIdx.x & 31) == 0) {
            mbar_arrive(smem_addr(&m->p_full[slot][0]));
            if (two) mbar_arrive(smem_addr(&m->p_full[slot][1]));
          }
        } else {
          // The reference that the weights are taken against moves only where a
          // weight could pass 2^kRise: their relative precision is the same below
          // that, and O is left alone.
          const bool move = (top - ref) * c_row > kRise<KV> || (ref == -INFINITY && top != -INFINITY);
          if (__any_sync(0xffffffffu, move || grown != 1.0f)) {
            float f = !move ? 1.0f : worth(ref, top, c_row);
            if (move) ref = top, sum *= f;
            f *= grown;
            __syncwarp();
            if (u > 0) {
#pragma unroll 1
              for (int i = 0; i < DP / 32; ++i) {
                tmem_load32(o_at + slot * DP + 32 * i, s[0]);
                tmem_wait_load(s[0]);
#pragma unroll
                for (int j = 0; j < 32; ++j) s[0][j] = __float_as_uint(__uint_as_float(s[0][j]) * f);
                tmem_store32(o_at + slot * DP + 32 * i, s[0]);
              }
            }
          }
          // (the unit's exponent, less the room, goes into the powers of two)
          const int shift = KV == SJD_BF16 ? 0 : static_cast<int>(__float_as_uint(unit.of) >> 23) - 127 - kRoom;
          float base = ref == -INFINITY ? 0.0f : ref * c_row;
          if (__any_sync(0xffffffffu, fabsf(base) > kFar)) less_reference<kTile>(s_at, ref, base);
          base += static_cast<float>(shift);
          Pair total[2] = {pair(0.0f, 0.0f), pair(0.0f, 0.0f)};
          tmem_load32(s_at, s[0]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (i < 2 || two) {
              uint32_t out[16];
              tmem_wait_load(s[i & 1]);
              if (i < 3) tmem_load32(s_at + 32 * (i + 1), s[(i + 1) & 1]);
              weights_of<KV>(s[i & 1], fv + 32 * i, c_row, base, out, total);
              tmem_store16(s_at + 16 * i, out);
            }
            if (i & 1) {
              tmem_wait_store();
              tc_fence_before();
              __syncwarp();
              if ((threadIdx.x & 31) == 0 && (i == 1 || two)) mbar_arrive(smem_addr(&m->p_full[slot][i / 2]));
            }
          }
          if (!two) tmem_wait_load(s[0]);
          const float2 ends = halves(add2(total[0], total[1]));
          sum += (ends.x + ends.y) * (KV == SJD_BF16 ? 1.0f : __uint_as_float(static_cast<uint32_t>(127 + shift) << 23));
        }
      } else if ((threadIdx.x & 31) == 0) {
        mbar_arrive(smem_addr(&m->p_full[slot][0]));
        if (two) mbar_arrive(smem_addr(&m->p_full[slot][1]));
      }
      __syncwarp();
    }
    // the end of the piece: O of both slots is complete
    wait(m, &m->o_full, w.piece & 1);
    tc_fence_after();
    float f[2] = {1.0f, 1.0f}, back[2] = {1.0f, 1.0f};
    const int tiles = w.k1 - w.k0;
    const bool take[2] = {NM == 1 || slot == 0, NM == 1 ? tiles > 1 : slot == 1};
    if constexpr (NM == 1) {
      named_barrier(2 + slot, 128);  // (the factors are done with)
      m->row[slot][0][row] = ref * row_unit;
      m->row[slot][1][row] = sum;
      named_barrier(1, 256);
      const float r1 = tiles > 1 ? m->row[1][0][row] : -INFINITY, r0s = m->row[0][0][row];
      const float s1 = tiles > 1 ? m->row[1][1][row] : 0.0f, s0 = m->row[0][1][row];
      ref = fmaxf(r0s, r1);
      f[0] = worth(r0s, ref, c);
      f[1] = worth(r1, ref, c);
      sum = s0 * f[0] + s1 * f[1];
      if constexpr (KV != SJD_BF16) {  // each slot knows its unit
        named_barrier(1, 256);
        m->row[slot][0][row] = unit.back();
        named_barrier(1, 256);
        back[0] = m->row[0][0][row];
        back[1] = tiles > 1 ? m->row[1][0][row] : 0.0f;
      }
    } else if (KV != SJD_BF16) {
      ref *= row_unit;
      back[0] = back[1] = unit.back();
    }
    const bool wholly = w.k0 == 0 && w.k1 == it.tiles;
    const bool bad = *const_cast<volatile int*>(&m->bad_values[w.piece & 3]) == w.piece + 1;
    // this thread's columns of its row
    constexpr int kColumns = NM == 1 ? DP / 2 : DP;
    const int column0 = NM == 1 ? slot * kColumns : 0;
    const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    const long long part = 2ll * blockIdx.x + (w.k0 == 0 ? 1 : 0);
    const long long token = static_cast<long long>(it.b) * p.c.n + t;
    const int g = r0 + row - t * G;
    const long long head = token * p.c.Hq + static_cast<long long>(it.kvh) * G + g;
    if (active) {
#pragma unroll 1
      for (int i = 0; i < kColumns / 32; ++i) {
        const int column = column0 + 32 * i;
        __syncwarp();
        float o[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) o[j] = 0.0f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (!take[e]) continue;
          uint32_t x[32];
          tmem_load32(o_at + e * DP + column, x);
          tmem_wait_load(x);
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float v = __uint_as_float(x[j]);
            o[j] = KV != SJD_BF16 ? fmaf(NM == 1 ? v * f[e] : v, back[e], o[j]) : NM == 1 ? fmaf(v, f[e], o[j]) : v;
          }
        }
        if (bad && valid) {
          float with[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) with[j] = o[j];
          add_bad_values<KV>(p, it, first_looked_over<NM>(p, it, w.k0), min(it.keys, w.k1 * kTile), t, column, with);
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = with[j];
        }
        if (valid && wholly) {
          __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.o) + row_index(p, head) * p.c.D + column;
#pragma unroll
          for (int j = 0; j < 32; j += 8)
            if (column + j < p.c.D)
              *reinterpret_cast<uint4*>(to + j) =
                  make_uint4(pack_bf16(o[j] * inverse, o[j + 1] * inverse), pack_bf16(o[j + 2] * inverse, o[j + 3] * inverse),
                             pack_bf16(o[j + 4] * inverse, o[j + 5] * inverse), pack_bf16(o[j + 6] * inverse, o[j + 7] * inverse));
        } else if (valid) {
          float* to = parts + part_index<NM>(p, part, (NM == 2 ? slot * kTile : 0) + row) * DP + column;
#pragma unroll
          for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
        }
      }
      if (valid && (NM == 2 || slot == 0)) {
        if (wholly) {
          if (p.lse) p.lse[row_index(p, head)] = log_of_sum(p, ref, sum);
        } else {
          part_rows[part_index<NM>(p, part, (NM == 2 ? slot * kTile : 0) + row)] = make_float2(ref, sum);
        }
      }
    }
    if (threadIdx.x == 0 && w.k0 == 0 && w.k1 < it.tiles) {
      // the rest of the item lies in the blocks after this one
      const long long beyond = m->start.tile + m->start.tiles - w.left + it.tiles - 1;
      shared[blockIdx.x] = {static_cast<int>(beyond / m->start.per - blockIdx.x + 1), it.kvh, it.b, it.mt, 0};
    }
    const bool last = w.left <= tiles;
    if (NM == 1) {  // both groups have read both accumulators and the rows' sums
      tc_fence_before();
      named_barrier(1, 256);
    } else {
      named_barrier(2 + slot, 128);
    }
    if (last) return;
    if (row == 0) w.next(p);
    named_barrier(2 + slot, 128);
  }
}

// The rows beyond each sequence's span: the block's sequences, a warp (of
// `step`) to a row.
__device__ __forceinline__ void clear_rows(const AttendParams& p, int row0, int step, int lane) {
  for (int b = blockIdx.x; b < p.c.B; b += gridDim.x) {
    const int2 span = span_of(p.c, b);
    const long long begin = (static_cast<long long>(b) * p.c.n + span.y) * p.c.Hq, end = (b + 1ll) * p.c.n * p.c.Hq;
    for (long long row = begin + row0; row < end; row += step) {
      for (int i = lane; i < p.c.D / 8; i += 32)
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.o) + row_index(p, row) * p.c.D + 8 * i) = make_uint4(0, 0, 0, 0);
      if (p.lse && lane == 0) p.lse[row_index(p, row)] = -INFINITY;
    }
  }
}

// The softmax of at most 128 / SP rows, SP = 2 or 4 copies of them in the tile
// (NM = 1). A warp has the 128 / SP keys of its copy.
template <int KV, int DP, int SP>
__device__ __forceinline__ void softmax_copies(const AttendParams& p, Misc<1>* m, unsigned char* queries, uint32_t tmem, float* parts, float2* part_rows,
                                               Shared* shared, bool join_here) {
  constexpr int kRows = kTile / SP, kKeys = kTile / SP, kChunks = kKeys / 32, kWarps = 4 / SP;  // of a copy
  const int slot = threadIdx.x / 128, at = threadIdx.x & 127, lane = threadIdx.x & 31, copy = at / kRows, row = at % kRows;
  const uint32_t lanes = static_cast<uint32_t>(at & ~31) << 16;
  const uint32_t s_at = tmem + lanes + slot * kTile, o_at = tmem + lanes + kOColumn + slot * DP;
  const int G = p.c.group;
  const float c = power_factor(p);
  auto copy_barrier = [&]() {  // the copy's warps
    if constexpr (kWarps == 1) __syncwarp();
    else named_barrier(4 + slot * SP + copy, 32 * kWarps);
  };
  Walk<1>& w = m->walk[slot];
  const Item& it = w.it;
  if (m->start.tiles <= 0) return;
  if (at == 0) w.begin(p, m->start);
  named_barrier(2 + slot, 128);
  uint32_t sp = 0;
  for (;;) {
    const bool valid = row < it.rows, active = (at & ~31) % kRows < it.rows;
    const int t = by_group(p.c, row);
    const int units = (w.k1 - w.k0 + 1 - slot) / 2, k_first = w.k0 + slot;
    const int limit = !valid ? 0x7fffffff : p.mask_kind == SJD_MASK_CAUSAL ? it.start + t + 1 : it.keys;
    const int whole = !valid ? 0x7fffffff : p.mask_kind == SJD_MASK_GIVEN ? it.start : limit;
    const int common = common_keys<1>(p, it);
    float ref = -INFINITY, sum = 0.0f, c_row = c, row_unit = 1.0f;
    Unit unit;
    // the factors of key `at` of a tile, as in softmax_rows
    float next_k = 0.0f, next_v = 0.0f;
    int page = kNoPage;
    auto factors = [&](int u) {
      const int key = (k_first + 2 * u) * kTile + at;
      const uint32_t v = vector_in(p.c, page, key, it.kvh);
      next_k = next_v = 0.0f;
      if (v != kNoVector) next_k = p.c.ks[v], next_v = p.c.vs[v];
      page = u + 1 < units ? key_page(p.c, it, key + 2 * kTile) : kNoPage;
    };
    if (KV != SJD_BF16 && units > 0) {
      page = key_page(p.c, it, k_first * kTile + at);
      factors(0);
    }
#pragma unroll 1
    for (int u = 0; u < units; ++u) {
      const int tile_key = (k_first + 2 * u) * kTile, key0 = tile_key + copy * kKeys;
      const bool two = it.keys - tile_key > kHalf;
      float grown = 1.0f;
      if constexpr (KV != SJD_BF16) {
        const bool apart = tile_key + kTile > common;
        const bool bad_k = apart && next_k != next_k, bad_v = apart && !(next_v < INFINITY);
        copy_barrier();  // all have used the factors of the tile before
        m->row[slot][0][at] = bad_k ? kLeast : fmaxf(next_k, next_k == next_k ? kLeast : next_k);
        m->row[slot][1][at] = value_factor(bad_v ? 0.0f : next_v, unit.wide);
        const unsigned poison = __ballot_sync(0xffffffffu, bad_k);
        if (bad_v) m->bad_values[w.piece & 3] = w.piece + 1;
        const ushort2 range = range_of_factors(next_v, tile_key + at < it.keys);
        if (lane == 0) m->poison[slot][at / 32] = poison, m->range[slot][at / 32] = range;
        copy_barrier();
        if (u + 1 < units) factors(u + 1);
        if (!unit.wide) {
          const ushort2* of = m->range[slot] + copy * kChunks;
          grown = take_factors(unit, SP == 4 ? of[0] : joint(of[0], of[1]), ref != -INFINITY);
          if (unit.wide) {  // (the same for the copy)
            m->row[slot][1][at] = log2f(m->row[slot][1][at]);
            copy_barrier();
          }
        }
      }
      wait(m, &m->s_full[slot], sp);
      sp ^= 1;
      tc_fence_after();
      if (active) {
        const uint32_t* poison = m->poison[slot] + copy * kChunks;
        uint32_t bad = 0;
        if (KV != SJD_BF16) bad = SP == 4 ? poison[0] : poison[0] | poison[1];
        const bool mixed = !__all_sync(0xffffffffu, key0 + kKeys <= whole) || bad;
        float top = -INFINITY;
        if (KV != SJD_BF16 && u == 0) {
          row_unit = __uint_as_float(static_cast<uint32_t>(127 + m->exponents[w.piece & 1][at]) << 23);
          c_row = fminf(fmaxf(c * row_unit, 1e-37f), FLT_MAX);
        }
        const float* fk = m->row[slot][0] + copy * kKeys;
        const float* fv = m->row[slot][1] + copy * kKeys;
        // (64 scores do not stay in registers: they are read again for their weights)
        uint32_t s[32];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          tmem_load32(s_at + copy * kKeys + 32 * i, s);
          tmem_wait_load(s);
          if (mixed) {
            const int n = limit - (key0 + 32 * i);
            uint32_t seen = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
            if (p.mask_kind == SJD_MASK_GIVEN && valid) {
              const uint8_t* mask = p.mask + p.mask_b * it.b + p.mask_r * t - it.start;
              const int a = max(key0 + 32 * i, it.start), e = min(key0 + 32 * i + 32, it.keys);
#pragma unroll 8
              for (int key = a; key < e; ++key)
                if (!mask[key]) seen &= ~(1u << (key - key0 - 32 * i));
            }
            const uint32_t none = KV != SJD_BF16 ? seen & poison[i] : 0u;
#pragma unroll
            for (int j = 0; j < 32; ++j) s[j] = seen >> j & 1 ? (none >> j & 1 ? 0x7fc00000u : s[j]) : 0xff800000u;
            __syncwarp();
          }
          if (KV != SJD_BF16) times_factors(s, fk + 32 * i);
          if (kChunks > 1 && (KV != SJD_BF16 || mixed)) tmem_store32(s_at + copy * kKeys + 32 * i, s);
          top = largest_of(s, top);
        }
        if (kChunks > 1) tmem_wait_store();
        // (wide_weights' steps in place: with a call the other tiles lose registers too, 16 tokens
        // over 32768 252 us instead of 209; 32 chunks of 64 rows over 8100 211 instead of 203)
        const bool wide = KV != SJD_BF16 && unit.wide;
        float f = 1.0f;
        bool turn;
        if (wide) {
          const float behind = wide_move(top, c_row, ref, sum, unit.low);
          __syncwarp();
          const float from = ref == -INFINITY ? 0.0f : ref;
#pragma unroll 1
          for (int i = 0; i < kChunks; ++i) {
            if (kChunks > 1) {
              tmem_load32(s_at + copy * kKeys + 32 * i, s);
              tmem_wait_load(s);
            }
            unit.low = wide_largest(s, fv + 32 * i, from, c_row, unit.low);
            if (kChunks > 1) tmem_store32(s_at + copy * kKeys + 32 * i, s);
          }
          if (kChunks > 1) tmem_wait_store();
          const float now = wide_unit(unit.of, unit.low);
          f = exp2_fast(behind + (unit.of - now));
          turn = behind != 0.0f || now != unit.of;
          unit.of = now;
        } else {
          const bool move = (top - ref) * c_row > kRise<KV> || (ref == -INFINITY && top != -INFINITY);
          turn = move || grown != 1.0f;
          if (move) f = worth(ref, top, c_row), ref = top, sum *= f;
          f *= grown;
        }
        __syncwarp();
        if (u > 0 && __any_sync(0xffffffffu, turn)) {
#pragma unroll 1
          for (int i = 0; i < DP / 16; ++i) {
            uint32_t o[16];
            tmem_load16(o_at + 16 * i, o);
            tmem_wait_load(o);
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
            tmem_store16(o_at + 16 * i, o);
          }
        }
        if (wide) {
#pragma unroll 1
          for (int i = 0; i < kChunks; ++i) {
            if (kChunks > 1) {
              tmem_load32(s_at + copy * kKeys + 32 * i, s);
              tmem_wait_load(s);
            }
            uint32_t out[16];
            sum += wide_weights_of(s, fv + 32 * i, unit.of, out);
            tmem_store16(s_at + 16 * (copy * kChunks + i), out);
          }
        } else {
          uint32_t out[kChunks][16];
          const int shift = KV == SJD_BF16 ? 0 : static_cast<int>(__float_as_uint(unit.of) >> 23) - 127 - kRoom;
          float base = ref == -INFINITY ? 0.0f : ref * c_row;
          if (__any_sync(0xffffffffu, fabsf(base) > kFar)) {
            if constexpr (kChunks == 1) {
              const float from = ref == -INFINITY ? 0.0f : ref;
              base = 0.0f;
#pragma unroll
              for (int j = 0; j < 32; ++j) s[j] = __float_as_uint(__uint_as_float(s[j]) - from);
            } else {
              less_reference<kKeys>(s_at + copy * kKeys, ref, base);
            }
          }
          base += static_cast<float>(shift);
          Pair total[2] = {pair(0.0f, 0.0f), pair(0.0f, 0.0f)};
#pragma unroll
          for (int i = 0; i < kChunks; ++i) {
            if (kChunks > 1) {
              tmem_load32(s_at + copy * kKeys + 32 * i, s);
              tmem_wait_load(s);
            }
            weights_of<KV>(s, fv + 32 * i, c_row, base, out[i], total);
          }
          const float2 ends = halves(add2(total[0], total[1]));
          sum += (ends.x + ends.y) * (KV == SJD_BF16 ? 1.0f : __uint_as_float(static_cast<uint32_t>(127 + shift) << 23));
#pragma unroll
          for (int i = 0; i < kChunks; ++i) tmem_store16(s_at + 16 * (copy * kChunks + i), out[i]);
        }
        // (the row's weights of the other copies' keys are 0)
        uint32_t none[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) none[j] = 0;
#pragma unroll
        for (int i = kChunks; i < 4; ++i) tmem_store16(s_at + 16 * ((copy * kChunks + i) % 4), none);
        tmem_wait_store();
        tc_fence_before();
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(smem_addr(&m->p_full[slot][0]));
        if (two) mbar_arrive(smem_addr(&m->p_full[slot][1]));
      }
    }
    // The end of the piece: the 2 SP accumulators of a row are added up by way
    // of the queries' shared memory, a quarter of the columns at a time.
    wait(m, &m->o_full, w.piece & 1);
    tc_fence_after();
    const int tiles = w.k1 - w.k0;
    copy_barrier();  // (the factors are done with)
    ref *= row_unit;
    m->row[slot][0][at] = units > 0 && active ? ref : -INFINITY;
    m->row[slot][1][at] = units > 0 && active ? sum : 0.0f;
    named_barrier(1, 256);
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2 * SP; ++i) most = fmaxf(most, m->row[i & 1][0][i / 2 * kRows + row]);
    const float own = units > 0 && active ? worth(ref, most, c) : 0.0f, back = KV == SJD_BF16 ? 1.0f : unit.back();
    const bool wholly = w.k0 == 0 && w.k1 == it.tiles;
    const bool bad = *const_cast<volatile int*>(&m->bad_values[w.piece & 3]) == w.piece + 1;
    const long long part = 2ll * blockIdx.x + (w.k0 == 0 ? 1 : 0);
    constexpr int kColumns = DP / 4, kFours = kColumns / 4;
    float4* sums = reinterpret_cast<float4*>(queries);
#pragma unroll 1
    for (int round = 0; round < 4; ++round) {
      const int column = round * kColumns;
      float4* mine = sums + (slot * kTile + at) * kFours;
      if (active) {
#pragma unroll
        for (int i = 0; i < kColumns / 16; ++i) {
          uint32_t o[16];
          if (units > 0) {
            tmem_load16(o_at + column + 16 * i, o);
            tmem_wait_load(o);
          }
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            // (a copy without weights has nothing, whatever its accumulator holds)
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (units > 0 && ref != -INFINITY)
              v = make_float4(__uint_as_float(o[j]) * own * back, __uint_as_float(o[j + 1]) * own * back, __uint_as_float(o[j + 2]) * own * back, __uint_as_float(o[j + 3]) * own * back);
            mine[(4 * i + j / 4) ^ (lane & (kFours - 1))] = v;
          }
        }
      }
      named_barrier(1, 256);
      for (int i = threadIdx.x; i < kRows * kFours; i += 256) {
        const int r = i / kFours, four = i % kFours, col = column + 4 * four;
        if (r >= it.rows) break;
        float top = -INFINITY, all = 0.0f;
#pragma unroll
        for (int k = 0; k < 2 * SP; ++k) top = fmaxf(top, m->row[k & 1][0][k / 2 * kRows + r]);
        float o[4] = {};
#pragma unroll
        for (int k = 0; k < 2 * SP; ++k) {
          const int from = k / 2 * kRows + r;
          const float its = m->row[k & 1][0][from];
          all += m->row[k & 1][1][from] * worth(its, top, c);
          const float4 v = sums[((k & 1) * kTile + from) * kFours + (four ^ (from & (kFours - 1)))];
          o[0] += v.x, o[1] += v.y, o[2] += v.z, o[3] += v.w;
        }
        const int its_t = by_group(p.c, r), g = r - its_t * G;
        const int keys_end = min(it.keys, w.k1 * kTile);
        if (KV == SJD_BF16 && all == all) {
          // An infinity that all rows see is in the tile, and the copies that have other keys
          // made 0 * inf of it: where that left a NaN, the values that are not finite tell.
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            const float v = i == 0 ? o[0] : i == 1 ? o[1] : i == 2 ? o[2] : o[3];
            if (v == v) continue;
            float x[1] = {0.0f};
            add_bad_values<KV>(p, it, w.k0 * kTile, keys_end, its_t, col + i, x);
            if (x[0] == 0.0f) continue;
            if (i == 0) o[0] = x[0];
            else if (i == 1) o[1] = x[0];
            else if (i == 2) o[2] = x[0];
            else o[3] = x[0];
          }
        }
        if (bad) add_bad_values<KV>(p, it, first_looked_over<1>(p, it, w.k0), keys_end, its_t, col, o);
        const long long head = (static_cast<long long>(it.b) * p.c.n + its_t) * p.c.Hq + static_cast<long long>(it.kvh) * G + g;
        const bool some = all > 0.0f || all != all;
        if (wholly) {
          const float inverse = some ? 1.0f / all : 0.0f;
          if (col < p.c.D)
            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.o) + row_index(p, head) * p.c.D + col) =
                make_uint2(pack_bf16(o[0] * inverse, o[1] * inverse), pack_bf16(o[2] * inverse, o[3] * inverse));
          if (p.lse && col == 0) p.lse[row_index(p, head)] = log_of_sum(p, top, all);
        } else {
          *reinterpret_cast<float4*>(parts + part_index<1>(p, part, r) * DP + col) = make_float4(o[0], o[1], o[2], o[3]);
          if (col == 0) part_rows[part_index<1>(p, part, r)] = make_float2(top, all);
        }
      }
      named_barrier(1, 256);
    }
    tc_fence_before();
    if (!wholly) {
      const long long begin = m->start.tile + m->start.tiles - w.left - w.k0, end = begin + it.tiles - 1, per = m->start.per;
      const int first = static_cast<int>(SJD_KV_IDX(p.c.status, begin / per, gridDim.x)), count = static_cast<int>(end / per) - first + 1;
      if (!join_here) {
        if (threadIdx.x == 0 && w.k0 == 0) shared[blockIdx.x] = {count, it.kvh, it.b, it.mt, 0};
      } else {
        // the block whose part is the last to be there joins them all, in their order
        __threadfence();
        named_barrier(1, 256);
        if (threadIdx.x == 0) {
          m->last = atomicAdd(&shared[first].done, 1) == count - 1;
          if (m->last) shared[first].done = 0;
          __threadfence();
        }
        named_barrier(1, 256);
        if (m->last) {
          // every part's factor, and each row's sum in the place after them
          float* factor = reinterpret_cast<float*>(queries);
          auto part_at = [&](int k, int r) { return part_index<1>(p, 2ll * (first + k) + (k == 0 ? 1 : 0), r); };
          const int rows = it.rows;
          for (int r = threadIdx.x / 32; r < rows; r += 8) {
            const float2 rs = lane < count ? __ldcg(&part_rows[part_at(lane, r)]) : make_float2(-INFINITY, 0.0f);
            float top = rs.x;
            for (int k = 16; k > 0; k /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
            const float f = worth(rs.x, top, c);
            float all = rs.y * f;
            for (int k = 16; k > 0; k /= 2) all += __shfl_xor_sync(0xffffffffu, all, k);
            const bool some = all > 0.0f || all != all;
            factor[32 * r + lane] = f * (some ? 1.0f / all : 0.0f);
            if (p.lse && lane == 0) {
              const int its_t = by_group(p.c, r);
              const long long head = (static_cast<long long>(it.b) * p.c.n + its_t) * p.c.Hq + static_cast<long long>(it.kvh) * G + r - its_t * G;
              p.lse[row_index(p, head)] = log_of_sum(p, top, all);
            }
          }
          named_barrier(1, 256);
          constexpr int kAcross = DP / 4;
          for (int i = threadIdx.x; i < rows * kAcross; i += 256) {
            const int r = i / kAcross, col = i % kAcross * 4;
            float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
            for (int k = 0; k < count; ++k) {
              const float f = factor[32 * r + k];
              const float4 v = __ldcg(reinterpret_cast<const float4*>(parts + part_at(k, r) * DP + col));
              o.x = fmaf(v.x, f, o.x), o.y = fmaf(v.y, f, o.y), o.z = fmaf(v.z, f, o.z), o.w = fmaf(v.w, f, o.w);
            }
            const int its_t = by_group(p.c, r);
            const long long head = (static_cast<long long>(it.b) * p.c.n + its_t) * p.c.Hq + static_cast<long long>(it.kvh) * G + r - its_t * G;
            if (col < p.c.D)
              *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.o) + row_index(p, head) * p.c.D + col) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
          }
          named_barrier(1, 256);  // (the queries' memory is used no more)
        }
      }
    }
    if (threadIdx.x == 0) mbar_arrive(smem_addr(&m->q_empty));  // the queries' memory is free again
    const bool last = w.left <= tiles;
    named_barrier(2 + slot, 128);
    if (last) return;
    if (at == 0) w.next(p);
    named_barrier(2 + slot, 128);
  }
}

template <int KV, int DP, int NM, int SP>
__global__ void __launch_bounds__(kAttendThreads, 1) attend_kernel(const AttendParams p, float* parts, float2* part_rows, Shared* shared, bool join_here) {
  extern __shared__ __align__(1024) unsigned char raw[];
  using P = Plan<KV, DP, NM>;
  Misc<NM>* m = reinterpret_cast<Misc<NM>*>(raw + P::kAtMisc);
  const uint32_t smem = smem_addr(raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0);  // (the same for all lanes, to the compiler too)
  if (warp == kMmaWarp) tmem_alloc(smem_addr(&m->tmem), kTmemColumns);
  if (threadIdx.x == 256) {
    for (int i = 0; i < 5; ++i) {
      // (16-bit tiles are there when every thread's copies are, 8-bit ones when the warps have turned them into fp16)
      const int loaders = KV == SJD_BF16 ? 128 : 4;
      mbar_init(smem_addr(&m->k_full[i]), loaders), mbar_init(smem_addr(&m->k_empty[i]), 1);
      mbar_init(smem_addr(&m->v_full[i]), loaders), mbar_init(smem_addr(&m->v_empty[i]), 1);
    }
    mbar_init(smem_addr(&m->q_full), 4), mbar_init(smem_addr(&m->q_empty), SP > 1 ? 2 : 1), mbar_init(smem_addr(&m->o_full), 1);
    mbar_init(smem_addr(&m->drained), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&m->s_full[i]), 1), mbar_init(smem_addr(&m->p_full[i][0]), 4), mbar_init(smem_addr(&m->p_full[i][1]), 4);
    }
    m->abort = 0;
    for (int i = 0; i < 4; ++i) m->bad_values[i] = m->poison[0][i] = m->poison[1][i] = 0;
    fence_barrier_init();
  }
  wait_for_previous();
  let_next_start();
  if (warp == 0) locate<NM>(p, &m->start);
  if (threadIdx.x == 256) shared[blockIdx.x].parts = 0;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = m->tmem;
  if (warp < 8) {
    if constexpr (SP > 1) softmax_copies<KV, DP, SP>(p, m, raw, tmem, parts, part_rows, shared, join_here);
    else softmax_rows<KV, DP, NM>(p, m, tmem, parts, part_rows, shared);
  } else if (warp < 12) {
    load_operand<KV, DP, NM, SP, false>(p, m, smem);
  } else if (warp < 16) {
    load_operand<KV, DP, NM, SP, true>(p, m, smem);
  } else if (warp == kMmaWarp) {
    issue_products<KV, DP, NM>(p, m, smem, tmem);
  } else if (SP > 1 && join_here) {
    clear_rows(p, warp - 16, kMmaWarp - 16, threadIdx.x & 31);
  }
  copy_wait_all();  // (also where a wait ran out)
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_free(tmem, kTmemColumns);
  }
  if (threadIdx.x == 0 && m->abort) atomicOr(p.c.status, status_bit(SJD_ERR_TIMEOUT));
}

// Joins the parts of the item that block x began and others went on with; and
// clears the rows beyond each sequence's span. A warp takes a row.
constexpr int kJoinWarps = 8;

template <int DP>
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const AttendParams p, const float* parts, const float2* part_rows,
                                                               const Shared* shared, int rows_per_item) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, G = p.c.group;
  wait_for_previous();
  let_next_start();
  const float c = power_factor(p);
  const Shared s = shared[blockIdx.x];
  const int row0 = blockIdx.y * kJoinWarps + warp, step = gridDim.y * kJoinWarps;
  if (s.parts > 1) {
    const int2 span = span_of(p.c, s.b);
    for (int row = row0; row < rows_per_item; row += step) {
      const int r = s.mt * rows_per_item + row;
      if (r >= span.y * G) break;
      auto part_at = [&](int i) {
        return static_cast<long long>(SJD_KV_IDX(p.c.status, (2ll * (blockIdx.x + i) + (i == 0 ? 1 : 0)) * rows_per_item + row, 2ll * gridDim.x * rows_per_item));
      };
      float top = -INFINITY;
      for (int i = lane; i < s.parts; i += 32) top = fmaxf(top, part_rows[part_at(i)].x);
      for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      float sum = 0.0f, o[DP / 32] = {};
#pragma unroll 4
      for (int i = 0; i < s.parts; ++i) {
        const float2 rs = part_rows[part_at(i)];
        const float f = worth(rs.x, top, c);
        sum += rs.y * f;
        const float* x = parts + part_at(i) * DP + lane * (DP / 32);
        if constexpr (DP == 128) {
          const float4 v = *reinterpret_cast<const float4*>(x);
          o[0] = fmaf(v.x, f, o[0]), o[1] = fmaf(v.y, f, o[1]), o[2] = fmaf(v.z, f, o[2]), o[3] = fmaf(v.w, f, o[3]);
        } else {
          const float2 v = *reinterpret_cast<const float2*>(x);
          o[0] = fmaf(v.x, f, o[0]), o[1] = fmaf(v.y, f, o[1]);
        }
      }
      const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
      const int t = by_group(p.c, r), g = r - t * G;
      const long long head = (static_cast<long long>(s.b) * p.c.n + t) * p.c.Hq + static_cast<long long>(s.kvh) * G + g;
      __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.o) + row_index(p, head) * p.c.D + lane * (DP / 32);
      if (lane * (DP / 32) < p.c.D) {
#pragma unroll
        for (int j = 0; j < DP / 32; j += 2) *reinterpret_cast<uint32_t*>(to + j) = pack_bf16(o[j] * inverse, o[j + 1] * inverse);
      }
      if (p.lse && lane == 0) p.lse[row_index(p, head)] = log_of_sum(p, top, sum);
    }
  }
  clear_rows(p, row0, step, lane);
}

template <int KV, int DP, int NM, int SP>
cudaError_t launch(const AttendParams& p, int sms, unsigned char* scratch, cudaStream_t s) {
  const int blocks = sms < kMaxAttendBlocks ? sms : kMaxAttendBlocks;
  const size_t rows = static_cast<size_t>(kTile) * NM * 2 * blocks;
  Shared* shared = reinterpret_cast<Shared*>(scratch);
  float2* part_rows = reinterpret_cast<float2*>(scratch + kMaxAttendBlocks * sizeof(Shared));
  float* parts = reinterpret_cast<float*>(part_rows + rows);
  // At most 32 rows, of which at most 22 blocks have a part (an item is at most
  // one of kv_heads equal shares of the tiles): the last of them to be done joins
  // them, which saves a launch (one token of two sequences of 300:
  // 13.0 us a call against 14.6; 64 rows of nine parts take longer that way, 28.7
  // against 18.5).
  const bool join_here = SP == 4 && p.c.Hkv >= 8;
  static_assert(kMaxAttendBlocks / 8 + 2 <= 32, "a lane to a part");
  const cudaError_t e =
      launch_early(attend_kernel<KV, DP, NM, SP>, blocks, kAttendThreads, shared_bytes<KV, DP, NM>(), s, p, parts, part_rows, shared, join_here);
  if (e != cudaSuccess || join_here) return e;
  return launch_early(join_kernel<DP>, dim3(blocks, 8), 32 * kJoinWarps, 0, s, p, parts, part_rows, shared, kTile * NM);
}

// 256 rows to an item share each tile that is loaded between two products;
// fewer leave the tile's other rows idle, or to copies. 32 sequences over 8100, 8 key heads
// of 128, by the rows of an item (bf16 / e4m3): 32 138 / 141 us, 64
// 144 / 200, 128 146 / 204, 256 214 / 355; 132 rows, in an item of 256, 189 / 292.
template <int KV, int DP>
cudaError_t launch_of(const AttendParams& p, int sms, unsigned char* scratch, cudaStream_t s) {
  const long long rows = static_cast<long long>(p.c.n) * p.c.group;
  if (rows <= kTile / 4) return launch<KV, DP, 1, 4>(p, sms, scratch, s);
  if (rows <= kTile / 2) return launch<KV, DP, 1, 2>(p, sms, scratch, s);
  if (rows <= kTile) return launch<KV, DP, 1, 1>(p, sms, scratch, s);
  return launch<KV, DP, 2, 1>(p, sms, scratch, s);
}

template <int KV, int DP, int NM, int SP>
cudaError_t raise_limit() {
  return cudaFuncSetAttribute(attend_kernel<KV, DP, NM, SP>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared_bytes<KV, DP, NM>());
}
template <int KV, int DP>
cudaError_t raise_limits() {
  cudaError_t e = raise_limit<KV, DP, 1, 4>();
  if (e == cudaSuccess) e = raise_limit<KV, DP, 1, 2>();
  if (e == cudaSuccess) e = raise_limit<KV, DP, 1, 1>();
  return e == cudaSuccess ? raise_limit<KV, DP, 2, 1>() : e;
}

}  // namespace

cudaError_t prepare_attend(int kv_dtype, int head_dim) {
  const bool small = head_dim <= 64;
  if (kv_dtype == SJD_BF16) return small ? raise_limits<SJD_BF16, 64>() : raise_limits<SJD_BF16, 128>();
  if (kv_dtype == SJD_E4M3) return small ? raise_limits<SJD_E4M3, 64>() : raise_limits<SJD_E4M3, 128>();
  return small ? raise_limits<SJD_S8, 64>() : raise_limits<SJD_S8, 128>();
}

size_t attend_counter_bytes() { return kMaxAttendBlocks * sizeof(Shared); }

size_t attend_scratch_bytes(int head_dim, long long rows) {
  const size_t per = (rows > kTile ? 2 : 1) * static_cast<size_t>(kTile), dp = head_dim <= 64 ? 64 : 128;
  return kMaxAttendBlocks * (sizeof(Shared) + 2 * per * (sizeof(float2) + dp * sizeof(float)));
}

cudaError_t launch_attend(const AttendParams& p, int kv_dtype, int sms, unsigned char* scratch, cudaStream_t s) {
  const bool small = p.c.D <= 64;
  if (kv_dtype == SJD_BF16) return small ? launch_of<SJD_BF16, 64>(p, sms, scratch, s) : launch_of<SJD_BF16, 128>(p, sms, scratch, s);
  if (kv_dtype == SJD_E4M3) return small ? launch_of<SJD_E4M3, 64>(p, sms, scratch, s) : launch_of<SJD_E4M3, 128>(p, sms, scratch, s);
  return small ? launch_of<SJD_S8, 64>(p, sms, scratch, s) : launch_of<SJD_S8, 128>(p, sms, scratch, s);
}

}  // namespace sjd_kv_ops
