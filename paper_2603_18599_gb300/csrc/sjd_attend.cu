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
// of 256 rows. 8-11 load keys, 12-15 the queries and values, one thread of
// warp 16 issues the products: those of one slot run while the other's
// softmax does.

#include <cfloat>

#include "sjd_kv_device.cuh"
#include "sjd_tcgen05.cuh"

namespace sjd_kv_ops {

namespace {

constexpr int kTile = 128;              // rows of a product, and keys of a tile
constexpr int kAttendThreads = 17 * 32;
constexpr int kMmaWarp = 16;
constexpr uint32_t kTmemColumns = 512;  // S of the two slots (P over them), then O of the two
constexpr uint32_t kOColumn = 2 * kTile;
constexpr long long kWaitClocks = 4000000000ll;  // about two seconds
constexpr float kRise = 8.0f;           // a row's reference maximum moves when it is behind by more than 2^8

__host__ __device__ constexpr uint32_t tile_bytes(int dp) { return static_cast<uint32_t>(kTile) * dp * 2; }

// Shared memory: queries, rings of key and value tiles (1024-byte aligned),
// then the small things.
template <int DP, int NM>
struct Plan {
  static constexpr uint32_t kQ = NM * tile_bytes(DP);
  static constexpr int kK = DP == 128 ? 3 : 5;                       // key tiles
  static constexpr int kV = DP == 128 ? (NM == 1 ? 3 : 2) : 5;       // value tiles
  static constexpr uint32_t kAtK = kQ, kAtV = kAtK + kK * tile_bytes(DP), kAtMisc = kAtV + kV * tile_bytes(DP);
};

struct Misc {
  unsigned long long k_full[5], k_empty[5], v_full[5], v_empty[5], q_full, q_empty, s_full[2], p_full[2], o_full;
  uint32_t tmem;
  int abort;
  int bad_values[4];       // number of the piece (modulo 4) in which a value that some rows do not see is not finite
  int first[4];            // the block's first item: key head, sequence, row tile, key tile
  long long first_tile, tiles;  // the block's part of all key tiles
  float row[2][2][kTile];  // per slot: factors of the tile's keys and values; at the end the rows' maxima and sums
};

template <int DP, int NM>
constexpr uint32_t shared_bytes() {
  return Plan<DP, NM>::kAtMisc + static_cast<uint32_t>(sizeof(Misc));
}

// What a block leaves for the joining kernel: the item of which it has the
// first part, if other blocks have the rest.
struct Shared {
  int parts, kvh, b, mt;
};

__device__ __forceinline__ void wait(Misc* m, unsigned long long* bar, uint32_t parity) {
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

// An item's position and its keys.
struct Item {
  int kvh, b, mt;       // key head, sequence, tile of 128 NM rows
  int start, count;     // the sequence's span
  int rows;             // rows of the sequence (count * G)
  int keys;             // keys that some row of the item sees: 0 .. keys - 1
  int tiles;            // of 128 keys
};

template <int NM>
__device__ __forceinline__ int keys_of(const AttendParams& p, int start, int count, int mt) {
  if (p.mask_kind != SJD_MASK_CAUSAL) return start + count;
  const int G = p.c.Hq / p.c.Hkv;
  return start + (min((mt + 1) * (kTile * NM), count * G) - 1) / G + 1;
}

// Key tiles of one key head of sequence b, all its items.
template <int NM>
__device__ int tiles_of(const AttendParams& p, int b) {
  const int2 span = span_of(p.c, b);
  const int items = (span.y * (p.c.Hq / p.c.Hkv) + kTile * NM - 1) / (kTile * NM);
  int sum = 0;
  for (int mt = 0; mt < items; ++mt) sum += (keys_of<NM>(p, span.x, span.y, mt) + kTile - 1) / kTile;
  return sum;
}

template <int NM>
__device__ __forceinline__ void fill(const AttendParams& p, Item& it) {
  it.rows = it.count * (p.c.Hq / p.c.Hkv);
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

  __device__ __forceinline__ bool begin(const AttendParams& p, const Misc* m) {
    left = m->tiles;
    if (left <= 0) return false;
    it.kvh = m->first[0], it.b = m->first[1], it.mt = m->first[2];
    const int2 span = span_of(p.c, it.b);
    it.start = span.x, it.count = span.y;
    fill<NM>(p, it);
    k0 = m->first[3];
    k1 = static_cast<int>(min(static_cast<long long>(it.tiles), k0 + left));
    piece = 0;
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

// Where the block's part begins (warp 0).
template <int NM>
__device__ void locate(const AttendParams& p, Misc* m) {
  const int lane = threadIdx.x & 31;
  long long per_head = 0;
  for (int b0 = 0; b0 < p.c.B; b0 += 32) {
    long long x = b0 + lane < p.c.B ? tiles_of<NM>(p, b0 + lane) : 0;
    for (int o = 16; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    per_head += x;
  }
  const long long all = per_head * p.c.Hkv, per = (all + gridDim.x - 1) / gridDim.x, from = blockIdx.x * per;
  const long long mine = max(0ll, min(per, all - from));
  if (lane == 0) m->first_tile = from, m->tiles = mine;
  if (mine == 0) return;
  const int kvh = static_cast<int>(from / per_head);
  long long rest = from % per_head;
  for (int b0 = 0; b0 < p.c.B; b0 += 32) {
    const long long x = b0 + lane < p.c.B ? tiles_of<NM>(p, b0 + lane) : 0;
    long long upto = x;
    for (int o = 1; o < 32; o *= 2) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, upto > rest);
    if (past) {
      const int at = __ffs(past) - 1;
      rest -= __shfl_sync(0xffffffffu, upto - x, at);
      if (lane == 0) {
        const int2 span = span_of(p.c, b0 + at);
        int mt = 0, t;
        while (rest >= (t = (keys_of<NM>(p, span.x, span.y, mt) + kTile - 1) / kTile)) rest -= t, ++mt;
        m->first[0] = kvh, m->first[1] = b0 + at, m->first[2] = mt, m->first[3] = static_cast<int>(rest);
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
  return it.start + it.mt * (kTile * NM) / (p.c.Hq / p.c.Hkv) + 1;
}

// Byte offset of a 16-byte piece (8 bf16 columns) of a row in a tile.
__device__ __forceinline__ uint32_t piece_at(int row, int piece) {
  return static_cast<uint32_t>((piece >> 3) * (kTile * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
}

// The bf16 values of 8 codes, exactly.
template <int KV>
__device__ __forceinline__ uint32_t two_values(uint32_t x) {
  // x: one code in each half word, in its upper byte (e4m3) or its lower one (s8)
  __nv_bfloat162 a, b;
  if constexpr (KV == SJD_E4M3) {
    // sign, exponent and fraction in bf16's places, the exponent 120 short
    const uint32_t v = (x & 0x80008000u) | ((x >> 4) & 0x07f007f0u), up = 0x7b807b80u;  // 2^120
    a = *reinterpret_cast<const __nv_bfloat162*>(&v);
    b = *reinterpret_cast<const __nv_bfloat162*>(&up);
    a = __hmul2(a, b);
  } else {
    // 128 + (low seven bits), less 128 or, of a negative one, 256
    const uint32_t v = (x & 0x007f007fu) | 0x43004300u, w = (x & 0x00800080u) | 0x43004300u;
    a = *reinterpret_cast<const __nv_bfloat162*>(&v);
    b = *reinterpret_cast<const __nv_bfloat162*>(&w);
    a = __hsub2(a, b);
  }
  return *reinterpret_cast<const uint32_t*>(&a);
}
template <int KV>
__device__ __forceinline__ uint4 eight_values(uint2 w) {
  constexpr uint32_t lo = KV == SJD_E4M3 ? 0x1404 : 0x4140, hi = KV == SJD_E4M3 ? 0x3424 : 0x4342;
  return make_uint4(two_values<KV>(__byte_perm(w.x, 0, lo)), two_values<KV>(__byte_perm(w.x, 0, hi)),
                    two_values<KV>(__byte_perm(w.y, 0, lo)), two_values<KV>(__byte_perm(w.y, 0, hi)));
}

// --- loading --------------------------------------------------------------------

// Slot (in vectors) of key `key` of the item's key head, -1 for none.
__device__ __forceinline__ long long vector_at(const Cache& c, const Item& it, int key) {
  if (key >= it.keys) return -1;
  const long long s = slot_of(c, it.b, key);
  return s < 0 ? -1 : s + static_cast<long long>(it.kvh) * c.ps;
}

// Queries of the item: rows of 16-byte pieces, zeros beyond.
template <int DP, int NM>
__device__ __forceinline__ void load_queries(const AttendParams& p, const Item& it, uint32_t smem, int tid) {
  constexpr int kPieces = DP / 8;
  const int G = p.c.Hq / p.c.Hkv, pieces = p.c.D / 8;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q.p) + it.b * p.q.sb + static_cast<long long>(it.kvh) * G * p.q.sh;
  const int piece = tid % kPieces;
#pragma unroll 8
  for (int row = tid / kPieces; row < kTile * NM; row += 128 / kPieces) {
    const int r = it.mt * (kTile * NM) + row, t = r / G, g = r - t * G;
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

// The four warps of one operand, keys (IS_V false) or values, go through the
// block's tiles. A thread has the piece tid % (DP / 8) of every 128 / (DP /
// 8)-th row; a lane finds the slot of row (warp * 32 + lane) of the next tile
// while this one's copies run, and the others ask it by shuffles.
template <int KV, int DP, int NM, bool IS_V>
__device__ __forceinline__ void load_operand(const AttendParams& p, Misc* m, uint32_t smem) {
  using P = Plan<DP, NM>;
  using Code = typename Codes<KV>::type;
  constexpr int kPieces = DP / 8, kStep = 32 / kPieces, kRounds = 32 / kStep;  // rows of a warp at a time; rounds
  constexpr int kStages = IS_V ? P::kV : P::kK, kLag = kStages - 1;
  const int tid = threadIdx.x & 127, warp = tid / 32, lane = tid & 31, piece = lane % kPieces;
  const uint32_t ring = smem + (IS_V ? P::kAtV : P::kAtK);
  unsigned long long* full = IS_V ? m->v_full : m->k_full;
  unsigned long long* empty = IS_V ? m->v_empty : m->k_empty;
  const Code* data = static_cast<const Code*>(IS_V ? p.c.v : p.c.k);
  const bool in = 8 * piece < p.c.D;
  Walk<NM> w;
  if (!w.begin(p, m)) return;
  int stage = 0;              // of the tile being loaded
  uint32_t round = 1;         // parity of the empty barriers' phase before it
  if constexpr (KV == SJD_BF16) {
    int owed = 0, owed_stage = 0;             // tiles whose arrival has not been told yet, and the first one's stage
    unsigned owed_mixed = 0;                  // of them, bit i: the i-th is to be looked over (take_out)
    int owed_piece = 0;
    auto tell = [&]() {
      if constexpr (IS_V) {
        if (owed_mixed & 1) {
          bool bad = false;
          for (int i = 0; i < kRounds; ++i) {
            const int row = warp * 32 + i * kStep + lane / kPieces;
            uint4* at = reinterpret_cast<uint4*>(__cvta_shared_to_generic(ring + owed_stage * tile_bytes(DP) + piece_at(row, piece)));
            uint4 v = *at;
            const bool a = take_out(v.x), b = take_out(v.y), c = take_out(v.z), d = take_out(v.w);
            if (a || b || c || d) *at = v, bad = true;
          }
          if (bad) m->bad_values[owed_piece & 3] = owed_piece + 1;
        }
        owed_mixed >>= 1;
      }
      fence_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_addr(&full[owed_stage]));
      if (++owed_stage == kStages) owed_stage = 0;
      --owed;
    };
    auto drain = [&]() {
      copy_wait<0>();
      while (owed > 0) tell();
    };
    do {
      long long mine = vector_at(p.c, w.it, w.k0 * kTile + warp * 32 + lane);
      if constexpr (IS_V) {
        drain();
        wait(m, &m->q_empty, (w.piece & 1) ^ 1);
        load_queries<DP, NM>(p, w.it, smem, tid);
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&m->q_full));
        owed_piece = w.piece;
      }
      const int common = IS_V ? common_keys<NM>(p, w.it) : 0;
      for (int k = w.k0; k < w.k1; ++k) {
        wait(m, &empty[stage], round);
        const uint32_t to = ring + stage * tile_bytes(DP);
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
          const int row = i * kStep + lane / kPieces;
          const long long at = __shfl_sync(0xffffffffu, mine, row);
          const bool here = at >= 0 && in;
          copy16(to + piece_at(warp * 32 + row, piece), here ? data + at * p.c.D + 8 * piece : data, here ? 16 : 0);
        }
        copy_commit();
        if (k + 1 < w.k1) mine = vector_at(p.c, w.it, (k + 1) * kTile + warp * 32 + lane);
        if constexpr (IS_V) {
          if ((k + 1) * kTile > common) owed_mixed |= 1u << owed;
        }
        ++owed;
        if (++stage == kStages) stage = 0, round ^= 1;
        if (owed > kLag) {
          copy_wait<kLag>();
          tell();
        }
      }
    } while (w.next(p));
    drain();
  } else {
    // 8 codes to a thread and row, two tiles in registers: one on its way while
    // the other is turned into bf16
    uint2 now[kRounds], then[kRounds];
    auto fetch = [&](uint2 (&to)[kRounds], const Item& it, int k) {
      const long long mine = vector_at(p.c, it, k * kTile + warp * 32 + lane);
#pragma unroll
      for (int i = 0; i < kRounds; ++i) {
        const long long at = __shfl_sync(0xffffffffu, mine, i * kStep + lane / kPieces);
        to[i] = at >= 0 && in ? *reinterpret_cast<const uint2*>(data + at * p.c.D + 8 * piece) : make_uint2(0, 0);
      }
    };
    fetch(now, w.it, w.k0);
    bool more = true;
    while (more) {
      if constexpr (IS_V) {
        wait(m, &m->q_empty, (w.piece & 1) ^ 1);
        load_queries<DP, NM>(p, w.it, smem, tid);
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&m->q_full));
      }
      const int k1 = w.k1;
      for (int k = w.k0; k < k1; ++k) {
        if (k + 1 < k1) {
          fetch(then, w.it, k + 1);
        } else {
          more = w.next(p);
          if (more) fetch(then, w.it, w.k0);
        }
        wait(m, &empty[stage], round);
        const uint32_t to = ring + stage * tile_bytes(DP);
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
          const int row = warp * 32 + i * kStep + lane / kPieces;
          *reinterpret_cast<uint4*>(__cvta_shared_to_generic(to + piece_at(row, piece))) = eight_values<KV>(now[i]);
          now[i] = then[i];
        }
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&full[stage]));
        if (++stage == kStages) stage = 0, round ^= 1;
      }
    }
  }
}

// --- products -------------------------------------------------------------------

template <int DP, int NM>
__device__ __forceinline__ void issue_products(const AttendParams& p, Misc* m, uint32_t smem, uint32_t tmem) {
  using P = Plan<DP, NM>;
  constexpr uint32_t kQK = product_kind(kTile, kTile, false), kPV = product_kind(kTile, DP, true);
  Walk<NM> w;
  if (!w.begin(p, m)) return;
  int ks = 0, vs = 0;
  uint32_t kp = 0, vp = 0, pp[2] = {0, 0};
  do {
    const int units = NM * (w.k1 - w.k0);  // of a slot and a tile, the slots in turn
    auto scores = [&](int u) {
      const int slot = u & 1;
      if (NM == 1 || slot == 0) wait(m, &m->k_full[ks], kp);
      tc_fence_after();
      const uint32_t q = smem + (NM == 2 ? slot * tile_bytes(DP) : 0), k = smem + P::kAtK + ks * tile_bytes(DP);
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) {
        const uint32_t at = (i / 4) * (kTile * 128) + (i % 4) * 32;
        mma_ss(tmem + slot * kTile, operand_k(q + at), operand_k(k + at), kQK, i > 0);
      }
      mma_commit(smem_addr(&m->s_full[slot]));
      if (NM == 1 || slot == 1) {
        mma_commit(smem_addr(&m->k_empty[ks]));
        if (++ks == P::kK) ks = 0, kp ^= 1;
      }
      if (u + 1 == units) mma_commit(smem_addr(&m->q_empty));
    };
    wait(m, &m->q_full, w.piece & 1);
    scores(0);
    if (units > 1) scores(1);
    for (int u = 0; u < units; ++u) {
      const int slot = u & 1;
      if (NM == 1 || slot == 0) wait(m, &m->v_full[vs], vp);
      wait(m, &m->p_full[slot], pp[slot]);
      pp[slot] ^= 1;
      tc_fence_after();
      const uint32_t v = smem + P::kAtV + vs * tile_bytes(DP);
#pragma unroll
      for (int i = 0; i < kTile / 16; ++i)
        mma_ts(tmem + kOColumn + slot * DP, tmem + slot * kTile + i * 8, operand_n(v + i * 2048, kTile * 128), kPV, u >= 2 || i > 0);
      if (NM == 1 || slot == 1) {
        mma_commit(smem_addr(&m->v_empty[vs]));
        if (++vs == P::kV) vs = 0, vp ^= 1;
      }
      if (u + 2 < units) scores(u + 2);
    }
    mma_commit(smem_addr(&m->o_full));
  } while (w.next(p));
  // (the last commits' arrivals are waited for below, so that no product is in flight when the block ends)
  wait(m, &m->o_full, w.piece & 1);
}

// --- softmax --------------------------------------------------------------------

// Values that were taken out of the tiles (take_out), for the rows that see them.
template <int KV, int N>
__device__ __noinline__ void add_bad_values(const AttendParams& p, const Item& it, int k0, int k1, int t, int column, float (&o)[N]) {
  if constexpr (KV == SJD_BF16) {
    const int end = min(it.keys, k1 * kTile);
    for (int key = max(k0 * kTile, it.start); key < end; ++key) {
      const bool seen = p.mask_kind == SJD_MASK_CAUSAL ? key <= it.start + t
                                                       : p.mask[p.mask_b * it.b + p.mask_r * t + (key - it.start)] != 0;
      const long long at = seen ? vector_at(p.c, it, key) : -1;
      if (at < 0) continue;
      const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.c.v) + at * p.c.D;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (column + i >= p.c.D) break;
        const float x = __bfloat162float(v[column + i]);
        if (!(fabsf(x) <= FLT_MAX)) o[i] += x;
      }
    }
  }
}

template <int KV, int DP, int NM>
__device__ __forceinline__ void softmax_rows(const AttendParams& p, Misc* m, uint32_t tmem, float* parts, float2* part_rows, Shared* shared) {
  const int slot = threadIdx.x / 128, row = threadIdx.x & 127, warp_row = row & ~31;
  const uint32_t lanes = static_cast<uint32_t>(warp_row) << 16;
  const uint32_t s_at = tmem + lanes + slot * kTile;
  const int G = p.c.Hq / p.c.Hkv;
  const float c = fabsf(p.scale) * 1.4426950408889634f;  // log2 e: weights are powers of two
  Walk<NM> w;
  if (!w.begin(p, m)) return;
  long long at_tile = m->first_tile;  // number, among all, of the piece's first tile
  uint32_t sp = 0;
  do {
    const Item& it = w.it;
    const int r0 = it.mt * (kTile * NM) + (NM == 2 ? slot * kTile : 0), r = r0 + row;
    const bool valid = r < it.rows, active = r0 + warp_row < it.rows;
    const int t = r / G, g = r - t * G;
    const int tiles = w.k1 - w.k0, units = NM == 2 ? tiles : (tiles + 1 - slot) / 2, stride = NM == 2 ? 1 : 2;
    const int k_first = w.k0 + (NM == 2 ? 0 : slot);
    // keys below `whole` are seen, those from `limit` on are not (a given mask tells between)
    const int limit = !valid ? 0x7fffffff : p.mask_kind == SJD_MASK_CAUSAL ? it.start + t + 1 : it.keys;
    const int whole = !valid ? 0x7fffffff : p.mask_kind == SJD_MASK_GIVEN ? it.start : limit;
    float ref = -INFINITY, sum = 0.0f;
    float next_k = 0.0f, next_v = 0.0f;
    auto factors = [&](int k) {
      if constexpr (KV != SJD_BF16) {
        const long long at = vector_at(p.c, it, k * kTile + row);
        next_k = at >= 0 ? p.c.ks[at] * c : 0.0f;
        next_v = at >= 0 ? p.c.vs[at] : 0.0f;
      }
    };
    if (units > 0) factors(k_first);
    for (int u = 0; u < units; ++u) {
      const int key0 = (k_first + u * stride) * kTile;
      if constexpr (KV != SJD_BF16) {
        named_barrier(2 + slot, 128);
        m->row[slot][0][row] = next_k;
        m->row[slot][1][row] = next_v;
        named_barrier(2 + slot, 128);
        if (u + 1 < units) factors(k_first + (u + 1) * stride);
      }
      wait(m, &m->s_full[slot], sp);
      sp ^= 1;
      tc_fence_after();
      if (active) {
        const bool mixed = !__all_sync(0xffffffffu, key0 + kTile <= whole);
        uint32_t seen[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
        if (mixed) {
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
              for (int key = a; key < e; ++key)
                if (!mask[key]) seen[i] &= ~(1u << (key - key0 - 32 * i));
            }
          }
        }
        __syncwarp();
        // the largest score
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t s[32];
          tmem_load32(s_at + 32 * i, s);
          tmem_wait_load(s);
          float a[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          if (mixed) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              const float x = __uint_as_float(s[j]) * (KV == SJD_BF16 ? 1.0f : m->row[slot][0][32 * i + j]);
              a[j & 3] = fmaxf(a[j & 3], seen[i] >> j & 1 ? x : -INFINITY);
            }
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              a[j & 3] = fmaxf(a[j & 3], __uint_as_float(s[j]) * (KV == SJD_BF16 ? 1.0f : m->row[slot][0][32 * i + j]));
          }
          top = fmaxf(top, fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])));
        }
        if (KV == SJD_BF16 && top != -INFINITY) top *= c;
        // The reference moves only where a weight could pass 2^8: the weights'
        // relative precision is the same below that, and O is left alone.
        const bool move = top > ref + kRise || (ref == -INFINITY && top != -INFINITY);
        if (__any_sync(0xffffffffu, move)) {
          const float f = !move ? 1.0f : ref == -INFINITY ? 0.0f : exp2_fast(ref - top);
          if (move) ref = top, sum *= f;
          __syncwarp();
          if (u > 0) {
            for (int i = 0; i < DP / 32; ++i) {
              uint32_t o[32];
              tmem_load32(tmem + lanes + kOColumn + slot * DP + 32 * i, o);
              tmem_wait_load(o);
#pragma unroll
              for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              tmem_store32(tmem + lanes + kOColumn + slot * DP + 32 * i, o);
            }
          }
        }
        const float base = ref == -INFINITY ? 0.0f : ref;
        float a[4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t s[32], out[16];
          tmem_load32(s_at + 32 * i, s);
          tmem_wait_load(s);
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            float x[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              x[e] = exp2_fast(fmaf(__uint_as_float(s[j + e]), KV == SJD_BF16 ? c : m->row[slot][0][32 * i + j + e], -base));
              if (mixed && !(seen[i] >> (j + e) & 1)) x[e] = 0.0f;
              a[(j + e) & 3] += x[e];
              if (KV != SJD_BF16) {
                const float f = m->row[slot][1][32 * i + j + e];
                x[e] = mixed && !(seen[i] >> (j + e) & 1) ? 0.0f : x[e] * f;
              }
            }
            out[j / 2] = pack_bf16(x[0], x[1]);
          }
          tmem_store16(s_at + 16 * i, out);
        }
        sum += (a[0] + a[1]) + (a[2] + a[3]);
        tmem_wait_store();
        tc_fence_before();
      }
      __syncwarp();
      if ((threadIdx.x & 31) == 0) mbar_arrive(smem_addr(&m->p_full[slot]));
    }
    // the end of the piece: O of both slots is complete
    wait(m, &m->o_full, w.piece & 1);
    tc_fence_after();
    float f[2] = {1.0f, 1.0f};
    bool take[2] = {NM == 1 || slot == 0, NM == 1 ? tiles > 1 : slot == 1};
    if constexpr (NM == 1) {
      named_barrier(2 + slot, 128);  // (all of the group are done with the factors)
      m->row[slot][0][row] = ref;
      m->row[slot][1][row] = sum;
      named_barrier(1, 256);
      const float r1 = tiles > 1 ? m->row[1][0][row] : -INFINITY, r0s = m->row[0][0][row];
      const float s1 = tiles > 1 ? m->row[1][1][row] : 0.0f, s0 = m->row[0][1][row];
      ref = fmaxf(r0s, r1);
      f[0] = r0s == -INFINITY ? 0.0f : exp2_fast(r0s - ref);
      f[1] = r1 == -INFINITY ? 0.0f : exp2_fast(r1 - ref);
      sum = s0 * f[0] + s1 * f[1];
    }
    const bool wholly = w.k0 == 0 && w.k1 == it.tiles;
    const bool bad = KV == SJD_BF16 && *const_cast<volatile int*>(&m->bad_values[w.piece & 3]) == w.piece + 1;
    // this thread's columns of its row
    constexpr int kColumns = NM == 1 ? DP / 2 : DP;
    const int column0 = NM == 1 ? slot * kColumns : 0;
    const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    const long long part = 2ll * blockIdx.x + (w.k0 == 0 ? 1 : 0);
    const long long token = static_cast<long long>(it.b) * p.c.n + t;
    const long long head = token * p.c.Hq + static_cast<long long>(it.kvh) * G + g;
    if (active) {
#pragma unroll
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
          tmem_load32(tmem + lanes + kOColumn + e * DP + column, x);
          tmem_wait_load(x);
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = NM == 1 ? fmaf(__uint_as_float(x[j]), f[e], o[j]) : __uint_as_float(x[j]);
        }
        if (KV == SJD_BF16 && bad && valid) {
          float with[32];
          for (int j = 0; j < 32; ++j) with[j] = o[j];
          add_bad_values<KV>(p, it, w.k0, w.k1, t, column, with);
          for (int j = 0; j < 32; ++j) o[j] = with[j];
        }
        if (valid && wholly) {
          __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.o) + head * p.c.D + column;
#pragma unroll
          for (int j = 0; j < 32; j += 8)
            if (column + j < p.c.D)
              *reinterpret_cast<uint4*>(to + j) =
                  make_uint4(pack_bf16(o[j] * inverse, o[j + 1] * inverse), pack_bf16(o[j + 2] * inverse, o[j + 3] * inverse),
                             pack_bf16(o[j + 4] * inverse, o[j + 5] * inverse), pack_bf16(o[j + 6] * inverse, o[j + 7] * inverse));
        } else if (valid) {
          float* to = parts + (part * (kTile * NM) + (NM == 2 ? slot * kTile : 0) + row) * DP + column;
#pragma unroll
          for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
        }
      }
      if (valid && (NM == 2 || slot == 0)) {
        if (wholly) {
          if (p.lse) p.lse[head] = sum > 0.0f || sum != sum ? (ref + log2f(sum)) * 0.69314718055994531f : -INFINITY;
        } else {
          part_rows[part * (kTile * NM) + (NM == 2 ? slot * kTile : 0) + row] = make_float2(ref, sum);
        }
      }
    }
    if (threadIdx.x == 0 && w.k0 == 0 && w.k1 < it.tiles) {
      // the rest of the item lies in the blocks after this one
      const long long per = m->tiles, beyond = at_tile + it.tiles - 1;
      shared[blockIdx.x] = {static_cast<int>(beyond / per - blockIdx.x + 1), it.kvh, it.b, it.mt};
    }
    if constexpr (NM == 1) {
      tc_fence_before();
      named_barrier(1, 256);  // both groups have read both accumulators and the rows' sums
    }
    at_tile += w.k1 - w.k0;
  } while (w.next(p));
}

template <int KV, int DP, int NM>
__global__ void __launch_bounds__(kAttendThreads, 1) attend_kernel(const AttendParams p, float* parts, float2* part_rows, Shared* shared) {
  extern __shared__ __align__(1024) unsigned char raw[];
  using P = Plan<DP, NM>;
  Misc* m = reinterpret_cast<Misc*>(raw + P::kAtMisc);
  const uint32_t smem = smem_addr(raw);
  const int warp = threadIdx.x / 32;
  if (warp == 0) locate<NM>(p, m);
  if (warp == kMmaWarp) tmem_alloc(smem_addr(&m->tmem), kTmemColumns);
  if (threadIdx.x == 128) {
    for (int i = 0; i < 5; ++i) {
      mbar_init(smem_addr(&m->k_full[i]), 4), mbar_init(smem_addr(&m->k_empty[i]), 1);
      mbar_init(smem_addr(&m->v_full[i]), 4), mbar_init(smem_addr(&m->v_empty[i]), 1);
    }
    mbar_init(smem_addr(&m->q_full), 4), mbar_init(smem_addr(&m->q_empty), 1), mbar_init(smem_addr(&m->o_full), 1);
    for (int i = 0; i < 2; ++i) mbar_init(smem_addr(&m->s_full[i]), 1), mbar_init(smem_addr(&m->p_full[i]), 4);
    m->abort = 0;
    for (int i = 0; i < 4; ++i) m->bad_values[i] = 0;
    shared[blockIdx.x].parts = 0;
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = m->tmem;
  if (warp < 8) {
    softmax_rows<KV, DP, NM>(p, m, tmem, parts, part_rows, shared);
  } else if (warp < 12) {
    load_operand<KV, DP, NM, false>(p, m, smem);
  } else if (warp < 16) {
    load_operand<KV, DP, NM, true>(p, m, smem);
  } else {
    if ((threadIdx.x & 31) == 0) issue_products<DP, NM>(p, m, smem, tmem);
    __syncwarp();
  }
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
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, G = p.c.Hq / p.c.Hkv;
  const Shared s = shared[blockIdx.x];
  const int row0 = blockIdx.y * kJoinWarps + warp, step = gridDim.y * kJoinWarps;
  if (s.parts > 1) {
    const int2 span = span_of(p.c, s.b);
    for (int row = row0; row < rows_per_item; row += step) {
      const int r = s.mt * rows_per_item + row;
      if (r >= span.y * G) break;
      auto part_at = [&](int i) { return (2ll * (blockIdx.x + i) + (i == 0 ? 1 : 0)) * rows_per_item + row; };
      float top = -INFINITY;
      for (int i = lane; i < s.parts; i += 32) top = fmaxf(top, part_rows[part_at(i)].x);
      for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      float sum = 0.0f, o[DP / 32] = {};
#pragma unroll 4
      for (int i = 0; i < s.parts; ++i) {
        const float2 rs = part_rows[part_at(i)];
        const float f = rs.x == -INFINITY ? 0.0f : exp2_fast(rs.x - top);
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
      const int t = r / G, g = r - t * G;
      const long long head = (static_cast<long long>(s.b) * p.c.n + t) * p.c.Hq + static_cast<long long>(s.kvh) * G + g;
      __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.o) + head * p.c.D + lane * (DP / 32);
      if (lane * (DP / 32) < p.c.D) {
#pragma unroll
        for (int j = 0; j < DP / 32; j += 2) *reinterpret_cast<uint32_t*>(to + j) = pack_bf16(o[j] * inverse, o[j + 1] * inverse);
      }
      if (p.lse && lane == 0) p.lse[head] = sum > 0.0f || sum != sum ? (top + log2f(sum)) * 0.69314718055994531f : -INFINITY;
    }
  }
  for (int b = blockIdx.x; b < p.c.B; b += gridDim.x) {
    const int2 span = span_of(p.c, b);
    const long long begin = (static_cast<long long>(b) * p.c.n + span.y) * p.c.Hq, end = (b + 1ll) * p.c.n * p.c.Hq;
    for (long long row = begin + row0; row < end; row += step) {
      for (int i = lane; i < p.c.D / 8; i += 32)
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.o) + row * p.c.D + 8 * i) = make_uint4(0, 0, 0, 0);
      if (p.lse && lane == 0) p.lse[row] = -INFINITY;
    }
  }
}

template <int KV, int DP, int NM>
cudaError_t launch(const AttendParams& p, int sms, unsigned char* scratch, cudaStream_t s) {
  const int blocks = sms < kMaxAttendBlocks ? sms : kMaxAttendBlocks;
  const size_t rows = static_cast<size_t>(kTile) * NM * 2 * blocks;
  Shared* shared = reinterpret_cast<Shared*>(scratch);
  float2* part_rows = reinterpret_cast<float2*>(scratch + kMaxAttendBlocks * sizeof(Shared));
  float* parts = reinterpret_cast<float*>(part_rows + rows);
  auto* kernel = attend_kernel<KV, DP, NM>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared_bytes<DP, NM>());
  if (e != cudaSuccess) return e;
  kernel<<<blocks, kAttendThreads, shared_bytes<DP, NM>(), s>>>(p, parts, part_rows, shared);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  join_kernel<DP><<<dim3(blocks, 8), 32 * kJoinWarps, 0, s>>>(p, parts, part_rows, shared, kTile * NM);
  return cudaGetLastError();
}

template <int KV>
cudaError_t launch_of(const AttendParams& p, int sms, unsigned char* scratch, cudaStream_t s) {
  const bool two = static_cast<long long>(p.c.n) * (p.c.Hq / p.c.Hkv) > kTile;
  if (p.c.D <= 64) return two ? launch<KV, 64, 2>(p, sms, scratch, s) : launch<KV, 64, 1>(p, sms, scratch, s);
  return two ? launch<KV, 128, 2>(p, sms, scratch, s) : launch<KV, 128, 1>(p, sms, scratch, s);
}

}  // namespace

size_t attend_scratch_bytes(int head_dim, long long rows) {
  const size_t per = (rows > kTile ? 2 : 1) * static_cast<size_t>(kTile), dp = head_dim <= 64 ? 64 : 128;
  return kMaxAttendBlocks * (sizeof(Shared) + 2 * per * (sizeof(float2) + dp * sizeof(float)));
}

cudaError_t launch_attend(const AttendParams& p, int kv_dtype, int sms, unsigned char* scratch, cudaStream_t s) {
  if (kv_dtype == SJD_BF16) return launch_of<SJD_BF16>(p, sms, scratch, s);
  if (kv_dtype == SJD_E4M3) return launch_of<SJD_E4M3>(p, sms, scratch, s);
  return launch_of<SJD_S8>(p, sms, scratch, s);
}

}  // namespace sjd_kv_ops
