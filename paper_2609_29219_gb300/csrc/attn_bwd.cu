// Attention's backward pass for GB300 (sm_103a): TMA + mbarrier rings, tcgen05 MMAs with TMEM
// accumulators, warp-specialised loader / MMA / elementwise roles.
//
// With S = scale Q K^T, P = exp(S - LSE) (0 where masked), dP = dO V^T and, per query row,
// delta = dO . O - dLSE,
//     dS = P o (dP - delta),   dV = P^T dO,   dK = scale dS^T Q,   dQ = scale dS K
// (dK and dV summed over the query heads of a kv head).  P is recomputed from LSE, which the
// forward pass returns, so no score leaves the chip.
//
// Two launches:
//   attn_bwd_rows_kernel  delta and LSE of every query row, negated and in base 2, into the
//                         workspace in tiles of 128 rows; the item counters, and dQ of ragged queries
//                         that see no key, zeroed
//   attn_bwd_kernel       persistent CTAs.  First the items (kv tile of 128 keys of a kv head):
//                         dK and dV stay in TMEM while the CTA walks the query tiles of every
//                         head of the group.  Then the items (query tile of 128 rows of a head):
//                         dQ stays in TMEM while the CTA walks the keys.
// A gradient's sum stays in TMEM over a whole item, or a share of one, in a fixed order: no atomics on
// values, the same bits each time.  The price is that S and dP are computed in both walks: seven
// products of 128 x 128 x D per pair of tiles instead of five.  What it saves is fp32 sums of dQ in
// memory, 512 D bytes for every pair of tiles, added in an order that would have to be kept.  What the plan
// deals in shares (bwd.h; 512 items of H32/8 S8192 too) does pass through memory in fp32: one partial sum
// a share.
// Items are taken from a counter, long ones first, so CTAs that finish the kv items early start on
// the query items.
//
// P and dS are rounded to bf16 where they become operands of dV, dK and dQ, as the forward rounds P:
// in 32 bits they would take a slower kind of product, twice the TMEM, and operands Q, K and dO of
// that type.  A gradient's error against 64 bits is 0.0024 of its norm; 0.0017 with one rounding, at the end.
//
// What bounds it: the tensor pipe and the hand-overs around it.  A step of a kv item (D = 128) is four
// products, 2048 clocks of the pipe, and takes 2940: the score products read both operands from
// shared memory, at all of its bandwidth, so that dK and the next dP take 1440 to 1600 clocks
// together, dV and the next S 1250 to 1380; a query item's step takes 2110 for its three (1536).
// GB300, on the device alone (graph replays): B4 H32 S2048 D128 causal 355 to 359 us (958 to 968 TFLOP/s
// of the five products that the gradients need, 1.4 times that of the seven), B1 H32/8 S8192 1073 to 1093
// (1257 to 1281; under the power limit), D64 H64/16 S8192 1650 to 1657 (829 to 833; not traced).  Call after
// call: 371 to 388, 1166 to 1256.
#include <cuda.h>
#include <cuda_bf16.h>

#include <cmath>
#include <cstring>
#include <mutex>

#include "bwd.h"
#include "kernels.h"
#include "ptx.cuh"

namespace loom {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTile = 128;   // queries and keys per tile
constexpr int kEltWarps = 8;  // elementwise warps: four for each half of a tile's columns
constexpr int kLoader = kEltWarps, kMma0 = kEltWarps + 1, kMma1 = kEltWarps + 2;
// Ragged batches have one more warp, which clears what follows a sequence's end (clean_tiles).
constexpr int kCleaner = kMma1 + 1;
template <bool VARLEN>
constexpr int kThreads = (VARLEN ? kCleaner + 1 : kMma1 + 1) * 32;
constexpr int kShortItem = 4;  // steps
constexpr int kRowThreads = 256, kRowsPerBlock = 32;  // of the row statistics
constexpr int kStat = 2 * kTile;  // floats of a query tile's row statistics: -LSE (base 2), then -delta

template <int D>
struct BwdCfg {
  static constexpr int NBOX = D / 64;  // 128-byte-swizzled boxes of 64 columns per tile
  static constexpr uint32_t BOX_BYTES = kTile * 128;
  static constexpr uint32_t TILE_BYTES = NBOX * BOX_BYTES;
  // An item's own two tiles: D = 64 has room to load the next item's beside them.
  static constexpr int NOWN = D == 128 ? 1 : 2;
  // kv items: K, V, then rings of Q and dO tiles and of row statistics
  static constexpr int NQ = D == 128 ? 3 : 4, ND = D == 128 ? 2 : 4;
  static constexpr uint32_t K_OFF = 0, V_OFF = NOWN * TILE_BYTES;
  static constexpr uint32_t QR_OFF = 2 * NOWN * TILE_BYTES, DOR_OFF = QR_OFF + NQ * TILE_BYTES;
  static constexpr uint32_t ST_OFF = DOR_OFF + ND * TILE_BYTES;
  static constexpr uint32_t KV_END = ST_OFF + ND * kStat * 4;
  // query items: Q, dO, then rings of K and V tiles
  static constexpr int NK = D == 128 ? 3 : 5, NV = D == 128 ? 2 : 4;
  static constexpr uint32_t Q_OFF = 0, DO_OFF = NOWN * TILE_BYTES;
  static constexpr uint32_t KR_OFF = 2 * NOWN * TILE_BYTES, VR_OFF = KR_OFF + NK * TILE_BYTES;
  static constexpr uint32_t Q_END = VR_OFF + NV * TILE_BYTES;
  static constexpr uint32_t ITEM_OFF = KV_END > Q_END ? KV_END : Q_END;  // two item records
  static constexpr uint32_t BAR_OFF = ITEM_OFF + 2 * 64;
  static constexpr int NBAR = 8 * NOWN + 3 * NQ + 2 * ND + 11 + 3 * NK + 3 * NV + 8 + 8;
  static constexpr uint32_t TMEM_PTR_OFF = BAR_OFF + NBAR * 8;
  static constexpr uint32_t ABORT_OFF = TMEM_PTR_OFF + 8;
  static constexpr uint32_t BYTES = ABORT_OFF + 16;  // from a 1024-byte boundary
  static_assert(BYTES <= 227 * 1024, "shared memory budget");
  // TMEM: S / P at 0, dP / dS at 128; kv items dV at 256, dK at 256 + D; query items dQ at 256, two
  // buffers of dS at 384 and 448
  static constexpr uint32_t S_COL = 0, DP_COL = 128, DV_COL = 256, DK_COL = 256 + D, DQ_COL = 256, DS_COL = 384;
};

struct BwdParams {
  __nv_bfloat16 *dq, *dk, *dv;
  const float* stats;       // [planes][tiles][2][128]
  unsigned int* counters;   // [0] kv items, [1] query items; from [64] on, arrivals at split items
  float* partial;           // gradients of the shares of split items
  int kv_split, q_split;    // shares that an item's steps are dealt to at most
  int kv_slots;             // kv items that counters and partial gradients have room for; query items follow
  int B, Hq, Hkv, Sq, Skv, causal;
  int wide;                 // dq, dk and dv are 32-byte aligned
  int lg;                   // a query plane's rows are those of 2^lg heads of one kv head
  float c;                  // scale * log2(e)
  float scale;
  int q_tiles, kv_tiles;    // dense: tiles per plane
  int stat_tiles;           // tiles of row statistics per plane
  int q_items, kv_items;    // dense: items
  int q_block, kv_block;    // planes whose tiles are dealt together (see item order)
  const int32_t *cu_q, *cu_k;
  int total_q, total_k;
  KernelCtl ctl;
};

// Query planes.  The rows of a plane are the rows of 2^lg query heads of one kv head, ordered by
// query: row i is query i >> lg of the plane's head i mod 2^lg.  A tile of 128 rows then has 128 >> lg
// queries of each, so that few or odd numbers of queries still fill tiles (chunk of 515 queries, 4
// heads per kv head: 17 tiles instead of 20; one query of 8 heads: one tile instead of 8).
//
// One item as the roles see it.  Rows are counted within the sequence's plane.
struct Item {
  int n;          // steps of this share (0: gradients are zero); -1: no item is left, -2: an empty share
  int row0;       // first row of the item's own tile (keys / queries)
  int plane;      // kv items: kv plane; query items: query plane
  int other;      // kv items: first query plane of the group; query items: kv plane
  int t0, nt;     // kv items: query tiles t0 .. t0 + nt - 1 of each plane
  int g, t;       // the share's first step: plane of the group (kv items), tile
  int shares;     // shares of the item that have steps
  int id, share;  // the item, and which of its shares this is
  int sq, skv;    // lengths in queries (that see a key) and keys
  int qb, kb;     // first query (that sees a key) and key row of the sequence (0 for dense)
  int stat0;      // first tile of the sequence within a plane's row statistics
};
static_assert(sizeof(Item) <= 64, "item record");

// ---------------------------------------------------------------- item order
// Dense: blocks of `block` planes; within a block tile by tile over the planes, the longest
// tiles first.  Planes in flight together share what they walk in L2.
struct DenseItem {
  int tile, plane;
};
__device__ __forceinline__ DenseItem dense_item(int idx, int tiles, int planes, int block) {
  const int per = block * tiles, blk = idx / per, in = idx - blk * per;
  const int p0 = blk * block, nb = min(block, planes - p0);
  return {in / nb, p0 + in % nb};
}

// Ragged: sequences in order; a cursor that only moves forward (a CTA's indices grow).
struct Cursor {
  int b;
  long long first;  // index of sequence b's first item
  int tiles;        // its tiles per plane
};
__device__ __forceinline__ int seq_tiles(const int32_t* cu, int b, int lg) {
  const int n = cu[b + 1] - cu[b];
  return n > 0 ? ((n << lg) + kTile - 1) / kTile : 0;
}
__device__ __forceinline__ bool cursor_to(Cursor& cur, const int32_t* cu, int lg, int B, int planes, long long idx) {
  if (cur.b < 0) cur = {0, 0, seq_tiles(cu, 0, lg)};
  while (cur.b < B && idx >= cur.first + static_cast<long long>(cur.tiles) * planes) {
    cur.first += static_cast<long long>(cur.tiles) * planes;
    ++cur.b;
    cur.tiles = cur.b < B ? seq_tiles(cu, cur.b, lg) : 0;
  }
  return cur.b < B;
}
// Queries at a ragged sequence's start that see no key (causal, more queries than keys).  The walks
// begin behind them: masked by a probability of zero alone, a NaN or an infinity of theirs would reach
// the others' gradients.
__device__ __forceinline__ int unseen_queries(int sq, int skv, int causal) { return causal ? max(0, sq - skv) : 0; }
// First tile of sequence b in a plane's row statistics: tiles of different sequences never meet.
__device__ __forceinline__ int ragged_stat0(const int32_t* cu_q, int b, int lg) {
  return static_cast<int>((static_cast<long long>(cu_q[b]) << lg) / kTile) + b;
}

// KV: item idx of the kv items, else of the query items.
// An item is split where the plan deals its steps in shares: these accumulate a run of its
// steps each, write what they have in fp32, and the last one to arrive adds them up in their order.
template <bool KV, bool VARLEN, bool SPLIT>
__device__ __forceinline__ Item make_item(const BwdParams& p, long long idx, Cursor& cur) {
  Item it;
  it.n = -1;
  const int split = KV ? p.kv_split : p.q_split;
  if constexpr (SPLIT) {
    it.share = static_cast<int>(idx % split);
    idx /= split;
    it.id = static_cast<int>(idx);
  }
  int tile, b;
  const int G = p.Hq / p.Hkv >> p.lg, HP = p.Hq >> p.lg;  // query planes of a kv head, of a sequence
  if constexpr (VARLEN) {
    const int planes = KV ? p.Hkv : HP;
    const int32_t* cu = KV ? p.cu_k : p.cu_q;
    if (!cursor_to(cur, cu, KV ? 0 : p.lg, p.B, planes, idx)) return it;
    b = cur.b;
    const int in = static_cast<int>(idx - cur.first);
    tile = in / planes;
    it.plane = in % planes;
    it.other = KV ? it.plane * G : it.plane / G;
    it.qb = p.cu_q[b];
    it.kb = p.cu_k[b];
    it.sq = p.cu_q[b + 1] - it.qb;
    it.skv = p.cu_k[b + 1] - it.kb;
    const int unseen = unseen_queries(it.sq, it.skv, p.causal);
    it.qb += unseen;
    it.sq -= unseen;
    it.stat0 = ragged_stat0(p.cu_q, b, p.lg);
    // (causal query tiles are longest at the sequence's end)
    if (!KV && p.causal) tile = cur.tiles - 1 - tile;
  } else {
    if (idx >= (KV ? p.kv_items : p.q_items)) return it;
    const DenseItem d = KV ? dense_item(static_cast<int>(idx), p.kv_tiles, p.B * p.Hkv, p.kv_block)
                           : dense_item(static_cast<int>(idx), p.q_tiles, p.B * HP, p.q_block);
    it.plane = d.plane;
    if constexpr (KV) {
      b = d.plane / p.Hkv;
      it.other = b * HP + (d.plane - b * p.Hkv) * G;
    } else {
      b = d.plane / HP;
      it.other = b * p.Hkv + (d.plane - b * HP) / G;
    }
    tile = !KV && p.causal ? p.q_tiles - 1 - d.tile : d.tile;
    it.qb = it.kb = it.stat0 = 0;
    it.sq = p.Sq;
    it.skv = p.Skv;
  }
  it.row0 = tile * kTile;
  const int off = it.skv - it.sq;  // query i sees keys <= i + off
  if constexpr (KV) {
    const int tiles = ((it.sq << p.lg) + kTile - 1) / kTile;
    it.t0 = p.causal ? min(tiles, (max(0, min(it.sq, it.row0 - off)) << p.lg) / kTile) : 0;
    it.nt = tiles - it.t0;
    const int steps = it.nt * G;
    it.n = steps;
    it.g = 0;
    it.t = it.t0;
    if constexpr (SPLIT) {
      it.shares = max(1, min(split, steps));
      const int lo = static_cast<int>(static_cast<long long>(steps) * it.share / it.shares);
      it.n = it.share < it.shares ? static_cast<int>(static_cast<long long>(steps) * (it.share + 1) / it.shares) - lo : -2;
      it.g = it.nt > 0 ? lo / it.nt : 0;
      it.t += lo - it.g * it.nt;
    }
  } else {
    const int seen = p.causal ? min(it.skv, ((it.row0 + kTile) >> p.lg) + off) : it.skv;
    // (ragged: the sequence has a tile for the unseen queries too)
    const int steps = seen > 0 && (!VARLEN || it.row0 < it.sq << p.lg) ? (seen + kTile - 1) / kTile : 0;
    it.n = steps;
    it.t = 0;
    if constexpr (SPLIT) {
      it.shares = max(1, min(split, steps));
      it.t = static_cast<int>(static_cast<long long>(steps) * it.share / it.shares);
      it.n = it.share < it.shares ? static_cast<int>(static_cast<long long>(steps) * (it.share + 1) / it.shares) - it.t : -2;
    }
  }
  return it;
}

// ---------------------------------------------------------------- shared pieces
// Items pass from the loader to the other roles through two records.
struct ItemRing {
  uint32_t full, empty;  // two barriers each
  Item* rec;
};
__device__ __forceinline__ bool ring_put(const ItemRing& r, int i, const Item& it, const KernelCtl& ctl, const Abort& ab) {
  if (i >= 2 && !mbar_wait(r.empty + 8 * (i & 1), ((i >> 1) - 1) & 1, ctl, ab)) return false;
  r.rec[i & 1] = it;
  mbar_arrive(r.full + 8 * (i & 1));
  return true;
}
// The i-th item, read by a whole warp.
__device__ __forceinline__ bool ring_get(const ItemRing& r, int i, Item& it, const KernelCtl& ctl, const Abort& ab) {
  if (!mbar_wait_warp(r.full + 8 * (i & 1), (i >> 1) & 1, ctl, ab)) return false;
  it = r.rec[i & 1];
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(r.empty + 8 * (i & 1));
  return true;
}
// A whole warp's wait for two barriers at once, by different lanes: a wait costs the MMA warp some
// 150 clocks even if the phase is over, and it has no time to spare.
__device__ __forceinline__ bool wait_two(uint32_t bar0, uint32_t par0, uint32_t bar1, uint32_t par1, const KernelCtl& ctl,
                                         const Abort& ab) {
  const bool odd = threadIdx.x & 1;
  return mbar_wait_warp(odd ? bar1 : bar0, odd ? par1 : par0, ctl, ab);
}
__device__ __forceinline__ bool wait_three(uint32_t bar0, uint32_t par0, uint32_t bar1, uint32_t par1, uint32_t bar2,
                                           uint32_t par2, const KernelCtl& ctl, const Abort& ab) {
  const int i = threadIdx.x & 3;
  return mbar_wait_warp(i == 0 ? bar0 : i == 1 ? bar1 : bar2, i == 0 ? par0 : i == 1 ? par1 : par2, ctl, ab);
}
// One arrival for a warp whose lanes are all done with what the barrier guards.
__device__ __forceinline__ void warp_arrive(uint32_t bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
template <bool VARLEN>
constexpr int kItemReaders = kEltWarps + (VARLEN ? 3 : 2);  // the elementwise warps, the MMA warps and the cleaner

// A tile of a query plane: 128 >> lg queries of 2^lg heads, from row `row` of the plane of a sequence
// that starts at query qb.
template <int D, bool VARLEN>
__device__ __forceinline__ void load_q_tile(uint32_t dst, const CUtensorMap* map, int plane, int qb, int row, int lg,
                                            uint32_t bar) {
  using C = BwdCfg<D>;
  const int query = qb + (row >> lg);
#pragma unroll
  for (int x = 0; x < C::NBOX; ++x)
    tma_load_4d(dst + x * C::BOX_BYTES, map, x * 64, 0, VARLEN ? plane : query, VARLEN ? query : plane, bar);
}
template <int D, bool VARLEN>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int plane, int row, uint32_t bar) {
  using C = BwdCfg<D>;
#pragma unroll
  for (int x = 0; x < C::NBOX; ++x)
    tma_load_3d(dst + x * C::BOX_BYTES, map, x * 64, VARLEN ? plane : row, VARLEN ? row : plane, bar);
}

// A ragged batch's last tile of a sequence goes on with the next sequence's rows, which must not
// reach this one's gradients whatever they hold (a NaN or an infinity times a zero probability
// would): rows [n, 128) become zeros before anything reads the tile.  A warp of its own does it,
// between the arrival of each tile and the MMA warps: in those, it would cost a step's critical path
// 1000 clocks (ragged batch of 8, 100 to 2048 tokens: 320 us; here 295), and so do products that stop at the last
// row.
template <int D>
__device__ __forceinline__ void zero_rows(uint32_t tile, int n) {
  using C = BwdCfg<D>;
  for (int x = 0; x < C::NBOX; ++x)
    for (uint32_t o = n * 128 + (threadIdx.x & 31) * 16; o < C::BOX_BYTES; o += 512)
      st_shared_v4(tile + x * C::BOX_BYTES + o, 0, 0, 0, 0);
  fence_proxy_async_smem();
}
// One tile of a ring, at step m: n rows of it belong to the sequence.
template <int D, int SLOTS>
__device__ __forceinline__ bool clean_tile(uint32_t ring, uint32_t full, uint32_t clean, int m, int n, const KernelCtl& ctl,
                                           const Abort& ab) {
  const int slot = m % SLOTS;
  if (!mbar_wait_warp(full + 8 * slot, m / SLOTS & 1, ctl, ab)) return false;
  if (n < kTile) zero_rows<D>(ring + slot * BwdCfg<D>::TILE_BYTES, n);
  warp_arrive(clean + 8 * slot);
  return true;
}

// The MMAs of one pair of tiles.  D[128 x 128] = A B^T, both K-major in shared memory.
template <int D>
__device__ __forceinline__ void issue_scores(uint32_t d_tmem, uint32_t a, uint32_t b) {
  using C = BwdCfg<D>;
  constexpr uint32_t idesc = idesc_bf16(kTile, kTile, 0, 0);
  const uint64_t da = sdesc_sw128(a, 16, 1024), db = sdesc_sw128(b, 16, 1024);
#pragma unroll
  for (int x = 0; x < C::NBOX; ++x)
    mma_ss_k64_el(d_tmem, da + x * (C::BOX_BYTES >> 4), db + x * (C::BOX_BYTES >> 4), idesc, x > 0);
}
// D[128 x D] += A B over 64 of the tile's rows: A in TMEM (packed bf16), B's rows 64 h .. 64 h + 63.
template <int D>
__device__ __forceinline__ void issue_grad_half(uint32_t d_tmem, uint32_t a_tmem, uint32_t b, int h, bool acc) {
  using C = BwdCfg<D>;
  constexpr uint32_t idesc = idesc_bf16(kTile, D, 0, 1);
  mma_ts_k64_el(d_tmem, a_tmem, sdesc_sw128(b, C::BOX_BYTES, 1024) + h * 64 * (128 >> 4), idesc, acc ? 1u : 0u);
}
// The same over chunk c (32 rows) of each half of the tile: A's halves are 64 columns apart.
template <int D>
__device__ __forceinline__ void issue_grad_chunks(uint32_t d_tmem, uint32_t a_tmem, uint32_t b, int c, bool acc) {
  using C = BwdCfg<D>;
  constexpr uint32_t idesc = idesc_bf16(kTile, D, 0, 1);
  const uint64_t db = sdesc_sw128(b, C::BOX_BYTES, 1024) + c * 32 * (128 >> 4);
  mma_ts_k32_el(d_tmem, a_tmem + 16 * c, db, idesc, acc ? 1u : 0u);
  mma_ts_k32_el(d_tmem, a_tmem + 64 + 16 * c, db + 64 * (128 >> 4), idesc, 1u);
}
// A word whose lowest n bits are set.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

// 64 TMEM columns of this thread's lane.
__device__ __forceinline__ void ld64(uint32_t tm, uint32_t* r) {
  tmem_ld32(tm, r);
  tmem_ld32(tm + 32, r + 32);
  tmem_wait_ld();
  reg_fence32(r);
  reg_fence32(r + 32);
}

// A gradient row's COLS values from TMEM, scaled, as bf16 to global memory: dst is this thread's row,
// store whether there is one.  Lanes 2 i and 2 i + 1 swap halves of 64-byte pieces first, so that a
// warp's 32-byte stores meet 16 rows each instead of 32: a store instruction takes the load/store
// unit a clock per 128-byte line, and a tile's 16-byte stores row by row 2 us of an item's end.
// wide: the tensors are 32-byte aligned (else 16-byte stores, row by row).
__device__ __forceinline__ void st_global_v8(__nv_bfloat16* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
// Where a row goes, and the neighbouring lane's.
struct RowOut {
  __nv_bfloat16 *mine, *other;
  bool store, other_store, wide;
};
__device__ __forceinline__ RowOut row_out(__nv_bfloat16* dst, bool store, bool wide) {
  return {dst,
          reinterpret_cast<__nv_bfloat16*>(__shfl_xor_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), 1)), store,
          static_cast<bool>(__shfl_xor_sync(0xffffffffu, store, 1)), wide};
}
__device__ __forceinline__ void store_32(const RowOut& out, int c, const uint32_t* r, uint64_t s2) {
  const bool odd = threadIdx.x & 1;
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint64_t x = mul2(f2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), s2);
    w[i] = pack_bf16x2(f2lo(x), f2hi(x));
  }
  if (out.wide) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? w[i] : w[8 + i], 1);
      if (odd)
        w[i] = got;
      else
        w[8 + i] = got;
    }
    // w[0..7]: of the even lane's row, w[8..15]: of the odd lane's
    const int at = c + (odd ? 16 : 0);
    if (odd ? out.other_store : out.store) st_global_v8((odd ? out.other : out.mine) + at, w);
    if (odd ? out.store : out.other_store) st_global_v8((odd ? out.mine : out.other) + at, w + 8);
  } else if (out.store) {
    uint4* d = reinterpret_cast<uint4*>(out.mine + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}

// The end of an item for one warp: its 32 rows and COLS columns of the gradient, from TMEM at tm.
// shares > 1: an item's share.  The warp writes its part of the sum (float4s of four columns, lanes
// side by side), and of the shares' warps with the same rows and columns the last one to arrive at
// `arrivals` adds the parts, in the shares' order.
struct Finish {  // what is kept of an item until its end
  __nv_bfloat16* dst;  // this lane's row
  int id;
  uint32_t bits;       // shares, share << 8, store << 16 (there is such a row)
};
// part0: this lane's first float4 of share 0's part, part_step: floats from share to share.
template <int COLS, bool SPLIT>
__device__ __forceinline__ void finish_rows(const Finish& f, uint32_t tm, float scale, bool wide, uint32_t bar_acce,
                                            float* part0, size_t part_step, unsigned int* arrivals) {
  const RowOut out = row_out(f.dst, f.bits >> 16, wide);
  const int shares = SPLIT ? f.bits & 255 : 1, share = f.bits >> 8 & 255;
  const uint64_t s2 = f2(scale, scale);
  uint32_t r[32];
#pragma unroll 1
  for (int c = 0; c < COLS; c += 32) {
    tmem_ld32(tm + c, r);
    tmem_wait_ld();
    reg_fence32(r);
    if (shares == 1) {
      store_32(out, c, r, s2);
    } else {
      float4* d = reinterpret_cast<float4*>(part0 + share * part_step) + (c / 4) * kTile;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        d[i * kTile] = make_float4(__uint_as_float(r[4 * i]), __uint_as_float(r[4 * i + 1]), __uint_as_float(r[4 * i + 2]),
                                   __uint_as_float(r[4 * i + 3]));
    }
  }
  tc_fence_before();
  warp_arrive(bar_acce);
  if (!SPLIT || shares == 1) return;
  __threadfence();
  __syncwarp();
  unsigned int before = 0;
  if ((threadIdx.x & 31) == 0) before = atomicAdd(arrivals, 1u);
  if (__shfl_sync(0xffffffffu, before, 0) != static_cast<unsigned int>(shares) - 1) return;
  __threadfence();
#pragma unroll 1
  for (int c = 0; c < COLS; c += 32) {
    float a[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) a[i] = 0.f;
#pragma unroll 1
    for (int s = 0; s < shares; ++s) {
      const float4* d = reinterpret_cast<const float4*>(part0 + s * part_step) + (c / 4) * kTile;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 v = __ldcg(d + i * kTile);
        a[4 * i] += v.x, a[4 * i + 1] += v.y, a[4 * i + 2] += v.z, a[4 * i + 3] += v.w;
      }
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(a[i]);
    store_32(out, c, r, s2);
  }
}
template <int COLS>
__device__ __forceinline__ void store_zeros(__nv_bfloat16* dst) {
#pragma unroll
  for (int c = 0; c < COLS; c += 8) *reinterpret_cast<uint4*>(dst + c) = make_uint4(0, 0, 0, 0);
}

struct Shared {
  uint32_t base, bars, tmem;
  ItemRing items;
  Abort ab, drain_ab;
};

// P^T of the queries e0 .. e0 + 31 of this thread's 64 (and its key row) from S^T in s: left in s
// as fp32, and in pk as bf16.  nl: -LSE of the 64 queries in shared memory.
__device__ __forceinline__ void probs_t(uint32_t* s, uint32_t* pk, uint32_t nl, uint64_t c2, int e0) {
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const int e = e0 + i;
    const uint4 l4 = ld_shared_v4(nl + 4 * e);
    const uint64_t x0 = fma2(f2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2,
                             f2(__uint_as_float(l4.x), __uint_as_float(l4.y)));
    const uint64_t x1 = fma2(f2(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])), c2,
                             f2(__uint_as_float(l4.z), __uint_as_float(l4.w)));
    const float p0 = ex2(f2lo(x0)), p1 = ex2(f2hi(x0)), p2 = ex2(f2lo(x1)), p3 = ex2(f2hi(x1));
    s[e] = __float_as_uint(p0);
    s[e + 1] = __float_as_uint(p1);
    s[e + 2] = __float_as_uint(p2);
    s[e + 3] = __float_as_uint(p3);
    pk[i / 2] = pack_bf16x2(p0, p1);
    pk[i / 2 + 1] = pack_bf16x2(p2, p3);
  }
}
// dS^T = P^T (dP^T - delta) of the same, from dP^T in d, as bf16.  nd: -delta of the 64 queries.
__device__ __forceinline__ void dprobs_t(const uint32_t* s, const uint32_t* d, uint32_t* pk, uint32_t nd, int e0) {
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const int e = e0 + i;
    const uint4 l4 = ld_shared_v4(nd + 4 * e);
    const uint64_t x0 = mul2(add2(f2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])),
                                  f2(__uint_as_float(l4.x), __uint_as_float(l4.y))),
                             f2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])));
    const uint64_t x1 = mul2(add2(f2(__uint_as_float(d[e + 2]), __uint_as_float(d[e + 3])),
                                  f2(__uint_as_float(l4.z), __uint_as_float(l4.w))),
                             f2(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])));
    pk[i / 2] = pack_bf16x2(f2lo(x0), f2hi(x0));
    pk[i / 2 + 1] = pack_bf16x2(f2lo(x1), f2hi(x1));
  }
}

// ---------------------------------------------------------------- kv items: dK and dV
// Per step n (one query tile of one head):
//   MMA warps    S^T = K Q^T | dP^T = V dO^T, and once the elementwise warps have written P^T and
//                dS^T (bf16, over S^T and dP^T):  dV += P^T dO,  dK += dS^T Q.  One warp issues
//                dV_n, S_n+1, the other dK_n, dP_n+1: the tensor pipe has the products of one
//                step's P while dS is computed, and those of dS while the next P is; and while
//                one warp waits (150 to 240 clocks a wait, done or not), the other issues.
//   elementwise  a thread has key row = TMEM lane, 64 of the tile's 128 queries (warps 0-3 the
//                first half, 4-7 the second).
template <int D, bool VARLEN, bool SPLIT>
__device__ __forceinline__ void kv_items(const BwdParams& p, const Shared& sh, const CUtensorMap* tm_q,
                                         const CUtensorMap* tm_do, const CUtensorMap* tm_k, const CUtensorMap* tm_v) {
  using C = BwdCfg<D>;
  constexpr int NQ = C::NQ, ND = C::ND;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const KernelCtl& ctl = p.ctl;
  const Abort& ab = sh.ab;
  constexpr int NO = C::NOWN;
  const uint32_t bar_k = sh.bars, bar_v = bar_k + 8 * NO, bar_ke = bar_v + 8 * NO, bar_ve = bar_ke + 8 * NO;
  const uint32_t bar_q = bar_ve + 8 * NO, bar_qe = bar_q + 8 * NQ, bar_do = bar_qe + 8 * NQ;
  const uint32_t bar_s = bar_do + 8 * C::ND, bar_dp = bar_s + 8, bar_p = bar_dp + 8, bar_ds = bar_p + 16;
  const uint32_t bar_acc = bar_ds + 16, bar_acce = bar_acc + 8, bar_drain = bar_acce + 8;
  const uint32_t bar_si = bar_drain + 8;  // [step % 2] the next step's S has been issued
  // what an MMA of a tile waits for: ragged, the tile's clearing
  const uint32_t bar_qc = VARLEN ? bar_si + 16 : bar_q, bar_doc = VARLEN ? bar_qc + 8 * NQ : bar_do;
  const uint32_t sb = sh.base;

  if (warp == kLoader) {
    if (lane == 0) {
      int n = 0, filled = 0;  // steps and items with steps so far
      int in_flight_k = 0, in_flight_q = 0, in_flight_do = 0;
      bool ok = true;
      Cursor cur{-1, 0, 0};
      // The first item is the CTA's own, the others come from the counter: fetched when the loads of
      // the item before are out (any earlier, and long items go to CTAs that are not done), but before
      // the loads of a short one, since the answer takes as long as such an item.
      long long idx = blockIdx.x;
      for (int i = 0; ok; ++i) {
        const Item it = make_item<true, VARLEN, SPLIT>(p, idx, cur);
        if (!(ok = ring_put(sh.items, i, it, ctl, ab)) || it.n == -1) break;
        if (it.n <= kShortItem) idx = static_cast<long long>(gridDim.x) + atomicAdd(p.counters, 1u);
        int g = it.g, t = it.t;  // plane of the group, tile
        for (int j = 0; j < it.n; ++j, ++n) {
          const int qs = n % NQ, ds = n % ND;
          if (j == 0) {
            const int o = filled % NO;
            if (filled >= NO && !(ok = mbar_wait(bar_ke + 8 * o, (filled / NO - 1) & 1, ctl, ab))) break;
            mbar_expect_tx(bar_k + 8 * o, C::TILE_BYTES);
            load_tile<D, VARLEN>(sb + C::K_OFF + o * C::TILE_BYTES, tm_k, it.plane, it.kb + it.row0, bar_k + 8 * o);
            in_flight_k = filled + 1;
          }
          if (n >= NQ && !(ok = mbar_wait(bar_qe + 8 * qs, (n / NQ - 1) & 1, ctl, ab))) break;
          if (ctl.inject == 4 && n == 1) break;  // test hook: never load this tile
          mbar_expect_tx(bar_q + 8 * qs, C::TILE_BYTES);
          load_q_tile<D, VARLEN>(sb + C::QR_OFF + qs * C::TILE_BYTES, tm_q, it.other + g, it.qb, t * kTile, p.lg, bar_q + 8 * qs);
          in_flight_q = n + 1;
          if (j == 0) {
            const int o = filled % NO;
            if (filled >= NO && !(ok = mbar_wait(bar_ve + 8 * o, (filled / NO - 1) & 1, ctl, ab))) break;
            mbar_expect_tx(bar_v + 8 * o, C::TILE_BYTES);
            load_tile<D, VARLEN>(sb + C::V_OFF + o * C::TILE_BYTES, tm_v, it.plane, it.kb + it.row0, bar_v + 8 * o);
            ++filled;
          }
          // dV and dK of step n - ND are done, and so are dP, issued before dK, and the reading of the
          // step's row statistics
          if (n >= ND && !(ok = mbar_wait(bar_qe + 8 * ((n - ND) % NQ), (n - ND) / NQ & 1, ctl, ab))) break;
          mbar_expect_tx(bar_do + 8 * ds, C::TILE_BYTES + kStat * 4);
          load_q_tile<D, VARLEN>(sb + C::DOR_OFF + ds * C::TILE_BYTES, tm_do, it.other + g, it.qb, t * kTile, p.lg, bar_do + 8 * ds);
          bulk_g2s(sb + C::ST_OFF + ds * (kStat * 4),
                   p.stats + (static_cast<size_t>(it.other + g) * p.stat_tiles + it.stat0 + t) * kStat, kStat * 4,
                   bar_do + 8 * ds);
          in_flight_do = n + 1;
          if (++t == it.t0 + it.nt) ++g, t = it.t0;
        }
        if (it.n > kShortItem) idx = static_cast<long long>(gridDim.x) + atomicAdd(p.counters, 1u);
        if (ctl.inject == 4 && n == 1) break;
      }
      // copies still in flight must land before the shared memory is used for anything else
      for (int m = max(0, in_flight_k - NO); m < in_flight_k; ++m) mbar_wait(bar_k + 8 * (m % NO), (m / NO) & 1, ctl, sh.drain_ab);
      for (int m = max(0, filled - NO); m < filled; ++m) mbar_wait(bar_v + 8 * (m % NO), (m / NO) & 1, ctl, sh.drain_ab);
      for (int m = max(0, in_flight_q - NQ); m < in_flight_q; ++m) mbar_wait(bar_q + 8 * (m % NQ), (m / NQ) & 1, ctl, sh.drain_ab);
      for (int m = max(0, in_flight_do - ND); m < in_flight_do; ++m)
        mbar_wait(bar_do + 8 * (m % ND), (m / ND) & 1, ctl, sh.drain_ab);
    }
    __syncwarp();
  } else if (VARLEN && warp == kCleaner) {
    int n = 0;
    bool ok = true;
    Item it;
    for (int i = 0; ok; ++i) {
      if (!(ok = ring_get(sh.items, i, it, ctl, ab)) || it.n == -1) break;
      int t = it.t;
      for (int j = 0; ok && j < it.n; ++j, ++n) {
        const int rows = (it.sq << p.lg) - t * kTile;  // of the step's query tile, within the sequence
        if (++t == it.t0 + it.nt) t = it.t0;
        ok = clean_tile<D, NQ>(sb + C::QR_OFF, bar_q, bar_qc, n, rows, ctl, ab) &&
             clean_tile<D, ND>(sb + C::DOR_OFF, bar_do, bar_doc, n, rows, ctl, ab);
      }
    }
  } else if (warp >= kMma0) {
    const bool first = warp == kMma0;  // S and dV, or dP and dK
    const uint32_t tm = sh.tmem;
    int n = 0, filled = 0;
    bool ok = true;
    Item it;
    for (int i = 0; ok; ++i) {
      if (!(ok = ring_get(sh.items, i, it, ctl, ab)) || it.n == -1) break;
      if (it.n <= 0) continue;
      const int own = filled % NO, own_ph = filled / NO & 1;
      auto q_tile = [&](int j) { return sb + C::QR_OFF + (n + j) % NQ * C::TILE_BYTES; };
      auto do_tile = [&](int j) { return sb + C::DOR_OFF + (n + j) % ND * C::TILE_BYTES; };
      if (first) {
        auto scores = [&](int j) {
          issue_scores<D>(tm + C::S_COL, sb + C::K_OFF + own * C::TILE_BYTES, q_tile(j));
          tc_commit_el(bar_s);
          if (j + 1 == it.n) tc_commit_el(bar_ke + 8 * own);
        };
        if (!(ok = wait_two(bar_k + 8 * own, own_ph, bar_qc + 8 * (n % NQ), n / NQ & 1, ctl, ab))) break;
        scores(0);
        // the gradients of the item before must have been read out
        if (filled > 0 && !(ok = mbar_wait_warp(bar_acce, (filled - 1) & 1, ctl, ab))) break;
        for (int j = 0; j < it.n; ++j) {
          const int m = n + j;
          const uint32_t par = m & 1;
          const bool more = j + 1 < it.n;
          // (dense: P was made with statistics that came with the dO tile)
          const uint32_t bd = VARLEN ? bar_doc + 8 * (m % ND) : bar_p, pd = VARLEN ? m / ND & 1 : par;
          if (!(ok = wait_three(bar_p, par, bd, pd, more ? bar_qc + 8 * ((m + 1) % NQ) : bar_p, more ? (m + 1) / NQ & 1 : par, ctl,
                                ab)))
            break;
          tc_fence_after();
          issue_grad_chunks<D>(tm + C::DV_COL, tm + C::S_COL, do_tile(j), 0, j > 0);
          if (!(ok = mbar_wait_warp(bar_p + 8, par, ctl, ab))) break;
          tc_fence_after();
          issue_grad_chunks<D>(tm + C::DV_COL, tm + C::S_COL, do_tile(j), 1, true);
          if (more) scores(j + 1);
          if (lane == 0) mbar_arrive(bar_si + 8 * (m & 1));
          __syncwarp();
          tc_commit_el(bar_qe + 8 * (m % NQ));
        }
      } else {
        auto dprobs = [&](int j) {
          issue_scores<D>(tm + C::DP_COL, sb + C::V_OFF + own * C::TILE_BYTES, do_tile(j));
          tc_commit_el(bar_dp);
          if (j + 1 == it.n) tc_commit_el(bar_ve + 8 * own);
        };
        if (!(ok = wait_two(bar_v + 8 * own, own_ph, bar_doc + 8 * (n % ND), n / ND & 1, ctl, ab))) break;
        dprobs(0);
        if (filled > 0 && !(ok = mbar_wait_warp(bar_acce, (filled - 1) & 1, ctl, ab))) break;
        for (int j = 0; j < it.n; ++j) {
          const int m = n + j;
          const uint32_t par = m & 1;
          const bool more = j + 1 < it.n;
          // dK goes behind the next S in the tensor pipe: the next P waits for that S
          if (!(ok = wait_three(bar_ds, par, bar_si + 8 * (m & 1), m >> 1 & 1, more ? bar_doc + 8 * ((m + 1) % ND) : bar_ds,
                                more ? (m + 1) / ND & 1 : par, ctl, ab)))
            break;
          tc_fence_after();
          issue_grad_chunks<D>(tm + C::DK_COL, tm + C::DP_COL, q_tile(j), 0, j > 0);
          if (!(ok = mbar_wait_warp(bar_ds + 8, par, ctl, ab))) break;
          tc_fence_after();
          issue_grad_chunks<D>(tm + C::DK_COL, tm + C::DP_COL, q_tile(j), 1, true);
          tc_commit_el(bar_qe + 8 * (m % NQ));
          if (more) dprobs(j + 1);
        }
      }
      if (!ok) break;
      tc_commit_el(bar_acc);
      n += it.n;
      ++filled;
    }
    // every MMA issued above is done before TMEM or shared memory is used for anything else
    tc_commit_el(bar_drain);
    mbar_wait_warp(bar_drain, 0, ctl, sh.drain_ab);
  } else {
    const int half = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t tm = sh.tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_tm = tm + C::S_COL + 64 * half, dp_tm = tm + C::DP_COL + 64 * half;
    const uint64_t c2 = f2(p.c, p.c);
    int n = 0, filled = 0;
    bool ok = true, pending = false;
    Finish fin{};
    // An item's gradients are stored after the first step of the next one, whose products the MMA
    // warps issue meanwhile.
    auto finish = [&]() -> bool {
      if (!mbar_wait_warp(bar_acc, filled & 1, ctl, ab)) return false;
      tc_fence_after();
      constexpr size_t step = 2 * D * kTile;  // dV and dK of a share: D x 128 floats each
      finish_rows<D, SPLIT>(fin, tm + (half ? C::DK_COL : C::DV_COL), half ? p.scale : 1.f, p.wide, bar_acce,
                     p.partial + static_cast<size_t>(fin.id) * p.kv_split * step + half * (D * kTile) + 4 * r, step,
                     p.counters + 64 + static_cast<size_t>(fin.id) * kEltWarps + warp);
      ++filled;
      pending = false;
      return true;
    };
    Item it;
    for (int i = 0; ok; ++i) {
      if (!(ok = ring_get(sh.items, i, it, ctl, ab)) || it.n == -1) break;
      const int off = it.skv - it.sq, key = it.row0 + r;
      int t = it.t;
      for (int j = 0; j < it.n; ++j, ++n) {
        const int slot = n % ND;
        const uint32_t st = sb + C::ST_OFF + slot * (kStat * 4) + 256 * half;
        const int q0 = t * kTile + 64 * half;
        if (++t == it.t0 + it.nt) t = it.t0;
        // (the statistics come with the dO tile)
        if (!(ok = wait_two(bar_s, n & 1, bar_do + 8 * slot, n / ND & 1, ctl, ab))) break;
        tc_fence_after();
        uint32_t s[64];
        ld64(s_tm, s);
        if (p.causal && (q0 >> p.lg) + off < it.row0 + kTile - 1) {
          // queries from key - off on see this key
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const uint32_t hidden = low_bits((max(0, min(it.sq, key - off)) << p.lg) - q0 - 32 * g);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (hidden & (1u << e)) s[32 * g + e] = __float_as_uint(-INFINITY);
          }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t pk[16];
          probs_t(s, pk, st, c2, 32 * c);
          tmem_st16(s_tm + 16 * c, pk);
          tmem_wait_st();
          tc_fence_before();
          warp_arrive(bar_p + 8 * c);
          if (c == 0) reg_fence32(s + 32);  // keeps the second chunk's arithmetic behind the first's hand-over
        }
        if (!(ok = mbar_wait_warp(bar_dp, n & 1, ctl, ab))) break;
        tc_fence_after();
        uint32_t d[64];
        ld64(dp_tm, d);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t pk[16];
          dprobs_t(s, d, pk, st + kTile * 4, 32 * c);
          tmem_st16(dp_tm + 16 * c, pk);
          tmem_wait_st();
          tc_fence_before();
          warp_arrive(bar_ds + 8 * c);
          if (c == 0) reg_fence32(d + 32);
        }
        if (pending && !(ok = finish())) break;
      }
      if (!ok) break;
      // warps 0-3 store dV, warps 4-7 dK
      const bool store = key < it.skv;
      const long long row = VARLEN ? static_cast<long long>(it.kb + key) * p.Hkv + it.plane
                                   : static_cast<long long>(it.plane) * p.Skv + key;
      __nv_bfloat16* const at = (half ? p.dk : p.dv) + (store ? row : 0) * D;
      if (it.n > 0) {
        fin = {at, SPLIT ? it.id : 0, SPLIT ? static_cast<uint32_t>(it.shares | it.share << 8 | store << 16) : store << 16};
        pending = true;
      } else if (it.n == 0 && store) {  // (another item's may be pending)
        store_zeros<D>(at);
      }
    }
    if (ok && pending) finish();
  }
}

// ---------------------------------------------------------------- query items: dQ
// Per step n (one kv tile):  S = Q K^T,  dP = dO V^T,  dQ += dS K.  P never leaves the registers;
// dS has two TMEM buffers of its own, so S and dP of the next step are issued as soon as the
// elementwise warps have loaded this step's.  They may therefore finish the next dS before the MMA
// warp has looked at this one: each buffer has barriers of its own, and is written again once dQ of
// two steps before is done.
template <int D, bool VARLEN, bool SPLIT>
__device__ __forceinline__ void q_items(const BwdParams& p, const Shared& sh, const CUtensorMap* tm_q,
                                        const CUtensorMap* tm_do, const CUtensorMap* tm_k, const CUtensorMap* tm_v) {
  using C = BwdCfg<D>;
  constexpr int NK = C::NK, NV = C::NV;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const KernelCtl& ctl = p.ctl;
  const Abort& ab = sh.ab;
  constexpr int NO = C::NOWN;
  const uint32_t bar_q = sh.bars, bar_do = bar_q + 8 * NO, bar_qe = bar_do + 8 * NO, bar_doe = bar_qe + 8 * NO;
  const uint32_t bar_k = bar_doe + 8 * NO, bar_ke = bar_k + 8 * NK, bar_v = bar_ke + 8 * NK;
  // bar_dpf[step % NV]: dP is in registers, and so V's slot is free
  const uint32_t bar_s = bar_v + 8 * NV, bar_dp = bar_s + 8, bar_sf = bar_dp + 8, bar_dpf = bar_sf + 8;
  const uint32_t bar_ds = bar_dpf + 8 * NV, bar_acc = bar_ds + 16, bar_acce = bar_acc + 8, bar_drain = bar_acce + 8;
  const uint32_t bar_kc = VARLEN ? bar_drain + 8 : bar_k, bar_vc = VARLEN ? bar_kc + 8 * NK : bar_v;  // as in kv_items
  const uint32_t sb = sh.base;

  if (warp == kLoader) {
    if (lane == 0) {
      int n = 0, filled = 0;
      int in_flight_q = 0, in_flight_k = 0, in_flight_v = 0;
      bool ok = true;
      Cursor cur{-1, 0, 0};
      unsigned int idx = atomicAdd(p.counters + 1, 1u);
      for (int i = 0; ok; ++i) {
        const Item it = make_item<false, VARLEN, SPLIT>(p, idx, cur);
        if (!(ok = ring_put(sh.items, i, it, ctl, ab)) || it.n == -1) break;
        if (it.n <= kShortItem) idx = atomicAdd(p.counters + 1, 1u);
        for (int j = 0; j < it.n; ++j, ++n) {
          if (j == 0) {
            const int o = filled % NO;
            if (filled >= NO && !(ok = mbar_wait(bar_qe + 8 * o, (filled / NO - 1) & 1, ctl, ab))) break;
            mbar_expect_tx(bar_q + 8 * o, C::TILE_BYTES);
            load_q_tile<D, VARLEN>(sb + C::Q_OFF + o * C::TILE_BYTES, tm_q, it.plane, it.qb, it.row0, p.lg, bar_q + 8 * o);
            in_flight_q = filled + 1;
          }
          const int ks = n % NK, kp = n / NK, vs = n % NV, vp = n / NV;
          if (kp > 0 && !(ok = mbar_wait(bar_ke + 8 * ks, (kp - 1) & 1, ctl, ab))) break;
          mbar_expect_tx(bar_k + 8 * ks, C::TILE_BYTES);
          load_tile<D, VARLEN>(sb + C::KR_OFF + ks * C::TILE_BYTES, tm_k, it.other, it.kb + (it.t + j) * kTile, bar_k + 8 * ks);
          in_flight_k = n + 1;
          if (j == 0) {
            const int o = filled % NO;
            if (filled >= NO && !(ok = mbar_wait(bar_doe + 8 * o, (filled / NO - 1) & 1, ctl, ab))) break;
            mbar_expect_tx(bar_do + 8 * o, C::TILE_BYTES);
            load_q_tile<D, VARLEN>(sb + C::DO_OFF + o * C::TILE_BYTES, tm_do, it.plane, it.qb, it.row0, p.lg, bar_do + 8 * o);
            ++filled;
          }
          if (vp > 0 && !(ok = mbar_wait(bar_dpf + 8 * vs, (vp - 1) & 1, ctl, ab))) break;
          mbar_expect_tx(bar_v + 8 * vs, C::TILE_BYTES);
          load_tile<D, VARLEN>(sb + C::VR_OFF + vs * C::TILE_BYTES, tm_v, it.other, it.kb + (it.t + j) * kTile, bar_v + 8 * vs);
          in_flight_v = n + 1;
        }
        if (it.n > kShortItem) idx = atomicAdd(p.counters + 1, 1u);
      }
      for (int m = max(0, in_flight_q - NO); m < in_flight_q; ++m) mbar_wait(bar_q + 8 * (m % NO), (m / NO) & 1, ctl, sh.drain_ab);
      for (int m = max(0, filled - NO); m < filled; ++m) mbar_wait(bar_do + 8 * (m % NO), (m / NO) & 1, ctl, sh.drain_ab);
      for (int m = max(0, in_flight_k - NK); m < in_flight_k; ++m) mbar_wait(bar_k + 8 * (m % NK), (m / NK) & 1, ctl, sh.drain_ab);
      for (int m = max(0, in_flight_v - NV); m < in_flight_v; ++m) mbar_wait(bar_v + 8 * (m % NV), (m / NV) & 1, ctl, sh.drain_ab);
    }
    __syncwarp();
  } else if (VARLEN && warp == kCleaner) {
    int n = 0;
    bool ok = true;
    Item it;
    for (int i = 0; ok; ++i) {
      if (!(ok = ring_get(sh.items, i, it, ctl, ab)) || it.n == -1) break;
      for (int j = 0; ok && j < it.n; ++j, ++n) {
        const int rows = it.skv - (it.t + j) * kTile;
        ok = clean_tile<D, NK>(sb + C::KR_OFF, bar_k, bar_kc, n, rows, ctl, ab) &&
             clean_tile<D, NV>(sb + C::VR_OFF, bar_v, bar_vc, n, rows, ctl, ab);
      }
    }
  } else if (warp >= kMma0) {
    const bool first = warp == kMma0;  // S and dP, or dQ
    const uint32_t tm = sh.tmem;
    int n = 0, filled = 0;
    bool ok = true;
    Item it;
    for (int i = 0; ok; ++i) {
      if (!(ok = ring_get(sh.items, i, it, ctl, ab)) || it.n == -1) break;
      if (it.n <= 0) continue;
      const int own = filled % NO, own_ph = filled / NO & 1;
      auto k_tile = [&](int j) { return sb + C::KR_OFF + (n + j) % NK * C::TILE_BYTES; };
      if (first) {
        for (int j = 0; j < it.n; ++j) {
          const int m = n + j, ks = m % NK, vs = m % NV;
          const uint32_t bk = bar_kc + 8 * ks, pk = m / NK & 1, bv = bar_vc + 8 * vs, pv = m / NV & 1;
          const uint32_t v = sb + C::VR_OFF + vs * C::TILE_BYTES;
          // the tiles, and S and dP of the step before in registers
          if (j == 0 && !(ok = mbar_wait_warp(bar_q + 8 * own, own_ph, ctl, ab))) break;
          if (!(ok = wait_two(bk, pk, m > 0 ? bar_sf : bk, m > 0 ? (m - 1) & 1 : pk, ctl, ab))) break;
          tc_fence_after();
          issue_scores<D>(tm + C::S_COL, sb + C::Q_OFF + own * C::TILE_BYTES, k_tile(j));
          tc_commit_el(bar_s);
          if (j + 1 == it.n) tc_commit_el(bar_qe + 8 * own);
          if (j == 0 && !(ok = mbar_wait_warp(bar_do + 8 * own, own_ph, ctl, ab))) break;
          if (!(ok = wait_two(bv, pv, m > 0 ? bar_dpf + 8 * ((m - 1) % NV) : bv, m > 0 ? (m - 1) / NV & 1 : pv, ctl, ab))) break;
          tc_fence_after();
          issue_scores<D>(tm + C::DP_COL, sb + C::DO_OFF + own * C::TILE_BYTES, v);
          tc_commit_el(bar_dp);
          if (j + 1 == it.n) tc_commit_el(bar_doe + 8 * own);
        }
      } else {
        // the gradient of the item before must have been read out
        if (filled > 0 && !(ok = mbar_wait_warp(bar_acce, (filled - 1) & 1, ctl, ab))) break;
        for (int j = 0; j < it.n; ++j) {
          const int m = n + j;
          if (!(ok = mbar_wait_warp(bar_ds + 8 * (m & 1), m >> 1 & 1, ctl, ab))) break;
          tc_fence_after();
          for (int h = 0; h < 2; ++h)
            issue_grad_half<D>(tm + C::DQ_COL, tm + C::DS_COL + 64 * (m & 1) + 32 * h, k_tile(j), h, j > 0 || h > 0);
          tc_commit_el(bar_ke + 8 * (m % NK));
        }
        if (ok) tc_commit_el(bar_acc);
      }
      if (!ok) break;
      n += it.n;
      ++filled;
    }
    tc_commit_el(bar_drain);
    mbar_wait_warp(bar_drain, 0, ctl, sh.drain_ab);
  } else {
    const int half = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t tm = sh.tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint64_t c2 = f2(p.c, p.c);
    int n = 0, filled = 0;
    bool ok = true, pending = false;
    Finish fin{};
    auto finish = [&]() -> bool {  // as in kv_items
      if (!mbar_wait_warp(bar_acc, filled & 1, ctl, ab)) return false;
      tc_fence_after();
      constexpr size_t step = D * kTile;
      const size_t kv_part = p.kv_split > 1 ? static_cast<size_t>(p.kv_slots) * p.kv_split * 2 * step : 0;
      finish_rows<D / 2, SPLIT>(fin, tm + C::DQ_COL + half * (D / 2), p.scale, p.wide, bar_acce,
                         p.partial + kv_part + static_cast<size_t>(fin.id) * p.q_split * step + half * (D / 2 * kTile) + 4 * r,
                         step, p.counters + 64 + (static_cast<size_t>(p.kv_slots) + fin.id) * kEltWarps + warp);
      ++filled;
      pending = false;
      return true;
    };
    Item it;
    for (int i = 0; ok; ++i) {
      if (!(ok = ring_get(sh.items, i, it, ctl, ab)) || it.n == -1) break;
      const int q = (it.row0 + r) >> p.lg;
      const float* st = p.stats + (static_cast<size_t>(it.plane) * p.stat_tiles + it.stat0 + it.row0 / kTile) * kStat + r;
      const float nl = __ldg(st), nd = __ldg(st + kTile);
      const uint64_t nl2 = f2(nl, nl), nd2 = f2(nd, nd);
      const int limit = p.causal ? min(it.skv, q + it.skv - it.sq + 1) : it.skv;  // keys [0, limit) are seen
      for (int j = 0; j < it.n; ++j, ++n) {
        const int k0 = (it.t + j) * kTile + 64 * half;
        if (!(ok = mbar_wait_warp(bar_s, n & 1, ctl, ab))) break;
        tc_fence_after();
        uint32_t s[64];
        ld64(tm + C::S_COL + 64 * half, s);
        tc_fence_before();
        warp_arrive(bar_sf);
        if (k0 + 64 > limit) {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const uint32_t visible = low_bits(limit - k0 - 32 * g);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(visible & (1u << e))) s[32 * g + e] = __float_as_uint(-INFINITY);
          }
        }
#pragma unroll
        for (int e = 0; e < 64; e += 2) {
          const uint64_t x = fma2(f2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2, nl2);
          s[e] = __float_as_uint(ex2(f2lo(x)));
          s[e + 1] = __float_as_uint(ex2(f2hi(x)));
        }
        // ... and dQ of two steps before is done with this step's buffer of dS
        const int m2 = n - 2;
        if (!(ok = wait_two(bar_dp, n & 1, m2 >= 0 ? bar_ke + 8 * (m2 % NK) : bar_dp, m2 >= 0 ? m2 / NK & 1 : n & 1, ctl, ab))) break;
        tc_fence_after();
        uint32_t d[64], pk[32];
        ld64(tm + C::DP_COL + 64 * half, d);
        tc_fence_before();
        warp_arrive(bar_dpf + 8 * (n % NV));
#pragma unroll
        for (int e = 0; e < 64; e += 2) {
          const uint64_t x = mul2(add2(f2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), nd2),
                                  f2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])));
          pk[e / 2] = pack_bf16x2(f2lo(x), f2hi(x));
        }
        tmem_st32(tm + C::DS_COL + 64 * (n & 1) + 32 * half, pk);
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(bar_ds + 8 * (n & 1));
        if (pending && !(ok = finish())) break;
      }
      if (!ok) break;
      const bool store = q < it.sq;
      const long long head = (static_cast<long long>(it.plane) << p.lg) + ((it.row0 + r) & ((1 << p.lg) - 1));
      const long long row = VARLEN ? static_cast<long long>(it.qb + q) * p.Hq + head : head * p.Sq + q;
      __nv_bfloat16* const at = p.dq + (store ? row : 0) * D + half * (D / 2);
      if (it.n > 0) {
        fin = {at, SPLIT ? it.id : 0, SPLIT ? static_cast<uint32_t>(it.shares | it.share << 8 | store << 16) : store << 16};
        pending = true;
      } else if (it.n == 0 && store) {
        store_zeros<D / 2>(at);
      }
    }
    if (ok && pending) finish();
  }
}

template <int D, bool VARLEN, bool SPLIT>
__global__ void __launch_bounds__(kThreads<VARLEN>, 1)
    attn_bwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do,
                    const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const BwdParams p) {
  using C = BwdCfg<D>;
  // 128-byte-swizzled tiles start at 1024-byte boundaries.  The tiles leave no room to round the
  // base up (D = 128): it is aligned by declaration, and a launch where it is not does nothing but
  // say so.
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  if (sbase & 1023u) {
    if (threadIdx.x == 0) atomicOr(p.ctl.err, kErrTimeout);
    return;
  }
  const int warp = threadIdx.x >> 5;
  uint32_t* tmem_ptr = reinterpret_cast<uint32_t*>(smem + C::TMEM_PTR_OFF);
  volatile int* flags = reinterpret_cast<volatile int*>(smem + C::ABORT_OFF);

  // Barriers of the kv items and of the query items: [0, kv) and [kv, ..), each with an item ring.
  constexpr int kKvBars = 4 * C::NOWN + 3 * C::NQ + 2 * C::ND + 11, kQBars = 4 * C::NOWN + 3 * C::NK + 3 * C::NV + 8;
  static_assert(kKvBars + kQBars + 8 <= C::NBAR, "barrier space");
  const uint32_t bars = sbase + C::BAR_OFF;
  const uint32_t kv_bars = bars, q_bars = bars + 8 * kKvBars, ring_bars = q_bars + 8 * kQBars;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kKvBars + kQBars; ++i) mbar_init(bars + 8 * i, 1);
    // the elementwise warps arrive on these
    const uint32_t bar_p = kv_bars + 8 * (4 * C::NOWN + 2 * C::NQ + C::ND + 2);
    for (int i = 0; i < 4; ++i) mbar_init(bar_p + 8 * i, kEltWarps);  // p[2], ds[2]
    mbar_init(bar_p + 8 * 4, 2);                                      // acc: both MMA warps
    mbar_init(bar_p + 8 * 5, kEltWarps);                              // acc_empty
    mbar_init(bar_p + 8 * 6, 2);                                      // drain: both MMA warps
    for (int i = 0; i < C::NQ; ++i) mbar_init(kv_bars + 8 * (4 * C::NOWN + C::NQ + i), 2);  // q_empty: dV and dK
    const uint32_t bar_sf = q_bars + 8 * (4 * C::NOWN + 2 * C::NK + C::NV + 2);
    for (int i = 0; i < 1 + C::NV + 2; ++i) mbar_init(bar_sf + 8 * i, kEltWarps);  // S free, dP free[NV], ds[2]
    const uint32_t bar_qacce = bar_sf + 8 * (1 + C::NV + 3);
    mbar_init(bar_qacce, kEltWarps);
    mbar_init(bar_qacce + 8, 2);  // drain: both MMA warps
    for (int i = 0; i < 2; ++i) {  // two rings: full[2], empty[2]
      mbar_init(ring_bars + 32 * i, 1);
      mbar_init(ring_bars + 32 * i + 8, 1);
      mbar_init(ring_bars + 32 * i + 16, kItemReaders<VARLEN>);
      mbar_init(ring_bars + 32 * i + 24, kItemReaders<VARLEN>);
    }
    flags[0] = 0;
    flags[1] = 0;
    fence_barrier_init();
  }
  if (warp == kMma0) tmem_alloc(smem_u32(tmem_ptr), 512);
  if (threadIdx.x == kLoader * 32) {
    prefetch_tensormap(&tm_q);
    prefetch_tensormap(&tm_do);
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // the row statistics and the zeroed counters come from the kernel before this one
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  Item* rec = reinterpret_cast<Item*>(smem + C::ITEM_OFF);
  static_assert(sizeof(Item) * 2 <= 128, "item records");
  Shared sh{sbase, kv_bars, *tmem_ptr, {ring_bars, ring_bars + 16, rec}, {flags}, {flags + 1}};
  kv_items<D, VARLEN, SPLIT>(p, sh, &tm_q, &tm_do, &tm_k, &tm_v);
  // The rings' shared memory and TMEM change hands: every role is done, its copies have landed
  // and its MMAs are complete.
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (flags[0] == 0 && flags[1] == 0) {
    sh.bars = q_bars;
    sh.items.full = ring_bars + 32;
    sh.items.empty = ring_bars + 48;
    q_items<D, VARLEN, SPLIT>(p, sh, &tm_q, &tm_do, &tm_k, &tm_v);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kMma0) {
    tc_fence_after();
    tmem_dealloc(*tmem_ptr, 512);
  }
}

// ---------------------------------------------------------------- row statistics
// kTile / kRowsPerBlock blocks per tile of 128 rows of a query plane: -LSE log2(e) and dLSE - dO . O for each row.
// Rows past the end, and rows whose LSE is -inf, get -inf and 0, so P = 0 and dS = 0 whatever their dLSE
// and O are.  A ragged sequence's rows are counted from its first query that sees a key; dQ of those before it
// becomes zeros here.  Bound by reading dO and O once; D / 8 lanes of 16 bytes take a row.
template <int D, bool VARLEN>
__global__ void __launch_bounds__(kRowThreads)
    attn_bwd_rows_kernel(const __nv_bfloat16* dout, const __nv_bfloat16* o, const float* lse, const float* dlse, float* stats,
                         unsigned int* counters, int n_counters, int B, int H, int Sq, int lg, int stat_tiles,
                         const int32_t* cu_q, const int32_t* cu_k, int causal, __nv_bfloat16* dq) {
  constexpr int LPR = D / 8, PASSES = kRowsPerBlock * LPR / kRowThreads;  // lanes per row
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  for (int i = static_cast<int>(blockIdx.x) * kRowThreads + static_cast<int>(threadIdx.x); i < n_counters;
       i += static_cast<int>(gridDim.x) * kRowThreads)
    counters[i] = 0;
  const int at_tile = static_cast<int>(blockIdx.x / (kTile / kRowsPerBlock)), part = static_cast<int>(blockIdx.x % (kTile / kRowsPerBlock));
  const int plane = at_tile / stat_tiles, tile = at_tile % stat_tiles;
  int row0 = tile * kTile, n = Sq, qb = 0, unseen = 0;
  if constexpr (VARLEN) {
    int lo = 0, hi = B - 1;  // the last sequence that starts at this tile or before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (ragged_stat0(cu_q, mid, lg) <= tile)
        lo = mid;
      else
        hi = mid - 1;
    }
    qb = cu_q[lo];
    n = cu_q[lo + 1] - qb;
    row0 = (tile - ragged_stat0(cu_q, lo, lg)) * kTile;
    if (row0 < 0 || row0 >= n << lg) return;  // a tile of no sequence
    unseen = unseen_queries(n, cu_k[lo + 1] - cu_k[lo], causal);
    n -= unseen;
  }
  const int l = threadIdx.x % LPR, r0 = part * kRowsPerBlock + static_cast<int>(threadIdx.x) / LPR;
  float* st = stats + static_cast<size_t>(at_tile) * kStat;
  uint4 x[PASSES], y[PASSES];
  float nl[PASSES], dl[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = row0 + r0 + i * (kRowThreads / LPR), query = row >> lg;
    const long long head = (static_cast<long long>(plane) << lg) + (row & ((1 << lg) - 1));
    const long long at = VARLEN ? static_cast<long long>(qb + unseen + query) * H + head : head * Sq + query;
    if (VARLEN && query < unseen)
      *reinterpret_cast<uint4*>(dq + (static_cast<long long>(qb + query) * H + head) * D + 8 * l) = make_uint4(0, 0, 0, 0);
    x[i] = y[i] = make_uint4(0, 0, 0, 0);
    nl[i] = -INFINITY;
    dl[i] = 0.f;
    if (query < n) {
      x[i] = *reinterpret_cast<const uint4*>(dout + at * D + 8 * l);
      y[i] = *reinterpret_cast<const uint4*>(o + at * D + 8 * l);
      if (l == 0) {
        const long long s = VARLEN ? head * Sq + qb + unseen + query : at;
        const float e = lse[s];
        nl[i] = e == -INFINITY ? -INFINITY : -e * kLog2e;
        if (dlse) dl[i] = dlse[s];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const uint32_t xw[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, yw[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) a = fmaf(bf16hi(xw[w]), bf16hi(yw[w]), fmaf(bf16lo(xw[w]), bf16lo(yw[w]), a));
#pragma unroll
    for (int m = LPR / 2; m > 0; m >>= 1) a += __shfl_xor_sync(0xffffffffu, a, m);
    if (l == 0) {
      const int r = r0 + i * (kRowThreads / LPR);
      st[r] = nl[i];
      st[kTile + r] = nl[i] == -INFINITY ? 0.f : dl[i] - a;
    }
  }
}

// ---------------------------------------------------------------- host side
using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &qres) == cudaSuccess &&
        qres == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(ptr);
  });
  return fn;
}

// 64-column x 128-row boxes of dense planes [planes, rows, D] (innermost first D, rows, planes), or
// of packed tokens [rows, H, D] (D, H, rows).
bool make_map(CUtensorMap* map, const void* base, int D, long long rows, long long planes, bool tokens) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t row = static_cast<cuuint64_t>(D) * 2;
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(tokens ? planes : rows),
                        static_cast<cuuint64_t>(tokens ? rows : planes)};
  cuuint64_t strides[2] = {row, row * dims[1]};
  cuuint32_t box[3] = {64, tokens ? 1u : static_cast<cuuint32_t>(kTile), tokens ? static_cast<cuuint32_t>(kTile) : 1u};
  cuuint32_t estr[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of query planes of 2^lg heads: dense [planes, queries, heads, D] (innermost first D, heads,
// queries, planes), packed tokens [queries, planes, heads, D] (D, heads, planes, queries).
bool make_q_map(CUtensorMap* map, const void* base, int D, long long queries, long long planes, int lg, bool tokens) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t row = static_cast<cuuint64_t>(D) * 2, nq = static_cast<cuuint64_t>(queries);
  const cuuint64_t np = static_cast<cuuint64_t>(planes), heads = 1ull << lg;
  cuuint64_t dims[4] = {static_cast<cuuint64_t>(D), heads, tokens ? np : nq, tokens ? nq : np};
  cuuint64_t strides[3] = {tokens ? row : row * nq, tokens ? row << lg : row, tokens ? (row << lg) * np : (row << lg) * nq};
  const cuuint32_t q = static_cast<cuuint32_t>(kTile >> lg);
  cuuint32_t box[4] = {64, 1u << lg, tokens ? 1u : q, tokens ? q : 1u};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class Kernel, class... Args>
cudaError_t launch(Kernel kernel, int grid, int threads, uint32_t smem, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D, bool VARLEN>
cudaError_t launch_d(const BwdArgs& a, const KernelCtl& ctl, cudaStream_t stream) {
  using C = BwdCfg<D>;
  static PerDeviceOnce configured;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const auto whole = attn_bwd_kernel<D, VARLEN, false>, shared = attn_bwd_kernel<D, VARLEN, true>;
  if (!configured.run(dev, [&] {
        return cudaFuncSetAttribute(whole, cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES) == cudaSuccess &&
               cudaFuncSetAttribute(shared, cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES) == cudaSuccess;
      }))
    return cudaErrorInvalidValue;
  CUtensorMap mq, mdo, mk, mv;
  const int lg = bwd_pack_log2(a.Hq / a.Hkv);
  const long long q_planes = (VARLEN ? a.Hq : static_cast<long long>(a.B) * a.Hq) >> lg;
  const long long kv_planes = VARLEN ? a.Hkv : static_cast<long long>(a.B) * a.Hkv;
  if (!make_q_map(&mq, a.q, D, a.Sq, q_planes, lg, VARLEN) || !make_q_map(&mdo, a.dout, D, a.Sq, q_planes, lg, VARLEN) ||
      !make_map(&mk, a.k, D, a.Skv, kv_planes, VARLEN) || !make_map(&mv, a.v, D, a.Skv, kv_planes, VARLEN))
    return cudaErrorInvalidValue;
  const int stat_tiles = static_cast<int>(bwd_stat_tiles(a.B, a.Sq, lg, VARLEN));
  const BwdPlan plan = bwd_plan(a.B, a.Hq, a.Hkv, a.Sq, a.Skv, D, VARLEN, a.causal != 0, sms);
  unsigned int* counters = static_cast<unsigned int*>(a.workspace);
  float* stats = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + plan.stats_at);
  e = launch(attn_bwd_rows_kernel<D, VARLEN>, static_cast<int>(q_planes * stat_tiles) * (kTile / kRowsPerBlock), kRowThreads, 0, stream,
             static_cast<const __nv_bfloat16*>(a.dout), static_cast<const __nv_bfloat16*>(a.o), a.lse, a.dlse, stats, counters,
             plan.counters, a.B, a.Hq, a.Sq, lg, stat_tiles, a.cu_q, a.cu_k, a.causal,
             static_cast<__nv_bfloat16*>(a.dq));
  if (e != cudaSuccess) return e;
  BwdParams p;
  memset(&p, 0, sizeof(p));
  p.dq = static_cast<__nv_bfloat16*>(a.dq);
  p.dk = static_cast<__nv_bfloat16*>(a.dk);
  p.dv = static_cast<__nv_bfloat16*>(a.dv);
  p.stats = stats;
  p.counters = counters;
  p.partial = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + plan.partial_at);
  p.kv_split = plan.kv_split;
  p.q_split = plan.q_split;
  p.kv_slots = static_cast<int>(plan.kv_items);
  p.B = a.B;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.Sq = a.Sq;
  p.Skv = a.Skv;
  p.causal = a.causal;
  p.wide = ((reinterpret_cast<uintptr_t>(a.dq) | reinterpret_cast<uintptr_t>(a.dk) | reinterpret_cast<uintptr_t>(a.dv)) & 31) == 0;
  p.lg = lg;
  p.c = a.scale * kLog2e;
  p.scale = a.scale;
  p.stat_tiles = stat_tiles;
  p.cu_q = a.cu_q;
  p.cu_k = a.cu_k;
  p.ctl = ctl;
  long long items;
  if constexpr (VARLEN) {
    p.total_q = a.Sq;
    p.total_k = a.Skv;
    items = static_cast<long long>(a.B) *
            (static_cast<long long>(a.Hkv) * ((a.max_k + kTile - 1) / kTile) * p.kv_split +
             q_planes * (((static_cast<long long>(a.max_q) << lg) + kTile - 1) / kTile) * p.q_split);
  } else {
    p.q_tiles = static_cast<int>(((static_cast<long long>(a.Sq) << lg) + kTile - 1) / kTile);
    p.kv_tiles = (a.Skv + kTile - 1) / kTile;
    p.q_items = static_cast<int>(q_planes * p.q_tiles);
    p.kv_items = static_cast<int>(kv_planes * p.kv_tiles);
    p.kv_block = plan.kv_block;
    p.q_block = plan.q_block;
    items = static_cast<long long>(p.q_items) * p.q_split + static_cast<long long>(p.kv_items) * p.kv_split;
  }
  const int grid = static_cast<int>(items > 0 && items < sms ? items : sms);
  // (the kernel that can split costs a launch that does not 7 %: B4 H32 S2048 causal 354 -> 379 us)
  return launch(plan.kv_split > 1 || plan.q_split > 1 ? shared : whole, grid, kThreads<VARLEN>, C::BYTES, stream, mq, mdo, mk, mv, p);
}

}  // namespace

cudaError_t launch_attn_bwd(const BwdArgs& a, const KernelCtl& ctl, cudaStream_t stream) {
  if (a.cu_q) return a.D == 128 ? launch_d<128, true>(a, ctl, stream) : launch_d<64, true>(a, ctl, stream);
  return a.D == 128 ? launch_d<128, false>(a, ctl, stream) : launch_d<64, false>(a, ctl, stream);
}

}  // namespace loom
