// Attention of a chunk of new tokens per sequence over a paged KV cache: TMA + mbarrier ring over the
// pages, tcgen05 MMAs with TMEM accumulators, warp-specialised loader / MMA / softmax roles, and the
// work of a call dealt out evenly whatever mixture of lengths it holds.
//
// Per query row, over key tiles of 128, with scores s_j = scale q.k_j in units of log 2:
//     m' = max(m, max_j s_j),  l' = l 2^(m-m') + sum_j 2^(s_j-m'),  o' = o 2^(m-m') + sum_j 2^(s_j-m') v_j
//     O = o / l,  LSE = (m + log2 l) ln 2;
// parts (m_p, l_p, o_p) of a row's keys join as M = max m_p, l = sum 2^(m_p-M) l_p, o = sum 2^(m_p-M) o_p.
//
// Rows.  The `gt` query heads of a kv head (all of its group, up to 128) are rows next to one another: row
// i of a tile is token i / gt, head i % gt of the plane, TQ = 128 / gt tokens a tile, so that single tokens
// and drafts fill as few tiles as they can and a key is read once for all of them.  A unit of work is a
// pair of query tiles (256 rows; the second may be missing) of a plane of a sequence, against the keys
// that it sees.  Two tiles alternate on the tensor pipe, each over all of the keys; a single tile's
// even key tiles go one tile's way and its odd ones the other's, whose sums are joined in the end (O in
// TMEM, m and l through shared memory), so that its steps overlap too.
//
// Dealing.  All units lie on one line, in order, each as long as its modelled cost: kUnitCost and a
// weight per key.  CTA c of G takes the c-th of G equal stretches of the line's W, cut to
// whole key tiles of the units it starts and ends in.  So the CTAs finish together for any mixture of
// prompts and single tokens, no list of items is made in memory, and nothing depends on timing: the
// sequences' prefix sum and a binary search give each CTA its first unit, and one warp walks on from there,
// a few units ahead of the others.  A unit that lies in one stretch is finished there.  The pieces of a
// cut one go to the workspace in 32 bits; the last warp to bring its rows' piece joins all of them in the
// pieces' order.
//
// What bounds it: many queries, the tensor cores, as the prefill kernel, whose step this one repeats
// (two query tiles alternate on the tensor pipe, P in TMEM); few queries, the cache's bandwidth; small calls,
// latencies.  GB300, H32/8 D 128, on the device alone: 2048 tokens after 30000 in 637 to 651 us, 1599 to 1634 TFLOP/s (call
// after call from Python, under the power cap, 718 to 732 us, 1422 to 1450 TFLOP/s); 16 single
// tokens of 4K to 8K keys in 73.8 us, 5.5 TB/s; 31 of 100 to 12K and 481 tokens of a prompt in 138 us,
// 5.7 TB/s; one of 500 keys in 10.3 us.  Two tiles' alternation and 128 keys a tile: a step of both
// takes 2900 clocks for 2048 of the tensor pipe, and TMEM has room for no third S and O.
#include <cuda.h>
#include <cuda_bf16.h>

#include <chrono>
#include <mutex>

#include "chunk.h"
#include "ptx.cuh"

namespace loom {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRescaleThreshold = 8.0f;  // base-2 units; P <= 2^8 between rescales

// The line's units: a key of a pair of tiles costs 1 << kKeyLg2, of a single tile 1 << kKeyLg1; a unit kUnitCost more.
// (1000, 1400, 2000 and 3000: 8192 tokens alone 377, 354, 357 and 359 us, 2048 alone 50.0, 50.0, 48.9 and 49.9, 512 after 3584
// 45.8, 46.0, 44.7 and 44.3, 48 drafts 23.9, 23.6, 23.3 and 23.2, 16 tokens of 4K to 8K keys 74.0, 73.8, 73.8 and 74.9.)
constexpr int kKeyLg2 = 3, kKeyLg1 = 2, kUnitCost = 2000;
// The least that a CTA is given of units that are longer: they are not cut into shorter pieces.  (1000, 2000, 3000, 6000 and
// 12000: one token of 500 keys 11.4, 10.5, 10.3, 10.3 and 10.3 us, of 1024 15.0, 16.7, 16.5, 16.0 and 15.8, of 4096 21.6, 19.6,
// 19.8, 24.3 and 41.4, four of 4096 25.5, 23.3, 25.7, 27.3 and 43.9, 48 drafts 23.4, 23.3, 23.3, 23.3 and 27.2.)
constexpr int kLeastStretch = 3000;
// A cut that would leave less than this of a unit's tiles on one side falls on its end: joining a piece costs more
// than the unevenness.  It concerns single tiles: a pair's key tile costs as much by itself, so a pair is cut where the line says.
// With every cut, so, and with twice this: 128 tokens, 64 wide, after 10 to 500 39.5, 37.5 and 36.8 us; 48 drafts 23.5, 23.3
// and 23.9; one token of 4096 keys 19.3, 19.8 and 22.6; 16 of 4K to 8K 73.8, 73.8 and 74.2.
constexpr int kSnap = 1024;

template <int D>
struct ChunkCfg {
  static constexpr int BM = 128, BN = 128;
  static constexpr int NR = D == 128 ? 2 : 4;       // slots of the K ring, and of the V ring
  static constexpr int THREADS = 384;               // 8 softmax warps, K loader, MMA, V loader, scheduler
  // Units that the scheduler is ahead: at D = 128 what shared memory has room for.  (D = 64, 128 tokens after 10 to 500:
  // 4 and five slots a ring 44.7 us, 8 and four 41.4; longer units the same.)
  static constexpr int NREC = D == 128 ? 4 : 8;
  static constexpr int NBOX = D / 64;               // 128-byte swizzled boxes per row of a tile
  static constexpr uint32_t BOX_BYTES = BM * 128;
  static constexpr uint32_t TILE_BYTES = NBOX * BOX_BYTES;
  static constexpr uint32_t Q_OFF = 0;
  static constexpr uint32_t RING_OFF = 2 * TILE_BYTES;
  static constexpr uint32_t STG_OFF = RING_OFF + 2 * NR * TILE_BYTES;  // 4 KB for each softmax warp
  static constexpr uint32_t ML_OFF = STG_OFF + 8 * 4096;               // [BM] (m, l): see bar_ml
  static constexpr uint32_t BAR_OFF = ML_OFF + BM * 8;
  // q[2], qe[2], full[2][NR], empty[2][NR], s[2], p[2][2], o[2], oe[2], ml, mle, drain, rec[NREC], rece[NREC]
  static constexpr int NBAR = 4 + 4 * NR + 2 + 4 + 2 + 2 + 3 + 2 * NREC;
  static constexpr uint32_t REC_OFF = (BAR_OFF + NBAR * 8 + 15) / 16 * 16;  // [NREC] Item
  static constexpr uint32_t LINE_OFF = REC_OFF + NREC * 80;                 // Line, and the Walk to its start
  static constexpr uint32_t SUM_OFF = LINE_OFF + 96;  // the scan's sums, one per warp, and numbers of units
  static constexpr uint32_t TMEM_PTR_OFF = SUM_OFF + THREADS / 32 * 12;
  static constexpr uint32_t ABORT_OFF = TMEM_PTR_OFF + 8;
  static constexpr uint32_t BYTES = ABORT_OFF + 16 + 1024;  // + alignment slack
  static constexpr uint32_t S_COL = 0;       // + t * BN
  static constexpr uint32_t O_COL = 2 * BN;  // + t * D
  static_assert(BYTES <= 227 * 1024, "shared memory budget");
  static_assert(O_COL + 2 * D <= 512, "TMEM budget");
};

struct ChunkParams {
  __nv_bfloat16* o;
  float* lse;
  const int32_t *cu_q, *seqlens, *table;
  float* part;                // [2 G][groups][D / 4][32] float4: the rows of cut units' pieces
  float2* part_ml;            // [2 G][groups][32]: their (m, l); l < 0: no keys, no row
  unsigned long long* count;  // [G][8]: pieces of a 32-row group that have come
  unsigned long long tag;     // of this process, in the upper 48 bits of a count
  int groups;                 // 32-row groups of a unit that the workspace has room for
  int B, Hq, total_q, causal;
  int gt, planes, planes_per_kv, tq;  // heads of a plane, planes of a token, tokens of a tile
  int num_pages, page, max_pages, hnd, Hkv;
  float c;  // scale log2(e)
  KernelCtl ctl;
};

// ---------------------------------------------------------------- the line of work
// a / b of numbers that are not negative: nearly always below 2^32, where it takes a fifth of the time.
__device__ __forceinline__ long long quotient(long long a, long long b) {
  if (((a | b) >> 32) == 0) return static_cast<unsigned>(a) / static_cast<unsigned>(b);
  return a / b;
}
struct Seq {
  int qb, sq, skv, pairs;  // first token, tokens, keys, pairs of query tiles
};
__device__ __forceinline__ Seq load_seq(const ChunkParams& p, int b) {
  Seq s;
  // (offsets that decrease or leave the tensor are the caller's mistake; they reach no other memory)
  s.qb = min(max(p.cu_q[b], 0), p.total_q);
  s.sq = min(max(p.cu_q[b + 1], s.qb), p.total_q) - s.qb;
  const long long cap = static_cast<long long>(p.max_pages) * p.page;
  s.skv = static_cast<int>(min(max(static_cast<long long>(p.seqlens[b]), 0ll), cap));
  s.pairs = static_cast<int>((static_cast<unsigned>(s.sq) + 2u * p.tq - 1) / (2u * p.tq));
  return s;
}
// Keys that the queries before token `end` of a sequence see.
__device__ __forceinline__ int keys_until(const ChunkParams& p, const Seq& s, long long end) {
  if (!p.causal) return s.skv;
  return static_cast<int>(max(0ll, min(end, static_cast<long long>(s.sq)) + s.skv - s.sq));
}
__device__ __forceinline__ int key_tiles(int keys) { return static_cast<int>((static_cast<unsigned>(keys) + 127u) / 128u); }
__device__ __forceinline__ int key_lg(const ChunkParams& p, const Seq& s, int pair) {
  return s.sq - 2ll * p.tq * pair > p.tq ? kKeyLg2 : kKeyLg1;
}
__device__ __forceinline__ long long unit_cost(const ChunkParams& p, const Seq& s, int pair) {
  return kUnitCost + (static_cast<long long>(keys_until(p, s, 2ll * p.tq * (pair + 1))) << key_lg(p, s, pair));
}
// Cost of a plane's pairs before pair i < pairs (all of them of two tiles, none past the sequence's end).
__device__ __forceinline__ long long cost_before(const ChunkParams& p, const Seq& s, int i) {
  long long keys = static_cast<long long>(i) * s.skv;
  if (p.causal) {
    // pair j sees off + step (j + 1) keys, from the first j where that is positive
    const long long step = 2ll * p.tq, off = static_cast<long long>(s.skv) - s.sq;
    const long long j0 = off >= 0 ? 0 : quotient(-off, step);
    const long long n = i - j0;
    keys = n > 0 ? n * off + step * ((j0 + 1 + i) * n / 2) : 0;
  }
  return static_cast<long long>(i) * kUnitCost + (keys << kKeyLg2);
}
__device__ __forceinline__ long long plane_cost(const ChunkParams& p, const Seq& s) {
  return s.pairs ? cost_before(p, s, s.pairs - 1) + unit_cost(p, s, s.pairs - 1) : 0;
}
// The line, W long and dealt to G CTAs, and this CTA's stretch of it.
struct Line {
  long long W, x0, x1;
  long long each;  // W / G
  int rest, G;     // W % G
  __device__ __forceinline__ void set(long long length, int units, int ctas, int cta) {
    W = length;
    G = ctas;
    // (as many for each unit, so that equal ones are not cut where they need not be)
    if (units < ctas && W < static_cast<long long>(ctas) * kLeastStretch)
      G = max(1, min(ctas, units * max(1, static_cast<int>(W) / (max(units, 1) * kLeastStretch))));
    each = quotient(W, G);
    rest = static_cast<int>(W - each * G);
    x0 = cta < G ? bound(cta) : W;
    x1 = cta + 1 < G ? bound(cta + 1) : W;
  }
  // Where CTA c's stretch begins.
  __device__ __forceinline__ long long bound(int c) const { return each * c + min(c, rest); }
};
// Key tiles of a unit that lie before the place d > 0 behind its beginning.
__device__ __forceinline__ int tiles_before(long long d, int key_lg, int tiles) {
  const long long t = (d - kUnitCost + (128 << key_lg) - 1) >> (key_lg + 7);
  const int n = t < 0 ? 0 : t < tiles ? static_cast<int>(t) : tiles;
  return min(n, tiles - n) < (kSnap + (128 << key_lg) - 1) >> (key_lg + 7) ? (2 * n < tiles ? 0 : tiles) : n;
}

// A place on the line: unit `pair` of a plane of sequence b, which begins at `at`.
struct Walk {
  int b, plane, pair;
  long long at;
  Seq s;
};
// A unit, or the piece of it that this CTA has; shared memory's record of it is 80 bytes.
struct Item {
  int b, plane, t0, qb, sq, skv;  // t0: its first token within the sequence
  int lo, n;                      // first key tile and key tiles here (n < 0: there are no more items)
  int n0, n1;                     // of these, the steps of S, P and O number 0 and number 1
  int tiles;                      // all its key tiles
  int two;                        // it has two query tiles
  int key_lg;                     // a key's cost
  int first, pieces;              // cut: the first CTA that has a piece, and how many have (written before the next record)
  long long at, cost;             // its place on the line
  __device__ __forceinline__ bool cut() const { return n < tiles; }
};
static_assert(sizeof(Item) == 80, "fits its record");

// The first sequence from b on that brings tokens (B: none does), found by a whole warp, 256 sequences at a time.
// (GB300, one token of 500 keys as the first of 4096 sequences: 309 us where idle ones were walked one at a time, and ahead of
// the unit that was at hand; 24.9 so, of which 14 are the prefix sum over them all; a million idle ones outlasted the other roles'
// waits.)
__device__ __noinline__ int next_sequence(const ChunkParams& p, int b) {
  const unsigned B = static_cast<unsigned>(p.B), lane = threadIdx.x & 31;
#pragma unroll 1
  for (unsigned from = static_cast<unsigned>(b); from < B; from += 256) {  // (of all lanes alike)
    unsigned found = B;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
      const unsigned r = from + 32 * i + lane;
      if (r < B && min(max(p.cu_q[r + 1], 0), p.total_q) > min(max(p.cu_q[r], 0), p.total_q)) found = r;  // (as load_seq has it)
    }
    found = __reduce_min_sync(0xffffffffu, found);
    if (found < B) return static_cast<int>(found);
  }
  return p.B;
}

// The CTA's next piece, and the walk to it; false past the stretch's end.  (All lanes of a warp alike.)
__device__ __forceinline__ bool next_item(const ChunkParams& p, const Line& ln, Walk& w, Item& it) {
#pragma unroll 1
  while (w.b < p.B && w.at < ln.x1) {
    // (past a sequence's end only here: the last unit of a stretch waits for no other sequence)
    if (w.pair == w.s.pairs) {
      w.pair = 0;
      if (++w.plane == p.planes) {
        w.plane = 0;
        ++w.b;
#pragma unroll 1
        while (w.b < p.B) {
          w.s = load_seq(p, w.b);
          if (w.s.pairs) break;
          w.b = next_sequence(p, w.b + 1);
        }
        if (w.b >= p.B) break;
      }
    }
    const long long step = 2ll * p.tq;
    it.b = w.b;
    it.plane = w.plane;
    it.qb = w.s.qb;
    it.sq = w.s.sq;
    it.skv = w.s.skv;
    it.t0 = static_cast<int>(step * w.pair);
    it.two = w.s.sq - it.t0 > p.tq;
    it.key_lg = it.two ? kKeyLg2 : kKeyLg1;
    const int keys = keys_until(p, w.s, step * (w.pair + 1));
    it.tiles = key_tiles(keys);
    it.at = w.at;
    it.cost = kUnitCost + (static_cast<long long>(keys) << it.key_lg);
    it.lo = ln.x0 > it.at ? tiles_before(ln.x0 - it.at, it.key_lg, it.tiles) : 0;
    const int hi = ln.x1 < it.at + it.cost ? tiles_before(ln.x1 - it.at, it.key_lg, it.tiles) : it.tiles;
    it.n = hi - it.lo;
    it.n0 = it.two ? max(0, min(hi, key_tiles(keys_until(p, w.s, it.t0 + p.tq))) - it.lo) : (it.n + 1) / 2;
    it.n1 = it.two ? it.n : it.n / 2;
    w.at += it.cost;
    ++w.pair;
    // (a unit without keys belongs to the CTA in whose stretch it begins)
    if (it.n > 0 || (it.tiles == 0 && ln.x0 <= it.at)) return true;
  }
  return false;
}

// The walk to this CTA's first unit, from the sequence s, number b, that begins at `at`.
__device__ __forceinline__ Walk walk_from(const ChunkParams& p, const Line& ln, int b, const Seq& s, long long at) {
  Walk w;
  w.b = b;
  w.s = s;
  const long long plane = plane_cost(p, w.s);
  w.plane = static_cast<int>(quotient(ln.x0 - at, plane));
  const long long r = ln.x0 - at - w.plane * plane;
  int lo = 0, hi = w.s.pairs;  // the last pair that begins at r or before
#pragma unroll 1
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (cost_before(p, w.s, mid) <= r)
      lo = mid;
    else
      hi = mid;
  }
  w.pair = lo;
  w.at = at + w.plane * plane + cost_before(p, w.s, lo);
  return w;
}

__device__ __forceinline__ void st_shared_u32(uint32_t addr, uint32_t v) {
  asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ int ld_shared_i32(uint32_t addr) {
  int v;
  asm volatile("ld.shared.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// The pieces of a cut unit, found by a whole warp: the first CTA that has one (its last unit; the others' pieces
// are their CTAs' first), and which of the 32 CTAs from `from` on have one.
__device__ __forceinline__ int first_cta(const Line& ln, const Item& it) {
  int c = min(ln.G - 1, static_cast<int>(static_cast<float>(it.at) / static_cast<float>(ln.W) * ln.G));
#pragma unroll 1
  while (c > 0 && ln.bound(c) > it.at) --c;
#pragma unroll 1
  while (c + 1 < ln.G && ln.bound(c + 1) <= it.at) ++c;
  // (it may begin in a stretch that holds none of its key tiles)
#pragma unroll 1
  while (c + 1 < ln.G && tiles_before(ln.bound(c + 1) - it.at, it.key_lg, it.tiles) == 0) ++c;
  return c;
}
__device__ __forceinline__ uint32_t piece_ctas(const Line& ln, const Item& it, int from) {
  const int c = from + static_cast<int>(threadIdx.x & 31);
  bool has = false;
  if (c < ln.G) {
    const long long begin = ln.bound(c) - it.at, end = (c + 1 < ln.G ? ln.bound(c + 1) : ln.W) - it.at;
    const int lo = begin > 0 ? tiles_before(begin, it.key_lg, it.tiles) : 0;
    const int hi = end < it.cost ? tiles_before(end, it.key_lg, it.tiles) : it.tiles;
    has = end > 0 && begin < it.cost && lo < hi;
  }
  return __ballot_sync(0xffffffffu, has);
}
// How many pieces a cut unit has; and their places in the workspace, in order, into the warp's list in shared
// memory (4 bytes each, one for each CTA at most).
__device__ __forceinline__ int count_pieces(const Line& ln, const Item& it, int first) {
  int n = 0;
#pragma unroll 1
  for (int from = first; from < ln.G && ln.bound(from) < it.at + it.cost; from += 32) n += __popc(piece_ctas(ln, it, from));
  return n;
}
__device__ __forceinline__ void list_pieces(const Line& ln, const Item& it, int first, uint32_t list) {
  const int lane = static_cast<int>(threadIdx.x & 31);
  int n = 0;
#pragma unroll 1
  for (int from = first; from < ln.G && ln.bound(from) < it.at + it.cost; from += 32) {
    const uint32_t ctas = piece_ctas(ln, it, from);
    const int c = from + lane;
    if (ctas >> lane & 1u) st_shared_u32(list + 4 * (n + __popc(ctas & ((1u << lane) - 1u))), c == first ? 2 * c + 1 : 2 * c);
    n += __popc(ctas);
  }
  __syncwarp();
}

// mbar_wait_warp as a call: in line at each of the roles' waits it made the kernel longer than the instruction
// cache, and what runs once a unit was fetched anew each time.
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, const KernelCtl& ctl, const Abort& ab) {
  return mbar_wait_warp(bar, parity, ctl, ab);
}
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, const KernelCtl& ctl, const Abort& ab) {
  return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) || wait_long(bar, parity, ctl, ab);
}

// ---------------------------------------------------------------- softmax
// One online-softmax step of one query row (this thread's TMEM lane) over a 128-key tile of S in TMEM at
// s_tm: mask keys >= limit, move the running max lazily, write P = 2^(S c - m) as bf16 over the first
// half of S's columns in two halves (arriving on bar_p and bar_p + 8 after each), rescale O at o_tm where
// the max moved, and add to the row's sum.  S is only ready after the tile's previous P.V (issued before it by
// the same warp), so the rescale needs no wait.  P is rounded to bf16 because the product takes one type for P and V, and V is
// the cache's; l sums the weights before that, in 32 bits.  A weight is off by half a step at most, to either side, which
// puts an output's error at 0.0023 of the norm where its own rounding to bf16 is 0.0017; LSE has nothing of it.
template <int D>
__device__ __forceinline__ bool chunk_step(uint32_t s_tm, uint32_t o_tm, uint32_t bar_s, uint32_t par_s, uint32_t bar_p,
                                           bool first, int limit, float c, float& m_run, float& l_run, const KernelCtl& ctl,
                                           const Abort& ab) {
  constexpr int BN = 128;
  if (!mbar_wait_warp(bar_s, par_s, ctl, ab)) return false;
  tc_fence_after();
  uint32_t s[BN];
#pragma unroll
  for (int ch = 0; ch < BN / 32; ++ch) tmem_ld32(s_tm + ch * 32, s + ch * 32);
  tmem_wait_ld();
#pragma unroll
  for (int ch = 0; ch < BN / 32; ++ch) reg_fence32(s + ch * 32);
  if (limit < BN) {
#pragma unroll
    for (int g = 0; g < BN / 32; ++g) {
      const int n = limit - 32 * g;  // visible keys of the 32
      const uint32_t visible = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (!(visible & (1u << i))) s[32 * g + i] = __float_as_uint(-INFINITY);
    }
  }
  float mm[8];
#pragma unroll
  for (int g = 0; g < 8; ++g) mm[g] = __uint_as_float(s[g]);
#pragma unroll
  for (int i = 8; i + 16 <= BN; i += 16)
#pragma unroll
    for (int g = 0; g < 8; ++g) mm[g] = max3(mm[g], __uint_as_float(s[i + g]), __uint_as_float(s[i + 8 + g]));
#pragma unroll
  for (int g = 0; g < 8; ++g) mm[g] = fmaxf(mm[g], __uint_as_float(s[BN - 8 + g]));
  const float mx = fmaxf(max3(mm[0], mm[1], mm[2]), max3(max3(mm[3], mm[4], mm[5]), mm[6], mm[7]));
  const float m_new = fmaxf(m_run, mx * c);
  const bool need = m_new > m_run + kRescaleThreshold;
  const float alpha = need ? ex2(m_run - m_new) : 1.f;
  if (need) m_run = m_new;
  const float ms = m_run == -INFINITY ? 0.f : m_run;
  const uint64_t nms2 = f2(-ms, -ms), c2 = f2(c, c);
  uint64_t acc[4] = {0, 0, 0, 0};
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    uint32_t pk[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const int e = 64 * half + 2 * i;
      const uint64_t x = fma2(f2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2, nms2);
      const float p0 = ex2(f2lo(x)), p1 = ex2(f2hi(x));
      acc[i & 3] = add2(acc[i & 3], f2(p0, p1));
      pk[i] = pack_bf16x2(p0, p1);
    }
    tmem_st32(s_tm + 32 * half, pk);
    tmem_wait_st();
    if (half == 0 && !first && __any_sync(0xffffffffu, need)) {
      const uint64_t a2 = f2(alpha, alpha);
#pragma unroll 1
      for (int ch = 0; ch < D / 32; ++ch) {
        uint32_t rr[32];
        tmem_ld32(o_tm + ch * 32, rr);
        tmem_wait_ld();
        reg_fence32(rr);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint64_t x = mul2(f2(__uint_as_float(rr[2 * i]), __uint_as_float(rr[2 * i + 1])), a2);
          rr[2 * i] = __float_as_uint(f2lo(x));
          rr[2 * i + 1] = __float_as_uint(f2hi(x));
        }
        tmem_st32(o_tm + ch * 32, rr);
      }
      tmem_wait_st();
    }
    tc_fence_before();
    mbar_arrive(bar_p + 8 * half);
  }
  const uint64_t a01 = add2(add2(acc[0], acc[1]), add2(acc[2], acc[3]));
  l_run = l_run * alpha + (f2lo(a01) + f2hi(a01));
  return true;
}

__device__ __forceinline__ void st_shared_f2(uint32_t addr, float a, float b) {
  asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(a), "f"(b) : "memory");
}

// 64 columns of this warp's 32 rows, packed bf16 pairs of each lane's own row in w, to the rows' places in O (my_at:
// this row's first column, in 16 bytes from o; < 0: not a row): through the warp's 4 KB of shared memory, so that
// a store writes whole 128-byte lines (from the lanes' own rows it would touch 32 lines).
__device__ __forceinline__ void store_rows(uint32_t stg, const uint32_t* w, int my_at, uint4* o) {
  const int lane = threadIdx.x & 31, j = lane % 8;
#pragma unroll
  for (int c = 0; c < 8; ++c)
    st_shared_v4(stg + lane * 128 + ((c ^ (lane & 7)) << 4), w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = k * 4 + lane / 8, at = __shfl_sync(0xffffffffu, my_at, r);
    const uint4 v = ld_shared_v4(stg + r * 128 + ((j ^ (r & 7)) << 4));
    if (at >= 0) o[at + j] = v;
  }
  __syncwarp();
}

__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2; }

// Counts one more piece of a 32-row group: how many have come.  A count without the tag (see ChunkParams) is
// whatever the workspace held before, and begins anew; a launch leaves its counts at zero.
__device__ __forceinline__ int count_piece(unsigned long long* at, unsigned long long tag) {
  // (released: the warp's pieces before it; acquired: the others' behind it)
  const auto add = [&]() {
    unsigned long long was;
    asm volatile("atom.acq_rel.gpu.global.add.u64 %0, [%1], 1;" : "=l"(was) : "l"(at) : "memory");
    return was;
  };
  unsigned long long was = add();
  while ((was ^ tag) >> 16) {
    const unsigned long long seen = was + 1;
    asm volatile("atom.acq_rel.gpu.global.cas.b64 %0, [%1], %2, %3;" : "=l"(was) : "l"(at), "l"(seen), "l"(tag + 1) : "memory");
    if (was == seen) return 1;
    if ((was ^ tag) >> 16)
      --was;  // (another's count on top of what there was)
    else
      was = add();
  }
  return static_cast<int>(was & 0xffff) + 1;
}

// What a unit, or a piece of it, has to say of one query row (this thread's TMEM lane): its place in O, in 16 bytes
// from the unit's first token (-1: not a row), and in LSE (or null), and its sums, O's in TMEM: weight 0 of that at o_tm, and with
// `both` weight 1 of that at o_tm + D.
struct RowSums {
  int at;
  float* lse_at;
  float m, l, w0, w1;
  bool has, both;  // key tiles were walked here
  bool any;        // the warp has a row
};

// 32 columns of a row's O from column c on, weighted and summed.
template <int D>
__device__ __forceinline__ void load_o(uint32_t o_tm, int c, const RowSums& r, float scale, uint32_t* out) {
  tmem_ld32(o_tm + c, out);
  tmem_wait_ld();
  reg_fence32(out);
  const uint64_t a = f2(r.w0 * scale, r.w0 * scale);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint64_t x = mul2(f2(__uint_as_float(out[2 * i]), __uint_as_float(out[2 * i + 1])), a);
    out[2 * i] = __float_as_uint(f2lo(x)), out[2 * i + 1] = __float_as_uint(f2hi(x));
  }
  if (r.both) {
    uint32_t other[32];
    tmem_ld32(o_tm + D + c, other);
    tmem_wait_ld();
    reg_fence32(other);
    const uint64_t b = f2(r.w1 * scale, r.w1 * scale);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint64_t x = fma2(f2(__uint_as_float(other[2 * i]), __uint_as_float(other[2 * i + 1])), b,
                              f2(__uint_as_float(out[2 * i]), __uint_as_float(out[2 * i + 1])));
      out[2 * i] = __float_as_uint(f2lo(x)), out[2 * i + 1] = __float_as_uint(f2hi(x));
    }
  }
}
// O has been read out of TMEM: the next item's P.V may overwrite it.
__device__ __forceinline__ void release_o(const RowSums& r, uint32_t bar_oe, uint32_t bar_oe1) {
  tc_fence_before();
  mbar_arrive(bar_oe);
  if (r.both) mbar_arrive(bar_oe1);
}

// Joins the pieces of a warp's rows, 1 << lg of which lie side by side in the lanes, each lane with U chunks of 16
// bytes of a row at a time, of two pieces, whose loads are on their way together.  (What runs once a unit is fetched
// anew each time, at 100 clocks for eight instructions, so that code weighs more than rounds.)
template <int D>
__device__ __forceinline__ void join_pieces(const ChunkParams& p, uint32_t list, int pieces, const float2* ml, const float4* part,
                                            int rows, int lg, const RowSums& r, long long unit_at) {
  constexpr int U = 8;
  const int lane = threadIdx.x & 31, my = min(lane & ((1 << lg) - 1), rows - 1), parts = 32 >> lg;
  const size_t ml_slot = static_cast<size_t>(p.groups) * 32, part_slot = ml_slot * (D / 4);
  ml += my;
  part += my + (lane >> lg) * 32;
  float M = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < pieces; k0 += 4) {
    float2 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = __ldcg(ml + ld_shared_i32(list + 4 * min(k0 + k, pieces - 1)) * ml_slot);
    float M_new = M;
#pragma unroll
    for (int k = 0; k < 4; ++k) M_new = fmaxf(M_new, x[k].x);
    const float base = M_new == -INFINITY ? 0.f : M_new;
    l *= ex2(M - base);
    M = M_new;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k0 + k < pieces && !(x[k].y < 0.f)) l = fmaf(ex2(x[k].x - base), x[k].y, l);
  }
  const float base = M == -INFINITY ? 0.f : M, inv = l == 0.f ? 0.f : 1.f / l;
  const int at = __shfl_sync(0xffffffffu, r.at, my);
  __nv_bfloat16* o = p.o + unit_at + static_cast<long long>(at) * 8 + (lane >> lg) * 4;
#pragma unroll 1
  for (int block = 0; block < D / 4; block += U * parts) {  // (of all lanes alike)
    float acc[4 * U];
#pragma unroll
    for (int i = 0; i < 4 * U; ++i) acc[i] = 0.f;
#pragma unroll 1
    for (int k0 = 0; k0 < pieces; k0 += 2) {
      float2 x[2];
      float4 v[2][U];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const size_t slot = ld_shared_i32(list + 4 * min(k0 + k, pieces - 1));
        x[k] = __ldcg(ml + slot * ml_slot);
        const float4* from = part + slot * part_slot + block * 32;
#pragma unroll
        for (int i = 0; i < U; ++i) v[k][i] = __ldcg(from + i * parts * 32);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (k0 + k >= pieces || x[k].y < 0.f) continue;  // (no keys of the row's tile: nothing was written there)
        const float w = ex2(x[k].x - base) * inv;
#pragma unroll
        for (int i = 0; i < U; ++i) {
          acc[4 * i] = fmaf(w, v[k][i].x, acc[4 * i]);
          acc[4 * i + 1] = fmaf(w, v[k][i].y, acc[4 * i + 1]);
          acc[4 * i + 2] = fmaf(w, v[k][i].z, acc[4 * i + 2]);
          acc[4 * i + 3] = fmaf(w, v[k][i].w, acc[4 * i + 3]);
        }
      }
    }
    if ((lane & ((1 << lg) - 1)) < rows)
#pragma unroll
      for (int i = 0; i < U; ++i)
        *reinterpret_cast<uint2*>(o + (block + i * parts) * 4) =
            make_uint2(pack_bf16x2(acc[4 * i], acc[4 * i + 1]), pack_bf16x2(acc[4 * i + 2], acc[4 * i + 3]));
  }
  // (every lane below `rows` has its own row)
  if (r.lse_at) *r.lse_at = row_lse(M, l);
}

// Counts one of the pieces of this warp's rows of a cut unit; true for the last to come.
__device__ __forceinline__ bool last_piece(const ChunkParams& p, int pieces, int first, int warp) {
  int come = 0;
  if ((threadIdx.x & 31) == 0) {
    unsigned long long* count = p.count + static_cast<size_t>(first) * 8 + warp;
    come = count_piece(count, p.tag);
    if (come == pieces) *reinterpret_cast<volatile unsigned long long*>(count) = p.tag;
  }
  return __shfl_sync(0xffffffffu, come, 0) == pieces;
}

// A whole unit: this warp's 32 rows are stored.  (Not inlined, like the next: its registers would spill the softmax
// loop's.)
template <int D>
__device__ __noinline__ void finish_unit(const ChunkParams& p, const RowSums r, long long unit_at, uint32_t o_tm, uint32_t bar_oe,
                                         uint32_t bar_oe1, uint32_t stg) {
  const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
  const uint64_t inv2 = f2(inv * r.w0, inv * r.w0);
  uint4* o = reinterpret_cast<uint4*>(p.o + unit_at);
#pragma unroll 1
  for (int h = 0; h < D / 64; ++h) {  // (code that runs once a unit: the shorter, the sooner it is fetched)
    uint32_t w[64];
    if (r.both) {
      load_o<D>(o_tm, 64 * h, r, inv, w);
      load_o<D>(o_tm, 64 * h + 32, r, inv, w + 32);
    } else if (r.has) {
      tmem_ld32(o_tm + 64 * h, w);
      tmem_ld32(o_tm + 64 * h + 32, w + 32);
      tmem_wait_ld();
      reg_fence32(w);
      reg_fence32(w + 32);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const uint64_t x = mul2(f2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])), inv2);
        w[2 * i] = __float_as_uint(f2lo(x)), w[2 * i + 1] = __float_as_uint(f2hi(x));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 64; ++i) w[i] = 0;
    }
    if (r.has && h + 1 == D / 64) release_o(r, bar_oe, bar_oe1);
#pragma unroll
    for (int i = 0; i < 32; ++i) w[i] = pack_bf16x2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    store_rows(stg, w, r.at < 0 ? r.at : r.at + 8 * h, o);
  }
  if (r.lse_at) *r.lse_at = row_lse(r.m, r.l);
}

// A piece of a cut unit: this warp's 32 rows go to the workspace, each 16 bytes of a row beside the other lanes'
// (one store: 512 bytes in a row).  The last warp to bring its piece of the rows joins all of them, in the
// pieces' order.  Not inlined: it is rare, and its registers would spill the softmax loop's.
template <int D>
__device__ __noinline__ void finish_piece(const ChunkParams& p, const Line& ln, const Item& it, const RowSums r, long long unit_at,
                                          uint32_t o_tm, uint32_t bar_oe, uint32_t bar_oe1, uint32_t stg, int warp) {
  const int lane = threadIdx.x & 31, group = it.two ? warp : warp & 3;
  const bool row = r.at >= 0;
  const int slot = it.lo == 0 ? 2 * static_cast<int>(blockIdx.x) + 1 : 2 * static_cast<int>(blockIdx.x);
  if (r.any) {
    float4* mine = reinterpret_cast<float4*>(p.part) + (static_cast<size_t>(slot) * p.groups + group) * (D / 4) * 32 + lane;
    if (r.has) {
#pragma unroll 1
      for (int ch = 0; ch < D / 32; ++ch) {
        uint32_t rr[32];
        load_o<D>(o_tm, ch * 32, r, 1.f, rr);
        if (row)
#pragma unroll
          for (int u = 0; u < 8; ++u)
            mine[(ch * 8 + u) * 32] = make_float4(__uint_as_float(rr[4 * u]), __uint_as_float(rr[4 * u + 1]),
                                                  __uint_as_float(rr[4 * u + 2]), __uint_as_float(rr[4 * u + 3]));
      }
    }
    if (row) p.part_ml[(static_cast<size_t>(slot) * p.groups + group) * 32 + lane] = make_float2(r.m, r.has ? r.l : -1.f);
  }
  if (r.has) release_o(r, bar_oe, bar_oe1);
  if (!r.any) return;
  __syncwarp();
  if (!last_piece(p, it.pieces, it.first, warp)) return;
  __syncwarp();
  list_pieces(ln, it, it.first, stg);
  // The warp's rows (its first lanes') are spread over all lanes: 1 << lg of them side by side, each lane with
  // every (32 >> lg)-th 16 bytes of its row.
  const int rows = __popc(__ballot_sync(0xffffffffu, row));
  // (at least 8, or 16 at D = 64: a row's chunks are as many as its lanes take at a time)
  const int lg = max(D == 128 ? 3 : 4, 32 - __clz(rows - 1));
  const float2* ml = p.part_ml + group * 32;
  const float4* part = reinterpret_cast<const float4*>(p.part) + static_cast<size_t>(group) * (D / 4) * 32;
  join_pieces<D>(p, stg, it.pieces, ml, part, rows, lg, r, unit_at);
  __syncwarp();  // the list has been read
}

// After a wait has given up, a softmax warp counts the pieces that it has not brought all the same, so that every
// count is whole again at the launch's end: a captured launch may be replayed on this workspace.
__device__ __noinline__ void count_rest(const ChunkParams& p, const Line& ln, int b, long long at, int warp, int counted) {
  if (ln.x0 >= ln.x1) return;
  Walk w = walk_from(p, ln, b, load_seq(p, b), at);
  Item it;
  while (next_item(p, ln, w, it)) {
    // the warp's first row, if it has rows: as the softmax role has it
    const int i = (warp & 3) * 32, token = it.t0 + (it.two ? (warp >> 2) * p.tq : 0) + i / p.gt;
    if (!it.cut() || (!it.two && warp >= 4) || i / p.gt >= p.tq || token >= it.sq) continue;
    if (--counted >= 0) continue;
    const int first = first_cta(ln, it);
    last_piece(p, count_pieces(ln, it, first), first, warp);
  }
}

template <int D>
__global__ void __launch_bounds__(ChunkCfg<D>::THREADS, 1)
    chunk_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                 const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ ChunkParams p) {
  using C = ChunkCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_base = smem_u32(smem_raw);
  const uint32_t sbase = (raw_base + 1023u) & ~1023u;  // for the 128-byte swizzled tiles
  uint8_t* smem = smem_raw + (sbase - raw_base);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  const uint32_t bar_q = sbase + C::BAR_OFF;           // [2] Q_t loaded
  const uint32_t bar_qe = bar_q + 16;                  // [2] Q_t no longer read
  const uint32_t bar_full = bar_qe + 16;               // [2][NR] slots of the K ring and of the V ring filled
  const uint32_t bar_empty = bar_full + 16 * C::NR;    // [2][NR] and no longer read
  const uint32_t bar_s = bar_empty + 16 * C::NR;       // [2] S_t ready
  const uint32_t bar_p = bar_s + 16;                   // [2][2] half h of P_t written (h = 0: and O_t rescaled)
  const uint32_t bar_o = bar_p + 32;                   // [2] O_t of the item complete
  const uint32_t bar_oe = bar_o + 16;                  // [2] O_t read out
  const uint32_t bar_ml = bar_oe + 16;                 // m and l of a single tile's odd key tiles are there
  const uint32_t bar_mle = bar_ml + 8;                 // and read
  const uint32_t bar_drain = bar_mle + 8;
  const uint32_t bar_rec = bar_drain + 8;              // [NREC] a record is written
  const uint32_t bar_rece = bar_rec + 8 * C::NREC;     // [NREC] and read by the other roles' warps
  uint32_t* tmem_ptr = reinterpret_cast<uint32_t*>(smem + C::TMEM_PTR_OFF);
  Abort ab{reinterpret_cast<volatile int*>(smem + C::ABORT_OFF)};

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(bar_q + 8 * t, 1);
      mbar_init(bar_qe + 8 * t, 1);
      mbar_init(bar_s + 8 * t, 1);
      mbar_init(bar_p + 16 * t, C::BM);
      mbar_init(bar_p + 16 * t + 8, C::BM);
      mbar_init(bar_o + 8 * t, 1);
      mbar_init(bar_oe + 8 * t, C::BM);
    }
    for (int s = 0; s < 2 * C::NR; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1);
    }
    mbar_init(bar_ml, C::BM);
    mbar_init(bar_mle, C::BM);
    mbar_init(bar_drain, 1);
    for (int i = 0; i < C::NREC; ++i) {
      mbar_init(bar_rec + 8 * i, 1);
      mbar_init(bar_rece + 8 * i, C::THREADS / 32 - 1);
    }
    *ab.flag = 0;
    *(ab.flag + 1) = 0;
    fence_barrier_init();
  }
  // rows of the Q tiles that no load fills (a tile has tq gt rows): zeros, so that their scores are too
  {
    const int rows = p.tq * p.gt, n = (C::BM - rows) * 8;
#pragma unroll 1
    for (int i = threadIdx.x; i < 2 * C::NBOX * n; i += C::THREADS)
      st_shared_v4(sbase + C::Q_OFF + i / n * C::BOX_BYTES + rows * 128 + i % n * 16, 0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  if (warp == 9) tmem_alloc(smem_u32(tmem_ptr), 512);
  // The set-up above touches no global memory; from here on the previous kernel's writes must be visible.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");

  // The line's length, and the sequence in which this CTA's stretch begins: a prefix sum over the sequences.
  Line& ln = *reinterpret_cast<Line*>(smem + C::LINE_OFF);
  volatile long long* start = reinterpret_cast<volatile long long*>(smem + C::LINE_OFF + sizeof(Line));  // sequence, its place
  Seq& start_seq = *reinterpret_cast<Seq*>(smem + C::LINE_OFF + sizeof(Line) + 16);
  static_assert(sizeof(Line) + 16 + sizeof(Seq) <= 96, "fits");
  {
    volatile long long* sums = reinterpret_cast<volatile long long*>(smem + C::SUM_OFF);
    constexpr int kWarps = C::THREADS / 32;
    Line l;
    volatile int* unit_sums = reinterpret_cast<volatile int*>(smem + C::SUM_OFF + C::THREADS / 32 * 8);
    const int G = static_cast<int>(gridDim.x);
    int units = 0;
    l.x0 = 0;
    const bool one = p.B <= C::THREADS;
    // (one round: the sum of all and this CTA's sequence from the same scan; else a round for each)
#pragma unroll 1
    for (int round = 0; round < (one ? 1 : 2); ++round) {
      long long before = 0;
#pragma unroll 1
      for (int b0 = 0; b0 < p.B; b0 += C::THREADS) {
        const int b = b0 + static_cast<int>(threadIdx.x);
        long long cost = 0;
        int n = 0;
        Seq s;
        if (b < p.B) {
          s = load_seq(p, b);
          cost = p.planes * plane_cost(p, s);
          n = min(s.pairs, 1 << 15) * min(p.planes, 1 << 10);  // (more than there are CTAs is enough)
        }
        n = __reduce_add_sync(0xffffffffu, min(n, 1 << 15));
        long long x = cost;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const long long y = __shfl_up_sync(0xffffffffu, x, d);
          if (lane >= d) x += y;
        }
        if (lane == 31) sums[warp] = x, unit_sums[warp] = n;
        __syncthreads();
        long long all = 0;
        x += before - cost;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
          const long long y = sums[i];
          if (i < warp) x += y;
          all += y;
          if (round == 0) units = min(units + unit_sums[i], 1 << 20);
        }
        if (one) {
          l.set(all, units, G, blockIdx.x);
        }
        if ((one || round == 1) && x <= l.x0 && l.x0 < x + cost) {
          start[0] = b;
          start[1] = x;
          start_seq = s;
        }
        before += all;
        __syncthreads();
      }
      if (!one && round == 0) {
        l.set(before, units, G, blockIdx.x);
      }
    }
    if (threadIdx.x == 0) ln = l;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_ptr;

  // The items, for the other roles' warps: item number i, once its record is written (null where a wait gave up, or
  // past the last one); a warp gives the record back when it needs no more of it.
  int rec_n = 0, counted = 0;  // counted: (softmax warps) pieces of cut units that this warp has counted
  const auto take_item = [&]() -> const Item* {
    const int i = rec_n % C::NREC;
    if (!wait_warp(bar_rec + 8 * i, (rec_n / C::NREC) & 1, p.ctl, ab)) return nullptr;
    const Item* it = reinterpret_cast<const Item*>(smem + C::REC_OFF + i * 80);
    return *reinterpret_cast<const volatile int*>(&it->n) < 0 ? nullptr : it;
  };
  const auto give_item = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_rece + 8 * (rec_n % C::NREC));
    ++rec_n;
  };

  if (warp == 11) {
    // ------------------------------------------------------------------ scheduler (whole warp, all lanes alike)
    Walk walk;
    walk.b = p.B;
    const Line l = ln;
    if (l.x0 < l.x1) walk = walk_from(p, l, static_cast<int>(start[0]), start_seq, start[1]);
    bool more = true;
#pragma unroll 1
    for (int k = 0; more; ++k) {
      Item it;
      more = next_item(p, l, walk, it);
      if (!more) it.n = -1;
      const int i = k % C::NREC;
      if (k >= C::NREC && !wait_warp(bar_rece + 8 * i, (k / C::NREC - 1) & 1, p.ctl, ab)) break;
      Item& rec = *reinterpret_cast<Item*>(smem + C::REC_OFF + i * 80);
      if (lane == 0) {
        rec = it;
        mbar_arrive(bar_rec + 8 * i);
      }
      __syncwarp();
      if (more && it.cut()) {
        const int first = first_cta(l, it), pieces = count_pieces(l, it, first);
        if (lane == 0) rec.first = first, rec.pieces = pieces;
      }
    }
  } else if (warp == 8 || warp == 10) {
    // ------------------------------------------------------------------ loaders (whole warps): Q and K, and V
    // Lane 0 waits and expects; a tile's pieces of min(page, 64) keys are copied by one lane each.
    const bool is_v = warp == 10;
    const CUtensorMap* map = is_v ? &tm_v : &tm_k;
    if (lane == 0) {
      if (!is_v) prefetch_tensormap(&tm_q);
      prefetch_tensormap(map);
    }
    const uint32_t full = bar_full + (is_v ? 8 * C::NR : 0), empty = bar_empty + (is_v ? 8 * C::NR : 0);
    const uint32_t ring = sbase + C::RING_OFF + (is_v ? C::NR * C::TILE_BYTES : 0);
    int pos = 0, issued = 0, skipped = -1, q_issued0 = 0, q_issued1 = 0;
    bool ok = true;
    const int rows = min(p.page, 64), rows_lg = 31 - __clz(rows);  // (8, 16, 32 or 64)
    const uint32_t q_bytes = static_cast<uint32_t>(C::NBOX * p.tq * p.gt * 128);
    int q_single = 0;  // the Q tile that the next single tile takes: they take turns
    const auto load_q = [&](int t, int plane, int token) -> bool {
      const int n = t ? q_issued1 : q_issued0;
      if (n > 0 && !wait_warp(bar_qe + 8 * t, (n - 1) & 1, p.ctl, ab)) return false;
      if (lane == 0) {
        mbar_expect_tx(bar_q + 8 * t, q_bytes);
        for (int x = 0; x < C::NBOX; ++x)
          tma_load_4d(sbase + C::Q_OFF + t * C::TILE_BYTES + x * C::BOX_BYTES, &tm_q, x * 64, 0, plane, token, bar_q + 8 * t);
      }
      __syncwarp();
      (t ? q_issued1 : q_issued0) = n + 1;
      return true;
    };
    const Item* rec;
    while (ok && (rec = take_item())) {
      const int lo = rec->lo, end = lo + rec->n, skv = rec->skv, plane = rec->plane, token = rec->qb + rec->t0, n0 = rec->n0;
      const bool two = rec->two;
      const int32_t* table = p.table + static_cast<size_t>(rec->b) * p.max_pages;
      give_item();
      if (lo == end) continue;  // no keys: nothing to load
      // the pages of the 32 pieces from key tile j on, this lane's (none past the sequence's keys)
      const auto pages_from = [&](int j) {
        const unsigned key = static_cast<unsigned>(j) * C::BN + lane * rows;
        if (key >= static_cast<unsigned>(skv)) return -1;
        return table[p.page > 64 ? key / static_cast<unsigned>(p.page) : key >> rows_lg];
      };
      // (32 pieces are `ahead` tiles; the next ones are looked up while these are loaded)
      const int ahead = 1 << (rows_lg - 2);
      int window = pages_from(lo), next_window = -1;
      if (!is_v && n0 > 0 && !(ok = load_q(two ? 0 : q_single, plane, token))) break;
      q_single ^= !two;
      const int hk = plane / p.planes_per_kv;
#pragma unroll 1
      for (int j = lo; j < end; ++j, ++pos) {
        const int slot = pos % C::NR;
        if (pos >= C::NR && !(ok = wait_warp(empty + 8 * slot, (pos / C::NR - 1) & 1, p.ctl, ab))) break;
        issued = pos + 1;
        if (p.ctl.inject == 5 && !is_v && pos == 1) {  // test hook: never load this tile
          skipped = pos;
          continue;
        }
        if (((j - lo) & (ahead - 1)) == 0) {
          if (j > lo) window = next_window;
          next_window = j + ahead < end ? pages_from(j + ahead) : -1;
        }
        const int page = __shfl_sync(0xffffffffu, window, ((j - lo) << (7 - rows_lg)) + lane);  // (of a width of 32)
        const int pieces = (min(C::BN, skv - j * C::BN) + rows - 1) >> rows_lg;
        if (lane == 0) mbar_expect_tx(full + 8 * slot, static_cast<uint32_t>(C::NBOX * pieces * rows * 128));
        __syncwarp();
        if (lane < pieces) {
          // NHD view [keys of all pages, Hkv, D]: (dim, kv head, key); HND view [pages x Hkv, page, D]:
          // (dim, row in page, page x Hkv + kv head).  A page that there is not: past the end, which reads as zeros.
          const unsigned key = static_cast<unsigned>(j * C::BN + lane * rows);
          const int in = p.page > 64 ? static_cast<int>(key % static_cast<unsigned>(p.page)) : 0;
          const bool bad = page < 0 || page >= p.num_pages;
          const int y = p.hnd ? in : hk;
          const int z = p.hnd ? (bad ? p.num_pages * p.Hkv : page * p.Hkv + hk) : (bad ? p.num_pages * p.page : page * p.page + in);
#pragma unroll
          for (int x = 0; x < C::NBOX; ++x)
            tma_load_3d(ring + slot * C::TILE_BYTES + x * C::BOX_BYTES + lane * rows * 128, map, x * 64, y, z, full + 8 * slot);
        }
        if (j == lo && !is_v && two && !(ok = load_q(1, plane, token + p.tq))) break;
      }
    }
    // drain copies still in flight before the CTA may exit
    if (lane == 0) {
      Abort no_abort{ab.flag + 1};
      if (q_issued0 > 0) mbar_wait(bar_q, (q_issued0 - 1) & 1, p.ctl, no_abort);
      if (q_issued1 > 0) mbar_wait(bar_q + 8, (q_issued1 - 1) & 1, p.ctl, no_abort);
      for (int ps = max(0, issued - C::NR); ps < issued; ++ps)
        if (ps != skipped) mbar_wait(full + 8 * (ps % C::NR), (ps / C::NR) & 1, p.ctl, no_abort);
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------------ MMA issuer (whole warp, one lane elected)
    constexpr uint32_t idesc_s = idesc_bf16(C::BM, C::BN, 0, 0);  // Q, K both K-major
    constexpr uint32_t idesc_pv = idesc_bf16(C::BM, D, 0, 1);     // P from TMEM, V MN-major
    const uint64_t dq0 = sdesc_sw128(sbase + C::Q_OFF, 16, 1024);
    const uint64_t dk0 = sdesc_sw128(sbase + C::RING_OFF, 16, 1024);
    const uint64_t dv0 = sdesc_sw128(sbase + C::RING_OFF + C::NR * C::TILE_BYTES, C::BOX_BYTES, 1024);
    constexpr uint32_t kTile16 = C::TILE_BYTES >> 4, kBox16 = C::BOX_BYTES >> 4;
    const auto wait_k = [&](int n) { return wait_warp(bar_full + 8 * (n % C::NR), (n / C::NR) & 1, p.ctl, ab); };
    const auto wait_v = [&](int n) { return wait_warp(bar_full + 8 * (C::NR + n % C::NR), (n / C::NR) & 1, p.ctl, ab); };
    int q0 = 0, q1 = 0, q_single = 0;  // loads so far of Q tile 0 and 1; the one that the next single tile takes
    int pos = 0;                       // key tiles so far
    int cnt0 = 0, cnt1 = 0, items0 = 0, items1 = 0;  // steps of S, P and O number 0 and 1, items that had some
    // S_t = Q K^T with the query tile q and K number n
    const auto issue_s = [&](int t, int q, int n) {
      const uint64_t a = dq0 + q * kTile16, b = dk0 + (n % C::NR) * kTile16;
#pragma unroll
      for (int x = 0; x < C::NBOX; ++x)
        mma_ss_k64_el(tmem + C::S_COL + t * C::BN, a + x * kBox16, b + x * kBox16, idesc_s, x > 0);
      tc_commit_el(bar_s + 8 * t);
    };
    // O_t += P_t V with V number n, the half written first as soon as it is there; step i of number t's
    const auto issue_pv = [&](int t, int n, int i) -> bool {
      const uint64_t b = dv0 + (n % C::NR) * kTile16;
      const int cnt = t ? cnt1 : cnt0, items = t ? items1 : items0;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (!wait_warp(bar_p + 16 * t + 8 * half, (cnt + i) & 1, p.ctl, ab)) return false;
        // O_t of the item before must have been read out
        if (half == 0 && i == 0 && items > 0 && !wait_warp(bar_oe + 8 * t, (items - 1) & 1, p.ctl, ab)) return false;
        tc_fence_after();
        mma_ts_k64_el(tmem + C::O_COL + t * D, tmem + C::S_COL + t * C::BN + half * 32, b + half * 64 * (128 >> 4), idesc_pv,
                      i > 0 || half > 0 ? 1u : 0u);
      }
      return true;
    };
    const auto free_slot = [&](int ring, int n) { tc_commit_el(bar_empty + 8 * (ring * C::NR + n % C::NR)); };
    // The items' loops have one place each that issues a number's S and P.V (the MMAs take 36 instructions each,
    // and a prologue and an end of their own doubled that); the first steps are only S.
    // Two query tiles: S0 S1 | PV0 S0' | PV1 S1' | ...: the tensor pipe works on one tile while the other's softmax
    // runs.  Tile 0 stops at its own diagonal.
    const auto two_tiles = [&](int n0, int n) -> bool {
#pragma unroll 1
      for (int i = -1; i < n; ++i) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int nt = t ? n : n0;
          if (i >= 0 && i < nt) {
            if (!issue_pv(t, pos + i, i)) return false;
            if (i + 1 == nt) tc_commit_el(bar_o + 8 * t);
            if (t == 1) free_slot(1, pos + i);
          }
          if (i + 1 >= nt) continue;
          if (i < 0 && !wait_warp(bar_q + 8 * t, (t ? q1++ : q0++) & 1, p.ctl, ab)) return false;
          if ((t == 0 || n0 <= i + 1) && !wait_k(pos + i + 1)) return false;
          // (the next V is awaited while P.V keeps the tensor pipe busy; at D = 64 that would hold S back)
          if (D == 128 && t == 1 && i >= 0 && !wait_v(pos + i + 1)) return false;
          tc_fence_after();
          issue_s(t, t, pos + i + 1);
          if (t == 1) free_slot(0, pos + i + 1);
          if (i + 2 == nt) tc_commit_el(bar_qe + 8 * t);  // the Q tile's last S of the item
          if (t == 1 && (D != 128 || i < 0) && !wait_v(pos + i + 1)) return false;
        }
      }
      return true;
    };
    // One query tile: key tile x goes the way of number x % 2.
    const auto one_tile = [&](int n) -> bool {
      const int q = q_single;
      q_single ^= 1;
#pragma unroll 1
      for (int x = -2; x < n; ++x) {
        const int t = x & 1, k = x + 2;
        if (x >= 0) {
          if (!wait_v(pos + x) || !issue_pv(t, pos + x, x >> 1)) return false;
          free_slot(1, pos + x);
          if (k >= n) tc_commit_el(bar_o + 8 * t);
        }
        if (k >= n) continue;
        if (k == 0 && !wait_warp(bar_q + 8 * q, (q ? q1++ : q0++) & 1, p.ctl, ab)) return false;
        if (!wait_k(pos + k)) return false;
        tc_fence_after();
        issue_s(t, q, pos + k);
        free_slot(0, pos + k);
        if (k + 1 == n) tc_commit_el(bar_qe + 8 * q);
      }
      return true;
    };
    while (const Item* rec = take_item()) {
      const int n = rec->n, n0 = rec->n0, n1 = rec->n1;
      const bool two = rec->two;
      give_item();
      if (n == 0) continue;
      if (!(two ? two_tiles(n0, n) : one_tile(n))) break;
      cnt0 += n0;
      cnt1 += n1;
      pos += n;
      items0 += n0 > 0;
      items1 += n1 > 0;
    }
    // wait for every MMA issued above before TMEM may be released
    Abort no_abort{ab.flag + 1};
    tc_commit_el(bar_drain);
    wait_warp(bar_drain, 0, p.ctl, no_abort);
  } else {
    // ------------------------------------------------------------------ softmax
    const int t = warp >> 2;                         // S, P and O number t are this warpgroup's
    const int row_in_tile = (warp & 3) * 32 + lane;  // == TMEM lane
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_tm = tmem + lane_addr + C::S_COL + t * C::BN;
    const uint32_t o_tm = tmem + lane_addr + C::O_COL + t * D;
    const uint32_t my_s = bar_s + 8 * t, my_p = bar_p + 16 * t, my_o = bar_o + 8 * t, my_oe = bar_oe + 8 * t;
    const uint32_t stg = sbase + C::STG_OFF + warp * 4096;
    const uint32_t ml = sbase + C::ML_OFF + row_in_tile * 8;
    const int row_token = row_in_tile / p.gt, row_head = row_in_tile - row_token * p.gt;
    int cnt = 0, items = 0;  // this warpgroup's steps so far, items that had some
    int pos = 0, shared = 0, items1 = 0;  // key tiles so far; single tiles that both had steps of; items of number 1
    bool alive = true;
    while (const Item* rec = alive ? take_item() : nullptr) {
      const Item& it = *rec;
      const int n = t == 0 ? it.n0 : it.n1;
      const int token = it.t0 + (it.two ? t * p.tq : 0) + row_token;
      const bool row = row_token < p.tq && token < it.sq;
      const bool any = __any_sync(0xffffffffu, row);
      const int query = min(token, it.sq - 1);  // (a row that is none: masked like the last)
      const int limit = (p.causal ? max(0, query - it.sq + 1 + it.skv) : it.skv) - it.lo * C::BN;
      // The unit's last tile here, where it reaches past the sequence's keys: what V's rows hold there (other
      // keys, or nothing that was ever written) must not meet P = 0, so they are cleared, by the
      // warps whose P.V comes first.
      const int over = it.skv - (it.lo + it.n - 1) * C::BN;  // keys of the last tile
      const bool clears = over < C::BN && (it.two ? (t == 0 ? it.n0 == it.n : it.n0 < it.n) : t == ((it.n - 1) & 1));
      float m_run = -INFINITY, l_run = 0.f;
#pragma unroll 1
      for (int i = 0; alive && i < n; ++i) {
        const int j = it.two ? i : 2 * i + t;  // key tile
        if (clears && j + 1 == it.n) {
          const int vn = pos + j, slot = vn % C::NR;
          // (S first: it is issued behind the P.V of the tile that had V's slot before, without which V's barrier
          // could be two phases behind, which a wait by parity takes for done)
          alive = wait_warp(my_s, (cnt + i) & 1, p.ctl, ab) && wait_warp(bar_full + 8 * (C::NR + slot), (vn / C::NR) & 1, p.ctl, ab);
          if (!alive) break;
          // (a thread clears its row, from a chunk of its own on: no two lanes of eight meet in a bank)
          const uint32_t v = sbase + C::RING_OFF + (C::NR + slot) * C::TILE_BYTES + row_in_tile * 128;
          if (row_in_tile >= over)
#pragma unroll
            for (int x = 0; x < C::NBOX * 8; ++x) st_shared_v4(v + x / 8 * C::BOX_BYTES + (((x + lane) & 7) << 4), 0, 0, 0, 0);
          fence_proxy_async_smem();
        }
        if (any) {
          alive = chunk_step<D>(s_tm, o_tm, my_s, (cnt + i) & 1, my_p, i == 0, limit - j * C::BN, p.c, m_run, l_run, p.ctl, ab);
        } else if ((alive = wait_warp(my_s, (cnt + i) & 1, p.ctl, ab))) {  // a warp without rows keeps step
          mbar_arrive(my_p);
          mbar_arrive(my_p + 8);
        }
      }
      const bool both = !it.two && it.n1 > 0;
      if (!it.two && t == 1) {
        // the odd key tiles of a single tile: O stays in TMEM, m and l go to the even ones' warps
        if (both) {
          alive = alive && (shared == 0 || wait_warp(bar_mle, (shared - 1) & 1, p.ctl, ab));
          if (alive) {
            st_shared_f2(ml, m_run, l_run);
            mbar_arrive(bar_ml);
            alive = wait_warp(my_o, items & 1, p.ctl, ab);  // (a wait by parity may not miss a phase)
          }
        }
      } else {
        alive = alive && (n == 0 || wait_warp(my_o, items & 1, p.ctl, ab));
        RowSums r{-1, nullptr, m_run, l_run, 1.f, 0.f, n > 0, both, any};
        if (both) {
          alive = alive && wait_warp(bar_o + 8, items1 & 1, p.ctl, ab) && wait_warp(bar_ml, shared & 1, p.ctl, ab);
          if (alive) {
            const float2 other = ld_shared_f2(ml);
            mbar_arrive(bar_mle);
            r.m = fmaxf(m_run, other.x);
            const float base = r.m == -INFINITY ? 0.f : r.m;
            r.w0 = ex2(m_run - base);
            r.w1 = ex2(other.x - base);
            r.l = r.w0 * l_run + r.w1 * other.y;
          }
        }
        tc_fence_after();
        const long long unit_at = static_cast<long long>(it.qb + it.t0) * p.Hq * D;  // its first token's place in O
        if (row) {
          const int head = it.plane * p.gt + row_head;
          r.at = ((token - it.t0) * p.Hq + head) * (D / 8);
          if (p.lse) r.lse_at = p.lse + static_cast<size_t>(head) * p.total_q + it.qb + token;
        }
        if (it.cut()) {
          // (the next record: behind it the numbers of the pieces are there; where a wait gave up, see count_rest)
          alive = alive && wait_warp(bar_rec + 8 * ((rec_n + 1) % C::NREC), ((rec_n + 1) / C::NREC) & 1, p.ctl, ab);
          if (!alive) break;
          finish_piece<D>(p, ln, it, r, unit_at, o_tm, my_oe, bar_oe + 8, stg, warp);
          counted += any;
        } else if (alive && any) {
          finish_unit<D>(p, r, unit_at, o_tm, my_oe, bar_oe + 8, stg);
        } else if (alive && n > 0) {
          release_o(r, my_oe, bar_oe + 8);
        }
      }
      cnt += n;
      items += n > 0;
      pos += it.n;
      shared += both;
      items1 += it.n1 > 0;
      give_item();
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (ab.raised() && warp < 8) count_rest(p, ln, static_cast<int>(start[0]), start[1], warp, counted);
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

bool encode(CUtensorMap* map, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const EncodeTiledFn enc = encode_fn();
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, ones,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// q [total_q, planes, gt, D] in boxes of 64 columns x a plane's heads x a tile's tokens, whose rows land one
// after another as the tile has them.
bool q_map(CUtensorMap* map, const ChunkArgs& a, int gt, int tq) {
  const cuuint64_t row = static_cast<cuuint64_t>(a.D) * 2;
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(a.D), static_cast<cuuint64_t>(gt), static_cast<cuuint64_t>(a.Hq / gt),
                              static_cast<cuuint64_t>(a.total_q)};
  const cuuint64_t strides[3] = {row, row * gt, row * a.Hq};
  const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(gt), 1, static_cast<cuuint32_t>(tq)};
  return encode(map, 4, a.q, dims, strides, box);
}

// A paged cache in boxes of 64 columns x `rows` keys of one kv head:
//   NHD [num_pages, page, Hkv, D] as [keys of all pages, Hkv, D];  HND [num_pages, Hkv, page, D] as [pages x Hkv, page, D]
bool cache_map(CUtensorMap* map, const void* cache, const ChunkArgs& a, int rows) {
  const bool hnd = a.pages.layout == kPagedHND;
  const cuuint64_t row = static_cast<cuuint64_t>(a.D) * 2, inner = hnd ? a.pages.page_size : a.Hkv;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(a.D), inner,
                              static_cast<cuuint64_t>(a.pages.num_pages) * (hnd ? a.Hkv : a.pages.page_size)};
  const cuuint64_t strides[2] = {row, row * inner};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(hnd ? rows : 1), static_cast<cuuint32_t>(hnd ? 1 : rows)};
  return encode(map, 3, cache, dims, strides, box);
}

// Query heads of a plane: the largest divisor of the group that a tile has rows for.
int plane_heads(int group) {
  int gt = group < 128 ? group : 128;
  while (group % gt) --gt;
  return gt;
}

// 32-row groups that a unit of a call with total_q tokens may have.
int row_groups(int total_q, int gt) {
  const int tq = 128 / gt;
  const auto groups = [&](long long tokens) { return static_cast<int>((tokens * gt + 31) / 32); };
  return total_q <= tq ? groups(total_q) : 4 + groups((total_q < 2 * tq ? total_q : 2 * tq) - tq);
}

constexpr size_t kCountBytes = 16384;  // counts of up to 256 CTAs

// 48 bits that no other process has and that memory holds by chance only.
unsigned long long process_tag() {
  static const unsigned long long tag = [] {
    unsigned long long z = static_cast<unsigned long long>(std::chrono::system_clock::now().time_since_epoch().count());
    z = (z ^ z >> 31) * 0x9E3779B97F4A7C15ull;
    z = (z ^ z >> 29) * 0xBF58476D1CE4E5B9ull;
    return (z ^ z >> 32) << 16;
  }();
  return tag;
}

template <int D>
cudaError_t launch_d(const ChunkArgs& a, const KernelCtl& ctl, cudaStream_t stream) {
  using C = ChunkCfg<D>;
  static PerDeviceOnce configured;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  if (!configured.run(dev, [] {
        return cudaFuncSetAttribute(chunk_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES) == cudaSuccess;
      }))
    return cudaErrorInvalidValue;
  const int ctas = sms < 256 ? sms : 256;
  ChunkParams p{};
  p.gt = plane_heads(a.Hq / a.Hkv);
  p.tq = 128 / p.gt;
  p.planes = a.Hq / p.gt;
  p.planes_per_kv = p.planes / a.Hkv;
  const int rows = a.pages.page_size < 64 ? a.pages.page_size : 64;
  CUtensorMap mq, mk, mv;
  if (!q_map(&mq, a, p.gt, p.tq) || !cache_map(&mk, a.k, a, rows) || !cache_map(&mv, a.v, a, rows)) return cudaErrorInvalidValue;
  p.o = static_cast<__nv_bfloat16*>(a.o);
  p.lse = a.lse;
  p.cu_q = a.cu_q;
  p.seqlens = a.seqlens;
  p.table = a.pages.block_table;
  p.groups = row_groups(a.total_q, p.gt);
  char* ws = static_cast<char*>(a.workspace);
  p.count = reinterpret_cast<unsigned long long*>(ws);
  p.part_ml = reinterpret_cast<float2*>(ws + kCountBytes);
  p.part = reinterpret_cast<float*>(ws + kCountBytes + static_cast<size_t>(2 * ctas) * p.groups * 32 * sizeof(float2));
  p.tag = process_tag();
  p.B = a.B;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.total_q = a.total_q;
  p.causal = a.causal;
  p.num_pages = a.pages.num_pages;
  p.page = a.pages.page_size;
  p.max_pages = a.pages.max_pages;
  p.hnd = a.pages.layout == kPagedHND;
  p.c = a.scale * kLog2e;
  p.ctl = ctl;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = C::BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, chunk_kernel<D>, mq, mk, mv, p);
}

}  // namespace

size_t chunk_workspace_bytes(int Hq, int Hkv, int total_q, int D, int sms) {
  const size_t slots = 2 * static_cast<size_t>(sms < 256 ? sms : 256);
  return kCountBytes + slots * row_groups(total_q, plane_heads(Hq / Hkv)) * 32 * (sizeof(float2) + D * sizeof(float));
}

cudaError_t launch_chunk_paged(const ChunkArgs& a, const KernelCtl& ctl, cudaStream_t stream) {
  return a.D == 128 ? launch_d<128>(a, ctl, stream) : launch_d<64>(a, ctl, stream);
}

}  // namespace loom
