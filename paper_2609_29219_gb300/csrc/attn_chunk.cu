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
// that it sees.
//
// Dealing.  All units lie on one line, in order, each as long as its modelled cost: kUnitCost and a
// weight per key.  CTA c of G takes the stretch [W c / G, W (c + 1) / G) of the line's W, cut to
// whole key tiles of the units it starts and ends in.  So the CTAs finish together for any mixture of
// prompts and single tokens, no list of items is made or stored, and nothing depends on timing: the
// offsets' prefix sum and a binary search give each CTA its first unit.  A unit that lies in one stretch
// is finished there.  The pieces of a cut one go to the workspace in 32 bits; the last warp to bring its
// rows' piece joins all of them in the pieces' order.
//
// What bounds it: many queries, the tensor cores, as the prefill kernel, whose step this one repeats
// (two query tiles alternate on the tensor pipe, P in TMEM); few queries, the cache's bandwidth.
#include <cuda.h>
#include <cuda_bf16.h>

#include <atomic>
#include <chrono>
#include <mutex>

#include "chunk.h"
#include "ptx.cuh"

namespace loom {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRescaleThreshold = 8.0f;  // base-2 units; P <= 2^8 between rescales

// The line's units.  A key of a pair of tiles costs kKeyCost2, of a single tile kKeyCost1; a unit kUnitCost more.
constexpr int kKeyCost2 = 8, kKeyCost1 = 6, kUnitCost = 1024;

template <int D>
struct ChunkCfg {
  static constexpr int BM = 128, BN = 128;
  static constexpr int NSLOT = D == 128 ? 4 : 10;   // K/V ring slots
  static constexpr int NKE = NSLOT / 2;
  static constexpr int THREADS = 320;               // 8 softmax warps, loader, MMA
  static constexpr int NBOX = D / 64;               // 128-byte swizzled boxes per row of a tile
  static constexpr uint32_t BOX_BYTES = BM * 128;
  static constexpr uint32_t TILE_BYTES = NBOX * BOX_BYTES;
  static constexpr uint32_t Q_OFF = 0;
  static constexpr uint32_t RING_OFF = 2 * TILE_BYTES;
  static constexpr uint32_t STG_OFF = RING_OFF + NSLOT * TILE_BYTES;  // 4 KB for each softmax warp
  static constexpr uint32_t BAR_OFF = STG_OFF + 8 * 4096;
  // q[2], qe[2], full[NSLOT], empty[NKE], s[2], p[2][2], o[2], oe[2], drain
  static constexpr int NBAR = 4 + NSLOT + NKE + 2 + 4 + 2 + 2 + 1;
  static constexpr uint32_t START_OFF = BAR_OFF + NBAR * 8;  // where this CTA's stretch begins (Start)
  static constexpr uint32_t SUM_OFF = START_OFF + 32;        // the scan's sums, one per warp
  static constexpr uint32_t TMEM_PTR_OFF = SUM_OFF + 16 * 8;
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
  unsigned long long tag;     // of this launch, in the upper 48 bits of a count
  int groups;                 // 32-row groups of a unit that the workspace has room for
  int B, Hq, total_q, causal;
  int gt, planes, planes_per_kv, tq;  // heads of a plane, planes of a token, tokens of a tile
  int num_pages, page, max_pages, hnd, Hkv;
  float c;  // scale log2(e)
  KernelCtl ctl;
};

// ---------------------------------------------------------------- the line of work
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
  s.pairs = static_cast<int>((static_cast<long long>(s.sq) + 2 * p.tq - 1) / (2 * p.tq));
  return s;
}
// Keys that the queries before token `end` of a sequence see.
__device__ __forceinline__ int keys_until(const ChunkParams& p, const Seq& s, long long end) {
  if (!p.causal) return s.skv;
  return static_cast<int>(max(0ll, min(end, static_cast<long long>(s.sq)) + s.skv - s.sq));
}
__device__ __forceinline__ int key_cost(const ChunkParams& p, const Seq& s, int pair) {
  return s.sq - 2ll * p.tq * pair > p.tq ? kKeyCost2 : kKeyCost1;
}
__device__ __forceinline__ long long unit_cost(const ChunkParams& p, const Seq& s, int pair) {
  return kUnitCost + static_cast<long long>(key_cost(p, s, pair)) * keys_until(p, s, 2ll * p.tq * (pair + 1));
}
// Cost of a plane's pairs before pair i < pairs (all of them of two tiles, none past the sequence's end).
__device__ __forceinline__ long long cost_before(const ChunkParams& p, const Seq& s, int i) {
  long long keys = static_cast<long long>(i) * s.skv;
  if (p.causal) {
    // pair j sees off + step (j + 1) keys, from the first j where that is positive
    const long long step = 2ll * p.tq, off = static_cast<long long>(s.skv) - s.sq;
    const long long j0 = off >= 0 ? 0 : -off / step;
    const long long n = i - j0;
    keys = n > 0 ? n * off + step * ((j0 + 1 + i) * n / 2) : 0;
  }
  return static_cast<long long>(i) * kUnitCost + kKeyCost2 * keys;
}
__device__ __forceinline__ long long plane_cost(const ChunkParams& p, const Seq& s) {
  return s.pairs ? cost_before(p, s, s.pairs - 1) + unit_cost(p, s, s.pairs - 1) : 0;
}
// The line's place where CTA c of G begins.
__device__ __forceinline__ long long bound_of(long long W, int G, int c) {
  return W / G * c + static_cast<int>(W % G) * c / G;
}
// Key tiles of a unit that lie before the place d > 0 behind its beginning.
__device__ __forceinline__ int tiles_before(long long d, int key, int tiles) {
  d -= kUnitCost;
  if (d <= 0) return 0;
  const long long t = (d + key * 128 - 1) / (key * 128);
  return t < tiles ? static_cast<int>(t) : tiles;
}

// What a CTA knows of its stretch.
struct Line {
  long long W, x0, x1;
  int G;
};
// A place on the line: unit `pair` of a plane of sequence b, which begins at `at`.
struct Walk {
  int b, plane, pair;
  long long at;
  Seq s;
};
// A unit, or the piece of it that this CTA has.
struct Item {
  int b, plane, t0, qb, sq, skv;  // t0: its first token within the sequence
  long long at, cost;             // its place on the line
  int key, tiles;                 // a key's cost, all its key tiles
  int lo, n0, n;                  // first key tile, key tiles of tile 0 and of tile 1 here
  bool two;                       // it has a tile 0 (a single tile is tile 1)
  __device__ __forceinline__ bool cut() const { return n < tiles; }
};

// The CTA's next piece, and the walk behind it; false past the stretch's end.
__device__ __forceinline__ bool next_item(const ChunkParams& p, const Line& ln, Walk& w, Item& it) {
  while (w.b < p.B && w.at < ln.x1) {
    const long long step = 2ll * p.tq;
    it.b = w.b;
    it.plane = w.plane;
    it.qb = w.s.qb;
    it.sq = w.s.sq;
    it.skv = w.s.skv;
    it.t0 = static_cast<int>(step * w.pair);
    it.two = w.s.sq - it.t0 > p.tq;
    it.key = it.two ? kKeyCost2 : kKeyCost1;
    const int keys = keys_until(p, w.s, step * (w.pair + 1));
    it.tiles = (keys + 127) / 128;
    it.at = w.at;
    it.cost = kUnitCost + static_cast<long long>(it.key) * keys;
    it.lo = ln.x0 > it.at ? tiles_before(ln.x0 - it.at, it.key, it.tiles) : 0;
    const int hi = ln.x1 < it.at + it.cost ? tiles_before(ln.x1 - it.at, it.key, it.tiles) : it.tiles;
    it.n = hi - it.lo;
    it.n0 = it.two ? max(0, min(hi, (keys_until(p, w.s, it.t0 + p.tq) + 127) / 128) - it.lo) : 0;
    w.at += it.cost;
    if (++w.pair == w.s.pairs) {
      w.pair = 0;
      if (++w.plane == p.planes) {
        w.plane = 0;
        while (++w.b < p.B) {
          w.s = load_seq(p, w.b);
          if (w.s.pairs) break;
        }
      }
    }
    // (a unit without keys belongs to the CTA in whose stretch it begins)
    if (it.n > 0 || (it.tiles == 0 && ln.x0 <= it.at)) return true;
  }
  return false;
}

// The pieces of a cut unit: calls f(slot) with each piece's place in the workspace, in order, and returns
// the CTA that has the first.  The first piece is its CTA's last unit, the others' are their CTAs' first.
template <class F>
__device__ __forceinline__ int for_pieces(const Line& ln, const Item& it, F f) {
  int c = min(ln.G - 1, static_cast<int>(static_cast<double>(it.at) / static_cast<double>(ln.W) * ln.G));
  while (c > 0 && bound_of(ln.W, ln.G, c) > it.at) --c;
  while (c + 1 < ln.G && bound_of(ln.W, ln.G, c + 1) <= it.at) ++c;
  int first = -1;
  for (int lo = 0; lo < it.tiles && c < ln.G; ++c) {
    const long long end = c + 1 < ln.G ? bound_of(ln.W, ln.G, c + 1) : ln.W;
    const int hi = end < it.at + it.cost ? tiles_before(end - it.at, it.key, it.tiles) : it.tiles;
    if (hi > lo) {
      f(lo == 0 ? 2 * c + 1 : 2 * c);
      if (first < 0) first = c;
    }
    lo = hi;
  }
  return first;
}

// ---------------------------------------------------------------- softmax
// One online-softmax step of one query row (this thread's TMEM lane) over a 128-key tile of S in TMEM at
// s_tm: mask keys >= limit, move the running max lazily, write P = 2^(S c - m) as bf16 over the first
// half of S's columns in two halves (arriving on bar_p and bar_p + 8 after each), rescale O at o_tm where
// the max moved, and add to the row's sum.  S is only ready after the tile's previous P.V (issued before it by
// the same warp), so the rescale needs no wait.  before_p() runs before the first arrival.
template <int D, class F>
__device__ __forceinline__ bool chunk_step(uint32_t s_tm, uint32_t o_tm, uint32_t bar_s, uint32_t par_s, uint32_t bar_p,
                                           bool first, int limit, float c, float& m_run, float& l_run, const KernelCtl& ctl,
                                           const Abort& ab, F before_p) {
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
    if (half == 0 && !before_p()) return false;
    tc_fence_before();
    mbar_arrive(bar_p + 8 * half);
  }
  const uint64_t a01 = add2(add2(acc[0], acc[1]), add2(acc[2], acc[3]));
  l_run = l_run * alpha + (f2lo(a01) + f2hi(a01));
  return true;
}

// 64 columns of this warp's 32 rows, packed bf16 pairs of each lane's own row in w, to the rows' places in O (my_at:
// this row's first column, in elements; < 0: not a row): through the warp's 4 KB of shared memory, so that
// a store writes whole 128-byte lines (from the lanes' own rows it would touch 32 lines).
__device__ __forceinline__ void store_rows(uint32_t stg, const uint32_t* w, long long my_at, __nv_bfloat16* o) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c = 0; c < 8; ++c)
    st_shared_v4(stg + lane * 128 + ((c ^ (lane & 7)) << 4), w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = k * 4 + lane / 8, j = lane % 8;
    const long long at = __shfl_sync(0xffffffffu, my_at, r);
    const uint4 v = ld_shared_v4(stg + r * 128 + ((j ^ (r & 7)) << 4));
    if (at >= 0) reinterpret_cast<uint4*>(o + at)[j] = v;
  }
  __syncwarp();
}

__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2; }

// Counts one more piece of a 32-row group: how many have come (tag: see ChunkParams; a count of another launch, or
// whatever else the workspace held, counts as none).
__device__ __forceinline__ int count_piece(unsigned long long* at, unsigned long long tag) {
  unsigned long long seen = *reinterpret_cast<volatile unsigned long long*>(at), mine;
  while (true) {
    mine = ((seen ^ tag) >> 16 ? tag : seen) + 1;
    const unsigned long long was = atomicCAS(at, seen, mine);
    if (was == seen) return static_cast<int>(mine & 0xffff);
    seen = was;
  }
}

// What a cut unit's piece has to say of one query row (this thread's TMEM lane).
struct PieceRow {
  long long at;    // its place in O, in elements
  float* lse_at;   // and in LSE, or null
  float m, l;
  bool has_tiles;  // this CTA walked key tiles of the row's tile
  bool row, any;   // it is a row; the warp has one
  bool alive;      // no wait has given up
};

// A piece of a cut unit: this warp's 32 rows go to the workspace, each 16 bytes of a row beside the other lanes'
// (one store: 512 bytes in a row).  The last warp to bring its piece of the rows joins all of them, in the
// pieces' order.  A CTA that gave up counts its pieces all the same, so that the counts are whole again at the
// launch's end.  Not inlined: it is rare, and its registers would spill the softmax loop's.
template <int D>
__device__ __noinline__ void finish_piece(const ChunkParams& p, const Line& ln, const Item& it, const PieceRow r, uint32_t o_tm,
                                          uint32_t bar_oe, uint32_t stg, int warp) {
  const int lane = threadIdx.x & 31, group = it.two ? warp : warp & 3;
  const auto part_of = [&](int slot) {
    return reinterpret_cast<float4*>(p.part) + (static_cast<size_t>(slot) * p.groups + group) * (D / 4) * 32 + lane;
  };
  const auto ml_of = [&](int slot) { return p.part_ml + (static_cast<size_t>(slot) * p.groups + group) * 32 + lane; };
  const int slot = it.lo == 0 ? 2 * static_cast<int>(blockIdx.x) + 1 : 2 * static_cast<int>(blockIdx.x);
  if (r.alive && r.any) {
    float4* mine = part_of(slot);
    if (r.has_tiles) {
#pragma unroll
      for (int ch = 0; ch < D / 32; ++ch) {
        uint32_t rr[32];
        tmem_ld32(o_tm + ch * 32, rr);
        tmem_wait_ld();
        reg_fence32(rr);
        if (r.row)
#pragma unroll
          for (int u = 0; u < 8; ++u)
            mine[(ch * 8 + u) * 32] = make_float4(__uint_as_float(rr[4 * u]), __uint_as_float(rr[4 * u + 1]),
                                                  __uint_as_float(rr[4 * u + 2]), __uint_as_float(rr[4 * u + 3]));
      }
    }
    if (r.row) *ml_of(slot) = make_float2(r.m, r.has_tiles ? r.l : -1.f);
  }
  if (r.alive && r.has_tiles) {
    tc_fence_before();
    mbar_arrive(bar_oe);
  }
  if (!r.any) return;
  int pieces = 0;
  const int first = for_pieces(ln, it, [&](int) { ++pieces; });
  unsigned long long* count = p.count + static_cast<size_t>(first) * 8 + warp;
  __threadfence();
  __syncwarp();
  int come = 0;
  if (lane == 0) {
    come = count_piece(count, p.tag);
    if (come == pieces) *reinterpret_cast<volatile unsigned long long*>(count) = p.tag;
  }
  come = __shfl_sync(0xffffffffu, come, 0);
  if (!r.alive || come != pieces) return;
  __syncwarp();
  __threadfence();
  float M = -INFINITY, l = 0.f;
  for_pieces(ln, it, [&](int s) {
    if (r.row) M = fmaxf(M, __ldcg(ml_of(s)).x);
  });
  const float base = M == -INFINITY ? 0.f : M;
  for_pieces(ln, it, [&](int s) {
    if (!r.row) return;
    const float2 ml = __ldcg(ml_of(s));
    if (!(ml.y < 0.f)) l = fmaf(ex2(ml.x - base), ml.y, l);
  });
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
  for (int h = 0; h < D / 64; ++h) {
    float acc[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) acc[i] = 0.f;
    for_pieces(ln, it, [&](int s) {
      if (!r.row) return;
      const float2 ml = __ldcg(ml_of(s));
      if (ml.y < 0.f) return;
      const float weight = ex2(ml.x - base);
      const float4* from = part_of(s) + h * 16 * 32;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float4 v = __ldcg(from + i * 32);
        acc[4 * i] = fmaf(weight, v.x, acc[4 * i]);
        acc[4 * i + 1] = fmaf(weight, v.y, acc[4 * i + 1]);
        acc[4 * i + 2] = fmaf(weight, v.z, acc[4 * i + 2]);
        acc[4 * i + 3] = fmaf(weight, v.w, acc[4 * i + 3]);
      }
    });
    uint32_t w[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) w[i] = pack_bf16x2(acc[2 * i] * inv, acc[2 * i + 1] * inv);
    store_rows(stg, w, r.at < 0 ? r.at : r.at + 64 * h, p.o);
  }
  if (r.lse_at) *r.lse_at = row_lse(M, l);
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
  const uint32_t bar_full = bar_qe + 16;               // [NSLOT]
  const uint32_t bar_empty = bar_full + 8 * C::NSLOT;  // [NKE] K number n and the V before it are no longer read
  const uint32_t bar_s = bar_empty + 8 * C::NKE;       // [2] S_t ready
  const uint32_t bar_p = bar_s + 16;                   // [2][2] half h of P_t written (h = 0: and O_t rescaled)
  const uint32_t bar_o = bar_p + 32;                   // [2] O_t of the item complete
  const uint32_t bar_oe = bar_o + 16;                  // [2] O_t read out
  const uint32_t bar_drain = bar_oe + 16;
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
    for (int s = 0; s < C::NSLOT; ++s) mbar_init(bar_full + 8 * s, 1);
    for (int n = 0; n < C::NKE; ++n) mbar_init(bar_empty + 8 * n, 1);
    mbar_init(bar_drain, 1);
    *ab.flag = 0;
    *(ab.flag + 1) = 0;
    fence_barrier_init();
  }
  // rows of the Q tiles that no load fills (a tile has tq gt rows): zeros, so that their scores are too
  {
    const int rows = p.tq * p.gt, n = (C::BM - rows) * 8;
    for (int i = threadIdx.x; i < 2 * C::NBOX * n; i += C::THREADS)
      st_shared_v4(sbase + C::Q_OFF + i / n * C::BOX_BYTES + rows * 128 + i % n * 16, 0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  if (warp == 9) tmem_alloc(smem_u32(tmem_ptr), 512);
  // The set-up above touches no global memory; from here on the previous kernel's writes must be visible.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");

  // The line's length, and the sequence in which this CTA's stretch begins: a prefix sum over the sequences.
  Line ln;
  Walk walk;
  {
    volatile long long* sums = reinterpret_cast<volatile long long*>(smem + C::SUM_OFF);
    volatile long long* start = reinterpret_cast<volatile long long*>(smem + C::START_OFF);
    constexpr int kWarps = C::THREADS / 32;
    ln.G = static_cast<int>(gridDim.x);
    ln.W = ln.x0 = ln.x1 = 0;
    const bool one = p.B <= C::THREADS;
    // (one round: the sum of all and this CTA's sequence from the same scan; else a round for each)
    for (int round = 0; round < (one ? 1 : 2); ++round) {
      long long before = 0;
      for (int b0 = 0; b0 < p.B; b0 += C::THREADS) {
        const int b = b0 + static_cast<int>(threadIdx.x);
        long long cost = 0;
        if (b < p.B) cost = p.planes * plane_cost(p, load_seq(p, b));
        long long x = cost;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const long long y = __shfl_up_sync(0xffffffffu, x, d);
          if (lane >= d) x += y;
        }
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        long long all = 0;
        x += before - cost;
        for (int i = 0; i < kWarps; ++i) {
          const long long y = sums[i];
          if (i < warp) x += y;
          all += y;
        }
        if (one) {
          ln.W = all;
          ln.x0 = bound_of(ln.W, ln.G, blockIdx.x);
        }
        if ((one || round == 1) && x <= ln.x0 && ln.x0 < x + cost) {
          start[0] = b;
          start[1] = x;
        }
        before += all;
        __syncthreads();
      }
      if (!one && round == 0) {
        ln.W = before;
        ln.x0 = bound_of(ln.W, ln.G, blockIdx.x);
      }
    }
    ln.x1 = static_cast<int>(blockIdx.x) + 1 < ln.G ? bound_of(ln.W, ln.G, blockIdx.x + 1) : ln.W;
    walk.b = p.B;
    if (ln.x0 < ln.x1) {
      walk.b = static_cast<int>(start[0]);
      walk.s = load_seq(p, walk.b);
      const long long plane = plane_cost(p, walk.s), in = ln.x0 - start[1];
      walk.plane = static_cast<int>(in / plane);
      const long long r = in - walk.plane * plane;
      int lo = 0, hi = walk.s.pairs;  // the last pair that begins at r or before
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (cost_before(p, walk.s, mid) <= r)
          lo = mid;
        else
          hi = mid;
      }
      walk.pair = lo;
      walk.at = start[1] + walk.plane * plane + cost_before(p, walk.s, lo);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_ptr;
  Item it{};

  if (warp == 8) {
    // ------------------------------------------------------------------ loader (whole warp)
    // Lane 0 waits and expects; a tile's pieces of min(page, 64) keys are looked up and copied by one lane each.
    if (lane == 0) {
      prefetch_tensormap(&tm_q);
      prefetch_tensormap(&tm_k);
      prefetch_tensormap(&tm_v);
    }
    int pos = 0, issued = 0, skipped = -1, q_issued[2] = {0, 0};
    bool ok = true;
    const int rows = min(p.page, 64);
    const uint32_t q_bytes = static_cast<uint32_t>(C::NBOX * p.tq * p.gt * 128);
    const auto load_q = [&](int t) -> bool {
      const int n = q_issued[t];
      if (n > 0 && !mbar_wait_warp(bar_qe + 8 * t, (n - 1) & 1, p.ctl, ab)) return false;
      if (lane == 0) {
        mbar_expect_tx(bar_q + 8 * t, q_bytes);
        const int token = it.qb + it.t0 + (it.two && t == 1 ? p.tq : 0);
        for (int x = 0; x < C::NBOX; ++x)
          tma_load_4d(sbase + C::Q_OFF + t * C::TILE_BYTES + x * C::BOX_BYTES, &tm_q, x * 64, 0, it.plane, token, bar_q + 8 * t);
      }
      __syncwarp();
      q_issued[t] = n + 1;
      return true;
    };
    while (ok && next_item(p, ln, walk, it)) {
      if (it.n == 0) continue;  // no keys: nothing to load
      const int32_t* table = p.table + static_cast<size_t>(it.b) * p.max_pages;
      // the page of this lane's piece of key tile j (none past the sequence's keys)
      const auto page_of = [&](int j) {
        const int key = j * C::BN + lane * rows;
        return lane * rows < C::BN && key < it.skv ? table[key / p.page] : -1;
      };
      int page = page_of(it.lo);
      if (!(ok = load_q(it.n0 > 0 ? 0 : 1))) break;
      const int hk = it.plane / p.planes_per_kv;
      for (int jj = 0; jj < 2 * it.n; ++jj, ++pos) {  // K_0, [Q_1], V_0, K_1, V_1, ...
        if (jj == 1 && it.n0 > 0 && !(ok = load_q(1))) break;
        const int slot = pos % C::NSLOT;
        // the slot's last tile, at position pos - NSLOT, is released with K number n
        if (pos >= C::NSLOT) {
          const int n = (pos - C::NSLOT + 1) >> 1;
          if (!(ok = mbar_wait_warp(bar_empty + 8 * (n % C::NKE), (n / C::NKE) & 1, p.ctl, ab))) break;
        }
        issued = pos + 1;
        if (p.ctl.inject == 5 && pos == 2) {  // test hook: never load this tile
          skipped = pos;
          continue;
        }
        const int j = it.lo + (jj >> 1), key0 = j * C::BN;
        const int pieces = (min(C::BN, it.skv - key0) + rows - 1) / rows;
        if (lane == 0) mbar_expect_tx(bar_full + 8 * slot, static_cast<uint32_t>(C::NBOX * pieces * rows * 128));
        __syncwarp();
        if (lane < pieces) {
          // NHD view [keys of all pages, Hkv, D]: (dim, kv head, key); HND view [pages x Hkv, page, D]:
          // (dim, row in page, page x Hkv + kv head).  A page that there is not: past the end, which reads as zeros.
          const int key = key0 + lane * rows, in = key % p.page;
          const bool bad = page < 0 || page >= p.num_pages;
          const int y = p.hnd ? in : hk;
          const int z = p.hnd ? (bad ? p.num_pages * p.Hkv : page * p.Hkv + hk) : (bad ? p.num_pages * p.page : page * p.page + in);
          const CUtensorMap* map = (jj & 1) ? &tm_v : &tm_k;
#pragma unroll
          for (int x = 0; x < C::NBOX; ++x)
            tma_load_3d(sbase + C::RING_OFF + slot * C::TILE_BYTES + x * C::BOX_BYTES + lane * rows * 128, map, x * 64, y, z,
                        bar_full + 8 * slot);
        }
        if ((jj & 1) && j + 1 < it.lo + it.n) page = page_of(j + 1);
      }
    }
    // drain copies still in flight before the CTA may exit
    if (lane == 0) {
      Abort no_abort{ab.flag + 1};
      for (int t = 0; t < 2; ++t)
        if (q_issued[t] > 0) mbar_wait(bar_q + 8 * t, (q_issued[t] - 1) & 1, p.ctl, no_abort);
      for (int ps = max(0, issued - C::NSLOT); ps < issued; ++ps)
        if (ps != skipped) mbar_wait(bar_full + 8 * (ps % C::NSLOT), (ps / C::NSLOT) & 1, p.ctl, no_abort);
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------------ MMA issuer (whole warp, one lane elected)
    constexpr uint32_t idesc_s = idesc_bf16(C::BM, C::BN, 0, 0);  // Q, K both K-major
    constexpr uint32_t idesc_pv = idesc_bf16(C::BM, D, 0, 1);     // P from TMEM, V MN-major
    const uint64_t dq0 = sdesc_sw128(sbase + C::Q_OFF, 16, 1024);
    const uint64_t dk0 = sdesc_sw128(sbase + C::RING_OFF, 16, 1024);
    const uint64_t dv0 = sdesc_sw128(sbase + C::RING_OFF, C::BOX_BYTES, 1024);
    constexpr uint32_t kTile16 = C::TILE_BYTES >> 4, kBox16 = C::BOX_BYTES >> 4;
    const auto wait_slot = [&](int ps) {
      return mbar_wait_warp(bar_full + 8 * (ps % C::NSLOT), (ps / C::NSLOT) & 1, p.ctl, ab);
    };
    const auto issue_s = [&](int t, int kpos) {
      const uint64_t a = dq0 + t * kTile16, b = dk0 + (kpos % C::NSLOT) * kTile16;
#pragma unroll
      for (int x = 0; x < C::NBOX; ++x)
        mma_ss_k64_el(tmem + C::S_COL + t * C::BN, a + x * kBox16, b + x * kBox16, idesc_s, x > 0);
    };
    const auto issue_pv = [&](int t, int vpos, bool acc, int half) {
      const uint64_t b = dv0 + (vpos % C::NSLOT) * kTile16 + half * 64 * (128 >> 4);
      mma_ts_k64_el(tmem + C::O_COL + t * D, tmem + C::S_COL + t * C::BN + half * 32, b, idesc_pv, acc ? 1u : 0u);
    };
    int pos = 0, cnt0 = 0, cnt1 = 0;  // ring position of K_0; S/P uses so far per tile
    int n0 = 0, n1 = 0;               // items so far that had a tile 0, a tile 1
    bool ok = true;
    while (ok && next_item(p, ln, walk, it)) {
      const int nt0 = it.n0, nt = it.n;
      if (nt == 0) continue;
      if (nt0 > 0) {
        if (!(ok = mbar_wait_warp(bar_q, n0 & 1, p.ctl, ab) && wait_slot(pos))) break;
        tc_fence_after();
        issue_s(0, pos);
        tc_commit_el(bar_s);
        if (nt0 == 1) tc_commit_el(bar_qe);  // every S of tile 0 issued
      }
      if (!(ok = mbar_wait_warp(bar_q + 8, n1 & 1, p.ctl, ab) && (nt0 > 0 || wait_slot(pos)))) break;
      tc_fence_after();
      issue_s(1, pos);
      tc_commit_el(bar_s + 8);
      tc_commit_el(bar_empty + 8 * ((pos >> 1) % C::NKE));
      if (!(ok = wait_slot(pos + 1))) break;
      if (nt == 1) tc_commit_el(bar_qe + 8);  // every S of tile 1 issued
      for (int j = 0; j < nt; ++j) {
        const int vpos = pos + 2 * j + 1, kpos = pos + 2 * j + 2;
        const bool more = j + 1 < nt;
        if (j < nt0) {  // query tile 0 stops at its own diagonal
          if (!(ok = mbar_wait_warp(bar_p, (cnt0 + j) & 1, p.ctl, ab))) break;
          // O_0 of the previous item must have been read out
          if (j == 0 && n0 > 0 && !(ok = mbar_wait_warp(bar_oe, (n0 - 1) & 1, p.ctl, ab))) break;
          tc_fence_after();
          issue_pv(0, vpos, j > 0, 0);
          if (!(ok = mbar_wait_warp(bar_p + 8, (cnt0 + j) & 1, p.ctl, ab))) break;
          tc_fence_after();
          issue_pv(0, vpos, true, 1);
          if (j + 1 == nt0) tc_commit_el(bar_o);
        }
        if (more) {
          if (!(ok = wait_slot(kpos))) break;
          tc_fence_after();
          if (j + 1 < nt0) {
            issue_s(0, kpos);
            tc_commit_el(bar_s);
            if (j + 2 == nt0) tc_commit_el(bar_qe);  // tile 0's last S of the item
          }
        }
        if (!(ok = mbar_wait_warp(bar_p + 16, (cnt1 + j) & 1, p.ctl, ab))) break;
        if (j == 0 && n1 > 0 && !(ok = mbar_wait_warp(bar_oe + 8, (n1 - 1) & 1, p.ctl, ab))) break;
        tc_fence_after();
        issue_pv(1, vpos, j > 0, 0);
        if (!(ok = mbar_wait_warp(bar_p + 24, (cnt1 + j) & 1, p.ctl, ab))) break;
        tc_fence_after();
        issue_pv(1, vpos, true, 1);
        if (!more) {
          tc_commit_el(bar_o + 8);
        } else {
          // (the next V is awaited while P.V keeps the tensor pipe busy; at D = 64 that would hold S back)
          if (D == 128 && !(ok = wait_slot(vpos + 2))) break;
          issue_s(1, kpos);
          tc_commit_el(bar_s + 8);
          tc_commit_el(bar_empty + 8 * ((kpos >> 1) % C::NKE));
          if (D != 128 && !(ok = wait_slot(vpos + 2))) break;
          if (j + 2 == nt) tc_commit_el(bar_qe + 8);  // tile 1's last S of the item
        }
      }
      if (!ok) break;
      cnt0 += nt0;
      cnt1 += nt;
      pos += 2 * nt;
      n0 += nt0 > 0;
      ++n1;
    }
    // wait for every MMA issued above before TMEM may be released
    Abort no_abort{ab.flag + 1};
    tc_commit_el(bar_drain);
    mbar_wait_warp(bar_drain, 0, p.ctl, no_abort);
  } else {
    // ------------------------------------------------------------------ softmax
    const int t = warp >> 2;                         // query tile of this warpgroup
    const int row_in_tile = (warp & 3) * 32 + lane;  // == TMEM lane
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_tm = tmem + lane_addr + C::S_COL + t * C::BN;
    const uint32_t o_tm = tmem + lane_addr + C::O_COL + t * D;
    const uint32_t my_s = bar_s + 8 * t, my_p = bar_p + 16 * t, my_o = bar_o + 8 * t, my_oe = bar_oe + 8 * t;
    const uint32_t stg = sbase + C::STG_OFF + warp * 4096;
    const int row_token = row_in_tile / p.gt, row_head = row_in_tile - row_token * p.gt;
    int cnt = 0, items = 0;  // S tiles of this query tile so far, items that had it
    int pos = 0;             // ring position of the item's K_0
    bool alive = true;
    while (next_item(p, ln, walk, it)) {
      const int n = t == 0 ? it.n0 : it.n;
      const int first_token = it.t0 + (it.two && t == 1 ? p.tq : 0);
      const bool has_tile = t == 1 || it.two;
      const int token = first_token + row_token;
      const bool row = has_tile && row_token < p.tq && token < it.sq;
      const bool any = __any_sync(0xffffffffu, row);
      const int query = min(token, it.sq - 1);  // (a row that is none: masked like the last)
      const int limit = (p.causal ? max(0, query + it.skv - it.sq + 1) : it.skv) - it.lo * C::BN;
      // The unit's last tile here, where it reaches past the sequence's keys: what V's rows hold there (other
      // keys, or nothing that was ever written) must not meet P = 0, so they are cleared, by the
      // warps of tile 0 if it takes part in the step, which P.V of tile 1 follows.
      const int over = it.skv - (it.lo + it.n - 1) * C::BN;  // keys of the last tile
      const bool clears = over < C::BN && (t == 0 ? it.n0 == it.n : it.n0 < it.n);
      float m_run = -INFINITY, l_run = 0.f;
      for (int j = 0; alive && j < n; ++j) {
        const auto before_p = [&]() -> bool {
          if (!clears || j + 1 < it.n) return true;
          const int vpos = pos + 2 * j + 1, slot = vpos % C::NSLOT;
          if (!mbar_wait_warp(bar_full + 8 * slot, (vpos / C::NSLOT) & 1, p.ctl, ab)) return false;
          const uint32_t v = sbase + C::RING_OFF + slot * C::TILE_BYTES;
          const int chunks = (C::BN - over) * 8;
          for (int i = row_in_tile; i < C::NBOX * chunks; i += C::BM)
            st_shared_v4(v + i / chunks * C::BOX_BYTES + over * 128 + i % chunks * 16, 0, 0, 0, 0);
          fence_proxy_async_smem();
          return true;
        };
        if (any) {
          alive = chunk_step<D>(s_tm, o_tm, my_s, (cnt + j) & 1, my_p, j == 0, limit - j * C::BN, p.c, m_run, l_run, p.ctl, ab,
                                before_p);
        } else if (mbar_wait_warp(my_s, (cnt + j) & 1, p.ctl, ab) && before_p()) {  // a warp without rows keeps step
          mbar_arrive(my_p);
          mbar_arrive(my_p + 8);
        } else {
          alive = false;
        }
      }
      alive = alive && (n == 0 || mbar_wait_warp(my_o, items & 1, p.ctl, ab));
      tc_fence_after();
      const int head = it.plane * p.gt + row_head;
      const long long at = row ? (static_cast<long long>(it.qb + token) * p.Hq + head) * D : -1;
      float* lse_at = row && p.lse ? p.lse + static_cast<size_t>(head) * p.total_q + it.qb + token : nullptr;
      if (!it.cut()) {
        if (alive && any) {
          const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
          const uint64_t inv2 = f2(inv, inv);
          uint32_t w[D / 2];
          if (n > 0) {
#pragma unroll
            for (int ch = 0; ch < D / 32; ch += 2) {
              uint32_t rr[2][32];
              tmem_ld32(o_tm + ch * 32, rr[0]);
              tmem_ld32(o_tm + ch * 32 + 32, rr[1]);
              tmem_wait_ld();
              reg_fence32(rr[0]);
              reg_fence32(rr[1]);
#pragma unroll
              for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  const uint64_t x = mul2(f2(__uint_as_float(rr[u][2 * i]), __uint_as_float(rr[u][2 * i + 1])), inv2);
                  w[(ch + u) * 16 + i] = pack_bf16x2(f2lo(x), f2hi(x));
                }
            }
            tc_fence_before();
            mbar_arrive(my_oe);  // O is in registers: the next item's P.V may overwrite it
          } else {
#pragma unroll
            for (int i = 0; i < D / 2; ++i) w[i] = 0;
          }
#pragma unroll
          for (int h = 0; h < D / 64; ++h) store_rows(stg, w + 32 * h, at < 0 ? at : at + 64 * h, p.o);
          if (lse_at) *lse_at = row_lse(m_run, l_run);
        } else if (alive && n > 0) {
          mbar_arrive(my_oe);
        }
      } else {
        finish_piece<D>(p, ln, it, {at, lse_at, m_run, l_run, n > 0, row, any, alive}, o_tm, my_oe, stg, warp);
      }
      cnt += n;
      items += n > 0;
      pos += 2 * it.n;
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
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

// A launch's tag: 48 bits that no other launch of this process has and that memory holds by chance only.
unsigned long long launch_tag() {
  static std::atomic<unsigned long long> n{static_cast<unsigned long long>(
      std::chrono::steady_clock::now().time_since_epoch().count())};
  unsigned long long z = n.fetch_add(1) * 0x9E3779B97F4A7C15ull;
  z ^= z >> 29;
  z *= 0xBF58476D1CE4E5B9ull;
  z ^= z >> 32;
  return z << 16;
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
  p.tag = launch_tag();
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
