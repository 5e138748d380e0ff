// Attention's backward pass: the launch interface between the C ABI (loom_api.cu) and the
// kernels (attn_bwd.cu).
#pragma once

#include <cstddef>
#include <cstdint>

#include "kernels.h"

namespace loom {

struct BwdArgs {
  const void *dout, *q, *k, *v, *o;  // dense [B, H, S, D]; ragged [total, H, D] (bf16)
  const float* lse;                  // [B, Hq, Sq]; ragged [Hq, total_q]
  const float* dlse;                 // like lse, or null
  void *dq, *dk, *dv;
  void* workspace;
  int B, Hq, Hkv, Sq, Skv, D, causal;  // ragged: Sq, Skv are the totals
  float scale;
  const int32_t *cu_q, *cu_k;  // ragged: [B + 1] on the device; null: dense
  int max_q, max_k;            // ragged: they only bound the launch
};

// Query heads of a kv head whose rows make one plane, as a power of two: the largest that divides
// the group, up to 32.
inline int bwd_pack_log2(int G) {
  int lg = 0;
  while (lg < 5 && (G >> lg) % 2 == 0) ++lg;
  return lg;
}
// Tiles of 128 rows that a plane of 2^lg heads has in the workspace's row statistics.
inline long long bwd_stat_tiles(int B, long long Sq, int lg, bool ragged) {
  return ragged ? (Sq << lg) / 128 + B : ((Sq << lg) + 127) / 128;
}
// How a call's work is dealt, and its workspace.  The kernel has two kinds of items: a tile of 128
// keys of a kv head, whose steps are the query tiles of the group's heads that see it, and a tile of
// 128 rows of a query plane, whose steps are the kv tiles it sees.  Where whole items would leave SMs
// idle at the end, an item's steps are split into shares (with partial sums in fp32 in the workspace): few
// and long items, but also the 512 of H32/8 S8192 causal, in two.
struct BwdPlan {
  int kv_split, q_split;        // shares of an item, powers of two
  int kv_block, q_block;        // dense: planes whose tiles are dealt together
  long long kv_items, q_items;  // (ragged: at most)
  int counters;                 // 64, then one for each elementwise warp of each item where items are split
  size_t stats_at, partial_at, bytes;
};
// Planes whose tiles are dealt together: as many as have what their items walk at a time (bytes a plane)
// in L2 at once, since the longest tiles of them all go first, but at least a round of CTAs.  A kv plane
// walks the query planes of its group one after another, and one of them is counted.  With all of the
// group's (another choice only where a group is no power of two), GB300, us, one / all: B8 H28/4 S2048 causal
// 607 / 590, B2 S16384 7756 / 7716, B4 H28/4 S8192 4008 / 4030, D64 2974 / 3023, B2 H15/5 S8192 993 / 1010;
// ten shapes 0.2 % apart on average.
inline int bwd_planes_per_block(double bytes, long long tiles, int sms, long long planes) {
  const double fit = 48e6 / bytes;
  const long long n = fit > planes ? planes : static_cast<long long>(fit), round = (sms + tiles - 1) / tiles;
  return static_cast<int>(n < round ? round : n);
}
inline BwdPlan bwd_plan(int B, int Hq, int Hkv, long long Sq, long long Skv, int D, bool ragged, bool causal, int sms) {
  const int lg = bwd_pack_log2(Hq / Hkv), G = Hq / Hkv >> lg;
  const long long seqs = ragged ? 1 : B;
  const long long q_planes = seqs * (Hq >> lg), kv_planes = seqs * Hkv, stat_tiles = bwd_stat_tiles(B, Sq, lg, ragged);
  BwdPlan p{};
  p.kv_items = kv_planes * (ragged ? Skv / 128 + B : (Skv + 127) / 128);
  p.q_items = q_planes * stat_tiles;
  // The splits of the least score: all of the work spread over the SMs and part of the longest share of
  // each kind, or the longest share if that is more, query items' after the kv items' full rounds.  A
  // share of a split item writes and reads its partial sums, and the last one to arrive adds the others';
  // the kernel that can split takes longer over whole kv items too.  The constants are fitted: they choose
  // best among 1 to 16 shares of kv items and 1 to 8 of query items over 7000 random dense shapes (1 to 96
  // heads, 32 to 8000 queries and keys), where the choices take 1.7 % longer than the best ones on average,
  // no splits 16 %.  They are about microseconds, but no step times (those at D = 128 are 1.6 and 1.1, not
  // 1.1 and 0.67; at D = 64 steps are shorter, not longer), and not tried outside those shapes: a ragged
  // batch enters as if all its sequences had the average length.  GB300, us, unsplit / split: B1 H8/1 S2000
  // causal 158 / 47, B1 H32/8 S2048 causal 136 / 100; B1 H16/16 S2048 causal, an item for each SM and more,
  // 52 / 73.
  const auto tiles = [&](long long rows) {
    return ragged ? static_cast<double>(rows) / B / 128 + 0.5 : static_cast<double>((rows + 127) / 128);
  };
  const double kv_steps = G * tiles(Sq << lg), q_steps = tiles(Skv);
  const double seen = causal ? 1 - 0.5 * static_cast<double>(Sq < Skv ? Sq : Skv) / static_cast<double>(Skv > 0 ? Skv : 1) : 1;
  const double kv_step = D == 128 ? 1.1 : 1.5, q_step = D == 128 ? 0.67 : 0.95, kv_part = D == 128 ? 6 : 7, q_part = 2;
  double best = 1e300;
  // Items of eight steps and more that keep less than a third of the SMs busy always have two shares or
  // more.  By the score alone 1.5 % of random shapes of 1 to 32 heads would have whole items instead: 37 of
  // those, 16 to 21 us, take 0.96 to 1.13 times as long in shares, 1.04 on average, so the rule gains
  // nothing; it keeps few long items in the form that they are tested in.
  const int least = kv_steps >= 8 && p.kv_items + p.q_items <= sms / 3 ? 2 : 1;
  for (int a = least; a <= 16 && (a == 1 || a <= kv_steps); a *= 2)
    for (int b = 1; b <= 8 && (b == 1 || b <= q_steps); b *= 2) {
      // (a quarter of a gigabyte of partial sums of each kind at most)
      if (a > 1 && p.kv_items * a * 1024.0 * D > 2.7e8) continue;
      if (b > 1 && p.q_items * b * 512.0 * D > 2.7e8) continue;
      const double k_all = kv_steps * seen * kv_step + 2.5 + (a > 1 ? a * kv_part : b > 1 ? 0.9 : 0);
      const double q_all = q_steps * seen * q_step + 2.1 + (b > 1 ? b * q_part : 0);
      const double k_long = kv_steps * kv_step / a + 2.5 + (a > 1 ? 4.3 + 1.1 * a : 0);
      const double q_long = q_steps * q_step / b + 2.1 + (b > 1 ? 0.35 * b : 0);
      const double spread = (p.kv_items * k_all + p.q_items * q_all) / sms + 0.42 * k_long + 0.16 * q_long;
      const double rounds = static_cast<double>(p.kv_items * a / sms) * (k_all / a), q_end = 0.85 * rounds + q_long;
      const double longest = k_long > q_end ? k_long : q_end, score = spread > longest ? spread : longest;
      if (score < best) best = score, p.kv_split = a, p.q_split = b;
    }
  if (!ragged) {
    const double row = 4.0 * D;  // a query's dO and Q, a key's K and V
    p.kv_block = bwd_planes_per_block(row * Sq * (1 << lg), (Skv + 127) / 128, sms, kv_planes);
    p.q_block = bwd_planes_per_block(row * Skv / G, stat_tiles, sms, q_planes);
  }
  const bool any = p.kv_split > 1 || p.q_split > 1;
  p.counters = 64 + (any ? static_cast<int>((p.kv_items + p.q_items) * 8) : 0);
  p.stats_at = (static_cast<size_t>(p.counters) * 4 + 255) / 256 * 256;
  p.partial_at = p.stats_at + static_cast<size_t>(q_planes) * static_cast<size_t>(stat_tiles) * 1024;
  p.bytes = p.partial_at + (p.kv_split > 1 ? static_cast<size_t>(p.kv_items) * p.kv_split * 1024 * D : 0) +
            (p.q_split > 1 ? static_cast<size_t>(p.q_items) * p.q_split * 512 * D : 0);
  return p;
}

// The workspace of a call, causal or not.
inline size_t bwd_workspace(int B, int Hq, int Hkv, long long Sq, long long Skv, int D, bool ragged, int sms) {
  const size_t full = bwd_plan(B, Hq, Hkv, Sq, Skv, D, ragged, false, sms).bytes;
  const size_t causal = bwd_plan(B, Hq, Hkv, Sq, Skv, D, ragged, true, sms).bytes;
  return full > causal ? full : causal;
}

cudaError_t launch_attn_bwd(const BwdArgs& a, const KernelCtl& ctl, cudaStream_t stream);

}  // namespace loom
