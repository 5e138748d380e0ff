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
// 128 rows of a query plane, whose steps are the kv tiles it sees.  Where items are few and long, an
// item's steps are split into shares (with partial sums in fp32 in the workspace).
struct BwdPlan {
  int kv_split, q_split;        // shares of an item, powers of two
  long long kv_items, q_items;  // (ragged: at most)
  int counters;                 // 64, then one for each elementwise warp of each item where items are split
  size_t stats_at, partial_at, bytes;
};
inline BwdPlan bwd_plan(int B, int Hq, int Hkv, long long Sq, long long Skv, int D, bool ragged, int sms) {
  const int lg = bwd_pack_log2(Hq / Hkv), G = Hq / Hkv >> lg;
  const long long seqs = ragged ? 1 : B;
  const long long q_planes = seqs * (Hq >> lg), kv_planes = seqs * Hkv, stat_tiles = bwd_stat_tiles(B, Sq, lg, ragged);
  BwdPlan p{};
  p.kv_items = kv_planes * (ragged ? Skv / 128 + B : (Skv + 127) / 128);
  p.q_items = q_planes * stat_tiles;
  // Steps of an item (ragged: of a sequence of average length), a kv item's of about 1.4 us and a
  // query item's of 1.2 (D = 128).  The splits are those of the least estimate: the time of all
  // steps spread over the SMs, 4 us for each share (its partial sums), and half the longest share,
  // but no less than one share of each kind one after the other.  GB300, us, unsplit / split: B1 H8/1
  // S2000 causal 158 / 49, B2 H16/2 S512 causal 50 / 31, B1 H8/1 S300 causal 32 / 24; a chunk of 515 at 3001,
  // H32/8, has an item for each SM and stays whole (70; 97 in two and four shares).
  const double rows = static_cast<double>(Sq) / (ragged ? B : 1) * (1 << lg), keys = static_cast<double>(Skv) / (ragged ? B : 1);
  const double kv_us = 1.4 * G * (rows < 128 ? 1 : rows / 128), q_us = 1.2 * (keys < 128 ? 1 : keys / 128);
  const double all = (p.kv_items * kv_us + p.q_items * q_us) / sms;
  double best = 1e300;
  for (int a = 1; a <= 16 && (a == 1 || kv_us / a >= 2.8); a *= 2)
    for (int b = 1; b <= 16 && (b == 1 || q_us / b >= 2.4); b *= 2) {
      // (a quarter of a gigabyte of partial sums of each kind at most)
      if (a > 1 && p.kv_items * a * 1024.0 * D > 2.7e8) continue;
      if (b > 1 && p.q_items * b * 512.0 * D > 2.7e8) continue;
      const double k = kv_us / a, q = q_us / b, shares = (a > 1 ? p.kv_items * a : 0) + (b > 1 ? p.q_items * b : 0);
      const double spread = all + 4.0 * shares / sms + 0.5 * (k > q ? k : q), chain = k + q + (a > 1 ? 4 : 0) + (b > 1 ? 4 : 0);
      const double us = spread > chain ? spread : chain;
      if (us < best) best = us, p.kv_split = a, p.q_split = b;
    }
  const bool any = p.kv_split > 1 || p.q_split > 1;
  p.counters = 64 + (any ? static_cast<int>((p.kv_items + p.q_items) * 8) : 0);
  p.stats_at = (static_cast<size_t>(p.counters) * 4 + 255) / 256 * 256;
  p.partial_at = p.stats_at + static_cast<size_t>(q_planes) * static_cast<size_t>(stat_tiles) * 1024;
  p.bytes = p.partial_at + (p.kv_split > 1 ? static_cast<size_t>(p.kv_items) * p.kv_split * 1024 * D : 0) +
            (p.q_split > 1 ? static_cast<size_t>(p.q_items) * p.q_split * 512 * D : 0);
  return p;
}

cudaError_t launch_attn_bwd(const BwdArgs& a, const KernelCtl& ctl, cudaStream_t stream);

}  // namespace loom
