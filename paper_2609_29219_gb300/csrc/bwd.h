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
// Workspace: 256 bytes of counters, then 2 x 128 floats for each tile of 128 rows of each plane.
inline size_t bwd_workspace_bytes(int B, int Hq, int Hkv, long long Sq, bool ragged) {
  const int lg = bwd_pack_log2(Hq / Hkv);
  const size_t planes = (ragged ? static_cast<size_t>(Hq) : static_cast<size_t>(B) * Hq) >> lg;
  return 256 + planes * static_cast<size_t>(bwd_stat_tiles(B, Sq, lg, ragged)) * 1024;
}

cudaError_t launch_attn_bwd(const BwdArgs& a, const KernelCtl& ctl, cudaStream_t stream);

}  // namespace loom
