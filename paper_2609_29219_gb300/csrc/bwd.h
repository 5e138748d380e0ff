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

// Rows of 128 queries per head that the workspace's row statistics have.
inline long long bwd_stat_tiles(int B, long long Sq, bool ragged) {
  return ragged ? Sq / 128 + B : (Sq + 127) / 128;
}
// Workspace: 256 bytes of counters, then 2 x 128 floats for each tile of 128 queries of each head.
inline size_t bwd_workspace_bytes(int B, int Hq, long long Sq, bool ragged) {
  const size_t planes = ragged ? static_cast<size_t>(Hq) : static_cast<size_t>(B) * Hq;
  return 256 + planes * static_cast<size_t>(bwd_stat_tiles(B, Sq, ragged)) * 1024;
}

cudaError_t launch_attn_bwd(const BwdArgs& a, const KernelCtl& ctl, cudaStream_t stream);

}  // namespace loom
