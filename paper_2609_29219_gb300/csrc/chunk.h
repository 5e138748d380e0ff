// Attention of a chunk of new tokens over a paged cache: the launch interface between the C ABI
// (loom_api.cu) and the kernel (attn_chunk.cu).
#pragma once

#include <cstddef>
#include <cstdint>

#include "kernels.h"
#include "paged.h"

namespace loom {

struct ChunkArgs {
  const void* q;           // [total_q, Hq, D] bf16
  const void* k;           // the caches (PagedKV), bf16
  const void* v;
  const int32_t* cu_q;     // [B + 1] on the device
  const int32_t* seqlens;  // [B] on the device
  void* o;                 // [total_q, Hq, D] bf16
  float* lse;              // [Hq, total_q] or null
  void* workspace;
  int B, Hq, Hkv, total_q, D, causal;
  float scale;
  PagedKV pages;
};

constexpr int kMaxChunkHeads = 65536;  // query heads: what a unit's places in O leave room for in 32 bits

size_t chunk_workspace_bytes(int Hq, int Hkv, int total_q, int D, int sms);
cudaError_t launch_chunk_paged(const ChunkArgs& a, const KernelCtl& ctl, cudaStream_t stream);

}  // namespace loom
