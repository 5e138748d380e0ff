// Norms of q and k per head with the position rotation: the launch interface between the C
// ABI (loom_api.cu) and the kernels (qkv_rope.cu).
#pragma once

#include <cstddef>
#include <cstdint>

#include "kernels.h"

namespace loom {

// A head's values of one token, as [tokens][heads][D] with any distance between tokens and
// between heads: value 0 of (t, h) is at tok(t) + h * head, in elements.
struct QkvPlace {
  int S;               // > 0: tokens come as T / S sequences, head-major ([B, H, S, D])
  int H;               // heads (for S > 0, and for S = 0 packed tokens [T, H, D])
  const int32_t* slots;  // cache: token t goes to row slots[t] (null: not a cache)
  int page, n_slots;   // cache: rows per page, rows in all (a slot outside is not written)
  long long page_elems, row_elems, head_elems;  // cache: strides
};

struct QkvArgs {
  const void* qkv;       // [T, >= (Hq + 2 Hkv) D] bf16, rows row_elems apart
  long long row_elems;
  const void* q_weight;  // [D]
  const void* k_weight;  // [D]
  int weights_f32;       // the weights are fp32 (else bf16)
  const float* cos;      // [P, R / 2]
  const float* sin;      // [P, R / 2]
  const int32_t* positions;  // [T], or null: t (S = 0) or t % S; with axes [n_axes, T]
  int n_axes;                // 0: one position a token; else pair i turns by that of its axis
  long long pos_stride;      // axes: from one axis' positions to the next's
  unsigned long long axis_of[2];  // axes: two bits for each pair of a head
  int T, Hq, Hkv, D, R, P, interleaved;
  float eps;
  QkvPlace q_at, kv_at;
  void *q, *k, *v;       // forward: written; backward: dq, dk, dv, read
  // backward
  void* dqkv;            // [T, >= (Hq + 2 Hkv) D] bf16, rows drow_elems apart
  long long drow_elems;
  float *dq_weight, *dk_weight;  // [D]
  float* partial;        // [blocks][2][D] (workspace)
};

constexpr int kMaxAxes = 4;  // what two bits tell apart

// Heads (Hq + 2 Hkv) of a token at most in the backward pass.
constexpr int kMaxBwdHeads = 16384;

cudaError_t launch_qkv_norm_rope(const QkvArgs& a, cudaStream_t stream);
cudaError_t launch_qkv_norm_rope_bwd(const QkvArgs& a, cudaStream_t stream);
// Bytes of workspace of the backward pass: a partial sum of the weights' gradients per block.
size_t qkv_bwd_workspace_bytes(int D);

}  // namespace loom
