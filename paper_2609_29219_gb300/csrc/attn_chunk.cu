// Attention of a chunk of new tokens per sequence over a paged KV cache: one block per (query token,
// query head) walks its visible keys 128 at a time with a running maximum m and sum l,
//     m' = max(m, max_j s_j),  l' = l 2^(m-m') + sum_j 2^(s_j-m'),  o' = o 2^(m-m') + sum_j 2^(s_j-m') v_j
// (scores in units of log 2), and stores o / l and (m + log2 l) ln 2.
#include <cuda_bf16.h>

#include "chunk.h"
#include "ptx.cuh"

namespace loom {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct ChunkParams {
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* o;
  float* lse;
  const int32_t *cu_q, *seqlens, *table;
  int B, Hq, Hkv, total_q, causal;
  int num_pages, page, max_pages, hnd;
  float c;  // scale log2(e)
};

template <int D>
__global__ void __launch_bounds__(128) chunk_simple_kernel(const ChunkParams p) {
  __shared__ float q[D], prob[128], red[4];
  __shared__ long long rows[128];
  const int token = blockIdx.x, h = blockIdx.y, hk = h / (p.Hq / p.Hkv), tid = threadIdx.x;
  if (token >= p.cu_q[p.B]) return;
  int b = 0, hi = p.B;
  while (hi - b > 1) {
    const int mid = (b + hi) / 2;
    if (p.cu_q[mid] <= token)
      b = mid;
    else
      hi = mid;
  }
  const int n = p.cu_q[b + 1] - p.cu_q[b];
  const long long cap = static_cast<long long>(p.max_pages) * p.page;
  const int len = static_cast<int>(min(max(static_cast<long long>(p.seqlens[b]), 0ll), cap));
  const int limit = p.causal ? min(len, max(0, token - p.cu_q[b] + len - n + 1)) : len;
  const size_t at = (static_cast<size_t>(token) * p.Hq + h) * D;
  if (tid < D) q[tid] = __bfloat162float(p.q[at + tid]);
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int j0 = 0; j0 < limit; j0 += 128) {
    const int j = j0 + tid;
    long long row = -1;
    float s = -INFINITY;
    __syncthreads();
    if (j < limit) {
      const int page = p.table[static_cast<size_t>(b) * p.max_pages + j / p.page];
      const bool bad = page < 0 || page >= p.num_pages;
      if (!bad)
        row = (p.hnd ? (static_cast<long long>(page) * p.Hkv + hk) * p.page + j % p.page
                     : (static_cast<long long>(page) * p.page + j % p.page) * p.Hkv + hk) * D;
      s = 0.f;
      if (!bad)
        for (int d = 0; d < D; ++d) s = fmaf(q[d], __bfloat162float(p.k[row + d]), s);
      s *= p.c;
    }
    rows[tid] = row;
    float mx = s;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    if ((tid & 31) == 0) red[tid >> 5] = mx;
    __syncthreads();
    const float m_new = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m);
    const float base = m_new == -INFINITY ? 0.f : m_new;  // (all NaN: stays NaN)
    const float pr = exp2f(s - base), alpha = exp2f(m - base);
    prob[tid] = pr;
    m = m_new;
    __syncthreads();
    l *= alpha;
    o *= alpha;
    const int keys = min(128, limit - j0);
    for (int i = 0; i < keys; ++i) {
      l += prob[i];
      if (tid < D && rows[i] >= 0) o = fmaf(prob[i], __bfloat162float(p.v[rows[i] + tid]), o);
    }
  }
  if (tid < D) p.o[at + tid] = __float2bfloat16_rn(l == 0.f ? 0.f : o / l);
  if (tid == 0 && p.lse) p.lse[static_cast<size_t>(h) * p.total_q + token] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

size_t chunk_workspace_bytes(int, int, int, int, int) { return 256; }

cudaError_t launch_chunk_paged(const ChunkArgs& a, const KernelCtl&, cudaStream_t stream) {
  const ChunkParams p{static_cast<const __nv_bfloat16*>(a.q), static_cast<const __nv_bfloat16*>(a.k),
                      static_cast<const __nv_bfloat16*>(a.v), static_cast<__nv_bfloat16*>(a.o), a.lse, a.cu_q, a.seqlens,
                      a.pages.block_table, a.B, a.Hq, a.Hkv, a.total_q, a.causal, a.pages.num_pages, a.pages.page_size,
                      a.pages.max_pages, a.pages.layout == kPagedHND, a.scale * kLog2e};
  const dim3 grid(static_cast<unsigned>(a.total_q), static_cast<unsigned>(a.Hq));
  if (a.D == 128)
    chunk_simple_kernel<128><<<grid, 128, 0, stream>>>(p);
  else
    chunk_simple_kernel<64><<<grid, 128, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace loom
