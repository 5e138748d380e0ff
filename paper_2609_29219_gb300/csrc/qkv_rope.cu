// From a packed QKV projection to what attention takes: an RMS norm of each query and key head,
// the position rotation, and the split into q, k, v (or into a cache); and its gradients.
//
// A token's projection row holds Hq query heads, Hkv key heads and Hkv value heads of D values.
// For a query or key head x with norm weight w and the token's angles (c, s):
//     r = (mean_i x_i^2 + eps)^(-1/2),   z = r x w,   y = rotation of the first R values of z:
//     y_a = z_a c - z_b s,  y_b = z_b c + z_a s   for each pair (a, b): (i, i + R/2), or
//     interleaved (2i, 2i + 1).
// Backward, with dy given:  g = rotation transposed of dy,  u = g w,
//     dw = sum over tokens and heads of g r x,   dx = r (u - r x mean_i(u_i r x_i)).
// Value heads are copied.  All arithmetic is fp32; a value is rounded once, when it is stored.
//
// What bounds it: the projection is read once and written once, and no value meets another
// outside its head, so it is the memory's bandwidth.  A head is D / 8 lanes of 16 bytes; a warp
// takes a token and UNR steps of 256 / D heads, all of whose loads are issued before the first
// is used, so that the token's angles and the weights are loaded once for all of them and enough
// bytes are in flight.  The norm's sum is shuffled within the head's lanes, and so is the pair's
// partner of the half-split form, which lies R / 16 lanes away.
#include <cuda_bf16.h>

#include "kernels.h"
#include "ptx.cuh"
#include "qkv.h"

namespace loom {
namespace {

constexpr int kWarps = 8;             // per block
constexpr int kMaxBwdBlocks = 152 * 4;  // partial sums of the weights' gradients

struct QkvParams {
  const __nv_bfloat16* x;
  long long row_elems;
  const void *wq, *wk;
  const float *cos, *sin;
  const int32_t* pos;
  int T, Hq, Hkv, R, P;
  int chunks;        // warps' shares of a token
  long long units;   // T * chunks
  float eps;
  QkvPlace q_at, kv_at;
  __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* dx;
  long long drow_elems;
  float* partial;
};

__device__ __forceinline__ uint4 ld_stream(const __nv_bfloat16* p) {
  return __ldcs(reinterpret_cast<const uint4*>(p));
}

// Value 0 of token t's head 0 in a place without a cache, and the distance between heads.
template <int D>
__device__ __forceinline__ long long place_token(const QkvPlace& at, int t, long long& head) {
  if (at.S > 0) {
    const int b = t / at.S, s = t - b * at.S;
    head = static_cast<long long>(at.S) * D;
    return (static_cast<long long>(b) * at.H * at.S + s) * D;
  }
  head = D;
  return static_cast<long long>(t) * at.H * D;
}

__device__ __forceinline__ void unpack8(const uint4& u, float* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16lo(w[i]);
    f[2 * i + 1] = bf16hi(w[i]);
  }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

template <bool W_F32>
__device__ __forceinline__ void load_weight(const void* w, int i0, float* f) {
  if constexpr (W_F32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(w) + i0);
    const float4 a = __ldg(p), b = __ldg(p + 1);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  } else {
    unpack8(__ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w) + i0)), f);
  }
}

// This lane's angles: y_i = z_i c_i + partner(z)_i s_i, with the pair's sign in s (BWD: of the
// transposed rotation).  src: the lane that holds the partners (half-split).
template <int D, bool INTER, bool BWD>
__device__ __forceinline__ void load_angles(const QkvParams& p, int t, int lane, float* c, float* s, int& src) {
  constexpr int LPH = D / 8;
  const int l = lane % LPH, i0 = 8 * l;
  src = lane;
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = 1.f, s[i] = 0.f;
  if (i0 >= p.R) return;
  int pos = p.pos ? __ldg(p.pos + t) : p.q_at.S > 0 ? t % p.q_at.S : t;
  pos = min(max(pos, 0), p.P - 1);
  const int half = p.R / 2;
  const long long row = static_cast<long long>(pos) * half;
  if constexpr (INTER) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p.cos + row + i0 / 2));
    const float4 b = __ldg(reinterpret_cast<const float4*>(p.sin + row + i0 / 2));
    const float cc[4] = {a.x, a.y, a.z, a.w}, ss[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[2 * i] = c[2 * i + 1] = cc[i];
      s[2 * i] = BWD ? ss[i] : -ss[i];
      s[2 * i + 1] = BWD ? -ss[i] : ss[i];
    }
  } else {
    const bool first = i0 < half;
    const int at = first ? i0 : i0 - half;
    src = first ? lane + half / 8 : lane - half / 8;
    const float sign = first == BWD ? 1.f : -1.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(p.cos + row + at) + h);
      const float4 b = __ldg(reinterpret_cast<const float4*>(p.sin + row + at) + h);
      c[4 * h] = a.x, c[4 * h + 1] = a.y, c[4 * h + 2] = a.z, c[4 * h + 3] = a.w;
      s[4 * h] = sign * b.x, s[4 * h + 1] = sign * b.y, s[4 * h + 2] = sign * b.z, s[4 * h + 3] = sign * b.w;
    }
  }
}

template <bool INTER>
__device__ __forceinline__ void rotate8(const float* z, const float* c, const float* s, int src, float* y) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float other = INTER ? z[i ^ 1] : __shfl_sync(0xffffffffu, z[i], src);
    y[i] = fmaf(other, s[i], z[i] * c[i]);
  }
}

// Sum over the LPH lanes of a head.
template <int LPH>
__device__ __forceinline__ float head_sum(float a) {
#pragma unroll
  for (int m = LPH / 2; m > 0; m >>= 1) a += __shfl_xor_sync(0xffffffffu, a, m);
  return a;
}

template <int D, bool INTER, bool W_F32, int UNR>
__global__ void __launch_bounds__(kWarps * 32) qkv_norm_rope_kernel(const QkvParams p) {
  constexpr int LPH = D / 8, RPW = 32 / LPH;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const long long unit = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (unit >= p.units) return;
  const int lane = threadIdx.x & 31, i0 = 8 * (lane % LPH);
  const int t = static_cast<int>(unit / p.chunks);
  const int row0 = static_cast<int>(unit - static_cast<long long>(t) * p.chunks) * (RPW * UNR) + lane / LPH;
  const int heads = p.Hq + 2 * p.Hkv;
  uint4 raw[UNR];
  const __nv_bfloat16* x = p.x + static_cast<long long>(t) * p.row_elems + i0;
#pragma unroll
  for (int u = 0; u < UNR; ++u) {
    const int h = row0 + u * RPW;
    raw[u] = h < heads ? ld_stream(x + static_cast<long long>(h) * D) : make_uint4(0, 0, 0, 0);
  }
  float c[8], s[8], wq[8], wk[8];
  int src;
  load_angles<D, INTER, false>(p, t, lane, c, s, src);
  load_weight<W_F32>(p.wq, i0, wq);
  load_weight<W_F32>(p.wk, i0, wk);
  long long q_head, kv_head;
  const long long q_tok = place_token<D>(p.q_at, t, q_head);
  long long kv_tok;
  bool kv_ok = true;
  if (p.kv_at.slots) {
    const int slot = __ldg(p.kv_at.slots + t);
    kv_ok = slot >= 0 && slot < p.kv_at.n_slots;
    const int page = kv_ok ? slot / p.kv_at.page : 0;
    kv_tok = page * p.kv_at.page_elems + static_cast<long long>(slot - page * p.kv_at.page) * p.kv_at.row_elems;
    kv_head = p.kv_at.head_elems;
  } else {
    kv_tok = place_token<D>(p.kv_at, t, kv_head);
  }
#pragma unroll
  for (int u = 0; u < UNR; ++u) {
    const int h = row0 + u * RPW;
    const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
    float z[8], y[8];
    unpack8(raw[u], z);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(z[i], z[i], ss);
    const float r = rsqrtf(head_sum<LPH>(ss) * (1.f / D) + p.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = z[i] * r * (is_q ? wq[i] : wk[i]);
    rotate8<INTER>(z, c, s, src, y);
    const uint4 out = is_v ? raw[u] : pack8(y);
    if (h < heads && (is_q || kv_ok)) {
      __nv_bfloat16* dst = is_q ? p.q + q_tok + h * q_head
                           : is_v ? p.v + kv_tok + (h - p.Hq - p.Hkv) * kv_head
                                  : p.k + kv_tok + (h - p.Hq) * kv_head;
      *reinterpret_cast<uint4*>(dst + i0) = out;
    }
  }
}

// The gradients.  Blocks walk the (token, share) units in a fixed order, each lane adding up what
// its eight values give to the weights' gradients; a block's sum goes to the workspace, where
// qkv_weight_grad_kernel adds the blocks' in their order: no atomics, the same bits each time.
template <int D, bool INTER, bool W_F32, int UNR>
__global__ void __launch_bounds__(kWarps * 32) qkv_norm_rope_bwd_kernel(const QkvParams p) {
  constexpr int LPH = D / 8, RPW = 32 / LPH;
  __shared__ float sums[kWarps][2 * D];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i0 = 8 * (lane % LPH);
  const int heads = p.Hq + 2 * p.Hkv;
  float wq[8], wk[8], gq[8], gk[8];
  load_weight<W_F32>(p.wq, i0, wq);
  load_weight<W_F32>(p.wk, i0, wk);
#pragma unroll
  for (int i = 0; i < 8; ++i) gq[i] = gk[i] = 0.f;
  const long long step = static_cast<long long>(gridDim.x) * kWarps;
  for (long long unit = static_cast<long long>(blockIdx.x) * kWarps + warp; unit < p.units; unit += step) {
    const int t = static_cast<int>(unit / p.chunks);
    const int row0 = static_cast<int>(unit - static_cast<long long>(t) * p.chunks) * (RPW * UNR) + lane / LPH;
    long long q_head, kv_head;
    const long long q_tok = place_token<D>(p.q_at, t, q_head), kv_tok = place_token<D>(p.kv_at, t, kv_head);
    const __nv_bfloat16* x = p.x + static_cast<long long>(t) * p.row_elems + i0;
    uint4 rdy[UNR], rx[UNR];
#pragma unroll
    for (int u = 0; u < UNR; ++u) {
      const int h = row0 + u * RPW;
      const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
      rdy[u] = rx[u] = make_uint4(0, 0, 0, 0);
      if (h < heads) {
        const __nv_bfloat16* dy = is_q ? p.q + q_tok + h * q_head
                                  : is_v ? p.v + kv_tok + (h - p.Hq - p.Hkv) * kv_head
                                         : p.k + kv_tok + (h - p.Hq) * kv_head;
        rdy[u] = ld_stream(dy + i0);
        if (!is_v) rx[u] = ld_stream(x + static_cast<long long>(h) * D);
      }
    }
    float c[8], s[8];
    int src;
    load_angles<D, INTER, true>(p, t, lane, c, s, src);
#pragma unroll
    for (int u = 0; u < UNR; ++u) {
      const int h = row0 + u * RPW;
      const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
      float n[8], dy[8], g[8];
      unpack8(rx[u], n);
      unpack8(rdy[u], dy);
      rotate8<INTER>(dy, c, s, src, g);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(n[i], n[i], ss);
      const float r = rsqrtf(head_sum<LPH>(ss) * (1.f / D) + p.eps);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        n[i] *= r;
        const float gn = is_v ? 0.f : g[i] * n[i];
        if (is_q)
          gq[i] += gn;
        else
          gk[i] += gn;
        g[i] *= is_q ? wq[i] : wk[i];
        dot = fmaf(g[i], n[i], dot);
      }
      dot = head_sum<LPH>(dot) * (1.f / D);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = r * fmaf(-dot, n[i], g[i]);
      if (h < heads)
        *reinterpret_cast<uint4*>(p.dx + static_cast<long long>(t) * p.drow_elems + static_cast<long long>(h) * D + i0) =
            is_v ? rdy[u] : pack8(g);
    }
  }
  // the warp's head groups, then the block's warps
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int m = LPH; m < 32; m <<= 1) {
      gq[i] += __shfl_xor_sync(0xffffffffu, gq[i], m);
      gk[i] += __shfl_xor_sync(0xffffffffu, gk[i], m);
    }
  }
  if (lane < LPH) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sums[warp][i0 + i] = gq[i];
      sums[warp][D + i0 + i] = gk[i];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kWarps * 32) {
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) a += sums[w][i];
    p.partial[static_cast<size_t>(blockIdx.x) * (2 * D) + i] = a;
  }
}

// Adds the blocks' partial sums [n][2 D] in a fixed order: a block takes 32 of the 2 D columns.
__global__ void __launch_bounds__(1024) qkv_weight_grad_kernel(const float* partial, int n, int D, float* dwq, float* dwk) {
  __shared__ float sums[32][33];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 32 + x;
  float a = 0.f;
  for (int i = y; i < n; i += 32) a += partial[static_cast<size_t>(i) * (2 * D) + col];
  sums[y][x] = a;
  __syncthreads();
  a = sums[x][y];  // column y's sum over the rows that thread row x took
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) a += __shfl_xor_sync(0xffffffffu, a, m);
  if (x == 0) {
    const int i = blockIdx.x * 32 + y;
    (i < D ? dwq[i] : dwk[i - D]) = a;
  }
}

// A launch as a programmatic dependent of the kernel before it in the stream: every kernel here
// waits for that one (griddepcontrol.wait) before its first access to memory.
template <class Kernel, class... Args>
cudaError_t launch(Kernel kernel, int grid, int threads, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

QkvParams params_of(const QkvArgs& a, int unroll) {
  QkvParams p{};
  p.x = static_cast<const __nv_bfloat16*>(a.qkv);
  p.row_elems = a.row_elems;
  p.wq = a.q_weight;
  p.wk = a.k_weight;
  p.cos = a.cos;
  p.sin = a.sin;
  p.pos = a.positions;
  p.T = a.T;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.R = a.R;
  p.P = a.P;
  const int rows = 256 / a.D * unroll;  // heads that a warp takes
  p.chunks = (a.Hq + 2 * a.Hkv + rows - 1) / rows;
  p.units = static_cast<long long>(a.T) * p.chunks;
  p.eps = a.eps;
  p.q_at = a.q_at;
  p.kv_at = a.kv_at;
  p.q = static_cast<__nv_bfloat16*>(a.q);
  p.k = static_cast<__nv_bfloat16*>(a.k);
  p.v = static_cast<__nv_bfloat16*>(a.v);
  p.dx = static_cast<__nv_bfloat16*>(a.dqkv);
  p.drow_elems = a.drow_elems;
  p.partial = a.partial;
  return p;
}

template <int D, int UNR>
cudaError_t launch_fwd_u(const QkvArgs& a, cudaStream_t stream) {
  const QkvParams p = params_of(a, UNR);
  const long long blocks = (p.units + kWarps - 1) / kWarps;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  const int g = static_cast<int>(blocks);
  if (a.interleaved)
    return a.weights_f32 ? launch(qkv_norm_rope_kernel<D, true, true, UNR>, g, kWarps * 32, stream, p)
                         : launch(qkv_norm_rope_kernel<D, true, false, UNR>, g, kWarps * 32, stream, p);
  return a.weights_f32 ? launch(qkv_norm_rope_kernel<D, false, true, UNR>, g, kWarps * 32, stream, p)
                       : launch(qkv_norm_rope_kernel<D, false, false, UNR>, g, kWarps * 32, stream, p);
}

template <int D>
cudaError_t launch_fwd_d(const QkvArgs& a, cudaStream_t stream) {
  return launch_fwd_u<D, 4>(a, stream);
}

template <int D, int UNR>
cudaError_t launch_bwd_u(const QkvArgs& a, cudaStream_t stream) {
  const QkvParams p = params_of(a, UNR);
  const long long blocks = (p.units + kWarps - 1) / kWarps;
  const int g = static_cast<int>(blocks < kMaxBwdBlocks ? blocks : kMaxBwdBlocks);
  cudaError_t e;
  if (a.interleaved)
    e = a.weights_f32 ? launch(qkv_norm_rope_bwd_kernel<D, true, true, UNR>, g, kWarps * 32, stream, p)
                      : launch(qkv_norm_rope_bwd_kernel<D, true, false, UNR>, g, kWarps * 32, stream, p);
  else
    e = a.weights_f32 ? launch(qkv_norm_rope_bwd_kernel<D, false, true, UNR>, g, kWarps * 32, stream, p)
                      : launch(qkv_norm_rope_bwd_kernel<D, false, false, UNR>, g, kWarps * 32, stream, p);
  if (e != cudaSuccess) return e;
  return launch(qkv_weight_grad_kernel, 2 * D / 32, 1024, stream, static_cast<const float*>(p.partial), g, D, a.dq_weight,
                a.dk_weight);
}

}  // namespace

cudaError_t launch_qkv_norm_rope(const QkvArgs& a, cudaStream_t stream) {
  return a.D == 128 ? launch_fwd_d<128>(a, stream) : launch_fwd_d<64>(a, stream);
}

cudaError_t launch_qkv_norm_rope_bwd(const QkvArgs& a, cudaStream_t stream) {
  return a.D == 128 ? launch_bwd_u<128, 4>(a, stream) : launch_bwd_u<64, 4>(a, stream);
}

size_t qkv_bwd_workspace_bytes(int D) { return static_cast<size_t>(kMaxBwdBlocks) * 2 * D * sizeof(float); }

}  // namespace loom
