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
// outside its head, so it is the memory's bandwidth, and after that the instructions per value:
// at 100 instructions for 16 bytes of a lane they took as long as the memory (8192 tokens, H32/8,
// D 128: 49 us; 33 with what follows).  So the norm's factor is applied last, and weight and angle
// are multiplied once for all of a token's heads:
//     y_i = r (x_i A_i + x_partner(i) B_i),   A_i = w_i c_i,   B_i = w_partner(i) (+-) s_i;
// the arithmetic is on pairs of floats, and the partner's values are shuffled as packed bf16.
// A head is D / 8 lanes of 16 bytes; a warp takes a unit, up to UNR steps of 256 / D heads of one
// kind (query, key or value) of a token, and issues the loads of all of them before it uses the
// first.
#include <cuda_bf16.h>

#include <type_traits>

#include "kernels.h"
#include "ptx.cuh"
#include "qkv.h"

namespace loom {
namespace {

constexpr int kWarps = 8;  // per block (the forward's: at most)
constexpr int kBwdBlocksPerSm = 2, kBwdStages = 2;
constexpr int kMaxBwdBlocks = 152 * kBwdBlocksPerSm;  // as many as are resident; partial sums of the weights' gradients
// Steps of a unit: one where the call is over as soon as its longest warp, else four, or two where
// four would leave a third of the steps without heads (units of two steps fewer than 3/2 of those of
// four).  GB300, device us with one / two / four steps, forward and backward: 30 tokens H32/8 D 128
// (184320 values) backward 4.0 / 4.1 / 4.6; 200 tokens (1228800) 6.3 / 6.1 / 5.2; 20000 tokens 137 /
// 95 / 80 and 264 / 160 / 122; H9/3 (units 9 / 5 / 4) 52 / 39 / 42 and 95 / 66 / 66; H4/4 (6 / 3 / 3)
// 34 / 25 / 31 and 60 / 40 / 49; H28/4 (18 / 9 / 6) 107 / 75 / 70 and 207 / 126 / 108.  Eight steps:
// forward of 8192 tokens H32/8 35.5 (four: 34.7; both in blocks of eight warps).
constexpr long long kManyValues = 1 << 18;

struct QkvParams {
  const __nv_bfloat16* x;
  long long row_elems;
  const void *wq, *wk;
  int w_f32;
  const float *cos, *sin;
  const int32_t* pos;
  int T, Hq, Hkv, R, P;
  int q_units, kv_units;  // units of a token's query heads, of its key heads (and of its value heads)
  long long units;        // of all tokens
  float eps;
  QkvPlace q_at, kv_at;
  __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* dx;
  long long drow_elems;
  float* partial;
};

// Unit `unit`: which token's heads of which kind, from head h0 on (counted within the kind).
enum Kind { kQuery, kKey, kValue };
struct Unit {
  int t, kind, h0, heads;  // heads: of the kind
};
template <int D, int UNR>
__device__ __forceinline__ Unit unit_of(const QkvParams& p, long long unit) {
  const int per = p.q_units + 2 * p.kv_units;
  const long long token = unit / per;
  const int t = token < p.T ? static_cast<int>(token) : p.T;
  int u = static_cast<int>(unit - token * per);
  if (u < p.q_units) return {t, kQuery, u * (256 / D * UNR), p.Hq};
  u -= p.q_units;
  const int kind = u < p.kv_units ? kKey : kValue;
  return {t, kind, (u - (kind == kValue ? p.kv_units : 0)) * (256 / D * UNR), p.Hkv};
}

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

// Eight packed bf16 as four pairs of floats, and back.
__device__ __forceinline__ void unpack8(const uint4& u, uint64_t* f) {
  f[0] = f2(bf16lo(u.x), bf16hi(u.x));
  f[1] = f2(bf16lo(u.y), bf16hi(u.y));
  f[2] = f2(bf16lo(u.z), bf16hi(u.z));
  f[3] = f2(bf16lo(u.w), bf16hi(u.w));
}
__device__ __forceinline__ uint4 pack8(const uint64_t* f) {
  return make_uint4(pack_bf16x2(f2lo(f[0]), f2hi(f[0])), pack_bf16x2(f2lo(f[1]), f2hi(f[1])), pack_bf16x2(f2lo(f[2]), f2hi(f[2])),
                    pack_bf16x2(f2lo(f[3]), f2hi(f[3])));
}

// Eight weights from i0 on.
__device__ __forceinline__ void load_weight(const QkvParams& p, int kind, int i0, float* f) {
  const void* w = kind == kQuery ? p.wq : p.wk;
  if (p.w_f32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(w) + i0);
    const float4 a = __ldg(q), b = __ldg(q + 1);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  } else {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w) + i0));
    f[0] = bf16lo(u.x), f[1] = bf16hi(u.x), f[2] = bf16lo(u.y), f[3] = bf16hi(u.y);
    f[4] = bf16lo(u.z), f[5] = bf16hi(u.z), f[6] = bf16lo(u.w), f[7] = bf16hi(u.w);
  }
}

// The lane whose values are the partners of this lane's (half-split pairs; else this lane).
template <int D, bool INTER>
__device__ __forceinline__ int partner_lane(const QkvParams& p, int lane) {
  const int i0 = 8 * (lane % (D / 8)), half = p.R / 2;
  return INTER || i0 >= p.R ? lane : i0 < half ? lane + half / 8 : lane - half / 8;
}

// The position whose angles token t takes.
__device__ __forceinline__ int position(const QkvParams& p, int t) {
  const int pos = p.pos ? __ldg(p.pos + t) : p.q_at.S > 0 ? t % p.q_at.S : t;
  return min(max(pos, 0), p.P - 1);
}

// The angles of the eight values from i0 on, from their position's R / 2 = half cosines and sines:
// y_i = z_i c_i + partner(z)_i s_i, with the pair's sign in s (BWD: of the transposed rotation).
template <bool INTER, bool BWD>
__device__ __forceinline__ void angles(const float* cos, const float* sin, int i0, int half, float* c, float* s) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = 1.f, s[i] = 0.f;
  if (i0 >= 2 * half) return;
  if constexpr (INTER) {
    const float4 a = *reinterpret_cast<const float4*>(cos + i0 / 2), b = *reinterpret_cast<const float4*>(sin + i0 / 2);
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
    const float sign = first == BWD ? 1.f : -1.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 a = *(reinterpret_cast<const float4*>(cos + at) + h), b = *(reinterpret_cast<const float4*>(sin + at) + h);
      c[4 * h] = a.x, c[4 * h + 1] = a.y, c[4 * h + 2] = a.z, c[4 * h + 3] = a.w;
      s[4 * h] = sign * b.x, s[4 * h + 1] = sign * b.y, s[4 * h + 2] = sign * b.z, s[4 * h + 3] = sign * b.w;
    }
  }
}

// The partners of eight packed values.
template <bool INTER>
__device__ __forceinline__ uint4 partners(const uint4& u, int src) {
  if constexpr (INTER)
    return make_uint4(__funnelshift_l(u.x, u.x, 16), __funnelshift_l(u.y, u.y, 16), __funnelshift_l(u.z, u.z, 16),
                      __funnelshift_l(u.w, u.w, 16));
  else
    return make_uint4(__shfl_sync(0xffffffffu, u.x, src), __shfl_sync(0xffffffffu, u.y, src), __shfl_sync(0xffffffffu, u.z, src),
                      __shfl_sync(0xffffffffu, u.w, src));
}

__device__ __forceinline__ float sum8(const uint64_t* a, const uint64_t* b) {
  const uint64_t s = add2(fma2(a[1], b[1], mul2(a[0], b[0])), fma2(a[3], b[3], mul2(a[2], b[2])));
  return f2lo(s) + f2hi(s);
}
// Sum over the LPH lanes of a head.
template <int LPH>
__device__ __forceinline__ float head_sum(float a) {
#pragma unroll
  for (int m = LPH / 2; m > 0; m >>= 1) a += __shfl_xor_sync(0xffffffffu, a, m);
  return a;
}

// Value 0 of token t's head 0 of a kind where it is written (backward: read), and the distance
// between heads; a token whose cache slot lies outside the cache has no such place.
template <int D>
__device__ __forceinline__ __nv_bfloat16* place(const QkvParams& p, const Unit& u, long long& head) {
  __nv_bfloat16* base = u.kind == kQuery ? p.q : u.kind == kKey ? p.k : p.v;
  const QkvPlace& at = u.kind == kQuery ? p.q_at : p.kv_at;
  if (u.kind == kQuery || !at.slots) return base + place_token<D>(at, u.t, head);
  const int slot = __ldg(at.slots + u.t);
  head = at.head_elems;
  if (slot < 0 || slot >= at.n_slots) return nullptr;
  const int page = slot / at.page;
  return base + page * at.page_elems + static_cast<long long>(slot - page * at.page) * at.row_elems;
}

template <int D, bool INTER, int UNR>
__global__ void __launch_bounds__(kWarps * 32) qkv_norm_rope_kernel(const QkvParams p) {
  constexpr int LPH = D / 8, RPW = 32 / LPH;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const long long unit = static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (unit >= p.units) return;
  const Unit u = unit_of<D, UNR>(p, unit);
  const int lane = threadIdx.x & 31, i0 = 8 * (lane % LPH), h0 = u.h0 + lane / LPH;
  const int first = u.kind == kQuery ? 0 : u.kind == kKey ? p.Hq : p.Hq + p.Hkv;
  const __nv_bfloat16* x = p.x + static_cast<long long>(u.t) * p.row_elems + static_cast<long long>(first + h0) * D + i0;
  uint4 raw[UNR];
#pragma unroll
  for (int s = 0; s < UNR; ++s)
    raw[s] = h0 + s * RPW < u.heads ? ld_stream(x + s * RPW * D) : make_uint4(0, 0, 0, 0);
  long long head;
  __nv_bfloat16* dst = place<D>(p, u, head);
  if (!dst) return;
  dst += h0 * head + i0;
  if (u.kind == kValue) {
#pragma unroll
    for (int s = 0; s < UNR; ++s)
      if (h0 + s * RPW < u.heads) __stcs(reinterpret_cast<uint4*>(dst + s * RPW * head), raw[s]);
    return;
  }
  const int src = partner_lane<D, INTER>(p, lane);
  uint64_t a[4], b[4];
  {
    float c[8], s[8], w[8], wp[8];
    const long long row = static_cast<long long>(position(p, u.t)) * (p.R / 2);
    angles<INTER, false>(p.cos + row, p.sin + row, i0, p.R / 2, c, s);
    load_weight(p, u.kind, i0, w);
    load_weight(p, u.kind, 8 * (src % LPH), wp);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = f2(w[2 * i] * c[2 * i], w[2 * i + 1] * c[2 * i + 1]);
      b[i] = INTER ? f2(wp[2 * i + 1] * s[2 * i], wp[2 * i] * s[2 * i + 1]) : f2(wp[2 * i] * s[2 * i], wp[2 * i + 1] * s[2 * i + 1]);
    }
  }
#pragma unroll
  for (int s = 0; s < UNR; ++s) {
    uint64_t z[4], o[4];
    unpack8(raw[s], z);
    unpack8(partners<INTER>(raw[s], src), o);
    const float r = rsqrtf(head_sum<LPH>(sum8(z, z)) * (1.f / D) + p.eps);
    const uint64_t r2 = f2(r, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = mul2(fma2(o[i], b[i], mul2(z[i], a[i])), r2);
    if (h0 + s * RPW < u.heads) __stcs(reinterpret_cast<uint4*>(dst + s * RPW * head), pack8(z));
  }
}

// The gradients.  With g the rotation transposed of dy and u = g w:  dx = r u - x r^3 mean(u x) and
// dw += r g x.  A warp takes the same heads of every so many tokens (the grid's warps are a multiple
// of a token's units, or the last few have nothing to do), each lane adding up what its eight values give to the weight's gradient; a
// block's sum goes to the workspace, where qkv_weight_grad_kernel adds the blocks' in their order: no
// atomics, the same bits each time.  While a warp works on a token the next one's dy, x and angles are
// on their way to its part of shared memory (held in registers they were requested only after the
// last token's use: 8192 tokens H32/8 D 128 59 us, here 49.6; with three stages 53.6, with three blocks
// on an SM 53.6).
template <int UNR>
struct BwdStage {  // of a warp
  uint4 dy[UNR][32], x[UNR][32];  // each lane's own
  float cos[64], sin[64];         // of the token; R / 2 of them
};

__device__ __forceinline__ void copy16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

template <int D, bool INTER, int UNR>
__global__ void __launch_bounds__(kWarps * 32, kBwdBlocksPerSm) qkv_norm_rope_bwd_kernel(const QkvParams p) {
  constexpr int LPH = D / 8, RPW = 32 / LPH;
  extern __shared__ __align__(16) uint8_t bwd_smem[];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i0 = 8 * (lane % LPH);
  const int src = partner_lane<D, INTER>(p, lane);
  Unit u = unit_of<D, UNR>(p, static_cast<long long>(blockIdx.x) * kWarps + warp);
  const int tokens = static_cast<int>(gridDim.x) * kWarps / (p.q_units + 2 * p.kv_units);  // from one to the next
  if (u.t >= tokens) u.t = p.T;
  const int h0 = u.h0 + lane / LPH;
  const int first = u.kind == kQuery ? 0 : u.kind == kKey ? p.Hq : p.Hq + p.Hkv;
  const long long at = static_cast<long long>(first + h0) * D + i0;
  const int half = p.R / 2;
  BwdStage<UNR>* stages = reinterpret_cast<BwdStage<UNR>*>(bwd_smem) + kBwdStages * warp;
  uint64_t w[4], gw[4];
  {
    float wf[8];
    load_weight(p, u.kind, i0, wf);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = f2(wf[2 * i], wf[2 * i + 1]);
      gw[i] = f2(0.f, 0.f);
    }
  }
  const auto after = [&](int t) { return p.T - t > tokens ? t + tokens : p.T; };
  // requests token t, whose position is pos
  const auto request = [&](BwdStage<UNR>& st, int t, int pos) {
    Unit v = u;
    v.t = t;
    long long head;
    const __nv_bfloat16* dy = place<D>(p, v, head) + i0;
    dy += h0 * head;
    const __nv_bfloat16* x = p.x + static_cast<long long>(t) * p.row_elems + at;
#pragma unroll
    for (int s = 0; s < UNR; ++s)
      if (h0 + s * RPW < u.heads) {
        copy16(&st.dy[s][lane], dy + s * RPW * head);
        if (u.kind != kValue) copy16(&st.x[s][lane], x + s * RPW * D);
      }
    if (u.kind != kValue && 4 * (lane & 15) < half) {
      const float* from = (lane < 16 ? p.cos : p.sin) + static_cast<long long>(pos) * half + 4 * (lane & 15);
      copy16((lane < 16 ? st.cos : st.sin) + 4 * (lane & 15), from);
    }
  };
  int to = u.t, ahead = 0, now = 0, free = 0;  // the token requested next, its position; stages
  const auto request_next = [&] {
    if (to < p.T) {
      request(stages[free], to, ahead);
      to = after(to);
      if (to < p.T) ahead = position(p, to);
    }
    free = free + 1 < kBwdStages ? free + 1 : 0;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (to < p.T) ahead = position(p, to);
#pragma unroll
  for (int i = 0; i + 1 < kBwdStages; ++i) request_next();
  for (; u.t < p.T; u.t = after(u.t), now = now + 1 < kBwdStages ? now + 1 : 0) {
    request_next();
    asm volatile("cp.async.wait_group %0;" ::"n"(kBwdStages - 1) : "memory");
    __syncwarp();
    const BwdStage<UNR>& st = stages[now];
    __nv_bfloat16* dx = p.dx + static_cast<long long>(u.t) * p.drow_elems + at;
    if (u.kind == kValue) {
#pragma unroll
      for (int s = 0; s < UNR; ++s)
        if (h0 + s * RPW < u.heads) __stcs(reinterpret_cast<uint4*>(dx + s * RPW * D), st.dy[s][lane]);
      continue;
    }
    uint64_t c[4], s[4];
    {
      float cf[8], sf[8];
      angles<INTER, true>(st.cos, st.sin, i0, half, cf, sf);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = f2(cf[2 * i], cf[2 * i + 1]);
        s[i] = f2(sf[2 * i], sf[2 * i + 1]);
      }
    }
#pragma unroll
    for (int k = 0; k < UNR; ++k) {
      const bool in = h0 + k * RPW < u.heads;
      const uint4 rdy = in ? st.dy[k][lane] : make_uint4(0, 0, 0, 0), rx = in ? st.x[k][lane] : make_uint4(0, 0, 0, 0);
      uint64_t z[4], g[4], o[4];
      unpack8(rx, z);
      unpack8(rdy, g);
      unpack8(partners<INTER>(rdy, src), o);
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = fma2(o[i], s[i], mul2(g[i], c[i]));
      const float r = rsqrtf(head_sum<LPH>(sum8(z, z)) * (1.f / D) + p.eps);
      const uint64_t r2 = f2(r, r);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        gw[i] = fma2(mul2(g[i], z[i]), r2, gw[i]);
        g[i] = mul2(g[i], w[i]);
      }
      const float m = -(r * r) * (head_sum<LPH>(sum8(g, z)) * (1.f / D));
      const uint64_t m2 = f2(m, m);
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = mul2(fma2(z[i], m2, g[i]), r2);
      if (in) __stcs(reinterpret_cast<uint4*>(dx + k * RPW * D), pack8(g));
    }
    __syncwarp();  // every lane has read the angles before the next request
  }
  __syncthreads();  // the stages become the warps' sums
  float(*sums)[2 * D] = reinterpret_cast<float(*)[2 * D]>(bwd_smem);
  // the warp's head groups, then the block's warps
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float a = i & 1 ? f2hi(gw[i / 2]) : f2lo(gw[i / 2]);
#pragma unroll
    for (int m = LPH; m < 32; m <<= 1) a += __shfl_xor_sync(0xffffffffu, a, m);
    if (lane < LPH) {
      sums[warp][i0 + i] = u.kind == kQuery ? a : 0.f;
      sums[warp][D + i0 + i] = u.kind == kKey ? a : 0.f;
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

// Adds the blocks' partial sums [n][2 D] in a fixed order: a block takes 8 of the 2 D columns, 128
// threads each.
__global__ void __launch_bounds__(1024) qkv_weight_grad_kernel(const float* partial, int n, int D, float* dwq, float* dwk) {
  __shared__ float sums[128][9], parts[4][8];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int x = threadIdx.x & 7, y = threadIdx.x >> 3;
  float a = 0.f;
#pragma unroll 4
  for (int i = y; i < n; i += 128) a += partial[static_cast<size_t>(i) * (2 * D) + blockIdx.x * 8 + x];
  sums[y][x] = a;
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;  // warp: column warp % 8, rows 32 (warp / 8) ..
  a = sums[(warp >> 3) * 32 + lane][warp & 7];
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) a += __shfl_xor_sync(0xffffffffu, a, m);
  if (lane == 0) parts[warp >> 3][warp & 7] = a;
  __syncthreads();
  if (threadIdx.x < 8) {
    const int i = blockIdx.x * 8 + x;
    (i < D ? dwq[i] : dwk[i - D]) = (parts[0][x] + parts[1][x]) + (parts[2][x] + parts[3][x]);
  }
}

// A launch as a programmatic dependent of the kernel before it in the stream: every kernel here
// waits for that one (griddepcontrol.wait) before its first access to memory.
template <class Kernel, class... Args>
cudaError_t launch(Kernel kernel, int grid, int threads, size_t smem, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
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
  p.w_f32 = a.weights_f32;
  p.cos = a.cos;
  p.sin = a.sin;
  p.pos = a.positions;
  p.T = a.T;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.R = a.R;
  p.P = a.P;
  const int heads = 256 / a.D * unroll;  // of a unit
  p.q_units = (a.Hq + heads - 1) / heads;
  p.kv_units = (a.Hkv + heads - 1) / heads;
  p.units = static_cast<long long>(a.T) * (p.q_units + 2 * p.kv_units);
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

// Blocks of four warps, whose places are free again sooner, where there are more warps than are
// resident (64 registers: 32 an SM); else of eight, of which there are fewer to start.  GB300, device us
// with eight / four / two warps: 8192 tokens H32/8 D 128 35.2 / 33.0 / 32.7, 30000 tokens 118 / 111 / 111,
// H16/2 D 64 41.9 / 40.0 / 60.9; 579 tokens H32/8 4.0 / 4.3 / 4.2.
template <int D, int UNR>
cudaError_t launch_fwd_u(const QkvArgs& a, cudaStream_t stream) {
  const QkvParams p = params_of(a, UNR);
  const int warps = p.units > 152 * 32 ? kWarps / 2 : kWarps;
  const long long blocks = (p.units + warps - 1) / warps;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  const int g = static_cast<int>(blocks);
  return a.interleaved ? launch(qkv_norm_rope_kernel<D, true, UNR>, g, warps * 32, 0, stream, p)
                       : launch(qkv_norm_rope_kernel<D, false, UNR>, g, warps * 32, 0, stream, p);
}

template <int D, int UNR>
cudaError_t launch_bwd_u(const QkvArgs& a, cudaStream_t stream) {
  const QkvParams p = params_of(a, UNR);
  // blocks whose warps are a multiple of a token's units (unless that is more than there is room for),
  // as many as there is room for or need of
  const int per = p.q_units + 2 * p.kv_units;
  static_assert(kMaxBwdHeads / (256 / D * 4) + 3 <= kMaxBwdBlocks * kWarps, "a token's units have a warp each");
  int unit = 1;
  while (unit < kMaxBwdBlocks && unit * kWarps % per) ++unit;
  const long long need = (p.units + static_cast<long long>(unit) * kWarps - 1) / (static_cast<long long>(unit) * kWarps);
  const int most = kMaxBwdBlocks / unit, g = static_cast<int>(need < most ? need : most) * unit;
  constexpr size_t smem = kBwdStages * kWarps * sizeof(BwdStage<UNR>);
  static_assert(smem >= kWarps * 2 * D * sizeof(float), "the stages hold the sums");
  const auto inter = qkv_norm_rope_bwd_kernel<D, true, UNR>, split = qkv_norm_rope_bwd_kernel<D, false, UNR>;
  static PerDeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.run(dev, [&] {
        return cudaFuncSetAttribute(inter, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess &&
               cudaFuncSetAttribute(split, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess;
      }))
    return cudaErrorInvalidValue;
  e = launch(a.interleaved ? inter : split, g, kWarps * 32, smem, stream, p);
  if (e != cudaSuccess) return e;
  return launch(qkv_weight_grad_kernel, 2 * D / 8, 1024, 0, stream, static_cast<const float*>(p.partial), g, D, a.dq_weight,
                a.dk_weight);
}

// Calls f(std::integral_constant<int, steps>) with the steps of a unit.
template <class F>
cudaError_t with_steps(const QkvArgs& a, F f) {
  if (static_cast<long long>(a.T) * (a.Hq + 2 * a.Hkv) * a.D < kManyValues) return f(std::integral_constant<int, 1>());
  const int heads = 256 / a.D;  // of a step
  const auto units = [&](int n) { return (a.Hq + heads * n - 1) / (heads * n) + 2 * ((a.Hkv + heads * n - 1) / (heads * n)); };
  return 2 * units(2) < 3 * units(4) ? f(std::integral_constant<int, 2>()) : f(std::integral_constant<int, 4>());
}

template <int D>
cudaError_t launch_fwd_d(const QkvArgs& a, cudaStream_t stream) {
  return with_steps(a, [&](auto n) { return launch_fwd_u<D, decltype(n)::value>(a, stream); });
}
template <int D>
cudaError_t launch_bwd_d(const QkvArgs& a, cudaStream_t stream) {
  return with_steps(a, [&](auto n) { return launch_bwd_u<D, decltype(n)::value>(a, stream); });
}

}  // namespace

cudaError_t launch_qkv_norm_rope(const QkvArgs& a, cudaStream_t stream) {
  return a.D == 128 ? launch_fwd_d<128>(a, stream) : launch_fwd_d<64>(a, stream);
}

cudaError_t launch_qkv_norm_rope_bwd(const QkvArgs& a, cudaStream_t stream) {
  return a.D == 128 ? launch_bwd_d<128>(a, stream) : launch_bwd_d<64>(a, stream);
}

size_t qkv_bwd_workspace_bytes(int D) { return static_cast<size_t>(kMaxBwdBlocks) * 2 * D * sizeof(float); }

}  // namespace loom
