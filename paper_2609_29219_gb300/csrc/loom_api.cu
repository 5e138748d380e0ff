// C ABI of the library (declared in include/loom_attn.h): argument validation, the
// device error word, the analytic model hook for the decode split count, and dispatch
// to the kernels.  No device memory is allocated here: the error word is a
// file-scope __device__ variable whose address is looked up once per device.
#include <cmath>
#include <cstdint>
#include <mutex>
#include <utility>
#include <vector>

#include "../../include/loom_attn.h"
#include "bwd.h"
#include "chunk.h"
#include "gemm.h"
#include "gemm_model.h"
#include "kernels.h"
#include "model.h"
#include "paged.h"
#include "qkv.h"
#include "varlen.h"

namespace loom {
namespace {

__device__ uint32_t g_error_word = 0;

constexpr uint64_t kDefaultTimeoutNs = 2000000000ull;  // 2 s
uint64_t g_timeout_ns = kDefaultTimeoutNs;
int g_inject = 0;
int g_prefill_design = 0;
int g_prefill_slots = 0;  // test hook: the two-tile prefill's K/V ring depth (0: the model's)
int g_gemm_tile_n = 0;  // test hook: forced GEMM tile width (0: the model's choice)
int g_gemm_splits = 0;  // test hook: forced GEMM split count (0: the model's choice)
int g_gemm_pair = 0;    // test hook: 1 forces CTA-pair tiles, -1 forbids them, 0: the model's choice
int g_gemm_stages = 0;  // test hook: GEMM ring depth (0: the model's; a compiled neighbour otherwise)
int g_gemm_group = 0;   // test hook: tile rows per group of the GEMM tile order (0: the default)
int g_gemm_k_alt = 0;   // test hook: -1 stops the CTA-pair GEMM walking K backwards every other round
int g_decode_form = 0;     // test hook: the Flash Decode form (0: the model's; kDecode* otherwise)
int g_decode_cluster = 0;  // test hook: the cluster decode form's cluster size (0: the model's)
int g_decode_stage_plan = 0;  // test hook: a compiled ablation stage plan of the decode split kernel
// test hook: the split + merge form's split kernel on a contiguous cache (DecodeArgs::tc)
int g_decode_tc = 1;

constexpr int kMaxDevices = 64;
uint32_t* g_err_ptr[kMaxDevices] = {};
std::mutex g_err_mutex;

// Device address of the error word on the current device (looked up once per device).
uint32_t* error_word_ptr() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  std::lock_guard<std::mutex> lock(g_err_mutex);
  if (!g_err_ptr[dev]) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_error_word) != cudaSuccess) return nullptr;
    g_err_ptr[dev] = static_cast<uint32_t*>(p);
  }
  return g_err_ptr[dev];
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int current_sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return sms;
}

// The current device's SMs, or the model's count without a device.
int sms_or_model() {
  const int sms = current_sm_count();
  return sms > 0 ? sms : model::kGb300.num_sms;
}

struct SplitKey {
  int B, Hq, Hkv, Skv, D, sms, tc;
  bool operator==(const SplitKey& o) const {
    return B == o.B && Hq == o.Hq && Hkv == o.Hkv && Skv == o.Skv && D == o.D && sms == o.sms && tc == o.tc;
  }
};
std::vector<std::pair<SplitKey, int>> g_split_cache;
std::mutex g_split_mutex;

bool make_ctl(KernelCtl* ctl) {
  ctl->err = error_word_ptr();
  ctl->timeout_ns = g_timeout_ns;
  ctl->inject = g_inject;
  return ctl->err != nullptr;
}

}  // namespace
}  // namespace loom

using namespace loom;

extern "C" {

const char* loom_status_string(loom_status s) {
  switch (s) {
    case LOOM_OK: return "LOOM_OK";
    case LOOM_ERR_INVALID_ARG: return "LOOM_ERR_INVALID_ARG";
    case LOOM_ERR_UNSUPPORTED: return "LOOM_ERR_UNSUPPORTED";
    case LOOM_ERR_MISALIGNED: return "LOOM_ERR_MISALIGNED";
    case LOOM_ERR_WORKSPACE: return "LOOM_ERR_WORKSPACE";
    case LOOM_ERR_CUDA: return "LOOM_ERR_CUDA";
    case LOOM_ERR_TIMEOUT: return "LOOM_ERR_TIMEOUT";
  }
  return "LOOM_ERR_UNKNOWN";
}

loom_status loom_attn_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int B,
                          int Hq, int Hkv, int Sq, int Skv, int D, int causal, float scale,
                          void* stream) {
  if (!q || !k || !v || !o) return LOOM_ERR_INVALID_ARG;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Skv <= 0 || D <= 0) return LOOM_ERR_INVALID_ARG;
  if (Hq % Hkv != 0) return LOOM_ERR_INVALID_ARG;
  if (causal != 0 && causal != 1) return LOOM_ERR_INVALID_ARG;
  if (causal && Sq > Skv) return LOOM_ERR_INVALID_ARG;
  if (!std::isfinite(scale) || scale <= 0.f) return LOOM_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return LOOM_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return LOOM_ERR_MISALIGNED;
  if (lse && (reinterpret_cast<uintptr_t>(lse) & 3u)) return LOOM_ERR_MISALIGNED;
  // TMA views use 32-bit coordinates: rows and planes must fit
  if (static_cast<long long>(B) * Hq > 0x7fffffff || static_cast<long long>(B) * Hkv > 0x7fffffff)
    return LOOM_ERR_UNSUPPORTED;
  KernelCtl ctl;
  if (!make_ctl(&ctl)) return LOOM_ERR_CUDA;
  FwdArgs a{q, k, v, o, lse, B, Hq, Hkv, Sq, Skv, D, causal, scale, g_prefill_design, g_prefill_slots};
  return launch_fwd(a, ctl, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK
                                                                               : LOOM_ERR_CUDA;
}

int loom_attn_fwd_cluster(int B, int Hq, int Hkv, int Sq, int Skv, int D, int causal) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || Sq <= 0 || Skv <= 0 || (D != 64 && D != 128)) return 0;
  if ((causal != 0 && causal != 1) || (causal && Sq > Skv) || static_cast<long long>(B) * Hq > 0x7fffffff) return 0;
  const FwdArgs a{nullptr, nullptr, nullptr, nullptr, nullptr, B, Hq, Hkv, Sq, Skv, D, causal, 1.f, g_prefill_design,
                  g_prefill_slots};
  const int n = fwd_cluster_of(a);
  cudaGetLastError();
  return n;
}

int loom_attn_decode_num_splits(int B, int Hq, int Hkv, int Skv, int D) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Skv <= 0 || Hq % Hkv != 0) return 0;
  if (D != 64 && D != 128) return 0;
  const int sms = sms_or_model();
  // The enumeration costs ~0.1 ms of host time: remember the answer per problem shape.
  // the split + merge form's split kernel runs on the tensor cores for a contiguous cache
  // (a paged cache takes the same split count, with the CUDA-core kernel)
  const int tc = (g_decode_tc != 0 && Hq / Hkv <= kDecodeTcMaxGroup) ? 1 : 0;
  const SplitKey key{B, Hq, Hkv, Skv, D, sms, tc};
  {
    std::lock_guard<std::mutex> lock(g_split_mutex);
    for (const auto& e : g_split_cache)
      if (e.first == key) return e.second;
  }
  // Both Flash Decode forms compete (Eq. 9); the cluster form's CTA slots come from the
  // device, or from the GB300 estimate when no device answers.
  const bool device = current_sm_count() > 0;
  const int G = Hq / Hkv;
  // (the CUDA-core persistent split kernel is a candidate only where the tensor-core one
  // does not run)
  const int slots = tc ? 0 : device ? decode_persistent_slots(D, G) : sms * model::decode_stage(D).ctas_per_sm;
  const int splits = model::choose_decode_plan(
                         B, Hq, Hkv, Skv, D, sms,
                         [&](int cs) {
                           return device ? decode_max_clusters(D, G, cs) : model::decode_default_clusters(sms, cs, D);
                         },
                         slots, model::kGb300, tc != 0)
                         .splits;
  std::lock_guard<std::mutex> lock(g_split_mutex);
  if (g_split_cache.size() >= 256) g_split_cache.erase(g_split_cache.begin());
  g_split_cache.emplace_back(key, splits);
  return splits;
}

size_t loom_attn_decode_workspace_bytes(int B, int Hq, int Hkv, int Skv, int D, int num_splits) {
  if (num_splits == 0) {
    num_splits = loom_attn_decode_num_splits(B, Hq, Hkv, Skv, D);
    if (num_splits > 0) num_splits = decode_ragged_splits(B, Hq, Hkv, Skv, D, num_splits, sms_or_model());
  }
  if (num_splits <= 0 || num_splits > kMaxDecodeSplits) return 0;
  if (B <= 0 || Hq <= 0 || (D != 64 && D != 128)) return 0;
  return decode_workspace_bytes(B, Hq, D, num_splits);
}

}  // extern "C"

namespace loom {
// Every check of the contiguous decode entry points that comes before the workspace: on
// LOOM_OK, *splits is the split count the call will use (the model's when num_splits = 0).
int decode_check_args(const void* q, const void* k_cache, const void* v_cache, const int32_t* seqlens_k,
                      const void* o, const float* lse, int B, int Hq, int Hkv, int Skv, int D, float scale,
                      int num_splits, int* splits) {
  if (!q || !k_cache || !v_cache || !o) return LOOM_ERR_INVALID_ARG;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Skv <= 0 || D <= 0) return LOOM_ERR_INVALID_ARG;
  if (Hq % Hkv != 0) return LOOM_ERR_INVALID_ARG;
  if (!std::isfinite(scale) || scale <= 0.f) return LOOM_ERR_INVALID_ARG;
  if (num_splits < 0) return LOOM_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return LOOM_ERR_UNSUPPORTED;
  if (num_splits > kMaxDecodeSplits) return LOOM_ERR_UNSUPPORTED;
  if (static_cast<long long>(B) * Hq * (num_splits ? num_splits : 1) > 0x7fffffffLL ||
      static_cast<long long>(B) > 65535)
    return LOOM_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o))
    return LOOM_ERR_MISALIGNED;
  if ((lse && (reinterpret_cast<uintptr_t>(lse) & 3u)) ||
      (seqlens_k && (reinterpret_cast<uintptr_t>(seqlens_k) & 3u)))
    return LOOM_ERR_MISALIGNED;
  if (num_splits == 0) num_splits = loom_attn_decode_num_splits(B, Hq, Hkv, Skv, D);
  if (num_splits <= 0) return LOOM_ERR_INVALID_ARG;
  *splits = num_splits;
  return LOOM_OK;
}

namespace {
// With the model's count and lengths on the device, lays the partials out for the larger
// count of a ragged batch where the workspace holds it: *splits becomes that count and the
// model's is returned (0: nothing changes).
int ragged_layout(bool lengths, int B, int Hq, int Hkv, int Skv, int D, size_t workspace_bytes, int* splits) {
  if (!lengths) return 0;
  const int r = decode_ragged_splits(B, Hq, Hkv, Skv, D, *splits, sms_or_model());
  if (r == *splits || decode_workspace_bytes(B, Hq, D, r) > workspace_bytes) return 0;
  const int equal = *splits;
  *splits = r;
  return equal;
}
}  // namespace
}  // namespace loom

extern "C" {

loom_status loom_attn_decode(const void* q, const void* k_cache, const void* v_cache,
                             const int32_t* seqlens_k, void* o, float* lse, void* workspace,
                             size_t workspace_bytes, int B, int Hq, int Hkv, int Skv, int D,
                             float scale, int num_splits, void* stream) {
  const int by_model = num_splits == 0 ? 1 : 0;
  const int st = decode_check_args(q, k_cache, v_cache, seqlens_k, o, lse, B, Hq, Hkv, Skv, D, scale, num_splits,
                                   &num_splits);
  if (st != LOOM_OK) return static_cast<loom_status>(st);
  const size_t need = decode_workspace_bytes(B, Hq, D, num_splits);
  if (!workspace || workspace_bytes < need) return LOOM_ERR_WORKSPACE;
  if (!aligned16(workspace)) return LOOM_ERR_MISALIGNED;
  const int equal_splits = ragged_layout(by_model && seqlens_k, B, Hq, Hkv, Skv, D, workspace_bytes, &num_splits);
  KernelCtl ctl;
  if (!make_ctl(&ctl)) return LOOM_ERR_CUDA;
  const size_t rows = static_cast<size_t>(B) * Hq * num_splits;
  float* o_part = static_cast<float*>(workspace);
  float* lse_part = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                             (rows * D * sizeof(float) + 255) / 256 * 256);
  DecodeArgs a{q, k_cache, v_cache, seqlens_k, o, lse, o_part, lse_part, B, Hq, Hkv, Skv, D,
               num_splits, scale, g_decode_form, g_decode_cluster, g_decode_stage_plan, by_model, g_decode_tc,
               decode_sched_word(workspace, B, Hq, D, num_splits), equal_splits};
  return launch_decode(a, ctl, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK
                                                                                 : LOOM_ERR_CUDA;
}

loom_status loom_attn_fwd_varlen(const void* q, const void* k, const void* v, void* o, float* lse,
                                 const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int B,
                                 int Hq, int Hkv, int total_q, int total_k, int max_seqlen_q, int D,
                                 int causal, float scale, void* stream) {
  if (!q || !k || !v || !o || !cu_seqlens_q || !cu_seqlens_k) return LOOM_ERR_INVALID_ARG;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || D <= 0 || total_q < 0 || total_k < 0 || max_seqlen_q < 0)
    return LOOM_ERR_INVALID_ARG;
  if (Hq % Hkv != 0) return LOOM_ERR_INVALID_ARG;
  if (!std::isfinite(scale) || scale <= 0.f) return LOOM_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return LOOM_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return LOOM_ERR_MISALIGNED;
  if ((reinterpret_cast<uintptr_t>(cu_seqlens_q) & 3u) || (reinterpret_cast<uintptr_t>(cu_seqlens_k) & 3u) ||
      (lse && (reinterpret_cast<uintptr_t>(lse) & 3u)))
    return LOOM_ERR_MISALIGNED;
  if (total_q == 0) return LOOM_OK;
  if (total_k == 0) return LOOM_ERR_UNSUPPORTED;
  // work items (query-tile pairs x heads) are at most (total_q / 256 + B) * Hq
  if ((static_cast<long long>(total_q) / 256 + B) * Hq > 0x7fffffffLL) return LOOM_ERR_UNSUPPORTED;
  KernelCtl ctl;
  if (!make_ctl(&ctl)) return LOOM_ERR_CUDA;
  FwdVarlenArgs a{q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, B, Hq, Hkv, total_q, total_k, max_seqlen_q, D,
                  causal ? 1 : 0, scale};
  return launch_fwd_varlen(a, ctl, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
}

loom_status loom_attn_decode_paged(const void* q, const void* k_cache, const void* v_cache,
                                   const int32_t* block_table, const int32_t* seqlens_k, void* o,
                                   float* lse, void* workspace, size_t workspace_bytes, int B, int Hq,
                                   int Hkv, int num_pages, int page_size, int max_pages, int kv_layout,
                                   int D, float scale, int num_splits, void* stream) {
  if (!q || !k_cache || !v_cache || !o || !block_table || !seqlens_k) return LOOM_ERR_INVALID_ARG;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || num_pages <= 0 || page_size <= 0 || max_pages <= 0 || D <= 0)
    return LOOM_ERR_INVALID_ARG;
  if (Hq % Hkv != 0) return LOOM_ERR_INVALID_ARG;
  if (!std::isfinite(scale) || scale <= 0.f) return LOOM_ERR_INVALID_ARG;
  if (num_splits < 0) return LOOM_ERR_INVALID_ARG;
  if (kv_layout != kPagedNHD && kv_layout != kPagedHND) return LOOM_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return LOOM_ERR_UNSUPPORTED;
  if (!paged_page_size_ok(page_size)) return LOOM_ERR_UNSUPPORTED;
  if (static_cast<long long>(num_pages) * page_size > 0x7fffffffLL ||
      static_cast<long long>(num_pages) * Hkv > 0x7fffffffLL ||
      static_cast<long long>(max_pages) * page_size > 0x7fffffffLL ||
      static_cast<long long>(B) * max_pages > 0x7fffffffLL)
    return LOOM_ERR_UNSUPPORTED;
  if (num_splits > kMaxDecodeSplits) return LOOM_ERR_UNSUPPORTED;
  if (static_cast<long long>(B) * Hq * (num_splits ? num_splits : 1) > 0x7fffffffLL ||
      static_cast<long long>(B) > 65535)
    return LOOM_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o)) return LOOM_ERR_MISALIGNED;
  if ((reinterpret_cast<uintptr_t>(block_table) & 3u) || (reinterpret_cast<uintptr_t>(seqlens_k) & 3u) ||
      (lse && (reinterpret_cast<uintptr_t>(lse) & 3u)))
    return LOOM_ERR_MISALIGNED;
  const int Skv = max_pages * page_size;
  const int by_model = num_splits == 0 ? 1 : 0;
  if (num_splits == 0) num_splits = loom_attn_decode_num_splits(B, Hq, Hkv, Skv, D);
  if (num_splits <= 0) return LOOM_ERR_INVALID_ARG;
  const size_t need = decode_workspace_bytes(B, Hq, D, num_splits);
  if (!workspace || workspace_bytes < need) return LOOM_ERR_WORKSPACE;
  if (!aligned16(workspace)) return LOOM_ERR_MISALIGNED;
  const int equal_splits = ragged_layout(by_model && seqlens_k, B, Hq, Hkv, Skv, D, workspace_bytes, &num_splits);
  KernelCtl ctl;
  if (!make_ctl(&ctl)) return LOOM_ERR_CUDA;
  const size_t rows = static_cast<size_t>(B) * Hq * num_splits;
  float* o_part = static_cast<float*>(workspace);
  float* lse_part = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                             (rows * D * sizeof(float) + 255) / 256 * 256);
  DecodeArgs a{q, k_cache, v_cache, seqlens_k, o, lse, o_part, lse_part, B, Hq, Hkv, Skv, D, num_splits, scale,
               g_decode_form, g_decode_cluster, 0, by_model, g_decode_tc,
               decode_sched_word(workspace, B, Hq, D, num_splits), equal_splits};
  PagedKV pk{block_table, num_pages, page_size, max_pages, kv_layout};
  return launch_decode_paged(a, pk, ctl, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK
                                                                                          : LOOM_ERR_CUDA;
}

namespace {
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Sizes of a backward call that have a workspace: items and row statistics within 32 bits.
bool bwd_sizes_fit(int B, int Hq, int Hkv, long long Sq, long long Skv, bool ragged) {
  const int lg = bwd_pack_log2(Hq / Hkv);
  const long long heads = ragged ? Hq : static_cast<long long>(B) * Hq;
  const long long kv_planes = ragged ? Hkv : static_cast<long long>(B) * Hkv;
  return heads <= 0x7fffffffLL && Sq << lg <= 0x3fffffffLL && Skv <= 0x3fffffffLL &&
         (heads >> lg) * bwd_stat_tiles(B, Sq, lg, ragged) <= 0x1fffffffLL &&
         kv_planes * (Skv / 128 + (ragged ? B : 1)) <= 0x3fffffffLL;
}

loom_status bwd_call(const BwdArgs& a, size_t workspace_bytes, void* stream) {
  const bool ragged = a.cu_q != nullptr;
  if (a.Hq % a.Hkv != 0) return LOOM_ERR_INVALID_ARG;
  if (!std::isfinite(a.scale) || a.scale <= 0.f) return LOOM_ERR_INVALID_ARG;
  if (a.D != 64 && a.D != 128) return LOOM_ERR_UNSUPPORTED;
  if (!bwd_sizes_fit(a.B, a.Hq, a.Hkv, a.Sq, a.Skv, ragged)) return LOOM_ERR_UNSUPPORTED;
  for (const void* p : {a.dout, a.q, a.k, a.v, a.o, static_cast<const void*>(a.dq), static_cast<const void*>(a.dk),
                        static_cast<const void*>(a.dv)})
    if (!aligned16(p)) return LOOM_ERR_MISALIGNED;
  if (!aligned4(a.lse) || !aligned4(a.dlse) || !aligned4(a.cu_q) || !aligned4(a.cu_k)) return LOOM_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.Sq == 0 || a.Skv == 0) {  // ragged: no queries or no keys at all, so no gradient
    const size_t row = static_cast<size_t>(a.D) * 2;
    cudaError_t e = cudaSuccess;
    if (a.Sq > 0) e = cudaMemsetAsync(a.dq, 0, row * a.Hq * a.Sq, s);
    if (e == cudaSuccess && a.Skv > 0) e = cudaMemsetAsync(a.dk, 0, row * a.Hkv * a.Skv, s);
    if (e == cudaSuccess && a.Skv > 0) e = cudaMemsetAsync(a.dv, 0, row * a.Hkv * a.Skv, s);
    return e == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
  }
  if (!a.workspace || workspace_bytes < bwd_workspace(a.B, a.Hq, a.Hkv, a.Sq, a.Skv, a.D, ragged, sms_or_model()))
    return LOOM_ERR_WORKSPACE;
  if (!aligned16(a.workspace)) return LOOM_ERR_MISALIGNED;
  KernelCtl ctl;
  if (!make_ctl(&ctl)) return LOOM_ERR_CUDA;
  return launch_attn_bwd(a, ctl, s) == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
}
}  // namespace

size_t loom_attn_bwd_workspace_bytes(int B, int Hq, int Hkv, int Sq, int Skv, int D) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Skv <= 0 || Hq % Hkv || (D != 64 && D != 128)) return 0;
  return bwd_sizes_fit(B, Hq, Hkv, Sq, Skv, false) ? bwd_workspace(B, Hq, Hkv, Sq, Skv, D, false, sms_or_model()) : 0;
}

size_t loom_attn_bwd_varlen_workspace_bytes(int B, int Hq, int Hkv, int total_q, int total_k, int D) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || total_q < 0 || total_k < 0 || Hq % Hkv || (D != 64 && D != 128)) return 0;
  return bwd_sizes_fit(B, Hq, Hkv, total_q, total_k, true) ? bwd_workspace(B, Hq, Hkv, total_q, total_k, D, true, sms_or_model()) : 0;
}

loom_status loom_attn_bwd_plan(int B, int Hq, int Hkv, int Sq, int Skv, int D, int causal, int ragged, int* plan) {
  if (!plan || B <= 0 || Hq <= 0 || Hkv <= 0 || Sq < !ragged || Skv < !ragged || D <= 0) return LOOM_ERR_INVALID_ARG;
  if (Hq % Hkv || (causal != 0 && causal != 1) || (ragged != 0 && ragged != 1) || (!ragged && causal && Sq > Skv))
    return LOOM_ERR_INVALID_ARG;
  if ((D != 64 && D != 128) || !bwd_sizes_fit(B, Hq, Hkv, Sq, Skv, ragged != 0)) return LOOM_ERR_UNSUPPORTED;
  const BwdPlan p = bwd_plan(B, Hq, Hkv, Sq, Skv, D, ragged != 0, causal != 0, sms_or_model());
  plan[0] = p.kv_split;
  plan[1] = p.q_split;
  plan[2] = p.kv_block;
  plan[3] = p.q_block;
  return LOOM_OK;
}

loom_status loom_attn_bwd(const void* dout, const void* q, const void* k, const void* v, const void* o, const float* lse,
                          const float* dlse, void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes, int B,
                          int Hq, int Hkv, int Sq, int Skv, int D, int causal, float scale, void* stream) {
  if (!dout || !q || !k || !v || !o || !lse || !dq || !dk || !dv) return LOOM_ERR_INVALID_ARG;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Skv <= 0 || D <= 0) return LOOM_ERR_INVALID_ARG;
  if ((causal != 0 && causal != 1) || (causal && Sq > Skv)) return LOOM_ERR_INVALID_ARG;
  const BwdArgs a{dout, q, k, v, o, lse, dlse, dq, dk, dv, workspace, B, Hq, Hkv, Sq, Skv, D, causal, scale,
                  nullptr, nullptr, 0, 0};
  return bwd_call(a, workspace_bytes, stream);
}

loom_status loom_attn_bwd_varlen(const void* dout, const void* q, const void* k, const void* v, const void* o,
                                 const float* lse, const float* dlse, void* dq, void* dk, void* dv,
                                 const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, void* workspace,
                                 size_t workspace_bytes, int B, int Hq, int Hkv, int total_q, int total_k, int max_seqlen_q,
                                 int max_seqlen_k, int D, int causal, float scale, void* stream) {
  if (!cu_seqlens_q || !cu_seqlens_k) return LOOM_ERR_INVALID_ARG;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || total_q < 0 || total_k < 0 || max_seqlen_q < 0 || max_seqlen_k < 0 || D <= 0)
    return LOOM_ERR_INVALID_ARG;
  if (total_q > 0 && (!dout || !q || !o || !lse || !dq)) return LOOM_ERR_INVALID_ARG;
  if (total_k > 0 && (!k || !v || !dk || !dv)) return LOOM_ERR_INVALID_ARG;
  if (causal != 0 && causal != 1) return LOOM_ERR_INVALID_ARG;
  const BwdArgs a{dout, q, k, v, o, lse, dlse, dq, dk, dv, workspace, B, Hq, Hkv, total_q, total_k, D, causal, scale,
                  cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k};
  return bwd_call(a, workspace_bytes, stream);
}

namespace {
// Sizes of a chunk call that there is a kernel for.
bool chunk_sizes_ok(int B, int Hq, int Hkv, int total_q, int D) {
  return (D == 64 || D == 128) && Hq <= kMaxChunkHeads && static_cast<long long>(total_q) * Hq <= 0x7fffffffLL;
}
}  // namespace

size_t loom_attn_chunk_paged_workspace_bytes(int B, int Hq, int Hkv, int total_q, int D) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || total_q < 0 || Hq % Hkv != 0 || !chunk_sizes_ok(B, Hq, Hkv, total_q, D)) return 0;
  return chunk_workspace_bytes(Hq, Hkv, total_q, D, sms_or_model());
}

loom_status loom_attn_chunk_paged(const void* q, const void* k_cache, const void* v_cache, const int32_t* block_table,
                                  const int32_t* cu_seqlens_q, const int32_t* seqlens_k, void* o, float* lse,
                                  void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int total_q,
                                  int num_pages, int page_size, int max_pages, int kv_layout, int D, int causal,
                                  float scale, void* stream) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || num_pages <= 0 || page_size <= 0 || max_pages <= 0 || D <= 0 || total_q < 0)
    return LOOM_ERR_INVALID_ARG;
  if (!k_cache || !v_cache || !block_table || !cu_seqlens_q || !seqlens_k || (total_q > 0 && (!q || !o)))
    return LOOM_ERR_INVALID_ARG;
  if (Hq % Hkv != 0) return LOOM_ERR_INVALID_ARG;
  if (causal != 0 && causal != 1) return LOOM_ERR_INVALID_ARG;
  if (!std::isfinite(scale) || scale <= 0.f) return LOOM_ERR_INVALID_ARG;
  if (kv_layout != kPagedNHD && kv_layout != kPagedHND) return LOOM_ERR_INVALID_ARG;
  if (!chunk_sizes_ok(B, Hq, Hkv, total_q, D) || !paged_page_size_ok(page_size)) return LOOM_ERR_UNSUPPORTED;
  if (static_cast<long long>(num_pages) * page_size > 0x7fffffffLL ||
      static_cast<long long>(num_pages) * Hkv > 0x7fffffffLL ||
      static_cast<long long>(max_pages) * page_size > 0x7fffffffLL ||
      static_cast<long long>(B) * max_pages > 0x7fffffffLL)
    return LOOM_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o)) return LOOM_ERR_MISALIGNED;
  if (!aligned4(block_table) || !aligned4(cu_seqlens_q) || !aligned4(seqlens_k) || !aligned4(lse)) return LOOM_ERR_MISALIGNED;
  if (total_q == 0) return LOOM_OK;
  if (!workspace || workspace_bytes < chunk_workspace_bytes(Hq, Hkv, total_q, D, sms_or_model())) return LOOM_ERR_WORKSPACE;
  if (!aligned16(workspace)) return LOOM_ERR_MISALIGNED;
  KernelCtl ctl;
  if (!make_ctl(&ctl)) return LOOM_ERR_CUDA;
  const ChunkArgs a{q, k_cache, v_cache, cu_seqlens_q, seqlens_k, o, lse, workspace, B, Hq, Hkv, total_q, D, causal, scale,
                    PagedKV{block_table, num_pages, page_size, max_pages, kv_layout}};
  return launch_chunk_paged(a, ctl, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
}

loom_status loom_paged_plan(const int32_t* new_lens, const int32_t* lens, int32_t* block_table, int32_t* free_pages,
                            const int32_t* free_count, int32_t* free_count_out, int32_t* cu_seqlens, int32_t* seqlens_k,
                            int32_t* positions, int32_t* slots, int32_t* granted, int B, int T, int num_pages,
                            int page_size, int max_pages, void* stream) {
  if (B <= 0 || T < 0 || num_pages <= 0 || page_size <= 0 || max_pages <= 0) return LOOM_ERR_INVALID_ARG;
  if (!new_lens || !lens || !block_table || !free_pages || !free_count || !free_count_out || !cu_seqlens || !seqlens_k ||
      !granted || (T > 0 && (!positions || !slots)))
    return LOOM_ERR_INVALID_ARG;
  if (B > kMaxPlanB || static_cast<long long>(num_pages) * page_size > 0x7fffffffLL ||
      static_cast<long long>(max_pages) * page_size > 0x7fffffffLL || static_cast<long long>(B) * max_pages > 0x7fffffffLL)
    return LOOM_ERR_UNSUPPORTED;
  for (const void* p : {static_cast<const void*>(new_lens), static_cast<const void*>(lens), static_cast<const void*>(block_table),
                        static_cast<const void*>(free_pages), static_cast<const void*>(free_count),
                        static_cast<const void*>(free_count_out), static_cast<const void*>(cu_seqlens),
                        static_cast<const void*>(seqlens_k), static_cast<const void*>(positions),
                        static_cast<const void*>(slots), static_cast<const void*>(granted)})
    if (!aligned4(p)) return LOOM_ERR_MISALIGNED;
  const PlanArgs a{new_lens, lens, block_table, free_pages, free_count, free_count_out, cu_seqlens, seqlens_k, positions, slots,
                   granted, B, T, num_pages, page_size, max_pages};
  return launch_paged_plan(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
}

namespace {
// The arguments that the three norm-and-rotation entry points share, checked; *a is filled in.
loom_status qkv_common(QkvArgs* a, const void* qkv, int64_t qkv_stride, const void* q_weight, const void* k_weight,
                       int weight_type, const float* cos, const float* sin, int table_rows, int rotary_dim, int interleaved,
                       const int32_t* positions, int T, int Hq, int Hkv, int D, float eps) {
  if (T < 0 || Hq <= 0 || Hkv <= 0 || D <= 0 || table_rows <= 0) return LOOM_ERR_INVALID_ARG;
  if (!q_weight || !k_weight || !cos || !sin || (T > 0 && !qkv)) return LOOM_ERR_INVALID_ARG;
  if (weight_type != LOOM_BF16 && weight_type != LOOM_FP32) return LOOM_ERR_INVALID_ARG;
  if (interleaved != 0 && interleaved != 1) return LOOM_ERR_INVALID_ARG;
  if (!std::isfinite(eps) || eps <= 0.f) return LOOM_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return LOOM_ERR_UNSUPPORTED;
  if (rotary_dim < 16 || rotary_dim > D || rotary_dim % 16) return LOOM_ERR_UNSUPPORTED;
  const long long heads = static_cast<long long>(Hq) + 2ll * Hkv;
  if (heads * D > 0x3fffffffLL) return LOOM_ERR_UNSUPPORTED;
  if (qkv_stride < heads * D) return LOOM_ERR_INVALID_ARG;
  if (qkv_stride % 8) return LOOM_ERR_MISALIGNED;
  if (!aligned16(qkv) || !aligned16(q_weight) || !aligned16(k_weight) || !aligned16(cos) || !aligned16(sin))
    return LOOM_ERR_MISALIGNED;
  if (!aligned4(positions)) return LOOM_ERR_MISALIGNED;
  a->qkv = qkv;
  a->row_elems = qkv_stride;
  a->q_weight = q_weight;
  a->k_weight = k_weight;
  a->weights_f32 = weight_type == LOOM_FP32;
  a->cos = cos;
  a->sin = sin;
  a->positions = positions;
  a->T = T;
  a->Hq = Hq;
  a->Hkv = Hkv;
  a->D = D;
  a->R = rotary_dim;
  a->P = table_rows;
  a->interleaved = interleaved;
  a->eps = eps;
  return LOOM_OK;
}

// Whether the tables have a row for each position that no positions given imply.
bool tables_reach(const int32_t* positions, int T, int seq_len, int table_rows) {
  return positions || T == 0 || (seq_len > 0 ? seq_len : T) <= table_rows;
}
}  // namespace

namespace {
// The positions of the calls with axes, checked; *a is filled in (after qkv_common).
loom_status axes_args(QkvArgs* a, int64_t positions_stride, int n_axes, const int* pair_axis) {
  if (n_axes < 1 || !pair_axis || positions_stride < a->T || (a->T > 0 && !a->positions)) return LOOM_ERR_INVALID_ARG;
  if (n_axes > kMaxAxes) return LOOM_ERR_UNSUPPORTED;
  for (int i = 0; i < a->R / 2; ++i) {
    if (pair_axis[i] < 0 || pair_axis[i] >= n_axes) return LOOM_ERR_INVALID_ARG;
    a->axis_of[i / 32] |= static_cast<unsigned long long>(pair_axis[i]) << (2 * (i % 32));
  }
  a->n_axes = n_axes;
  a->pos_stride = positions_stride;
  return LOOM_OK;
}

loom_status norm_rope_call(QkvArgs& a, void* q, void* k, void* v, int seq_len, void* stream) {
  if (seq_len < 0 || (seq_len > 0 && a.T % seq_len) || (a.T > 0 && (!q || !k || !v))) return LOOM_ERR_INVALID_ARG;
  if (!tables_reach(a.positions, a.T, seq_len, a.P)) return LOOM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v)) return LOOM_ERR_MISALIGNED;
  if (a.T == 0) return LOOM_OK;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_at.S = a.kv_at.S = seq_len;
  a.q_at.H = a.Hq;
  a.kv_at.H = a.Hkv;
  return launch_qkv_norm_rope(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
}

loom_status norm_rope_cache_call(QkvArgs& a, const int32_t* slots, void* q, void* k_cache, void* v_cache, int num_pages,
                                 int page_size, int kv_layout, void* stream) {
  if (num_pages <= 0 || page_size <= 0 || (kv_layout != kPagedNHD && kv_layout != kPagedHND)) return LOOM_ERR_INVALID_ARG;
  if (!k_cache || !v_cache || (a.T > 0 && (!q || !a.positions || !slots))) return LOOM_ERR_INVALID_ARG;
  if (static_cast<long long>(num_pages) * page_size > 0x7fffffffLL) return LOOM_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned4(slots)) return LOOM_ERR_MISALIGNED;
  if (a.T == 0) return LOOM_OK;
  a.q = q;
  a.k = k_cache;
  a.v = v_cache;
  a.q_at.H = a.Hq;
  a.kv_at.H = a.Hkv;
  a.kv_at.slots = slots;
  a.kv_at.page = page_size;
  a.kv_at.n_slots = num_pages * page_size;
  a.kv_at.page_elems = static_cast<long long>(page_size) * a.Hkv * a.D;
  a.kv_at.row_elems = kv_layout == kPagedNHD ? static_cast<long long>(a.Hkv) * a.D : a.D;
  a.kv_at.head_elems = kv_layout == kPagedNHD ? a.D : static_cast<long long>(page_size) * a.D;
  return launch_qkv_norm_rope(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
}

loom_status norm_rope_bwd_call(QkvArgs& a, const void* dq, const void* dk, const void* dv, void* dqkv, int64_t dqkv_stride,
                               float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes, int seq_len,
                               void* stream) {
  if (seq_len < 0 || (seq_len > 0 && a.T % seq_len) || (a.T > 0 && (!dq || !dk || !dv || !dqkv))) return LOOM_ERR_INVALID_ARG;
  if (!dq_weight || !dk_weight) return LOOM_ERR_INVALID_ARG;
  if (!tables_reach(a.positions, a.T, seq_len, a.P)) return LOOM_ERR_INVALID_ARG;
  if (dqkv_stride < (static_cast<int64_t>(a.Hq) + 2ll * a.Hkv) * a.D) return LOOM_ERR_INVALID_ARG;
  if (a.Hq + 2ll * a.Hkv > kMaxBwdHeads) return LOOM_ERR_UNSUPPORTED;
  if (dqkv_stride % 8 || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned16(dqkv) || !aligned4(dq_weight) ||
      !aligned4(dk_weight))
    return LOOM_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.T == 0) {
    const bool ok = cudaMemsetAsync(dq_weight, 0, a.D * sizeof(float), s) == cudaSuccess &&
                    cudaMemsetAsync(dk_weight, 0, a.D * sizeof(float), s) == cudaSuccess;
    return ok ? LOOM_OK : LOOM_ERR_CUDA;
  }
  if (!workspace || workspace_bytes < qkv_bwd_workspace_bytes(a.D)) return LOOM_ERR_WORKSPACE;
  if (!aligned16(workspace)) return LOOM_ERR_MISALIGNED;
  a.q = const_cast<void*>(dq);
  a.k = const_cast<void*>(dk);
  a.v = const_cast<void*>(dv);
  a.q_at.S = a.kv_at.S = seq_len;
  a.q_at.H = a.Hq;
  a.kv_at.H = a.Hkv;
  a.dqkv = dqkv;
  a.drow_elems = dqkv_stride;
  a.dq_weight = dq_weight;
  a.dk_weight = dk_weight;
  a.partial = static_cast<float*>(workspace);
  return launch_qkv_norm_rope_bwd(a, s) == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
}
}  // namespace

loom_status loom_qkv_norm_rope(const void* qkv, int64_t qkv_stride, const void* q_weight, const void* k_weight,
                               int weight_type, const float* cos, const float* sin, int table_rows, int rotary_dim,
                               int interleaved, const int32_t* positions, void* q, void* k, void* v, int T,
                               int seq_len, int Hq, int Hkv, int D, float eps, void* stream) {
  QkvArgs a{};
  const loom_status st = qkv_common(&a, qkv, qkv_stride, q_weight, k_weight, weight_type, cos, sin, table_rows, rotary_dim,
                                    interleaved, positions, T, Hq, Hkv, D, eps);
  return st != LOOM_OK ? st : norm_rope_call(a, q, k, v, seq_len, stream);
}

loom_status loom_qkv_norm_rope_cache(const void* qkv, int64_t qkv_stride, const void* q_weight, const void* k_weight,
                                     int weight_type, const float* cos, const float* sin, int table_rows,
                                     int rotary_dim, int interleaved, const int32_t* positions, const int32_t* slots,
                                     void* q, void* k_cache, void* v_cache, int num_pages, int page_size,
                                     int kv_layout, int T, int Hq, int Hkv, int D, float eps, void* stream) {
  QkvArgs a{};
  const loom_status st = qkv_common(&a, qkv, qkv_stride, q_weight, k_weight, weight_type, cos, sin, table_rows, rotary_dim,
                                    interleaved, positions, T, Hq, Hkv, D, eps);
  return st != LOOM_OK ? st : norm_rope_cache_call(a, slots, q, k_cache, v_cache, num_pages, page_size, kv_layout, stream);
}

size_t loom_qkv_norm_rope_bwd_workspace_bytes(int D) { return D == 64 || D == 128 ? qkv_bwd_workspace_bytes(D) : 0; }

loom_status loom_qkv_norm_rope_bwd(const void* dq, const void* dk, const void* dv, const void* qkv, int64_t qkv_stride,
                                   const void* q_weight, const void* k_weight, int weight_type, const float* cos,
                                   const float* sin, int table_rows, int rotary_dim, int interleaved,
                                   const int32_t* positions, void* dqkv, int64_t dqkv_stride, float* dq_weight,
                                   float* dk_weight, void* workspace, size_t workspace_bytes, int T, int seq_len,
                                   int Hq, int Hkv, int D, float eps, void* stream) {
  QkvArgs a{};
  const loom_status st = qkv_common(&a, qkv, qkv_stride, q_weight, k_weight, weight_type, cos, sin, table_rows, rotary_dim,
                                    interleaved, positions, T, Hq, Hkv, D, eps);
  return st != LOOM_OK ? st
                       : norm_rope_bwd_call(a, dq, dk, dv, dqkv, dqkv_stride, dq_weight, dk_weight, workspace, workspace_bytes,
                                            seq_len, stream);
}

loom_status loom_qkv_norm_rope_axes(const void* qkv, int64_t qkv_stride, const void* q_weight, const void* k_weight,
                                    int weight_type, const float* cos, const float* sin, int table_rows,
                                    int rotary_dim, int interleaved, const int32_t* positions,
                                    int64_t positions_stride, int n_axes, const int* pair_axis, void* q, void* k,
                                    void* v, int T, int seq_len, int Hq, int Hkv, int D, float eps, void* stream) {
  QkvArgs a{};
  loom_status st = qkv_common(&a, qkv, qkv_stride, q_weight, k_weight, weight_type, cos, sin, table_rows, rotary_dim,
                              interleaved, positions, T, Hq, Hkv, D, eps);
  if (st == LOOM_OK) st = axes_args(&a, positions_stride, n_axes, pair_axis);
  return st != LOOM_OK ? st : norm_rope_call(a, q, k, v, seq_len, stream);
}

loom_status loom_qkv_norm_rope_axes_cache(const void* qkv, int64_t qkv_stride, const void* q_weight,
                                          const void* k_weight, int weight_type, const float* cos, const float* sin,
                                          int table_rows, int rotary_dim, int interleaved, const int32_t* positions,
                                          int64_t positions_stride, int n_axes, const int* pair_axis,
                                          const int32_t* slots, void* q, void* k_cache, void* v_cache, int num_pages,
                                          int page_size, int kv_layout, int T, int Hq, int Hkv, int D, float eps,
                                          void* stream) {
  QkvArgs a{};
  loom_status st = qkv_common(&a, qkv, qkv_stride, q_weight, k_weight, weight_type, cos, sin, table_rows, rotary_dim,
                              interleaved, positions, T, Hq, Hkv, D, eps);
  if (st == LOOM_OK) st = axes_args(&a, positions_stride, n_axes, pair_axis);
  return st != LOOM_OK ? st : norm_rope_cache_call(a, slots, q, k_cache, v_cache, num_pages, page_size, kv_layout, stream);
}

loom_status loom_qkv_norm_rope_axes_bwd(const void* dq, const void* dk, const void* dv, const void* qkv,
                                        int64_t qkv_stride, const void* q_weight, const void* k_weight,
                                        int weight_type, const float* cos, const float* sin, int table_rows,
                                        int rotary_dim, int interleaved, const int32_t* positions,
                                        int64_t positions_stride, int n_axes, const int* pair_axis, void* dqkv,
                                        int64_t dqkv_stride, float* dq_weight, float* dk_weight, void* workspace,
                                        size_t workspace_bytes, int T, int seq_len, int Hq, int Hkv, int D, float eps,
                                        void* stream) {
  QkvArgs a{};
  loom_status st = qkv_common(&a, qkv, qkv_stride, q_weight, k_weight, weight_type, cos, sin, table_rows, rotary_dim,
                              interleaved, positions, T, Hq, Hkv, D, eps);
  if (st == LOOM_OK) st = axes_args(&a, positions_stride, n_axes, pair_axis);
  return st != LOOM_OK ? st
                       : norm_rope_bwd_call(a, dq, dk, dv, dqkv, dqkv_stride, dq_weight, dk_weight, workspace, workspace_bytes,
                                            seq_len, stream);
}

namespace {
loom_status gemm_call(const void* a, const void* b, void* c, int M, int N, int K, int b_kmajor, void* stream) {
  if (!a || !b || !c) return LOOM_ERR_INVALID_ARG;
  if (M <= 0 || N <= 0 || K <= 0) return LOOM_ERR_INVALID_ARG;
  if (!aligned16(a) || !aligned16(b) || !aligned16(c)) return LOOM_ERR_MISALIGNED;
  if (K % 8 != 0 || N % 8 != 0) return LOOM_ERR_UNSUPPORTED;  // 16-byte row strides for TMA
  KernelCtl ctl;
  if (!make_ctl(&ctl)) return LOOM_ERR_CUDA;
  GemmArgs g{a, b, c, M, N, K, g_gemm_tile_n, g_gemm_splits, g_gemm_pair, b_kmajor, g_gemm_stages, g_gemm_group, g_gemm_k_alt};
  return launch_gemm(g, ctl, static_cast<cudaStream_t>(stream)) == cudaSuccess ? LOOM_OK : LOOM_ERR_CUDA;
}
}  // namespace

loom_status loom_gemm_bf16(const void* a, const void* b, void* c, int M, int N, int K, void* stream) {
  return gemm_call(a, b, c, M, N, K, 0, stream);
}

loom_status loom_gemm_bf16_bt(const void* a, const void* b, void* c, int M, int N, int K, void* stream) {
  return gemm_call(a, b, c, M, N, K, 1, stream);
}

namespace {
// The model's GEMM choice: with the device's cluster occupancy when a device answers, else
// with the estimate of whole clusters in 8 equal SM groups of a GB300.
GemmChoice gemm_choice_any(int M, int N, int K, GemmChoice forced) {
  const GemmChoice c = gemm_choice(M, N, K, forced);
  if (c.tile_n != 0) return c;
  cudaGetLastError();
  const int sms = model::kGb300.num_sms;
  const model::GemmChoiceModel m = model::gemm_choose(
      M, N, K, sms, [sms](int, int S) { return model::gemm_default_slots(sms, S); }, model::kGb300,
      forced.tile_n, forced.splits, forced.pair >= 0 ? model::gemm_default_slots(sms, 2) : 0, forced.pair);
  return {m.bn, m.splits, m.pair ? 1 : 0};
}
}  // namespace

int loom_gemm_tile_n(int M, int N, int K) {
  if (M <= 0 || N <= 0 || K <= 0) return 0;
  return gemm_choice_any(M, N, K, {g_gemm_tile_n, g_gemm_splits, g_gemm_pair}).tile_n;
}

int loom_gemm_splits(int M, int N, int K) {
  if (M <= 0 || N <= 0 || K <= 0) return 0;
  return gemm_choice_any(M, N, K, {g_gemm_tile_n, g_gemm_splits, g_gemm_pair}).splits;
}

int loom_gemm_cta_pair(int M, int N, int K) {
  if (M <= 0 || N <= 0 || K <= 0) return 0;
  return gemm_choice_any(M, N, K, {g_gemm_tile_n, g_gemm_splits, g_gemm_pair}).pair;
}

double loom_model_gemm_time_us(int M, int N, int K, int tile_n, int splits, int num_sms) {
  if (M <= 0 || N <= 0 || K <= 0 || num_sms <= 0) return -1.0;
  if (tile_n == 512 && splits == 1)  // CTA-pair 256 x 256 tiles
    return model::gemm_pair_time_us(M, N, K, model::gemm_default_slots(num_sms, 2));
  if (tile_n != 64 && tile_n != 128 && tile_n != 192 && tile_n != 256) return -1.0;
  if (!model::gemm_split_supported(splits)) return -1.0;
  const model::GemmPlan p = model::gemm_plan_variant(tile_n);
  if (!p.feasible) return -1.0;
  if (splits == 1) return model::gemm_time_us(p, M, N, K, num_sms);
  return model::gemm_splitk_time_us(p, M, N, K, splits, model::gemm_default_slots(num_sms, splits));
}

void loom_debug_gemm_tile_n(int tile_n) {
  g_gemm_tile_n = (tile_n == 64 || tile_n == 128 || tile_n == 192 || tile_n == 256) ? tile_n : 0;
}

void loom_debug_gemm_splits(int splits) { g_gemm_splits = model::gemm_split_supported(splits) ? splits : 0; }

void loom_debug_gemm_cta_pair(int mode) { g_gemm_pair = (mode == 1 || mode == -1) ? mode : 0; }

void loom_debug_gemm_stages(int stages) { g_gemm_stages = stages > 0 ? stages : 0; }

void loom_debug_decode_tensor_cores(int mode) { g_decode_tc = (mode >= 0 && mode <= 2) ? mode : 1; }

void loom_debug_gemm_order(int group_rows, int k_alternate) {
  g_gemm_group = (group_rows >= 1 && group_rows <= 1024) ? group_rows : 0;
  g_gemm_k_alt = k_alternate < 0 ? -1 : 0;
}

loom_status loom_attn_check_error(void* stream) {
  if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) return LOOM_ERR_CUDA;
  uint32_t* p = error_word_ptr();
  if (!p) return LOOM_ERR_CUDA;
  uint32_t word = 0;
  if (cudaMemcpy(&word, p, sizeof word, cudaMemcpyDeviceToHost) != cudaSuccess) return LOOM_ERR_CUDA;
  if (word) {
    const uint32_t zero = 0;
    if (cudaMemcpy(p, &zero, sizeof zero, cudaMemcpyHostToDevice) != cudaSuccess) return LOOM_ERR_CUDA;
  }
  return (word & kErrTimeout) ? LOOM_ERR_TIMEOUT : LOOM_OK;
}

namespace {
void fill_plan(const model::FwdPlan& p, loom_fwd_plan* out) {
  out->design = p.design;
  out->s_buffers = p.s_buffers;
  out->bm = p.bm;
  out->bn = p.bn;
  out->q_tiles = p.q_tiles;
  out->kv_slots = p.kv_slots;
  out->b_lm = p.b_lm;
  out->b_ms = p.b_ms;
  out->smem_bytes = p.smem_bytes;
  out->tmem_cols = p.tmem_cols;
  out->t_load_ns = p.t_load_ns;
  out->t_mma_ns = p.t_mma_ns;
  out->t_softmax_ns = p.t_softmax_ns;
  out->t_iter_ns = p.t_iter_ns;
}
}  // namespace

loom_status loom_model_fwd_plan(int D, loom_fwd_plan* out) {
  if (!out) return LOOM_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return LOOM_ERR_UNSUPPORTED;
  fill_plan(model::fwd_plan(D), out);
  return LOOM_OK;
}

loom_status loom_model_fwd_plan_variant(int D, int design, loom_fwd_plan* out) {
  if (!out) return LOOM_ERR_INVALID_ARG;
  if ((D != 64 && D != 128) || design < 1 || design > 4) return LOOM_ERR_UNSUPPORTED;
  const model::FwdPlan p = model::fwd_plan_variant(D, design);
  if (!p.feasible) return LOOM_ERR_UNSUPPORTED;
  fill_plan(p, out);
  return LOOM_OK;
}

double loom_model_heg_pipe(double l, double m, double s, int b_lm, int b_ms) {
  return model::heg_pipe(l, m, s, b_lm != 0, b_ms != 0);
}

double loom_model_fwd_time_us(int B, int Hq, int Sq, int Skv, int D, int causal) {
  if (B <= 0 || Hq <= 0 || Sq <= 0 || Skv <= 0 || (D != 64 && D != 128)) return -1.0;
  return model::fwd_time_us(model::fwd_plan(D), B, Hq, Sq, Skv, D, causal != 0);
}

double loom_model_fwd_time_us_design(int design, int B, int Hq, int Sq, int Skv, int D, int causal) {
  if (B <= 0 || Hq <= 0 || Sq <= 0 || Skv <= 0 || (D != 64 && D != 128) || design < 1 || design > 4) return -1.0;
  const model::FwdPlan p = model::fwd_plan_variant(D, design);
  if (!p.feasible) return -1.0;
  return model::fwd_time_us(p, B, Hq, Sq, Skv, D, causal != 0);
}

double loom_model_decode_time_us(int splits, int B, int Hq, int Hkv, int Skv, int D, int num_sms) {
  if (splits <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || Skv <= 0 || num_sms <= 0 ||
      (D != 64 && D != 128))
    return -1.0;
  return model::decode_time_us(splits, B, Hq, Hkv, Skv, D, num_sms);
}

double loom_model_decode_tc_time_us(int splits, int B, int Hq, int Hkv, int Skv, int D, int num_sms) {
  if (splits <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || Skv <= 0 || num_sms <= 0 ||
      (D != 64 && D != 128) || Hq / Hkv > kDecodeTcMaxGroup)
    return -1.0;
  return model::decode_tc_time_us(splits, B, Hq, Hkv, Skv, D, num_sms);
}

int loom_attn_decode_form(int B, int Hq, int Hkv, int Skv, int D, int num_splits, int paged, int* cluster) {
  if (cluster) *cluster = 0;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Skv <= 0 || Hq % Hkv != 0 || (D != 64 && D != 128) || num_splits < 0 ||
      num_splits > kMaxDecodeSplits)
    return -1;
  const int by_model = num_splits == 0 ? 1 : 0;
  if (num_splits == 0) num_splits = loom_attn_decode_num_splits(B, Hq, Hkv, Skv, D);
  if (num_splits <= 0) return -1;
  DecodeArgs a{};
  a.by_model = by_model;
  a.B = B;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.Skv = Skv;
  a.D = D;
  a.splits = num_splits;
  a.form = g_decode_form;
  a.cluster = g_decode_cluster;
  a.tc = g_decode_tc;
  int cs = 0;
  const int form = decode_form_of(a, paged != 0, &cs);
  cudaGetLastError();
  if (cluster) *cluster = cs;
  return form;
}

double loom_model_decode_cluster_time_us(int splits, int cluster, int B, int Hq, int Hkv, int Skv, int D,
                                         int clusters) {
  if (splits <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || Skv <= 0 || clusters <= 0 ||
      (D != 64 && D != 128))
    return -1.0;
  const double t = model::decode_cluster_time_us(splits, cluster, B, Hq, Hkv, Skv, D, clusters);
  return t > 1e299 ? -1.0 : t;
}

double loom_model_decode_persistent_time_us(int splits, int B, int Hq, int Hkv, int Skv, int D, int ctas) {
  if (splits <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || Skv <= 0 || ctas <= 0 || (D != 64 && D != 128))
    return -1.0;
  return model::decode_persistent_time_us(splits, B, Hq, Hkv, Skv, D, ctas);
}

int loom_decode_max_clusters(int D, int G, int cluster) {
  if ((D != 64 && D != 128) || G <= 0 || cluster <= 0 || cluster > model::kMaxClusterSize) return 0;
  const int sms = current_sm_count();
  if (sms <= 0) return model::decode_default_clusters(model::kGb300.num_sms, cluster, D);
  const int n = decode_max_clusters(D, G, cluster);
  cudaGetLastError();
  return n;
}

int loom_decode_persistent_slots(int D, int G) {
  if ((D != 64 && D != 128) || G <= 0) return 0;
  const int sms = current_sm_count();
  if (sms <= 0) return model::kGb300.num_sms * model::decode_stage(D).ctas_per_sm;
  const int n = decode_persistent_slots(D, G);
  cudaGetLastError();
  return n;
}

void loom_debug_decode_form(int form, int cluster) {
  g_decode_form = (form == kDecodeSplitMerge || form == kDecodePersistent || form == kDecodeCluster) ? form : 0;
  g_decode_cluster = (cluster >= 1 && cluster <= model::kMaxClusterSize) ? cluster : 0;
}

int loom_debug_decode_stage_plan(int tokens, int stages, int ctas_per_sm) {
  const model::DecodeStagePlan& m = model::decode_stage(128);
  if (tokens == 0 || (tokens == m.tokens && stages == m.stages && ctas_per_sm == m.ctas_per_sm)) {
    g_decode_stage_plan = 0;
    return 1;
  }
  g_decode_stage_plan = decode_ablation_plan(tokens, stages, ctas_per_sm);
  return g_decode_stage_plan > 0 ? 1 : 0;
}

void loom_debug_set_timeout_ns(uint64_t ns) { g_timeout_ns = ns ? ns : kDefaultTimeoutNs; }

void loom_debug_inject(int mode) { g_inject = mode; }

void loom_debug_prefill_design(int design) {
  g_prefill_design = (design >= 1 && design <= 4) ? design : 0;
}

int loom_debug_prefill_slots(int D, int slots) {
  if (slots == 0 || (D == 128 && slots == model::fwd_plan_variant(128, 2).kv_slots) ||
      (D == 64 && slots == model::fwd_plan_variant(64, 2).kv_slots) || fwd_slots_compiled(D, slots)) {
    g_prefill_slots = slots;
    return 1;
  }
  g_prefill_slots = 0;
  return 0;
}

}  // extern "C"
