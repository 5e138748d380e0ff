// The bookkeeping of a serving step over a paged cache: offsets, positions, slots and new pages from
// the requests' lengths.
//
// With n_b new tokens, len_b cached ones and pages of s rows:
//     cu_b     = sum_{a<b} max(n_a, 0)
//     need_b   = ceil((len_b + n_b) / s) - ceil(len_b / s)      (0 where the row or the step has no room)
//     off_b    = sum_{a<b} need_a;   granted where need_b = 0 or off_b + need_b <= pages that are free
// The demands granted are a prefix of all demands, so one prefix sum decides them: page k of the step is
// the k-th from the end of the free list, request b's are off_b .. off_b + need_b - 1.
//
// What bounds it is a launch and the chain of latencies after it: lengths, prefix sums, the table's
// entry, the stores.  So it is one launch of one cluster whose blocks all compute the prefix sums for
// themselves (in shared memory) and share the tokens and pages; the one cluster barrier lies between the
// last read of the lengths and the free count and the first write, so that those may be updated in place.
#include <atomic>

#include "kernels.h"
#include "paged.h"
#include "ptx.cuh"

namespace loom {
namespace {

// Blocks of the cluster: 16 where the device has room for one of them, else 8 (which any has).  (4096 requests with 68648
// tokens, 256 with 22883: 4 blocks 31.2 and 13.5 us, 8 21.6 and 10.3, 16 17.2 and 9.3.)
constexpr int kThreads = 1024, kClusterBlocks = 16, kPortableBlocks = 8;
// Requests and tokens that one block deals with alone: it needs no 16 SMs of one GPC free at the same time.  On a device with
// nothing else to do a cluster is sooner all the same (alone and in a cluster: 4 requests with 4 tokens 5.0 and 4.8 us, 64
// with 64 6.2 and 5.8, 256 with 256 6.4 and 6.2, 512 with 1866 8.3 and 7.0, 1000 with 1450 8.6 and 7.6), and past these bounds
// by more (64 with 2846 8.0 and 6.1, 2000 with 2000 10.0 and 8.5, 4096 with 4096 13.6 and 9.6).
constexpr int kAloneTokens = 2048, kAloneRequests = 1024;

// Exclusive prefix sums of a and b over the block, and their totals.
struct Sums {
  long long a, b, all_a, all_b;
};
__device__ __forceinline__ Sums scan(long long a, long long b, long long (*part)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = a, y = b;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, x, d), v = __shfl_up_sync(0xffffffffu, y, d);
    if (lane >= d) x += u, y += v;
  }
  __syncthreads();  // the last call's sums have been read
  if (lane == 31) part[warp][0] = x, part[warp][1] = y;
  __syncthreads();
  long long p = part[lane][0], q = part[lane][1];
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, p, d), v = __shfl_up_sync(0xffffffffu, q, d);
    if (lane >= d) p += u, q += v;
  }
  const long long before_p = __shfl_sync(0xffffffffu, p, (warp + 31) & 31), before_q = __shfl_sync(0xffffffffu, q, (warp + 31) & 31);
  return {(warp ? before_p : 0) + x - a, (warp ? before_q : 0) + y - b, __shfl_sync(0xffffffffu, p, 31),
          __shfl_sync(0xffffffffu, q, 31)};
}

// Rows in pages, in 32 bits (rows and page - 1 are below 2^31), by a shift where it does: divisions of 64 bits took
// most of the kernel's instructions, and of 32 a third (4096 requests with 68648 tokens 18.9 us, so 17.2).
struct Pages {
  unsigned page;
  int lg;  // of a power of two; else -1
  __device__ __forceinline__ int whole(unsigned rows) const { return static_cast<int>(lg >= 0 ? rows >> lg : rows / page); }
  __device__ __forceinline__ int of(int rows) const { return whole(static_cast<unsigned>(rows) + page - 1u); }
};

// The largest b with at[b] <= x, of n + 1 values that never decrease, at[0] <= x < at[n].
__device__ __forceinline__ int holder(const int* at, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (at[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

enum : uint8_t { kGranted = 1, kOver = 2 };

__global__ void __launch_bounds__(kThreads) paged_plan_kernel(const PlanArgs p) {
  extern __shared__ int plan_smem[];
  __shared__ long long part[32][2];
  const int B = p.B;
  const Pages pages{static_cast<unsigned>(p.page), (p.page & (p.page - 1)) ? -1 : 31 - __clz(p.page)};
  int* cu = plan_smem;        // [B + 1] first token, p.T at most
  int* off = cu + B + 1;      // [B + 1] pages that the requests before ask for (one more than there are, at most)
  int* rel = off + B + 1;     // [B + 1] pages that the requests before give back, as many as there are at most
  int* len = rel + B + 1;     // [B] cached tokens
  uint8_t* state = reinterpret_cast<uint8_t*>(len + B);
  const int blocks = static_cast<int>(cluster_nctarank()), rank = static_cast<int>(cluster_ctarank());
  const int first = rank * kThreads + static_cast<int>(threadIdx.x), step = blocks * kThreads;
  const long long rows = static_cast<long long>(p.max_pages) * p.page;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");

  const int listed = min(max(*p.free_count, 0), p.num_pages);
  for (int b = threadIdx.x; b < B; b += kThreads) {
    cu[b] = p.new_lens[b];
    len[b] = static_cast<int>(min(max(static_cast<long long>(p.lens[b]), 0ll), rows));
  }
  __syncthreads();
  // A thread has a few requests in a row, so that two scans of the block do for any number of them (a scan for every
  // 1024 took 3 us each: 8192 requests 29.1 us for 16.8).
  // An odd number, so that the threads of a warp meet in no bank.
  const int each = (B + kThreads - 1) / kThreads | 1, b0 = min(B, each * static_cast<int>(threadIdx.x)), b1 = min(B, b0 + each);
  long long n_sum = 0, rel_sum = 0;
  for (int b = b0; b < b1; ++b) {
    n_sum += max(cu[b], 0);
    rel_sum += cu[b] < 0 ? pages.of(len[b]) : 0;
  }
  const Sums s = scan(n_sum, rel_sum, part);
  const long long given = s.all_b;
  // (0 where the row or the step has no room; off holds it until the sums are known)
  long long end = s.a, back = s.b, need_sum = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = cu[b], l = len[b];
    const long long begin = end;
    end += max(n, 0);
    const bool fits = n >= 0 && l + static_cast<long long>(n) <= rows && end <= p.T;
    const int need = fits && n > 0 ? pages.of(l + n) - pages.of(l) : 0;
    off[b] = need;
    need_sum += need;
    cu[b] = static_cast<int>(min(begin, static_cast<long long>(p.T)));
    rel[b] = static_cast<int>(min(back, static_cast<long long>(p.num_pages)));
    if (n < 0) back += pages.of(l);
    state[b] = n < 0 ? kOver : fits ? kGranted : 0;
  }
  const Sums t = scan(need_sum, 0, part);
  long long asked = t.a;
  for (int b = b0; b < b1; ++b) {
    const int need = off[b];
    off[b] = static_cast<int>(min(asked, static_cast<long long>(p.num_pages) + 1));
    asked += need;
    // (past all pages there are: the sorted offsets do not tell these apart)
    if (need && asked > p.num_pages) state[b] = 0;
  }
  if (threadIdx.x == 0) {
    cu[B] = static_cast<int>(min(s.all_a, static_cast<long long>(p.T)));
    rel[B] = static_cast<int>(min(given, static_cast<long long>(p.num_pages)));
    off[B] = static_cast<int>(min(t.all_a, static_cast<long long>(p.num_pages) + 1));
  }
  __syncthreads();
  const int total = static_cast<int>(min(listed + given, static_cast<long long>(p.num_pages)));
  // Where the demands pass the total: off is sorted, and every demand before the first that does is met.
  int taken = off[B];
  if (taken > total) taken = off[holder(off, B, total)];
  cluster_sync_all();  // every block has read what may be updated in place

  // entry i of the free list with the pages given back at its end
  const auto listed_page = [&](int i) {
    if (i < listed) return p.free_pages[i];
    const int b = holder(rel, B, i - listed);
    return p.block_table[static_cast<size_t>(b) * p.max_pages + (i - listed - rel[b])];
  };
  const auto fresh_page = [&](int k) { return listed_page(total - 1 - k); };
  const auto is_granted = [&](int b) { return state[b] == kGranted && (off[b + 1] == off[b] || off[b + 1] <= total); };

  for (int b = first; b < B; b += step) {
    const bool g = is_granted(b);
    const int n = cu[b + 1] - cu[b];
    p.cu[b] = cu[b];
    p.seqlens[b] = state[b] == kOver ? 0 : len[b] + (g ? n : 0);
    p.granted[b] = g ? n : 0;
  }
  if (first == 0) {
    p.cu[B] = cu[B];
    *p.free_count_out = total - taken;
  }
  for (int k = first; k < taken; k += step) {
    const int b = holder(off, B, k);
    p.block_table[static_cast<size_t>(b) * p.max_pages + pages.of(len[b]) + (k - off[b])] = fresh_page(k);
  }
  for (int i = listed + first; i < total - taken; i += step) p.free_pages[i] = listed_page(i);
  // A warp takes as many tokens in a row as it has to, looks for its first and last one's request among all, and
  // for the others between those (for each among all: 4096 requests of 15 tokens 18.3 us, here 16.6).
  const int lane = static_cast<int>(threadIdx.x & 31), warps = step / 32;
  const int mine = static_cast<int>(((static_cast<unsigned>(p.T) + warps - 1) / warps + 31) / 32 * 32);
  const long long t0 = static_cast<long long>(first / 32) * mine;
  if (t0 >= p.T) return;
  const int end_t = static_cast<int>(min(t0 + mine, static_cast<long long>(p.T))), real = min(end_t, cu[B]);  // (past real: padding)
  int low = 0, high = 0;
  if (t0 < real) low = holder(cu, B, static_cast<int>(t0)), high = holder(cu, B, real - 1);
#pragma unroll 4
  for (int i = 0; i < mine; i += 32) {
    const long long t = t0 + i + lane;
    if (t >= end_t) continue;
    int pos = 0, slot = -1;
    if (t < real) {
      const int b = low + holder(cu + low, high + 1 - low, static_cast<int>(t));
      if (is_granted(b)) {
        pos = len[b] + (static_cast<int>(t) - cu[b]);
        const int j = pages.whole(static_cast<unsigned>(pos)), held = pages.of(len[b]);
        const int at = j < held ? p.block_table[static_cast<size_t>(b) * p.max_pages + j] : fresh_page(off[b] + j - held);
        if (at >= 0 && at < p.num_pages) slot = at * p.page + (pos - j * p.page);
      }
    }
    p.positions[t] = pos;
    p.slots[t] = slot;
  }
}

constexpr size_t plan_smem_bytes(int B) { return (4 * static_cast<size_t>(B) + 3) * sizeof(int) + B; }
static_assert(plan_smem_bytes(kMaxPlanB) <= 200 * 1024, "prefix sums in shared memory");

// A launch of one cluster of `blocks`; attr has room for two.
cudaLaunchConfig_t plan_config(int blocks, size_t smem, cudaStream_t stream, cudaLaunchAttribute* attr) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(blocks);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cfg;
}

// Blocks of a cluster on the current device, known from its first call on.
int cluster_blocks(int dev) {
  static std::atomic<int> cache[64];
  const bool cached = dev >= 0 && dev < 64;
  if (cached) {
    const int c = cache[dev].load(std::memory_order_relaxed);
    if (c != 0) return c;
  }
  int clusters = 0;
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = plan_config(kClusterBlocks, plan_smem_bytes(kMaxPlanB), nullptr, attr);
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&clusters, paged_plan_kernel, &cfg) != cudaSuccess) {
    cudaGetLastError();
    clusters = 0;
  }
  const int blocks = clusters > 0 ? kClusterBlocks : kPortableBlocks;
  if (cached) cache[dev].store(blocks, std::memory_order_relaxed);
  return blocks;
}

}  // namespace

cudaError_t launch_paged_plan(const PlanArgs& a, cudaStream_t stream) {
  static PerDeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.run(dev, [] {
        return cudaFuncSetAttribute(paged_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, plan_smem_bytes(kMaxPlanB)) ==
                   cudaSuccess &&
               cudaFuncSetAttribute(paged_plan_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
      }))
    return cudaErrorInvalidValue;
  const int blocks = a.T <= kAloneTokens && a.B <= kAloneRequests ? 1 : cluster_blocks(dev);
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = plan_config(blocks, plan_smem_bytes(a.B), stream, attr);
  return cudaLaunchKernelEx(&cfg, paged_plan_kernel, a);
}

}  // namespace loom
