// The pages of a pool between requests: reference counts, tables and the copies that sharing and packing
// need. Everything is decided on the device (tables and counts live there and no call waits for the host):
//
//   page_plan   one cluster of eight CTAs: checks the call's tables against the counts, and only if all is well
//               ranks the free (or live) pages by prefix sums over the counts, writes the new tables and counts
//               and lists the page copies. Warp w of the cluster owns the w-th run of pages; ranks are the
//               counts of the runs before it plus ballots within it, so equal inputs give equal ids whatever
//               the schedule. Atomics only add integers.
//   page_copy   the listed pages of every layer, K and V (a page of a layer is contiguous).
//
// The plan is bound by latency (five or six passes over small arrays, a cluster barrier between them), the
// copies by memory: each copied byte is read once and written once.
#include "common.cuh"
#include "extend.h"

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

constexpr int kPlanCtas = 8;  // the largest portable cluster
constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kCopyThreads = 256;
constexpr int kMaxCopyLayers = 64;  // of one copy launch

// In the caller's workspace.
struct PageScratch {
  int* abort;   // [0]: the call is rejected, [1]: copies listed
  int* src;     // [copies] page copied from, to, and its live slots
  int* dst;
  int* live;
  int* fresh;   // fork: the new pages in order
  int* mark;    // [pages] entries of a page; compact, then: a moving page's number
};

struct PlanArgs {
  PageTables t;
  PageScratch s;
  const int32_t* refs_in;
  int32_t* refs_out;
  int fresh;   // fork: new pages of the call
  bool deep;
  int* status;
};

__device__ __forceinline__ int table_of_entry(const PageTables& t, int e) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= e) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Sums over the CTAs of the cluster, exchanged through shared memory.
struct Exchange {
  int total[kPlanCtas];  // written by every CTA into every CTA
  int bad[kPlanCtas];
  int warp_sum[kPlanWarps];
  int warp_before[kPlanWarps];
};
__device__ __forceinline__ void st_cluster_s32(const void* p, uint32_t rank, int v) {
  asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(mapa_shared(p, rank)), "r"(v) : "memory");
}

// All threads: `count` (lane 0 of each warp) summed over the cluster, with the sum of the warps before the
// caller's in *before; `bad` (any thread) ORed. Ends in a cluster barrier.
__device__ __forceinline__ int cluster_count(Exchange& x, int count, int bad, int* before, int* any_bad) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int block_bad = __syncthreads_or(bad);
  if (lane == 0) x.warp_sum[warp] = count;
  __syncthreads();
  if (warp == 0) {
    const int v = x.warp_sum[lane];
    int s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += u;
    }
    x.warp_before[lane] = s - v;
    const int total = __shfl_sync(0xffffffffu, s, 31);
    const int me = static_cast<int>(cluster_ctarank());
    if (lane < kPlanCtas) {
      st_cluster_s32(&x.total[me], lane, total);
      st_cluster_s32(&x.bad[me], lane, block_bad);
    }
  }
  __syncthreads();
  cluster_sync();
  int sum = 0, mine = 0, b = 0;
  const int me = static_cast<int>(cluster_ctarank());
#pragma unroll
  for (int i = 0; i < kPlanCtas; ++i) {
    if (i == me) mine = sum;
    sum += x.total[i];
    b |= x.bad[i];
  }
  *before = mine + x.warp_before[warp];
  *any_bad = b;
  return sum;
}

template <PageOp OP>
__global__ void __cluster_dims__(kPlanCtas, 1, 1) __launch_bounds__(kPlanThreads, 1)
    page_plan(const __grid_constant__ PlanArgs a) {
  static_assert(kPlanWarps == 32, "cluster_count scans one warp's worth of warps");
  __shared__ Exchange xa, xb;
  griddep_launch_dependents();
  const PageTables& t = a.t;
  const int P = t.num_pages, entries = t.first[t.n];
  const int lane = threadIdx.x & 31;
  const int me = static_cast<int>(cluster_ctarank());
  const int warp = me * kPlanWarps + (threadIdx.x >> 5);
  const int thread = me * kPlanThreads + threadIdx.x, threads = kPlanCtas * kPlanThreads;
  // this warp's pages [p0, p1)
  const int run = ((P + kPlanCtas * kPlanWarps - 1) / (kPlanCtas * kPlanWarps) + 31) & ~31;
  const int p0 = static_cast<int>(min(static_cast<int64_t>(P), static_cast<int64_t>(warp) * run));
  const int p1 = min(P, p0 + run);
  int bad = 0;

  // Entries of every page (release, compact); their ids are checked here, and a fork's counts too
  if (OP != kPageFork)
    for (int p = p0 + lane; p < p1; p += 32) a.s.mark[p] = 0;
  cluster_sync();  // and every CTA of the cluster runs, before its shared memory is written to
  for (int e = thread; e < entries; e += threads) {
    const int f = table_of_entry(t, e);
    const int id = t.table[f][e - t.first[f]];
    if (id < 0 || id >= P)
      bad = 1;
    else if (OP == kPageFork)
      bad |= a.refs_in[id] < 1;
    else
      atomicAdd(&a.s.mark[id], 1);
  }
  // fork: free pages; compact: live pages
  int count = 0;
  for (int p = p0 + lane; p - lane < p1; p += 32) {
    const int r = p < p1 ? a.refs_in[p] : 0;
    bad |= r < 0;
    const bool mine = p < p1 && (OP == kPageFork ? r == 0 : r > 0);
    count += __popc(__ballot_sync(0xffffffffu, mine));
  }
  int before, any_bad;
  const int total = cluster_count(xa, count, bad, &before, &any_bad);
  bool full = false;
  int below = 0;  // compact: live pages below `total`, those that stay
  if (OP == kPageFork) {
    full = total < a.fresh;
  } else {
    // every entry is counted now
    bad = 0;
    int stay = 0;
    for (int p = p0 + lane; p - lane < p1; p += 32) {
      const int r = p < p1 ? a.refs_in[p] : 0, m = p < p1 ? __ldcg(&a.s.mark[p]) : 0;
      bad |= OP == kPageCompact ? m != r : m > r;
      stay += __popc(__ballot_sync(0xffffffffu, r > 0 && p < total));
    }
    int unused, again;
    below = cluster_count(xb, stay, bad, &unused, &again);
    any_bad |= again;
  }
  if (any_bad || full) {
    if (thread == 0) {
      a.s.abort[0] = 1;
      a.s.abort[1] = 0;
      if (a.status) atomicOr(a.status, any_bad ? kStatusCounts : kStatusFull);
    }
    return;
  }
  const int copies = OP == kPageFork ? a.fresh : OP == kPageCompact ? total - below : 0;
  if (thread == 0) {
    a.s.abort[0] = 0;
    a.s.abort[1] = copies;
  }

  if (OP == kPageRelease) {
    for (int p = p0 + lane; p < p1; p += 32) a.refs_out[p] = a.refs_in[p] - __ldcg(&a.s.mark[p]);
    return;
  }

  if (OP == kPageFork) {
    for (int p = p0 + lane; p - lane < p1; p += 32) {
      const int r = p < p1 ? a.refs_in[p] : 1;
      const uint32_t free = __ballot_sync(0xffffffffu, r == 0);
      const int rank = before + __popc(free & ((1u << lane) - 1));
      const bool taken = r == 0 && rank < a.fresh;
      if (taken) a.s.fresh[rank] = p;
      if (p < p1) a.refs_out[p] = taken ? 1 : r;
      before += __popc(free);
    }
    cluster_sync();
    for (int e = thread; e < entries; e += threads) {
      const int f = table_of_entry(t, e), i = e - t.first[f];
      const int id = t.table[f][i], live = min(kPage, t.n_tokens[f] - i * kPage);
      int child = id;
      if (a.deep || live < kPage) {
        const int k = t.fresh0[f] + (a.deep ? i : 0);
        child = __ldcg(&a.s.fresh[k]);
        a.s.src[k] = id;
        a.s.dst[k] = child;
        a.s.live[k] = live;
      } else {
        atomicAdd(&a.refs_out[id], 1);
      }
      t.out[f][i] = child;
    }
    return;
  }

  // compact: `total` live pages stay in or move into [0, total); page p's number among the movers or holes
  for (int p = p0 + lane; p - lane < p1; p += 32) {
    const int r = p < p1 ? a.refs_in[p] : 0;
    const uint32_t live = __ballot_sync(0xffffffffu, r > 0);
    const int rank = before + __popc(live & ((1u << lane) - 1));  // live pages below p
    if (p < p1) {
      if (p >= total && r > 0) {
        a.s.src[rank - below] = p;
        a.s.mark[p] = rank - below;
      } else if (p < total && r == 0) {
        a.s.dst[p - rank] = p;
        a.s.live[p - rank] = kPage;
      }
    }
    before += __popc(live);
  }
  cluster_sync();
  for (int k = thread; k < copies; k += threads) a.refs_out[__ldcg(&a.s.dst[k])] = a.refs_in[__ldcg(&a.s.src[k])];
  if (a.refs_out != a.refs_in)
    for (int p = p0 + lane; p < min(p1, total); p += 32)
      if (a.refs_in[p] > 0) a.refs_out[p] = a.refs_in[p];
  for (int e = thread; e < entries; e += threads) {
    const int f = table_of_entry(t, e), i = e - t.first[f];
    const int id = t.table[f][i];
    t.out[f][i] = id < total ? id : __ldcg(&a.s.dst[__ldcg(&a.s.mark[id])]);
  }
  cluster_sync();  // in place, the movers' counts are read above
  for (int p = max(p0, total) + lane; p < p1; p += 32) a.refs_out[p] = 0;
}

struct CopyArgs {
  PageScratch s;
  __nv_bfloat16* pool[2 * kMaxCopyLayers];  // K of the layers, then V
  int pools;
  int n_kv_heads, head_dim;
};

__global__ void __launch_bounds__(kCopyThreads) page_copy(const __grid_constant__ CopyArgs a) {
  griddep_wait();
  if (a.s.abort[0]) return;
  const int64_t units = static_cast<int64_t>(a.s.abort[1]) * a.pools;
  const int head_vecs = kPage * a.head_dim / 8, page_vecs = a.n_kv_heads * head_vecs;  // 16 bytes each
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int k = static_cast<int>(u / a.pools), pool = static_cast<int>(u - static_cast<int64_t>(k) * a.pools);
    const int live_vecs = a.s.live[k] * a.head_dim / 8;
    const uint4* src = reinterpret_cast<const uint4*>(a.pool[pool]) + static_cast<int64_t>(a.s.src[k]) * page_vecs;
    uint4* dst = reinterpret_cast<uint4*>(a.pool[pool]) + static_cast<int64_t>(a.s.dst[k]) * page_vecs;
    constexpr int kBatch = 4;
    for (int i = threadIdx.x; i < page_vecs; i += kBatch * kCopyThreads) {
      uint4 v[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int j = i + b * kCopyThreads;
        if (j < page_vecs && j % head_vecs < live_vecs) v[b] = __ldcs(src + j);
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int j = i + b * kCopyThreads;
        if (j < page_vecs && j % head_vecs < live_vecs) __stcs(dst + j, v[b]);
      }
    }
  }
}

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

PageScratch scratch_of(void* workspace, int num_pages, int entries, size_t* bytes) {
  uint8_t* w = static_cast<uint8_t*>(workspace);
  size_t o = 256;
  auto take = [&](size_t n) {
    int* at = reinterpret_cast<int*>(w + o);
    o = align256(o + n * sizeof(int));
    return at;
  };
  PageScratch s;
  s.abort = reinterpret_cast<int*>(w);
  // a fork lists one copy an entry at most, a compaction one a page
  const size_t copies = static_cast<size_t>(std::max(num_pages, entries));
  s.src = take(copies);
  s.dst = take(copies);
  s.live = take(copies);
  s.fresh = take(copies);
  s.mark = take(num_pages);
  *bytes = o;
  return s;
}

int copy_launches(int n_layers) { return (n_layers + kMaxCopyLayers - 1) / kMaxCopyLayers; }

}  // namespace

size_t page_workspace(int num_pages, int entries) {
  size_t bytes;
  scratch_of(nullptr, num_pages, entries, &bytes);
  return bytes;
}

int page_launches(PageOp op, const PageTables& t, int n_layers) {
  if (op == kPageRelease || (op == kPageFork && t.fresh0[t.n] == 0)) return 1;
  return 1 + copy_launches(n_layers);
}

cudaError_t launch_pages(PageOp op, const PageTables& t, bool deep, const int32_t* refs_in, int32_t* refs_out,
                         const PagePool* pool, void* workspace, int num_sms, int* status, cudaStream_t stream) {
  PlanArgs a;
  std::memset(&a, 0, sizeof(a));
  a.t = t;
  size_t bytes;
  a.s = scratch_of(workspace, t.num_pages, t.first[t.n], &bytes);
  a.refs_in = refs_in;
  a.refs_out = refs_out;
  a.fresh = op == kPageFork ? t.fresh0[t.n] : 0;
  a.deep = deep;
  a.status = status;
  auto* plan = op == kPageFork ? page_plan<kPageFork> : op == kPageCompact ? page_plan<kPageCompact> : page_plan<kPageRelease>;
  cudaError_t e = launch_kernel(plan, dim3(kPlanCtas), dim3(kPlanThreads), 0, stream, a);
  if (e != cudaSuccess || op == kPageRelease || (op == kPageFork && a.fresh == 0)) return e;
  PdlScope pdl;
  for (int l0 = 0; l0 < pool->n_layers; l0 += kMaxCopyLayers) {
    CopyArgs c;
    std::memset(&c, 0, sizeof(c));
    c.s = a.s;
    const int n = std::min(kMaxCopyLayers, pool->n_layers - l0);
    for (int l = 0; l < n; ++l) {
      c.pool[l] = static_cast<__nv_bfloat16*>(pool->k[l0 + l]);
      c.pool[n + l] = static_cast<__nv_bfloat16*>(pool->v[l0 + l]);
    }
    c.pools = 2 * n;
    c.n_kv_heads = pool->n_kv_heads;
    c.head_dim = pool->head_dim;
    int64_t units = static_cast<int64_t>(num_sms) * 8;
    if (op == kPageFork) units = std::min(units, static_cast<int64_t>(a.fresh) * c.pools);
    e = launch_kernel(page_copy, dim3(static_cast<unsigned>(units)), dim3(kCopyThreads), 0, stream, c);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace crf
