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
// The plan is bound by latency (three to five passes over small arrays, a cluster barrier between them: 7-12 us), the
// copies by memory: each copied byte is read once and written once (1.9 GB of 16 KB pages 283 us, 98% of the copy
// rate; with the plan a private copy of a 16K-token prefix takes 305 us, packing 1.2 GB of 8 KB pages 200).
#include "common.cuh"
#include "extend.h"

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

constexpr int kPlanCtas = 8;  // the largest portable cluster
constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
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

// The tables in shared memory: the parameters come from memory at every launch, and a search through them would wait
// for it at every step.
struct Tables {
  int first[kMaxTables + 1];
  const int32_t* table[kMaxTables];
};
__device__ __forceinline__ int table_of_entry(const Tables& t, int n, int e) {
  int lo = 0, hi = n - 1;
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
  if (lane == 0) x.warp_sum[warp] = count;
  const int block_bad = __syncthreads_or(bad);
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
    __syncwarp();
  }
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

// Loads of a warp's loop that are in flight together.
constexpr int kBatch = 8;

// The warp's share of the call's entries, consecutive ones: fn(table, index in it, id) for each. The table is
// searched for once and followed from there: with that, release's own short way and the loads of a loop in flight
// together, giving 64 tables of 550 entries back takes 8.3 us a call instead of 12.3 (beside what the caller needs to name
// the tables: 60 us in the Python binding).
template <typename F>
__device__ __forceinline__ void for_entries(const Tables& t, int n, int warp, int lane, F&& fn) {
  const int entries = t.first[n], warps = kPlanCtas * kPlanWarps;
  const int per = (entries + warps - 1) / warps;
  const int e0 = static_cast<int>(min(static_cast<int64_t>(entries), static_cast<int64_t>(warp) * per)), e1 = min(entries, e0 + per);
  if (e0 >= e1) return;
  int f = table_of_entry(t, n, e0);
  for (int e = e0 + lane; e < e1; e += 32 * kBatch) {
    int at[kBatch], id[kBatch], i[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int x = e + 32 * b;
      if (x < e1) {
        while (x >= t.first[f + 1]) ++f;
        at[b] = f;
        i[b] = x - t.first[f];
        id[b] = t.table[f][i[b]];
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      if (e + 32 * b < e1) fn(at[b], i[b], id[b]);
  }
}

// The warp's run of pages [p0, p1): fn(page, what `load` reads of it or zeros, in the run) by whole warps.
template <typename L, typename F>
__device__ __forceinline__ void for_pages(int p0, int p1, int lane, L&& load, F&& fn) {
  for (int p = p0; p < p1; p += 32 * kBatch) {
    decltype(load(0)) v[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int x = p + 32 * b + lane;
      v[b] = decltype(load(0))();
      if (x < p1) v[b] = load(x);
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int x = p + 32 * b + lane;
      if (p + 32 * b < p1) fn(x, v[b], x < p1);
    }
  }
}

template <PageOp OP>
__global__ void __cluster_dims__(kPlanCtas, 1, 1) __launch_bounds__(kPlanThreads, 1)
    page_plan(const __grid_constant__ PlanArgs a) {
  static_assert(kPlanWarps == 32, "cluster_count scans one warp's worth of warps");
  __shared__ Exchange xa, xb;
  __shared__ Tables tables;
  griddep_launch_dependents();
  const PageTables& t = a.t;
  const int P = t.num_pages;
  const int lane = threadIdx.x & 31;
  const int me = static_cast<int>(cluster_ctarank());
  const int warp = me * kPlanWarps + (threadIdx.x >> 5);
  const int thread = me * kPlanThreads + threadIdx.x, threads = kPlanCtas * kPlanThreads;
  // this warp's pages [p0, p1)
  const int run = ((P + kPlanCtas * kPlanWarps - 1) / (kPlanCtas * kPlanWarps) + 31) & ~31;
  const int p0 = static_cast<int>(min(static_cast<int64_t>(P), static_cast<int64_t>(warp) * run));
  const int p1 = min(P, p0 + run);
  auto ref = [&](int p) { return a.refs_in[p]; };
  int bad = 0;
  for (int i = threadIdx.x; i <= t.n; i += kPlanThreads) {
    tables.first[i] = t.first[i];
    if (i < t.n) tables.table[i] = t.table[i];
  }
  griddep_wait();

  // Entries of every page (release, compact); their ids are checked here, and a fork's counts too
  if (OP != kPageFork)
    for (int p = p0 + lane; p < p1; p += 32) a.s.mark[p] = 0;
  cluster_sync();  // and every CTA of the cluster runs, before its shared memory is written to
  for_entries(tables, t.n, warp, lane, [&](int, int, int id) {
    if (id < 0 || id >= P)
      bad = 1;
    else if (OP == kPageFork)
      bad |= a.refs_in[id] < 1 || (!a.deep && a.refs_in[id] > 0x7fffffff - t.first[t.n]);  // room for the call's entries
    else
      atomicAdd(&a.s.mark[id], 1);
  });
  __syncwarp();
  if (OP == kPageRelease) {
    cluster_sync();  // every entry is counted
    auto both = [&](int p) { return make_int2(a.refs_in[p], __ldcg(&a.s.mark[p])); };
    for_pages(p0, p1, lane, both, [&](int, int2 v, bool) { bad |= v.x < 0 || v.y > v.x; });
    int unused, any;
    cluster_count(xa, 0, bad, &unused, &any);
    if (thread == 0) {
      a.s.abort[0] = any ? 1 : 0;
      a.s.abort[1] = 0;
      if (any && a.status) atomicOr(a.status, kStatusCounts);
    }
    if (any) return;
    for_pages(p0, p1, lane, both, [&](int p, int2 v, bool in) {
      if (in) a.refs_out[p] = v.x - v.y;
    });
    return;
  }
  // fork: free pages; compact: live pages
  int count = 0;
  for_pages(p0, p1, lane, ref, [&](int, int r, bool in) {
    bad |= r < 0;
    count += __popc(__ballot_sync(0xffffffffu, in && (OP == kPageFork ? r == 0 : r > 0)));
  });
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
    for_pages(p0, p1, lane, [&](int p) { return make_int2(a.refs_in[p], __ldcg(&a.s.mark[p])); }, [&](int p, int2 v, bool) {
      bad |= v.x != v.y;
      stay += __popc(__ballot_sync(0xffffffffu, v.x > 0 && p < total));
    });
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

  if (OP == kPageFork) {
    for_pages(p0, p1, lane, ref, [&](int p, int r, bool in) {
      const uint32_t free = __ballot_sync(0xffffffffu, in && r == 0);
      const int rank = before + __popc(free & ((1u << lane) - 1));
      const bool taken = in && r == 0 && rank < a.fresh;
      if (taken) a.s.fresh[rank] = p;
      if (in) a.refs_out[p] = taken ? 1 : r;
      before += __popc(free);
    });
    cluster_sync();
    for_entries(tables, t.n, warp, lane, [&](int f, int i, int id) {
      const int live = min(kPage, t.n_tokens[f] - i * kPage);
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
    });
    return;
  }

  // compact: `total` live pages stay in or move into [0, total); page p's number among the movers or holes
  for_pages(p0, p1, lane, ref, [&](int p, int r, bool in) {
    const uint32_t live = __ballot_sync(0xffffffffu, in && r > 0);
    const int rank = before + __popc(live & ((1u << lane) - 1));  // live pages below p
    if (in) {
      if (p >= total && r > 0) {
        a.s.src[rank - below] = p;
        a.s.mark[p] = rank - below;
      } else if (p < total && r == 0) {
        a.s.dst[p - rank] = p;
        a.s.live[p - rank] = kPage;
      }
    }
    before += __popc(live);
  });
  cluster_sync();
  for (int k = thread; k < copies; k += threads) a.refs_out[__ldcg(&a.s.dst[k])] = a.refs_in[__ldcg(&a.s.src[k])];
  if (a.refs_out != a.refs_in)
    for_pages(p0, min(p1, max(p0, total)), lane, ref, [&](int p, int r, bool in) {
      if (in && r > 0) a.refs_out[p] = r;
    });
  for_entries(tables, t.n, warp, lane, [&](int f, int i, int id) {
    t.out[f][i] = id < total ? id : __ldcg(&a.s.dst[__ldcg(&a.s.mark[id])]);
  });
  cluster_sync();  // in place, the movers' counts are read above
  for (int p = max(p0, total) + lane; p < p1; p += 32) a.refs_out[p] = 0;
}

// A copy unit: up to kCopyBytes of one listed page in one layer's K or V. One thread of a block moves units through
// a ring of shared-memory stages with bulk copies (a stage is refilled once the bulk store that read it has), so no
// registers stand between the load and the store and kCopyStages units a block are in flight.
constexpr int kCopyBytes = 16384;
constexpr int kCopyStages = 6;

struct CopyUnit {
  const uint8_t* src;
  uint8_t* dst;
  int heads, bytes;  // bytes of each head: its live slots
  bool whole;
};

struct CopyArgs {
  PageScratch s;
  uint8_t* pool[2 * kMaxCopyLayers];  // K of the layers, then V
  int pools;
  int heads, head_bytes, slot_bytes;  // of a page: kv heads, bytes of a head's 16 slots, of one slot
  int unit_heads, subs;               // heads of a unit, units of a page
  int* status;
};

__global__ void __launch_bounds__(32) page_copy(const __grid_constant__ CopyArgs a) {
  extern __shared__ __align__(128) uint8_t stages[];
  __shared__ __align__(8) uint64_t full[kCopyStages];
  __shared__ CopyUnit ring[kCopyStages];
  griddep_launch_dependents();
  griddep_wait();
  if (threadIdx.x != 0 || a.s.abort[0]) return;
  for (int i = 0; i < kCopyStages; ++i) mbar_init(&full[i], 1);
  fence_barrier_init();
  const int64_t units = static_cast<int64_t>(a.s.abort[1]) * a.pools * a.subs;
  const int64_t page_bytes = static_cast<int64_t>(a.heads) * a.head_bytes;
  auto unit_at = [&](int64_t u) {
    CopyUnit x;
    const int64_t kp = u / a.subs;
    const int sub = static_cast<int>(u - kp * a.subs);
    const int k = static_cast<int>(kp / a.pools);
    uint8_t* pool = a.pool[kp - static_cast<int64_t>(k) * a.pools];
    const int live = a.s.live[k];
    const int64_t at = static_cast<int64_t>(sub) * a.unit_heads * a.head_bytes;
    x.src = pool + a.s.src[k] * page_bytes + at;
    x.dst = pool + a.s.dst[k] * page_bytes + at;
    x.heads = min(a.unit_heads, a.heads - sub * a.unit_heads);
    x.bytes = live * a.slot_bytes;
    x.whole = live == kPage;
    return x;
  };
  volatile int abort_flag = 0;
  auto load = [&](int64_t u, int st) {
    const CopyUnit x = unit_at(u);
    ring[st] = x;
    const uint32_t to = smem_u32(stages + st * kCopyBytes);
    mbar_arrive_expect_tx(&full[st], x.heads * x.bytes);
    if (x.whole) {
      bulk_load(to, x.src, x.heads * x.bytes, &full[st]);
    } else {
      for (int h = 0; h < x.heads; ++h)
        bulk_load(to + h * a.head_bytes, x.src + h * a.head_bytes, x.bytes, &full[st]);
    }
  };
  auto store = [&](int st) {
    const CopyUnit x = ring[st];
    const uint32_t from = smem_u32(stages + st * kCopyBytes);
    if (x.whole) {
      bulk_store(x.dst, from, x.heads * x.bytes);
    } else {
      for (int h = 0; h < x.heads; ++h)
        bulk_store(x.dst + h * a.head_bytes, from + h * a.head_bytes, x.bytes);
    }
    bulk_commit();
  };
  // unit i of the block is in stage i % kCopyStages; loads run kCopyStages - 1 units ahead of stores
  const int64_t mine = units > blockIdx.x ? (units - blockIdx.x + gridDim.x - 1) / gridDim.x : 0;
  auto at = [&](int64_t i) { return blockIdx.x + i * gridDim.x; };
  constexpr int kAhead = kCopyStages - 1;
  int64_t asked = 0;
  for (; asked < kAhead && asked < mine; ++asked) load(at(asked), static_cast<int>(asked));
  int st = 0;
  uint32_t ph = 0;
  for (int64_t i = 0; i < mine; ++i) {
    if (!mbar_wait(&full[st], ph, &abort_flag, a.status)) break;
    store(st);
    if (asked < mine) {
      // the stage of unit asked was read by the store of unit asked - kCopyStages = i - 1
      bulk_wait_read<1>();
      load(at(asked), static_cast<int>(asked % kCopyStages));
      ++asked;
    }
    if (++st == kCopyStages) {
      st = 0;
      ph ^= 1;
    }
  }
  if (abort_flag) {
    // a load never came: the others land before the block's shared memory is released
    for (int64_t i = asked > kCopyStages ? asked - kCopyStages : 0; i < asked; ++i) {
      volatile int never = 0;
      mbar_wait(&full[i % kCopyStages], static_cast<uint32_t>((i / kCopyStages) & 1), &never, nullptr);
    }
  }
  bulk_wait_all();
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
  PdlScope pdl;
  cudaError_t e = launch_kernel(plan, dim3(kPlanCtas), dim3(kPlanThreads), 0, stream, a);
  if (e != cudaSuccess || op == kPageRelease || (op == kPageFork && a.fresh == 0)) return e;
  const int head_bytes = kPage * pool->head_dim * 2;
  constexpr int smem = kCopyStages * kCopyBytes;
  static PerDevice once;
  int dev = 0;
  if (once.pending(&dev)) {
    e = cudaFuncSetAttribute(page_copy, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    once.done(dev);
  }
  for (int l0 = 0; l0 < pool->n_layers; l0 += kMaxCopyLayers) {
    CopyArgs c;
    std::memset(&c, 0, sizeof(c));
    c.s = a.s;
    const int n = std::min(kMaxCopyLayers, pool->n_layers - l0);
    for (int l = 0; l < n; ++l) {
      c.pool[l] = static_cast<uint8_t*>(pool->k[l0 + l]);
      c.pool[n + l] = static_cast<uint8_t*>(pool->v[l0 + l]);
    }
    c.pools = 2 * n;
    c.heads = pool->n_kv_heads;
    c.head_bytes = head_bytes;
    c.slot_bytes = pool->head_dim * 2;
    c.unit_heads = std::min(pool->n_kv_heads, kCopyBytes / head_bytes);
    c.subs = (pool->n_kv_heads + c.unit_heads - 1) / c.unit_heads;
    c.status = status;
    int64_t blocks = static_cast<int64_t>(num_sms) * 2;  // resident together
    if (op == kPageFork) blocks = std::min(blocks, static_cast<int64_t>(a.fresh) * c.pools * c.subs);
    e = launch_kernel(page_copy, dim3(static_cast<unsigned>(blocks)), dim3(32), smem, stream, c);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace crf
