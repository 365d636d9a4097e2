// Attention of requests that share prefixes, a form of the kernel of chunk_attn.cuh.
//
// The rows of all requests of a group are packed into one axis for the keys that they share, as rows and heads are
// within a request, so that keys and values of the prefix are read, and multiplied, once for the group and not once a request.
// Their own keys are attended in one of two ways, whichever takes fewer units of work (share_prefixes):
//   folded   the pages of the requests' own keys are laid end to end behind the shared tiles; a row sees the shared keys and its
//            request's run of those behind them, two ranges as with sinks. The products of rows with the others' own keys are wasted; there is
//            one item a kv head instead of one more for every request, which each cost 4.6 us beside their steps
//   split    each request's own keys are items like any other, and the two parts of an output row are joined by their maxima and sums:
//              o = (e^(m1 - m) o1 + e^(m2 - m) o2) / (e^(m1 - m) l1 + e^(m2 - m) l2),  m = max(m1, m2)
//            with (m, l, o) the maximum, the sum of exponentials and their unnormalised product with v. Every segment then writes its part;
//            one merge joins an output row's parts of the group's item and of its request's, in order
// Where the rows of each request fill tiles of their own, sharing saves no products, and where there is little work in all it costs more
// latency than it saves: the requests are then attended one by one.
//
// Bound by latency at the usual sizes: 32 single rows (28 heads over 4) of 15000 shared keys and up to 600 of their own take 29 us (129 one by one),
// 64 of them 39 (241), 128 over 4000 keys 38 (137). A start of 4.5 us, some six steps a run of 1.6 to 2.4, q and the end of a part 5.5, the
// merge 7, where the bytes take 6.
#include "chunk_attn.cuh"

namespace crf {

namespace {

struct JoinArgs {
  ChunkAttnDesc d;
  AttnTable c;
  PrefixGroups g;
  int item0[kMaxEntries];
  const int* first;
  const int* last;
  const float* part;
  const float* part_ml;
  int rows;  // output rows times query heads
};

// The parts of one output row in one item: `count` of them, `rows` rows apart.
struct Parts {
  int64_t at, base;  // row of the first part's row; first row of the first part
  int rows, r, count;
};
__device__ __forceinline__ Parts parts_of(const JoinArgs& a, int e, int row, int h) {
  const int grp = a.d.n_q_heads / a.d.n_kv_heads;
  const int packed = (row - a.c.row0[e]) * grp + h % grp, all = a.c.rows[e] * grp, tile = narrow_form(all) ? kM : 2 * kM;
  const int qt = packed / tile, item = a.item0[e] + ((all + tile - 1) / tile - 1 - qt) * a.d.n_kv_heads + h / grp;
  Parts p;
  p.r = packed - qt * tile;
  p.rows = min(tile, all - qt * tile);
  p.base = __ldcg(a.first + item);
  p.count = static_cast<int>(__ldcg(a.last + item) - p.base) / p.rows + 1;
  p.at = p.base + p.r;
  return p;
}

// As chunk_attn_merge: a row by GROUPS groups of D / 4 lanes.
template <int D, int GROUPS>
__global__ void __launch_bounds__(kMergeThreads) chunk_attn_join(const __grid_constant__ JoinArgs a) {
  constexpr int kLanes = D / 4, kRows = kMergeThreads / (kLanes * GROUPS), kBatch = 4;
  __shared__ float4 red_o[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? kRows * kLanes : 1];
  __shared__ float2 red_ml[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? kRows : 1];
  griddep_launch_dependents();
  const ChunkAttnDesc& d = a.d;
  const int c = threadIdx.x % kLanes, q = threadIdx.x / kLanes % GROUPS, rr = threadIdx.x / (kLanes * GROUPS);
  const int b = min(static_cast<int>(blockIdx.x) * kRows + rr, a.rows - 1);  // a last block's spare rows repeat the last
  const int row = b / d.n_q_heads, h = b - row * d.n_q_heads;
  int lo = a.g.groups, hi = a.c.n - 1;  // the row's request, or its folded group
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.c.row0[mid] <= row) lo = mid; else hi = mid - 1;
  }
  const int group = a.g.of[lo - a.g.groups];
  griddep_wait();
  const Parts own = parts_of(a, lo, row, h);
  Parts shared = own;
  shared.count = 0;
  if (group >= 0) shared = parts_of(a, group, row, h);
  const int parts = shared.count + own.count;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = q; k0 < parts; k0 += kBatch * GROUPS) {
    float2 ml[kBatch];
    float4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int k = k0 + i * GROUPS;
      ml[i] = make_float2(-INFINITY, 0.f);
      if (k < parts) {
        const bool s = k < shared.count;
        const int rows = s ? shared.rows : own.rows, r = s ? shared.r : own.r;
        const int64_t base = (s ? shared.base : own.base) + static_cast<int64_t>(s ? k : k - shared.count) * rows;
        ml[i] = __ldcg(reinterpret_cast<const float2*>(a.part_ml) + base + r);
        v[i] = __ldcg(reinterpret_cast<const float4*>(a.part) + base * kLanes + (static_cast<int64_t>(c / 8) * rows + r) * 8 + row_unit(r, c % 8));
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (ml[i].y == 0.f) continue;  // nothing seen (its o holds no number)
      const float mn = fmaxf(m, ml[i].x), keep = m == -INFINITY ? 0.f : ex2_approx(m - mn), add = ex2_approx(ml[i].x - mn);
      o.x = o.x * keep + v[i].x * add;
      o.y = o.y * keep + v[i].y * add;
      o.z = o.z * keep + v[i].z * add;
      o.w = o.w * keep + v[i].w * add;
      l = l * keep + ml[i].y * add;
      m = mn;
    }
  }
  if (GROUPS > 1) {
    red_o[q][rr * kLanes + c] = o;
    if (c == 0) red_ml[q][rr] = make_float2(m, l);
    __syncthreads();
    if (q != 0) return;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) M = fmaxf(M, red_ml[i][rr].x);
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const float2 ml = red_ml[i][rr];
      if (ml.y == 0.f) continue;
      const float e = ex2_approx(ml.x - M);
      const float4 v = red_o[i][rr * kLanes + c];
      o.x += v.x * e;
      o.y += v.y * e;
      o.z += v.z * e;
      o.w += v.w * e;
      L += ml.y * e;
    }
    m = M;
    l = L;
  }
  const float inv = l != 0.f ? 1.0f / l : 0.f;
  *reinterpret_cast<uint2*>(d.out + row * d.out_row + h * d.out_head + c * 4) =
      make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  if (d.lse && c == 0) d.lse[static_cast<size_t>(row) * d.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Floats of a workspace's pieces, each a multiple of 64.
size_t round64(size_t n) { return (n + 63) & ~static_cast<size_t>(63); }
struct Pieces {
  size_t part, ml, items, total;
};
Pieces pieces_of(const AttnPlan& p, int head_dim) {
  Pieces x;
  if (p.shared) {
    x.part = round64(static_cast<size_t>(p.part_rows) * head_dim);
    x.ml = round64(static_cast<size_t>(p.part_rows) * 2);
    x.items = round64(2 * static_cast<size_t>(p.items));
  } else {
    x.part = part_floats(p.runs, head_dim, false);
    x.ml = part_floats(p.runs, head_dim, true);
    x.items = 0;
  }
  x.total = total_floats(p.runs, head_dim);
  return x;
}

template <int D, bool LEAN>
cudaError_t launch_prefix(const ChunkArgs<kPrefix>& a, const PrefixGroups& g, const AttnPlan& p, int num_sms, cudaStream_t stream) {
  PdlScope pdl;
  const cudaError_t e = launch_kernel_tc<D, LEAN, kPrefix>(a, p.runs.ctas, stream);
  if (e != cudaSuccess) return e;
  if (!p.shared) return launch_merge<D>(a.d, p.runs, a.part, a.part_ml, num_sms, stream);
  JoinArgs j;
  std::memset(&j, 0, sizeof(j));
  j.d = a.d;
  j.c = a.c;
  j.g = g;
  std::memcpy(j.item0, p.item0, sizeof(j.item0));
  j.first = a.prefix.first;
  j.last = a.prefix.last;
  j.part = a.part;
  j.part_ml = a.part_ml;
  int rows = 0;
  for (int i = g.groups; i < a.c.n; ++i) rows += a.c.rows[i];
  j.rows = rows * a.d.n_q_heads;
  constexpr int kRow = kMergeThreads / (D / 4);  // rows a block with one group each
  if (j.rows < 4 * kRow * num_sms) {
    constexpr int kRows8 = kRow / 8;
    return launch_kernel(chunk_attn_join<D, 8>, dim3((j.rows + kRows8 - 1) / kRows8), dim3(kMergeThreads), 0, stream, j);
  }
  return launch_kernel(chunk_attn_join<D, 1>, dim3((j.rows + kRow - 1) / kRow), dim3(kMergeThreads), 0, stream, j);
}

}  // namespace

void plan_prefix_attention(const AttnTable& a, bool shared, int n_q_heads, int n_kv_heads, bool causal, int num_sms, AttnPlan* p) {
  std::memset(p->run_rows, 0, sizeof(p->run_rows));
  p->shared = shared;
  p->items = 0;
  p->part_rows = 0;
  const int grp = n_q_heads / n_kv_heads;
  for (int i = 0; i < a.n; ++i) {
    const int rows = a.rows[i] * grp, tile = narrow_form(rows) ? kM : 2 * kM;
    p->item0[i] = p->items;
    p->items += (rows + tile - 1) / tile * n_kv_heads;
  }
  plan_runs<kPrefixCosts>(a, n_q_heads, n_kv_heads, causal, 0, num_sms, shared ? p->run_rows : nullptr, &p->runs);
  if (shared)
    for (int b = 0; b < p->runs.ctas; ++b) p->part_rows += p->run_rows[b];
}

void share_prefixes(const ChunkTable& c, const int* count, const int* keys, int n, int n_q_heads, int n_kv_heads, bool causal,
                    int num_sms, AttnTable* a, PrefixGroups* g) {
  std::memset(a, 0, sizeof(*a));
  std::memset(g, 0, sizeof(*g));
  const int grp = n_q_heads / n_kv_heads;
  // Units of one kv head's items of rows [r0, r0 + rows) of an entry of `t`.
  auto units = [&](const AttnTable& t, int i) {
    const int packed = t.rows[i] * grp;
    const bool narrow = narrow_form(packed);
    const int tile = narrow ? kM : 2 * kM;
    int64_t sum = 0;
    for (int q0 = 0; q0 < packed; q0 += tile) {
      const int steps = steps_of(t, i, q0, std::min(q0 + tile, packed) - 1, grp, causal, 0, narrow);
      sum += kPrefixCosts.segment(narrow) + static_cast<int64_t>(steps) * kPrefixCosts.step(narrow) +
             static_cast<int64_t>(steps - shared_steps(t, i, narrow, steps)) * kPrefixCosts.masked;
    }
    return sum;
  };
  // Entry i of `t`: request j, over its keys from key0 on.
  auto put_request = [&](AttnTable* t, int i, int j, int key0) {
    t->row0[i] = c.row0[j];
    t->rows[i] = rows_of(c, j);
    t->pos[i] = c.pos[j];
    t->key0[i] = key0;
    t->n_keys[i] = c.n_keys[j];
    t->sinks[i] = t->member0[i] = t->members[i] = 0;
    t->pt[i] = c.pt[j];
  };
  // The group of requests [r0, r1) over its shared keys alone.
  auto put_shared = [&](AttnTable* t, int i, int r0, int r1, int n_shared, const int32_t* pt) {
    t->row0[i] = c.row0[r0];
    t->rows[i] = c.row0[r1] - c.row0[r0];
    t->pos[i] = kMaxKeys;  // behind every key
    t->key0[i] = 0;
    t->n_keys[i] = n_shared;
    t->sinks[i] = t->member0[i] = t->members[i] = 0;
    t->pt[i] = pt;
  };
  // The same with its requests' own keys behind them. Members' numbers are those of the requests.
  auto put_folded = [&](AttnTable* t, int i, int r0, int r1, int n_shared, const int32_t* pt) {
    put_shared(t, i, r0, r1, n_shared, pt);
    t->sinks[i] = n_shared;
    t->member0[i] = r0;
    t->members[i] = r1 - r0;
    int page = 0;
    for (int j = r0; j < r1; ++j) {
      const int rows = rows_of(c, j);
      t->m_row0[j] = c.row0[j] - c.row0[r0];
      t->m_page0[j] = page;
      t->m_first[j] = n_shared / kPage;
      t->m_pos[j] = c.pos[j];
      t->m_keys[j] = c.n_keys[j];
      t->m_pt[j] = c.pt[j];
      if (rows == 0) continue;
      const int seen = causal && c.pos[j] + rows < c.n_keys[j] ? c.pos[j] + rows : c.n_keys[j];
      if (seen > n_shared) page += (seen + kPage - 1) / kPage - n_shared / kPage;
    }
  };
  static_assert(kMaxChunks <= kMaxEntries, "members are numbered as requests");
  a->num_pages = c.num_pages;
  enum Way : uint8_t { kApart, kSplit, kFolded } way[kMaxChunks];
  const int32_t* lead[kMaxChunks];
  AttnTable t;
  std::memset(&t, 0, sizeof(t));
  int64_t saved = 0;
  bool any_split = false;
  for (int i = 0, r = 0; i < n; r += count[i++]) {
    way[i] = kApart;
    lead[i] = nullptr;
    int64_t apart = 0, own = 0, pages = 0;
    for (int j = r; j < r + count[i]; ++j) {
      if (rows_of(c, j) == 0) continue;
      if (!lead[i]) lead[i] = c.pt[j];
      put_request(&t, 0, j, 0);
      apart += units(t, 0);
      put_request(&t, 0, j, keys[i]);
      own += units(t, 0);
      pages += std::max(0, c.n_keys[j] - keys[i]) / kPage + 2;
    }
    if (!lead[i] || keys[i] == 0) continue;
    put_shared(&t, 0, r, r + count[i], keys[i], lead[i]);
    const int64_t split = own + units(t, 0);
    int64_t folded = INT64_MAX;
    if (pages * kPage + keys[i] + kN <= kMaxKeys) {
      put_folded(&t, 0, r, r + count[i], keys[i], lead[i]);
      folded = units(t, 0);
    }
    if (folded < apart && folded <= split + split / 4) way[i] = kFolded;  // (a split group's parts cost every row of the call a join)
    else if (split < apart) way[i] = kSplit;
    if (way[i] != kApart) saved += apart - (way[i] == kSplit ? split : folded);
    any_split = any_split || way[i] == kSplit;
  }
  // Few long items cut over all SMs begin and end later than many short ones: wide rows' q and o, masks, more parts to merge. 32 rows over
  // 1000 shared keys (22 units an SM saved) take 20.1 us folded and 17.5 apart, drafts in two groups (11 units) 29 split and 21 apart;
  // 8 rows over 15000 (45 units) 20.5 folded and 41.6 apart. All of these are 28 heads over 4, and the units know nothing of a shared call's
  // fixed cost: timed both ways over 72 calls (8 to 32 rows or drafts, 1000 to 15000 keys, 28 heads over 4, 12 and 4 over 2), none was
  // shared to its loss, but 19 stood apart that sharing would have made 1 to 9 us faster, 8 rows of 12 heads over 2 and 15000 keys most
  // (25 apart, 16 folded).
  if (saved * n_kv_heads < static_cast<int64_t>(any_split ? 40 : 24) * num_sms)
    for (int i = 0; i < n; ++i) way[i] = kApart;
  for (int i = 0, r = 0; i < n; r += count[i++]) {
    g->any = g->any || way[i] != kApart;
    if (way[i] == kSplit) put_shared(a, g->groups++, r, r + count[i], keys[i], lead[i]);
  }
  a->n = g->groups;
  int16_t group = 0;
  for (int i = 0, r = 0; i < n; r += count[i++]) {
    if (way[i] == kFolded) {
      g->of[a->n - g->groups] = -1;
      put_folded(a, a->n++, r, r + count[i], keys[i], lead[i]);
      continue;
    }
    for (int j = r; j < r + count[i]; ++j) {
      g->of[a->n - g->groups] = way[i] == kSplit ? group : int16_t{-1};
      put_request(a, a->n++, j, way[i] == kSplit ? keys[i] : 0);
    }
    if (way[i] == kSplit) ++group;
  }
}

size_t prefix_attention_workspace(const AttnPlan& p, int head_dim) {
  const Pieces x = pieces_of(p, head_dim);
  return (x.part + x.ml + x.items + x.total) * sizeof(float);
}

cudaError_t launch_prefix_attention(const ChunkAttnDesc& d, const AttnTable& c, const PrefixGroups& g, const AttnPlan& p,
                                    void* workspace, int num_sms, cudaStream_t stream) {
  if (p.runs.ctas == 0) return cudaSuccess;
  ChunkArgs<kPrefix> a;
  std::memset(&a, 0, sizeof(a));
  const long pool_rows = static_cast<long>(c.num_pages) * d.n_kv_heads * kPage;
  if (!tensor_map_pool(&a.tmK, d.kpages, pool_rows, d.head_dim) || !tensor_map_pool(&a.tmV, d.vpages, pool_rows, d.head_dim))
    return cudaErrorInvalidValue;
  a.d = d;
  a.c = c;
  std::memcpy(a.run, p.runs.run, (p.runs.ctas + 1) * sizeof(RunStart));
  const Pieces x = pieces_of(p, d.head_dim);
  a.part = static_cast<float*>(workspace);
  a.part_ml = a.part + x.part;
  a.part_rows = p.runs.part_rows;
  a.total = a.part_ml + x.ml + x.items;
  a.prefix.on = p.shared;
  if (p.shared) {
    a.prefix.first = reinterpret_cast<int*>(a.part_ml + x.ml);
    a.prefix.last = a.prefix.first + p.items;
    std::memcpy(a.prefix.item0, p.item0, sizeof(a.prefix.item0));
    int row = 0;
    for (int b = 0; b < p.runs.ctas; ++b) {
      a.prefix.row0[b] = row;
      row += static_cast<int>(p.run_rows[b]);
    }
  }
  bool lean = true;
  for (int i = 0; i < c.n; ++i) lean = lean && static_cast<int64_t>(c.rows[i]) * (d.n_q_heads / d.n_kv_heads) <= kLeanRows;
  if (d.head_dim == 128)
    return lean ? launch_prefix<128, true>(a, g, p, num_sms, stream) : launch_prefix<128, false>(a, g, p, num_sms, stream);
  return lean ? launch_prefix<64, true>(a, g, p, num_sms, stream) : launch_prefix<64, false>(a, g, p, num_sms, stream);
}

}  // namespace crf
