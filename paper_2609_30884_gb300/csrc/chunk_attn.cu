// Attention of a chunk of new rows over their requests' cached keys, on tcgen05. Row r of a request at position
// p sees the keys lo <= j < hi with hi = min(n_keys, p + 1) (causal; n_keys otherwise) and lo = max(0, p - window + 1)
// (0 without a window): o = softmax(scale q k) v, lse = log sum exp(scale q k).
//
// The query heads of one kv head read the same keys, so a request's rows and the group's heads are packed into
// one axis (row r, head h of the group -> r group + h) and cut into tiles of 128 rows, the M of an MMA. Two chains
// S -> softmax -> P V run side by side in a CTA, so that one's products fill the other's softmax:
//   wide form    256 packed rows or a last part of them: chain t is query tile t, both read the same K/V tiles
//   narrow form  requests of at most 128 packed rows (one token of 7 heads: 7): one query tile, chain t takes
//                every other K/V tile, and the chains' (o, maximum, sum) meet in shared memory at the end
// A step of the pair of chains is one K/V tile (wide) or two (narrow).
//
// Work: the steps of all items (request, query tile or pair, kv head) laid end to end are dealt to one CTA per SM in
// equal runs (plan_chunk_attention). A run is a sequence of segments, whole items or parts of them; a part writes its
// unnormalised o, maximum and sum in fp32 to the workspace and chunk_attn_merge joins an item's parts in order of
// keys. The K/V ring runs on from segment to segment, so the copies of the next one land during this one's end.
//
// Warps: 0 gathers the pages of K and V tiles with TMA, 1 issues the MMAs, one thread of 2 finds the segments ahead, 3
// sees the ring's copies land, in order, and counts them (a chain that waited for a slot's phase itself could take
// the phase before for it: that one may be the other chain's, and copies land out of order),
// 4-7 and 8-11 are the chains' softmax (one packed row a thread; S from TMEM, P back over it as bf16, o
// rescaled there when the maximum grows by more than 2^8); they also bring q into shared memory (rows of any strides,
// packed heads). Warps whose 32 rows are all padding only keep the others company. As in the prefill attention
// (attention_tc.cu), the issuing warp waits only for each chain's P and commits only each chain's S; the softmax
// warps check that the next K/V tiles have landed and release the ring's slots. Every wait is bounded.
//
// Unseen slots may hold anything: pages that no row of the CTA sees are not fetched and stay out of P V; scores of
// unseen keys become -inf whatever they were; v of keys that no row sees is zeroed, and in tiles that only some rows
// see an infinite or NaN element of v is zeroed and given back, at the end, to the rows that see it (0 times infinity
// would be NaN in the others; infinities absorb whatever they are added to, so when does not matter).
#include "common.cuh"
#include "extend.h"
#include "tma_map.h"

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

constexpr int kM = 128;  // packed rows per query tile
constexpr int kN = 128;  // keys per K/V tile
constexpr int kPagesPerTile = kN / kPage;
constexpr int kThreads = 384;
constexpr int kMaxSlots = 6; // K/V ring
constexpr int kSegRing = 4;  // segments found ahead
// Steps of a chain after which its o starts anew. The tensor cores drop the low bits of every sum: in one chain of products
// o comes out short by 0.76e-6 of itself a tile (v of mean 1, standard deviation 0.5: 6e-3 over 2^20 keys, 0.1 over 2^24).
// So after this many tiles, 1e-4, o and the sum of weights are added to fp32 totals in the workspace, rounded to nearest
// (9728 rows over 2^24 keys: 2e-7). 2048 rows over 65536 keys take 1216 us with it, 1188 without; shorter runs
// have no totals.
constexpr int kChain = 128;
// setmaxnreg split: the first warpgroup (producer, issuer, finder) keeps kRegsCtl, the softmax warpgroups take
// kRegsSoftmax; the sum must fit what the CTA launched with.
constexpr int kRegsCtl = 80;
constexpr int kRegsSoftmax = 208;
constexpr int kRegsNeeded = 128 * kRegsCtl + 256 * kRegsSoftmax;
constexpr uint32_t kTmemCols = 512;  // S0 | S1 | O0 | O1, 128 each
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct ChunkArgs {
  CUtensorMap tmK, tmV;  // pages of the layer, box: one page of one kv head
  ChunkAttnDesc d;
  ChunkTable c;
  RunStart run[kMaxCtas + 1];
  // parts of cut items: o [slot][32-column block][row][32] with the 16-byte units of a row swizzled by it, and
  // [slot][row] maximum (log2 units) and sum. A CTA's first segment has slot 2 b, a later one 2 b + 1.
  float* part;
  float* part_ml;
  int part_rows;
  float* total;  // of chains longer than kChain: [CTA][chain][kTotals][row]
};

struct MergeArgs {
  ChunkAttnDesc d;
  const float* part;
  const float* part_ml;
  int part_rows, cuts;
  int rows[kMaxCtas + 1];  // packed rows of the cut items before each
  CutItem cut[kMaxCtas];
};

__host__ __device__ inline bool narrow_form(int packed_rows) { return packed_rows <= kM; }

// Keys [lo, hi) that rows at positions first .. last see in all; empty if hi <= lo. With the arguments swapped: the
// keys that every one of them sees.
struct KeyRange {
  int lo, hi;
};
__host__ __device__ inline KeyRange keys_of_rows(int first_pos, int last_pos, int n_keys, bool causal, int window) {
  KeyRange k;
  k.lo = window > 0 && first_pos + 1 > window ? first_pos + 1 - window : 0;
  k.hi = causal && last_pos + 1 < n_keys ? last_pos + 1 : n_keys;
  return k;
}
// K/V tiles [first, first + count) of packed rows q0 .. q1 of a request, and the steps that they make.
struct TileSpan {
  int first, count, steps;
};
__host__ __device__ inline TileSpan tiles_of(const KeyRange& k, bool narrow) {
  TileSpan s;
  s.first = k.lo / kN;
  s.count = k.hi > k.lo ? (k.hi + kN - 1) / kN - s.first : 0;
  s.steps = narrow ? (s.count + 1) / 2 : s.count;
  return s;
}

__device__ __forceinline__ void regs_dec_ctl() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsCtl)); }
__device__ __forceinline__ void regs_inc_softmax() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
}
__device__ __forceinline__ void softmax_groups_sync() {
  __syncwarp();
  asm volatile("barrier.sync 1, 256;" ::: "memory");
}
// The same, ANDing a flag over the eight warps, so that they leave a loop together.
__device__ __forceinline__ bool softmax_groups_and(bool flag) {
  uint32_t out;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred pi, po;\n\t"
      "setp.ne.u32 pi, %1, 0;\n\t"
      "barrier.red.and.pred po, 1, 256, pi;\n\t"
      "selp.u32 %0, 1, 0, po;\n\t}"
      : "=r"(out)
      : "r"(flag ? 1u : 0u)
      : "memory");
  return out != 0;
}
__device__ __forceinline__ void mbar_arrive_n(uint64_t* bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}

// Scores of keys outside [lo, hi) (relative to the tile) of the thread's row become -inf, 32 keys at a time; 32 keys
// that every row of the warp sees are left alone. A pass of its own over TMEM, on the few tiles that need it, keeps the
// softmax one short piece of code (with the mask in a second instance of it, a masked tile took 3300 cycles, and
// 6600 where its instructions were not cached, against 1250 unmasked).
__device__ __forceinline__ void mask_tile(uint32_t tS, int lo, int hi) {
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    if (!__any_sync(0xffffffffu, c * 32 < lo || c * 32 + 32 > hi)) continue;
    const int h = min(32, max(0, hi - c * 32)), l = min(32, max(0, lo - c * 32));
    const uint32_t below_h = h == 32 ? 0xffffffffu : (1u << h) - 1, below_l = l == 32 ? 0xffffffffu : (1u << l) - 1;
    const uint32_t seen = below_h & ~below_l;
    uint32_t x[32];
    tmem_ld32(tS + c * 32, x);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (!(seen & (1u << i))) x[i] = __float_as_uint(-INFINITY);
    tmem_st32(tS + c * 32, x);
  }
  tmem_st_wait();
}

// One packed row's share of a K/V tile: 128 raw scores from TMEM, running maximum and sum, o rescaled in TMEM when
// the maximum grows by more than 2^8, P (bf16, unnormalised) back over the scores. A row that has seen no key yet
// keeps a maximum of -inf.
template <int D>
__device__ __forceinline__ void softmax_tile(uint32_t tS, uint32_t tO, bool first, float sl2, float& m_run, float& l_run) {
  uint32_t sr[4][32];
#pragma unroll
  for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, sr[c]);
  tmem_ld_wait();
  float mx[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) mx[k] = -INFINITY;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      mx[i & 7] = fmax3(mx[i & 7], __uint_as_float(sr[c][2 * i]), __uint_as_float(sr[c][2 * i + 1]));
  const float mt = fmax3(fmax3(mx[0], mx[1], mx[2]), fmax3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7]));
  const bool grow = (mt - m_run) * sl2 > kRescaleThreshold;  // false while both are -inf
  const float alpha = grow ? ex2_approx((m_run - mt) * sl2) : 1.0f;
  if (!first && __any_sync(0xffffffffu, grow)) {
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      tmem_ld32(tO + c * 32, o);
      tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
      tmem_st32(tO + c * 32, o);
    }
    tmem_st_wait();
  }
  if (grow) {
    l_run *= alpha;
    m_run = mt;
  }
  const float neg_m = m_run == -INFINITY ? 0.f : -m_run * sl2;
  const uint64_t sl2x2 = f32x2(sl2, sl2), negm2 = f32x2(neg_m, neg_m);
  uint64_t rs2[2] = {f32x2(0.f, 0.f), f32x2(0.f, 0.f)};
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint32_t pk[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x0, x1;
      f32x2_split(fma_f32x2(f32x2(__uint_as_float(sr[c][2 * i]), __uint_as_float(sr[c][2 * i + 1])),
                            sl2x2, negm2), x0, x1);
      const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
      rs2[i & 1] = add_f32x2(rs2[i & 1], f32x2(p0, p1));
      // the product with v is bf16 x bf16: a weight is off by 2^-8 of itself at most; the sum keeps the fp32 one
      pk[i] = pack_bf16(p0, p1);
    }
    tmem_st16(tS + 16 * c, pk);
  }
  tmem_st_wait();
  float r0, r1, r2, r3;
  f32x2_split(rs2[0], r0, r1);
  f32x2_split(rs2[1], r2, r3);
  l_run += (r0 + r1) + (r2 + r3);
}

// The totals of a thread's row: o's columns, the sum of weights and the maximum that they were formed under, element i at
// total[i kM]. They are added to between two loops over tiles: a test in the one loop, with the maximum and the sum in
// registers, cost every call 2-6%.
template <int D>
constexpr int kTotals = D + 2;
// o and the sum of a chain's last steps into the row's totals; the first time there is nothing to add to.
template <int D>
__device__ __forceinline__ void add_to_totals(uint32_t tO, float* total, bool first, float sl2, float m_run, float& l_run) {
  const float m_was = first ? -INFINITY : __ldcg(total + (D + 1) * kM);
  const float keep = m_was == -INFINITY ? 0.f : ex2_approx((m_was - m_run) * sl2);
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    uint32_t o[32];
    float was[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) was[i] = first ? 0.f : __ldcg(total + (c * 32 + i) * kM);
    tmem_ld32(tO + c * 32, o);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 32; ++i) __stcg(total + (c * 32 + i) * kM, was[i] * keep + __uint_as_float(o[i]));
  }
  __stcg(total + D * kM, (first ? 0.f : __ldcg(total + D * kM)) * keep + l_run);
  __stcg(total + (D + 1) * kM, m_run);
  l_run = 0.f;
}
// The totals into o and the sum, at a segment's end.
template <int D>
__device__ __forceinline__ void add_totals(uint32_t tO, const float* total, float sl2, float m_run, float& l_run) {
  const float m_was = __ldcg(total + (D + 1) * kM);
  const float keep = m_was == -INFINITY ? 0.f : ex2_approx((m_was - m_run) * sl2);
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    uint32_t o[32];
    float was[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) was[i] = __ldcg(total + (c * 32 + i) * kM);
    tmem_ld32(tO + c * 32, o);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(was[i] * keep + __uint_as_float(o[i]));
    tmem_st32(tO + c * 32, o);
  }
  tmem_st_wait();
  l_run += __ldcg(total + D * kM) * keep;
}

__device__ __forceinline__ bool not_finite_bf16(uint32_t h) { return (h & 0x7F80u) == 0x7F80u; }

// LEAN: every request of the call has at most 64 packed rows (single tokens and short drafts), so that o at a segment's
// end takes half the space and the ring a slot more: 8 rows of 4K-16K keys, replayed from a graph, take 37.4 us instead of 39.5.
constexpr int kLeanRows = 64;
template <int D, bool LEAN>
struct Tile {
  static constexpr int kSlots = LEAN ? 6 : 5;
  static constexpr int kStageRows = LEAN ? kLeanRows : 128;
  static constexpr int HALVES = D / 64;
  static constexpr int Q_BYTES = kM * D * 2;
  static constexpr int KV_BYTES = kN * D * 2;
  static constexpr int HALF_ROWS_BYTES = kN * 128;    // one 64-column half of a query tile
  static constexpr int GROUP_BYTES = HALVES * 1024;   // 8 keys, all halves, in a K/V slot
  static constexpr int STAGE_BYTES = LEAN ? 2 * kM * 128 : 2 * kM * 256;  // q tiles; at a segment's end rows of o
  static constexpr int kSmem = STAGE_BYTES + kSlots * KV_BYTES + 1024;
};

// Where an element of a K/V slot lies: key, 16-byte unit of the head.
template <int D>
__device__ __forceinline__ uint4* slot_unit(uint8_t* slot, int key, int unit) {
  using T = Tile<D, false>;
  return reinterpret_cast<uint4*>(slot + (key >> 3) * T::GROUP_BYTES + (unit >> 3) * 1024 + (key & 7) * 128 +
                                  (((unit & 7) ^ (key & 7)) << 4));
}

// Keys [a0, a1) and [b0, b1) of a V tile, dealt to `threads`: those outside [lo, hi), which no row sees, become
// zeros, and so do infinite and NaN elements of the others (*dirty is set).
template <int D>
__device__ __forceinline__ void clean_v(uint8_t* slot, int a0, int a1, int b0, int b1, int lo, int hi, int thread,
                                        int threads, volatile int* dirty) {
  constexpr int kUnits = D / 8;
  const int unit = thread % kUnits, step = threads / kUnits, n = a1 - a0 + b1 - b0;
#pragma unroll 1
  for (int i = thread / kUnits; i < n; i += step) {
    const int key = i < a1 - a0 ? a0 + i : b0 + i - (a1 - a0);
    uint4* at = slot_unit<D>(slot, key, unit);
    uint4 v = make_uint4(0, 0, 0, 0);
    bool write = key < lo || key >= hi;
    if (!write) {
      v = *at;
      uint32_t* e = reinterpret_cast<uint32_t*>(&v);
      uint32_t any = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t bad = (not_finite_bf16(e[q]) ? 0x0000FFFFu : 0u) | (not_finite_bf16(e[q] >> 16) ? 0xFFFF0000u : 0u);
        e[q] &= ~bad;
        any |= bad;
      }
      write = any != 0;
      if (write) *dirty = 1;
    }
    if (write) *at = v;
  }
}

// A segment: the item's rows, and the keys that the CTA reads.
struct Segment {
  int g, q0, rows;      // kv head; the item's first packed row; packed rows of the request
  int pos, n_keys, row0;
  const int32_t* pt;
  bool end;             // no further segment
  bool narrow;
  int slot;             // of a part of an item; -1: the whole item
  int all_lo, all_hi;   // keys that some row sees
  KeyRange full0, full1;  // keys that all rows of a chain see
  int jb, J;            // K/V tiles; every one holds a key that some row sees
  int n0, n1;           // steps of the chains
  int quarters0, quarters1;  // warps of a chain with rows
};

struct Shared {
  uint64_t q_full, o_full, drain;
  uint64_t kv_full[kMaxSlots], kv_empty[kMaxSlots];
  uint64_t s_full[2], p_full[2];
  uint64_t seg_full[kSegRing], seg_empty[kSegRing];
  Segment seg[kSegRing];
  float2 ml[kM];       // narrow: chain 1's maxima and sums
  uint64_t tmem_free;  // the softmax warps are done with TMEM
  uint32_t landed;     // items of the ring that have landed, in order, over all segments
  uint32_t tmem_base;
  volatile int abort_flag;
  volatile int dirty;  // an infinite or NaN element of v was zeroed
};

// Walks a run's segments.
struct Walk {
  RunStart at;
  bool first = true;
  __device__ __forceinline__ void next(const ChunkArgs& a, Segment& w) {
    const RunStart& to = a.run[blockIdx.x + 1];
    w.end = at.req > to.req || (at.req == to.req && (at.qt < to.qt || (at.qt == to.qt && (at.g > to.g || (at.g == to.g && at.step >= to.step)))));
    if (w.end) return;
    const int i = at.req, grp = a.d.n_q_heads / a.d.n_kv_heads;
    const int rows = (a.c.row0[i + 1] - a.c.row0[i]) * grp;
    const bool narrow = narrow_form(rows);
    const int tile = narrow ? kM : 2 * kM, q0 = at.qt * tile;
    w.g = at.g;
    w.q0 = q0;
    w.rows = rows;
    w.pos = a.c.pos[i];
    w.n_keys = a.c.n_keys[i];
    w.row0 = a.c.row0[i];
    w.pt = a.c.pt[i];
    w.narrow = narrow;
    // keys of the chains' query tiles
    KeyRange some[2], full[2];
    int valid[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r0 = q0 + (narrow ? 0 : t * kM), r1 = min(r0 + kM, rows) - 1;
      valid[t] = max(0, r1 - r0 + 1);
      const int p0 = w.pos + r0 / grp, p1 = w.pos + r1 / grp;
      some[t] = keys_of_rows(p0, p1, w.n_keys, a.d.causal, a.d.window);
      full[t] = keys_of_rows(p1, p0, w.n_keys, a.d.causal, a.d.window);
      if (valid[t] == 0) some[t].hi = 0;
    }
    KeyRange all = {some[0].lo, max(some[0].hi, some[1].hi)};
    w.all_lo = all.lo;
    w.all_hi = all.hi;
    w.full0 = full[0];
    w.full1 = full[1];
    const TileSpan s = tiles_of(all, narrow);
    const bool last = to.req == i && to.qt == at.qt && to.g == at.g;  // the run ends within the item
    const int s1 = last ? min(to.step, s.steps) : s.steps, per = narrow ? 2 : 1;
    w.jb = s.first + at.step * per;
    w.J = min(s.count - at.step * per, (s1 - at.step) * per);
    w.n0 = narrow ? (w.J + 1) / 2 : min(w.J, max(0, (some[0].hi + kN - 1) / kN - w.jb));
    w.n1 = narrow ? w.J / 2 : min(w.J, max(0, (some[1].hi + kN - 1) / kN - w.jb));
    w.quarters0 = (valid[0] + 31) / 32;
    w.quarters1 = (valid[1] + 31) / 32;
    w.slot = at.step == 0 && s1 == s.steps ? -1 : 2 * static_cast<int>(blockIdx.x) + (first ? 0 : 1);
    first = false;
    // the next item
    at.step = s1;
    if (s1 < s.steps) return;  // the run's end
    at.step = 0;
    if (++at.g < a.d.n_kv_heads) return;
    at.g = 0;
    if (--at.qt >= 0) return;
    do ++at.req; while (at.req < a.c.n && a.c.row0[at.req + 1] == a.c.row0[at.req]);
    if (at.req < a.c.n) {
      const int r = (a.c.row0[at.req + 1] - a.c.row0[at.req]) * grp, t = narrow_form(r) ? kM : 2 * kM;
      at.qt = (r + t - 1) / t - 1;
    } else {
      at.qt = 0;
    }
  }
};

// The ring's sequence within a segment of J tiles: K0 V0 K1 V1 ... (wide), K0 K1 V0 V1 K2 K3 ... (narrow: both chains
// start early; a last odd tile alone).
__device__ __forceinline__ int item_k(bool narrow, int j) { return narrow ? 4 * (j >> 1) + (j & 1) : 2 * j; }
__device__ __forceinline__ int item_v(bool narrow, int j, int J) {
  return narrow ? 4 * (j >> 1) + (j + 1 == J && (j & 1) == 0 ? 1 : 2 + (j & 1)) : 2 * j + 1;
}
// K/V tile of a chain's step.
__device__ __forceinline__ int tile_of(bool narrow, int t, int s) { return narrow ? 2 * s + t : s; }
// Pages [first, last) of tile j that some row sees.
struct PageSpan {
  int lo, hi;  // of the segment, from its first tile's first page on
  __device__ __forceinline__ explicit PageSpan(const Segment& w)
      : lo(w.all_lo / kPage - w.jb * kPagesPerTile), hi((w.all_hi + kPage - 1) / kPage - w.jb * kPagesPerTile) {}
  __device__ __forceinline__ int first(int j) const { return max(0, lo - j * kPagesPerTile); }
  __device__ __forceinline__ int last(int j) const { return min(kPagesPerTile, hi - j * kPagesPerTile); }
};
// Wait until `items` items of the ring have landed: the count is monotonic, so no phase is mistaken for another. The
// outcome is uniform over the warp.
__device__ __forceinline__ uint32_t ld_acquire_shared(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.acquire.cta.shared::cta.u32 %0, [%1];" : "=r"(v) : "r"(smem_u32(p)) : "memory");
  return v;
}
__device__ __forceinline__ void st_release_shared(uint32_t* p, uint32_t v) {
  asm volatile("st.release.cta.shared::cta.u32 [%0], %1;" ::"r"(smem_u32(p)), "r"(v) : "memory");
}
__device__ __forceinline__ bool wait_landed(Shared& sh, int items, int* status) {
  unsigned long long t0 = 0;
  for (uint32_t it = 1;; ++it) {
    if (__all_sync(0xffffffffu, static_cast<int>(ld_acquire_shared(&sh.landed) - static_cast<uint32_t>(items)) >= 0)) return true;
    if ((it & 63u) == 0) {
      if (__any_sync(0xffffffffu, sh.abort_flag != 0)) return false;
      if ((it & 1023u) == 0) {
        const unsigned long long now = globaltimer_ns();
        if (t0 == 0) t0 = now;
        if (__any_sync(0xffffffffu, now - t0 > kWaitLimitNs)) {
          sh.abort_flag = 1;
          if (status && (threadIdx.x & 31) == 0) atomicOr(status, kStatusTimeout);
          return false;
        }
      }
    }
  }
}
// Slot of the ring `n` items on (n <= SLOTS).
template <int SLOTS>
__device__ __forceinline__ int slot_after(int slot, int n) {
  slot += n;
  return slot >= SLOTS ? slot - SLOTS : slot;
}
// 16-byte unit u of row r's 128 bytes (32 columns of fp32, or of bf16 in the first four) in the stage.
__device__ __forceinline__ int row_unit(int r, int u) { return u ^ (r & 7); }

template <int D, bool LEAN>
__global__ void __launch_bounds__(kThreads, 1) chunk_attn_kernel(const __grid_constant__ ChunkArgs a) {
  using T = Tile<D, LEAN>;
  constexpr int kSlots = T::kSlots;
  constexpr int Q_BYTES = T::Q_BYTES, KV_BYTES = T::KV_BYTES, GROUP_BYTES = T::GROUP_BYTES;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) Shared sh;
  griddep_launch_dependents();
  uint8_t* stage = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sKV = stage + T::STAGE_BYTES;
  const ChunkAttnDesc& d = a.d;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);  // uniform
  const int lane = threadIdx.x & 31;
  if (warp == 1) {
    tmem_alloc(&sh.tmem_base, kTmemCols);
    tmem_relinquish();
  } else if (threadIdx.x == 0) {
    mbar_init(&sh.q_full, 8);
    mbar_init(&sh.o_full, 1);
    mbar_init(&sh.drain, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&sh.s_full[t], 1);
      mbar_init(&sh.p_full[t], 4);  // the chain's first warp arrives for those without rows
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&sh.kv_full[i], 1);
      mbar_init(&sh.kv_empty[i], 3);  // both chains, or twice the one that reads it, and warp 3
    }
    for (int i = 0; i < kSegRing; ++i) {
      mbar_init(&sh.seg_full[i], 1);
      mbar_init(&sh.seg_empty[i], 11);
    }
    mbar_init(&sh.tmem_free, 8);
    sh.landed = 0;
    sh.abort_flag = 0;
    sh.dirty = 0;
    fence_barrier_init();
  }
  Walk walk;
  if (threadIdx.x == 64) {
    // the first segment, while the others set up
    walk.at = a.run[blockIdx.x];
    Segment w;
    walk.next(a, w);
    sh.seg[0] = w;
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  // Pages, their tables and q may come from the kernel before. Every role waits for it here, so that the bounded waits
  // below measure this kernel alone (the issuer's for q, say, would run out behind a kernel of over two seconds).
  griddep_wait();

  if (warp < 4) {
    regs_dec_ctl();
    if (warp == 0) {
      // ---------------------------------------------------------------- producer
      const bool issuer = elect_one();
      bool ok = true;
      int slot = 0, armed = 0;
      uint32_t ph = 0;
      for (int n = 0; ok; ++n) {
        ok = mbar_wait_warp(&sh.seg_full[n % kSegRing], (n / kSegRing) & 1, &sh.abort_flag, d.status);
        if (!ok) break;
        const Segment& w = sh.seg[n % kSegRing];
        if (w.end) break;
        const PageSpan pages(w);
        const int J = w.J, jb = w.jb, group = w.narrow ? 2 : 1;  // tiles whose K come before their V
        auto page_id = [&](int j) {
          const int p = lane & (kPagesPerTile - 1);
          int id = 0;
          if (p >= pages.first(j) && p < pages.last(j)) {
            id = w.pt[(jb + j) * kPagesPerTile + p];
            if (id < 0 || id >= a.c.num_pages) {
              if (d.status) atomicOr(d.status, kStatusBounds);
              id = 0;
            }
          }
          return id;
        };
        int id0 = J > 0 ? page_id(0) : 0, id1 = J > 1 ? page_id(1) : 0;
        for (int j0 = 0; j0 < J && ok; j0 += group) {
          // ids of the tiles after these, on their way while these are asked for
          const int next0 = j0 + 2 < J ? page_id(j0 + 2) : 0, next1 = w.narrow && j0 + 3 < J ? page_id(j0 + 3) : 0;
#pragma unroll 1
          for (int x = 0; x < 2 * group; ++x) {
            const int i = w.narrow ? x & 1 : 0, kv = w.narrow ? x >> 1 : x, j = j0 + i;
            if (j >= J) continue;
            ok = mbar_wait_warp(&sh.kv_empty[slot], ph ^ 1, &sh.abort_flag, d.status);
            if (!ok) break;
            const int pg0 = pages.first(j), pg1 = pages.last(j), ids = i ? id1 : id0;
            if (issuer) mbar_arrive_expect_tx(&sh.kv_full[slot], (pg1 - pg0) * (kPage / 8) * GROUP_BYTES);
            uint8_t* dst = sKV + slot * KV_BYTES;
            const CUtensorMap* map = kv == 0 ? &a.tmK : &a.tmV;
#pragma unroll
            for (int p = 0; p < kPagesPerTile; ++p) {
              const int at = (__shfl_sync(0xffffffffu, ids, p) * d.n_kv_heads + w.g) * (kPage / 8);
              if (issuer && p >= pg0 && p < pg1)
                tma_load_4d(dst + p * (kPage / 8) * GROUP_BYTES, map, &sh.kv_full[slot], 0, 0, 0, at);
            }
            ++armed;
            if (++slot == kSlots) {
              slot = 0;
              ph ^= 1;
            }
          }
          id0 = w.narrow ? next0 : id1;
          id1 = w.narrow ? next1 : next0;
        }
        __syncwarp();
        if (issuer) mbar_arrive(&sh.seg_empty[n % kSegRing]);
      }
      if (!ok) {
        // every copy issued lands before the CTA can exit: the last use of every slot
        volatile int never = 0;
        for (int i = 0; i < kSlots && i < armed; ++i) {
          const int u = armed - 1 - i;
          mbar_wait(&sh.kv_full[u % kSlots], static_cast<uint32_t>((u / kSlots) & 1), &never, nullptr);
        }
      }
    } else if (warp == 1) {
      // -------------------------------------------------------------- MMA issuer
      // S of both chains' first tiles, then P V and the next S of each chain in turn. MMAs of one thread execute in
      // issue order, so a chain's next S overwrites the score columns only after P V has read P from them.
      const bool issuer = elect_one();
      bool ok = true, issued = false;
      const uint32_t idesc_s = idesc_bf16_f32(kM, kN);
      const uint32_t idesc_o = idesc_bf16_f32(kM, D, false, true);
      const uint64_t qd = smem_desc(smem_u32(stage), 16, 1024, kSwizzle128B);
      const uint64_t kd = smem_desc(smem_u32(sKV), 16, GROUP_BYTES, kSwizzle128B);
      const uint64_t vd = smem_desc(smem_u32(sKV), 1024, GROUP_BYTES, kSwizzle128B);
      int base = 0, work = 0;      // ring items and segments with tiles before this one
      int done0 = 0, done1 = 0;    // the chains' steps before it
      for (int n = 0; ok; ++n) {
        ok = mbar_wait_warp(&sh.seg_full[n % kSegRing], (n / kSegRing) & 1, &sh.abort_flag, d.status);
        if (!ok) break;
        const Segment& w = sh.seg[n % kSegRing];
        if (w.end) break;
        const bool narrow = w.narrow;
        const PageSpan pages(w);
        const int J = w.J, n0 = w.n0, n1 = w.n1;
        auto issue_s = [&](int t, int slot) {
          const uint64_t q = qd + static_cast<uint32_t>((narrow ? 0 : t) * (Q_BYTES >> 4));
          const uint64_t k = kd + static_cast<uint32_t>(slot * (KV_BYTES >> 4));
          if (issuer) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              mma_bf16_ss(tmem + t * 128, q + (kk >> 2) * (T::HALF_ROWS_BYTES >> 4) + (kk & 3) * 2,
                          k + (kk >> 2) * 64 + (kk & 3) * 2, idesc_s, kk > 0 ? 1u : 0u);
            mma_commit(&sh.s_full[t]);
          }
        };
        if (J > 0) {
          ok = mbar_wait_warp(&sh.q_full, work & 1, &sh.abort_flag, d.status);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok || (t ? n1 : n0) == 0) continue;
            const int item = base + item_k(narrow, tile_of(narrow, t, 0));
            ok = wait_landed(sh, item + 1, d.status);
            if (!ok) continue;
            tc_fence_after();
            issue_s(t, item % kSlots);
            issued = true;
          }
          // slots of the chains' V and next K, formed ahead of the wait
          int vs[2], ks[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            vs[t] = (base + item_v(narrow, tile_of(narrow, t, 0), J)) % kSlots;
            ks[t] = (base + item_k(narrow, tile_of(narrow, t, 1))) % kSlots;
          }
          const int most = max(n0, n1), stride = narrow ? 4 : 2;
          for (int s = 0; s < most && ok; ++s) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const int steps = t ? n1 : n0, j = tile_of(narrow, t, s);
              if (!ok || s >= steps) continue;
              const int pg0 = pages.first(j), pg1 = pages.last(j);
              // a last odd tile of the narrow form has its V next to its K
              const int vslot = narrow && t == 0 && s > 0 && j + 1 == J ? slot_after<kSlots>(vs[t], kSlots - 1) : vs[t];
              const uint64_t v = vd + static_cast<uint32_t>(vslot * (KV_BYTES >> 4));
              const bool full = pg0 == 0 && pg1 == kPagesPerTile, anew = s % kChain == 0;
              // P of this step is in TMEM, and its V and the chain's next K have landed
              ok = mbar_wait_warp(&sh.p_full[t], ((t ? done1 : done0) + s) & 1, &sh.abort_flag, d.status);
              if (!ok) continue;
              tc_fence_after();
              if (issuer) {
                if (full) {
#pragma unroll
                  for (int kk = 0; kk < kN / 16; ++kk)
                    mma_bf16_ts(tmem + 256 + t * 128, tmem + t * 128 + kk * 8, v + kk * (2 * GROUP_BYTES >> 4), idesc_o,
                                (!anew || kk > 0) ? 1u : 0u);
                } else {
                  // 16 keys, one page, an MMA: pages that no row sees are left out
#pragma unroll 1
                  for (int kk = pg0; kk < pg1; ++kk)
                    mma_bf16_ts(tmem + 256 + t * 128, tmem + t * 128 + kk * 8, v + kk * (2 * GROUP_BYTES >> 4), idesc_o,
                                (!anew || kk > pg0) ? 1u : 0u);
                }
              }
              if (s + 1 < steps) issue_s(t, ks[t]);
              vs[t] = slot_after<kSlots>(vs[t], stride);
              ks[t] = slot_after<kSlots>(ks[t], stride);
            }
          }
          if (ok && issuer) mma_commit(&sh.o_full);
          base += 2 * J;
          done0 += n0;
          done1 += n1;
          ++work;
        }
        __syncwarp();
        if (issuer) mbar_arrive(&sh.seg_empty[n % kSegRing]);
      }
      if (!ok && issued && issuer) {
        mma_commit(&sh.drain);
        volatile int never = 0;
        mbar_wait(&sh.drain, 0, &never, nullptr);
      }
    } else if (threadIdx.x == 64) {
      // -------------------------------------------------------------- segments
      mbar_arrive(&sh.seg_full[0]);
      for (int n = 1;; ++n) {
        if (!mbar_wait(&sh.seg_empty[n % kSegRing], ((n / kSegRing) & 1) ^ 1, &sh.abort_flag, d.status)) break;
        Segment w;
        walk.next(a, w);
        sh.seg[n % kSegRing] = w;
        mbar_arrive(&sh.seg_full[n % kSegRing]);
        if (w.end) break;
      }
    } else if (warp == 3) {
      // -------------------------------------------------------------- landed copies, in order
      const bool issuer = elect_one();
      bool ok = true;
      uint32_t item = 0;
      int slot = 0;
      uint32_t ph = 0;
      for (int n = 0; ok; ++n) {
        ok = mbar_wait_warp(&sh.seg_full[n % kSegRing], (n / kSegRing) & 1, &sh.abort_flag, d.status);
        if (!ok) break;
        const Segment& w = sh.seg[n % kSegRing];
        if (w.end) break;
        const int items = 2 * w.J;
        for (int i = 0; i < items; ++i) {
          ok = mbar_wait_warp(&sh.kv_full[slot], ph, &sh.abort_flag, d.status);
          if (!ok) break;
          ++item;
          if (issuer) {
            st_release_shared(&sh.landed, item);
            mbar_arrive(&sh.kv_empty[slot]);
          }
          if (++slot == kSlots) {
            slot = 0;
            ph ^= 1;
          }
        }
        __syncwarp();
        if (issuer) mbar_arrive(&sh.seg_empty[n % kSegRing]);
      }
    }
  } else {
    regs_inc_softmax();
    // ---------------------------------------------------------------- q, softmax, epilogue
    const int t = (warp - 4) >> 2, tid = threadIdx.x - 128;
    const int quarter = warp & 3;
    const int r = quarter * 32 + lane;  // row of the query tile (= TMEM lane)
    const uint32_t lane_off = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t tS = tmem + lane_off + t * 128, tO = tmem + lane_off + 256 + t * 128;
    const float sl2 = kLog2e * d.scale;
    const int grp = d.n_q_heads / d.n_kv_heads;
    bool ok = true;
    int base = 0, work = 0, done = 0;  // ring items, segments with tiles, steps of the chain before this segment
    for (int n = 0;; ++n) {
      // The warps go from segment to segment together: the stage is free for q once all have left it
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&sh.seg_full[n % kSegRing], (n / kSegRing) & 1, &sh.abort_flag, d.status));
      ok = softmax_groups_and(ok);
      if (!ok) break;
      const Segment& w = sh.seg[n % kSegRing];
      if (w.end) break;
      const bool narrow = w.narrow;
      const PageSpan pages(w);
      const int J = w.J, jb = w.jb, n0 = w.n0, n1 = w.n1, last_row = w.rows - 1, row0 = w.row0;
      const int steps = t ? n1 : n0, quarters = t ? w.quarters1 : w.quarters0;
      if (J > 0) {
        // q: 16-byte units of a row side by side in a warp; rows behind the request's last are zeros
        constexpr int kUnits = D / 8, kStep = 256 / kUnits, kTurns = kM / kStep;
        const int u = tid % kUnits;
        int row = (w.q0 + tid / kUnits) / grp, h = w.q0 + tid / kUnits - row * grp;
        const int row_step = kStep / grp, h_step = kStep - row_step * grp;
        uint4 v[LEAN ? 1 : 2][kTurns];  // every load in flight
#pragma unroll
        for (int x = 0; x < (LEAN ? 1 : 2); ++x)
#pragma unroll
          for (int i = 0; i < kTurns; ++i) {
            v[x][i] = make_uint4(0, 0, 0, 0);
            if (w.q0 + x * kM + tid / kUnits + i * kStep <= last_row)
              v[x][i] = *reinterpret_cast<const uint4*>(d.q + (row0 + row) * d.q_row + (w.g * grp + h) * d.q_head + u * 8);
            row += row_step;
            h += h_step;
            if (h >= grp) {
              h -= grp;
              ++row;
            }
          }
#pragma unroll
        for (int x = 0; x < (LEAN ? 1 : 2); ++x) {
          if (x == 1 && narrow) break;
#pragma unroll
          for (int i = 0; i < kTurns; ++i) {
            const int rr = tid / kUnits + i * kStep;
            *reinterpret_cast<uint4*>(stage + x * Q_BYTES + (u >> 3) * T::HALF_ROWS_BYTES + rr * 128 +
                                      (((u & 7) ^ (rr & 7)) << 4)) = v[x][i];
          }
        }
        if (tid == 0) sh.dirty = 0;
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full);
      }
      const int R = w.q0 + (narrow ? 0 : t * kM) + r;  // packed row
      const int row = min(R, last_row) / grp;
      const KeyRange mine = keys_of_rows(w.pos + row, w.pos + row, w.n_keys, d.causal, d.window);
      float m_run = -INFINITY, l_run = 0.f;  // maximum in raw score units
      auto totals = [&]() { return a.total + static_cast<size_t>(2 * blockIdx.x + t) * (kTotals<D> * kM) + r; };
      const KeyRange full = t ? w.full1 : w.full0;  // keys that all rows of the chain see, and of the CTA
      const bool both = !narrow && n1 > 0 && n0 > 0;
      const int cta_lo = both ? max(w.full0.lo, w.full1.lo) : full.lo;
      const int cta_hi = both ? min(w.full0.hi, w.full1.hi) : full.hi;
      const int share = both ? 1 : 2;  // arrivals that release a slot
      auto release = [&](int item) {
        if (quarter == 0 && lane == 0) mbar_arrive_n(&sh.kv_empty[(base + item) % kSlots], share);
      };
      auto release_slot = [&](int slot) {
        if (quarter == 0 && lane == 0) mbar_arrive_n(&sh.kv_empty[slot], share);
      };
      if (quarter < quarters && steps > 0) {
        // the ring's items of this step: K and V and their slots
        const int stride = narrow ? 4 : 2;
        int ki = base + item_k(narrow, tile_of(narrow, t, 0)), vi = base + item_v(narrow, tile_of(narrow, t, 0), J);
        int ks = ki % kSlots, vs = vi % kSlots, last_vs = 0;
        for (int s0 = 0; s0 < steps && ok; s0 += kChain) {
          const int s1 = min(steps, s0 + kChain);
          if (s0 > 0) {
            // S of the step complete: so is o of the steps before, which this step's P V overwrites
            ok = __all_sync(0xffffffffu, mbar_wait(&sh.s_full[t], (done + s0) & 1, &sh.abort_flag, d.status));
            if (!ok) break;
            tc_fence_after();
            add_to_totals<D>(tO, totals(), s0 == kChain, sl2, m_run, l_run);
          }
          for (int s = s0; s < s1 && ok; ++s) {
            const int j = tile_of(narrow, t, s), k0 = (jb + j) * kN;
            if (narrow && t == 0 && s > 0 && j + 1 == J) {  // a last odd tile: its V is next to its K
              --vi;
              vs = slot_after<kSlots>(vs, kSlots - 1);
            }
            ok = __all_sync(0xffffffffu, mbar_wait(&sh.s_full[t], (done + s) & 1, &sh.abort_flag, d.status));
            if (!ok) break;
            tc_fence_after();
            // S of this step complete: so is P V of the step before; this chain is done with that V and this K
            release_slot(ks);
            if (s > 0) release_slot(last_vs);
            // the products that read this P also need V and the chain's next K: seen early, they need no wait later
            const int need = (s + 1 < steps ? max(vi, ki + stride) : vi) + 1;
            bool here = static_cast<int>(ld_acquire_shared(&sh.landed) - static_cast<uint32_t>(need)) >= 0;
            __syncwarp();
            if (k0 < full.lo || k0 + kN > full.hi) mask_tile(tS, mine.lo - k0, mine.hi - k0);
            softmax_tile<D>(tS, tO, s == s0, sl2, m_run, l_run);
            if (k0 < cta_lo || k0 + kN > cta_hi) {
              ok = wait_landed(sh, vi + 1, d.status);
              if (!ok) break;
              // the fetched pages' keys before those that all rows see, and behind them
              const int a0 = pages.first(j) * kPage, a1 = min(pages.last(j) * kPage, max(a0, cta_lo - k0));
              const int b1 = pages.last(j) * kPage, b0 = min(b1, max(a1, cta_hi - k0));
              clean_v<D>(sKV + vs * KV_BYTES, a0, a1, b0, b1, w.all_lo - k0, w.all_hi - k0, quarter * 32 + lane,
                         32 * quarters, &sh.dirty);
              fence_proxy_async_smem();
            }
            if (quarter == 0 && !__all_sync(0xffffffffu, here)) {
              ok = wait_landed(sh, need, d.status);
              if (!ok) break;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_n(&sh.p_full[t], quarter == 0 ? 5 - quarters : 1);
            last_vs = vs;
            ki += stride;
            vi += stride;
            ks = slot_after<kSlots>(ks, stride);
            vs = slot_after<kSlots>(vs, stride);
          }
        }
      }
      if (J > 0) {
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&sh.o_full, work & 1, &sh.abort_flag, d.status));
        tc_fence_after();
        if (ok && steps > 0) {
          // every product is done: what this chain has not released yet
          release(item_v(narrow, tile_of(narrow, t, steps - 1), J));
          if (both)
            for (int j = steps; j < J; ++j) {
              release(item_k(false, j));
              release(item_v(false, j, J));
            }
        }
      }
      __syncwarp();
      const bool rows_here = ok && quarter < quarters;
      if (rows_here && steps > kChain) add_totals<D>(tO, totals(), sl2, m_run, l_run);
      if (rows_here && J > 0 && sh.dirty != 0 && steps > 0) {
        // the zeroed elements of v, to the rows that see them
#pragma unroll 1
        for (int s = 0; s < (narrow ? steps : J); ++s) {
          const int k0 = (jb + tile_of(narrow, t, s)) * kN;
          if (k0 >= cta_lo && k0 + kN <= cta_hi) continue;
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld32(tO + c * 32, o);
            tmem_ld_wait();
#pragma unroll 1
            for (int key = max(k0, mine.lo); key < min(k0 + kN, mine.hi); ++key) {
              const int page = w.pt[key / kPage];
              if (page < 0 || page >= a.c.num_pages) continue;
              const __nv_bfloat16* src =
                  d.vpages + ((static_cast<size_t>(page) * d.n_kv_heads + w.g) * kPage + key % kPage) * D + c * 32;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float e = __bfloat162float(src[i]);
                if (!isfinite(e)) o[i] = __float_as_uint(__uint_as_float(o[i]) + e);
              }
            }
            __syncwarp();
            tmem_st32(tO + c * 32, o);
            tmem_st_wait();
          }
        }
      }
      // The stage is free of q: every product is done. Rows of o pass through it in blocks of 32 columns, 128 bytes a
      // row, units swizzled by the row: narrow, a block for each 32 columns, which chain 1 fills for chain 0; wide, two
      // 4 KB blocks a warp in turn. Loops not unrolled: this code runs once a segment, mostly out of the
      // instruction cache.
      const bool second = narrow && n1 > 0, store = R <= last_row;
      uint4* blocks = reinterpret_cast<uint4*>(stage);
      const int warp_at = narrow ? quarter * 256 : (t * 4 + quarter) * 512;             // the warp's rows in a block
      const int block_step = narrow ? T::kStageRows * 8 : 256, block_mask = narrow ? 3 : 1;  // 16-byte units
      if (second) {
        if (t == 1 && rows_here) {
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld32(tO + c * 32, o);
            tmem_ld_wait();
            if (store) {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                blocks[c * block_step + warp_at + lane * 8 + row_unit(r, i)] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
            __syncwarp();
          }
          sh.ml[r] = make_float2(m_run, l_run);
        }
        softmax_groups_sync();
      }
      if (rows_here && !(narrow && t == 1)) {
        float own = 1.f, other = 0.f;
        if (second && store) {
          const float m1 = sh.ml[r].x, l1 = sh.ml[r].y, m = fmaxf(m_run, m1);
          own = m_run == -INFINITY ? 0.f : ex2_approx((m_run - m) * sl2);
          other = m1 == -INFINITY ? 0.f : ex2_approx((m1 - m) * sl2);
          l_run = l_run * own + l1 * other;
          m_run = m;
        }
        const bool whole = w.slot < 0;
        if (whole) {
          const float inv = l_run != 0.f ? 1.0f / l_run : 0.f;
          own *= inv;
          other *= inv;
        }
        const int count = min(32, last_row - (R - lane) + 1);  // the warp's rows
        const int item_row = R - w.q0;
        const int h = w.g * grp + (min(R, last_row) - row * grp);
        // whole rows leave eight at a time, four lanes to 32 columns of each
        __nv_bfloat16* out[4];
        {
          const int64_t mine_at = (row0 + row) * d.out_row + h * d.out_head;
#pragma unroll
          for (int i = 0; i < 4; ++i) out[i] = d.out + __shfl_sync(0xffffffffu, mine_at, i * 8 + lane / 4) + (lane % 4) * 8;
        }
        float* part = a.part + (static_cast<size_t>(max(w.slot, 0)) * (D / 32) * a.part_rows + item_row) * 32;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          if (steps > 0) {
            tmem_ld32(tO + c * 32, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = 0;
          }
          uint4* block = blocks + (c & block_mask) * block_step + warp_at;
          if (!whole && !narrow && c >= 2) {
            // the bulk copy of the block's rows two turns ago has read them
            if (lane == 0) bulk_wait_read<1>();
            __syncwarp();
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (second && store) x = block[lane * 8 + row_unit(r, i)];
            uint32_t* e = &o[4 * i];
            e[0] = __float_as_uint(__uint_as_float(e[0]) * own + __uint_as_float(x.x) * other);
            e[1] = __float_as_uint(__uint_as_float(e[1]) * own + __uint_as_float(x.y) * other);
            e[2] = __float_as_uint(__uint_as_float(e[2]) * own + __uint_as_float(x.z) * other);
            e[3] = __float_as_uint(__uint_as_float(e[3]) * own + __uint_as_float(x.w) * other);
          }
          if (whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t* e = &o[8 * i];
              block[lane * 8 + row_unit(r, i)] =
                  make_uint4(pack_bf16(__uint_as_float(e[0]), __uint_as_float(e[1])), pack_bf16(__uint_as_float(e[2]), __uint_as_float(e[3])),
                             pack_bf16(__uint_as_float(e[4]), __uint_as_float(e[5])), pack_bf16(__uint_as_float(e[6]), __uint_as_float(e[7])));
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int rr = i * 8 + lane / 4;
              if (rr < count) *reinterpret_cast<uint4*>(out[i] + c * 32) = block[rr * 8 + row_unit(rr, lane % 4)];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              block[lane * 8 + row_unit(r, i)] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            // the block leaves as it lies here, one bulk copy (a lane's rows in 16-byte pieces took 13000 cycles a
            // 256-row item)
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              bulk_store(part + static_cast<size_t>(c) * a.part_rows * 32, smem_u32(block), count * 128);
              bulk_commit();
            }
          }
          __syncwarp();
        }
        if (!whole && lane == 0) bulk_wait_read<0>();
        if (!whole) {
          // a sum of 0 marks a part that the row sees nothing of
          if (store)
            reinterpret_cast<float2*>(a.part_ml)[static_cast<size_t>(w.slot) * a.part_rows + item_row] = make_float2(m_run * sl2, l_run);
        } else if (store && d.lse) {
          d.lse[static_cast<size_t>(row0 + row) * d.n_q_heads + h] = l_run == 0.f ? -INFINITY : (m_run * sl2 + log2f(l_run)) * kLn2;
        }
      }
      if (J > 0) {
        base += 2 * J;
        done += steps;
        ++work;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.seg_empty[n % kSegRing]);
    }
    if (lane == 0) bulk_wait_all();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.tmem_free);
  }

  __syncwarp();
  if (warp == 1) {
    // (a failed wait: the softmax warps' own waits have run out by then too)
    volatile int never = 0;
    mbar_wait_warp(&sh.tmem_free, 0, &never, d.status);
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
  __syncthreads();
}

// Joins the parts of cut items, in order of keys. A row of o (of a packed row and kv head) is joined by GROUPS groups of
// D / 4 lanes, which take every GROUPS-th part, 16 bytes of o a lane: one group where the rows fill the SMs, eight
// where they are few and their parts many.
constexpr int kMergeThreads = 256;
template <int D, int GROUPS>
__global__ void __launch_bounds__(kMergeThreads) chunk_attn_merge(const __grid_constant__ MergeArgs a) {
  constexpr int kLanes = D / 4, kRows = kMergeThreads / (kLanes * GROUPS);
  __shared__ float4 red_o[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? kRows * kLanes : 1];
  __shared__ float2 red_ml[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? kRows : 1];
  griddep_launch_dependents();
  const ChunkAttnDesc& d = a.d;
  const int c = threadIdx.x % kLanes, q = threadIdx.x / kLanes % GROUPS, rr = threadIdx.x / (kLanes * GROUPS);
  const int b = min(static_cast<int>(blockIdx.x) * kRows + rr, a.rows[a.cuts] - 1);  // a last block's spare rows repeat the last
  int lo = 0, hi = a.cuts - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.rows[mid] <= b) lo = mid; else hi = mid - 1;
  }
  const CutItem& it = a.cut[lo];
  const int r = b - a.rows[lo], parts = it.parts;
  // column 4 c of the row: block of 32 columns, and unit of it as the row swizzles them
  const size_t at = (static_cast<size_t>(c / 8) * a.part_rows + r) * 8 + row_unit(r, c % 8);
  griddep_wait();
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kBatch = 4;
  for (int k0 = q; k0 < parts; k0 += kBatch * GROUPS) {
    float2 ml[kBatch];
    float4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int k = k0 + i * GROUPS;
      ml[i] = make_float2(-INFINITY, 0.f);
      if (k < parts) {
        const size_t slot = k == 0 ? it.first_slot : 2 * (it.cta + k);
        ml[i] = __ldcg(reinterpret_cast<const float2*>(a.part_ml) + slot * a.part_rows + r);
        v[i] = __ldcg(reinterpret_cast<const float4*>(a.part) + slot * a.part_rows * (D / 4) + at);
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
  const int grp = d.n_q_heads / d.n_kv_heads, R = it.q0 + r, row = it.row0 + R / grp, h = it.g * grp + R % grp;
  *reinterpret_cast<uint2*>(d.out + row * d.out_row + h * d.out_head + c * 4) =
      make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  if (d.lse && c == 0) d.lse[static_cast<size_t>(row) * d.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ---------------------------------------------------------------- plan (host)
// What runs are dealt by, in units of a wide step's time. A narrow step reads two tiles; a segment costs something beside
// its steps (q, the masks, the end): 8192 rows from nothing took 427 us with 4 units, 369 with 6, 370 with 8, 377 with 10;
// 64 single rows over 2000 keys 60 us with 2 or 4, 55 with 6.
constexpr int kSegment = 6;
inline int step_units(bool narrow) { return narrow ? 2 : 1; }
// The merge's launch and run.
constexpr int kMerge = 2;

// Deals the items' steps to at most `ctas` runs of at most `budget` units each; false if they do not fit. `whole`:
// an item a run.
bool deal(const ChunkTable& c, int n_q_heads, int n_kv_heads, bool causal, int window, int ctas, int64_t budget, bool whole,
          ChunkPlan* p) {
  const int grp = n_q_heads / n_kv_heads;
  p->ctas = 0;
  p->part_rows = p->cuts = p->merge_rows = p->longest = 0;
  int64_t left = 0;     // of the current CTA's budget
  int here = 0;         // segments of the current CTA
  auto open = [&](int req, int qt, int g, int step) {
    p->run[p->ctas++] = RunStart{req, qt, g, step};
    left = budget;
    here = 0;
  };
  for (int i = 0; i < c.n; ++i) {
    const int rows = (c.row0[i + 1] - c.row0[i]) * grp;
    if (rows == 0) continue;
    const bool narrow = narrow_form(rows);
    const int unit = step_units(narrow), tile = narrow ? kM : 2 * kM, tiles = (rows + tile - 1) / tile;
    for (int qt = tiles - 1; qt >= 0; --qt) {
      const int q0 = qt * tile, q1 = std::min(q0 + tile, rows) - 1;
      const int steps = tiles_of(keys_of_rows(c.pos[i] + q0 / grp, c.pos[i] + q1 / grp, c.n_keys[i], causal, window), narrow).steps;
      for (int g = 0; g < n_kv_heads; ++g) {
        int step = 0, first_cta = -1, first_slot = 0, parts = 0;
        do {
          // a segment of at least one step (or the whole of an empty item) starts only where it fits the budget
          if (p->ctas == 0 || whole || left < kSegment + std::min(steps - step, 1) * unit) {
            if (p->ctas == ctas) return false;
            open(i, qt, g, step);
          }
          left -= kSegment;
          const int take = whole ? steps : static_cast<int>(std::min<int64_t>(steps - step, left / unit));
          p->longest = std::max(p->longest, take);
          if (parts++ == 0) {
            first_cta = p->ctas - 1;
            first_slot = 2 * first_cta + (here > 0 ? 1 : 0);
          }
          ++here;
          left -= take * unit;
          step += take;
        } while (step < steps);
        if (parts > 1) {
          p->rows[p->cuts] = p->merge_rows;
          p->cut[p->cuts++] = CutItem{c.row0[i], q0, g, first_slot, first_cta, parts};
          p->merge_rows += q1 - q0 + 1;
          p->part_rows = std::max(p->part_rows, q1 - q0 + 1);
        }
      }
    }
  }
  p->run[p->ctas] = RunStart{c.n, 0, 0, 0};
  p->rows[p->cuts] = p->merge_rows;
  return true;
}

}  // namespace

void plan_chunk_attention(const ChunkTable& c, int n_q_heads, int n_kv_heads, bool causal, int window, int num_sms, ChunkPlan* p) {
  const int grp = n_q_heads / n_kv_heads, ctas = std::min(num_sms, kMaxCtas);
  int64_t total = 0, items = 0;
  int longest = 0, least = 1;  // units of the longest item's steps, of a segment of one step
  for (int i = 0; i < c.n; ++i) {
    const int rows = (c.row0[i + 1] - c.row0[i]) * grp;
    if (rows == 0) continue;
    const bool narrow = narrow_form(rows);
    const int unit = step_units(narrow), tile = narrow ? kM : 2 * kM;
    least = std::max(least, kSegment + unit);
    for (int q0 = 0; q0 < rows; q0 += tile) {
      const int q1 = std::min(q0 + tile, rows) - 1;
      const int steps = tiles_of(keys_of_rows(c.pos[i] + q0 / grp, c.pos[i] + q1 / grp, c.n_keys[i], causal, window), narrow).steps;
      total += static_cast<int64_t>(n_kv_heads) * (steps * unit + kSegment);
      items += n_kv_heads;
      longest = std::max(longest, steps * unit);
    }
  }
  // An even share at first; runs that end early for want of a whole step, and the segments that they continue, need some
  // more. Few short items stay whole: the merge costs more than the steps that it saves.
  int64_t budget = std::max<int64_t>(least, (total + ctas - 1) / ctas);
  const bool whole = items <= ctas && longest <= budget - kSegment + kMerge;
  if (items > 2 * ctas) budget += kSegment;  // nearly every run continues a segment: fewer tries
  for (int tries = 0;; ++tries) {
    if (deal(c, n_q_heads, n_kv_heads, causal, window, ctas, budget, whole, p)) return;
    budget += tries < 12 ? 1 : budget / 8 + 1;
  }
}

namespace {

template <int D, bool LEAN>
cudaError_t launch_tc(const ChunkArgs& a, const ChunkPlan& p, int num_sms, cudaStream_t stream) {
  static PerDevice once;
  int dev = 0;
  if (once.pending(&dev)) {
    cudaError_t e = cudaFuncSetAttribute(chunk_attn_kernel<D, LEAN>, cudaFuncAttributeMaxDynamicSharedMemorySize, Tile<D, LEAN>::kSmem);
    if (e != cudaSuccess) return e;
    // setmaxnreg.inc waits until the CTA's register pool can serve it: refuse to launch a build whose launch
    // count leaves the split short
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, chunk_attn_kernel<D, LEAN>);
    if (e != cudaSuccess) return e;
    if (fa.numRegs * kThreads < kRegsNeeded) return cudaErrorInvalidConfiguration;
    once.done(dev);
  }
  PdlScope pdl;
  cudaError_t e = launch_kernel(chunk_attn_kernel<D, LEAN>, dim3(p.ctas), dim3(kThreads), Tile<D, LEAN>::kSmem, stream, a);
  if (e != cudaSuccess || p.cuts == 0) return e;
  MergeArgs m;
  std::memset(&m, 0, sizeof(m));
  m.d = a.d;
  m.part = a.part;
  m.part_ml = a.part_ml;
  m.part_rows = a.part_rows;
  m.cuts = p.cuts;
  std::memcpy(m.rows, p.rows, (p.cuts + 1) * sizeof(int));
  std::memcpy(m.cut, p.cut, p.cuts * sizeof(CutItem));
  constexpr int kRow = kMergeThreads / (D / 4);  // rows a block with one group each
  if (p.merge_rows < 4 * kRow * num_sms) {
    constexpr int kRows8 = kRow / 8;
    return launch_kernel(chunk_attn_merge<D, 8>, dim3((p.merge_rows + kRows8 - 1) / kRows8), dim3(kMergeThreads), 0, stream, m);
  }
  return launch_kernel(chunk_attn_merge<D, 1>, dim3((p.merge_rows + kRow - 1) / kRow), dim3(kMergeThreads), 0, stream, m);
}

size_t part_floats(const ChunkPlan& p, int head_dim, bool ml) {
  if (p.cuts == 0) return 0;
  return (static_cast<size_t>(2 * p.ctas) * p.part_rows * (ml ? 2 : head_dim) + 63) & ~static_cast<size_t>(63);
}
size_t total_floats(const ChunkPlan& p, int head_dim) {
  return p.longest > kChain ? static_cast<size_t>(2 * p.ctas) * (head_dim + 2) * kM : 0;
}

}  // namespace

size_t chunk_attention_workspace(const ChunkPlan& p, int head_dim) {
  return (part_floats(p, head_dim, false) + part_floats(p, head_dim, true) + total_floats(p, head_dim)) * sizeof(float);
}

cudaError_t launch_chunk_attention(const ChunkAttnDesc& d, const ChunkTable& c, const ChunkPlan& p, void* workspace,
                                   int num_sms, cudaStream_t stream) {
  if (p.ctas == 0) return cudaSuccess;
  ChunkArgs a;
  const long pool_rows = static_cast<long>(c.num_pages) * d.n_kv_heads * kPage;
  if (!tensor_map_pool(&a.tmK, d.kpages, pool_rows, d.head_dim) || !tensor_map_pool(&a.tmV, d.vpages, pool_rows, d.head_dim))
    return cudaErrorInvalidValue;
  a.d = d;
  a.c = c;
  std::memcpy(a.run, p.run, (p.ctas + 1) * sizeof(RunStart));
  a.part = static_cast<float*>(workspace);
  a.part_ml = a.part + part_floats(p, d.head_dim, false);
  a.part_rows = p.part_rows;
  a.total = a.part_ml + part_floats(p, d.head_dim, true);
  bool lean = true;
  for (int i = 0; i < c.n; ++i) lean = lean && static_cast<int64_t>(c.row0[i + 1] - c.row0[i]) * (d.n_q_heads / d.n_kv_heads) <= kLeanRows;
  if (d.head_dim == 128) return lean ? launch_tc<128, true>(a, p, num_sms, stream) : launch_tc<128, false>(a, p, num_sms, stream);
  return lean ? launch_tc<64, true>(a, p, num_sms, stream) : launch_tc<64, false>(a, p, num_sms, stream);
}

}  // namespace crf
