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
// A step of the pair of chains is one K/V tile (wide) or two (narrow). Where the items (request, kv head,
// query tiles) would leave SMs idle, each one's keys are cut into pieces of equally many steps; a piece writes its
// unnormalised o, maximum and sum in fp32 to the workspace and chunk_attn_merge joins them in order of keys.
//
// Warp roles, TMEM and the ring follow the prefill attention (attention_tc.cu): warp 0 gathers the pages of K and V
// tiles with TMA, warp 1 issues the MMAs, warps 4-7 and 8-11 are the chains' softmax (one packed row a thread,
// P back into TMEM as bf16, o rescaled there when the maximum grows by more than 2^8). Here the softmax warps also
// bring q into shared memory (rows of any strides, packed heads), and warps whose 32 rows are all padding do nothing.
//
// Unseen slots may hold anything: pages that no row of the CTA sees are not fetched; scores of unseen keys
// become -inf whatever they were; v of keys that no row sees is zeroed, and in tiles that only some rows see an
// infinite or NaN element of v is zeroed and given back, at the end, to the rows that see it (0 times infinity
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
// setmaxnreg split: the first warpgroup (producer, issuer) keeps kRegsCtl, the softmax warpgroups take
// kRegsSoftmax; the sum must fit what the CTA launched with.
constexpr int kRegsCtl = 80;
constexpr int kRegsSoftmax = 208;
constexpr int kRegsNeeded = 128 * kRegsCtl + 256 * kRegsSoftmax;
constexpr uint32_t kTmemCols = 512;  // S0 | S1 | O0 | O1, 128 each
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// How a call's work is cut. Items of request i: [item0[i], item0[i + 1]), longest first: query tile (or pair)
// from the last down, kv head, piece of `piece_steps` steps.
struct ChunkPlan {
  int item0[kMaxChunks + 1];
  int pieces[kMaxChunks];  // of each (query tile, head); 1: written straight to out
  int piece_steps;
  int split_rows[kMaxChunks + 1];  // packed rows x kv heads of split requests, prefix: the merge's rows
};

struct ChunkArgs {
  CUtensorMap tmK, tmV;  // pages of the layer, box: one page of one kv head
  ChunkAttnDesc d;
  ChunkTable c;
  ChunkPlan p;
  float* part;  // split items: [item][rows of an item][D] o, then [item][rows][2] maximum and sum
  float* part_ml;
  int part_rows;
};

__host__ __device__ inline bool narrow_form(int packed_rows) { return packed_rows <= kM; }

// Keys [lo, hi) that the rows a .. b (positions) of a request see in all; empty if hi <= lo.
struct KeyRange {
  int lo, hi;
};
__host__ __device__ inline KeyRange keys_of_rows(int first_pos, int last_pos, int n_keys, bool causal, int window) {
  KeyRange k;
  k.lo = window > 0 && first_pos + 1 > window ? first_pos + 1 - window : 0;
  k.hi = causal && last_pos + 1 < n_keys ? last_pos + 1 : n_keys;
  return k;
}

__device__ __forceinline__ void regs_dec_ctl() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsCtl)); }
__device__ __forceinline__ void regs_inc_softmax() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
}
__device__ __forceinline__ void softmax_groups_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

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

__device__ __forceinline__ bool not_finite_bf16(uint32_t h) { return (h & 0x7F80u) == 0x7F80u; }

template <int D>
struct Tile {
  static constexpr int HALVES = D / 64;
  static constexpr int Q_BYTES = kM * D * 2;
  static constexpr int KV_BYTES = kN * D * 2;
  static constexpr int HALF_ROWS_BYTES = kN * 128;    // one 64-column half of a query tile
  static constexpr int GROUP_BYTES = HALVES * 1024;   // 8 keys, all halves, in a K/V slot
  static constexpr int kSmem = 2 * Q_BYTES + 5 * KV_BYTES + 1024;  // wide: 2 q tiles, 5 slots; narrow: 1 and 6
};

// Where an element of a K/V slot lies: key, 16-byte unit of the head.
template <int D>
__device__ __forceinline__ uint4* slot_unit(uint8_t* slot, int key, int unit) {
  using T = Tile<D>;
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

// An item and the part of its keys that the CTA reads, found by one thread.
struct Item {
  int g, q0, rows;      // kv head; the item's first packed row; packed rows of the request
  int pos, n_keys, row0;
  const int32_t* pt;
  bool narrow, split;
  int all_lo, all_hi;   // keys that some row sees
  KeyRange full0, full1;  // keys that all rows of a chain see
  int jb, J;            // K/V tiles of the piece; every one holds a key that some row sees
  int n0, n1;           // steps of the chains
  int quarters0, quarters1;  // warps of a chain with rows
};

struct Shared {
  uint64_t q_full, o_full, drain;
  uint64_t kv_full[6], kv_empty[6];
  uint64_t s_full[2], p_full[2];
  Item w;
  uint32_t tmem_base;
  volatile int abort_flag;
  volatile int dirty;  // an infinite or NaN element of v was zeroed
};

__device__ __forceinline__ void find_item(const ChunkArgs& a, int idx, Item& w) {
  int i = 0, top = a.c.n - 1;
  while (i < top) {
    const int mid = (i + top + 1) >> 1;
    if (a.p.item0[mid] <= idx) i = mid; else top = mid - 1;
  }
  const int grp = a.d.n_q_heads / a.d.n_kv_heads, pieces = a.p.pieces[i];
  const int rows = (a.c.row0[i + 1] - a.c.row0[i]) * grp;
  const bool narrow = narrow_form(rows);
  const int tile = narrow ? kM : 2 * kM, tiles = (rows + tile - 1) / tile;
  idx -= a.p.item0[i];
  const int qt = idx / (a.d.n_kv_heads * pieces);
  idx -= qt * a.d.n_kv_heads * pieces;
  const int g = idx / pieces, piece = idx - g * pieces;
  const int q0 = (tiles - 1 - qt) * tile;
  w.g = g;
  w.q0 = q0;
  w.rows = rows;
  w.pos = a.c.pos[i];
  w.n_keys = a.c.n_keys[i];
  w.row0 = a.c.row0[i];
  w.pt = a.c.pt[i];
  w.narrow = narrow;
  w.split = pieces > 1;
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
  w.all_lo = some[0].lo;
  w.all_hi = max(some[0].hi, some[1].hi);
  w.full0 = full[0];
  w.full1 = full[1];
  const int jfirst = w.all_lo / kN, jend = w.all_hi > w.all_lo ? (w.all_hi + kN - 1) / kN : jfirst;
  const int per_piece = a.p.piece_steps * (narrow ? 2 : 1);
  w.jb = static_cast<int>(min(static_cast<int64_t>(jend), jfirst + static_cast<int64_t>(piece) * per_piece));
  w.J = min(jend - w.jb, per_piece);
  w.n0 = narrow ? (w.J + 1) / 2 : min(w.J, max(0, (some[0].hi + kN - 1) / kN - w.jb));
  w.n1 = narrow ? w.J / 2 : min(w.J, max(0, (some[1].hi + kN - 1) / kN - w.jb));
  w.quarters0 = (valid[0] + 31) / 32;
  w.quarters1 = (valid[1] + 31) / 32;
}

template <int D, bool NARROW>
__device__ __forceinline__ void attn_body(const ChunkArgs& a, uint8_t* smem, Shared& sh) {
  using T = Tile<D>;
  constexpr int Q_BYTES = T::Q_BYTES, KV_BYTES = T::KV_BYTES, GROUP_BYTES = T::GROUP_BYTES;
  constexpr int kSlots = NARROW ? 6 : 5;
  constexpr int kTiles = NARROW ? 1 : 2;  // query tiles of the item
  const ChunkAttnDesc& d = a.d;
  const Item& w = sh.w;
  uint8_t* sQ = smem;
  uint8_t* sKV = sQ + kTiles * Q_BYTES;
  const int J = w.J, jb = w.jb, n0 = w.n0, n1 = w.n1;
  auto tile_of = [&](int t, int s) { return NARROW ? 2 * s + t : s; };
  // The ring's sequence: K0 V0 K1 V1 ... (wide), K0 K1 V0 V1 K2 K3 ... (narrow: both chains start early; a last
  // odd tile alone)
  auto item_k = [&](int j) { return NARROW ? 4 * (j >> 1) + (j & 1) : 2 * j; };
  auto item_v = [&](int j) { return NARROW ? 4 * (j >> 1) + (j + 1 == J && (j & 1) == 0 ? 1 : 2 + (j & 1)) : 2 * j + 1; };
  // pages [first, last) of tile j that some row sees
  auto first_page = [&](int j) { return max(0, w.all_lo / kPage - (jb + j) * kPagesPerTile); };
  auto last_page = [&](int j) { return min(kPagesPerTile, (w.all_hi + kPage - 1) / kPage - (jb + j) * kPagesPerTile); };
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);  // uniform
  const int lane = threadIdx.x & 31;
  const uint32_t tmem = sh.tmem_base;

  if (warp < 4) {
    regs_dec_ctl();
    if (warp == 0) {
      // ---------------------------------------------------------------- producer
      const bool issuer = elect_one();
      bool ok = true;
      int armed = 0, slot = 0;
      uint32_t ph = 0;
      const int32_t* pt = w.pt;
      auto page_id = [&](int j) {
        const int p = lane & (kPagesPerTile - 1);
        int id = 0;
        if (p >= first_page(j) && p < last_page(j)) {
          id = pt[(jb + j) * kPagesPerTile + p];
          if (id < 0 || id >= a.c.num_pages) {
            if (d.status) atomicOr(d.status, kStatusBounds);
            id = 0;
          }
        }
        return id;
      };
      constexpr int kGroup = NARROW ? 2 : 1;  // tiles whose K come before their V
      int ids[kGroup], next_ids[kGroup];
#pragma unroll
      for (int i = 0; i < kGroup; ++i) ids[i] = i < J ? page_id(i) : 0;
      for (int j0 = 0; j0 < J && ok; j0 += kGroup) {
#pragma unroll
        for (int i = 0; i < kGroup; ++i) next_ids[i] = j0 + kGroup + i < J ? page_id(j0 + kGroup + i) : 0;
#pragma unroll
        for (int x = 0; x < 2 * kGroup; ++x) {
          const int i = x % kGroup, j = j0 + i, kv = x / kGroup;
          if (!ok || j >= J) continue;
          ok = mbar_wait_warp(&sh.kv_empty[slot], ph ^ 1, &sh.abort_flag, d.status);
          if (!ok) continue;
          const int pg0 = first_page(j), pg1 = last_page(j);
          if (issuer) mbar_arrive_expect_tx(&sh.kv_full[slot], (pg1 - pg0) * (kPage / 8) * GROUP_BYTES);
          uint8_t* dst = sKV + slot * KV_BYTES;
          const CUtensorMap* map = kv == 0 ? &a.tmK : &a.tmV;
#pragma unroll
          for (int p = 0; p < kPagesPerTile; ++p) {
            const int group = (__shfl_sync(0xffffffffu, ids[i], p) * d.n_kv_heads + w.g) * (kPage / 8);
            if (issuer && p >= pg0 && p < pg1)
              tma_load_4d(dst + p * (kPage / 8) * GROUP_BYTES, map, &sh.kv_full[slot], 0, 0, 0, group);
          }
          ++armed;
          if (++slot == kSlots) {
            slot = 0;
            ph ^= 1;
          }
        }
#pragma unroll
        for (int i = 0; i < kGroup; ++i) ids[i] = next_ids[i];
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
      bool ok = J == 0 || mbar_wait_warp(&sh.q_full, 0, &sh.abort_flag, d.status);
      bool issued = false;
      const uint32_t idesc_s = idesc_bf16_f32(kM, kN);
      const uint32_t idesc_o = idesc_bf16_f32(kM, D, false, true);
      const uint64_t qd = smem_desc(smem_u32(sQ), 16, 1024, kSwizzle128B);
      const uint64_t kd = smem_desc(smem_u32(sKV), 16, GROUP_BYTES, kSwizzle128B);
      const uint64_t vd = smem_desc(smem_u32(sKV), 1024, GROUP_BYTES, kSwizzle128B);
      auto issue_s = [&](int t, int slot) {
        const uint64_t q = qd + static_cast<uint32_t>((NARROW ? 0 : t) * (Q_BYTES >> 4));
        const uint64_t k = kd + static_cast<uint32_t>(slot * (KV_BYTES >> 4));
        if (issuer) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            mma_bf16_ss(tmem + t * 128, q + (kk >> 2) * (T::HALF_ROWS_BYTES >> 4) + (kk & 3) * 2,
                        k + (kk >> 2) * 64 + (kk & 3) * 2, idesc_s, kk > 0 ? 1u : 0u);
          mma_commit(&sh.s_full[t]);
        }
      };
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (!ok || (t ? n1 : n0) == 0) continue;
        const int item = item_k(tile_of(t, 0));
        ok = mbar_wait_warp(&sh.kv_full[item % kSlots], (item / kSlots) & 1, &sh.abort_flag, d.status);
        if (!ok) continue;
        tc_fence_after();
        issue_s(t, item % kSlots);
        issued = true;
      }
      const int most = max(n0, n1);
      for (int s = 0; s < most && ok; ++s) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (!ok || s >= (t ? n1 : n0)) continue;
          // P of this step is in TMEM, and its V and the chain's next K have landed
          ok = mbar_wait_warp(&sh.p_full[t], s & 1, &sh.abort_flag, d.status);
          if (!ok) continue;
          tc_fence_after();
          const int j = tile_of(t, s), pg0 = first_page(j), pg1 = last_page(j);
          const uint64_t v = vd + static_cast<uint32_t>((item_v(j) % kSlots) * (KV_BYTES >> 4));
          if (issuer) {
            // 16 keys, one page, an MMA: pages that no row sees are left out
#pragma unroll
            for (int kk = 0; kk < kN / 16; ++kk)
              if (kk >= pg0 && kk < pg1)
                mma_bf16_ts(tmem + 256 + t * 128, tmem + t * 128 + kk * 8, v + kk * (2 * GROUP_BYTES >> 4), idesc_o,
                            (s > 0 || kk > pg0) ? 1u : 0u);
          }
          if (s + 1 < (t ? n1 : n0)) issue_s(t, item_k(tile_of(t, s + 1)) % kSlots);
        }
      }
      if (ok) {
        if (issuer) mma_commit(&sh.o_full);
      } else if (issued && issuer) {
        mma_commit(&sh.drain);
        volatile int never = 0;
        mbar_wait(&sh.drain, 0, &never, nullptr);
      }
    }
  } else {
    regs_inc_softmax();
    // ---------------------------------------------------------------- q, softmax, epilogue
    const int t = (warp - 4) >> 2, tid = threadIdx.x - 128;
    const int quarter = warp & 3;
    const int steps = t ? n1 : n0, quarters = t ? w.quarters1 : w.quarters0;
    const int grp = d.n_q_heads / d.n_kv_heads, last_row = w.rows - 1, row0 = w.row0;
    const int r = quarter * 32 + lane;  // row of the query tile (= TMEM lane)
    {
      // q: 16-byte units of a row side by side in a warp; rows behind the request's last are zeros
      constexpr int kUnits = D / 8, kStep = 256 / kUnits, kTurns = kTiles * kM / kStep;
      const int u = tid % kUnits;
      int row = (w.q0 + tid / kUnits) / grp, h = w.q0 + tid / kUnits - row * grp;
      const int row_step = kStep / grp, h_step = kStep - row_step * grp;
      uint4 v[kTurns];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        v[i] = make_uint4(0, 0, 0, 0);
        if (w.q0 + tid / kUnits + i * kStep <= last_row)
          v[i] = *reinterpret_cast<const uint4*>(d.q + (row0 + row) * d.q_row + (w.g * grp + h) * d.q_head + u * 8);
        row += row_step;
        h += h_step;
        if (h >= grp) {
          h -= grp;
          ++row;
        }
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int at = tid / kUnits + i * kStep, rr = at & (kM - 1);
        *reinterpret_cast<uint4*>(sQ + (at / kM) * Q_BYTES + (u >> 3) * T::HALF_ROWS_BYTES + rr * 128 +
                                  (((u & 7) ^ (rr & 7)) << 4)) = v[i];
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.q_full);
    }
    const uint32_t lane_off = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t tO = tmem + lane_off + 256 + t * 128;
    const float sl2 = kLog2e * d.scale;
    const int R = w.q0 + (NARROW ? 0 : t * kM) + r;  // packed row
    const int row = min(R, last_row) / grp, p = w.pos + row;
    const KeyRange mine = keys_of_rows(p, p, w.n_keys, d.causal, d.window);
    float m_run = -INFINITY, l_run = 0.f;  // maximum in raw score units
    bool ok = true;
    const KeyRange full = t ? w.full1 : w.full0;  // keys that all rows of the chain see, and of the CTA
    const bool both = !NARROW && n1 > 0 && n0 > 0;
    const int cta_lo = both ? max(w.full0.lo, w.full1.lo) : full.lo;
    const int cta_hi = both ? min(w.full0.hi, w.full1.hi) : full.hi;
    if (quarter < quarters) {
      const uint32_t tS = tmem + lane_off + t * 128;
      for (int s = 0; s < steps && ok; ++s) {
        const int j = tile_of(t, s), k0 = (jb + j) * kN;
        ok = __all_sync(0xffffffffu, mbar_wait(&sh.s_full[t], s & 1, &sh.abort_flag, d.status));
        if (!ok) break;
        tc_fence_after();
        // S of this step complete: so is P V of the step before; this chain is done with that V and this K
        if (quarter == 0 && lane == 0) {
          mbar_arrive(&sh.kv_empty[item_k(j) % kSlots]);
          if (s > 0) mbar_arrive(&sh.kv_empty[item_v(tile_of(t, s - 1)) % kSlots]);
        }
        if (k0 < full.lo || k0 + kN > full.hi) mask_tile(tS, mine.lo - k0, mine.hi - k0);
        softmax_tile<D>(tS, tO, s == 0, sl2, m_run, l_run);
        const int vi = item_v(j);
        if (k0 < cta_lo || k0 + kN > cta_hi) {
          ok = __all_sync(0xffffffffu, mbar_wait(&sh.kv_full[vi % kSlots], (vi / kSlots) & 1, &sh.abort_flag, d.status));
          if (!ok) break;
          // the fetched pages' keys before those that all rows see, and behind them
          const int a0 = first_page(j) * kPage, a1 = min(last_page(j) * kPage, max(a0, cta_lo - k0));
          const int b1 = last_page(j) * kPage, b0 = min(b1, max(a1, cta_hi - k0));
          clean_v<D>(sKV + (vi % kSlots) * KV_BYTES, a0, a1, b0, b1, w.all_lo - k0, w.all_hi - k0, quarter * 32 + lane,
                     32 * quarters, &sh.dirty);
          fence_proxy_async_smem();
        }
        if (quarter == 0) {
          // the products that read this P also need V and the chain's next K: hand over once they have landed
          ok = __all_sync(0xffffffffu, mbar_wait(&sh.kv_full[vi % kSlots], (vi / kSlots) & 1, &sh.abort_flag, d.status));
          if (ok && s + 1 < steps) {
            const int ki = item_k(tile_of(t, s + 1));
            ok = __all_sync(0xffffffffu, mbar_wait(&sh.kv_full[ki % kSlots], (ki / kSlots) & 1, &sh.abort_flag, d.status));
          }
          if (!ok) break;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[t]);
      }
    }
    if (ok && J > 0) ok = __all_sync(0xffffffffu, mbar_wait(&sh.o_full, 0, &sh.abort_flag, d.status));
    tc_fence_after();
    const bool rows_here = ok && quarter < quarters;
    if (rows_here && sh.dirty != 0) {
      // the zeroed elements of v, to the rows that see them
#pragma unroll 1
      for (int s = 0; s < (NARROW ? steps : J) && steps > 0; ++s) {
        const int k0 = (jb + tile_of(t, s)) * kN;
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
    // The ring is free: every product is done. Rows of o pass through it, 16-byte units swizzled by the row.
    constexpr int kRowUnits = D / 4;  // of an fp32 row
    float4* xo = reinterpret_cast<float4*>(sKV);                  // narrow: chain 1's rows
    float2* xml = reinterpret_cast<float2*>(xo + kM * kRowUnits);  // and maxima and sums
    const bool second = NARROW && n1 > 0;
    auto unit_of = [&](int rr, int u, int units) { return rr * units + (u ^ (rr & (units - 1))); };
    // Loops of 32 columns, not unrolled: this code runs once a CTA, mostly out of the instruction cache (as straight
    // code for 128 columns it took an item of few rows 1500 cycles longer).
    if (second) {
      if (t == 1 && rows_here) {
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          tmem_ld32(tO + c * 32, o);
          tmem_ld_wait();
          if (R <= last_row) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              xo[unit_of(r, c * 8 + i, kRowUnits)] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                                 __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
          }
          __syncwarp();
        }
        xml[r] = make_float2(m_run, l_run);
      }
      softmax_groups_sync();
    }
    if (rows_here && !(NARROW && t == 1)) {
      const bool store = R <= last_row;
      float own = 1.f, other = 0.f;
      if (second && store) {
        const float m1 = xml[r].x, l1 = xml[r].y, m = fmaxf(m_run, m1);
        own = m_run == -INFINITY ? 0.f : ex2_approx((m_run - m) * sl2);
        other = m1 == -INFINITY ? 0.f : ex2_approx((m1 - m) * sl2);
        l_run = l_run * own + l1 * other;
        m_run = m;
      }
      if (!w.split) {
        const float inv = l_run != 0.f ? 1.0f / l_run : 0.f;
        own *= inv;
        other *= inv;
      }
      // behind chain 1's rows; wide: one 128-row block a chain
      uint8_t* stage = sKV + (NARROW ? kM * kRowUnits * 16 + kM * 8 : t * kM * kRowUnits * 16);
      uint4* rows = reinterpret_cast<uint4*>(stage);
      constexpr int kOutUnits = D / 8;  // of a bf16 row
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
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          if (second && store) x = xo[unit_of(r, c * 8 + i, kRowUnits)];
          uint32_t* e = &o[4 * i];
          e[0] = __float_as_uint(__uint_as_float(e[0]) * own + x.x * other);
          e[1] = __float_as_uint(__uint_as_float(e[1]) * own + x.y * other);
          e[2] = __float_as_uint(__uint_as_float(e[2]) * own + x.z * other);
          e[3] = __float_as_uint(__uint_as_float(e[3]) * own + x.w * other);
        }
        if (w.split) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            rows[unit_of(r, c * 8 + i, kRowUnits)] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t* e = &o[8 * i];
            rows[unit_of(r, c * 4 + i, kOutUnits)] =
                make_uint4(pack_bf16(__uint_as_float(e[0]), __uint_as_float(e[1])), pack_bf16(__uint_as_float(e[2]), __uint_as_float(e[3])),
                           pack_bf16(__uint_as_float(e[4]), __uint_as_float(e[5])), pack_bf16(__uint_as_float(e[6]), __uint_as_float(e[7])));
          }
        }
        __syncwarp();
      }
      const int h = w.g * grp + (min(R, last_row) - row * grp);
      const size_t pr = static_cast<size_t>(blockIdx.x) * a.part_rows + (R - w.q0);
      const int first = quarter * 32, count = min(32, last_row - (R - lane) + 1);  // the warp's rows
      if (w.split) {
        // fp32 rows as they lie here, one bulk copy a warp: 512-byte rows a lane in 16-byte pieces took 13000 cycles a
        // 256-row item
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          bulk_store(a.part + pr * D, smem_u32(rows + first * kRowUnits), count * kRowUnits * 16);
          bulk_commit();
        }
      } else {
        // whole rows side by side
        const int64_t mine_at = (row0 + row) * d.out_row + h * d.out_head;
#pragma unroll 1
        for (int i0 = 0; i0 < count; i0 += 32 / kOutUnits) {
          const int i = i0 + lane / kOutUnits, u = lane % kOutUnits;
          const int64_t at = __shfl_sync(0xffffffffu, mine_at, i);
          if (i < count) *reinterpret_cast<uint4*>(d.out + at + u * 8) = rows[unit_of(first + i, u, kOutUnits)];
        }
      }
      if (store) {
        if (w.split) {
          // a sum of 0 marks a piece that the row sees nothing of
          reinterpret_cast<float2*>(a.part_ml)[pr] = make_float2(m_run * sl2, l_run);
        } else if (d.lse) {
          d.lse[static_cast<size_t>(row0 + row) * d.n_q_heads + h] =
              l_run == 0.f ? -INFINITY : (m_run * sl2 + log2f(l_run)) * kLn2;
        }
      }
      if (w.split && lane == 0) bulk_wait_all();
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) chunk_attn_kernel(const __grid_constant__ ChunkArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) Shared sh;
  griddep_launch_dependents();
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  if (threadIdx.x / 32 == 1) {
    tmem_alloc(&sh.tmem_base, kTmemCols);
    tmem_relinquish();
  } else if (threadIdx.x == 64) {
    Item w;
    find_item(a, blockIdx.x, w);
    sh.w = w;
    mbar_init(&sh.q_full, 8);
    mbar_init(&sh.o_full, 1);
    mbar_init(&sh.drain, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&sh.s_full[t], 1);
      mbar_init(&sh.p_full[t], max(1, t ? w.quarters1 : w.quarters0));
    }
    // a ring slot is free once every chain that reads it has released it
    const int readers = w.narrow ? 1 : max(1, (w.n0 > 0) + (w.n1 > 0));
    for (int i = 0; i < 6; ++i) {
      mbar_init(&sh.kv_full[i], 1);
      mbar_init(&sh.kv_empty[i], readers);
    }
    sh.abort_flag = 0;
    sh.dirty = 0;
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_wait();  // q, the pages and their tables may come from the kernel before
  if (sh.w.narrow)
    attn_body<D, true>(a, smem, sh);
  else
    attn_body<D, false>(a, smem, sh);
}

// Joins the pieces of split items, in order of keys. A row of o (of a packed row and kv head of a split request) is
// joined by GROUPS groups of D / 4 lanes, which take every GROUPS-th piece, 16 bytes of o a lane: one group where
// the rows fill the SMs, eight where they are few and their pieces many.
constexpr int kMergeThreads = 256;
template <int D, int GROUPS>
__global__ void __launch_bounds__(kMergeThreads) chunk_attn_merge(const __grid_constant__ ChunkArgs a, int total) {
  constexpr int kLanes = D / 4, kRows = kMergeThreads / (kLanes * GROUPS);
  __shared__ float4 red_o[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? kRows * kLanes : 1];
  __shared__ float2 red_ml[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? kRows : 1];
  griddep_launch_dependents();
  const ChunkAttnDesc& d = a.d;
  const int c = threadIdx.x % kLanes, q = threadIdx.x / kLanes % GROUPS, rr = threadIdx.x / (kLanes * GROUPS);
  const int b = min(static_cast<int>(blockIdx.x) * kRows + rr, total - 1);  // a last block's spare rows repeat the last
  int lo = 0, hi = a.c.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.p.split_rows[mid] <= b) lo = mid; else hi = mid - 1;
  }
  const int grp = d.n_q_heads / d.n_kv_heads;
  const int rows = (a.c.row0[lo + 1] - a.c.row0[lo]) * grp;
  const int at = b - a.p.split_rows[lo], g = at / rows, R = at - g * rows;
  const int tile = narrow_form(rows) ? kM : 2 * kM, tiles = (rows + tile - 1) / tile, pieces = a.p.pieces[lo];
  const int item = a.p.item0[lo] + ((tiles - 1 - R / tile) * d.n_kv_heads + g) * pieces;
  griddep_wait();
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kBatch = 4;
  for (int k0 = q; k0 < pieces; k0 += kBatch * GROUPS) {
    float2 ml[kBatch];
    float4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int k = k0 + i * GROUPS;
      ml[i] = make_float2(-INFINITY, 0.f);
      if (k < pieces) {
        const size_t pr = static_cast<size_t>(item + k) * a.part_rows + R % tile;
        ml[i] = __ldcg(reinterpret_cast<const float2*>(a.part_ml) + pr);
        v[i] = __ldcg(reinterpret_cast<const float4*>(a.part + pr * D) + (c ^ (R % tile & (kLanes - 1))));
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
  const int row = a.c.row0[lo] + R / grp, h = g * grp + R % grp;
  *reinterpret_cast<uint2*>(d.out + row * d.out_row + h * d.out_head + c * 4) =
      make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  if (d.lse && c == 0) d.lse[static_cast<size_t>(row) * d.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ---------------------------------------------------------------- plan (host)
struct Shape {
  int tiles, steps;  // query tiles (or pairs) of a kv head, steps of the longest
};
Shape shape_of(const ChunkTable& c, int i, int grp, bool causal, int window) {
  const int rows = (c.row0[i + 1] - c.row0[i]) * grp;
  Shape s{0, 0};
  if (rows == 0) return s;
  const bool narrow = narrow_form(rows);
  const int tile = narrow ? kM : 2 * kM;
  s.tiles = (rows + tile - 1) / tile;
  // K/V tiles of the longest query tile: at most those that the whole request sees, and with a causal window
  // those that so many keys in a row can touch
  const KeyRange all = keys_of_rows(c.pos[i], c.pos[i] + (rows - 1) / grp, c.n_keys[i], causal, window);
  int64_t t = all.hi > all.lo ? (all.hi + kN - 1) / kN - all.lo / kN : 0;
  if (causal && window > 0) {
    const int64_t positions = (std::min(tile, rows) + grp - 2) / grp + 1, keys = window + positions - 1;
    t = std::min(t, (keys + kN - 2) / kN + 1);
  }
  s.steps = static_cast<int>(narrow ? (t + 1) / 2 : t);
  return s;
}

struct Planned {
  ChunkPlan p;
  int items, merge_rows, part_rows;
};

// A piece of s steps takes about s + kOverhead steps of time (a start, an end and its share of the merge), and
// pieces run one to an SM in waves. Of the piece lengths that just fill 1, 2, ... waves the cheapest is taken; no piece
// is cut where the items are many.
constexpr int kOverhead = 2;
constexpr int kMostWaves = 6;

Planned make_plan(const ChunkTable& c, int n_q_heads, int n_kv_heads, bool causal, int window, int num_sms) {
  Planned r;
  std::memset(&r, 0, sizeof(r));
  const int grp = n_q_heads / n_kv_heads;
  Shape sh[kMaxChunks];
  int longest = 1;
  for (int i = 0; i < c.n; ++i) {
    sh[i] = shape_of(c, i, grp, causal, window);
    longest = std::max(longest, sh[i].steps);
  }
  auto items = [&](int piece) {
    int64_t n = 0;
    for (int i = 0; i < c.n; ++i) n += static_cast<int64_t>(sh[i].tiles) * n_kv_heads * std::max(1, (sh[i].steps + piece - 1) / piece);
    return n;
  };
  const int64_t whole = items(longest);
  int best = longest;
  int64_t best_cost = (whole + num_sms - 1) / num_sms * (longest + kOverhead);
  for (int w = 1; w <= kMostWaves && whole < static_cast<int64_t>(w) * num_sms; ++w) {
    int a = 1, b = longest;  // the shortest piece whose items fit w waves
    while (a < b) {
      const int mid = (a + b) / 2;
      if (items(mid) <= static_cast<int64_t>(w) * num_sms) b = mid; else a = mid + 1;
    }
    const int64_t cost = static_cast<int64_t>(w) * (a + kOverhead) + 1;
    if (a < longest && cost < best_cost) {
      best = a;
      best_cost = cost;
    }
  }
  r.p.piece_steps = best;
  int64_t n = 0, blocks = 0;
  for (int i = 0; i < c.n; ++i) {
    r.p.item0[i] = static_cast<int>(n);
    r.p.split_rows[i] = static_cast<int>(blocks);
    r.p.pieces[i] = std::max(1, (sh[i].steps + best - 1) / best);
    n += static_cast<int64_t>(sh[i].tiles) * n_kv_heads * r.p.pieces[i];
    const int rows = (c.row0[i + 1] - c.row0[i]) * grp;
    if (r.p.pieces[i] > 1) {
      blocks += static_cast<int64_t>(rows) * n_kv_heads;
      r.part_rows = std::max(r.part_rows, narrow_form(rows) ? std::min(rows, kM) : 2 * kM);
    }
  }
  for (int i = c.n; i <= kMaxChunks; ++i) {
    r.p.item0[i] = static_cast<int>(n);
    r.p.split_rows[i] = static_cast<int>(blocks);
  }
  r.items = n > 0x7fffffff ? -1 : static_cast<int>(n);
  r.merge_rows = static_cast<int>(blocks);
  return r;
}

template <int D>
cudaError_t launch_tc(const ChunkArgs& a, const Planned& p, int num_sms, cudaStream_t stream) {
  static PerDevice once;
  int dev = 0;
  if (once.pending(&dev)) {
    cudaError_t e = cudaFuncSetAttribute(chunk_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Tile<D>::kSmem);
    if (e != cudaSuccess) return e;
    // setmaxnreg.inc waits until the CTA's register pool can serve it: refuse to launch a build whose launch
    // count leaves the split short
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, chunk_attn_kernel<D>);
    if (e != cudaSuccess) return e;
    if (fa.numRegs * kThreads < kRegsNeeded) return cudaErrorInvalidConfiguration;
    once.done(dev);
  }
  PdlScope pdl;
  cudaError_t e = launch_kernel(chunk_attn_kernel<D>, dim3(p.items), dim3(kThreads), Tile<D>::kSmem, stream, a);
  if (e != cudaSuccess || p.merge_rows == 0) return e;
  constexpr int kRow = kMergeThreads / (D / 4);  // rows a block with one group each
  if (p.merge_rows < 4 * kRow * num_sms) {
    constexpr int kRows8 = kRow / 8 > 0 ? kRow / 8 : 1;
    return launch_kernel(chunk_attn_merge<D, 8>, dim3((p.merge_rows + kRows8 - 1) / kRows8), dim3(kMergeThreads), 0, stream, a,
                         p.merge_rows);
  }
  return launch_kernel(chunk_attn_merge<D, 1>, dim3((p.merge_rows + kRow - 1) / kRow), dim3(kMergeThreads), 0, stream, a,
                       p.merge_rows);
}

size_t part_floats(const Planned& p, int head_dim, bool ml) {
  if (p.merge_rows == 0) return 0;
  return (static_cast<size_t>(p.items) * p.part_rows * (ml ? 2 : head_dim) + 63) & ~static_cast<size_t>(63);
}

}  // namespace

size_t chunk_attention_workspace(const ChunkTable& c, int n_q_heads, int n_kv_heads, int head_dim, bool causal,
                                 int window, int num_sms) {
  const Planned p = make_plan(c, n_q_heads, n_kv_heads, causal, window, num_sms);
  return (part_floats(p, head_dim, false) + part_floats(p, head_dim, true)) * sizeof(float);
}

int chunk_attention_launches(const ChunkTable& c, int n_q_heads, int n_kv_heads, int head_dim, bool causal, int window,
                             int num_sms) {
  return make_plan(c, n_q_heads, n_kv_heads, causal, window, num_sms).merge_rows ? 2 : 1;
}

cudaError_t launch_chunk_attention(const ChunkAttnDesc& d, const ChunkTable& c, void* workspace, int num_sms,
                                   cudaStream_t stream) {
  const Planned p = make_plan(c, d.n_q_heads, d.n_kv_heads, d.causal, d.window, num_sms);
  if (p.items == 0) return cudaSuccess;
  if (p.items < 0) return cudaErrorInvalidValue;
  ChunkArgs a;
  std::memset(&a, 0, sizeof(a));
  const long pool_rows = static_cast<long>(c.num_pages) * d.n_kv_heads * kPage;
  if (!tensor_map_pool(&a.tmK, d.kpages, pool_rows, d.head_dim) || !tensor_map_pool(&a.tmV, d.vpages, pool_rows, d.head_dim))
    return cudaErrorInvalidValue;
  a.d = d;
  a.c = c;
  a.p = p.p;
  a.part = static_cast<float*>(workspace);
  a.part_ml = a.part + part_floats(p, d.head_dim, false);
  a.part_rows = p.part_rows;
  return d.head_dim == 128 ? launch_tc<128>(a, p, num_sms, stream) : launch_tc<64>(a, p, num_sms, stream);
}

}  // namespace crf
