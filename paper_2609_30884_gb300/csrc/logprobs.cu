// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the gradient. For a row z:
//   lse = log sum exp z,   logprob = z_t - lse,   entropy = lse - sum p z  with  p = exp(z - lse),
// and with g, h the gradients of logprob and entropy
//   dz_v = g (1[v = t] - p_v) - h p_v (log p_v + entropy).
//
// Forward: bound by reading the row once. A lane keeps a running maximum m, s = sum 2^x and d = sum 2^x x with
// x = (z - m) log2 e, in fp32 (entropy = log s - d log 2 / s); differences are formed before the product, so that the rounding of
// m log2 e stays out. A row is one CTA's, or the CTAs of a cluster's where rows are few; their sums meet in shared memory.
//
// The alternatives take no pass of their own over the row. A lane's maximum is known when its sums are, and the lanes of a row are
// groups of its elements (with a cluster, the same lane of every CTA): at least k elements reach the k-th greatest of the
// groups' maxima, and those that reach it lie in groups that do. Sixteen rounds of counting over the block find that bound, to its
// 16 leading bits, where at most 64 lanes then reach it; the pieces of those lanes (a maximum is kept of each) are read again (from
// L2), and the elements that do, some 1.1 k of a long row, are ranked by counting. Keys (value, then lower index) order them, so the
// order in which threads list them does not matter. Where more lanes reach it the rounds go on to its 32nd bit. Such rows (many equal
// logits), and rows that rise along the vocabulary, are gone through again as a whole: those equal to an exact bound are taken in
// order of index, or the k-th greatest key is found digit by digit.
//
// Short rows are a warp's each, which does the same within itself: the groups are halves of the lanes' elements, their bound is
// found with ballots, halves of a strip that reach it are read again, and where the list does not hold what reaches it, the greatest
// key below the last is looked for k times: rows of ties, and rows in which fewer than k groups hold anything above -inf (16384 bf16
// rows of 512 with 12 numbers each and 20 alternatives 157 us, 27 of numbers throughout; of 4000 973 and 49; with 8 alternatives no slower).
//
// Rows start at any element: a row is cut at 16-byte addresses, its first and last pieces element by element.
#include "../../include/crf.h"
#include "rotary.cuh"

#include <algorithm>
#include <cstring>
#include <type_traits>

namespace crf {

namespace {

constexpr int kLogThreads = 256;   // at most; four blocks an SM: 1021 fp32 rows of 152064 take 88 us so, 96 with 512 threads and two
constexpr int kStrip = 1024;       // elements of a warp's step, of a short row or at a row's ends
constexpr int kWide = 8;           // 16-byte units of a lane in a step within a long row: 2001 bf16 rows of 151936 96 us, some 5 more with 4
constexpr int kList = 512;         // elements that are ranked by counting
constexpr int kChosen = 64;        // lanes that are read again, at most
constexpr int kPieces = 128;       // pieces of their elements, at most
constexpr int kRowWarps = 8;        // rows of a block where a row is a warp's
constexpr int kRowList = 256;       // elements that one of them ranks
constexpr int kRowStrips = 8;       // of such a row, at most
// Bytes of a next row: 2001 bf16 rows of 151936 with 8 alternatives 112 us, 113 without and 119 with 128 KB; with 32 alternatives 132, 130 and 140;
// 4000 fp32 rows of 20011 with 8 72, 78 and 72.
constexpr int kAheadBytes = 32768;
constexpr int kAhead = 4;          // units of them that a lane asks for at once
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFloor = -200.f;   // 2^x is 0 from here down; keeps an infinite x out of products

// The greater, or NaN if either is NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Whole numbers that order floats: NaN 1, -inf above it; 0 is below every value.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 1u;
  const uint32_t b = __float_as_uint(v + 0.f);  // both zeros are equal
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  if (order <= 1u) return NAN;
  return __uint_as_float(order >> 31 ? order & 0x7fffffffu : ~order);
}

// The maximum of units, NaN only while there is nothing else; of 16-bit types two elements an instruction, in the type.
template <typename T>
struct UnitMax {
  uint32_t m = 0x7fff7fffu;  // two NaN, of both types
  __device__ __forceinline__ void add(const Unit<T, 8>& u) {
    const uint4 w = *reinterpret_cast<const uint4*>(&u);
    for (const uint32_t x : {w.x, w.y, w.z, w.w}) {
      if constexpr (std::is_same_v<T, __half>) asm("max.f16x2 %0, %0, %1;" : "+r"(m) : "r"(x));
      else asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(x));
    }
  }
  __device__ __forceinline__ float value() const {
    const float2 f = unpack2(T(), m);
    return fmaxf(f.x, f.y);
  }
};
template <>
struct UnitMax<float> {
  float m = NAN;
  __device__ __forceinline__ void add(const Unit<float, 4>& u) { m = fmax3(fmax3(m, u.e[0], u.e[1]), u.e[2], u.e[3]); }
  __device__ __forceinline__ float value() const { return m; }
};

// A running maximum, sum of 2^x and sum of 2^x x.
struct Sums {
  float m, s, d;
  // over to the maximum `to` (not less than m)
  __device__ __forceinline__ void raise(float to) {
    if (s != 0.f) {  // NaN too: it stays one
      const float x = (m - to) * kLog2e, f = ex2_approx(x);
      d = f * (d + s * max_nan(x, kFloor));
      s *= f;
    }
    m = to;
  }
  __device__ __forceinline__ void add(const Sums& o) {
    Sums other = o;
    const float to = fmaxf(m, o.m);
    if (to == -INFINITY) {
      s += o.s;  // nothing, or NaN
      d += o.d;
      return;
    }
    raise(to);
    other.raise(to);
    s += other.s;
    d += other.d;
  }
};

struct LogShared {
  Sums part[kLogThreads / 32];
  Sums cta;                         // read by the cluster's first CTA, as is
  uint32_t lane[kLogThreads];       // the order of each lane's maximum, 0 without elements
  int chosen[kPieces];              // lane + kLogThreads piece
  int n_chosen, n_list, n_equal[kLogThreads / 32];
  unsigned long long list[kList];
  int digits[256];
  unsigned long long prefix;
  int left;
};

__device__ __forceinline__ uint32_t ld_cluster_u32(const void* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ float ld_cluster_f32(const void* p, uint32_t rank) { return __uint_as_float(ld_cluster_u32(p, rank)); }

template <typename T>
__device__ __forceinline__ float load_logit(const T* p) {
  float f[1];
  unpack(*reinterpret_cast<const Unit<T, 1>*>(p), f);
  return f[0];
}

// Adds a strip to a lane's sums, and says the maximum of the lane's elements of it, by halves (its even and odd units).
// Lane l has units l, l + 32 ... of the strip.
template <typename T, int kLoads>
__device__ __forceinline__ float2 add_strip(const T* base, int v0, int skew, int end, int lane, Sums& acc, bool& any) {
  using U = Unit<T, 16 / sizeof(T)>;
  constexpr int VEC = 16 / sizeof(T), kStep = 32 * VEC * kLoads;
  float half[2] = {NAN, NAN}, mx;
  if (v0 >= skew && v0 + kStep <= end) {
    U u[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) u[j] = *reinterpret_cast<const U*>(base + v0 + (j * 32 + lane) * VEC);
    UnitMax<T> even, odd;
#pragma unroll
    for (int j = 0; j < kLoads; j += 2) {
      even.add(u[j]);
      odd.add(u[j + 1]);
    }
    half[0] = even.value();
    half[1] = odd.value();
    mx = fmaxf(half[0], half[1]);
    if (mx > acc.m) acc.raise(mx);
    any = true;
    const float neg = acc.m == -INFINITY ? 0.f : -acc.m;
    const uint64_t neg2 = f32x2(neg, neg), l2e = f32x2(kLog2e, kLog2e), one = f32x2(1.f, 1.f);
    uint64_t s2 = f32x2(0.f, 0.f), d2 = f32x2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      float x[VEC];
      unpack(u[j], x);
#pragma unroll
      for (int i = 0; i < VEC; i += 2) {
        float t0, t1;
        f32x2_split(fma_f32x2(add_f32x2(f32x2(x[i], x[i + 1]), neg2), l2e, f32x2(0.f, 0.f)), t0, t1);
        t0 = max_nan(t0, kFloor);
        t1 = max_nan(t1, kFloor);
        const uint64_t e = f32x2(ex2_approx(t0), ex2_approx(t1));
        s2 = fma_f32x2(e, one, s2);
        d2 = fma_f32x2(e, f32x2(t0, t1), d2);
      }
    }
    float s0, s1;
    f32x2_split(s2, s0, s1);
    acc.s += s0 + s1;
    f32x2_split(d2, s0, s1);
    acc.d += s0 + s1;
  } else {
    // a first or last strip: units that lie inside the row as they are, the others element by element; what is outside is
    // NaN to the maxima and no part of the sums
    float x[kLoads * VEC];
    auto inside = [&](int j, int i) { const int v = v0 + (j * 32 + lane) * VEC + i; return v >= skew && v < end; };
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      float y[VEC];
      if (inside(j, 0) && inside(j, VEC - 1)) {
        unpack(*reinterpret_cast<const U*>(base + v0 + (j * 32 + lane) * VEC), y);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = inside(j, i) ? load_logit(base + v0 + (j * 32 + lane) * VEC + i) : NAN;
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[j * VEC + i] = y[i];
    }
#pragma unroll
    for (int i = 0; i < kLoads * VEC; ++i) half[i / VEC & 1] = fmaxf(half[i / VEC & 1], x[i]);
    mx = fmaxf(half[0], half[1]);
    if (mx > acc.m) acc.raise(mx);
    const float m = acc.m == -INFINITY ? 0.f : acc.m;
#pragma unroll
    for (int i = 0; i < kLoads * VEC; ++i) {
      if (!inside(i / VEC, i % VEC)) continue;
      any = true;
      const float t = max_nan((x[i] - m) * kLog2e, kFloor), e = ex2_approx(t);
      acc.s += e;
      acc.d += e * t;
    }
  }
  return make_float2(half[0], half[1]);
}

// Log probability of a logit from the row's maximum and the log of its sum (-inf: the row holds nothing). The maximum goes first:
// their sum, rounded at the size of the logits, would leave that rounding in (2e-3 at logits of 60000).
__device__ __forceinline__ float logprob_of(float z, float m, float log_s) { return log_s == -INFINITY ? -INFINITY : (z - m) - log_s; }

// A row's outputs but the alternatives, by one thread.
template <typename T>
__device__ __forceinline__ void put_row(const LogprobsDesc& d, int row, const T* z, const Sums& t) {
  const float log_s = logf(t.s);
  if (d.lse) d.lse[row] = t.s == 0.f ? -INFINITY : t.m + log_s;
  if (d.entropy) d.entropy[row] = t.s == 0.f ? 0.f : log_s - t.d * kLn2 / t.s;
  if (d.logprob) {
    int token = d.targets[row];
    float lp = 0.f;
    if (token != -1) {
      token = checked_token(token, d.vocab, d.status);
      lp = logprob_of(load_logit(z + token), t.m, log_s);
    }
    d.logprob[row] = lp;
  }
}
__device__ __forceinline__ void put_top(const LogprobsDesc& d, int row, int at, unsigned long long key, float m, float log_s) {
  const int64_t to = static_cast<int64_t>(row) * d.n_top + at;
  if (d.top_ids) d.top_ids[to] = static_cast<int32_t>(~static_cast<uint32_t>(key));
  if (d.top_logprobs) d.top_logprobs[to] = logprob_of(value_of(static_cast<uint32_t>(key >> 32)), m, log_s);
}

// C: CTAs of a row, a cluster. next: as many rows as have blocks on the SMs at a time.
template <typename T, int C>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(kLogThreads, 4) logprobs_kernel(const __grid_constant__ LogprobsDesc d, int next) {
  using U = Unit<T, 16 / sizeof(T)>;
  constexpr int VEC = 16 / sizeof(T), kLoads = kWide, kNarrow = kStrip / (32 * VEC), kStep = 32 * VEC * kLoads;
  static_assert(kStep % kStrip == 0, "a step at a row's ends is gone through in strips");
  __shared__ LogShared sh;
  griddep_launch_dependents();
  const int row = blockIdx.x / C, rank = C > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const T* z = static_cast<const T*>(d.z) + row * d.z_row;
  // virtual index v = element + skew: 16-byte aligned where v is a multiple of VEC
  const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int end = d.vocab + skew, strips = (end + kStep - 1) / kStep;
  const T* base = z - skew;  // never read before z
  // a lane's elements in pieces, a maximum each: those of each CTA of the cluster, or halves of every other step
  constexpr int kSplit = C > 1 ? C : 2, kHalves = C > 1 ? 1 : 2, kParts = kSplit * kHalves;
  Sums acc{-INFINITY, 0.f, 0.f};
  float piece[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};  // without a cluster
  bool any = false;
  int turn = 0;
  auto note = [&](float2 half) {
    if constexpr (C == 1) {
      if (d.n_top == 0) return;
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        if ((turn & 1) == i / 2) {
          piece[i] = fmaxf(piece[i], half.x);
          piece[i + 1] = fmaxf(piece[i + 1], half.y);
        }
    }
  };
  griddep_wait();
  for (int st = rank * warps + warp; st < strips; st += C * warps, ++turn) {
    // lane l has units l, l + 32 ... of the strip
    const int v0 = st * kStep;
    if (v0 >= skew && v0 + kStep <= end) {
      note(add_strip<T, kLoads>(base, v0, skew, end, lane, acc, any));
    } else {
#pragma unroll 1
      for (int v = v0; v < min(v0 + kStep, end); v += kStrip) note(add_strip<T, kNarrow>(base, v, skew, end, lane, acc, any));
    }
  }
  // While a block looks for alternatives it loads nothing: the beginning of the row that its place on the SM is likely to have next
  // is brought to L2 meanwhile (4000 fp32 rows of 20011 with 8 alternatives 72 us, 78 without).
  if (C == 1 && threadIdx.x == 0 && d.n_top > 0 && row + next < d.n_rows) {
    const uintptr_t from = (reinterpret_cast<uintptr_t>(z + next * d.z_row) + 15) & ~uintptr_t{15};
    const int bytes = min(kAheadBytes, (d.vocab - VEC) * static_cast<int>(sizeof(T))) & ~15;
    if (bytes > 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"(bytes) : "memory");
  }
  sh.lane[threadIdx.x] = any ? order_of(acc.m) : 0u;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) {
    Sums other;
    other.m = __shfl_xor_sync(0xffffffffu, acc.m, o);
    other.s = __shfl_xor_sync(0xffffffffu, acc.s, o);
    other.d = __shfl_xor_sync(0xffffffffu, acc.d, o);
    acc.add(other);
  }
  if (lane == 0) sh.part[warp] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < warps; ++w) acc.add(sh.part[w]);
    sh.cta = acc;
    sh.n_chosen = sh.n_list = 0;
  }
  uint32_t part[kParts];
  part[0] = sh.lane[threadIdx.x];
  uint32_t mine = part[0];
  if (C > 1) {
    cluster_sync();
    if (rank != 0) {
      cluster_sync();  // the first CTA has read what it needs
      return;
    }
#pragma unroll
    for (int r = 1; r < C; ++r) mine = max(mine, part[r % kParts] = ld_cluster_u32(&sh.lane[threadIdx.x], r));
    if (threadIdx.x == 0) {
      for (int r = 1; r < C; ++r) {
        Sums o;
        o.m = ld_cluster_f32(&sh.cta.m, r);
        o.s = ld_cluster_f32(&sh.cta.s, r);
        o.d = ld_cluster_f32(&sh.cta.d, r);
        acc.add(o);
      }
      sh.cta = acc;
    }
    cluster_sync();
  } else {
#pragma unroll
    for (int i = 0; i < kParts; ++i) part[i] = order_of(piece[i & 3]);
    __syncthreads();
  }
  const float m = sh.cta.m, log_s = logf(sh.cta.s);
  if (threadIdx.x == 0) put_row(d, row, z, sh.cta);
  const int k = d.n_top;
  if (k == 0) return;

  // ---------------------------------------------------------------- lanes that reach the k-th greatest maximum
  uint32_t least = 0;
  int reached = __syncthreads_count(mine > 0);
  if (reached >= k) {
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t cand = least | (1u << bit);
      const int n = __syncthreads_count(mine >= cand);
      if (n >= k) {
        least = cand;
        reached = n;
      }
      if (bit == 16 && reached <= kChosen) break;
    }
  }
  least = max(least, 1u);  // (fewer lanes than k: every element is listed)
  auto key = [&](uint32_t order, int v) { return static_cast<unsigned long long>(order) << 32 | ~static_cast<uint32_t>(v - skew); };
  // Into the list; n_list counts those that it has no room for as well.
  auto push = [&](bool in, uint32_t order, int v) {
    const uint32_t ins = __ballot_sync(0xffffffffu, in);
    if (ins == 0) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(&sh.n_list, __popc(ins));
    at = __shfl_sync(0xffffffffu, at, 0) + __popc(ins & ((1u << lane) - 1));
    if (in && at < kList) sh.list[at] = key(order, v);
  };
  bool again = reached > kChosen;
  if (!again) {
    if (mine >= least) {
#pragma unroll
      for (int i = 0; i < kParts; ++i)
        if (part[i] >= least) {
          const int at = atomicAdd(&sh.n_chosen, 1);
          if (at < kPieces) sh.chosen[at] = i * kLogThreads + threadIdx.x;
        }
    }
    __syncthreads();
    // piece i of warp w has the steps (i / kHalves) warps + w, (i / kHalves + kSplit) warps + w ... of the row, or a half of their units
    constexpr int kUnits = kLoads / kHalves;
    const int turns = (strips + kSplit * warps - 1) / (kSplit * warps), units = min(sh.n_chosen, kPieces) * turns * kUnits;
    auto unit_at = [&](int e) {
      const int pair = e / kUnits, at = sh.chosen[pair / turns], thread = at % kLogThreads, i = at / kLogThreads;
      return ((i / kHalves + pair % turns * kSplit) * warps + thread / 32) * kStep + ((e % kUnits * kHalves + i % kHalves) * 32 + thread % 32) * VEC;
    };
    for (int e0 = warp * 32; e0 < units; e0 += kAhead * blockDim.x) {
      U u[kAhead];  // all in flight
      int v[kAhead];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        const int e = e0 + q * blockDim.x + lane;
        v[q] = e < units ? unit_at(e) : end;
        if (v[q] >= skew && v[q] + VEC <= end) u[q] = *reinterpret_cast<const U*>(base + v[q]);
      }
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        if (e0 + q * static_cast<int>(blockDim.x) >= units) break;
        uint32_t o[VEC];
        if (v[q] >= skew && v[q] + VEC <= end) {
          float x[VEC];
          unpack(u[q], x);
#pragma unroll
          for (int i = 0; i < VEC; ++i) o[i] = order_of(x[i]);
        } else {
#pragma unroll
          for (int i = 0; i < VEC; ++i) o[i] = v[q] + i >= skew && v[q] + i < end ? order_of(load_logit(base + v[q] + i)) : 0u;
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) push(o[i] >= least, o[i], v[q] + i);
      }
    }
    __syncthreads();
    again = sh.n_list > kList || sh.n_list < k || sh.n_chosen > kPieces;  // (fewer than k: where NaN hides behind a maximum of -inf)
    if (sh.n_list < k) least = 1u;
  }
  if (again) {
    // ---------------------------------------------------------------- the whole row again, a run of it a warp
    const bool exact = reached > kChosen;
    const int runs = (end + 31) / 32, c0 = static_cast<int>(static_cast<int64_t>(runs) * warp / warps), c1 = static_cast<int>(static_cast<int64_t>(runs) * (warp + 1) / warps);
    auto order_at = [&](int v) { return v >= skew && v < end ? order_of(load_logit(base + v)) : 0u; };
    __syncthreads();
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
    int above = kList + 1;
    if (exact) {
      int equal = 0;
#pragma unroll 4
      for (int c = c0; c < c1; ++c) {
        const uint32_t o = order_at(c * 32 + lane);
        push(o > least, o, c * 32 + lane);
        equal += __popc(__ballot_sync(0xffffffffu, o == least));
      }
      if (lane == 0) sh.n_equal[warp] = equal;
      __syncthreads();
      above = sh.n_list;
      for (int w = equal = 0; w < warps; ++w) equal += sh.n_equal[w];
      __syncthreads();
      if (above + equal < k) {  // NaN behind a bound of -inf
        above = kList + 1;
        least = 1u;
      }
    }
    if (above <= kList - kMaxTop) {
      // all above the bound, and the first of those equal to it
      int at = above;
      for (int w = 0; w < warp; ++w) at += sh.n_equal[w];
      for (int c = c0; c < c1 && at < k; ++c) {
        const uint32_t o = order_at(c * 32 + lane), eqs = __ballot_sync(0xffffffffu, o == least);
        const int to = at + __popc(eqs & ((1u << lane) - 1));
        if (o == least && to < k) sh.list[to] = key(o, c * 32 + lane);
        at += __popc(eqs);
      }
      if (threadIdx.x == 0) sh.n_list = max(above, k);
    } else {
      // the k-th greatest key, a digit of eight bits at a time; then the keys that reach it
      if (threadIdx.x == 0) {
        sh.prefix = 0;
        sh.left = k;
        sh.n_list = 0;
      }
      for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += blockDim.x) sh.digits[i] = 0;
        __syncthreads();
        const unsigned long long prefix = sh.prefix;
#pragma unroll 4
        for (int c = c0; c < c1; ++c) {
          const uint32_t o = order_at(c * 32 + lane);
          const unsigned long long x = key(o, c * 32 + lane);
          if (o >= least && (shift == 56 || x >> (shift + 8) == prefix >> (shift + 8))) atomicAdd(&sh.digits[static_cast<int>(x >> shift) & 255], 1);
        }
        __syncthreads();
        if (warp == 0) {
          // lane l has the digits from 255 - 8 l down
          int sum = 0;
          for (int i = 0; i < 8; ++i) sum += sh.digits[255 - 8 * lane - i];
          int to = sum;
#pragma unroll
          for (int o = 1; o < 32; o *= 2) {
            const int up = __shfl_up_sync(0xffffffffu, to, o);
            if (lane >= o) to += up;
          }
          const int left = sh.left;
          __syncwarp();
          int at = to - sum;
          if (at < left && to >= left) {
            int i = 255 - 8 * lane;
            while (at + sh.digits[i] < left) at += sh.digits[i--];
            sh.prefix = prefix | static_cast<unsigned long long>(i) << shift;
            sh.left = left - at;
          }
        }
        __syncthreads();
      }
      const unsigned long long from = sh.prefix;
#pragma unroll 4
      for (int c = c0; c < c1; ++c) {
        const uint32_t o = order_at(c * 32 + lane);
        push(o != 0 && key(o, c * 32 + lane) >= from, o, c * 32 + lane);
      }
    }
    __syncthreads();
  }
  // ---------------------------------------------------------------- ranks: a key's lanes count those above it
  const int listed = sh.n_list, share = listed * 8 <= static_cast<int>(blockDim.x) ? 8 : 1, own = threadIdx.x % share;
  for (int i0 = 0; i0 < listed; i0 += blockDim.x / share) {
    const int i = i0 + static_cast<int>(threadIdx.x) / share;
    const unsigned long long it = i < listed ? sh.list[i] : 0ull;
    int before = 0;
#pragma unroll 4
    for (int j = own; j < listed; j += share) before += sh.list[j] > it;
    for (int o = share / 2; o > 0; o /= 2) before += __shfl_xor_sync(0xffffffffu, before, o);
    if (i < listed && before < k && own == 0) put_top(d, row, before, it, m, log_s);
  }
}

// ---------------------------------------------------------------- a warp a row
template <typename T>
__global__ void __launch_bounds__(32 * kRowWarps, 4) logprobs_rows_kernel(const __grid_constant__ LogprobsDesc d) {
  using U = Unit<T, 16 / sizeof(T)>;
  constexpr int VEC = 16 / sizeof(T), kLoads = kStrip / (32 * VEC);
  __shared__ unsigned long long lists[kRowWarps][kRowList];
  __shared__ uint32_t maxima[kRowWarps][2 * kRowStrips][32];    // of the halves of a lane's elements of each strip
  __shared__ uint16_t pieces[kRowWarps][2 * kRowStrips * 32];   // 32 (2 strip + half) + lane: those that are read again
  griddep_launch_dependents();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, row = blockIdx.x * (blockDim.x / 32) + warp;
  if (row >= d.n_rows) return;
  const T* z = static_cast<const T*>(d.z) + row * d.z_row;
  const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int end = d.vocab + skew, strips = (end + kStrip - 1) / kStrip;
  const T* base = z - skew;  // never read before z
  Sums acc{-INFINITY, 0.f, 0.f};
  bool any = false;
  griddep_wait();
  // the maxima of a lane's elements by halves: 64 groups of the row's elements
  float even = -INFINITY, odd = -INFINITY;
  for (int st = 0; st < strips; ++st) {
    const float2 half = add_strip<T, kLoads>(base, st * kStrip, skew, end, lane, acc, any);
    even = fmaxf(even, half.x);
    odd = fmaxf(odd, half.y);
    if (d.n_top > 0) {
      maxima[warp][2 * st][lane] = order_of(half.x);
      maxima[warp][2 * st + 1][lane] = order_of(half.y);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) {
    Sums other;
    other.m = __shfl_xor_sync(0xffffffffu, acc.m, o);
    other.s = __shfl_xor_sync(0xffffffffu, acc.s, o);
    other.d = __shfl_xor_sync(0xffffffffu, acc.d, o);
    acc.add(other);
  }
  if (lane == 0) put_row(d, row, z, acc);
  const int k = d.n_top;
  if (k == 0) return;
  const float m = acc.m, log_s = logf(acc.s);
  const uint32_t mine[2] = {any ? order_of(even) : 0u, any ? order_of(odd) : 0u};
  auto groups_from = [&](uint32_t order) { return __popc(__ballot_sync(0xffffffffu, mine[0] >= order)) + __popc(__ballot_sync(0xffffffffu, mine[1] >= order)); };
  uint32_t least = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit)
    if (groups_from(least | (1u << bit)) >= k) least |= 1u << bit;
  auto key = [&](uint32_t order, int v) { return static_cast<unsigned long long>(order) << 32 | ~static_cast<uint32_t>(v - skew); };
  unsigned long long* list = lists[warp];
  int n = 0;
  if (least > order_of(-INFINITY)) {
    int found = 0;
#pragma unroll 2
    for (int h = 0; h < 2 * strips; ++h) {
      const bool in = maxima[warp][h][lane] >= least;
      const uint32_t ins = __ballot_sync(0xffffffffu, in);
      if (in) pieces[warp][found + __popc(ins & ((1u << lane) - 1))] = static_cast<uint16_t>(h * 32 + lane);
      found += __popc(ins);
    }
    __syncwarp();
    constexpr int kUnits = kLoads / 2, kMany = VEC == 8 ? 4 : 6;  // what 64 registers hold; a lane's elements are the bits of a word
    const int units = found * kUnits;
    const float bound = value_of(least);  // above -inf, where floats compare as their orders do
    auto unit_at = [&](int e) {
      const int piece = pieces[warp][e / kUnits];
      return piece / 64 * kStrip + ((e % kUnits * 2 + piece / 32 % 2) * 32 + piece % 32) * VEC;
    };
    for (int e0 = 0; e0 < units && n <= kRowList; e0 += 32 * kMany) {
      U u[kMany];  // all in flight
      int v[kMany];
      uint32_t hits = 0;
#pragma unroll
      for (int q = 0; q < kMany; ++q) {
        const int e = e0 + q * 32 + lane;
        v[q] = e < units ? unit_at(e) : end;
        if (v[q] >= skew && v[q] + VEC <= end) u[q] = *reinterpret_cast<const U*>(base + v[q]);
      }
#pragma unroll
      for (int q = 0; q < kMany; ++q) {
        if (v[q] >= skew && v[q] + VEC <= end) {
          float x[VEC];
          unpack(u[q], x);
#pragma unroll
          for (int i = 0; i < VEC; ++i) hits |= static_cast<uint32_t>(x[i] >= bound) << (q * VEC + i);
        } else if (v[q] < end) {
#pragma unroll 1
          for (int i = 0; i < VEC; ++i)
            if (v[q] + i >= skew && v[q] + i < end && load_logit(base + v[q] + i) >= bound) hits |= 1u << (q * VEC + i);
        }
      }
      const int count = __popc(hits);
      int to = count;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int up = __shfl_up_sync(0xffffffffu, to, o);
        if (lane >= o) to += up;
      }
      int at = n + to - count;
      n += __shfl_sync(0xffffffffu, to, 31);
      if (n > kRowList) break;
      for (; hits; hits &= hits - 1) {
        const int bit = __ffs(hits) - 1, at_v = unit_at(e0 + bit / VEC * 32 + lane) + bit % VEC;
        list[at++] = key(order_of(load_logit(base + at_v)), at_v);
      }
    }
  } else if (d.vocab <= kRowList) {  // (groups without elements count, at -inf and below)
    for (int v = skew + lane; v < end; v += 32) list[v - skew] = key(order_of(load_logit(base + v)), v);
    n = d.vocab;
  }
  __syncwarp();
  if (n >= k && n <= kRowList) {
    for (int i = lane; i < n; i += 32) {
      const unsigned long long it = list[i];
      int before = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) before += list[j] > it;
      if (before < k) put_top(d, row, before, it, m, log_s);
    }
    return;
  }
  // many equal logits, or few that are no NaN: the greatest key below the last, k times
  unsigned long long last = ~0ull;
#pragma unroll 1
  for (int r = 0; r < k; ++r) {
    unsigned long long best = 0;
#pragma unroll 4
    for (int v = skew + lane; v < end; v += 32) {
      const unsigned long long it = key(order_of(load_logit(base + v)), v);
      if (it < last && it > best) best = it;
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0) put_top(d, row, r, best, m, log_s);
    last = best;
  }
}

// ---------------------------------------------------------------- gradient
constexpr int kGradThreads = 256, kGradLoads = 4;

struct LogGradArgs {
  LogprobsGradDesc d;
};

// One element's gradient: x = log p.
__device__ __forceinline__ float grad_of(float x, float g, float h, float entropy) {
  const float l = max_nan(x, kFloor);
  return -ex2_approx(l * kLog2e) * (g + h * (l + entropy));
}

// VEC elements a load where z and dz lie alike, else 1. A block takes kGradThreads kGradLoads units of a row.
template <typename T, int VEC>
__global__ void __launch_bounds__(kGradThreads) logprobs_grad_kernel(const __grid_constant__ LogGradArgs a) {
  using U = Unit<T, VEC>;
  griddep_launch_dependents();
  const LogprobsGradDesc& d = a.d;
  const int64_t row = blockIdx.y + static_cast<int64_t>(blockIdx.z) * gridDim.y;
  if (row >= d.n_rows) return;
  const T* z = static_cast<const T*>(d.z) + row * d.z_row;
  T* out = static_cast<T*>(d.dz) + row * d.dz_row;
  const int skew = VEC > 1 ? static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T)) : 0;
  const int end = d.vocab + skew, units = (end + VEC - 1) / VEC;
  const int u0 = blockIdx.x * (kGradThreads * kGradLoads) + threadIdx.x;
  griddep_wait();
  U u[kGradLoads];
#pragma unroll
  for (int j = 0; j < kGradLoads; ++j) {
    const int v = (u0 + j * kGradThreads) * VEC;
    if (v >= skew && v + VEC <= end) u[j] = *reinterpret_cast<const U*>(z - skew + v);
  }
  const float lse = d.lse[row];
  int t = d.targets ? d.targets[row] : -1;
  if (t != -1) t = checked_token(t, d.vocab, d.status);
  const float g = t != -1 && d.g_logprob ? d.g_logprob[row] : 0.f;
  const float h = d.g_entropy ? d.g_entropy[row] : 0.f, entropy = d.g_entropy ? d.entropy[row] : 0.f;
  const bool empty = lse == -INFINITY;  // a row without a finite logit has no gradient
#pragma unroll
  for (int j = 0; j < kGradLoads; ++j) {
    const int v = (u0 + j * kGradThreads) * VEC;
    if (v >= skew && v + VEC <= end) {
      float x[VEC];
      unpack(u[j], x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        float y = empty ? 0.f : grad_of(x[i] - lse, g, h, entropy);
        if (v + i - skew == t && !empty) y += g;
        x[i] = y;
      }
      pack(x, u[j]);
      *reinterpret_cast<U*>(out - skew + v) = u[j];
    } else if (u0 + j * kGradThreads < units) {
#pragma unroll 1
      for (int i = max(0, skew - v); i < VEC && v + i < end; ++i) {
        const int e = v + i - skew;
        float y = empty ? 0.f : grad_of(load_logit(z + e) - lse, g, h, entropy);
        if (e == t && !empty) y += g;
        const float f[1] = {y};
        pack(f, *reinterpret_cast<Unit<T, 1>*>(out + e));
      }
    }
  }
}

// ---------------------------------------------------------------- launches
template <typename T>
cudaError_t launch_type(const LogprobsDesc& d, int num_sms, cudaStream_t stream) {
  const int strips = (d.vocab + 15 + kStrip - 1) / kStrip;
  // Short rows are a warp's each, many of up to eight strips too: 16384 bf16 rows of 4000 take 34 us so without alternatives and 58
  // with 32, 70 and 168 as blocks; of 8000, 55 and 81, 81 and 182 as blocks; 2500 of 8000, 16 and 24, 18 and 34 as blocks. Fewer rows, or
  // longer ones, are faster as blocks (100 of 8000 with 32: 9, 15 a warp each).
  if (strips <= 2 || (strips <= kRowStrips && d.n_rows >= 16 * num_sms)) {
    const int w = std::max(1, std::min(kRowWarps, d.n_rows / num_sms));
    PdlScope pdl;
    return launch_kernel(logprobs_rows_kernel<T>, dim3((d.n_rows + w - 1) / w), dim3(32 * w), 0, stream, d);
  }
  // a row's CTAs: enough that few rows fill the SMs twice (100 and 200 fp32 rows of 152064 take 14 and 23 us so, 16
  // and 26 with once, 19 and 26 with three times), each with two steps at least, so that 32 alternatives find groups enough
  constexpr int kStep = 32 * 16 / static_cast<int>(sizeof(T)) * kWide;
  int c = 1;
  while (c < 8 && static_cast<int64_t>(d.n_rows) * c < 2 * num_sms && d.vocab >= 4 * c * kStep) c *= 2;
  // as few warps as take no more turns: 700 bf16 rows of 20011 ten steps a row by five warps, all resident at once
  const int steps = ((d.vocab + 15 + kStep - 1) / kStep + c - 1) / c, most = kLogThreads / 32, turns = (steps + most - 1) / most;
  const dim3 grid(static_cast<unsigned>(d.n_rows) * c), block(32 * ((steps + turns - 1) / turns));
  const int next = num_sms * (4 * kLogThreads / static_cast<int>(block.x));
  PdlScope pdl;
  switch (c) {
    case 1: return launch_kernel(logprobs_kernel<T, 1>, grid, block, 0, stream, d, next);
    case 2: return launch_kernel(logprobs_kernel<T, 2>, grid, block, 0, stream, d, next);
    case 4: return launch_kernel(logprobs_kernel<T, 4>, grid, block, 0, stream, d, next);
  }
  return launch_kernel(logprobs_kernel<T, 8>, grid, block, 0, stream, d, next);
}

template <typename T>
cudaError_t launch_grad_type(const LogprobsGradDesc& d, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  LogGradArgs a{d};
  // every row of z and dz starts at the same place of a 16-byte piece
  const bool alike = ((reinterpret_cast<uintptr_t>(d.z) ^ reinterpret_cast<uintptr_t>(d.dz)) & 15) == 0 && (d.n_rows == 1 || (d.z_row - d.dz_row) % VEC == 0);
  const int vec = alike ? VEC : 1;
  const int64_t per = static_cast<int64_t>(kGradThreads) * kGradLoads * vec;
  const unsigned rows = static_cast<unsigned>(std::min(d.n_rows, 32768)), z = static_cast<unsigned>((static_cast<int64_t>(d.n_rows) + rows - 1) / rows);
  const dim3 grid(static_cast<unsigned>((d.vocab + vec - 1 + per - 1) / per), rows, z);
  PdlScope pdl;
  return alike ? launch_kernel(logprobs_grad_kernel<T, VEC>, grid, dim3(kGradThreads), 0, stream, a)
               : launch_kernel(logprobs_grad_kernel<T, 1>, grid, dim3(kGradThreads), 0, stream, a);
}

}  // namespace

cudaError_t launch_logprobs(const LogprobsDesc& d, int num_sms, cudaStream_t stream) {
  switch (d.type) {
    case CRF_BF16: return launch_type<__nv_bfloat16>(d, num_sms, stream);
    case CRF_FP16: return launch_type<__half>(d, num_sms, stream);
    case CRF_FP32: return launch_type<float>(d, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

cudaError_t launch_logprobs_grad(const LogprobsGradDesc& d, cudaStream_t stream) {
  switch (d.type) {
    case CRF_BF16: return launch_grad_type<__nv_bfloat16>(d, stream);
    case CRF_FP16: return launch_grad_type<__half>(d, stream);
    case CRF_FP32: return launch_grad_type<float>(d, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace crf
