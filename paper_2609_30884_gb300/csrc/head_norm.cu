// RMS norms of query and key heads with the position rotation in the same pass, and the gradient. For a head x of n
// elements with gain w, r = 1 / sqrt(mean(x^2) + eps), and R the rotation at the row's position (rotary.cu):
//   y = R (w x r)                                        (products element by element)
// and for the gradient g of y, with u = R^T g and v = w u:
//   dw = sum over rows and heads of u x r,   dx = r (v - x r^2 mean(v x)).
// Sums and products are fp32; y and dx are rounded once to the type, dw stays fp32. The forward form also writes keys and
// values of new rows into the pages of a layer (values neither normed nor turned).
//
// Bound by memory: every element is read once and written once. As in rotary.cu a thread owns one 16-byte unit of a head (for
// the half layout two, the pair's halves), in four neighbouring heads, two in a gradient; here the lanes of a head, a power of
// two, are neighbours in a warp and join the sum of squares by shuffles. What it takes to stay near memory is few instructions: 512
// elements of a warp's step took 283 of them at first (16384 bf16 rows of 32 heads 58 us, the gradient 155; now 44, 90% of the
// copy rate, and 72, 83%). So places are found by shifts, arithmetic is on two elements an instruction, gains and angles are
// multiplied once for a thread's heads, and all of its heads' shuffles go level by level. (In the half layout of 16-bit heads that is more than
// the 80 registers that three blocks an SM leave: 32 to 52 bytes a thread are spilled.) Heads whose units are no such thing (odd
// sizes, strides or alignments, a half of the turning part that is no whole unit, more than 32 units) take a warp each, an element or
// a pair a lane, and are slow: 16384 bf16 rows of 32 heads of 128 that turn 8 elements 254 us, the gradient 866;
// of 80 that turn 40 199 and 732; 8192 fp32 rows of 16 heads of 256 63 and 192 interleaved, 107 and 136 where 64 elements turn.
//
// The gains' gradient: a thread keeps the same elements of its heads' part over all the rows that its block walks, so
// their sums stay in its registers; a block's sums meet in shared memory, the blocks' in a second small kernel, both in a
// fixed order: the same inputs give the same bits. The next rows' loads are on their way, and a batch of their angles formed, before the
// block's one barrier a batch.
#include "../../include/crf.h"
#include "rotary.cuh"

#include <algorithm>
#include <cstring>
#include <type_traits>

namespace crf {

namespace {

constexpr int kNormBatch = 4;   // heads of a thread
constexpr int kLoose = 8;       // elements of a lane in the form of a warp a head: 256 / 32

// How a call's heads lie in blocks.
struct Tiling {
  int log_lanes;            // of a head
  int units, rot_units;     // 16-byte units of a head, those that rotate
  int log_rows;             // of a block
  int slot0[3];             // each part's first slot (of a batch of heads)
  int slots, block_slots;   // of all parts; of a block
};
struct NormArgs {
  HeadNormDesc d;
  ChunkTable c;
  Tiling t;
};

// A thread's place: unit u of the heads [head, head + heads) of a part, row rb of the block's.
struct Place {
  int rb, part, head, heads;
  bool turning;
  int e0, e1;  // first elements of its piece(s)
  int pair;    // its first pair
};
template <int VEC, bool INTER, int BATCH>
__host__ __device__ __forceinline__ Place place_of(const Tiling& a, const RotaryDesc& d, int thread, int column) {
  Place t;
  const int u = thread & ((1 << a.log_lanes) - 1), rest = thread >> a.log_lanes;
  t.rb = rest & ((1 << a.log_rows) - 1);
  const int at = rest >> a.log_rows, slot = at + column * a.block_slots;
  const bool there = at < a.block_slots && slot < a.slots && u < a.units;
  t.part = slot >= a.slot0[2] ? 2 : slot >= a.slot0[1] ? 1 : 0;
  const int first = t.part == 0 ? 0 : t.part == 1 ? a.slot0[1] : a.slot0[2];
  const int all = t.part == 0 ? d.part[0].heads : t.part == 1 ? d.part[1].heads : d.part[2].heads;
  t.head = (slot - first) * BATCH;
  t.heads = !there ? 0 : all - t.head < BATCH ? all - t.head : BATCH;
  t.turning = u < a.rot_units;
  t.e0 = t.turning ? u * VEC : d.rot_dim + (u - a.rot_units) * VEC;
  t.e1 = t.turning && !INTER ? t.e0 + d.rot_dim / 2 : t.e0;
  t.pair = u * (INTER ? VEC / 2 : VEC);
  return t;
}
// Whether a thread of the gradient has a second unit: the other half of its pairs, or its next head. Threads behind the last head have none,
// wherever their place would be.
template <bool INTER>
__host__ __device__ __forceinline__ bool second_unit(const Place& p) {
  return INTER ? p.heads > 1 : p.heads > 0 && p.turning;
}

// Position of row r of a cache's requests, and its page as the table has it.
__device__ __forceinline__ void find_row(const ChunkTable& c, int r, int* pos, int* page) {
  const int i = chunk_of_row(c, r);
  *pos = c.pos[i] + (r - c.row0[i]);
  *page = c.pt[i][*pos / kPage];
}
// The page, or -1 where the pool has none such: writes to it are left out.
__device__ __forceinline__ int checked_row_page(const RotaryDesc& d, const ChunkTable& c, int page) {
  if (page >= 0 && page < c.num_pages) return page;
  if (d.status) atomicOr(d.status, kStatusBounds);
  return -1;
}
// Where a part's row goes, and the step from head to head.
__device__ __forceinline__ int64_t out_at(const RotaryDesc& d, const RotPart& t, int64_t row, int pos, int page) {
  return t.paged ? (static_cast<int64_t>(page) * d.n_kv_heads * kPage + pos % kPage) * d.head_dim : row * t.out_row;
}
__device__ __forceinline__ int64_t out_step(const RotaryDesc& d, const RotPart& t) {
  return t.paged ? static_cast<int64_t>(kPage) * d.head_dim : t.out_head;
}

// ---------------------------------------------------------------- two elements a word
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float sum_f32x2(uint64_t a) {
  float x, y;
  f32x2_split(a, x, y);
  return x + y;
}
__device__ __forceinline__ uint64_t swap_f32x2(uint64_t a) {
  float x, y;
  f32x2_split(a, x, y);
  return f32x2(y, x);
}
template <typename T, int VEC>
__device__ __forceinline__ void unpack_pairs(const uint4& raw, uint64_t (&p)[VEC / 2]) {
  Unit<T, VEC> u;
  *reinterpret_cast<uint4*>(&u) = raw;
  float f[VEC];
  unpack(u, f);
#pragma unroll
  for (int i = 0; i < VEC / 2; ++i) p[i] = f32x2(f[2 * i], f[2 * i + 1]);
}
template <typename T, int VEC>
__device__ __forceinline__ uint4 pack_pairs(const uint64_t (&p)[VEC / 2]) {
  float f[VEC];
#pragma unroll
  for (int i = 0; i < VEC / 2; ++i) f32x2_split(p[i], f[2 * i], f[2 * i + 1]);
  Unit<T, VEC> u;
  pack(f, u);
  return *reinterpret_cast<const uint4*>(&u);
}
// Sums over the lanes of a head, of N heads level by level.
template <int N>
__device__ __forceinline__ void head_sums(float (&v)[N], int log_lanes) {
  for (int o = (1 << log_lanes) >> 1; o > 0; o >>= 1) {
#pragma unroll
    for (int b = 0; b < N; ++b) v[b] += __shfl_xor_sync(0xffffffffu, v[b], o);
  }
}
// Angles of `rows` rows: cosines and sines [row][pair].
struct Angles {
  float cos[kRotMaxAngles], sin[kRotMaxAngles];
};
__device__ __forceinline__ void form_angles(const RotaryDesc& d, const int* pos, int log_rows, int rows, Angles& to) {
  const int pairs = d.rot_dim / 2;
  for (int i = threadIdx.x; i < pairs << log_rows; i += blockDim.x) {
    const int k = i >> log_rows, r = i & ((1 << log_rows) - 1);  // lanes of a warp share pairs
    if (r >= rows) continue;
    const float2 t = turn_cos_sin(static_cast<uint64_t>(static_cast<int64_t>(pos[r])) * d.turns[k]);
    to.cos[r * pairs + k] = t.x * d.magnitude;
    to.sin[r * pairs + k] = t.y * d.magnitude;
  }
}

// N neighbouring angles, from where N of them are aligned to what they take (at most 16 bytes).
template <int N>
__device__ __forceinline__ void load_angles(const float* from, float (&to)[N]) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(from + i);
      to[i] = v.x;
      to[i + 1] = v.y;
      to[i + 2] = v.z;
      to[i + 3] = v.w;
    }
  } else {
    static_assert(N == 2, "an angle a pair of 8 or 4 elements");
    const float2 v = *reinterpret_cast<const float2*>(from);
    to[0] = v.x;
    to[1] = v.y;
  }
}

// ---------------------------------------------------------------- forward, 16-byte units
// PAGED: rows of a cache's requests, whose positions and pages are found first; else the positions are given (and the barrier between is left out:
// 5003 fp16 rows 15.8 us, 16.9 with it).
template <typename T, int VEC, bool INTER, int BATCH, bool PAGED>
__global__ void __launch_bounds__(kRotThreads, BATCH == 1 ? 1 : 3) head_norm_kernel(const __grid_constant__ NormArgs a) {
  constexpr bool kTwo = !INTER;
  constexpr int P = VEC / 2, H = kTwo ? P : 1;
  __shared__ int s_pos[PAGED ? kRotMaxRows : 1], s_page[PAGED ? kRotMaxRows : 1];
  __shared__ __align__(16) Angles s_angle;
  griddep_launch_dependents();
  const RotaryDesc& d = a.d.r;
  const Place p = place_of<VEC, INTER, BATCH>(a.t, d, threadIdx.x, blockIdx.y);
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) << a.t.log_rows, row = row0 + p.rb;
  const int heads = row < d.n_rows ? p.heads : 0, here = static_cast<int>(min(static_cast<int64_t>(1) << a.t.log_rows, d.n_rows - row0));
  const RotPart t = p.part == 0 ? d.part[0] : p.part == 1 ? d.part[1] : d.part[2];
  const bool two = kTwo && p.turning;
  uint4 lo[BATCH], hi[kTwo ? BATCH : 1], wl, wh;
  griddep_wait();
  {
    const T* src = static_cast<const T*>(t.x) + row * t.x_row + p.head * t.x_head + p.e0;
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      if (b < heads) {
        lo[b] = *reinterpret_cast<const uint4*>(src);
        if constexpr (kTwo)
          if (two) hi[b] = *reinterpret_cast<const uint4*>(src + (p.e1 - p.e0));
      }
      src += t.x_head;
    }
  }
  if ((!PAGED || t.rotate) && heads > 0) {
    const T* gain = static_cast<const T*>(p.part == 0 ? a.d.gain[0] : a.d.gain[1]);
    wl = *reinterpret_cast<const uint4*>(gain + p.e0);
    if (two) wh = *reinterpret_cast<const uint4*>(gain + p.e1);
  }
  [[maybe_unused]] int looked_up = 0;
  if constexpr (PAGED) {
    if (threadIdx.x < here) find_row(a.c, static_cast<int>(row0) + threadIdx.x, &s_pos[threadIdx.x], &looked_up);
    __syncthreads();
  }
  form_angles(d, PAGED ? s_pos : d.positions + row0, a.t.log_rows, here, s_angle);
  if constexpr (PAGED)  // (the page is on its way while angles are formed)
    if (threadIdx.x < here) s_page[threadIdx.x] = checked_row_page(d, a.c, looked_up);
  __syncthreads();
  if (__all_sync(0xffffffffu, heads == 0)) return;
  const int page = PAGED ? s_page[p.rb] : 0;
  const int64_t step = PAGED ? out_step(d, t) : t.out_head;
  T* dst = static_cast<T*>(t.out) + (heads > 0 ? p.head * step + (PAGED ? out_at(d, t, row, s_pos[p.rb], page) : row * t.out_row) + p.e0 : 0);
  const bool write = heads > 0 && !(PAGED && t.paged && page < 0);
  if (PAGED && !t.rotate) {
    // (a warp may have normed heads beside these, so their lanes go on to the sums)
    if (write) {
#pragma unroll
      for (int b = 0; b < BATCH; ++b)
        if (b < heads) {
          *reinterpret_cast<uint4*>(dst + b * step) = lo[b];
          if constexpr (kTwo)
            if (two) *reinterpret_cast<uint4*>(dst + b * step + (p.e1 - p.e0)) = hi[b];
        }
    }
  }
  const bool norm = (!PAGED || t.rotate) && heads > 0;  // values go as they are
  float ss[BATCH];
#pragma unroll
  for (int b = 0; b < BATCH; ++b) {
    uint64_t sum = 0;
    if (norm && b < heads) {
      uint64_t x[P];
      unpack_pairs<T, VEC>(lo[b], x);
#pragma unroll
      for (int i = 0; i < P; ++i) sum = fma_f32x2(x[i], x[i], sum);
      if constexpr (kTwo)
        if (two) {
          unpack_pairs<T, VEC>(hi[b], x);
#pragma unroll
          for (int i = 0; i < P; ++i) sum = fma_f32x2(x[i], x[i], sum);
        }
    }
    ss[b] = sum_f32x2(sum);
  }
  head_sums(ss, a.t.log_lanes);
  if (!norm || !write) return;
  // Gains and angles: x' = x k0 + y k1, y' = y k2 + x k3 (half layout), (x, y) k0 + (y, x) k1 (interleaved); a unit that does not
  // turn has its gain alone.
  uint64_t k0[P], k1[P], k2[H], k3[H];
  unpack_pairs<T, VEC>(wl, k0);
  if (p.turning) {
    float c[INTER ? P : VEC], n[INTER ? P : VEC];
    load_angles(s_angle.cos + p.rb * (d.rot_dim / 2) + p.pair, c);
    load_angles(s_angle.sin + p.rb * (d.rot_dim / 2) + p.pair, n);
    if constexpr (INTER) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        k1[i] = swap_f32x2(mul_f32x2(k0[i], f32x2(n[i], -n[i])));  // (-s w_y, s w_x)
        k0[i] = mul_f32x2(k0[i], f32x2(c[i], c[i]));
      }
    } else {
      unpack_pairs<T, VEC>(wh, k2);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float c0 = c[2 * i], c1 = c[2 * i + 1], n0 = n[2 * i], n1 = n[2 * i + 1];
        k1[i] = mul_f32x2(k2[i], f32x2(-n0, -n1));
        k3[i] = mul_f32x2(k0[i], f32x2(n0, n1));
        k0[i] = mul_f32x2(k0[i], f32x2(c0, c1));
        k2[i] = mul_f32x2(k2[i], f32x2(c0, c1));
      }
    }
  }
  const float eps = p.part == 0 ? a.d.eps[0] : a.d.eps[1];
#pragma unroll
  for (int b = 0; b < BATCH; ++b) {
    if (b < heads) {
      const float r = rsqrtf(ss[b] * a.d.inv_dim + eps);
      const uint64_t r2 = f32x2(r, r);
      uint64_t x[P], o[P];
      unpack_pairs<T, VEC>(lo[b], x);
#pragma unroll
      for (int i = 0; i < P; ++i) x[i] = mul_f32x2(x[i], r2);
      if (!p.turning) {
#pragma unroll
        for (int i = 0; i < P; ++i) o[i] = mul_f32x2(x[i], k0[i]);
      } else if constexpr (INTER) {
#pragma unroll
        for (int i = 0; i < P; ++i) o[i] = fma_f32x2(swap_f32x2(x[i]), k1[i], mul_f32x2(x[i], k0[i]));
      } else {
        uint64_t y[P];
        unpack_pairs<T, VEC>(hi[b], y);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          y[i] = mul_f32x2(y[i], r2);
          o[i] = fma_f32x2(y[i], k1[i], mul_f32x2(x[i], k0[i]));
          y[i] = fma_f32x2(x[i], k3[i], mul_f32x2(y[i], k2[i]));
        }
        *reinterpret_cast<uint4*>(dst + (p.e1 - p.e0)) = pack_pairs<T, VEC>(y);
      }
      *reinterpret_cast<uint4*>(dst) = pack_pairs<T, VEC>(o);
    }
    dst += step;
  }
}

// ---------------------------------------------------------------- forward, a warp a head
// Lane l has the pairs l, l + 32 ... of the part that turns and the elements l, l + 32 ... of the rest.
// Elements of the lane's i-th pair.
__device__ __forceinline__ int2 pair_at(const RotaryDesc& d, int pair) {
  return d.interleaved ? make_int2(2 * pair, 2 * pair + 1) : make_int2(pair, pair + d.rot_dim / 2);
}
template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  float f[1];
  unpack(*reinterpret_cast<const Unit<T, 1>*>(p), f);
  return f[0];
}
template <typename T>
__device__ __forceinline__ void store1(T* p, float v) {
  const float f[1] = {v};
  pack(f, *reinterpret_cast<Unit<T, 1>*>(p));
}

template <typename T>
__global__ void __launch_bounds__(kRotThreads) head_norm_loose_kernel(const __grid_constant__ NormArgs a) {
  __shared__ int s_pos[1], s_page[1];
  __shared__ Angles s_angle;
  griddep_launch_dependents();
  const RotaryDesc& d = a.d.r;
  const int row = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int pairs = d.rot_dim / 2;
  griddep_wait();
  if (threadIdx.x == 0) {
    if (d.positions) {
      s_pos[0] = d.positions[row];
    } else {
      int looked_up;
      find_row(a.c, row, s_pos, &looked_up);
      s_page[0] = checked_row_page(d, a.c, looked_up);
    }
  }
  __syncthreads();
  form_angles(d, s_pos, 0, 1, s_angle);
  __syncthreads();
  const int page = d.positions ? 0 : s_page[0];
  for (int s = warp; s < a.t.slots; s += blockDim.x / 32) {
    const int p = s >= a.t.slot0[2] ? 2 : s >= a.t.slot0[1] ? 1 : 0;
    const RotPart t = p == 0 ? d.part[0] : p == 1 ? d.part[1] : d.part[2];
    const int head = s - (p == 0 ? 0 : p == 1 ? a.t.slot0[1] : a.t.slot0[2]);
    const T* src = static_cast<const T*>(t.x) + row * t.x_row + head * t.x_head;
    if (t.paged && page < 0) continue;
    T* dst = static_cast<T*>(t.out) + head * out_step(d, t) + out_at(d, t, row, s_pos[0], page);
    if (!t.rotate) {
      for (int e = lane; e < d.head_dim; e += 32) dst[e] = src[e];
      continue;
    }
    const T* gain = static_cast<const T*>(p == 0 ? a.d.gain[0] : a.d.gain[1]);
    float x[kLoose], y[kLoose / 2], ss = 0.f;  // the lane's pairs (x, y), then its other elements
#pragma unroll
    for (int i = 0; i < kLoose / 2; ++i)
      if (lane + 32 * i < pairs) {
        const int2 e = pair_at(d, lane + 32 * i);
        x[i] = load1(src + e.x);
        y[i] = load1(src + e.y);
        ss += x[i] * x[i] + y[i] * y[i];
      }
    for (int e = d.rot_dim + lane; e < d.head_dim; e += 32) {
      const float v = load1(src + e);
      ss += v * v;
    }
    const float r = rsqrtf(warp_sum(ss) * a.d.inv_dim + (p == 0 ? a.d.eps[0] : a.d.eps[1]));
#pragma unroll
    for (int i = 0; i < kLoose / 2; ++i)
      if (lane + 32 * i < pairs) {
        const int2 e = pair_at(d, lane + 32 * i);
        const float2 cs = make_float2(s_angle.cos[lane + 32 * i], s_angle.sin[lane + 32 * i]);
        const float u = x[i] * (r * load1(gain + e.x)), v = y[i] * (r * load1(gain + e.y));
        store1(dst + e.x, u * cs.x - v * cs.y);
        store1(dst + e.y, v * cs.x + u * cs.y);
      }
    // (read again: in place, a lane's own elements are still the old ones)
    for (int e = d.rot_dim + lane; e < d.head_dim; e += 32) store1(dst + e, load1(src + e) * (r * load1(gain + e)));
  }
}

// ---------------------------------------------------------------- gradient, 16-byte units
struct NormGradArgs {
  HeadNormGradDesc d;
  Tiling t;
  int row_blocks;           // blocks along the rows: each takes every row_blocks-th tile of rows
  int log_batch;
  float* partial;           // [part][block][head_dim]
};
// A thread's heads: as many as make four units of x and g.
template <bool INTER>
constexpr int kGradBatch = INTER ? 2 : 1;
constexpr int kGradUnits = 4;
// A thread's units of the next two tiles are on their way into places of its own in shared memory: in registers one tile took 128
// of them and two blocks an SM had too few bytes in flight. Angles are formed for a batch of 2^log_batch tiles, so that there is work for
// all threads and a barrier a batch: 16384 bf16 rows of 32 heads took 94 us with a barrier a tile, 82, 77 and 73 with batches of 2, 4 and 8. Positions go four batches ahead, because all threads read what a few of them copied: the next batch's
// have landed, and a barrier has followed, one batch before its angles are formed.
constexpr int kStages = 3, kPositions = 4, kLogBatch = 3;
struct NormGradShared {
  Angles angle[2];
  int pos[kPositions][kRotMaxRows];
};

__device__ __forceinline__ void copy_async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async4(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(kRotThreads, 2) head_norm_grad_kernel(const __grid_constant__ NormGradArgs a) {
  constexpr bool kTwo = !INTER;
  constexpr int P = VEC / 2, H = kTwo ? P : 1, B = kGradBatch<INTER>;
  __shared__ __align__(16) NormGradShared sh;
  extern __shared__ __align__(16) uint4 s_unit[];  // [stage][x, its second or next, g likewise][thread]; then sums [head's lanes][head_dim]
  griddep_launch_dependents();
  const RotaryDesc& d = a.d.r;
  const Place p = place_of<VEC, INTER, B>(a.t, d, threadIdx.x, blockIdx.y);
  const int q = p.part & 1, threads = blockDim.x;
  const RotPart t = q == 0 ? d.part[0] : d.part[1];
  const int64_t g_row = q == 0 ? a.d.g_row[0] : a.d.g_row[1], g_head = q == 0 ? a.d.g_head[0] : a.d.g_head[1];
  const bool second = second_unit<INTER>(p), two = kTwo && second;
  const int e1 = p.e1 - p.e0, log_rows = a.t.log_rows;
  const int64_t tiles = (static_cast<int64_t>(d.n_rows) + (1 << log_rows) - 1) >> log_rows;
  uint64_t acc_x[P], acc_y[H], wx[P], wy[H];
#pragma unroll
  for (int i = 0; i < P; ++i) acc_x[i] = wx[i] = 0;
#pragma unroll
  for (int i = 0; i < H; ++i) acc_y[i] = wy[i] = 0;
  const int64_t first_row = (static_cast<int64_t>(blockIdx.x) << log_rows) + p.rb, jump = static_cast<int64_t>(a.row_blocks) << log_rows;
  // where the thread reads next, two tiles ahead, and writes
  const T* x_at = static_cast<const T*>(t.x) + first_row * t.x_row + p.head * t.x_head + p.e0;
  const T* g_at = static_cast<const T*>(q == 0 ? a.d.grad[0] : a.d.grad[1]) + first_row * g_row + p.head * g_head + p.e0;
  T* o_at = static_cast<T*>(t.out) + first_row * t.out_row + p.head * t.out_head + p.e0;
  const int64_t x_jump = jump * t.x_row, g_jump = jump * g_row, o_jump = jump * t.out_row;
  const int log_all = log_rows + a.log_batch;  // rows of a batch
  int64_t f_row = first_row;
  int64_t pos_row = ((blockIdx.x + static_cast<int64_t>(threadIdx.x >> log_rows) * a.row_blocks) << log_rows) + (threadIdx.x & ((1 << log_rows) - 1));
  const int heads = p.heads;
  griddep_wait();
  auto fetch_pos = [&](int slot) {
    if (threadIdx.x < 1 << log_all && pos_row < d.n_rows) copy_async4(&sh.pos[slot][threadIdx.x], d.positions + pos_row);
    pos_row += jump << a.log_batch;
  };
  auto fetch = [&](int stage) {
    if (f_row < d.n_rows) {
      uint4* to = s_unit + stage * kGradUnits * threads + threadIdx.x;
      if (heads > 0) {
        copy_async16(to, x_at);
        copy_async16(to + 2 * threads, g_at);
      }
      if (second) {
        copy_async16(to + threads, x_at + (kTwo ? e1 : t.x_head));
        copy_async16(to + 3 * threads, g_at + (kTwo ? e1 : g_head));
      }
    }
    f_row += jump;
    x_at += x_jump;
    g_at += g_jump;
  };
  fetch_pos(0);
  fetch_pos(1);
  copy_async_commit();
  fetch_pos(2);
  fetch(0);
  copy_async_commit();
  fetch_pos(3);
  fetch(1);
  copy_async_commit();
  if (heads > 0) {
    const T* gain = static_cast<const T*>(q == 0 ? a.d.gain[0] : a.d.gain[1]);
    unpack_pairs<T, VEC>(*reinterpret_cast<const uint4*>(gain + p.e0), wx);
    if constexpr (kTwo)
      if (two) unpack_pairs<T, VEC>(*reinterpret_cast<const uint4*>(gain + p.e1), wy);
  }
  copy_async_wait<1>();
  __syncthreads();  // the first three batches' positions
  int64_t row = first_row;
  // of the batch from the tile of row `at` on (behind the last row: of no position in particular)
  auto angles = [&](int64_t at, int slot, Angles& to) {
    if (at - p.rb < d.n_rows) form_angles(d, sh.pos[slot], log_all, 1 << log_all, to);
  };
  angles(row, 0, sh.angle[0]);
  __syncthreads();
  int stage = 0, ahead = 2, pos = 0, buffer = 0, in = 0;  // in: the tile of the batch
  for (int64_t tile = blockIdx.x; tile < tiles; tile += a.row_blocks) {
    if (in == 0) fetch_pos(pos);  // (this batch's are free: all have passed the barrier behind them)
    fetch(ahead);
    copy_async_commit();
    copy_async_wait<2>();  // this tile's units; positions of a batch or more ahead
    const int angle = ((in << log_rows) + p.rb) * (d.rot_dim / 2) + p.pair;
    float c[INTER ? P : VEC], n[INTER ? P : VEC];
    if (p.turning) {
      load_angles(sh.angle[buffer].cos + angle, c);
      load_angles(sh.angle[buffer].sin + angle, n);
    }
    const uint4* from = s_unit + stage * kGradUnits * threads + threadIdx.x;
    const int now = row < d.n_rows ? heads : 0;
    // u: the gradient, turned back
    uint64_t x[B][P], y[H], u[B][P], v[H];
    float ss[B], dot[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      uint64_t s2 = 0, d2 = 0;
      if (b < now) {
        unpack_pairs<T, VEC>(from[b * threads], x[b]);
        unpack_pairs<T, VEC>(from[(2 + b) * threads], u[b]);
        if constexpr (kTwo) {
          if (two) {
            unpack_pairs<T, VEC>(from[threads], y);
            unpack_pairs<T, VEC>(from[3 * threads], v);
#pragma unroll
            for (int i = 0; i < P; ++i) {
              const float c0 = c[2 * i], c1 = c[2 * i + 1], n0 = n[2 * i], n1 = n[2 * i + 1];
              const uint64_t g = u[b][i], c2 = f32x2(c0, c1);
              u[b][i] = fma_f32x2(v[i], f32x2(n0, n1), mul_f32x2(g, c2));
              v[i] = fma_f32x2(g, f32x2(-n0, -n1), mul_f32x2(v[i], c2));
              s2 = fma_f32x2(y[i], y[i], s2);
              d2 = fma_f32x2(mul_f32x2(v[i], wy[i]), y[i], d2);
            }
          }
        } else if (p.turning) {
#pragma unroll
          for (int i = 0; i < P; ++i) u[b][i] = fma_f32x2(swap_f32x2(u[b][i]), f32x2(n[i], -n[i]), mul_f32x2(u[b][i], f32x2(c[i], c[i])));
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
          s2 = fma_f32x2(x[b][i], x[b][i], s2);
          d2 = fma_f32x2(mul_f32x2(u[b][i], wx[i]), x[b][i], d2);
        }
      }
      ss[b] = sum_f32x2(s2);
      dot[b] = sum_f32x2(d2);
    }
    head_sums(ss, a.t.log_lanes);
    head_sums(dot, a.t.log_lanes);
    const float eps = q == 0 ? a.d.eps[0] : a.d.eps[1];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (b < now) {
        const float r = rsqrtf(ss[b] * a.d.inv_dim + eps), m = -r * (r * r * (dot[b] * a.d.inv_dim));
        const uint64_t r2 = f32x2(r, r), m2 = f32x2(m, m);
        T* dst = o_at + b * t.out_head;
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const uint64_t ur = mul_f32x2(u[b][i], r2);
          acc_x[i] = fma_f32x2(ur, x[b][i], acc_x[i]);
          u[b][i] = fma_f32x2(ur, wx[i], mul_f32x2(x[b][i], m2));
        }
        *reinterpret_cast<uint4*>(dst) = pack_pairs<T, VEC>(u[b]);
        if constexpr (kTwo)
          if (two) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
              const uint64_t vr = mul_f32x2(v[i], r2);
              acc_y[i] = fma_f32x2(vr, y[i], acc_y[i]);
              v[i] = fma_f32x2(vr, wy[i], mul_f32x2(y[i], m2));
            }
            *reinterpret_cast<uint4*>(dst + e1) = pack_pairs<T, VEC>(v);
          }
      }
    }
    o_at += o_jump;
    row += jump;
    stage = stage == kStages - 1 ? 0 : stage + 1;
    ahead = ahead == kStages - 1 ? 0 : ahead + 1;
    if (++in == 1 << a.log_batch) {
      in = 0;
      buffer ^= 1;
      pos = (pos + 1) & (kPositions - 1);
      angles(row, pos, sh.angle[buffer]);
      __syncthreads();
    }
  }
  copy_async_wait<0>();
  __syncthreads();
  // the block's sums: a head's lanes side by side, then a thread an element, head after head
  float* s_sum = reinterpret_cast<float*>(s_unit);
  float* mine = s_sum + (threadIdx.x >> a.t.log_lanes) * d.head_dim + p.e0;
  if (heads > 0) {
#pragma unroll
    for (int i = 0; i < P; ++i) f32x2_split(acc_x[i], mine[2 * i], mine[2 * i + 1]);
    if constexpr (kTwo)
      if (two) {
#pragma unroll
        for (int i = 0; i < P; ++i) f32x2_split(acc_y[i], mine[e1 + 2 * i], mine[e1 + 2 * i + 1]);
      }
  }
  __syncthreads();
  const int block = blockIdx.y * a.row_blocks + blockIdx.x, blocks = a.row_blocks * gridDim.y;
  const int first = blockIdx.y * a.t.block_slots;  // the block's slots of part 0 come before those of part 1
  const int slots = min(a.t.slots - first, a.t.block_slots);
  const int all = slots << log_rows, split = min(max(a.t.slot0[1] - first, 0), slots) << log_rows;
  for (int i = threadIdx.x; i < d.n_parts * d.head_dim; i += blockDim.x) {
    const int part = i >= d.head_dim, e = i - part * d.head_dim;
    float sum = 0.f;
    for (int g = part ? split : 0; g < (part ? all : split); ++g) sum += s_sum[g * d.head_dim + e];
    a.partial[(static_cast<size_t>(part) * blocks + block) * d.head_dim + e] = sum;
  }
}

struct GradArgs {  // of the loose form
  HeadNormGradDesc d;
  float* partial;           // [part][block][head_dim]
};

// ---------------------------------------------------------------- gradient, a warp a head
template <typename T>
__global__ void __launch_bounds__(kRotThreads) head_norm_grad_loose_kernel(const __grid_constant__ GradArgs a) {
  __shared__ Angles s_angle;
  __shared__ float s_sum[kRotThreads / 32][2 * kMaxPairs];
  griddep_launch_dependents();
  const RotaryDesc& d = a.d.r;
  const int q = blockIdx.y, warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const RotPart t = q == 0 ? d.part[0] : d.part[1];
  const T* gain = static_cast<const T*>(a.d.gain[q]);
  const int pairs = d.rot_dim / 2;
  float acc_x[kLoose / 2], acc_y[kLoose / 2], acc_r[kLoose];
#pragma unroll
  for (int i = 0; i < kLoose / 2; ++i) acc_x[i] = acc_y[i] = 0.f;
#pragma unroll
  for (int i = 0; i < kLoose; ++i) acc_r[i] = 0.f;
  griddep_wait();
  for (int64_t row = blockIdx.x; row < d.n_rows; row += gridDim.x) {
    __syncthreads();  // the angles of the row before have been read
    form_angles(d, d.positions + row, 0, 1, s_angle);
    __syncthreads();
    for (int head = warp; head < t.heads; head += warps) {
      const T* src = static_cast<const T*>(t.x) + row * t.x_row + head * t.x_head;
      const T* grad = static_cast<const T*>(a.d.grad[q]) + row * a.d.g_row[q] + head * a.d.g_head[q];
      T* dst = static_cast<T*>(t.out) + row * t.out_row + head * t.out_head;
      float x[kLoose / 2], y[kLoose / 2], u[kLoose / 2], v[kLoose / 2], xr[kLoose], ur[kLoose], ss = 0.f, dot = 0.f;
#pragma unroll
      for (int i = 0; i < kLoose / 2; ++i)
        if (lane + 32 * i < pairs) {
          const int2 e = pair_at(d, lane + 32 * i);
          const float2 cs = make_float2(s_angle.cos[lane + 32 * i], -s_angle.sin[lane + 32 * i]);
          x[i] = load1(src + e.x);
          y[i] = load1(src + e.y);
          const float g = load1(grad + e.x), h = load1(grad + e.y);
          u[i] = g * cs.x - h * cs.y;
          v[i] = h * cs.x + g * cs.y;
          ss += x[i] * x[i] + y[i] * y[i];
          dot += u[i] * load1(gain + e.x) * x[i] + v[i] * load1(gain + e.y) * y[i];
        }
#pragma unroll
      for (int i = 0; i < kLoose; ++i) {
        const int e = d.rot_dim + lane + 32 * i;
        if (e < d.head_dim) {
          xr[i] = load1(src + e);
          ur[i] = load1(grad + e);
          ss += xr[i] * xr[i];
          dot += ur[i] * load1(gain + e) * xr[i];
        }
      }
      const float r = rsqrtf(warp_sum(ss) * a.d.inv_dim + a.d.eps[q]), c = r * r * (warp_sum(dot) * a.d.inv_dim);
#pragma unroll
      for (int i = 0; i < kLoose / 2; ++i)
        if (lane + 32 * i < pairs) {
          const int2 e = pair_at(d, lane + 32 * i);
          acc_x[i] += u[i] * (x[i] * r);
          acc_y[i] += v[i] * (y[i] * r);
          store1(dst + e.x, r * (u[i] * load1(gain + e.x) - x[i] * c));
          store1(dst + e.y, r * (v[i] * load1(gain + e.y) - y[i] * c));
        }
#pragma unroll
      for (int i = 0; i < kLoose; ++i) {
        const int e = d.rot_dim + lane + 32 * i;
        if (e < d.head_dim) {
          acc_r[i] += ur[i] * (xr[i] * r);
          store1(dst + e, r * (ur[i] * load1(gain + e) - xr[i] * c));
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kLoose / 2; ++i)
    if (lane + 32 * i < pairs) {
      const int2 e = pair_at(d, lane + 32 * i);
      s_sum[warp][e.x] = acc_x[i];
      s_sum[warp][e.y] = acc_y[i];
    }
#pragma unroll
  for (int i = 0; i < kLoose; ++i) {
    const int e = d.rot_dim + lane + 32 * i;
    if (e < d.head_dim) s_sum[warp][e] = acc_r[i];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < d.head_dim; e += blockDim.x) {
    float sum = 0.f;
    for (int w = 0; w < warps; ++w) sum += s_sum[w][e];
    a.partial[(static_cast<size_t>(q) * gridDim.x + blockIdx.x) * d.head_dim + e] = sum;
  }
}

// The blocks' sums of one part's gain: a block 32 elements, each warp every 32nd of the sums.
struct GainArgs {
  const float* partial;  // [part][block][head_dim]
  float* dgain[2];
  int blocks, head_dim;
};
__global__ void __launch_bounds__(1024) head_norm_gain_kernel(const __grid_constant__ GainArgs a) {
  __shared__ float s_sum[32][33];
  griddep_launch_dependents();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, e = blockIdx.x * 32 + lane, q = blockIdx.y;
  const float* partial = a.partial + static_cast<size_t>(q) * a.blocks * a.head_dim;
  griddep_wait();
  float sum = 0.f;
  if (e < a.head_dim) {
#pragma unroll 8
    for (int b = warp; b < a.blocks; b += 32) sum += __ldcg(partial + static_cast<size_t>(b) * a.head_dim + e);
  }
  s_sum[warp][lane] = sum;
  __syncthreads();
  // element `warp` of the block's, over the warps' sums
  sum = warp_sum(s_sum[lane][warp]);
  if (lane == 0 && blockIdx.x * 32 + warp < a.head_dim) (q == 0 ? a.dgain[0] : a.dgain[1])[blockIdx.x * 32 + warp] = sum;
}

// ---------------------------------------------------------------- launches
bool units_align(const RotPart& t, int vec) {
  return t.x_row % vec == 0 && t.x_head % vec == 0 && (reinterpret_cast<uintptr_t>(t.x) & 15) == 0 &&
         (reinterpret_cast<uintptr_t>(t.out) & 15) == 0 && (t.paged || (t.out_row % vec == 0 && t.out_head % vec == 0));
}
// Units of a head in the vector form and the lanes that they take; false where a head has no such form.
bool vector_form(const RotaryDesc& d, int vec, Tiling* a) {
  if (d.head_dim % vec || d.rot_dim % vec || (!d.interleaved && d.rot_dim / 2 % vec)) return false;
  a->rot_units = d.interleaved ? d.rot_dim / vec : d.rot_dim / 2 / vec;
  a->units = a->rot_units + (d.head_dim - d.rot_dim) / vec;
  a->log_lanes = 0;
  while (1 << a->log_lanes < a->units) ++a->log_lanes;
  return a->log_lanes <= 5;
}
// Deals the parts' heads to slots of at most `batch`, and slots and rows to blocks of up to 160 threads (two rows of 72 fill five warps
// where one leaves a quarter of three idle: an append of 3552 rows 14.9 us, 15.2 with up to 128; 256 are slower everywhere else).
void deal_slots(const RotaryDesc& d, int batch, bool few, Tiling* a) {
  a->slots = 0;
  for (int p = 0; p < 3; ++p) {
    a->slot0[p] = a->slots;
    if (p < d.n_parts) a->slots += (d.part[p].heads + batch - 1) / batch;
    else a->slot0[p] = 1 << 30;
  }
  a->block_slots = std::min(a->slots, kRotThreads >> a->log_lanes);
  a->log_rows = 0;
  while (!few && (a->block_slots << a->log_lanes << (a->log_rows + 1)) <= 160 && (2 << a->log_rows) <= kRotMaxRows &&
         (d.rot_dim / 2) << (a->log_rows + 1) <= kRotMaxAngles)
    ++a->log_rows;
}
int block_threads(const Tiling& a) { return ((a.block_slots << a.log_lanes << a.log_rows) + 31) / 32 * 32; }
unsigned columns_of(const Tiling& a) { return (a.slots + a.block_slots - 1) / a.block_slots; }

template <typename T, int BATCH>
cudaError_t launch_units(const NormArgs& a, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(a.d.r.n_rows) + (1 << a.t.log_rows) - 1) >> a.t.log_rows), columns_of(a.t));
  const dim3 block(block_threads(a.t));
  if constexpr (std::is_same_v<T, __nv_bfloat16>)  // as caches are
    if (!a.d.r.positions)
      return a.d.r.interleaved ? launch_kernel(head_norm_kernel<T, VEC, true, BATCH, true>, grid, block, 0, stream, a)
                               : launch_kernel(head_norm_kernel<T, VEC, false, BATCH, true>, grid, block, 0, stream, a);
  return a.d.r.interleaved ? launch_kernel(head_norm_kernel<T, VEC, true, BATCH, false>, grid, block, 0, stream, a)
                           : launch_kernel(head_norm_kernel<T, VEC, false, BATCH, false>, grid, block, 0, stream, a);
}
template <typename T>
cudaError_t launch_norm(NormArgs& a, int num_sms, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  const RotaryDesc& d = a.d.r;
  bool vec = vector_form(d, VEC, &a.t);
  for (int p = 0; p < d.n_parts; ++p)
    vec = vec && units_align(d.part[p], VEC) && (!d.part[p].rotate || (reinterpret_cast<uintptr_t>(a.d.gain[p]) & 15) == 0);
  PdlScope pdl;
  if (!vec) {
    a.t.log_lanes = 5;
    deal_slots(d, 1, true, &a.t);
    const int threads = std::min(kRotThreads, 32 * a.t.slots);
    return launch_kernel(head_norm_loose_kernel<T>, dim3(d.n_rows), dim3(threads), 0, stream, a);
  }
  // as in rotary.cu: four heads a thread where the rows alone fill the SMs, one where they are few
  const bool few = d.n_rows < 4 * num_sms;
  if (few) {
    deal_slots(d, 1, true, &a.t);
    if (a.t.slots <= 4096) return launch_units<T, 1>(a, stream);  // (more: keep the grid's second axis short)
  }
  deal_slots(d, kNormBatch, few, &a.t);
  return launch_units<T, kNormBatch>(a, stream);
}

// Sums of a gradient's blocks, two parts, to join.
int most_blocks(int num_sms) { return 8 * num_sms; }

template <typename T, bool INTER>
cudaError_t launch_grad_units(const NormGradArgs& a, int threads, int columns, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T), kMost = kStages * kGradUnits * kRotThreads * 16;
  static PerDevice once;
  int dev = 0;
  if (once.pending(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(head_norm_grad_kernel<T, VEC, INTER>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    once.done(dev);
  }
  // (the sums need less: 64 bytes of a thread's two heads or two halves)
  return launch_kernel(head_norm_grad_kernel<T, VEC, INTER>, dim3(a.row_blocks, columns), dim3(threads), kStages * kGradUnits * threads * 16, stream, a);
}
template <typename T>
cudaError_t launch_grad(const HeadNormGradDesc& g, float* partial, int num_sms, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  const RotaryDesc& d = g.r;
  NormGradArgs a;
  std::memset(&a, 0, sizeof(a));
  bool vec = vector_form(d, VEC, &a.t);
  for (int p = 0; p < d.n_parts; ++p)
    vec = vec && units_align(d.part[p], VEC) && g.g_row[p] % VEC == 0 && g.g_head[p] % VEC == 0 &&
          ((reinterpret_cast<uintptr_t>(g.gain[p]) | reinterpret_cast<uintptr_t>(g.grad[p])) & 15) == 0;
  if (vec) {
    deal_slots(d, d.interleaved ? kGradBatch<true> : kGradBatch<false>, d.n_rows < 4 * num_sms, &a.t);
    vec = static_cast<int>(columns_of(a.t)) <= most_blocks(num_sms) / 8;
  }
  PdlScope pdl;
  cudaError_t e;
  GainArgs sums{partial, {g.dgain[0], g.dgain[1]}, 0, d.head_dim};
  if (vec) {
    a.d = g;
    a.partial = partial;
    // as many blocks as are resident at a time: two of 256 threads an SM (their registers), four of 128
    const int columns = static_cast<int>(columns_of(a.t)), threads = block_threads(a.t), resident = std::min(8, 2 * kRotThreads / threads);
    const int64_t tiles = (static_cast<int64_t>(d.n_rows) + (1 << a.t.log_rows) - 1) >> a.t.log_rows;
    a.row_blocks = static_cast<int>(std::min<int64_t>(tiles, std::max(1, resident * num_sms / columns)));
    sums.blocks = a.row_blocks * columns;
    while (a.log_batch < kLogBatch && tiles >> a.log_batch > a.row_blocks && (1 << (a.t.log_rows + a.log_batch + 1)) <= kRotMaxRows &&
           (d.rot_dim / 2) << (a.t.log_rows + a.log_batch + 1) <= kRotMaxAngles)
      ++a.log_batch;
    e = d.interleaved ? launch_grad_units<T, true>(a, threads, columns, stream) : launch_grad_units<T, false>(a, threads, columns, stream);
  } else {
    sums.blocks = std::min(d.n_rows, 4 * num_sms);
    const GradArgs l{g, partial};
    e = launch_kernel(head_norm_grad_loose_kernel<T>, dim3(sums.blocks, d.n_parts), dim3(kRotThreads), 0, stream, l);
  }
  if (e != cudaSuccess) return e;
  return launch_kernel(head_norm_gain_kernel, dim3((d.head_dim + 31) / 32, d.n_parts), dim3(1024), 0, stream, sums);
}

}  // namespace

cudaError_t launch_head_norm(const HeadNormDesc& d, const ChunkTable* chunks, int num_sms, cudaStream_t stream) {
  if (d.r.n_rows < 1) return cudaSuccess;
  NormArgs a;
  std::memset(&a, 0, sizeof(a));
  a.d = d;
  if (chunks) a.c = *chunks;
  switch (d.r.type) {
    case CRF_BF16: return launch_norm<__nv_bfloat16>(a, num_sms, stream);
    case CRF_FP16: return launch_norm<__half>(a, num_sms, stream);
    case CRF_FP32: return launch_norm<float>(a, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

size_t head_norm_grad_workspace(int head_dim, int num_sms) {
  return 2 * static_cast<size_t>(most_blocks(num_sms)) * head_dim * sizeof(float);
}

cudaError_t launch_head_norm_grad(const HeadNormGradDesc& d, float* partial, int num_sms, cudaStream_t stream) {
  if (d.r.n_rows < 1) {
    for (int p = 0; p < d.r.n_parts; ++p) {
      const cudaError_t e = cudaMemsetAsync(d.dgain[p], 0, d.r.head_dim * sizeof(float), stream);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  switch (d.r.type) {
    case CRF_BF16: return launch_grad<__nv_bfloat16>(d, partial, num_sms, stream);
    case CRF_FP16: return launch_grad<__half>(d, partial, num_sms, stream);
    case CRF_FP32: return launch_grad<float>(d, partial, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace crf
