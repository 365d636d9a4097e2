// RMS norms of query and key heads with the position rotation in the same pass, and the gradient. For a head x of n
// elements with gain w, r = 1 / sqrt(mean(x^2) + eps), and R the rotation at the row's position (rotary.cu):
//   y = R (w x r)                                        (products element by element)
// and for the gradient g of y, with u = R^T g and v = w u:
//   dw = sum over rows and heads of u x r,   dx = r (v - x r^2 mean(v x)).
// Sums and products are fp32; y and dx are rounded once to the type, dw stays fp32. The forward form also writes keys and
// values of new rows into the pages of a layer (values neither normed nor turned).
//
// Bound by memory: every element is read once and written once. As in rotary.cu a thread owns one 16-byte unit of a head (for
// the half layout two, the pair's halves); here the lanes of a head, a power of two, are neighbours in a warp and join the sum
// of squares by shuffles. Heads whose units are no such thing (odd sizes, strides or alignments) take a warp each, an element
// or a pair a lane.
//
// The gains' gradient: a thread keeps the same elements of its part's heads over all the rows that its block walks, so
// their sums stay in its registers; a block's sums meet in shared memory, the blocks' in a second small kernel, both in a
// fixed order: the same inputs give the same bits.
#include "../../include/crf.h"
#include "rotary.cuh"

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

constexpr int kNormBatch = 4;   // heads of a thread, at most
constexpr int kGradBatch = 2;
constexpr int kMaxGradColumns = 4;  // blocks side by side over a row's heads
constexpr int kLoose = 8;       // elements of a lane in the form of a warp a head: 256 / 32

struct NormArgs {
  HeadNormDesc d;
  ChunkTable c;
  int lanes;                // of a head, a power of two
  int units, rot_units;     // 16-byte units of a head, those that rotate
  int rows;                 // of a block
  int batch;                // heads of a slot
  int slot0[3];             // each part's first slot
  int slots, block_slots;   // of all parts; of a block
};

// Sum over the `lanes` neighbours that share a head.
__device__ __forceinline__ float head_sum(float v, int lanes) {
  for (int o = lanes / 2; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A thread's place: unit u of head slot `slot` of row `row`.
struct Place {
  int u, rb, slot, part, head, heads;
  bool turning;
  int e0, e1;  // first elements of its piece(s)
};
template <int VEC, bool INTER, typename Args>
__device__ __forceinline__ Place place_of(const Args& a, const RotaryDesc& d) {
  Place t;
  t.u = threadIdx.x % a.lanes;
  const int rest = threadIdx.x / a.lanes;
  t.rb = rest % a.rows;
  t.slot = rest / a.rows + blockIdx.y * a.block_slots;
  const bool there = rest / a.rows < a.block_slots && t.slot < a.slots && t.u < a.units;
  t.part = t.slot >= a.slot0[2] ? 2 : t.slot >= a.slot0[1] ? 1 : 0;
  const int first = t.part == 0 ? 0 : t.part == 1 ? a.slot0[1] : a.slot0[2];
  const int all = t.part == 0 ? d.part[0].heads : t.part == 1 ? d.part[1].heads : d.part[2].heads;
  t.head = (t.slot - first) * a.batch;
  t.heads = there ? min(a.batch, all - t.head) : 0;
  t.turning = t.u < a.rot_units;
  t.e0 = t.turning ? t.u * VEC : d.rot_dim + (t.u - a.rot_units) * VEC;
  t.e1 = t.turning && !INTER ? t.e0 + d.rot_dim / 2 : t.e0;
  return t;
}

// Angles of `here` rows from row0 on: [row][pair].
__device__ __forceinline__ void form_angles(const RotaryDesc& d, const int* pos, int here, float2* angle) {
  const int pairs = d.rot_dim / 2;
  for (int i = threadIdx.x; i < here * pairs; i += blockDim.x) {
    const int k = i / here, r = i - k * here;  // lanes of a warp share few pairs
    const float2 t = turn_cos_sin(static_cast<uint64_t>(static_cast<int64_t>(pos[r])) * d.turns[k]);
    angle[r * pairs + k] = make_float2(t.x * d.magnitude, (d.inverse ? -t.y : t.y) * d.magnitude);
  }
}
// Positions, and the pages of rows that go into a cache (-1: no page of the pool).
__device__ __forceinline__ void find_row(const RotaryDesc& d, const ChunkTable& c, int r, int* pos, int* page) {
  *page = 0;
  if (d.positions) {
    *pos = d.positions[r];
    return;
  }
  const int i = chunk_of_row(c, r);
  *pos = c.pos[i] + (r - c.row0[i]);
  *page = c.pt[i][*pos / kPage];
  if (*page < 0 || *page >= c.num_pages) {
    if (d.status) atomicOr(d.status, kStatusBounds);
    *page = -1;  // its writes are left out
  }
}
// Where a part's row goes, and the step from head to head.
__device__ __forceinline__ int64_t out_at(const RotaryDesc& d, const RotPart& t, int64_t row, int pos, int page) {
  return t.paged ? (static_cast<int64_t>(page) * d.n_kv_heads * kPage + pos % kPage) * d.head_dim : row * t.out_row;
}
__device__ __forceinline__ int64_t out_step(const RotaryDesc& d, const RotPart& t) {
  return t.paged ? static_cast<int64_t>(kPage) * d.head_dim : t.out_head;
}

// The pair(s) of two pieces, or of one with its pairs side by side.
template <int VEC, bool INTER>
__device__ __forceinline__ void turn(float (&x)[VEC], float (&y)[VEC], const float2* cs) {
#pragma unroll
  for (int i = 0; i < (INTER ? VEC / 2 : VEC); ++i) {
    float& a = INTER ? x[(2 * i) % VEC] : x[i];
    float& b = INTER ? x[(2 * i + 1) % VEC] : y[i];
    const float af = a, bf = b;
    a = af * cs[i].x - bf * cs[i].y;
    b = bf * cs[i].x + af * cs[i].y;
  }
}

// ---------------------------------------------------------------- forward, 16-byte units
template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(kRotThreads) head_norm_kernel(const __grid_constant__ NormArgs a) {
  using U = Unit<T, VEC>;
  constexpr bool kTwo = !INTER;
  constexpr int kPairs = INTER ? VEC / 2 : VEC;
  __shared__ int s_pos[kRotMaxRows], s_page[kRotMaxRows];
  __shared__ float2 s_angle[kRotMaxAngles];
  griddep_launch_dependents();
  const RotaryDesc& d = a.d.r;
  const Place p = place_of<VEC, INTER>(a, d);
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * a.rows, row = row0 + p.rb;
  const int heads = row < d.n_rows ? p.heads : 0;
  const RotPart t = p.part == 0 ? d.part[0] : p.part == 1 ? d.part[1] : d.part[2];
  const T* gain = static_cast<const T*>(p.part == 0 ? a.d.gain[0] : p.part == 1 ? a.d.gain[1] : nullptr);
  const float eps = p.part == 0 ? a.d.eps[0] : a.d.eps[1];
  const bool two = kTwo && p.turning;
  U lo[kNormBatch], hi[kNormBatch], wl, wh;
  griddep_wait();
  {
    const T* src = static_cast<const T*>(t.x) + row * t.x_row + p.head * t.x_head;
#pragma unroll
    for (int b = 0; b < kNormBatch; ++b) {
      if (b < heads) {
        lo[b] = *reinterpret_cast<const U*>(src + p.e0);
        if (two) hi[b] = *reinterpret_cast<const U*>(src + p.e1);
      }
      src += t.x_head;
    }
  }
  if (gain && heads > 0) {
    wl = *reinterpret_cast<const U*>(gain + p.e0);
    if (two) wh = *reinterpret_cast<const U*>(gain + p.e1);
  }
  if (threadIdx.x < a.rows && row0 + threadIdx.x < d.n_rows)
    find_row(d, a.c, static_cast<int>(row0) + threadIdx.x, &s_pos[threadIdx.x], &s_page[threadIdx.x]);
  __syncthreads();
  form_angles(d, s_pos, static_cast<int>(min(static_cast<int64_t>(a.rows), d.n_rows - row0)), s_angle);
  __syncthreads();
  const int page = s_page[p.rb];
  const bool rotate = p.turning && t.rotate;
  float2 cs[kPairs];
  if (rotate && heads > 0) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) cs[i] = s_angle[p.rb * (d.rot_dim / 2) + p.u * kPairs + i];
  }
  const int64_t step = out_step(d, t);
  T* dst = static_cast<T*>(t.out) + (heads > 0 ? p.head * step + out_at(d, t, row, s_pos[p.rb], page) : 0);
  const bool write = heads > 0 && !(t.paged && page < 0);
#pragma unroll
  for (int b = 0; b < kNormBatch; ++b) {
    float x[VEC], y[VEC], ss = 0.f;
    if (b < heads && t.rotate) {
      unpack(lo[b], x);
      if (two) unpack(hi[b], y);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        ss += x[i] * x[i];
        if (two) ss += y[i] * y[i];
      }
    }
    ss = head_sum(ss, a.lanes);  // every lane takes part
    if (b < heads && write) {
      if (t.rotate) {
        const float r = rsqrtf(ss * a.d.inv_dim + eps);
        float w[VEC];
        unpack(wl, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] *= r * w[i];
        if (two) {
          unpack(wh, w);
#pragma unroll
          for (int i = 0; i < VEC; ++i) y[i] *= r * w[i];
        }
        if (rotate) turn<VEC, INTER>(x, y, cs);
        pack(x, lo[b]);
        if (two) pack(y, hi[b]);
      }
      *reinterpret_cast<U*>(dst + p.e0) = lo[b];
      if (two) *reinterpret_cast<U*>(dst + p.e1) = hi[b];
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
  __shared__ float2 s_angle[kMaxPairs];
  griddep_launch_dependents();
  const RotaryDesc& d = a.d.r;
  const int row = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int pairs = d.rot_dim / 2;
  griddep_wait();
  if (threadIdx.x == 0) find_row(d, a.c, row, s_pos, s_page);
  __syncthreads();
  form_angles(d, s_pos, 1, s_angle);
  __syncthreads();
  const int page = s_page[0];
  for (int s = warp; s < a.slots; s += blockDim.x / 32) {
    const int p = s >= a.slot0[2] ? 2 : s >= a.slot0[1] ? 1 : 0;
    const RotPart t = p == 0 ? d.part[0] : p == 1 ? d.part[1] : d.part[2];
    const int head = s - (p == 0 ? 0 : p == 1 ? a.slot0[1] : a.slot0[2]);
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
        const float2 cs = s_angle[lane + 32 * i];
        const float u = x[i] * (r * load1(gain + e.x)), v = y[i] * (r * load1(gain + e.y));
        store1(dst + e.x, u * cs.x - v * cs.y);
        store1(dst + e.y, v * cs.x + u * cs.y);
      }
    // (read again: in place, a lane's own elements are still the old ones)
    for (int e = d.rot_dim + lane; e < d.head_dim; e += 32) store1(dst + e, load1(src + e) * (r * load1(gain + e)));
  }
}

// ---------------------------------------------------------------- gradient, 16-byte units
struct GradArgs {
  HeadNormGradDesc d;
  int lanes, units, rot_units;
  int rows, batch, slot0[3], slots, block_slots;
  int row_blocks;           // blocks along the rows: each takes every row_blocks-th group of rows
  float* partial;           // [part][block][head_dim]
};

template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(kRotThreads) head_norm_grad_kernel(const __grid_constant__ GradArgs a) {
  using U = Unit<T, VEC>;
  constexpr bool kTwo = !INTER;
  constexpr int kPairs = INTER ? VEC / 2 : VEC;
  __shared__ int s_pos[kRotMaxRows];
  __shared__ float2 s_angle[kRotMaxAngles];
  extern __shared__ float s_sum[];  // [lane group][head_dim]
  griddep_launch_dependents();
  const RotaryDesc& d = a.d.r;
  const Place p = place_of<VEC, INTER>(a, d);
  const RotPart t = p.part == 0 ? d.part[0] : d.part[1];
  const T* gain = static_cast<const T*>(a.d.gain[p.part & 1]);
  const float eps = a.d.eps[p.part & 1];
  const int64_t g_row = a.d.g_row[p.part & 1], g_head = a.d.g_head[p.part & 1];
  const bool two = kTwo && p.turning;
  float acc_lo[VEC], acc_hi[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) acc_lo[i] = acc_hi[i] = 0.f;
  griddep_wait();
  U wl, wh;
  if (p.heads > 0) {
    wl = *reinterpret_cast<const U*>(gain + p.e0);
    if (two) wh = *reinterpret_cast<const U*>(gain + p.e1);
  }
  for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * a.rows; row0 < d.n_rows; row0 += static_cast<int64_t>(a.row_blocks) * a.rows) {
    const int64_t row = row0 + p.rb;
    const int heads = row < d.n_rows ? p.heads : 0;
    U xl[kGradBatch], xh[kGradBatch], gl[kGradBatch], gh[kGradBatch];
    {
      const T* src = static_cast<const T*>(t.x) + row * t.x_row + p.head * t.x_head;
      const T* grad = static_cast<const T*>(a.d.grad[p.part & 1]) + row * g_row + p.head * g_head;
#pragma unroll
      for (int b = 0; b < kGradBatch; ++b) {
        if (b < heads) {
          xl[b] = *reinterpret_cast<const U*>(src + p.e0);
          gl[b] = *reinterpret_cast<const U*>(grad + p.e0);
          if (two) {
            xh[b] = *reinterpret_cast<const U*>(src + p.e1);
            gh[b] = *reinterpret_cast<const U*>(grad + p.e1);
          }
        }
        src += t.x_head;
        grad += g_head;
      }
    }
    if (threadIdx.x < a.rows && row0 + threadIdx.x < d.n_rows) s_pos[threadIdx.x] = d.positions[row0 + threadIdx.x];
    __syncthreads();
    form_angles(d, s_pos, static_cast<int>(min(static_cast<int64_t>(a.rows), d.n_rows - row0)), s_angle);
    __syncthreads();
    float2 cs[kPairs];
    if (p.turning && heads > 0) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) cs[i] = s_angle[p.rb * (d.rot_dim / 2) + p.u * kPairs + i];
    }
    T* dst = static_cast<T*>(t.out) + row * t.out_row + p.head * t.out_head;
#pragma unroll
    for (int b = 0; b < kGradBatch; ++b) {
      float x[VEC], y[VEC], u[VEC], v[VEC], w[VEC], ss = 0.f, dot = 0.f;
      if (b < heads) {
        unpack(xl[b], x);
        unpack(gl[b], u);
        if (two) {
          unpack(xh[b], y);
          unpack(gh[b], v);
        }
        if (p.turning) turn<VEC, INTER>(u, v, cs);
        unpack(wl, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          ss += x[i] * x[i];
          dot += u[i] * w[i] * x[i];
        }
        if (two) {
          unpack(wh, w);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            ss += y[i] * y[i];
            dot += v[i] * w[i] * y[i];
          }
        }
      }
      ss = head_sum(ss, a.lanes);
      dot = head_sum(dot, a.lanes);
      if (b < heads) {
        const float r = rsqrtf(ss * a.d.inv_dim + eps), c = r * r * (dot * a.d.inv_dim);
        unpack(wl, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          acc_lo[i] += u[i] * (x[i] * r);
          u[i] = r * (u[i] * w[i] - x[i] * c);
        }
        pack(u, xl[b]);
        *reinterpret_cast<U*>(dst + p.e0) = xl[b];
        if (two) {
          unpack(wh, w);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            acc_hi[i] += v[i] * (y[i] * r);
            v[i] = r * (v[i] * w[i] - y[i] * c);
          }
          pack(v, xh[b]);
          *reinterpret_cast<U*>(dst + p.e1) = xh[b];
        }
      }
      dst += t.out_head;
    }
    // (the next rows' positions are written behind the reads of this round's: the angles' barrier lies between; the
    // angles themselves are written behind the next round's first barrier)
  }
  // the block's sums: lane groups side by side, then a thread an element, group after group
  float* mine = s_sum + threadIdx.x / a.lanes * d.head_dim;
  if (p.u < a.units) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      mine[p.e0 + i] = acc_lo[i];
      if (two) mine[p.e1 + i] = acc_hi[i];
    }
  }
  __syncthreads();
  const int block = blockIdx.y * a.row_blocks + blockIdx.x, blocks = a.row_blocks * gridDim.y;
  const int first = blockIdx.y * a.block_slots;  // the block's slots of part 0 come before those of part 1
  const int split = min(max(a.slot0[1] - first, 0), a.block_slots) * a.rows, all = min(a.slots - first, a.block_slots) * a.rows;
  for (int i = threadIdx.x; i < d.n_parts * d.head_dim; i += blockDim.x) {
    const int q = i / d.head_dim, e = i - q * d.head_dim;
    float sum = 0.f;
    for (int g = q ? split : 0; g < (q ? all : min(split, all)); ++g) sum += s_sum[g * d.head_dim + e];
    a.partial[(static_cast<size_t>(q) * blocks + block) * d.head_dim + e] = sum;
  }
}

// ---------------------------------------------------------------- gradient, a warp a head
template <typename T>
__global__ void __launch_bounds__(kRotThreads) head_norm_grad_loose_kernel(const __grid_constant__ GradArgs a) {
  __shared__ float2 s_angle[kMaxPairs];
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
  for (int64_t row = blockIdx.x; row < d.n_rows; row += a.row_blocks) {
    __syncthreads();  // the angles of the row before have been read
    form_angles(d, d.positions + row, 1, s_angle);
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
          const float2 cs = s_angle[lane + 32 * i];
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
    a.partial[(static_cast<size_t>(q) * a.row_blocks + blockIdx.x) * d.head_dim + e] = sum;
  }
}

// The blocks' sums of one part's gain: a warp takes eight elements, four lanes to each.
struct GainArgs {
  const float* partial;  // [part][block][head_dim]
  float* dgain[2];
  int blocks, head_dim;
};
__global__ void __launch_bounds__(256) head_norm_gain_kernel(const __grid_constant__ GainArgs a) {
  __shared__ float s_sum[8][32];
  griddep_launch_dependents();
  const int lane = threadIdx.x % 32, group = threadIdx.x / 32, e = blockIdx.x * 32 + lane, q = blockIdx.y;
  griddep_wait();
  float sum = 0.f;
  if (e < a.head_dim) {
    const float* at = a.partial + static_cast<size_t>(q) * a.blocks * a.head_dim + e;
    for (int b = group; b < a.blocks; b += 8) sum += __ldcg(at + static_cast<size_t>(b) * a.head_dim);
  }
  s_sum[group][lane] = sum;
  __syncthreads();
  if (group == 0 && e < a.head_dim) {
#pragma unroll
    for (int g = 1; g < 8; ++g) sum += s_sum[g][lane];
    (q == 0 ? a.dgain[0] : a.dgain[1])[e] = sum;
  }
}

// ---------------------------------------------------------------- launches
bool units_align(const RotPart& t, int vec) {
  return t.x_row % vec == 0 && t.x_head % vec == 0 && (reinterpret_cast<uintptr_t>(t.x) & 15) == 0 &&
         (reinterpret_cast<uintptr_t>(t.out) & 15) == 0 && (t.paged || (t.out_row % vec == 0 && t.out_head % vec == 0));
}
// Units of a head in the vector form and the lanes that they take; false where a head has no such form.
template <typename Args>
bool vector_form(const RotaryDesc& d, int vec, Args* a) {
  if (d.head_dim % vec || d.rot_dim % vec || (!d.interleaved && d.rot_dim / 2 % vec)) return false;
  a->rot_units = d.interleaved ? d.rot_dim / vec : d.rot_dim / 2 / vec;
  a->units = a->rot_units + (d.head_dim - d.rot_dim) / vec;
  a->lanes = 1;
  while (a->lanes < a->units) a->lanes *= 2;
  return a->lanes <= 32;
}
// Deals the parts' heads to slots of at most `batch`, and slots and rows to blocks of about `threads` threads.
template <typename Args>
void deal_slots(const RotaryDesc& d, int batch, bool few, int threads, Args* a) {
  a->batch = batch;
  a->slots = 0;
  for (int p = 0; p < 3; ++p) {
    a->slot0[p] = a->slots;
    if (p < d.n_parts) a->slots += (d.part[p].heads + batch - 1) / batch;
    else a->slot0[p] = 1 << 30;
  }
  a->block_slots = std::min(a->slots, kRotThreads / a->lanes);
  a->rows = few ? 1 : std::max(1, std::min(kRotMaxRows, threads / (a->lanes * a->block_slots)));
}
template <typename Args>
int block_threads(const Args& a) {
  return (a.lanes * a.block_slots * a.rows + 31) / 32 * 32;
}

template <typename T>
cudaError_t launch_norm(NormArgs& a, int num_sms, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  const RotaryDesc& d = a.d.r;
  bool vec = vector_form(d, VEC, &a);
  for (int p = 0; p < d.n_parts; ++p)
    vec = vec && units_align(d.part[p], VEC) && (!d.part[p].rotate || (reinterpret_cast<uintptr_t>(a.d.gain[p]) & 15) == 0);
  PdlScope pdl;
  if (!vec) {
    a.lanes = 32;
    deal_slots(d, 1, true, 32, &a);
    const int threads = std::min(kRotThreads, 32 * a.slots);
    return launch_kernel(head_norm_loose_kernel<T>, dim3(d.n_rows), dim3(threads), 0, stream, a);
  }
  // as in rotary.cu: slots of four heads where the rows alone fill the SMs, of one where they are few
  const bool few = d.n_rows < 4 * num_sms;
  deal_slots(d, few ? 1 : kNormBatch, few, 128, &a);
  if (few && a.slots > 4096) deal_slots(d, kNormBatch, few, 128, &a);  // keep the grid's second axis short
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(d.n_rows) + a.rows - 1) / a.rows),
                  (a.slots + a.block_slots - 1) / a.block_slots);
  return d.interleaved ? launch_kernel(head_norm_kernel<T, VEC, true>, grid, dim3(block_threads(a)), 0, stream, a)
                       : launch_kernel(head_norm_kernel<T, VEC, false>, grid, dim3(block_threads(a)), 0, stream, a);
}

// Blocks along the rows of a gradient, and so sums to join: up to six an SM.
int row_blocks_of(int64_t groups, int num_sms) { return static_cast<int>(std::min<int64_t>(groups, 6 * num_sms)); }

template <typename T>
cudaError_t launch_grad(GradArgs& a, int num_sms, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  const RotaryDesc& d = a.d.r;
  bool vec = vector_form(d, VEC, &a);
  for (int p = 0; p < d.n_parts; ++p)
    vec = vec && units_align(d.part[p], VEC) && a.d.g_row[p] % VEC == 0 && a.d.g_head[p] % VEC == 0 &&
          ((reinterpret_cast<uintptr_t>(a.d.gain[p]) | reinterpret_cast<uintptr_t>(a.d.grad[p])) & 15) == 0;
  PdlScope pdl;
  int blocks;
  cudaError_t e;
  if (vec) {
    const bool few = d.n_rows < 4 * num_sms;
    deal_slots(d, kGradBatch, few, 128, &a);
    vec = a.slots <= a.block_slots * kMaxGradColumns;
  }
  if (vec) {
    const int columns = (a.slots + a.block_slots - 1) / a.block_slots;
    a.row_blocks = row_blocks_of((static_cast<int64_t>(d.n_rows) + a.rows - 1) / a.rows, num_sms);
    blocks = a.row_blocks * columns;
    const int threads = block_threads(a);
    const size_t smem = static_cast<size_t>(threads / a.lanes) * d.head_dim * sizeof(float);  // at most 16 KB
    const dim3 grid(a.row_blocks, columns);
    e = d.interleaved ? launch_kernel(head_norm_grad_kernel<T, VEC, true>, grid, dim3(threads), smem, stream, a)
                      : launch_kernel(head_norm_grad_kernel<T, VEC, false>, grid, dim3(threads), smem, stream, a);
  } else {
    a.row_blocks = blocks = row_blocks_of(d.n_rows, num_sms);
    e = launch_kernel(head_norm_grad_loose_kernel<T>, dim3(blocks, d.n_parts), dim3(kRotThreads), 0, stream, a);
  }
  if (e != cudaSuccess) return e;
  GainArgs g{a.partial, {a.d.dgain[0], a.d.dgain[1]}, blocks, d.head_dim};
  return launch_kernel(head_norm_gain_kernel, dim3((d.head_dim + 31) / 32, d.n_parts), dim3(256), 0, stream, g);
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

size_t head_norm_grad_workspace(int n_rows, int head_dim, int num_sms) {
  return 2ull * kMaxGradColumns * row_blocks_of(n_rows, num_sms) * head_dim * sizeof(float);
}

cudaError_t launch_head_norm_grad(const HeadNormGradDesc& d, float* partial, int num_sms, cudaStream_t stream) {
  if (d.r.n_rows < 1) {
    for (int p = 0; p < d.r.n_parts; ++p) {
      const cudaError_t e = cudaMemsetAsync(d.dgain[p], 0, d.r.head_dim * sizeof(float), stream);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  GradArgs a;
  std::memset(&a, 0, sizeof(a));
  a.d = d;
  a.partial = partial;
  switch (d.r.type) {
    case CRF_BF16: return launch_grad<__nv_bfloat16>(a, num_sms, stream);
    case CRF_FP16: return launch_grad<__half>(a, num_sms, stream);
    case CRF_FP32: return launch_grad<float>(a, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace crf
