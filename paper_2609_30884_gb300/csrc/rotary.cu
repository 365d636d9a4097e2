// Rotary positions of query and key heads, and the write of new rows' keys and values into the pages of a
// layer: pair (x, y) of a head at position p becomes magnitude (x cos - y sin, y cos + x sin) of the angle
// p f, with f the pair's radians a position; the inverse map takes -sin (the transpose, hence the gradient).
//
// Angles: f / 2 pi is a fraction of a turn, held as a 64-bit integer in units of 2^-64 turns, so the product
// with the position drops whole turns by itself (integer arithmetic modulo 2^64) and is exact for the held f:
// at p = 2^31 the angle is off by at most 2^-33 turns. Its top 32 bits are split into a quadrant and a
// remainder of at most an eighth of a turn, whose sine and cosine are fp32 functions.
//
// Bound by memory: every element is read once and written once. A thread owns one 16-byte unit of a row (for the
// half layout two, the pair's halves) and every hg-th of its heads, the first kRotBatch of them asked for before the
// angles are formed. The block's angles are formed once, in shared memory, for all heads of its rows.
#include "../../include/crf.h"
#include "common.cuh"
#include "extend.h"

#include <cuda_fp16.h>

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotBatch = 4;        // heads in flight
constexpr int kRotMaxRows = 32;     // of a block
constexpr int kRotMaxAngles = 2048; // of a block: at most 8 a thread

struct RotaryArgs {
  RotaryDesc d;
  ChunkTable c;
  int units, rot_units, rows_per_block, head_slots, heads;
};

// Request of packed row r.
__device__ __forceinline__ int chunk_of_row(const ChunkTable& c, int r) {
  int lo = 0, hi = c.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (c.row0[mid] <= r) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// (cos, sin) of `turn` x 2^-64 turns.
__device__ __forceinline__ float2 turn_cos_sin(uint64_t turn) {
  const int s = static_cast<int>(static_cast<uint32_t>(turn >> 32));
  const int q = static_cast<int>((static_cast<uint32_t>(s) + 0x20000000u) >> 30);  // nearest quarter turn
  const int rem = static_cast<int>(static_cast<uint32_t>(s) - (static_cast<uint32_t>(q) << 30));
  const float x = static_cast<float>(rem) * 4.656612873077393e-10f;  // half turns: 2^-31
  float sn, cs;
  sincospif(x, &sn, &cs);
  const float c = (q & 1) ? sn : cs, n = (q & 1) ? cs : sn;
  return make_float2((q == 1 || q == 2) ? -c : c, (q == 2 || q == 3) ? -n : n);
}

__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(float v) { return v; }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ float from_f(float v) { return v; }

template <typename T, int VEC>
struct __align__(sizeof(T) * VEC) Unit {
  T e[VEC];
};

// VEC elements a unit (16 bytes), or 1: a rotating unit is then one pair of elements.
template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const __grid_constant__ RotaryArgs a) {
  using U = Unit<T, VEC>;
  constexpr bool kTwo = VEC == 1 || !INTER;  // a rotating unit is two pieces
  constexpr int kPairs = VEC == 1 ? 1 : (INTER ? VEC / 2 : VEC);
  __shared__ int s_pos[kRotMaxRows], s_page[kRotMaxRows];
  __shared__ float2 s_angle[kRotMaxAngles];  // [row][pair]
  griddep_launch_dependents();
  const RotaryDesc& d = a.d;
  const int R = a.rows_per_block;
  const int u = threadIdx.x % a.units, rest = threadIdx.x / a.units;
  const int rb = rest % R, h0 = rest / R;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * R, row = row0 + rb;
  const bool active = h0 < a.head_slots && row < d.n_rows;
  const bool turning = u < a.rot_units;
  // first element of the unit's piece(s)
  int e0, e1 = 0;
  if (!turning) {
    e0 = d.rot_dim + (u - a.rot_units) * VEC;
  } else if (VEC == 1) {
    e0 = INTER ? 2 * u : u;
    e1 = INTER ? 2 * u + 1 : u + d.rot_dim / 2;
  } else {
    e0 = u * VEC;
    e1 = e0 + d.rot_dim / 2;
  }
  const bool two = kTwo && turning;
  const int n0 = d.part[0].heads, n1 = n0 + d.part[1].heads;  // heads of parts that are not there: 0
  auto part_of = [&](int h) { return h < n0 ? 0 : h < n1 ? 1 : 2; };
  auto first_of = [&](int p) { return p == 0 ? 0 : p == 1 ? n0 : n1; };
  U lo[kRotBatch], hi[kRotBatch];
  auto load = [&](int h_base) {
#pragma unroll
    for (int b = 0; b < kRotBatch; ++b) {
      const int h = h_base + b * a.head_slots;
      if (!active || h >= a.heads) continue;
      const int p = part_of(h);
      const RotPart& t = d.part[p];
      const T* src = static_cast<const T*>(t.x) + row * t.x_row + (h - first_of(p)) * t.x_head;
      lo[b] = *reinterpret_cast<const U*>(src + e0);
      if (two) hi[b] = *reinterpret_cast<const U*>(src + e1);
    }
  };
  griddep_wait();
  load(h0);
  if (threadIdx.x < R && row0 + threadIdx.x < d.n_rows) {
    const int r = static_cast<int>(row0) + threadIdx.x;
    int pos, page = 0;
    if (d.positions) {
      pos = d.positions[r];
    } else {
      const int i = chunk_of_row(a.c, r);
      pos = a.c.pos[i] + (r - a.c.row0[i]);
      page = a.c.pt[i][pos / kPage];
      if (page < 0 || page >= a.c.num_pages) {
        if (d.status) atomicOr(d.status, kStatusBounds);
        page = -1;  // its writes are left out
      }
    }
    s_pos[threadIdx.x] = pos;
    s_page[threadIdx.x] = page;
  }
  __syncthreads();
  const int pairs = d.rot_dim / 2, here = static_cast<int>(min(static_cast<int64_t>(R), d.n_rows - row0));
  for (int i = threadIdx.x; i < here * pairs; i += kRotThreads) {
    const int k = i / here, r = i - k * here;  // lanes of a warp share few pairs
    const float2 t = turn_cos_sin(static_cast<uint64_t>(static_cast<int64_t>(s_pos[r])) * d.turns[k]);
    s_angle[r * pairs + k] = make_float2(t.x * d.magnitude, (d.inverse ? -t.y : t.y) * d.magnitude);
  }
  __syncthreads();
  if (!active) return;
  float2 cs[kPairs];
  if (turning) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) cs[i] = s_angle[rb * pairs + u * kPairs + i];
  }
  const int page = s_page[rb], slot = s_pos[rb] % kPage;
  const int64_t page_at = (static_cast<int64_t>(page) * d.n_kv_heads * kPage + slot) * d.head_dim;
  for (int h_base = h0; h_base < a.heads; h_base += kRotBatch * a.head_slots) {
    if (h_base != h0) load(h_base);
#pragma unroll
    for (int b = 0; b < kRotBatch; ++b) {
      const int h = h_base + b * a.head_slots;
      if (h >= a.heads) continue;
      const int p = part_of(h);
      const RotPart& t = d.part[p];
      if (turning && t.rotate) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          T& xe = kTwo ? lo[b].e[i] : lo[b].e[(2 * i) % VEC];
          T& ye = kTwo ? hi[b].e[i] : lo[b].e[(2 * i + 1) % VEC];
          const float xf = to_f(xe), yf = to_f(ye);
          xe = from_f<T>(xf * cs[i].x - yf * cs[i].y);
          ye = from_f<T>(yf * cs[i].x + xf * cs[i].y);
        }
      }
      if (t.paged && page < 0) continue;
      const int64_t at = t.paged ? page_at + static_cast<int64_t>(h - first_of(p)) * kPage * d.head_dim
                                 : row * t.out_row + (h - first_of(p)) * t.out_head;
      T* dst = static_cast<T*>(t.out) + at;
      *reinterpret_cast<U*>(dst + e0) = lo[b];
      if (two) *reinterpret_cast<U*>(dst + e1) = hi[b];
    }
  }
}

template <typename T, int VEC>
cudaError_t launch_vec(RotaryArgs& a, int num_sms, cudaStream_t stream) {
  const RotaryDesc& d = a.d;
  a.rot_units = VEC == 1 ? d.rot_dim / 2 : d.interleaved ? d.rot_dim / VEC : d.rot_dim / 2 / VEC;
  a.units = a.rot_units + (d.head_dim - d.rot_dim) / VEC;
  a.heads = 0;
  for (int p = 0; p < d.n_parts; ++p) a.heads += d.part[p].heads;
  // A block's threads: units x rows x head slots. Slots of a batch of heads each where the rows fill the SMs (few
  // angles are formed twice); more slots and fewer rows where they do not.
  const int room = kRotThreads / a.units;
  a.head_slots = std::max(1, std::min(room, (a.heads + 2 * kRotBatch - 1) / (2 * kRotBatch)));
  a.rows_per_block = std::max(1, std::min(kRotMaxRows, room / a.head_slots));
  while (a.rows_per_block > 1 && (static_cast<int64_t>(d.n_rows) + a.rows_per_block - 1) / a.rows_per_block < 4 * num_sms)
    a.rows_per_block /= 2;
  a.head_slots = std::min(a.heads, room / a.rows_per_block);
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(d.n_rows) + a.rows_per_block - 1) / a.rows_per_block));
  PdlScope pdl;
  return d.interleaved ? launch_kernel(rotary_kernel<T, VEC, true>, grid, dim3(kRotThreads), 0, stream, a)
                       : launch_kernel(rotary_kernel<T, VEC, false>, grid, dim3(kRotThreads), 0, stream, a);
}

template <typename T>
cudaError_t launch_type(RotaryArgs& a, int num_sms, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  const RotaryDesc& d = a.d;
  bool vec = d.head_dim % VEC == 0 && d.rot_dim % VEC == 0 && (d.interleaved || d.rot_dim / 2 % VEC == 0);
  for (int p = 0; p < d.n_parts; ++p) {
    const RotPart& t = d.part[p];
    vec = vec && t.x_row % VEC == 0 && t.x_head % VEC == 0 && (reinterpret_cast<uintptr_t>(t.x) & 15) == 0 &&
          (reinterpret_cast<uintptr_t>(t.out) & 15) == 0 && (t.paged || (t.out_row % VEC == 0 && t.out_head % VEC == 0));
  }
  return vec ? launch_vec<T, VEC>(a, num_sms, stream) : launch_vec<T, 1>(a, num_sms, stream);
}

}  // namespace

cudaError_t launch_rotary(const RotaryDesc& d, const ChunkTable* chunks, int num_sms, cudaStream_t stream) {
  if (d.n_rows < 1) return cudaSuccess;
  RotaryArgs a;
  a.d = d;
  if (chunks) a.c = *chunks;
  else std::memset(&a.c, 0, sizeof(a.c));
  switch (d.type) {
    case CRF_BF16: return launch_type<__nv_bfloat16>(a, num_sms, stream);
    case CRF_FP16: return launch_type<__half>(a, num_sms, stream);
    case CRF_FP32: return launch_type<float>(a, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace crf
