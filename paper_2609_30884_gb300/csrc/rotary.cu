// Rotary positions of query and key heads, and the write of new rows' keys and values into the pages of a
// layer: pair (x, y) of a head at position p becomes magnitude (x cos - y sin, y cos + x sin) of the angle
// p f, with f the pair's radians a position; the inverse map takes -sin (the transpose, hence the gradient).
//
// Angles: f / 2 pi is a fraction of a turn, held as a 64-bit integer in units of 2^-64 turns, so the product
// with the position drops whole turns by itself (integer arithmetic modulo 2^64) and is exact for the held f:
// at p = 2^31 the angle is off by at most 2^-33 turns. Its top 32 bits are split into a quadrant and a
// remainder of at most an eighth of a turn, whose sine and cosine are fp32 functions.
//
// Bound by memory: every element is read once and written once. A thread owns one 16-byte unit of a row's head
// (for the half layout two, the pair's halves), forms its sines and cosines once and walks the heads with four
// units in flight.
#include "../../include/crf.h"
#include "common.cuh"
#include "extend.h"

#include <cuda_fp16.h>

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotBatch = 4;  // heads in flight

struct RotaryArgs {
  RotaryDesc d;
  ChunkTable c;
  int units, rot_units, rows_per_block, heads, heads_per_block;
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
  __shared__ uint64_t turns[kMaxPairs];
  const RotaryDesc& d = a.d;
  for (int i = threadIdx.x; i < d.rot_dim / 2; i += kRotThreads) turns[i] = d.turns[i];
  __syncthreads();
  const int rb = threadIdx.x / a.units, u = threadIdx.x - rb * a.units;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * a.rows_per_block + rb;
  if (rb >= a.rows_per_block || row >= d.n_rows) return;
  int pos, page = 0, slot = 0;
  if (d.positions) {
    pos = d.positions[row];
  } else {
    const int i = chunk_of_row(a.c, static_cast<int>(row));
    pos = a.c.pos[i] + (static_cast<int>(row) - a.c.row0[i]);
    page = a.c.pt[i][pos / kPage];
    slot = pos % kPage;
    if (page < 0 || page >= a.c.num_pages) {
      if (d.status) atomicOr(d.status, kStatusBounds);
      page = -1;  // its writes are left out
    }
  }
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
  float cs[kPairs], sn[kPairs];
  if (turning) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 t = turn_cos_sin(static_cast<uint64_t>(static_cast<int64_t>(pos)) * turns[u * kPairs + i]);
      cs[i] = t.x * d.magnitude;
      sn[i] = (d.inverse ? -t.y : t.y) * d.magnitude;
    }
  }
  const int h_begin = blockIdx.y * a.heads_per_block, h_end = min(a.heads, h_begin + a.heads_per_block);
  int first = 0;  // heads of the parts before
  for (int p = 0; p < d.n_parts; ++p) {
    const RotPart& t = d.part[p];
    const int last = min(h_end, first + t.heads);
    const bool rotate = turning && t.rotate, two = kTwo && turning;
    const T* x = static_cast<const T*>(t.x) + row * t.x_row;
    T* out = static_cast<T*>(t.out);
    int64_t out_head = t.out_head;
    if (t.paged) {
      out += (static_cast<int64_t>(page) * d.n_kv_heads * kPage + slot) * d.head_dim;
      out_head = static_cast<int64_t>(kPage) * d.head_dim;
    } else {
      out += row * t.out_row;
    }
    for (int h0 = max(h_begin, first); h0 < last; h0 += kRotBatch) {
      U lo[kRotBatch], hi[kRotBatch];
#pragma unroll
      for (int b = 0; b < kRotBatch; ++b) {
        if (h0 + b >= last) continue;
        const T* src = x + (h0 + b - first) * t.x_head;
        lo[b] = *reinterpret_cast<const U*>(src + e0);
        if (two) hi[b] = *reinterpret_cast<const U*>(src + e1);
      }
#pragma unroll
      for (int b = 0; b < kRotBatch; ++b) {
        if (h0 + b >= last) continue;
        if (rotate) {
#pragma unroll
          for (int i = 0; i < kPairs; ++i) {
            T& xe = kTwo ? lo[b].e[i] : lo[b].e[(2 * i) % VEC];
            T& ye = kTwo ? hi[b].e[i] : lo[b].e[(2 * i + 1) % VEC];
            const float xf = to_f(xe), yf = to_f(ye);
            xe = from_f<T>(xf * cs[i] - yf * sn[i]);
            ye = from_f<T>(yf * cs[i] + xf * sn[i]);
          }
        }
        if (t.paged && page < 0) continue;
        T* dst = out + (h0 + b - first) * out_head;
        *reinterpret_cast<U*>(dst + e0) = lo[b];
        if (two) *reinterpret_cast<U*>(dst + e1) = hi[b];
      }
    }
    first += t.heads;
  }
}

template <typename T, int VEC>
cudaError_t launch_vec(RotaryArgs& a, int num_sms, cudaStream_t stream) {
  const RotaryDesc& d = a.d;
  a.rot_units = VEC == 1 ? d.rot_dim / 2 : d.interleaved ? d.rot_dim / VEC : d.rot_dim / 2 / VEC;
  a.units = a.rot_units + (d.head_dim - d.rot_dim) / VEC;
  a.rows_per_block = kRotThreads / a.units;
  a.heads = 0;
  for (int p = 0; p < d.n_parts; ++p) a.heads += d.part[p].heads;
  const int gx = static_cast<int>((static_cast<int64_t>(d.n_rows) + a.rows_per_block - 1) / a.rows_per_block);
  // few rows: the heads are dealt to more blocks, down to one batch each
  const int batches = (a.heads + kRotBatch - 1) / kRotBatch;
  const int gy = std::min(batches, std::max(1, (8 * num_sms + gx - 1) / gx));
  a.heads_per_block = (batches + gy - 1) / gy * kRotBatch;
  const dim3 grid(gx, (a.heads + a.heads_per_block - 1) / a.heads_per_block);
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
