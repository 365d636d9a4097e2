// Rotary positions of query and key heads, and the write of new rows' keys and values into the pages of a
// layer: pair (x, y) of a head at position p becomes magnitude (x cos - y sin, y cos + x sin) of the angle
// p f, with f the pair's radians a position; the inverse map takes -sin (the transpose, hence the gradient).
//
// Angles: f / 2 pi is a fraction of a turn, held as a 64-bit integer in units of 2^-64 turns, so the product
// with the position drops whole turns by itself (integer arithmetic modulo 2^64). Three things are rounded: the
// fraction itself, formed in 64-bit floating point, is off by a few 2^-53 of its value, which the position multiplies
// (2^-24 turns for the fastest pair at p = 2^31, 2^-38 at 131072); its units cost p 2^-64 turns; and the product's
// top 32 bits are kept, which costs up to 2^-32 turns. They are split into a quadrant and a remainder of at most an
// eighth of a turn, whose sine and cosine are fp32 functions.
//
// Bound by memory: every element is read once and written once. A thread owns one 16-byte unit of a row (for the
// half layout two, the pair's halves) in up to four neighbouring heads and asks for all of them before the angles are
// formed; a block's angles are formed once, in shared memory, for its rows' heads. A thread has one round of loads:
// with its heads dealt in rounds (28 heads over 5 threads), 16384 bf16 rows of 32 heads took 66 us, so 44
// (268 MB: 90% of the copy rate; fp32 82 us for 537 MB, 97%; interleaved 43).
#include "../../include/crf.h"
#include "rotary.cuh"

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

constexpr int kRotBatch = 4;        // heads of a thread, at most

struct RotaryArgs {
  RotaryDesc d;
  ChunkTable c;
  int units, rot_units;     // 16-byte units of a head, those that rotate
  int rows;                 // of a block
  int batch;                // heads of a slot
  int slot0[3];             // each part's first slot
  int slots, block_slots;   // of all parts; of a block
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
  const int R = a.rows;
  const int u = threadIdx.x % a.units, rest = threadIdx.x / a.units;
  const int rb = rest % R, slot = rest / R + blockIdx.y * a.block_slots;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * R, row = row0 + rb;
  const bool active = rest / R < a.block_slots && slot < a.slots && row < d.n_rows;
  // the slot's part and heads [head, head + heads)
  const int p = slot >= a.slot0[2] ? 2 : slot >= a.slot0[1] ? 1 : 0;
  const RotPart t = p == 0 ? d.part[0] : p == 1 ? d.part[1] : d.part[2];
  const int head = (slot - (p == 0 ? 0 : p == 1 ? a.slot0[1] : a.slot0[2])) * a.batch;
  const int heads = active ? min(a.batch, t.heads - head) : 0;
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
  U lo[kRotBatch], hi[kRotBatch];
  griddep_wait();
  {
    const T* src = static_cast<const T*>(t.x) + row * t.x_row + head * t.x_head;
#pragma unroll
    for (int b = 0; b < kRotBatch; ++b) {
      if (b < heads) {
        lo[b] = *reinterpret_cast<const U*>(src + e0);
        if (two) hi[b] = *reinterpret_cast<const U*>(src + e1);
      }
      src += t.x_head;
    }
  }
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
  for (int i = threadIdx.x; i < here * pairs; i += blockDim.x) {
    const int k = i / here, r = i - k * here;  // lanes of a warp share few pairs
    const float2 t = turn_cos_sin(static_cast<uint64_t>(static_cast<int64_t>(s_pos[r])) * d.turns[k]);
    s_angle[r * pairs + k] = make_float2(t.x * d.magnitude, (d.inverse ? -t.y : t.y) * d.magnitude);
  }
  __syncthreads();
  const int page = s_page[rb];
  if (!active || (t.paged && page < 0)) return;
  const bool rotate = turning && t.rotate;
  float2 cs[kPairs];
  if (rotate) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) cs[i] = s_angle[rb * pairs + u * kPairs + i];
  }
  const int64_t out_head = t.paged ? static_cast<int64_t>(kPage) * d.head_dim : t.out_head;
  T* dst = static_cast<T*>(t.out) + head * out_head +
           (t.paged ? (static_cast<int64_t>(page) * d.n_kv_heads * kPage + s_pos[rb] % kPage) * d.head_dim : row * t.out_row);
#pragma unroll
  for (int b = 0; b < kRotBatch; ++b) {
    if (b < heads) {
      if (rotate) {
        float x[VEC], y[VEC];
        unpack(lo[b], x);
        if (kTwo) unpack(hi[b], y);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          float& u0 = kTwo ? x[i] : x[(2 * i) % VEC];
          float& u1 = kTwo ? y[i] : x[(2 * i + 1) % VEC];
          const float xf = u0, yf = u1;
          u0 = xf * cs[i].x - yf * cs[i].y;
          u1 = yf * cs[i].x + xf * cs[i].y;
        }
        pack(x, lo[b]);
        if (kTwo) pack(y, hi[b]);
      }
      *reinterpret_cast<U*>(dst + e0) = lo[b];
      if (two) *reinterpret_cast<U*>(dst + e1) = hi[b];
    }
    dst += out_head;
  }
}

template <typename T, int VEC>
cudaError_t launch_vec(RotaryArgs& a, int num_sms, cudaStream_t stream) {
  const RotaryDesc& d = a.d;
  a.rot_units = VEC == 1 ? d.rot_dim / 2 : d.interleaved ? d.rot_dim / VEC : d.rot_dim / 2 / VEC;
  a.units = a.rot_units + (d.head_dim - d.rot_dim) / VEC;
  // Slots of four heads where the rows alone fill the SMs, of one head where they are few: a call of one row is then
  // a block or two with one head a thread.
  const bool few = d.n_rows < 4 * num_sms;
  a.batch = few ? 1 : kRotBatch;
  auto deal = [&]() {
    a.slots = 0;
    for (int p = 0; p < 3; ++p) {
      a.slot0[p] = a.slots;
      if (p < d.n_parts) a.slots += (d.part[p].heads + a.batch - 1) / a.batch;
      else a.slot0[p] = 1 << 30;
    }
  };
  deal();
  if (a.batch == 1 && a.slots > 4096) {  // heads beyond any row's: keep the grid's second axis short
    a.batch = kRotBatch;
    deal();
  }
  const int room = kRotThreads / a.units;
  a.block_slots = std::min(a.slots, room);
  // rows of a block: about 128 threads (16384 bf16 rows of 32 heads: 44 us; 47 with 256, 50 with 72)
  a.rows = few ? 1 : std::max(1, std::min(kRotMaxRows, 128 / (a.units * a.block_slots)));
  const int threads = (a.units * a.block_slots * a.rows + 31) / 32 * 32;
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(d.n_rows) + a.rows - 1) / a.rows),
                  (a.slots + a.block_slots - 1) / a.block_slots);
  PdlScope pdl;
  return d.interleaved ? launch_kernel(rotary_kernel<T, VEC, true>, grid, dim3(threads), 0, stream, a)
                       : launch_kernel(rotary_kernel<T, VEC, false>, grid, dim3(threads), 0, stream, a);
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
