// What the kernels that turn heads share: the angle of a position, the request of a packed row, and 16-byte units of
// elements as fp32 (rotary.cu says how angles are formed and what they are off by).
#pragma once

#include "common.cuh"
#include "extend.h"

#include <cuda_fp16.h>

namespace crf {

constexpr int kRotThreads = 256;    // at most
constexpr int kRotMaxRows = 32;     // of a block
constexpr int kRotMaxAngles = 1024; // of a block: 8 pairs a unit, about 128 threads, or one row

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

// A unit of VEC elements as fp32 and back, two elements a conversion where they are packed.
template <typename T, int VEC>
struct __align__(sizeof(T) * VEC) Unit {
  T e[VEC];
};
template <int VEC>
__device__ __forceinline__ void unpack(const Unit<float, VEC>& u, float (&f)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) f[i] = u.e[i];
}
template <int VEC>
__device__ __forceinline__ void pack(const float (&f)[VEC], Unit<float, VEC>& u) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) u.e[i] = f[i];
}
__device__ __forceinline__ float2 unpack2(__nv_bfloat16, uint32_t w) { return make_float2(bf16_lo(w), bf16_hi(w)); }
__device__ __forceinline__ float2 unpack2(__half, uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ uint32_t pack2(__nv_bfloat16, float a, float b) { return pack_bf16(a, b); }
__device__ __forceinline__ uint32_t pack2(__half, float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T>
__device__ __forceinline__ void unpack(const Unit<T, 8>& u, float (&f)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(&u);
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 g = unpack2(T(), v[i]);
    f[2 * i] = g.x;
    f[2 * i + 1] = g.y;
  }
}
template <typename T>
__device__ __forceinline__ void pack(const float (&f)[8], Unit<T, 8>& u) {
  *reinterpret_cast<uint4*>(&u) =
      make_uint4(pack2(T(), f[0], f[1]), pack2(T(), f[2], f[3]), pack2(T(), f[4], f[5]), pack2(T(), f[6], f[7]));
}
__device__ __forceinline__ void unpack(const Unit<__nv_bfloat16, 1>& u, float (&f)[1]) { f[0] = __bfloat162float(u.e[0]); }
__device__ __forceinline__ void unpack(const Unit<__half, 1>& u, float (&f)[1]) { f[0] = __half2float(u.e[0]); }
__device__ __forceinline__ void pack(const float (&f)[1], Unit<__nv_bfloat16, 1>& u) { u.e[0] = __float2bfloat16_rn(f[0]); }
__device__ __forceinline__ void pack(const float (&f)[1], Unit<__half, 1>& u) { u.e[0] = __float2half_rn(f[0]); }

}  // namespace crf
