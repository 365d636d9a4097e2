// Attention of a chunk of new rows over their requests' cached keys. Row r of a request at position p sees the
// keys lo <= j < hi with hi = min(n_keys, p + 1) (causal; n_keys otherwise) and lo = max(0, p - window + 1)
// (0 without a window): o = softmax(scale q k) v, lse = log sum exp(scale q k). One warp per (row, query head)
// walks the keys with a running maximum and sum.
#include "common.cuh"
#include "extend.h"

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

struct ChunkArgs {
  ChunkAttnDesc d;
  ChunkTable c;
};

template <int D>
__global__ void __launch_bounds__(256) chunk_attn_simple(const __grid_constant__ ChunkArgs a) {
  constexpr int E = D / 32;
  const ChunkAttnDesc& d = a.d;
  const int lane = threadIdx.x & 31;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int64_t r = w / d.n_q_heads;
  const int h = static_cast<int>(w - r * d.n_q_heads), g = h / (d.n_q_heads / d.n_kv_heads);
  if (r >= a.c.row0[a.c.n]) return;
  int i = 0;
  while (r >= a.c.row0[i + 1]) ++i;
  const int p = a.c.pos[i] + static_cast<int>(r - a.c.row0[i]);
  const int hi = d.causal ? min(a.c.n_keys[i], p + 1) : a.c.n_keys[i], lo = d.window ? max(0, p - d.window + 1) : 0;
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = __bfloat162float(d.q[r * d.q_row + h * d.q_head + lane * E + e]) * d.scale;
    o[e] = 0.f;
  }
  for (int j = lo; j < hi; ++j) {
    int page = a.c.pt[i][j / kPage];
    if (page < 0 || page >= a.c.num_pages) {
      if (lane == 0) atomicOr(d.status, kStatusBounds);
      page = 0;
    }
    const size_t at = ((static_cast<size_t>(page) * d.n_kv_heads + g) * kPage + j % kPage) * D + lane * E;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += q[e] * __bfloat162float(d.kpages[at + e]);
    s = warp_sum(s);
    const float mn = fmaxf(m, s), c = __expf(m - mn), w = __expf(s - mn);
    l = l * c + w;
    m = mn;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * c + w * __bfloat162float(d.vpages[at + e]);
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) d.out[r * d.out_row + h * d.out_head + lane * E + e] = __float2bfloat16_rn(o[e] * inv);
  if (d.lse && lane == 0) d.lse[r * d.n_q_heads + h] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace

size_t chunk_attention_workspace(const ChunkTable&, int, int, int, bool, int, int) { return 0; }
int chunk_attention_launches(const ChunkTable&, int, int, int, bool, int, int) { return 1; }

cudaError_t launch_chunk_attention(const ChunkAttnDesc& d, const ChunkTable& c, void*, int, cudaStream_t stream) {
  ChunkArgs a;
  a.d = d;
  a.c = c;
  const int64_t warps = static_cast<int64_t>(c.row0[c.n]) * d.n_q_heads;
  if (warps == 0) return cudaSuccess;
  const dim3 grid(static_cast<unsigned>((warps + 7) / 8));
  return d.head_dim == 128 ? launch_kernel(chunk_attn_simple<128>, grid, dim3(256), 0, stream, a)
                           : launch_kernel(chunk_attn_simple<64>, grid, dim3(256), 0, stream, a);
}

}  // namespace crf
