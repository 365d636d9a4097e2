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
#include "chunk_attn.cuh"

namespace crf {

void plan_chunk_attention(const ChunkTable& c, int n_q_heads, int n_kv_heads, bool causal, int window, int num_sms, ChunkPlan* p) {
  plan_runs(c, kCosts, n_q_heads, n_kv_heads, causal, window, num_sms, nullptr, p);
}

size_t chunk_attention_workspace(const ChunkPlan& p, int head_dim) {
  return (part_floats(p, head_dim, false) + part_floats(p, head_dim, true) + total_floats(p, head_dim)) * sizeof(float);
}

cudaError_t launch_chunk_attention(const ChunkAttnDesc& d, const ChunkTable& c, const ChunkPlan& p, void* workspace,
                                   int num_sms, cudaStream_t stream) {
  return launch_rows<kPlain>(d, c, p, workspace, num_sms, stream);
}

}  // namespace crf
