// Attention with sinks, a form of the kernel of chunk_attn.cuh: row r of a request at position p sees the window p - window < j <= p and,
// whatever the window, the keys j < sinks. An item's tiles are those of the sinks, then those of its rows' windows, numbered through; each
// has one range of keys a row, and one mask. A tile that holds keys of both ranges is gone through twice. Nothing between the ranges is read,
// not even its entries of the page table.
//
// Single rows: 16 with a window of 4096 of 4K-16K keys take 35 us; their 134 MB take 20 at the copy rate and 21 here, the rest are the start, whole
// steps of a run, one more masked tile an item, and the merge (128 runs, each item cut in two). Long chunks are bound by the chains of
// products and softmax: 4096 rows over a window of 4096 200 us, 1210 TFLOP/s of what the windows need; their masked ends are computed beside it.
#include "chunk_attn.cuh"

namespace crf {

void plan_sinks_attention(const SinksTable& c, int n_q_heads, int n_kv_heads, bool causal, int window, int num_sms, ChunkPlan* p) {
  plan_runs<kSinksCosts>(c, n_q_heads, n_kv_heads, causal, window, num_sms, nullptr, p);
}

cudaError_t launch_sinks_attention(const ChunkAttnDesc& d, const SinksTable& c, const ChunkPlan& p, void* workspace,
                                   int num_sms, cudaStream_t stream) {
  return launch_rows<kSinks>(d, c, p, workspace, num_sms, stream);
}

}  // namespace crf
