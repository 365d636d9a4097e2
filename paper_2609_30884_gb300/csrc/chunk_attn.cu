// Attention of new rows over cached keys, the plain form: the plan of its runs, its workspace and its launch. The kernel and what it is
// built on are in chunk_attn.cuh.
#include "chunk_attn.cuh"

namespace crf {

void plan_chunk_attention(const ChunkTable& c, int n_q_heads, int n_kv_heads, bool causal, int window, int num_sms, ChunkPlan* p) {
  plan_runs<kCosts>(c, n_q_heads, n_kv_heads, causal, window, num_sms, nullptr, p);
}

size_t chunk_attention_workspace(const ChunkPlan& p, int head_dim) {
  return (part_floats(p, head_dim, false) + part_floats(p, head_dim, true) + total_floats(p, head_dim)) * sizeof(float);
}

cudaError_t launch_chunk_attention(const ChunkAttnDesc& d, const ChunkTable& c, const ChunkPlan& p, void* workspace,
                                   int num_sms, cudaStream_t stream) {
  return launch_rows<kPlain>(d, c, p, workspace, num_sms, stream);
}

}  // namespace crf
