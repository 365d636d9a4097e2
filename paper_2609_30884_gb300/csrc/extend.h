// Launchers of the calls that extend a cache with new tokens: rotary positions, norms of heads, writes of new keys and
// values, attention of a chunk over the pages, the pages' reference counts, and log probabilities of tokens.
#pragma once

#include "kernels.h"

namespace crf {

constexpr int kMaxChunks = 128;  // equals CRF_MAX_CHUNKS (api_extend.cu checks that)
constexpr int kMaxTables = 512;  // equals CRF_MAX_TABLES
constexpr int kMaxPairs = 128;   // rotary pairs of a head
constexpr int kMaxKeys = 1 << 26;  // equals CRF_MAX_KEYS
constexpr int kMaxTop = 32;      // equals CRF_MAX_TOP
constexpr int kMaxVocab = 1 << 20;  // equals CRF_MAX_VOCAB

// The requests of a call: rows [row0[i], row0[i + 1]) are request i's, at positions pos[i] on.
struct ChunkTable {
  int n, num_pages;
  int row0[kMaxChunks + 1];
  int pos[kMaxChunks];
  int n_keys[kMaxChunks];
  const int32_t* pt[kMaxChunks];
};

// ---------------------------------------------------------------- rotary positions
struct RotPart {
  const void* x;
  void* out;  // strided heads, or a layer's pages
  int64_t x_row, x_head, out_row, out_head;
  int heads;
  bool rotate, paged;
};
struct RotaryDesc {
  RotPart part[3];
  int n_parts;
  int head_dim, rot_dim;
  bool interleaved, inverse;
  float magnitude;
  int n_rows;
  const int32_t* positions;    // [n_rows], or null: the rows of `chunks`
  int n_kv_heads;              // of paged parts
  int type;                    // CRF_BF16 ...
  uint64_t turns[kMaxPairs];   // turns a position of pair i, in units of 2^-64
  int* status;
};
cudaError_t launch_rotary(const RotaryDesc& d, const ChunkTable* chunks, int num_sms, cudaStream_t stream);

// ---------------------------------------------------------------- norms of heads
// Parts that are rotated are normed first, with the gain and eps of their number.
struct HeadNormDesc {
  RotaryDesc r;
  const void* gain[2];
  float eps[2];
  float inv_dim;               // 1 / head_dim
};
cudaError_t launch_head_norm(const HeadNormDesc& d, const ChunkTable* chunks, int num_sms, cudaStream_t stream);
// r.part: x and, as out, its gradient; r.inverse is set.
struct HeadNormGradDesc {
  RotaryDesc r;
  const void* gain[2];
  const void* grad[2];         // of the outputs
  int64_t g_row[2], g_head[2];
  float eps[2];
  float inv_dim;
  float* dgain[2];
};
size_t head_norm_grad_workspace(int head_dim, int num_sms);
cudaError_t launch_head_norm_grad(const HeadNormGradDesc& d, float* partial, int num_sms, cudaStream_t stream);

// ---------------------------------------------------------------- log probabilities
struct LogprobsDesc {
  const void* z;
  int64_t z_row;
  int type, n_rows, vocab, n_top;
  const int32_t* targets;      // null with logprob
  float* logprob;              // each output may be null
  float* entropy;
  float* lse;
  int32_t* top_ids;            // [n_rows][n_top]
  float* top_logprobs;
  int* status;
};
cudaError_t launch_logprobs(const LogprobsDesc& d, int num_sms, cudaStream_t stream);
struct LogprobsGradDesc {
  const void* z;
  void* dz;
  int64_t z_row, dz_row;
  int type, n_rows, vocab;
  const int32_t* targets;
  const float* lse;
  const float* entropy;        // read with g_entropy
  const float* g_logprob;      // may be null
  const float* g_entropy;      // may be null
  int* status;
};
cudaError_t launch_logprobs_grad(const LogprobsGradDesc& d, cudaStream_t stream);

// ---------------------------------------------------------------- chunk attention
struct ChunkAttnDesc {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  int64_t q_row, q_head, out_row, out_head;
  float* lse;                  // [rows][n_q_heads] or null
  const __nv_bfloat16* kpages;
  const __nv_bfloat16* vpages;
  int n_q_heads, n_kv_heads, head_dim;
  float scale;
  bool causal;
  int window;                  // 0: none
  int* status;
};
// The requests of a call whose rows see the first `sinks` keys whatever their window.
struct SinksTable : ChunkTable {
  int sinks;
};
// The entries of a call whose requests share prefixes: entry i's rows [row0[i], row0[i] + rows[i]) over the keys from key0[i] on. A split group's shared keys are an entry (at a position behind
// all of them), before the entries of requests. A folded group is one entry for all: its sinks are the shared keys, behind which, from the
// next tile on, the pages of its members' own keys are laid end to end; member m's rows begin m_row0[m] behind the entry's, its pages at
// m_page0[m], the first of them being page m_first[m] of its table.
constexpr int kMaxEntries = kMaxChunks + kMaxChunks / 2;
struct AttnTable {
  int n, num_pages;
  int row0[kMaxEntries];
  int rows[kMaxEntries];
  int pos[kMaxEntries];
  int key0[kMaxEntries];
  int n_keys[kMaxEntries];
  int sinks[kMaxEntries];
  int member0[kMaxEntries];  // folded: members [member0, member0 + members)
  int members[kMaxEntries];  // 0: not folded
  const int32_t* pt[kMaxEntries];
  int m_row0[kMaxChunks];
  int m_page0[kMaxChunks];
  int m_first[kMaxChunks];
  int m_pos[kMaxChunks];
  int m_keys[kMaxChunks];
  const int32_t* m_pt[kMaxChunks];
};
constexpr int kMaxCtas = 256;
// Where a CTA's run begins: step `step` of item (request, query tile or pair qt, kv head g); request = c.n: the end.
// Items go through the requests in order, query tiles from the last down, heads.
struct RunStart {
  int req, qt, g, step;
};
// A cut item: part k is in slot first_slot (k = 0) or 2 (cta + k).
struct CutItem {
  int row0, q0, g, first_slot, cta, parts;
};
// How a call's work is dealt: one run a CTA, and the items that runs cut.
struct ChunkPlan {
  int ctas, cuts;
  int part_rows, merge_rows;  // rows of the largest cut item, of all
  int longest;                // steps of the longest segment
  RunStart run[kMaxCtas + 1];
  int rows[kMaxCtas + 1];     // packed rows of the cut items before each
  CutItem cut[kMaxCtas];
};
void plan_chunk_attention(const ChunkTable& c, int n_q_heads, int n_kv_heads, bool causal, int window, int num_sms,
                          ChunkPlan* p);
size_t chunk_attention_workspace(const ChunkPlan& p, int head_dim);
cudaError_t launch_chunk_attention(const ChunkAttnDesc& d, const ChunkTable& c, const ChunkPlan& p, void* workspace,
                                   int num_sms, cudaStream_t stream);

void plan_sinks_attention(const SinksTable& c, int n_q_heads, int n_kv_heads, bool causal, int window, int num_sms, ChunkPlan* p);
cudaError_t launch_sinks_attention(const ChunkAttnDesc& d, const SinksTable& c, const ChunkPlan& p, void* workspace,
                                   int num_sms, cudaStream_t stream);

// Attention of requests that share prefixes.
struct AttnPlan {
  ChunkPlan runs;
  bool shared;                      // the table has split groups; every segment is a part
  int items;
  int64_t part_rows;                // of all parts
  int64_t run_rows[kMaxCtas];
  int item0[kMaxEntries];           // items of the entries before
};
// The split groups' entries are the table's first; of[i] is that of entry groups + i, or -1.
struct PrefixGroups {
  int groups;
  bool any;                  // some group is split or folded
  int16_t of[kMaxChunks];
};
void plan_prefix_attention(const AttnTable& a, bool shared, int n_q_heads, int n_kv_heads, bool causal, int num_sms, AttnPlan* p);
// The table of requests in runs of count[i] that share their first keys[i] keys. A group is folded, split, or its requests stand apart,
// whichever takes the fewest units of work.
void share_prefixes(const ChunkTable& c, const int* count, const int* keys, int n, int n_q_heads, int n_kv_heads, bool causal,
                    int num_sms, AttnTable* a, PrefixGroups* g);
size_t prefix_attention_workspace(const AttnPlan& p, int head_dim);
cudaError_t launch_prefix_attention(const ChunkAttnDesc& d, const AttnTable& a, const PrefixGroups& g, const AttnPlan& p,
                                    void* workspace, int num_sms, cudaStream_t stream);

// ---------------------------------------------------------------- pages
// Entries [first[i], first[i + 1]) of a call are table i's.
struct PageTables {
  int n, num_pages;
  int first[kMaxTables + 1];
  int fresh0[kMaxTables + 1];  // fork: new pages of the tables before i
  int n_tokens[kMaxTables];
  const int32_t* table[kMaxTables];
  int32_t* out[kMaxTables];
};
struct PagePool {
  void* const* k;  // host arrays of the layers' pools
  void* const* v;
  int n_layers, n_kv_heads, head_dim;
};
enum PageOp : int { kPageFork, kPageCompact, kPageRelease };
size_t page_workspace(int num_pages, int entries);
// The plan (one kernel: checks, counts, tables, the list of copies) and, with a pool, the copies.
int page_launches(PageOp op, const PageTables& t, int n_layers);
cudaError_t launch_pages(PageOp op, const PageTables& t, bool deep, const int32_t* refs_in, int32_t* refs_out,
                         const PagePool* pool, void* workspace, int num_sms, int* status, cudaStream_t stream);

}  // namespace crf
