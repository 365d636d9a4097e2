// Launchers of the calls that extend a cache with new tokens: rotary positions, writes of new keys and
// values, attention of a chunk over the pages, and the pages' reference counts.
#pragma once

#include "kernels.h"

namespace crf {

constexpr int kMaxChunks = 128;  // equals CRF_MAX_CHUNKS (api_extend.cu checks that)
constexpr int kMaxTables = 512;  // equals CRF_MAX_TABLES
constexpr int kMaxPairs = 128;   // rotary pairs of a head

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
