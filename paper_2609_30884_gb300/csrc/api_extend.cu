// C ABI of the calls that extend a recovered cache with new tokens: argument checks and launches (see
// include/crf.h).
#include "api.h"
#include "common.cuh"
#include "extend.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <limits>

using namespace crf;

namespace {

// The arrays that kernels take are sized by the one and filled up to the other.
static_assert(kMaxChunks == CRF_MAX_CHUNKS && kMaxTables == CRF_MAX_TABLES && kMaxTop == CRF_MAX_TOP && kMaxVocab == CRF_MAX_VOCAB &&
                  kMaxKeys == CRF_MAX_KEYS,
              "limits of the ABI and of the kernels differ");

// The context's device for the length of a call, then the caller's again.
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    err_ = cudaGetDevice(&prev_);
    if (err_ == cudaSuccess && prev_ != device) {
      err_ = cudaSetDevice(device);
      moved_ = err_ == cudaSuccess;
    }
  }
  ~DeviceScope() {
    if (moved_) cudaSetDevice(prev_);
  }
  cudaError_t error() const { return err_; }

 private:
  int prev_ = 0;
  bool moved_ = false;
  cudaError_t err_;
};

// No C++ exception leaves a C entry.
template <typename F>
crf_status guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(CRF_ENOMEM, "host error: %s", e.what());
  }
}

// ---------------------------------------------------------------- rotary positions
double rope_base(const crf_rope& r) {
  return r.scaling == CRF_ROPE_BASE ? r.theta * std::pow(r.factor, r.rot_dim / (r.rot_dim - 2.0)) : r.theta;
}

crf_status check_rope(const crf_rope& r) {
  if (r.head_dim < 2 || r.head_dim > 2 * kMaxPairs || r.rot_dim < 2 || r.rot_dim % 2 || r.rot_dim > r.head_dim)
    return fail(CRF_EUNSUPPORTED, "rope: rot_dim %d must be even, 2..head_dim, and head_dim %d 2..%d", r.rot_dim,
                r.head_dim, 2 * kMaxPairs);
  if (r.layout != CRF_ROPE_HALF && r.layout != CRF_ROPE_INTERLEAVED) return fail(CRF_EINVAL, "rope: unknown layout %d", r.layout);
  if (r.scaling < CRF_ROPE_PLAIN || r.scaling > CRF_ROPE_BANDS) return fail(CRF_EINVAL, "rope: unknown scaling %d", r.scaling);
  if (!(r.theta > 0) || !std::isfinite(r.theta)) return fail(CRF_EINVAL, "rope: theta must be positive and finite");
  if (!std::isfinite(static_cast<float>(r.magnitude))) return fail(CRF_EINVAL, "rope: magnitude must be finite");
  if (r.scaling != CRF_ROPE_PLAIN && (!(r.factor >= 1) || !std::isfinite(r.factor)))
    return fail(CRF_EINVAL, "rope: factor must be finite and at least 1");
  if (r.scaling == CRF_ROPE_BASE && r.rot_dim == 2) return fail(CRF_EUNSUPPORTED, "rope: base scaling needs rot_dim > 2");
  if (r.scaling == CRF_ROPE_BANDS &&
      (!(r.low >= 0) || !(r.high > r.low) || !std::isfinite(r.high) || !(r.original > 0) || !std::isfinite(r.original)))
    return fail(CRF_EINVAL, "rope: bands need 0 <= low < high and original > 0, all finite");
  // the base in use; from the smallest normal number on, every frequency is finite
  const double base = rope_base(r);
  if (!std::isfinite(base) || base < std::numeric_limits<double>::min())
    return fail(CRF_EINVAL, "rope: the base is out of range");
  return CRF_OK;
}

// Turns a position of every pair, as a fraction of one turn in units of 2^-64.
void fill_turns(const crf_rope& r, uint64_t* turns) {
  const double two_pi = 6.283185307179586476925286766559;
  const double step = -2.0 / r.rot_dim * std::log2(rope_base(r));
  for (int i = 0; i < r.rot_dim / 2; ++i) {
    double f = std::exp2(step * i);
    if (r.scaling == CRF_ROPE_LINEAR) f /= r.factor;
    if (r.scaling == CRF_ROPE_BANDS) {
      double g = (r.original * f / two_pi - r.low) / (r.high - r.low);
      g = g < 0 ? 0 : g > 1 ? 1 : g;
      f *= g + (1 - g) / r.factor;
    }
    double t = f / two_pi;
    t -= std::floor(t);
    // t < 1; a product that rounds up to a whole turn is none
    const double units = t * 18446744073709551616.0;
    turns[i] = units >= 18446744073709551616.0 ? 0 : static_cast<uint64_t>(units);
  }
}

// Heads of `type` elements of `size` bytes; `out` too unless it is not read.
crf_status check_heads(const crf_heads& h, size_t size, bool has_out, const char* name) {
  if (!h.x || (has_out && !h.out)) return fail(CRF_EINVAL, "%s: null pointer", name);
  if (h.heads < 1 || h.heads > 65535) return fail(CRF_EINVAL, "%s: %d heads, 1..65535 wanted", name, h.heads);
  const int64_t most = int64_t{1} << 40;
  if (h.x_row < 0 || h.x_head < 0 || (has_out && (h.out_row < 0 || h.out_head < 0)) || h.x_row > most || h.x_head > most ||
      (has_out && (h.out_row > most || h.out_head > most)))
    return fail(CRF_EINVAL, "%s: a stride is negative or over 2^40", name);
  if ((reinterpret_cast<uintptr_t>(h.x) | (has_out ? reinterpret_cast<uintptr_t>(h.out) : 0)) & (size - 1))
    return fail(CRF_EINVAL, "%s: not aligned to its elements", name);
  return CRF_OK;
}

// The stride of an axis of one says nothing, whatever its value: it is set to one that every form takes.
crf_heads settled(crf_heads h, int64_t rows, int dim) {
  const int64_t step = (dim + 7) / 8 * 8;
  if (rows <= 1) h.x_row = h.out_row = step;
  if (h.heads == 1) h.x_head = h.out_head = step;
  return h;
}

RotPart part_of(const crf_heads& h, bool rotate) {
  RotPart p;
  p.x = h.x;
  p.out = h.out;
  p.x_row = h.x_row;
  p.x_head = h.x_head;
  p.out_row = h.out_row;
  p.out_head = h.out_head;
  p.heads = h.heads;
  p.rotate = rotate;
  p.paged = false;
  return p;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

// Outputs of rows and heads must not share elements: the strides are at least the extents they step over,
// in one order or the other.
crf_status check_out(const crf_heads& h, int64_t rows, int dim, const char* name) {
  // n steps and dim more within `outer`; a product could overflow
  auto fits = [dim](int64_t n, int64_t step, int64_t outer) { return outer >= dim && n <= (outer - dim) / step; };
  const bool head_ok = h.heads == 1 || h.out_head >= dim, row_ok = rows <= 1 || h.out_row >= dim;
  const bool rows_outer = head_ok && (rows <= 1 || (h.heads == 1 ? row_ok : fits(h.heads - 1, h.out_head, h.out_row)));
  const bool heads_outer = row_ok && (h.heads == 1 || (rows <= 1 ? head_ok : fits(rows - 1, h.out_row, h.out_head)));
  if (!rows_outer && !heads_outer) return fail(CRF_ESHAPE, "%s: the strides make output rows or heads overlap", name);
  return CRF_OK;
}

// ---------------------------------------------------------------- chunks
crf_status fill_chunks(const crf_chunk* chunks, int n, bool attend, int num_pages, ChunkTable* t) {
  if (!chunks) return fail(CRF_EINVAL, "chunks is null");
  if (n < 1 || n > CRF_MAX_CHUNKS) return fail(CRF_EINVAL, "n_chunks %d out of range (1..%d)", n, CRF_MAX_CHUNKS);
  std::memset(t, 0, sizeof(*t));
  t->n = n;
  t->num_pages = num_pages;
  int64_t rows = 0;
  for (int i = 0; i < n; ++i) {
    const crf_chunk& c = chunks[i];
    // 2^30 leaves room for tile arithmetic in 32 bits
    if (c.n_new < 0 || c.pos < 0 || c.n_keys < 0 || c.n_keys > (1 << 30) || static_cast<int64_t>(c.pos) + c.n_new > (1 << 30))
      return fail(CRF_EINVAL, "chunk %d: n_new, pos or n_keys out of range", i);
    // a query tile's keys have to pass within the kernels' wait limit (1.6 us for 128 of them: 0.8 s)
    if (attend && c.n_keys > CRF_MAX_KEYS) return fail(CRF_EUNSUPPORTED, "chunk %d: n_keys over %d", i, CRF_MAX_KEYS);
    if (!c.page_table && (attend ? c.n_new > 0 && c.n_keys > 0 : c.n_new > 0))
      return fail(CRF_EINVAL, "chunk %d: page table is null", i);
    if (!aligned4(c.page_table)) return fail(CRF_EINVAL, "chunk %d: page table misaligned", i);
    t->row0[i] = static_cast<int>(rows);
    t->pos[i] = c.pos;
    t->n_keys[i] = c.n_keys;
    t->pt[i] = c.page_table;
    rows += c.n_new;
    if (rows > (1 << 30)) return fail(CRF_EINVAL, "too many rows");
  }
  for (int i = n; i <= CRF_MAX_CHUNKS; ++i) t->row0[i] = static_cast<int>(rows);
  return CRF_OK;
}

crf_status check_pool_shape(int n_kv_heads, int head_dim, int num_pages) {
  if (head_dim != 64 && head_dim != 128) return fail(CRF_EUNSUPPORTED, "head_dim %d unsupported (64 or 128)", head_dim);
  if (n_kv_heads < 1) return fail(CRF_EINVAL, "n_kv_heads must be positive");
  if (num_pages < 1 || num_pages > (1 << 30)) return fail(CRF_EINVAL, "num_pages %d out of range", num_pages);
  // a page's 8-slot groups are counted in 32 bits
  if (static_cast<int64_t>(num_pages) * n_kv_heads > (1 << 30))
    return fail(CRF_EUNSUPPORTED, "num_pages x n_kv_heads over 2^30");
  return CRF_OK;
}

crf_status check_layer(const crf_kv_pool* pool, int layer) {
  if (!pool || !pool->k_pages || !pool->v_pages) return fail(CRF_EINVAL, "kv pool is null");
  if (layer < 0) return fail(CRF_EINVAL, "layer %d out of range", layer);
  if (!pool->k_pages[layer] || !pool->v_pages[layer] || !aligned16(pool->k_pages[layer]) || !aligned16(pool->v_pages[layer]))
    return fail(CRF_EINVAL, "kv pool layer %d null or misaligned", layer);
  return CRF_OK;
}

crf_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return CRF_OK;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return fail(CRF_EINVAL, "workspace null or not 256-byte aligned");
  if (have < need) return fail(CRF_ENOMEM, "workspace %zu bytes, %zu needed", have, need);
  return CRF_OK;
}

// rows: 0 where they are not known yet
crf_status check_attention(int n_q_heads, int n_kv_heads, int window, int64_t rows) {
  if (n_q_heads < 1 || n_kv_heads < 1) return fail(CRF_EINVAL, "heads must be positive");
  if (n_q_heads % n_kv_heads) return fail(CRF_ESHAPE, "%d query heads are no multiple of %d kv heads", n_q_heads, n_kv_heads);
  if (window < 0) return fail(CRF_EINVAL, "window must be >= 0");
  if (rows * n_q_heads > (1 << 30)) return fail(CRF_EUNSUPPORTED, "rows x query heads over 2^30");
  return CRF_OK;
}

// ---------------------------------------------------------------- heads of a call
// The arguments that calls on rows of heads share, checked, and their descriptor; it is left unset where there are no rows.
crf_status rotary_call(crf_ctx* ctx, const crf_rope* rope, const crf_heads* parts, int n_parts, int type, int n_rows,
                       const int32_t* positions, RotaryDesc* d) {
  if (!ctx || !rope || !parts) return fail(CRF_EINVAL, "null argument");
  crf_status s = check_rope(*rope);
  if (s != CRF_OK) return s;
  if (n_parts < 1 || n_parts > 2) return fail(CRF_EINVAL, "n_parts %d out of range (1 or 2)", n_parts);
  if (type < CRF_BF16 || type > CRF_FP32) return fail(CRF_EUNSUPPORTED, "unknown element type %d", type);
  if (n_rows < 0) return fail(CRF_EINVAL, "n_rows must be >= 0");
  if (n_rows == 0) return CRF_OK;
  if (!positions || !aligned4(positions)) return fail(CRF_EINVAL, "positions null or misaligned");
  std::memset(d, 0, sizeof(*d));
  for (int p = 0; p < n_parts; ++p) {
    const char* name = p ? "part 1" : "part 0";
    const crf_heads h = settled(parts[p], n_rows, rope->head_dim);
    s = check_heads(h, type == CRF_FP32 ? 4 : 2, true, name);
    if (s != CRF_OK) return s;
    s = check_out(h, n_rows, rope->head_dim, name);
    if (s != CRF_OK) return s;
    if (h.x == h.out && (h.x_row != h.out_row || h.x_head != h.out_head))
      return fail(CRF_ESHAPE, "%s: in place with other strides", name);
    d->part[p] = part_of(h, true);
  }
  d->n_parts = n_parts;
  d->head_dim = rope->head_dim;
  d->rot_dim = rope->rot_dim;
  d->interleaved = rope->layout == CRF_ROPE_INTERLEAVED;
  d->magnitude = static_cast<float>(rope->magnitude);
  d->n_rows = n_rows;
  d->positions = positions;
  d->type = type;
  d->status = ctx->status_dev;
  fill_turns(*rope, d->turns);
  return CRF_OK;
}

// The same of an append; no rows: t->row0[t->n] is 0 and *d unset.
crf_status append_call(crf_ctx* ctx, const crf_rope* rope, const crf_kv_pool* pool, int layer, int n_kv_heads, int head_dim,
                       const crf_chunk* chunks, int n_chunks, const crf_heads* q, const crf_heads* k, const crf_heads* v,
                       RotaryDesc* d, ChunkTable* t) {
  if (!ctx || !pool || !k || !v) return fail(CRF_EINVAL, "null argument");
  crf_status s = check_pool_shape(n_kv_heads, head_dim, pool->num_pages);
  if (s != CRF_OK) return s;
  s = check_layer(pool, layer);
  if (s != CRF_OK) return s;
  if (q && !rope) return fail(CRF_EINVAL, "q needs rope: there is nothing else to do with it");
  if (rope) {
    s = check_rope(*rope);
    if (s != CRF_OK) return s;
    if (rope->head_dim != head_dim) return fail(CRF_ESHAPE, "rope head_dim %d != head_dim %d", rope->head_dim, head_dim);
  }
  s = fill_chunks(chunks, n_chunks, false, pool->num_pages, t);
  if (s != CRF_OK) return s;
  const int rows = t->row0[t->n];
  if (rows == 0) return CRF_OK;
  const crf_heads hk = settled(*k, rows, head_dim), hv = settled(*v, rows, head_dim);
  s = check_heads(hk, 2, false, "k");
  if (s != CRF_OK) return s;
  s = check_heads(hv, 2, false, "v");
  if (s != CRF_OK) return s;
  if (k->heads != n_kv_heads || v->heads != n_kv_heads)
    return fail(CRF_ESHAPE, "k has %d and v %d heads, the pool %d", k->heads, v->heads, n_kv_heads);
  std::memset(d, 0, sizeof(*d));
  if (q) {
    const crf_heads hq = settled(*q, rows, head_dim);
    s = check_heads(hq, 2, true, "q");
    if (s != CRF_OK) return s;
    s = check_out(hq, rows, head_dim, "q");
    if (s != CRF_OK) return s;
    if (hq.x == hq.out && (hq.x_row != hq.out_row || hq.x_head != hq.out_head))
      return fail(CRF_ESHAPE, "q: in place with other strides");
    d->part[d->n_parts++] = part_of(hq, true);
  }
  RotPart kp = part_of(hk, rope != nullptr), vp = part_of(hv, false);
  kp.paged = vp.paged = true;
  kp.out = pool->k_pages[layer];
  vp.out = pool->v_pages[layer];
  d->part[d->n_parts++] = kp;
  d->part[d->n_parts++] = vp;
  d->head_dim = head_dim;
  d->rot_dim = rope ? rope->rot_dim : 2;
  if (rope) {
    d->interleaved = rope->layout == CRF_ROPE_INTERLEAVED;
    d->magnitude = static_cast<float>(rope->magnitude);
    fill_turns(*rope, d->turns);
  } else {
    d->rot_dim = head_dim;  // whole heads of units that no part rotates
  }
  d->n_rows = rows;
  d->n_kv_heads = n_kv_heads;
  d->type = CRF_BF16;
  d->status = ctx->status_dev;
  return CRF_OK;
}

crf_status check_norms(const crf_norm* norms, int n, int type, const void** gain, float* eps) {
  if (!norms) return fail(CRF_EINVAL, "norms is null");
  for (int i = 0; i < n; ++i) {
    if (!norms[i].gain || (reinterpret_cast<uintptr_t>(norms[i].gain) & (type == CRF_FP32 ? 3 : 1)))
      return fail(CRF_EINVAL, "norm %d: gain null or misaligned", i);
    if (!(norms[i].eps >= 0.f) || !std::isfinite(norms[i].eps)) return fail(CRF_EINVAL, "norm %d: eps must be finite and at least 0", i);
    gain[i] = norms[i].gain;
    eps[i] = norms[i].eps;
  }
  return CRF_OK;
}

// ---------------------------------------------------------------- logits
crf_status check_logits(int type, int n_rows, int vocab) {
  if (type < CRF_BF16 || type > CRF_FP32) return fail(CRF_EUNSUPPORTED, "unknown element type %d", type);
  if (vocab < 1 || vocab > CRF_MAX_VOCAB) return fail(CRF_EUNSUPPORTED, "vocab %d out of range (1..%d)", vocab, CRF_MAX_VOCAB);
  if (n_rows < 0) return fail(CRF_EINVAL, "n_rows must be >= 0");
  if (n_rows > (1 << 24)) return fail(CRF_EUNSUPPORTED, "n_rows %d over 2^24", n_rows);
  return CRF_OK;
}
crf_status check_rows_of(const void* x, int type, int n_rows, int vocab, int64_t stride, const char* name) {
  if (!x) return fail(CRF_EINVAL, "%s is null", name);
  if (reinterpret_cast<uintptr_t>(x) & (type == CRF_FP32 ? 3 : 1)) return fail(CRF_EINVAL, "%s: not aligned to its elements", name);
  if (n_rows > 1 && (stride < vocab || stride > (int64_t{1} << 40)))
    return fail(CRF_ESHAPE, "%s: row stride under vocab, or over 2^40", name);
  return CRF_OK;
}

// The sizes of an attention call, checked, and its table.
crf_status attention_sizes(crf_ctx* ctx, int n_q_heads, int n_kv_heads, int head_dim, const crf_chunk* chunks, int n_chunks,
                           int window, int sinks, ChunkTable* t) {
  if (!ctx) return fail(CRF_EINVAL, "ctx is null");
  crf_status s = check_attention(n_q_heads, n_kv_heads, window, 0);
  if (s != CRF_OK) return s;
  if (sinks < 0) return fail(CRF_EINVAL, "sinks must be >= 0");
  s = check_pool_shape(n_kv_heads, head_dim, 1);
  if (s != CRF_OK) return s;
  s = fill_chunks(chunks, n_chunks, true, 1, t);
  return s != CRF_OK ? s : check_attention(n_q_heads, n_kv_heads, window, t->row0[t->n]);
}

// The arguments that attention calls share, checked, and their descriptor; it is left unset where there are no rows.
crf_status attention_call(crf_ctx* ctx, const crf_kv_pool* pool, int layer, int n_kv_heads, int head_dim, const crf_chunk* chunks,
                          int n_chunks, const crf_heads* q, float* lse, float scale, int causal, int window, ChunkTable* t,
                          ChunkAttnDesc* d) {
  if (!ctx || !pool || !q) return fail(CRF_EINVAL, "null argument");
  crf_status s = check_pool_shape(n_kv_heads, head_dim, pool->num_pages);
  if (s != CRF_OK) return s;
  s = check_layer(pool, layer);
  if (s != CRF_OK) return s;
  s = check_attention(q->heads, n_kv_heads, window, 0);
  if (s != CRF_OK) return s;
  // the kernel multiplies scores by scale log2(e), in fp32
  if (!(scale >= 0.f) || !std::isfinite(scale * 1.4426950408889634f))
    return fail(CRF_EINVAL, "scale must be positive and under 2.35e38, or 0 for 1/sqrt(head_dim)");
  s = fill_chunks(chunks, n_chunks, true, pool->num_pages, t);
  if (s != CRF_OK) return s;
  const int rows = t->row0[t->n];
  if (rows == 0) return CRF_OK;
  s = check_attention(q->heads, n_kv_heads, window, rows);
  if (s != CRF_OK) return s;
  const crf_heads hq = settled(*q, rows, head_dim);
  s = check_heads(hq, 16, true, "q");
  if (s != CRF_OK) return s;
  if ((hq.x_row | hq.x_head | hq.out_row | hq.out_head) % 8)
    return fail(CRF_EUNSUPPORTED, "q: strides must be multiples of 8 elements");
  s = check_out(hq, rows, head_dim, "q");
  if (s != CRF_OK) return s;
  if (q->x == q->out) return fail(CRF_EINVAL, "q: o may not be written over q");
  if (!aligned4(lse)) return fail(CRF_EINVAL, "lse misaligned");
  d->q = static_cast<const __nv_bfloat16*>(q->x);
  d->out = static_cast<__nv_bfloat16*>(q->out);
  d->q_row = hq.x_row;
  d->q_head = hq.x_head;
  d->out_row = hq.out_row;
  d->out_head = hq.out_head;
  d->lse = lse;
  d->kpages = static_cast<const __nv_bfloat16*>(pool->k_pages[layer]);
  d->vpages = static_cast<const __nv_bfloat16*>(pool->v_pages[layer]);
  d->n_q_heads = q->heads;
  d->n_kv_heads = n_kv_heads;
  d->head_dim = head_dim;
  d->scale = scale > 0.f ? scale : static_cast<float>(1.0 / std::sqrt(static_cast<double>(head_dim)));
  d->causal = causal != 0;
  d->window = window;
  d->status = ctx->status_dev;
  return CRF_OK;
}

crf_status run_chunk_attention(crf_ctx* ctx, const ChunkAttnDesc& d, const ChunkTable& t, void* workspace, size_t ws_bytes,
                               cudaStream_t st) {
  ChunkPlan plan;
  plan_chunk_attention(t, d.n_q_heads, d.n_kv_heads, d.causal, d.window, ctx->num_sms, &plan);
  const crf_status s = check_workspace(workspace, ws_bytes, chunk_attention_workspace(plan, d.head_dim));
  if (s != CRF_OK) return s;
  DeviceScope dev(ctx->device);
  CRF_CUDA(dev.error());
  ProfScope ps(ctx, kPChunkAttn, st, plan.cuts ? 2 : 1);
  CRF_CUDA(launch_chunk_attention(d, t, plan, workspace, ctx->num_sms, st));
  return CRF_OK;
}

// The requests' groups, checked, and the table of those that share.
crf_status prefix_groups(const ChunkTable& t, const crf_prefix* prefixes, int n, int n_q_heads, int n_kv_heads, bool causal, int num_sms,
                         AttnTable* a, PrefixGroups* g) {
  if (!prefixes) return fail(CRF_EINVAL, "prefixes is null");
  if (n < 1 || n > t.n) return fail(CRF_EINVAL, "n_prefixes %d out of range (1..%d)", n, t.n);
  int count[CRF_MAX_CHUNKS], keys[CRF_MAX_CHUNKS], at = 0;
  for (int i = 0; i < n; ++i) {
    count[i] = prefixes[i].n_chunks;
    keys[i] = prefixes[i].n_shared;
    if (count[i] < 1 || count[i] > t.n - at) return fail(CRF_EINVAL, "prefix %d: n_chunks %d, %d requests are left", i, count[i], t.n - at);
    for (int j = at; j < at + count[i]; ++j) {
      if (t.row0[j + 1] == t.row0[j]) continue;
      if (keys[i] < 0 || keys[i] > t.n_keys[j] || (causal && keys[i] > t.pos[j]))
        return fail(CRF_EINVAL, "prefix %d: n_shared %d beyond the keys of chunk %d, or its new rows", i, keys[i], j);
    }
    at += count[i];
  }
  if (at != t.n) return fail(CRF_EINVAL, "the prefixes have %d requests, the call %d", at, t.n);
  share_prefixes(t, count, keys, n, n_q_heads, n_kv_heads, causal, num_sms, a, g);
  return CRF_OK;
}

crf_status check_parts(const AttnPlan& p) {
  if (p.part_rows > (1 << 30)) return fail(CRF_EUNSUPPORTED, "the rows' parts are over 2^30");
  return CRF_OK;
}

// ---------------------------------------------------------------- pages
crf_status fill_tables(const crf_pages* tables, int n, int num_pages, bool has_out, bool deep, PageTables* t) {
  if (!tables) return fail(CRF_EINVAL, "tables is null");
  if (n < 1 || n > CRF_MAX_TABLES) return fail(CRF_EINVAL, "n_tables %d out of range (1..%d)", n, CRF_MAX_TABLES);
  if (num_pages < 1 || num_pages > (1 << 30)) return fail(CRF_EINVAL, "num_pages %d out of range", num_pages);
  std::memset(t, 0, sizeof(*t));
  t->n = n;
  t->num_pages = num_pages;
  int64_t entries = 0, fresh = 0;
  for (int i = 0; i < n; ++i) {
    const crf_pages& p = tables[i];
    if (p.n_tokens < 0 || p.n_tokens > (1 << 30)) return fail(CRF_EINVAL, "table %d: n_tokens out of range", i);
    if (p.n_tokens > 0 && (!p.table || (has_out && !p.out))) return fail(CRF_EINVAL, "table %d: null pointer", i);
    if (!aligned4(p.table) || (has_out && !aligned4(p.out))) return fail(CRF_EINVAL, "table %d: misaligned pointer", i);
    t->first[i] = static_cast<int>(entries);
    t->fresh0[i] = static_cast<int>(fresh);
    t->n_tokens[i] = p.n_tokens;
    t->table[i] = p.table;
    t->out[i] = p.out;
    const int count = (p.n_tokens + kPage - 1) / kPage;
    entries += count;
    fresh += deep ? count : (p.n_tokens % kPage != 0);
    if (entries > (1 << 30)) return fail(CRF_EINVAL, "too many table entries");
  }
  for (int i = n; i <= CRF_MAX_TABLES; ++i) {
    t->first[i] = static_cast<int>(entries);
    t->fresh0[i] = static_cast<int>(fresh);
  }
  return CRF_OK;
}

crf_status run_pages(crf_ctx* ctx, PageOp op, const crf_kv_pool* pool, int n_layers, int n_kv_heads, int head_dim,
                     int num_pages, const int32_t* refs_in, int32_t* refs_out, const crf_pages* tables, int n_tables,
                     bool deep, void* workspace, size_t ws_bytes, void* stream) {
  if (!ctx) return fail(CRF_EINVAL, "ctx is null");
  if (!refs_in || !refs_out || !aligned4(refs_in) || !aligned4(refs_out))
    return fail(CRF_EINVAL, "reference counts null or misaligned");
  if (op != kPageRelease) {
    if (n_layers < 1) return fail(CRF_EINVAL, "n_layers must be positive");
    crf_status s = check_pool_shape(n_kv_heads, head_dim, num_pages);
    if (s != CRF_OK) return s;
    for (int l = 0; l < n_layers; ++l) {
      s = check_layer(pool, l);
      if (s != CRF_OK) return s;
    }
  }
  PageTables t;
  crf_status s = fill_tables(tables, n_tables, num_pages, op != kPageRelease, deep, &t);
  if (s != CRF_OK) return s;
  s = check_workspace(workspace, ws_bytes, page_workspace(num_pages, t.first[t.n]));
  if (s != CRF_OK) return s;
  DeviceScope dev(ctx->device);
  CRF_CUDA(dev.error());
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  PagePool pp{};
  if (pool) pp = PagePool{pool->k_pages, pool->v_pages, n_layers, n_kv_heads, head_dim};
  ProfScope ps(ctx, op == kPageRelease ? kPPagePlan : kPPageCopy, st, page_launches(op, t, n_layers));
  CRF_CUDA(launch_pages(op, t, deep, refs_in, refs_out, &pp, workspace, ctx->num_sms, ctx->status_dev, st));
  return CRF_OK;
}

}  // namespace

extern "C" {

crf_status crf_rotary(crf_ctx* ctx, const crf_rope* rope, const crf_heads* parts, int n_parts, int type, int n_rows,
                      const int32_t* positions, int inverse, void* stream) {
  return guarded([&]() -> crf_status {
    RotaryDesc d;
    const crf_status s = rotary_call(ctx, rope, parts, n_parts, type, n_rows, positions, &d);
    if (s != CRF_OK || n_rows == 0) return s;
    d.inverse = inverse != 0;
    DeviceScope dev(ctx->device);
    CRF_CUDA(dev.error());
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope ps(ctx, kPRotary, st);
    CRF_CUDA(launch_rotary(d, nullptr, ctx->num_sms, st));
    return CRF_OK;
  });
}

crf_status crf_norm_rotary(crf_ctx* ctx, const crf_rope* rope, const crf_heads* parts, const crf_norm* norms, int n_parts,
                           int type, int n_rows, const int32_t* positions, void* stream) {
  return guarded([&]() -> crf_status {
    HeadNormDesc d;
    std::memset(&d, 0, sizeof(d));
    crf_status s = rotary_call(ctx, rope, parts, n_parts, type, n_rows, positions, &d.r);
    if (s != CRF_OK) return s;
    s = check_norms(norms, n_parts, type, d.gain, d.eps);
    if (s != CRF_OK || n_rows == 0) return s;
    d.inv_dim = 1.0f / rope->head_dim;
    DeviceScope dev(ctx->device);
    CRF_CUDA(dev.error());
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope ps(ctx, kPHeadNorm, st);
    CRF_CUDA(launch_head_norm(d, nullptr, ctx->num_sms, st));
    return CRF_OK;
  });
}

crf_status crf_norm_rotary_workspace_size(crf_ctx* ctx, int head_dim, int n_rows, size_t* bytes) {
  return guarded([&]() -> crf_status {
    if (!ctx || !bytes) return fail(CRF_EINVAL, "null argument");
    if (head_dim < 2 || head_dim > 2 * kMaxPairs) return fail(CRF_EUNSUPPORTED, "head_dim %d unsupported", head_dim);
    if (n_rows < 0) return fail(CRF_EINVAL, "n_rows must be >= 0");
    *bytes = align256(head_norm_grad_workspace(head_dim, ctx->num_sms));
    return CRF_OK;
  });
}

crf_status crf_norm_rotary_grad(crf_ctx* ctx, const crf_rope* rope, const crf_heads* parts, const crf_norm* norms,
                                const crf_heads* grads, float* const* dgains, int n_parts, int type, int n_rows,
                                const int32_t* positions, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&]() -> crf_status {
    HeadNormGradDesc d;
    std::memset(&d, 0, sizeof(d));
    crf_status s = rotary_call(ctx, rope, parts, n_parts, type, n_rows, positions, &d.r);
    if (s != CRF_OK) return s;
    s = check_norms(norms, n_parts, type, d.gain, d.eps);
    if (s != CRF_OK) return s;
    if (!grads || !dgains) return fail(CRF_EINVAL, "null argument");
    d.r.n_parts = n_parts;
    d.r.head_dim = rope->head_dim;
    d.r.inverse = true;
    d.inv_dim = 1.0f / rope->head_dim;
    for (int p = 0; p < n_parts; ++p) {
      if (!dgains[p] || !aligned4(dgains[p])) return fail(CRF_EINVAL, "dgains[%d] null or misaligned", p);
      d.dgain[p] = dgains[p];
      if (n_rows == 0) continue;
      const char* name = p ? "grads 1" : "grads 0";
      const crf_heads g = settled(grads[p], n_rows, rope->head_dim);
      s = check_heads(g, type == CRF_FP32 ? 4 : 2, false, name);
      if (s != CRF_OK) return s;
      if (g.heads != parts[p].heads) return fail(CRF_ESHAPE, "%s: %d heads, x has %d", name, g.heads, parts[p].heads);
      if (g.x == d.r.part[p].out && (g.x_row != d.r.part[p].out_row || g.x_head != d.r.part[p].out_head))
        return fail(CRF_ESHAPE, "%s: written over with other strides", name);
      d.grad[p] = g.x;
      d.g_row[p] = g.x_row;
      d.g_head[p] = g.x_head;
    }
    if (n_parts == 2) {
      const uintptr_t a = reinterpret_cast<uintptr_t>(dgains[0]), b = reinterpret_cast<uintptr_t>(dgains[1]);
      if ((a < b ? b - a : a - b) < rope->head_dim * sizeof(float)) return fail(CRF_EINVAL, "dgains overlap: each part writes its own");
    }
    s = check_workspace(workspace, ws_bytes, head_norm_grad_workspace(rope->head_dim, ctx->num_sms));
    if (s != CRF_OK) return s;
    DeviceScope dev(ctx->device);
    CRF_CUDA(dev.error());
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope ps(ctx, kPHeadNormGrad, st, n_rows ? 2 : 0);
    CRF_CUDA(launch_head_norm_grad(d, static_cast<float*>(workspace), ctx->num_sms, st));
    return CRF_OK;
  });
}

crf_status crf_cache_append(crf_ctx* ctx, const crf_rope* rope, const crf_kv_pool* pool, int layer, int n_kv_heads,
                            int head_dim, const crf_chunk* chunks, int n_chunks, const crf_heads* q, const crf_heads* k,
                            const crf_heads* v, void* stream) {
  return guarded([&]() -> crf_status {
    RotaryDesc d;
    ChunkTable t;
    const crf_status s = append_call(ctx, rope, pool, layer, n_kv_heads, head_dim, chunks, n_chunks, q, k, v, &d, &t);
    if (s != CRF_OK || t.row0[t.n] == 0) return s;
    DeviceScope dev(ctx->device);
    CRF_CUDA(dev.error());
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope ps(ctx, kPAppend, st);
    CRF_CUDA(launch_rotary(d, &t, ctx->num_sms, st));
    return CRF_OK;
  });
}

crf_status crf_cache_append_normed(crf_ctx* ctx, const crf_rope* rope, const crf_kv_pool* pool, int layer, int n_kv_heads,
                                   int head_dim, const crf_chunk* chunks, int n_chunks, const crf_heads* q,
                                   const crf_norm* q_norm, const crf_heads* k, const crf_norm* k_norm, const crf_heads* v,
                                   void* stream) {
  return guarded([&]() -> crf_status {
    if (!rope || !k_norm || (q && !q_norm)) return fail(CRF_EINVAL, "null argument");
    HeadNormDesc d;
    std::memset(&d, 0, sizeof(d));
    crf_norm norms[2] = {q ? *q_norm : *k_norm, *k_norm};  // part 0 is q, or k without it
    crf_status s = check_norms(norms, q ? 2 : 1, CRF_BF16, d.gain, d.eps);
    if (s != CRF_OK) return s;
    ChunkTable t;
    s = append_call(ctx, rope, pool, layer, n_kv_heads, head_dim, chunks, n_chunks, q, k, v, &d.r, &t);
    if (s != CRF_OK || t.row0[t.n] == 0) return s;
    d.inv_dim = 1.0f / head_dim;
    DeviceScope dev(ctx->device);
    CRF_CUDA(dev.error());
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope ps(ctx, kPHeadNorm, st);
    CRF_CUDA(launch_head_norm(d, &t, ctx->num_sms, st));
    return CRF_OK;
  });
}

crf_status crf_logprobs(crf_ctx* ctx, const void* logits, int type, int n_rows, int vocab, int64_t row_stride,
                        const int32_t* targets, float* logprob, float* entropy, float* lse, int n_top, int32_t* top_ids,
                        float* top_logprobs, void* stream) {
  return guarded([&]() -> crf_status {
    if (!ctx) return fail(CRF_EINVAL, "ctx is null");
    crf_status s = check_logits(type, n_rows, vocab);
    if (s != CRF_OK) return s;
    if (n_top < 0 || n_top > CRF_MAX_TOP || n_top > vocab)
      return fail(CRF_EUNSUPPORTED, "n_top %d out of range (0..%d, at most vocab)", n_top, CRF_MAX_TOP);
    if (n_rows == 0) return CRF_OK;
    s = check_rows_of(logits, type, n_rows, vocab, row_stride, "logits");
    if (s != CRF_OK) return s;
    if (logprob && !targets) return fail(CRF_EINVAL, "logprob needs targets");
    if (n_top && !top_ids && !top_logprobs) return fail(CRF_EINVAL, "n_top without an output for it");
    if (!aligned4(targets) || !aligned4(logprob) || !aligned4(entropy) || !aligned4(lse) || !aligned4(top_ids) || !aligned4(top_logprobs))
      return fail(CRF_EINVAL, "targets or an output misaligned");
    LogprobsDesc d;
    d.z = logits;
    d.z_row = n_rows == 1 ? 0 : row_stride;
    d.type = type;
    d.n_rows = n_rows;
    d.vocab = vocab;
    d.n_top = n_top;
    d.targets = targets;
    d.logprob = logprob;
    d.entropy = entropy;
    d.lse = lse;
    d.top_ids = top_ids;
    d.top_logprobs = top_logprobs;
    d.status = ctx->status_dev;
    DeviceScope dev(ctx->device);
    CRF_CUDA(dev.error());
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope ps(ctx, kPLogprobs, st);
    CRF_CUDA(launch_logprobs(d, ctx->num_sms, st));
    return CRF_OK;
  });
}

crf_status crf_logprobs_grad(crf_ctx* ctx, const void* logits, int type, int n_rows, int vocab, int64_t row_stride,
                             const int32_t* targets, const float* lse, const float* entropy, const float* g_logprob,
                             const float* g_entropy, void* d_logits, int64_t d_row_stride, void* stream) {
  return guarded([&]() -> crf_status {
    if (!ctx) return fail(CRF_EINVAL, "ctx is null");
    crf_status s = check_logits(type, n_rows, vocab);
    if (s != CRF_OK || n_rows == 0) return s;
    s = check_rows_of(logits, type, n_rows, vocab, row_stride, "logits");
    if (s != CRF_OK) return s;
    s = check_rows_of(d_logits, type, n_rows, vocab, d_row_stride, "d_logits");
    if (s != CRF_OK) return s;
    if (logits == d_logits && n_rows > 1 && row_stride != d_row_stride) return fail(CRF_ESHAPE, "d_logits: in place with another stride");
    if (!lse) return fail(CRF_EINVAL, "lse is null");
    if (g_logprob && !targets) return fail(CRF_EINVAL, "g_logprob needs targets");
    if (g_entropy && !entropy) return fail(CRF_EINVAL, "g_entropy needs entropy");
    if (!aligned4(targets) || !aligned4(lse) || !aligned4(entropy) || !aligned4(g_logprob) || !aligned4(g_entropy))
      return fail(CRF_EINVAL, "targets, lse, entropy or a gradient misaligned");
    LogprobsGradDesc d;
    d.z = logits;
    d.dz = d_logits;
    d.z_row = n_rows == 1 ? 0 : row_stride;
    d.dz_row = n_rows == 1 ? 0 : d_row_stride;
    d.type = type;
    d.n_rows = n_rows;
    d.vocab = vocab;
    d.targets = g_logprob ? targets : nullptr;
    d.lse = lse;
    d.entropy = entropy;
    d.g_logprob = g_logprob;
    d.g_entropy = g_entropy;
    d.status = ctx->status_dev;
    DeviceScope dev(ctx->device);
    CRF_CUDA(dev.error());
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope ps(ctx, kPLogprobsGrad, st);
    CRF_CUDA(launch_logprobs_grad(d, st));
    return CRF_OK;
  });
}

crf_status crf_chunk_attention_workspace_size(crf_ctx* ctx, int n_q_heads, int n_kv_heads, int head_dim,
                                              const crf_chunk* chunks, int n_chunks, int causal, int window,
                                              size_t* bytes) {
  return crf_chunk_attention_sinks_workspace_size(ctx, n_q_heads, n_kv_heads, head_dim, chunks, n_chunks, causal, window, 0, bytes);
}

crf_status crf_chunk_attention_sinks_workspace_size(crf_ctx* ctx, int n_q_heads, int n_kv_heads, int head_dim,
                                                    const crf_chunk* chunks, int n_chunks, int causal, int window,
                                                    int sinks, size_t* bytes) {
  return guarded([&]() -> crf_status {
    if (!bytes) return fail(CRF_EINVAL, "null argument");
    ChunkTable t;
    crf_status s = attention_sizes(ctx, n_q_heads, n_kv_heads, head_dim, chunks, n_chunks, window, sinks, &t);
    if (s != CRF_OK) return s;
    size_t need;
    if (window > 0 && sinks > 0) {
      const SinksTable a{t, sinks};
      ChunkPlan plan;
      plan_sinks_attention(a, n_q_heads, n_kv_heads, causal != 0, window, ctx->num_sms, &plan);
      need = chunk_attention_workspace(plan, head_dim);
    } else {
      ChunkPlan plan;
      plan_chunk_attention(t, n_q_heads, n_kv_heads, causal != 0, window, ctx->num_sms, &plan);
      need = chunk_attention_workspace(plan, head_dim);
    }
    *bytes = align256(need);
    return CRF_OK;
  });
}

crf_status crf_chunk_attention(crf_ctx* ctx, const crf_kv_pool* pool, int layer, int n_kv_heads, int head_dim,
                               const crf_chunk* chunks, int n_chunks, const crf_heads* q, float* lse, float scale,
                               int causal, int window, void* workspace, size_t ws_bytes, void* stream) {
  return crf_chunk_attention_sinks(ctx, pool, layer, n_kv_heads, head_dim, chunks, n_chunks, q, lse, scale, causal, window, 0,
                                   workspace, ws_bytes, stream);
}

crf_status crf_chunk_attention_sinks(crf_ctx* ctx, const crf_kv_pool* pool, int layer, int n_kv_heads, int head_dim,
                                     const crf_chunk* chunks, int n_chunks, const crf_heads* q, float* lse, float scale,
                                     int causal, int window, int sinks, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&]() -> crf_status {
    ChunkTable t;
    ChunkAttnDesc d;
    crf_status s = attention_call(ctx, pool, layer, n_kv_heads, head_dim, chunks, n_chunks, q, lse, scale, causal, window, &t, &d);
    if (s != CRF_OK) return s;
    if (sinks < 0) return fail(CRF_EINVAL, "sinks must be >= 0");
    if (t.row0[t.n] == 0) return CRF_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (window > 0 && sinks > 0) {
      const SinksTable a{t, sinks};
      ChunkPlan plan;
      plan_sinks_attention(a, q->heads, n_kv_heads, causal != 0, window, ctx->num_sms, &plan);
      s = check_workspace(workspace, ws_bytes, chunk_attention_workspace(plan, head_dim));
      if (s != CRF_OK) return s;
      DeviceScope dev(ctx->device);
      CRF_CUDA(dev.error());
      ProfScope ps(ctx, kPChunkAttn, st, plan.cuts ? 2 : 1);
      CRF_CUDA(launch_sinks_attention(d, a, plan, workspace, ctx->num_sms, st));
      return CRF_OK;
    }
    return run_chunk_attention(ctx, d, t, workspace, ws_bytes, st);
  });
}

crf_status crf_prefix_attention_workspace_size(crf_ctx* ctx, int n_q_heads, int n_kv_heads, int head_dim,
                                               const crf_chunk* chunks, int n_chunks, const crf_prefix* prefixes,
                                               int n_prefixes, int causal, size_t* bytes) {
  return guarded([&]() -> crf_status {
    if (!bytes) return fail(CRF_EINVAL, "null argument");
    ChunkTable t;
    crf_status s = attention_sizes(ctx, n_q_heads, n_kv_heads, head_dim, chunks, n_chunks, 0, 0, &t);
    if (s != CRF_OK) return s;
    AttnTable a;
    PrefixGroups g;
    s = prefix_groups(t, prefixes, n_prefixes, n_q_heads, n_kv_heads, causal != 0, ctx->num_sms, &a, &g);
    if (s != CRF_OK) return s;
    size_t need;
    if (g.any) {
      AttnPlan plan;
      plan_prefix_attention(a, g.groups > 0, n_q_heads, n_kv_heads, causal != 0, ctx->num_sms, &plan);
      s = check_parts(plan);
      if (s != CRF_OK) return s;
      need = prefix_attention_workspace(plan, head_dim);
    } else {
      ChunkPlan plan;
      plan_chunk_attention(t, n_q_heads, n_kv_heads, causal != 0, 0, ctx->num_sms, &plan);
      need = chunk_attention_workspace(plan, head_dim);
    }
    *bytes = align256(need);
    return CRF_OK;
  });
}

crf_status crf_prefix_attention(crf_ctx* ctx, const crf_kv_pool* pool, int layer, int n_kv_heads, int head_dim,
                                const crf_chunk* chunks, int n_chunks, const crf_prefix* prefixes, int n_prefixes,
                                const crf_heads* q, float* lse, float scale, int causal, void* workspace, size_t ws_bytes,
                                void* stream) {
  return guarded([&]() -> crf_status {
    ChunkTable t;
    ChunkAttnDesc d;
    crf_status s = attention_call(ctx, pool, layer, n_kv_heads, head_dim, chunks, n_chunks, q, lse, scale, causal, 0, &t, &d);
    if (s != CRF_OK) return s;
    AttnTable a;
    PrefixGroups g;
    s = prefix_groups(t, prefixes, n_prefixes, q->heads, n_kv_heads, causal != 0, ctx->num_sms, &a, &g);
    if (s != CRF_OK || t.row0[t.n] == 0) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!g.any) return run_chunk_attention(ctx, d, t, workspace, ws_bytes, st);
    AttnPlan plan;
    plan_prefix_attention(a, g.groups > 0, q->heads, n_kv_heads, causal != 0, ctx->num_sms, &plan);
    s = check_parts(plan);
    if (s != CRF_OK) return s;
    s = check_workspace(workspace, ws_bytes, prefix_attention_workspace(plan, head_dim));
    if (s != CRF_OK) return s;
    DeviceScope dev(ctx->device);
    CRF_CUDA(dev.error());
    ProfScope ps(ctx, kPPrefixAttn, st, plan.shared || plan.runs.cuts ? 2 : 1);
    CRF_CUDA(launch_prefix_attention(d, a, g, plan, workspace, ctx->num_sms, st));
    return CRF_OK;
  });
}

crf_status crf_pages_workspace_size(crf_ctx* ctx, int num_pages, const crf_pages* tables, int n_tables, size_t* bytes) {
  return guarded([&]() -> crf_status {
    if (!ctx || !tables || !bytes) return fail(CRF_EINVAL, "null argument");
    if (n_tables < 1 || n_tables > CRF_MAX_TABLES) return fail(CRF_EINVAL, "n_tables %d out of range (1..%d)", n_tables, CRF_MAX_TABLES);
    if (num_pages < 1 || num_pages > (1 << 30)) return fail(CRF_EINVAL, "num_pages %d out of range", num_pages);
    int64_t entries = 0;
    for (int i = 0; i < n_tables; ++i) {
      if (tables[i].n_tokens < 0 || tables[i].n_tokens > (1 << 30)) return fail(CRF_EINVAL, "table %d: n_tokens out of range", i);
      entries += (tables[i].n_tokens + kPage - 1) / kPage;
    }
    if (entries > (1 << 30)) return fail(CRF_EINVAL, "too many table entries");
    *bytes = page_workspace(num_pages, static_cast<int>(entries));
    return CRF_OK;
  });
}

crf_status crf_pages_fork(crf_ctx* ctx, const crf_kv_pool* pool, int n_layers, int n_kv_heads, int head_dim,
                          const int32_t* refs_in, int32_t* refs_out, const crf_pages* tables, int n_tables, int deep,
                          void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&]() -> crf_status {
    if (!pool) return fail(CRF_EINVAL, "kv pool is null");
    return run_pages(ctx, kPageFork, pool, n_layers, n_kv_heads, head_dim, pool->num_pages, refs_in, refs_out, tables,
                     n_tables, deep != 0, workspace, ws_bytes, stream);
  });
}

crf_status crf_pages_compact(crf_ctx* ctx, const crf_kv_pool* pool, int n_layers, int n_kv_heads, int head_dim,
                             const int32_t* refs_in, int32_t* refs_out, const crf_pages* tables, int n_tables,
                             void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&]() -> crf_status {
    if (!pool) return fail(CRF_EINVAL, "kv pool is null");
    return run_pages(ctx, kPageCompact, pool, n_layers, n_kv_heads, head_dim, pool->num_pages, refs_in, refs_out, tables,
                     n_tables, false, workspace, ws_bytes, stream);
  });
}

crf_status crf_pages_release(crf_ctx* ctx, int num_pages, const int32_t* refs_in, int32_t* refs_out,
                             const crf_pages* tables, int n_tables, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&]() -> crf_status {
    return run_pages(ctx, kPageRelease, nullptr, 0, 0, 0, num_pages, refs_in, refs_out, tables, n_tables, false,
                     workspace, ws_bytes, stream);
  });
}

}  // extern "C"
