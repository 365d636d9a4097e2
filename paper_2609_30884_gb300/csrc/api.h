// What the translation units of the C ABI layer share: the context, error reporting and per-launch timing.
#pragma once

#include "../../include/crf.h"
#include "kernels.h"

#include <cstddef>
#include <cstdint>
#include <vector>

struct crf_ctx {
  int device;
  int num_sms;
  int* status_dev;
  // per-launch timing (crf_profile_enable)
  bool prof_on = false;
  std::vector<cudaEvent_t> ev;
  int ev_used = 0;
  struct Rec {
    int kind, idx, kernels;
  };
  std::vector<Rec> rec;
  int dropped = 0;
};

namespace crf {

enum ProfKind : int {
  kPQkv, kPO, kPGateUp, kPDown, kPAttn, kPNorm, kPEmbed, kPCopy,
  kPDecode, kPLmHead, kPKl, kPDrift, kPCheck, kPRotary, kPAppend, kPChunkAttn, kPPagePlan, kPPageCopy,
  kPHeadNorm, kPHeadNormGrad, kPLogprobs, kPLogprobsGrad, kPPrefixAttn, kPNumKinds
};

// Brackets the launches issued in its lifetime with two events on `st` when
// profiling is on; `kernels` is how many kernels those launches are.
struct ProfScope {
  crf_ctx* c;
  int kind, kernels, idx;
  cudaStream_t st;
  ProfScope(crf_ctx* c_, int kind_, cudaStream_t st_, int kernels_ = 1)
      : c(c_), kind(kind_), kernels(kernels_), idx(-1), st(st_) {
    if (!c->prof_on) return;
    if (c->ev_used + 2 > static_cast<int>(c->ev.size())) {
      c->dropped += kernels;
      return;
    }
    idx = c->ev_used;
    c->ev_used += 2;
    cudaEventRecord(c->ev[idx], st);
  }
  ~ProfScope() {
    if (idx >= 0) {
      cudaEventRecord(c->ev[idx + 1], st);
      c->rec.push_back({kind, idx, kernels});
    }
  }
};

// Records the message of crf_last_error and returns `st`.
crf_status fail(crf_status st, const char* fmt, ...);

#define CRF_CUDA(expr)                                                                  \
  do {                                                                                  \
    cudaError_t _e = (expr);                                                            \
    if (_e != cudaSuccess)                                                              \
      return fail(CRF_ECUDA, "%s failed: %s (%s:%d)", #expr, cudaGetErrorString(_e), __FILE__, \
                  __LINE__);                                                            \
  } while (0)

inline size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace crf
