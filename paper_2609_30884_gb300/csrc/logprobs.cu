// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the gradient. For a row z:
//   lse = log sum exp z,   logprob = z_t - lse,   entropy = lse - sum p z  with  p = exp(z - lse),
// and with g, h the gradients of logprob and entropy
//   dz_v = g (1[v = t] - p_v) - h p_v (log p_v + entropy).
//
// Forward: bound by reading the row once. A lane keeps a running maximum m, s = sum 2^x and d = sum 2^x x with
// x = (z - m) log2 e, in fp32 (entropy = log s - d log 2 / s); differences are formed before the product, so that the rounding of
// m log2 e stays out. A row is one CTA's, or the CTAs of a cluster's where rows are few; their sums meet in shared memory.
//
// The alternatives take no pass of their own over the row. The maximum of every 256 elements (a segment) is noted on the
// way. Keys (value, then lower index) order all elements; the k greatest elements lie in the k segments of greatest maxima, because a
// segment that is left out has k segments before it, each with an element of a greater key than any of its own. So k segments
// are read again (from L2), and the elements that reach the k-th greatest maximum, some 1.5 k of them as a rule, are ranked by
// counting. Where they are many (equal logits, rows that rise along the vocabulary), the k-th greatest key is found by
// bisection first. Nothing here depends on the order in which threads run.
//
// Rows start at any element: a row is cut at 16-byte addresses, its first and last pieces element by element.
#include "../../include/crf.h"
#include "rotary.cuh"

#include <algorithm>
#include <cstring>

namespace crf {

namespace {

constexpr int kLogThreads = 512;   // at most
constexpr int kStrip = 1024;       // elements of a warp's step
constexpr int kSegment = 256;      // elements that share a maximum
constexpr int kList = 512;         // elements that are ranked by counting
constexpr int kLogSmem = ((kMaxVocab + 16) / kSegment + 8 + kMaxTop * kSegment) * 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFloor = -200.f;   // 2^x is 0 from here down; keeps an infinite x out of products

// The greater, or NaN if either is NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Whole numbers that order floats: NaN 1, -inf above it; 0 is below every value.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 1u;
  const uint32_t b = __float_as_uint(v + 0.f);  // both zeros are equal
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  if (order <= 1u) return NAN;
  return __uint_as_float(order >> 31 ? order & 0x7fffffffu : ~order);
}

// A running maximum, sum of 2^x and sum of 2^x x.
struct Sums {
  float m, s, d;
  // over to the maximum `to` (not less than m)
  __device__ __forceinline__ void raise(float to) {
    if (s != 0.f) {  // NaN too: it stays one
      const float x = (m - to) * kLog2e, f = ex2_approx(x);
      d = f * (d + s * max_nan(x, kFloor));
      s *= f;
    }
    m = to;
  }
  __device__ __forceinline__ void add(const Sums& o) {
    Sums other = o;
    const float to = fmaxf(m, o.m);
    if (to == -INFINITY) {
      s += o.s;  // nothing, or NaN
      d += o.d;
      return;
    }
    raise(to);
    other.raise(to);
    s += other.s;
    d += other.d;
  }
};

struct LogArgs {
  LogprobsDesc d;
  int segments;  // room for a row's
};

struct LogShared {
  Sums part[kLogThreads / 32];
  Sums cta;                         // read by the cluster's first CTA
  int count[2][kLogThreads / 32];
  int chosen[kMaxTop];              // segments
  unsigned long long list[kList];
  int n_list, n_above, n_equal[kLogThreads / 32];
};

__device__ __forceinline__ uint32_t ld_cluster_u32(const void* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ float ld_cluster_f32(const void* p, uint32_t rank) { return __uint_as_float(ld_cluster_u32(p, rank)); }

// Threads' counts, summed over the block. Calls take turns at the two rows of `count`, so one barrier a call is enough.
__device__ __forceinline__ int block_count(LogShared& sh, int mine, int& turn) {
  const int warps = blockDim.x / 32;
  const int w = __reduce_add_sync(0xffffffffu, mine);
  if (threadIdx.x % 32 == 0) sh.count[turn & 1][threadIdx.x / 32] = w;
  __syncthreads();
  int n = 0;
  for (int i = 0; i < warps; ++i) n += sh.count[turn & 1][i];
  ++turn;
  return n;
}

template <typename T>
__device__ __forceinline__ float load_logit(const T* p) {
  float f[1];
  unpack(*reinterpret_cast<const Unit<T, 1>*>(p), f);
  return f[0];
}

// C: CTAs of a row, a cluster.
template <typename T, int C>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(kLogThreads, 2) logprobs_kernel(const __grid_constant__ LogArgs a) {
  constexpr int VEC = 16 / sizeof(T), kLoads = kStrip / (32 * VEC), kPerSegment = kSegment / (32 * VEC);
  static_assert(kPerSegment >= 1 && kLoads == 4 * kPerSegment, "a strip is four segments");
  __shared__ LogShared sh;
  extern __shared__ uint32_t s_dyn[];
  uint32_t* s_max = s_dyn;                   // [segment of the row]: those of this CTA's strips; then of all
  uint32_t* s_key = s_dyn + a.segments;      // [chosen segment][256]: orders
  griddep_launch_dependents();
  const LogprobsDesc& d = a.d;
  const int row = blockIdx.x / C, rank = C > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const bool top = d.n_top > 0;
  const T* z = static_cast<const T*>(d.z) + row * d.z_row;
  // virtual index v = element + skew: 16-byte aligned where v is a multiple of VEC
  const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int end = d.vocab + skew, strips = (end + kStrip - 1) / kStrip, segments = (end + kSegment - 1) / kSegment;
  const T* base = z - skew;  // never read before z
  Sums acc{-INFINITY, 0.f, 0.f};
  griddep_wait();
  for (int st = rank * warps + warp; st < strips; st += C * warps) {
    const int v0 = st * kStrip;
    float seg[4];
    if (v0 >= skew && v0 + kStrip <= end) {
      Unit<T, VEC> u[kLoads];
#pragma unroll
      for (int j = 0; j < kLoads; ++j) u[j] = *reinterpret_cast<const Unit<T, VEC>*>(base + v0 + (j * 32 + lane) * VEC);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        seg[g] = NAN;
#pragma unroll
        for (int j = g * kPerSegment; j < (g + 1) * kPerSegment; ++j) {
          float x[VEC];
          unpack(u[j], x);
#pragma unroll
          for (int i = 0; i < VEC; i += 2) seg[g] = fmax3(seg[g], x[i], x[i + 1]);
        }
      }
      const float mx = fmaxf(fmaxf(seg[0], seg[1]), fmaxf(seg[2], seg[3]));
      if (mx > acc.m) acc.raise(mx);
      const float neg = acc.m == -INFINITY ? 0.f : -acc.m;
      const uint64_t neg2 = f32x2(neg, neg), l2e = f32x2(kLog2e, kLog2e), one = f32x2(1.f, 1.f);
      uint64_t s2 = f32x2(0.f, 0.f), d2 = f32x2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        float x[VEC];
        unpack(u[j], x);
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
          float t0, t1;
          f32x2_split(fma_f32x2(add_f32x2(f32x2(x[i], x[i + 1]), neg2), l2e, f32x2(0.f, 0.f)), t0, t1);
          t0 = max_nan(t0, kFloor);
          t1 = max_nan(t1, kFloor);
          const uint64_t e = f32x2(ex2_approx(t0), ex2_approx(t1));
          s2 = fma_f32x2(e, one, s2);
          d2 = fma_f32x2(e, f32x2(t0, t1), d2);
        }
      }
      float s0, s1;
      f32x2_split(s2, s0, s1);
      acc.s += s0 + s1;
      f32x2_split(d2, s0, s1);
      acc.d += s0 + s1;
    } else {
      // a first or last strip, element by element; what lies outside the row is NaN to the maxima and no part of the sums
      float x[kStrip / 32];
      auto inside = [&](int j) { const int v = v0 + j * 32 + lane; return v >= skew && v < end; };
#pragma unroll
      for (int j = 0; j < kStrip / 32; ++j) x[j] = inside(j) ? load_logit(base + v0 + j * 32 + lane) : NAN;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        seg[g] = NAN;
#pragma unroll
        for (int j = 0; j < kSegment / 32; ++j) seg[g] = fmaxf(seg[g], x[g * (kSegment / 32) + j]);
      }
      const float mx = fmaxf(fmaxf(seg[0], seg[1]), fmaxf(seg[2], seg[3]));
      if (mx > acc.m) acc.raise(mx);
      const float m = acc.m == -INFINITY ? 0.f : acc.m;
#pragma unroll
      for (int j = 0; j < kStrip / 32; ++j) {
        if (!inside(j)) continue;
        const float t = max_nan((x[j] - m) * kLog2e, kFloor), e = ex2_approx(t);
        acc.s += e;
        acc.d += e * t;
      }
    }
    if (top) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        // (a lane without elements says 1, as one of NaN alone does)
        const uint32_t o = __reduce_max_sync(0xffffffffu, order_of(seg[g]));
        if (lane == 0 && st * 4 + g < segments) s_max[st * 4 + g] = o;
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) {
    Sums other;
    other.m = __shfl_xor_sync(0xffffffffu, acc.m, o);
    other.s = __shfl_xor_sync(0xffffffffu, acc.s, o);
    other.d = __shfl_xor_sync(0xffffffffu, acc.d, o);
    acc.add(other);
  }
  if (lane == 0) sh.part[warp] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < warps; ++w) acc.add(sh.part[w]);
    sh.cta = acc;
  }
  if (C > 1) {
    cluster_sync();
    if (rank != 0) {
      cluster_sync();  // the first CTA has read what it needs
      return;
    }
    if (threadIdx.x == 0) {
      for (int r = 1; r < C; ++r) {
        Sums o;
        o.m = ld_cluster_f32(&sh.cta.m, r);
        o.s = ld_cluster_f32(&sh.cta.s, r);
        o.d = ld_cluster_f32(&sh.cta.d, r);
        acc.add(o);
      }
      sh.cta = acc;
    }
    if (top)
      for (int i = threadIdx.x; i < segments; i += blockDim.x) {
        const int r = i / 4 / warps % C;
        if (r != 0) s_max[i] = ld_cluster_u32(s_max + i, r);
      }
    cluster_sync();
  } else {
    __syncthreads();
  }
  const float s = sh.cta.s, log_s = logf(s), lse = s == 0.f ? -INFINITY : sh.cta.m + log_s;
  if (threadIdx.x == 0) {
    if (d.lse) d.lse[row] = lse;
    if (d.entropy) d.entropy[row] = s == 0.f ? 0.f : log_s - sh.cta.d * kLn2 / s;
    if (d.logprob) {
      int t = d.targets[row];
      float lp = 0.f;
      if (t != -1) {
        t = checked_token(t, d.vocab, d.status);
        const float v = load_logit(z + t);
        lp = s == 0.f ? -INFINITY : v - lse;
      }
      d.logprob[row] = lp;
    }
  }
  if (!top) return;

  // ---------------------------------------------------------------- the k segments of greatest maxima
  int turn = 0;
  const int k = d.n_top, take = min(k, segments);
  uint32_t least = 0;  // the `take`-th greatest maximum
  if (segments > take) {
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t cand = least | (1u << bit);
      int n = 0;
      for (int i = threadIdx.x; i < segments; i += blockDim.x) n += s_max[i] >= cand;
      if (block_count(sh, n, turn) >= take) least = cand;
    }
  }
  // all above it, and the first of those equal to it
  {
    int above = 0;
    for (int i = threadIdx.x; i < segments; i += blockDim.x) above += s_max[i] > least;
    const int n_above = block_count(sh, above, turn);
    if (threadIdx.x == 0) sh.n_above = sh.n_list = 0;
    __syncthreads();
    int before = 0;  // equal ones in the rounds and warps before
    for (int i0 = 0; i0 < segments; i0 += blockDim.x) {
      const int i = i0 + threadIdx.x;
      const uint32_t v = i < segments ? s_max[i] : 0u;
      const bool eq = i < segments && v == least;
      if (i < segments && v > least) sh.chosen[atomicAdd(&sh.n_above, 1)] = i;
      const uint32_t mask = __ballot_sync(0xffffffffu, eq);
      if (lane == 0) sh.n_equal[warp] = __popc(mask);
      __syncthreads();
      int at = before;
      for (int w = 0; w < warps; ++w) {
        if (w < warp) at += sh.n_equal[w];
        before += sh.n_equal[w];
      }
      at += __popc(mask & ((1u << lane) - 1));
      if (eq && n_above + at < take) sh.chosen[n_above + at] = i;
      __syncthreads();
    }
  }
  // ---------------------------------------------------------------- their elements
  for (int c = warp; c < take; c += warps) {
    const int v0 = sh.chosen[c] * kSegment;
#pragma unroll
    for (int j = 0; j < kSegment; j += 32) {
      const int v = v0 + j + lane;
      s_key[c * kSegment + j + lane] = v >= skew && v < end ? order_of(load_logit(base + v)) : 0u;
    }
  }
  __syncthreads();
  auto key_of = [&](int e) {
    const int v = sh.chosen[e / kSegment] * kSegment + e % kSegment - skew;
    return static_cast<unsigned long long>(s_key[e]) << 32 | ~static_cast<uint32_t>(v);
  };
  // The list: elements that reach the k-th greatest maximum (every element where the segments are fewer than k).
  const uint32_t reach = max(least, 1u);
  const int elements = take * kSegment;
  int n = 0;
  for (int e = threadIdx.x; e < elements; e += blockDim.x) n += s_key[e] >= reach;
  const int reached = block_count(sh, n, turn);
  unsigned long long from = static_cast<unsigned long long>(reach) << 32;
  if (reached > kList) {
    from = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long cand = from | (1ull << bit);
      n = 0;
      for (int e = threadIdx.x; e < elements; e += blockDim.x) n += s_key[e] != 0 && key_of(e) >= cand;
      if (block_count(sh, n, turn) >= k) from = cand;
    }
  }
  for (int e = threadIdx.x; e < elements; e += blockDim.x)
    if (s_key[e] != 0 && key_of(e) >= from) sh.list[atomicAdd(&sh.n_list, 1)] = key_of(e);
  __syncthreads();
  const int listed = sh.n_list;
  for (int i = threadIdx.x; i < listed; i += blockDim.x) {
    const unsigned long long mine = sh.list[i];
    int before = 0;
    for (int j = 0; j < listed; ++j) before += sh.list[j] > mine;
    if (before < k) {
      if (d.top_ids) d.top_ids[static_cast<int64_t>(row) * k + before] = static_cast<int32_t>(~static_cast<uint32_t>(mine));
      if (d.top_logprobs) {
        const float v = value_of(static_cast<uint32_t>(mine >> 32));
        d.top_logprobs[static_cast<int64_t>(row) * k + before] = s == 0.f ? -INFINITY : v - lse;
      }
    }
  }
}

// ---------------------------------------------------------------- gradient
constexpr int kGradThreads = 256, kGradLoads = 4;

struct LogGradArgs {
  LogprobsGradDesc d;
};

// One element's gradient: x = log p.
__device__ __forceinline__ float grad_of(float x, float g, float h, float entropy) {
  const float l = max_nan(x, kFloor);
  return -ex2_approx(l * kLog2e) * (g + h * (l + entropy));
}

// VEC elements a load where z and dz lie alike, else 1. A block takes kGradThreads kGradLoads units of a row.
template <typename T, int VEC>
__global__ void __launch_bounds__(kGradThreads) logprobs_grad_kernel(const __grid_constant__ LogGradArgs a) {
  using U = Unit<T, VEC>;
  griddep_launch_dependents();
  const LogprobsGradDesc& d = a.d;
  const int64_t row = blockIdx.y + static_cast<int64_t>(blockIdx.z) * gridDim.y;
  if (row >= d.n_rows) return;
  const T* z = static_cast<const T*>(d.z) + row * d.z_row;
  T* out = static_cast<T*>(d.dz) + row * d.dz_row;
  const int skew = VEC > 1 ? static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T)) : 0;
  const int end = d.vocab + skew, units = (end + VEC - 1) / VEC;
  const int u0 = blockIdx.x * (kGradThreads * kGradLoads) + threadIdx.x;
  griddep_wait();
  U u[kGradLoads];
#pragma unroll
  for (int j = 0; j < kGradLoads; ++j) {
    const int v = (u0 + j * kGradThreads) * VEC;
    if (v >= skew && v + VEC <= end) u[j] = *reinterpret_cast<const U*>(z - skew + v);
  }
  const float lse = d.lse[row];
  int t = d.targets ? d.targets[row] : -1;
  if (t != -1) t = checked_token(t, d.vocab, d.status);
  const float g = t != -1 && d.g_logprob ? d.g_logprob[row] : 0.f;
  const float h = d.g_entropy ? d.g_entropy[row] : 0.f, entropy = d.g_entropy ? d.entropy[row] : 0.f;
  const bool empty = lse == -INFINITY;  // a row without a finite logit has no gradient
#pragma unroll
  for (int j = 0; j < kGradLoads; ++j) {
    const int v = (u0 + j * kGradThreads) * VEC;
    if (v >= skew && v + VEC <= end) {
      float x[VEC];
      unpack(u[j], x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        float y = empty ? 0.f : grad_of(x[i] - lse, g, h, entropy);
        if (v + i - skew == t && !empty) y += g;
        x[i] = y;
      }
      pack(x, u[j]);
      *reinterpret_cast<U*>(out - skew + v) = u[j];
    } else if (u0 + j * kGradThreads < units) {
#pragma unroll 1
      for (int i = max(0, skew - v); i < VEC && v + i < end; ++i) {
        const int e = v + i - skew;
        float y = empty ? 0.f : grad_of(load_logit(z + e) - lse, g, h, entropy);
        if (e == t && !empty) y += g;
        const float f[1] = {y};
        pack(f, *reinterpret_cast<Unit<T, 1>*>(out + e));
      }
    }
  }
}

// ---------------------------------------------------------------- launches
template <typename T, int C>
cudaError_t launch_log(const LogArgs& a, int threads, cudaStream_t stream) {
  const size_t smem = a.d.n_top > 0 ? (static_cast<size_t>(a.segments) + static_cast<size_t>(a.d.n_top) * kSegment) * sizeof(uint32_t) : 0;
  static PerDevice once;
  int dev = 0;
  if (once.pending(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(logprobs_kernel<T, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLogSmem);
    if (e != cudaSuccess) return e;
    once.done(dev);
  }
  PdlScope pdl;
  return launch_kernel(logprobs_kernel<T, C>, dim3(static_cast<unsigned>(a.d.n_rows) * C), dim3(threads), smem, stream, a);
}

template <typename T>
cudaError_t launch_type(const LogprobsDesc& d, int num_sms, cudaStream_t stream) {
  LogArgs a;
  a.d = d;
  a.segments = ((d.vocab + 15) / kSegment + 1 + 3) / 4 * 4;
  const int strips = (d.vocab + 15 + kStrip - 1) / kStrip;
  // a row's CTAs: enough that few rows fill the SMs, each with a strip a warp at least
  int c = 1;
  while (c < 8 && static_cast<int64_t>(d.n_rows) * c < num_sms && strips >= 2 * c) c *= 2;
  const int threads = 32 * std::min(kLogThreads / 32, (strips + c - 1) / c);
  switch (c) {
    case 1: return launch_log<T, 1>(a, threads, stream);
    case 2: return launch_log<T, 2>(a, threads, stream);
    case 4: return launch_log<T, 4>(a, threads, stream);
  }
  return launch_log<T, 8>(a, threads, stream);
}

template <typename T>
cudaError_t launch_grad_type(const LogprobsGradDesc& d, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  LogGradArgs a{d};
  // every row of z and dz starts at the same place of a 16-byte piece
  const bool alike = ((reinterpret_cast<uintptr_t>(d.z) ^ reinterpret_cast<uintptr_t>(d.dz)) & 15) == 0 && (d.n_rows == 1 || (d.z_row - d.dz_row) % VEC == 0);
  const int vec = alike ? VEC : 1;
  const int64_t per = static_cast<int64_t>(kGradThreads) * kGradLoads * vec;
  const unsigned rows = static_cast<unsigned>(std::min(d.n_rows, 32768)), z = static_cast<unsigned>((static_cast<int64_t>(d.n_rows) + rows - 1) / rows);
  const dim3 grid(static_cast<unsigned>((d.vocab + vec - 1 + per - 1) / per), rows, z);
  PdlScope pdl;
  return alike ? launch_kernel(logprobs_grad_kernel<T, VEC>, grid, dim3(kGradThreads), 0, stream, a)
               : launch_kernel(logprobs_grad_kernel<T, 1>, grid, dim3(kGradThreads), 0, stream, a);
}

}  // namespace

cudaError_t launch_logprobs(const LogprobsDesc& d, int num_sms, cudaStream_t stream) {
  switch (d.type) {
    case CRF_BF16: return launch_type<__nv_bfloat16>(d, num_sms, stream);
    case CRF_FP16: return launch_type<__half>(d, num_sms, stream);
    case CRF_FP32: return launch_type<float>(d, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

cudaError_t launch_logprobs_grad(const LogprobsGradDesc& d, cudaStream_t stream) {
  switch (d.type) {
    case CRF_BF16: return launch_grad_type<__nv_bfloat16>(d, stream);
    case CRF_FP16: return launch_grad_type<__half>(d, stream);
    case CRF_FP32: return launch_grad_type<float>(d, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace crf
