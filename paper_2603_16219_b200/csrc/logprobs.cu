// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits, in one read of the logits.
//
// Sums.  A thread walks its share of a row in chunks of 64 bytes.  With l = c x, c = log2(e)/temperature, it keeps
//   S = sum 2^(l - ref),   W = sum 2^(l - ref) (l - ref)
// for a reference that follows its largest l at a distance of at most 8, so that S and W are rescaled for hardly any chunk; brought
// together at M = max l they give  lse = M + log2 S  and  entropy = log2 S - W/S, in units of log 2.  The difference of logits is
// formed before it is scaled, so that entries of the type's lowest value, and rows of nothing else, stay in float32's range.
//
// The likeliest tokens.  Besides the sums a thread leaves nothing behind but the maximum of each of its slots (one or several
// chunks) in shared memory.  The n_top-th largest of the threads' maxima is a value that at least n_top entries reach, and only
// the slots that reach it, hardly more than n_top of them, are read again, from L2, by warps that keep their best entries as
// a list of one 64-bit key a lane (larger value first, then lower id).  So the stream carries no selection at all.  A slot whose best
// possible key does not beat the list's is not read: rows with many equal entries (a masked vocabulary) cost little more.
//
// Few rows are split over clusters of up to 8 CTAs, whose parts the first one joins through distributed shared memory.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "f32x2.cuh"
#include "paged.h"
#include "specsteer.h"

namespace specsteer {
namespace {

typedef long long i64;
constexpr int kLogThreads = 256, kLogWarps = kLogThreads / 32;
constexpr int kVecs = 4;             // vectors of 16 bytes a thread has in a chunk
constexpr int kSlots = 16;           // of a thread at most
constexpr float kSlack = 8.f;        // how far l may be above the reference
constexpr float kLeast = 1024.f;     // and below: there a weight is zero, and its product with the distance too

// The types of logits: elements of a vector, the pair in a 32-bit word (16-bit types), -inf in every element, the largest of a vector.
template <int DT> struct Logit;
template <> struct Logit<SPECSTEER_F32> {
  typedef float type;
  static constexpr int N = 4;
  static constexpr uint32_t kNone = 0xff800000u;
  static __device__ __forceinline__ float one(const float* x) { return *x; }
  static __device__ __forceinline__ float2 pair(const uint4& v, int i) {
    return i == 0 ? make_float2(__uint_as_float(v.x), __uint_as_float(v.y)) : make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  static __device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
  }
  static __device__ __forceinline__ float largest(const uint4 (&v)[kVecs]) {
    float m = __uint_as_float(v[0].x);
#pragma unroll
    for (int u = 0; u < kVecs; ++u) m = max3_nan(max3_nan(m, __uint_as_float(v[u].x), __uint_as_float(v[u].y)), __uint_as_float(v[u].z), __uint_as_float(v[u].w));
    return m;
  }
};
template <> struct Logit<SPECSTEER_BF16> {
  typedef __nv_bfloat16 type;
  static constexpr int N = 8;
  static constexpr uint32_t kNone = 0xff80ff80u;
  static __device__ __forceinline__ float one(const type* x) { return __bfloat162float(*x); }
  static __device__ __forceinline__ float2 pair(const uint4& v, int i) {
    const uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
    return make_float2(bf16lo(w), bf16hi(w));
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float largest(const uint4 (&v)[kVecs]) {
    uint32_t m = v[0].x;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) m = max2(max2(m, v[u].x), max2(v[u].y, max2(v[u].z, v[u].w)));
    m = max2(m, (m >> 16) | (m << 16));
    return bf16lo(m);
  }
};
template <> struct Logit<SPECSTEER_F16> {
  typedef __half type;
  static constexpr int N = 8;
  static constexpr uint32_t kNone = 0xfc00fc00u;
  static __device__ __forceinline__ float one(const type* x) { return __half2float(*x); }
  static __device__ __forceinline__ float2 pair(const uint4& v, int i) {
    const uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float largest(const uint4 (&v)[kVecs]) {
    uint32_t m = v[0].x;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) m = max2(max2(m, v[u].x), max2(v[u].y, max2(v[u].z, v[u].w)));
    m = max2(m, (m >> 16) | (m << 16));
    return __half2float(__ushort_as_half((unsigned short)m));
  }
};

// S and W of a thread, with their reference (a logit; none yet: -inf).
struct Sums {
  float ref, s, w;
};
__device__ __forceinline__ void rescale(Sums& a, float to, float c) {
  if (a.ref == kNegInf) {
    a.s = a.s == a.s ? 0.f : a.s;   // NaN stays
    a.w = 0.f;
  } else {
    const float d = fmaxf((a.ref - to) * c, -kLeast), f = ex2(d);
    a.w = fmaf(a.s, d, a.w) * f;
    a.s *= f;
  }
  a.ref = to;
}
// Takes a chunk in; returns its largest entry.
template <int DT> __device__ __forceinline__ float take(Sums& a, const uint4 (&v)[kVecs], float c) {
  typedef Logit<DT> L;
  const float mx = L::largest(v);
  if (mx > kNegInf && mx < -kNegInf) {
    if (a.ref == kNegInf || (mx - a.ref) * c > kSlack) rescale(a, mx, c);
    const float2 c2 = make_float2(c, c), r2 = make_float2(-a.ref, -a.ref);
    float2 s[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, w[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
#pragma unroll
      for (int i = 0; i < L::N / 2; ++i) {
        float2 t = mul2(add2(L::pair(v[u], i), r2), c2);
        t = make_float2(fmaxf(t.x, -kLeast), fmaxf(t.y, -kLeast));
        const float2 e = make_float2(ex2(t.x), ex2(t.y));
        s[i & 1] = add2(s[i & 1], e);
        w[i & 1] = fma2(e, t, w[i & 1]);
      }
    }
    s[0] = add2(s[0], s[1]);
    w[0] = add2(w[0], w[1]);
    a.s += s[0].x + s[0].y;
    a.w += w[0].x + w[0].y;
  } else if (mx != kNegInf) {
    a.s = __int_as_float(0x7fc00000);   // NaN or +inf: the row has no probabilities
  }
  return mx;
}

// ---- lists of the best entries: one descending key a lane, 0 = empty ------------------------------------------------
__device__ __forceinline__ void list_insert(u64& mine, u64 key, int lane) {
  const int pos = __popc(__ballot_sync(kFullMask, mine > key));
  const u64 up = __shfl_up_sync(kFullMask, mine, 1);
  if (lane > pos) mine = up;
  else if (lane == pos) mine = key;
}
// The 32 largest of two descending lists, `other` given back to front.
__device__ __forceinline__ u64 list_merge(u64 mine, u64 other, int lane) {
  u64 x = mine > other ? mine : other;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const u64 y = __shfl_xor_sync(kFullMask, x, o);
    x = ((lane & o) != 0) == (x > y) ? y : x;
  }
  return x;
}
// 32 floats of a warp in descending order.
__device__ __forceinline__ float sort_desc(float x, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
    for (int o = size >> 1; o > 0; o >>= 1) {
      const float y = __shfl_xor_sync(kFullMask, x, o);
      const bool low = ((lane & o) != 0) != ((lane & size) != 0 && size < 32);
      x = low ? fminf(x, y) : fmaxf(x, y);
    }
  }
  return x;
}
__device__ __forceinline__ float sorted_merge(float mine, float other, int lane) {
  float x = fmaxf(mine, other);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float y = __shfl_xor_sync(kFullMask, x, o);
    x = (lane & o) ? fminf(x, y) : fmaxf(x, y);
  }
  return x;
}

struct LogShared {
  float slot[kSlots][kLogThreads];   // largest entry of each slot
  float sorted[kLogWarps][32];
  u64 list[kLogWarps][32];           // [0]: the CTA's
  float red[3][kLogWarps];
  Sums sums;                         // the CTA's, at its largest entry
  float all[2];                      // the row's M, log2 S
  int bad;
};

template <int DT>
__global__ void __launch_bounds__(kLogThreads, 3) logprobs_kernel(const specsteer_token_logprobs_desc p) {
  typedef Logit<DT> L;
  typedef typename L::type T;
  __shared__ LogShared sh;
  cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int n_part = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float nan = __int_as_float(0x7fc00000);
  for (i64 r = blockIdx.x / n_part; r < p.R; r += gridDim.x / n_part) {
    const T* x = (const T*)p.logits + r * p.ld_row;
    const float temp = p.temperature ? p.temperature[r] : 1.f;
    const float c = kLog2e / temp;
    // the first of the given tokens, on their way early
    float given = 0.f;
    int token = -1;
    if (part == 0 && tid < p.n_tokens) {
      token = p.token[r * p.ld_tok + tid];
      if (token >= 0 && token < p.V) given = L::one(x + token);
    }
    // [0, head): entries before the first 16-byte boundary; then whole vectors; the rest behind them
    const int off = (int)(((uintptr_t)x & 15u) / sizeof(T));
    const int head = min(p.V, off ? L::N - off : 0), n_vec = (p.V - head) / L::N, rest = p.V - head - n_vec * L::N;
    const int v0 = (int)((i64)n_vec * part / n_part), v1 = (int)((i64)n_vec * (part + 1) / n_part);
    const uint4* vec = reinterpret_cast<const uint4*>(x + head) + v0;
    const int n = v1 - v0, iters = (n + kVecs * kLogThreads - 1) / (kVecs * kLogThreads);
    const int per_slot = max(1, (iters + kSlots - 1) / kSlots), slots = (iters + per_slot - 1) / per_slot;
    Sums a{kNegInf, 0.f, 0.f};
    const uint4 none = make_uint4(L::kNone, L::kNone, L::kNone, L::kNone);
    auto load = [&](int it, uint4 (&v)[kVecs]) {
#pragma unroll
      for (int u = 0; u < kVecs; ++u) {
        const i64 i = ((i64)it * kVecs + u) * kLogThreads + tid;
        v[u] = i < n ? __ldg(vec + i) : none;
      }
    };
    // entries outside the vectors: the first part's, one a thread
    float single = kNegInf;
    int single_at = 0x7fffffff;
    if (part == 0 && tid < head + rest) {
      single_at = tid < head ? tid : p.V - rest + (tid - head);
      single = L::one(x + single_at);
    }
    float top = kNegInf, slot_top = kNegInf;
    {
      uint4 v[kVecs], next[kVecs];
      load(0, v);
      int left = per_slot, slot = 0;
      for (int it = 0; it < iters; ++it) {
        if (it + 1 < iters) load(it + 1, next);
        slot_top = fmaxf(slot_top, take<DT>(a, v, c));
        if (--left == 0 || it + 1 == iters) {
          sh.slot[slot++][tid] = slot_top;
          top = fmaxf(top, slot_top);
          slot_top = kNegInf;
          left = per_slot;
        }
#pragma unroll
        for (int u = 0; u < kVecs; ++u) v[u] = next[u];
      }
    }
    // the threads' maxima, sorted, before the single entries join them: those are offered to the list in any case
    if (p.n_top > 0) sh.sorted[warp][lane] = sort_desc(top, lane);
    if (single_at != 0x7fffffff) {
      if (single > kNegInf && single < -kNegInf) {
        if (a.ref == kNegInf || (single - a.ref) * c > kSlack) rescale(a, single, c);
        const float t = fmaxf((single - a.ref) * c, -kLeast), e = ex2(t);
        a.s += e;
        a.w = fmaf(e, t, a.w);
        top = fmaxf(top, single);
      } else if (single != kNegInf) {
        a.s = nan;
      }
    }
    // the CTA's largest entry, and the sums there
    const float m = warp_max(top);
    if (lane == 0) sh.red[0][warp] = m;
    __syncthreads();
    float most = sh.red[0][0];
#pragma unroll
    for (int w = 1; w < kLogWarps; ++w) most = fmaxf(most, sh.red[0][w]);
    rescale(a, most == kNegInf ? 0.f : most, c);
    const float ws = warp_sum(a.s), ww = warp_sum(a.w);
    if (lane == 0) { sh.red[1][warp] = ws; sh.red[2][warp] = ww; }
    if (p.n_top > 0) {
      // the n_top-th largest of the threads' maxima
      float best = sh.sorted[0][lane];
#pragma unroll
      for (int w = 1; w < kLogWarps; ++w) best = sorted_merge(best, sh.sorted[w][31 - lane], lane);
      const float tau = __shfl_sync(kFullMask, best, p.n_top - 1);
      // the slots that reach it, of this warp's own threads
      u64 mine = 0, last = 0;
      auto offer = [&](float value, int at, bool there) {
        const u64 key = entry_key(value + 0.f, at);
        uint32_t todo = __ballot_sync(kFullMask, there && key > last);
        while (todo) {
          const int src = __ffs(todo) - 1;
          todo &= todo - 1;
          list_insert(mine, __shfl_sync(kFullMask, key, src), lane);
        }
        last = __shfl_sync(kFullMask, mine, p.n_top - 1);
      };
      if (warp == 0) offer(single, single_at, single_at != 0x7fffffff);
      for (int s = 0; s < slots; ++s) {
        const float value = sh.slot[s][tid];
        const i64 from = (i64)s * per_slot * kVecs * kLogThreads;   // of the slot's vectors; this lane's first is tid behind
        uint32_t todo = __ballot_sync(kFullMask, value >= tau);
        while (todo) {
          const int src = __ffs(todo) - 1;
          todo &= todo - 1;
          const int first_vec = (int)(from + warp * 32 + src);
          const u64 bound = entry_key(__shfl_sync(kFullMask, value, src) + 0.f, head + (v0 + first_vec) * L::N);
          if (bound <= last) continue;
          const int entries = per_slot * kVecs * L::N;
          for (int e0 = 0; e0 < entries; e0 += 32) {
            const int e = e0 + lane;
            const i64 i = first_vec + (i64)(e / L::N) * kLogThreads;
            const bool there = e < entries && i < n;
            const int at = there ? head + (v0 + (int)i) * L::N + e % L::N : 0;
            offer(there ? L::one(x + at) : 0.f, at, there);
          }
        }
      }
      sh.list[warp][lane] = mine;
    }
    __syncthreads();
    if (warp == 0) {
      if (p.n_top > 0) {
        u64 best = sh.list[0][lane];
#pragma unroll
        for (int w = 1; w < kLogWarps; ++w) best = list_merge(best, sh.list[w][31 - lane], lane);
        sh.list[0][lane] = best;
      }
      if (lane == 0) {
        float s = 0.f, w = 0.f;
#pragma unroll
        for (int i = 0; i < kLogWarps; ++i) { s += sh.red[1][i]; w += sh.red[2][i]; }
        sh.sums = Sums{most, s, w};
      }
    }
    if (n_part > 1) cluster.sync();
    else __syncthreads();
    if (part == 0) {
      if (warp == 0) {
        u64 best = p.n_top > 0 ? sh.list[0][lane] : 0;
        if (n_part > 1 && p.n_top > 0)
          for (int i = 1; i < n_part; ++i) best = list_merge(best, cluster.map_shared_rank(&sh.list[0][0], i)[31 - lane], lane);
        // the parts' sums, a lane each
        Sums b{kNegInf, 0.f, 0.f};
        if (lane < n_part) b = *cluster.map_shared_rank(&sh.sums, lane);
        const float M = warp_max(b.ref);
        rescale(b, M, c);
        const float s = warp_sum(b.s), w = warp_sum(b.w), l2s = log2f(s), lse = fmaf(l2s, kLn2, M / temp);
        const bool bad_temp = !(temp > 0.f && temp < -kNegInf);
        const bool bad = bad_temp || !(s > 0.f && s < -kNegInf) || !(fabsf(lse) < -kNegInf);
        if (lane == 0) {
          if (p.lse) p.lse[r] = bad ? nan : lse;
          if (p.entropy) p.entropy[r] = bad ? nan : (l2s - w / s) * kLn2;
          if (bad && p.row_status) atomicOr(p.row_status + r, bad_temp ? SPECSTEER_REQ_BAD_PARAM : SPECSTEER_REQ_NONFINITE);
          sh.all[0] = M;
          sh.all[1] = l2s;
          sh.bad = bad;
        }
        if (lane < p.n_top) {
          p.top_id[r * p.n_top + lane] = bad ? -1 : (int)(0xffffffffu - (uint32_t)best);
          p.top_logprob[r * p.n_top + lane] = bad ? nan : ((order_val((uint32_t)(best >> 32)) - M) * c - l2s) * kLn2;
        }
      }
      __syncthreads();
      const float M = sh.all[0], l2s = sh.all[1];
      for (int i = tid; i < p.n_tokens; i += kLogThreads) {
        if (i != tid) {
          token = p.token[r * p.ld_tok + i];
          if (token >= 0 && token < p.V) given = L::one(x + token);
        }
        const bool outside = token < 0 || token >= p.V;
        if (outside && token != -1 && p.row_status) atomicOr(p.row_status + r, SPECSTEER_REQ_BAD_TOKEN);
        p.logprob[r * p.ld_tok + i] = sh.bad ? nan : outside ? kNegInf : ((given - M) * c - l2s) * kLn2;
      }
    }
    if (n_part > 1) cluster.sync();   // nobody overwrites its part, or leaves, before the first has read it
    else __syncthreads();
  }
}

template <int DT> cudaError_t launch(const specsteer_token_logprobs_desc* d, int split, int grid, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid * split);
  cfg.blockDim = dim3(kLogThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<DT>, *d);
}

}  // namespace
}  // namespace specsteer

using namespace specsteer;

extern "C" specsteer_status specsteer_token_logprobs(const specsteer_token_logprobs_desc* d, void* cuda_stream) {
  if (!d || d->R < 0 || d->V < 1 || d->n_tokens < 0 || d->n_top < 0 || d->n_top > SPECSTEER_TOP_MAX || d->n_top > d->V || d->ld_row < d->V) return SPECSTEER_ERR_INVALID_ARG;
  if (d->dtype != SPECSTEER_F32 && d->dtype != SPECSTEER_BF16 && d->dtype != SPECSTEER_F16) return SPECSTEER_ERR_INVALID_ARG;
  if (d->n_tokens > 0 && d->ld_tok < d->n_tokens) return SPECSTEER_ERR_INVALID_ARG;
  if (d->R == 0) return SPECSTEER_OK;
  if (!d->logits || (d->n_tokens > 0 && (!d->token || !d->logprob)) || (d->n_top > 0 && (!d->top_id || !d->top_logprob))) return SPECSTEER_ERR_INVALID_ARG;
  const int sm = current_sm_count();
  if (sm <= 0) return SPECSTEER_ERR_CUDA;
  // Parts of a row: while the rows do not fill the SMs eight times over and a part keeps a chunk a thread.
  const long long chunks = (long long)d->V * (d->dtype == SPECSTEER_F32 ? 4 : 2) / (16 * kVecs * kLogThreads);
  int split = 1;
  while (split < 8 && (long long)d->R * split < 8ll * sm && chunks >= 2 * split) split *= 2;
  const int grid = d->R < (1 << 20) ? d->R : (1 << 20);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  const cudaError_t e = d->dtype == SPECSTEER_F32 ? launch<SPECSTEER_F32>(d, split, grid, s)
                        : d->dtype == SPECSTEER_BF16 ? launch<SPECSTEER_BF16>(d, split, grid, s) : launch<SPECSTEER_F16>(d, split, grid, s);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return SPECSTEER_ERR_CUDA;
  }
  return SPECSTEER_OK;
}
