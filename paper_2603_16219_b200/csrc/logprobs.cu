// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits.
//
// A block takes a row: a pass for the maximum, one for the sums, and one for each of the likeliest tokens (the largest key
// below the last one found).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "common.cuh"
#include "specsteer.h"

namespace specsteer {
namespace {

typedef long long i64;
constexpr int kLogThreads = 256, kLogWarps = kLogThreads / 32;

__device__ __forceinline__ float load_f32(const float* x) { return *x; }
__device__ __forceinline__ float load_f32(const __nv_bfloat16* x) { return __bfloat162float(*x); }
__device__ __forceinline__ float load_f32(const __half* x) { return __half2float(*x); }

__device__ __forceinline__ float block_sum(float v, float* scratch) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < kLogWarps; ++w) v += scratch[w];
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kLogThreads) logprobs_kernel(const specsteer_token_logprobs_desc p) {
  __shared__ float scratch[kLogWarps];
  __shared__ u64 keys[kLogWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float nan = __int_as_float(0x7fc00000);
  for (i64 r = blockIdx.x; r < p.R; r += gridDim.x) {
    const T* x = (const T*)p.logits + r * p.ld_row;
    const float temp = p.temperature ? p.temperature[r] : 1.f;
    const float c = kLog2e / temp;
    float m = kNegInf;
    for (int j = tid; j < p.V; j += kLogThreads) m = fmaxf(m, load_f32(x + j));
    __syncthreads();
    m = warp_max(m);
    if (lane == 0) scratch[warp] = m;
    __syncthreads();
    for (int w = 0; w < kLogWarps; ++w) m = fmaxf(m, scratch[w]);
    const float ref = m * c;   // weights are 2^(c x - ref)
    float s = 0.f, w = 0.f;
    for (int j = tid; j < p.V; j += kLogThreads) {
      const float a = fmaf(load_f32(x + j), c, -ref), e = exp2f(a);
      s += e;
      if (e != 0.f) w = fmaf(e, a, w);
    }
    s = block_sum(s, scratch);
    w = block_sum(w, scratch);
    const bool bad_temp = !(temp > 0.f) || isinf(temp);
    const bool bad = bad_temp || !(s > 0.f) || isinf(s) || !isfinite(ref);
    const float l2s = log2f(s);
    if (tid == 0) {
      if (p.lse) p.lse[r] = bad ? nan : (ref + l2s) * kLn2;
      if (p.entropy) p.entropy[r] = bad ? nan : (l2s - w / s) * kLn2;
      if (bad && p.row_status) atomicOr(p.row_status + r, bad_temp ? SPECSTEER_REQ_BAD_PARAM : SPECSTEER_REQ_NONFINITE);
    }
    for (int i = tid; i < p.n_tokens; i += kLogThreads) {
      const int t = p.token[r * p.ld_tok + i];
      const bool outside = t < 0 || t >= p.V;
      if (outside && t != -1 && p.row_status) atomicOr(p.row_status + r, SPECSTEER_REQ_BAD_TOKEN);
      p.logprob[r * p.ld_tok + i] = bad ? nan : outside ? kNegInf : (fmaf(load_f32(x + t), c, -ref) - l2s) * kLn2;
    }
    u64 last = ~0ull;
    for (int k = 0; k < p.n_top; ++k) {
      u64 best = 0;
      for (int j = tid; j < p.V; j += kLogThreads) {
        const u64 key = entry_key(load_f32(x + j) + 0.f, j);
        if (key < last && key > best) best = key;
      }
      for (int o = 16; o > 0; o >>= 1) {
        const u64 y = __shfl_xor_sync(kFullMask, best, o);
        best = y > best ? y : best;
      }
      __syncthreads();
      if (lane == 0) keys[warp] = best;
      __syncthreads();
      for (int i = 0; i < kLogWarps; ++i) best = keys[i] > best ? keys[i] : best;
      last = best;
      if (tid == 0) {
        p.top_id[r * p.n_top + k] = bad ? -1 : (int)(0xffffffffu - (uint32_t)best);
        p.top_logprob[r * p.n_top + k] = bad ? nan : (fmaf(order_val((uint32_t)(best >> 32)), c, -ref) - l2s) * kLn2;
      }
    }
  }
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
  cudaStream_t s = (cudaStream_t)cuda_stream;
  const int grid = d->R < (1 << 20) ? d->R : (1 << 20);
  if (d->dtype == SPECSTEER_F32) logprobs_kernel<float><<<grid, kLogThreads, 0, s>>>(*d);
  else if (d->dtype == SPECSTEER_BF16) logprobs_kernel<__nv_bfloat16><<<grid, kLogThreads, 0, s>>>(*d);
  else logprobs_kernel<__half><<<grid, kLogThreads, 0, s>>>(*d);
  return cudaGetLastError() == cudaSuccess ? SPECSTEER_OK : SPECSTEER_ERR_CUDA;
}
