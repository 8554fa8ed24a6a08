// What the two kernels of the chunk attention share: the request's geometry and its checks.
#pragma once
#include "common.cuh"
#include "internal.h"
#include "paged.h"
#include "specsteer.h"

namespace specsteer {

// The most that the index arithmetic takes of keys, requests, and (the tensor-core kernel) rows: a step past the end must not
// overflow 32 bits.
constexpr int kAttnMaxKv = 0x7fffffff - 4096;

struct AttnRequest {
  int row0, n, kv;   // first row of q, rows, keys in the cache; n = 0 when the request is refused
  bool bad;
};
__device__ __forceinline__ AttnRequest attn_request(const specsteer_attention_desc& p, int b) {
  AttnRequest r;
  r.row0 = p.cu_new[b];
  const int end = p.cu_new[b + 1];
  r.kv = p.kv_len[b];
  r.bad = r.row0 < 0 || end < r.row0 || end > p.T || r.kv < 0 || r.kv > kAttnMaxKv ||
          r.kv > (long long)p.table_width * p.page_size;
  r.n = r.bad ? 0 : end - r.row0;
  return r;
}

// The keys [lo, hi) that row i of a request sees (empty when hi <= lo).
__device__ __forceinline__ void attn_span(const specsteer_attention_desc& p, const AttnRequest& r, int i, int& lo, int& hi) {
  hi = r.kv - r.n + i + 1;
  lo = p.window > 0 && hi > p.window ? hi - p.window : 0;
}

// The tensor-core kernel: whether it takes a (checked) descriptor, the workspace it needs, the launch.
bool attention_tc_takes(const specsteer_attention_desc* d);
size_t attention_tc_workspace(const specsteer_attention_desc* d);
cudaError_t launch_attention_tc(const specsteer_attention_desc* d, cudaStream_t s);

}  // namespace specsteer
