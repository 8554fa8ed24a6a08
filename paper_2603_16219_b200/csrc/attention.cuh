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

// The keys of the chunk itself that a row sees, for trees of drafts (specsteer_tree_attention).
struct TreeMask {
  const uint32_t* bits;    // [T][ld]; nullptr: a chain
  long long ld;
  int words;
  const int* positions;    // [T], read with a window only
};

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
// The same for a tree, whose rows must be in the cache and in the mask.
__device__ __forceinline__ AttnRequest attn_request_tree(const specsteer_attention_desc& p, const TreeMask& m, int b) {
  AttnRequest r = attn_request(p, b);
  if (!r.bad && (r.kv < r.n || r.n > 32ll * m.words)) { r.bad = true; r.n = 0; }
  return r;
}
// Where the cached keys before the chunk begin that a row of a tree at position pos sees.
__device__ __forceinline__ int tree_lo(const specsteer_attention_desc& p, int pos) {
  return p.window > 0 && pos >= p.window ? pos - p.window + 1 : 0;
}
// That of row i: a position is at least that of the root and at most the row's own place.
__device__ __forceinline__ int tree_row_lo(const specsteer_attention_desc& p, const TreeMask& m, const AttnRequest& r, int i) {
  if (p.window <= 0) return 0;
  const int past = r.kv - r.n;
  return tree_lo(p, min(max(m.positions[(long long)r.row0 + i], past), past + i));
}
// Bits [at, at + 32) of a row's n bits (at may be negative; what lies outside is 0).
__device__ __forceinline__ uint32_t tree_bits(const TreeMask& m, long long row, int n, int at) {
  if (at <= -32 || at >= n) return 0u;
  const uint32_t* bits = m.bits + row * m.ld;
  const int w = at >> 5;
  const uint32_t low = w >= 0 ? bits[w] : 0u, high = 32 * (w + 1) < n ? bits[w + 1] : 0u;
  const uint32_t got = __funnelshift_r(low, high, at & 31);
  return n - at >= 32 ? got : got & ((1u << (n - at)) - 1u);
}

// The keys [lo, hi) that row i of a request sees (empty when hi <= lo).
__device__ __forceinline__ void attn_span(const specsteer_attention_desc& p, const AttnRequest& r, int i, int& lo, int& hi) {
  hi = r.kv - r.n + i + 1;
  lo = p.window > 0 && hi > p.window ? hi - p.window : 0;
}

// The tensor-core kernel: whether it takes a (checked) descriptor, the workspace it needs, the launch.
bool attention_tc_takes(const specsteer_attention_desc* d);
size_t attention_tc_workspace(const specsteer_attention_desc* d);
cudaError_t launch_attention_tc(const specsteer_attention_desc* d, const TreeMask& tree, cudaStream_t s);

}  // namespace specsteer
