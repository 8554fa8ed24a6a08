// Trees of drafts: the ancestors and positions of their rows, and the path that is kept when a round is over.
//
//   tree_plan_kernel   a block a request: parents into shared memory, then a thread a row climbs to its root.  Ancestors come
//                      in falling order, so the words of a row's mask are written one after the other as the climb leaves
//                      them, and no mask is held in registers.  Bound by latency: launch, parents' trip, the climb.  A tree of 9 rows 1.8 us,
//                      256 trees of 3 to 200 rows 3.3 us.  The climb is a chain of reads of shared memory, one a step: a bushy tree of 1024 rows
//                      23 us, a star of as many 18 us, a chain of 1024, where every row climbs to the front, 441 us.
//   tree_keep_kernel   every block of a request finds the path for itself (a pass over the rows gives each row its confirmed
//                      child, then as many steps as the path is long), and moves its share of the keys and values.  A
//                      thread owns a column, 16 bytes of one head in one layer's keys or values, and moves it along the path:
//                      rows only move towards the front, so what a column's later steps read its earlier ones have not written.
//                      Bound by latency: rows, their parents' choices, table, keys.  A tree of 9 rows in 36 layers 3.9 us, 64 trees
//                      of 15 to 32 rows in 16 layers 5.9 us (11 MB moved).
#include <cuda_runtime.h>

#include "common.cuh"
#include "paged.h"
#include "specsteer.h"

namespace specsteer {
namespace {

typedef long long i64;
constexpr int kMaxRows = SPECSTEER_TREE_MAX_ROWS;
constexpr int kTreeThreads = 256;
constexpr int kMoves = 4;          // rows of a path moved together

// Rows [row0, row0 + n) of request b and the tokens cached before them; false when the offsets or lengths make no sense.
struct TreeRequest { int row0, n, past; };
__device__ __forceinline__ bool tree_request(const int* cu_new, const int* kv_len, int T, int b, TreeRequest* r) {
  r->row0 = cu_new[b];
  const int end = cu_new[b + 1], kv = kv_len[b];
  const bool ok = r->row0 >= 0 && end >= r->row0 && end <= T && kv >= end - r->row0;
  r->n = ok ? end - r->row0 : 0;
  r->past = kv - r->n;
  return ok;
}

__global__ void __launch_bounds__(kTreeThreads) tree_plan_kernel(const specsteer_tree_plan_desc p) {
  __shared__ int parent_s[kMaxRows];
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= p.B) {   // rows behind the last request's
    __shared__ int end_s[kTreeThreads / 32];
    int end = max(0, p.cu_new[p.B]);
    for (int b = tid; b < p.B; b += kTreeThreads) {   // (offsets that go down: behind every request that is accepted)
      TreeRequest rq;
      if (tree_request(p.cu_new, p.kv_len, p.T, b, &rq)) end = max(end, rq.row0 + rq.n);
    }
    end = __reduce_max_sync(kFullMask, end);
    if ((tid & 31) == 0) end_s[tid >> 5] = end;
    __syncthreads();
    for (int w = 0; w < kTreeThreads / 32; ++w) end = max(end, end_s[w]);
    const i64 step = (i64)(gridDim.x - p.B) * kTreeThreads;
    for (i64 t = end + (i64)(blockIdx.x - p.B) * kTreeThreads + tid; t < p.T; t += step) {
      for (int w = 0; w < p.mask_words; ++w) p.mask[t * p.ld_mask + w] = 0u;
      if (p.positions) p.positions[t] = -1;
    }
    return;
  }
  const int b = blockIdx.x;
  TreeRequest rq;
  if (!tree_request(p.cu_new, p.kv_len, p.T, b, &rq)) {
    if (tid == 0 && p.req_status) atomicOr(p.req_status + b, SPECSTEER_REQ_BAD_LEN);
    return;
  }
  const bool fits = rq.n <= kMaxRows && rq.n <= 32 * p.mask_words;
  int bad = 0;
  if (fits) {
    for (int i = tid; i < rq.n; i += kTreeThreads) {
      const int j = p.parent[rq.row0 + i];
      const bool ok = j >= -1 && j < i;
      bad |= !ok;
      parent_s[i] = ok ? j : -1;
    }
  }
  bad = __syncthreads_or(bad);
  if (tid == 0 && p.req_status && (bad || !fits)) atomicOr(p.req_status + b, fits ? SPECSTEER_REQ_BAD_PARENT : SPECSTEER_REQ_BAD_LEN);
  for (int i = tid; i < rq.n; i += kTreeThreads) {
    uint32_t* row = p.mask + (i64)(rq.row0 + i) * p.ld_mask;
    int w = p.mask_words - 1, pos = -1;
    if (fits) {
      int j = i, depth = 0;
      uint32_t bits = 0u;
      do {
        if (p.window == 0 || depth < p.window) {
          for (; w > (j >> 5); --w) { row[w] = bits; bits = 0u; }
          bits |= 1u << (j & 31);
        }
        j = parent_s[j];
        ++depth;
      } while (j >= 0);
      row[w--] = bits;
      pos = rq.past + depth - 1;
    }
    for (; w >= 0; --w) row[w] = 0u;
    if (p.positions) p.positions[rq.row0 + i] = pos;
  }
}

// ---- keep -----------------------------------------------------------------------------------------------------------
template <int BYTES> struct Word;
template <> struct Word<16> { typedef uint4 type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };

// BYTES moved at once: 16, or an element where strides or pointers are not 16-byte multiples.  ES: bytes of an element.
template <int BYTES, int ES>
__global__ void __launch_bounds__(kTreeThreads) tree_keep_kernel(const specsteer_tree_keep_desc p) {
  typedef typename Word<BYTES>::type W;
  __shared__ int next_s[kMaxRows], path_s[kMaxRows];
  __shared__ int4 move_s[kMaxRows];   // page and place a row of the path comes from, page (-1: it stays) and place it goes to
  __shared__ int len_s;
  const int tid = threadIdx.x, b = blockIdx.x;
  const bool first = blockIdx.y == 0;
  TreeRequest rq;
  bool ok = tree_request(p.cu_new, p.kv_len, p.T, b, &rq) && rq.n <= kMaxRows;
  if (p.n_layers > 0 && (i64)rq.past + rq.n > (i64)p.table_width * p.page_size) ok = false;
  if (!ok) rq.n = 0;
  for (int i = tid; i < rq.n; i += kTreeThreads) next_s[i] = 0x7fffffff;
  __syncthreads();
  for (int i = tid; i < rq.n; i += kTreeThreads) {
    const int j = p.parent[rq.row0 + i];
    if (j < 0 || j >= i) continue;
    const int choice = p.choice[rq.row0 + j];
    if (choice >= 0 && p.token[rq.row0 + i] == choice) atomicMin(next_s + j, i);   // the lowest, whoever comes first
  }
  __syncthreads();
  if (tid == 0) {
    int len = 0;
    for (int j = 0; rq.n > 0 && j != 0x7fffffff && len < p.max_out; j = next_s[j]) path_s[len++] = j;
    len_s = len;
  }
  __syncthreads();
  const int len = len_s;
  if (first) {
    for (int i = tid; i < p.max_out; i += kTreeThreads) {
      const int j = i < len ? path_s[i] : -1;
      if (p.path) p.path[(i64)b * p.max_out + i] = j;
      if (p.out_tokens) p.out_tokens[(i64)b * p.max_out + i] = j >= 0 ? p.choice[rq.row0 + j] : -1;
    }
    if (tid == 0) {
      p.n_out[b] = len;
      if (!ok && p.req_status) atomicOr(p.req_status + b, SPECSTEER_REQ_BAD_LEN);
    }
  }
  if (p.n_layers == 0 || len < 2) return;
  for (int i = 1 + tid; i < len; i += kTreeThreads) {
    int4 m = make_int4(0, 0, -1, 0);
    if (path_s[i] != i) {
      const int from = rq.past + path_s[i], to = rq.past + i;
      const int* table = p.block_table + (i64)b * p.ld_table;
      const int pf = table[from / p.page_size], pt = table[to / p.page_size];
      if (pf >= 0 && pf < p.n_pages && pt >= 0 && pt < p.n_pages) m = make_int4(pf, from % p.page_size, pt, to % p.page_size);
      else if (first && p.req_status) atomicOr(p.req_status + b, SPECSTEER_REQ_BAD_PAGE);
    }
    move_s[i] = m;
  }
  __syncthreads();
  const int per_head = p.D * ES / BYTES;
  const i64 columns = (i64)p.n_layers * p.Hkv * per_head;
  for (i64 c = (i64)blockIdx.y * kTreeThreads + tid; c < columns; c += (i64)gridDim.y * kTreeThreads) {
    const int e = (int)(c % per_head) * (BYTES / ES);
    const int h = (int)(c / per_head % p.Hkv), layer = (int)(c / per_head / p.Hkv);
    char* kc = (char*)p.k_cache + (layer * p.kc_layer + h * p.kc_head + e) * ES;
    char* vc = (char*)p.v_cache + (layer * p.vc_layer + h * p.vc_head + e) * ES;
    // kMoves rows' loads together: what a row's place is read for, if at all, is a row before it
    for (int i0 = 1; i0 < len; i0 += kMoves) {
      W k[kMoves], v[kMoves];
#pragma unroll
      for (int j = 0; j < kMoves; ++j) {
        const int4 m = i0 + j < len ? move_s[i0 + j] : make_int4(0, 0, -1, 0);
        if (m.z < 0) continue;
        k[j] = *(const W*)(kc + (m.x * p.kc_page + m.y * p.kc_slot) * ES);
        v[j] = *(const W*)(vc + (m.x * p.vc_page + m.y * p.vc_slot) * ES);
      }
#pragma unroll
      for (int j = 0; j < kMoves; ++j) {
        const int4 m = i0 + j < len ? move_s[i0 + j] : make_int4(0, 0, -1, 0);
        if (m.z < 0) continue;
        *(W*)(kc + (m.z * p.kc_page + m.w * p.kc_slot) * ES) = k[j];
        *(W*)(vc + (m.z * p.vc_page + m.w * p.vc_slot) * ES) = v[j];
      }
    }
  }
}

}  // namespace
}  // namespace specsteer

using namespace specsteer;

extern "C" specsteer_status specsteer_tree_plan(const specsteer_tree_plan_desc* d, void* cuda_stream) {
  if (!d || d->B < 0 || d->T < 0 || d->mask_words < 1 || d->mask_words > SPECSTEER_TREE_MAX_ROWS / 32 || d->ld_mask < d->mask_words || d->window < 0)
    return SPECSTEER_ERR_INVALID_ARG;
  if (!d->cu_new || (d->B > 0 && !d->kv_len) || (d->T > 0 && (!d->parent || !d->mask))) return SPECSTEER_ERR_INVALID_ARG;
  if (d->T == 0 && d->B == 0) return SPECSTEER_OK;
  if (d->B > 0x7fffffff - 4096) return SPECSTEER_ERR_INVALID_ARG;
  const int tail = d->T / kTreeThreads + 1;
  tree_plan_kernel<<<d->B + (tail < 64 ? tail : 64), kTreeThreads, 0, (cudaStream_t)cuda_stream>>>(*d);
  return cudaGetLastError() == cudaSuccess ? SPECSTEER_OK : SPECSTEER_ERR_CUDA;
}

extern "C" specsteer_status specsteer_tree_keep(const specsteer_tree_keep_desc* d, void* cuda_stream) {
  if (!d || d->B < 0 || d->T < 0 || d->max_out < 1 || d->n_layers < 0) return SPECSTEER_ERR_INVALID_ARG;
  if (d->B > 0 && (!d->cu_new || !d->kv_len || !d->n_out)) return SPECSTEER_ERR_INVALID_ARG;
  if (d->B > 0 && d->T > 0 && (!d->parent || !d->token || !d->choice)) return SPECSTEER_ERR_INVALID_ARG;
  int es = 2;
  bool vec = true;
  if (d->n_layers > 0) {
    if (d->Hkv <= 0 || d->D <= 0 || d->page_size <= 0 || d->n_pages <= 0 || d->table_width <= 0 || d->ld_table < d->table_width) return SPECSTEER_ERR_INVALID_ARG;
    if (d->dtype != SPECSTEER_F32 && d->dtype != SPECSTEER_BF16 && d->dtype != SPECSTEER_F16) return SPECSTEER_ERR_INVALID_ARG;
    if ((long long)d->Hkv * d->D > 0x7fffffff) return SPECSTEER_ERR_INVALID_ARG;
    if (d->B > 0 && (!d->block_table || !d->k_cache || !d->v_cache)) return SPECSTEER_ERR_INVALID_ARG;
    es = d->dtype == SPECSTEER_F32 ? 4 : 2;
    const int extent[4] = {d->n_layers, d->n_pages, d->page_size, d->Hkv};
    const long long k[4] = {d->kc_layer, d->kc_page, d->kc_slot, d->kc_head}, v[4] = {d->vc_layer, d->vc_page, d->vc_slot, d->vc_head};
    vec = (long long)d->D * es % 16 == 0 && ((uintptr_t)d->k_cache & 15u) == 0 && ((uintptr_t)d->v_cache & 15u) == 0;
    for (int i = 0; i < 4; ++i) {
      if (k[i] < 0 || v[i] < 0 || (extent[i] > 1 && (!k[i] || !v[i]))) return SPECSTEER_ERR_INVALID_ARG;   // places that share memory
      vec = vec && (extent[i] == 1 || (k[i] * es % 16 == 0 && v[i] * es % 16 == 0));
    }
  }
  if (d->B == 0) return SPECSTEER_OK;
  const long long columns = (long long)d->n_layers * d->Hkv * d->D / (vec ? 16 / es : 1);
  const long long blocks = d->n_layers > 0 ? (columns + kTreeThreads - 1) / kTreeThreads : 1;
  const dim3 grid(d->B, (unsigned)(blocks < 64 ? blocks : 64));
  cudaStream_t s = (cudaStream_t)cuda_stream;
  if (vec && es == 2) tree_keep_kernel<16, 2><<<grid, kTreeThreads, 0, s>>>(*d);
  else if (vec) tree_keep_kernel<16, 4><<<grid, kTreeThreads, 0, s>>>(*d);
  else if (es == 2) tree_keep_kernel<2, 2><<<grid, kTreeThreads, 0, s>>>(*d);
  else tree_keep_kernel<4, 4><<<grid, kTreeThreads, 0, s>>>(*d);
  return cudaGetLastError() == cudaSuccess ? SPECSTEER_OK : SPECSTEER_ERR_CUDA;
}
