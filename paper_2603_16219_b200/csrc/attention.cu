// Attention of a chunk of new tokens over the paged cache: the host side, and the generic kernel that takes every shape.
//
// The generic kernel computes the definition in float32 on the CUDA cores, one block per 16 rows (a row is a token and
// a query head of one kv head) with the running maximum and sum of a softmax over tiles of 32 keys.  When that gives few
// blocks, a cluster of 8 shares each: its CTAs take the key tiles in turn and put their sums together through
// distributed shared memory.  Measured on shapes the tensor-core kernel takes: five rows of one request 39 us (15 there), 64
// single tokens 0.99 ms (0.08), four prompt chunks 23 ms (0.31).  It is bound by the shared-memory reads of its two inner
// loops (five for four products of a score, one for two of a result), which only a tile per warp would change; it is
// there for the shapes that the tensor-core kernel leaves, not for speed.
#include <cooperative_groups.h>

#include <cmath>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attention.cuh"

namespace specsteer {
namespace {

constexpr int kGenRows = 16, kGenKeys = 32, kGenThreads = 128, kGenWarps = kGenThreads / 32, kGenSplit = 8, kGenCtas = 4;
constexpr int kGenMaxD = SPECSTEER_ATTENTION_MAX_D;

__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f32(float x, __nv_bfloat16* y) { *y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_f32(float x, __half* y) { *y = __float2half_rn(x); }

// Blocks of kGenRows rows are numbered request by request; a block finds its request from the lengths (device data).
// Four CTAs an SM, which the host's rule for splitting blocks counts on: without the bound the trees' form takes 139 registers, three
// CTAs, and 64 trees of 15 to 32 rows over 130 to 4000 keys, 16/4 heads of 256, 6.05 ms instead of 4.62 (chains of the same lengths 4.63, 4.56).
template <typename T, bool TREE>
__global__ void __launch_bounds__(kGenThreads, kGenCtas) attention_generic_kernel(const specsteer_attention_desc p, const TreeMask tree) {
  __shared__ float qs[kGenRows][kGenMaxD];   // the queries; at the end of a split block its sums
  __shared__ T ks[kGenKeys][kGenMaxD + 2];   // an odd number of words a row: 8 keys in 8 banks
  __shared__ float ps[kGenRows][kGenKeys];
  __shared__ float alpha_s[kGenRows], l_s[kGenRows], m_s[kGenRows];
  __shared__ int page_s[kGenKeys];
  __shared__ long long sum_s[kGenThreads / 32];
  __shared__ int found_b, bad_page;
  __shared__ long long found_at;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int n_split = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int G = p.Hq / p.Hkv, hk = blockIdx.y, D = p.D;
  const T* q = (const T*)p.q;
  const T* kc = (const T*)p.k_cache;
  const T* vc = (const T*)p.v_cache;
  // A weight is 2^(post (s pre - m)): with a large scale the difference comes first, so that a score times the scale may pass
  // float32's range; with a small one the product, so that the difference of two scores may.  natural: of a maximum.
  const float c = p.scale * kLog2e, pre = c < 1.f ? c : 1.f, post = c < 1.f ? 1.f : c, natural = c < 1.f ? kLn2 : p.scale;

  auto request = [&](int b) { return TREE ? attn_request_tree(p, tree, b) : attn_request(p, b); };
  if (blockIdx.x == 0 && hk == 0 && p.req_status)
    for (int b = tid; b < p.B; b += kGenThreads)
      if (request(b).bad) atomicOr(p.req_status + b, SPECSTEER_REQ_BAD_LEN);

  // blk runs over this block's share of all blocks; `before` = blocks of the requests ahead of request `b0`
  long long before = 0;
  int b0 = 0;
  for (long long blk = blockIdx.x / n_split;; blk += gridDim.x / n_split) {
    // find the request of block blk: running sums over kGenThreads requests at a time
    if (tid == 0) found_b = -1;
    __syncthreads();
    while (b0 < p.B) {
      const int b = b0 + tid;
      long long mine = 0;
      if (b < p.B) mine = ((long long)request(b).n * G + kGenRows - 1) / kGenRows;
      long long x = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(kFullMask, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) sum_s[warp] = x;
      __syncthreads();
      long long total = 0;
      for (int w = 0; w < kGenThreads / 32; ++w) {
        if (w < warp) x += sum_s[w];
        total += sum_s[w];
      }
      const long long begin = before + x - mine;
      if (mine > 0 && blk >= begin && blk < begin + mine) { found_b = b; found_at = begin; }
      __syncthreads();
      if (found_b >= 0) break;
      before += total;
      b0 += kGenThreads;
    }
    if (found_b < 0) return;
    const int b = found_b;
    const AttnRequest rq = request(b);
    const int past = rq.kv - rq.n;                         // keys before the chunk
    const long long r0 = (blk - found_at) * kGenRows;      // first row of the block within the request and kv head
    const long long n_rows = (long long)rq.n * G;
    if (tid == 0) bad_page = 0;
    for (int e = tid; e < kGenRows * D; e += kGenThreads) {
      const int r = e / D, d = e - r * D;
      const long long rr = r0 + r;
      float x = 0.f;
      if (rr < n_rows) x = to_f32(q[(rq.row0 + rr / G) * p.q_tok + (hk * G + rr % G) * p.q_head + d]);
      qs[r][d] = x;
    }
    // 8 threads a row: this thread's row and its 4 keys of a tile
    const int row = tid >> 3, sub = tid & 7;
    const long long my_row = r0 + row;
    int lo = 0, hi = 0;
    if (my_row < n_rows) {
      attn_span(p, rq, (int)(my_row / G), lo, hi);
      if (TREE) { lo = tree_row_lo(p, tree, rq, (int)(my_row / G)); hi = rq.kv; }
    }
    const int last_row = (int)((r0 + kGenRows < n_rows ? r0 + kGenRows : n_rows) - 1 - r0);
    int blo, bhi, tmp;
    attn_span(p, rq, (int)(r0 / G), blo, tmp);
    attn_span(p, rq, (int)((r0 + last_row) / G), tmp, bhi);
    if (TREE) { blo = tree_lo(p, past); bhi = rq.kv; }
    float m = kNegInf, l = 0.f;
    float acc[kGenRows][2];
#pragma unroll
    for (int r = 0; r < kGenRows; ++r) acc[r][0] = acc[r][1] = 0.f;

    for (int k0 = blo + part * kGenKeys; k0 < bhi; k0 += n_split * kGenKeys) {
      __syncthreads();
      if (tid < kGenKeys) {
        const int j = k0 + tid;
        int page = -1;
        if (j < bhi) {
          page = p.block_table[(long long)b * p.ld_table + j / p.page_size];
          if (page < 0 || page >= p.n_pages) { page = -1; bad_page = 1; }
        }
        page_s[tid] = page;
      }
      __syncthreads();
      // a warp takes every fourth key: 16 loads a thread on their way together
      for (int d0 = lane; d0 < D; d0 += 64) {
        T x[kGenKeys / kGenWarps][2];
#pragma unroll
        for (int i = 0; i < kGenKeys / kGenWarps; ++i) {
          const int j = warp + i * kGenWarps;
          const T* k = kc + page_s[j] * p.kc_page + ((k0 + j) % p.page_size) * p.kc_slot + hk * p.kc_head;
          x[i][0] = x[i][1] = T(0.f);
          if (page_s[j] >= 0) x[i][0] = k[d0];
          if (page_s[j] >= 0 && d0 + 32 < D) x[i][1] = k[d0 + 32];
        }
#pragma unroll
        for (int i = 0; i < kGenKeys / kGenWarps; ++i) {
          ks[warp + i * kGenWarps][d0] = x[i][0];
          if (d0 + 32 < D) ks[warp + i * kGenWarps][d0 + 32] = x[i][1];
        }
      }
      __syncthreads();
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      for (int d = 0; d < D; ++d) {
        const float x = qs[row][d];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = fmaf(x, to_f32(ks[sub + 8 * i][d]), s[i]);
      }
      bool seen[4];
      float mt = kNegInf;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = k0 + sub + 8 * i;
        seen[i] = j >= lo && j < hi && page_s[sub + 8 * i] >= 0;
        if (TREE && j >= past) seen[i] = j < hi && page_s[sub + 8 * i] >= 0 && (tree_bits(tree, rq.row0 + my_row / G, rq.n, j - past) & 1u);
        s[i] *= pre;
        if (seen[i]) mt = s[i] > mt || s[i] != s[i] ? s[i] : mt;   // a NaN stays
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) {
        const float y = __shfl_xor_sync(kFullMask, mt, o);
        mt = y > mt || y != y ? y : mt;
      }
      const float m_new = mt > m || mt != mt ? mt : m;
      const float ref = m_new == kNegInf ? 0.f : m_new;
      const float alpha = m == kNegInf ? 0.f : exp2f((m - ref) * post);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = exp2f((s[i] - ref) * post);
        if (seen[i]) sum += w;
        ps[row][sub + 8 * i] = seen[i] ? w : -1.f;   // -1: not seen, its v is not touched (a NaN there stays away)
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(kFullMask, sum, o);
      l = l * alpha + sum;
      m = m_new;
      if (sub == 0) alpha_s[row] = alpha;
      __syncthreads();
#pragma unroll
      for (int r = 0; r < kGenRows; ++r) {
        const float a = alpha_s[r];
        acc[r][0] *= a;
        acc[r][1] *= a;
      }
      for (int j0 = 0; j0 < kGenKeys; j0 += 8) {
        float v0[8], v1[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = j0 + i;
          const T* v = vc + page_s[j] * p.vc_page + ((k0 + j) % p.page_size) * p.vc_slot + hk * p.vc_head;
          v0[i] = v1[i] = 0.f;
          if (page_s[j] >= 0 && tid < D) v0[i] = to_f32(v[tid]);
          if (page_s[j] >= 0 && tid + kGenThreads < D) v1[i] = to_f32(v[tid + kGenThreads]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
          for (int r = 0; r < kGenRows; ++r) {
            const float w = ps[r][j0 + i];
            if (!(w < 0.f)) {
              acc[r][0] = fmaf(w, v0[i], acc[r][0]);
              acc[r][1] = fmaf(w, v1[i], acc[r][1]);
            }
          }
        }
      }
    }
    if (sub == 0) { l_s[row] = l; m_s[row] = m; }
    __syncthreads();
    if (tid == 0 && bad_page && p.req_status) atomicOr(p.req_status + b, SPECSTEER_REQ_BAD_PAGE);
    auto finish = [&](int r, float top, float sum, float a0, float a1) {
      const long long rr = r0 + r;
      if (rr >= n_rows) return;
      T* o = (T*)p.out + (rq.row0 + rr / G) * p.o_tok + (hk * G + rr % G) * p.o_head;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      if (tid < D) from_f32(a0 * inv, o + tid);
      if (tid + kGenThreads < D) from_f32(a1 * inv, o + tid + kGenThreads);
      if (tid == 0 && p.lse) p.lse[(rq.row0 + rr / G) * p.Hq + hk * G + rr % G] = top == kNegInf ? kNegInf : fmaf(top, natural, log2f(sum) * kLn2);
    };
    if (n_split == 1) {
#pragma unroll
      for (int r = 0; r < kGenRows; ++r) finish(r, m_s[r], l_s[r], acc[r][0], acc[r][1]);
    } else {
#pragma unroll
      for (int r = 0; r < kGenRows; ++r) {
        if (tid < D) qs[r][tid] = acc[r][0];
        if (tid + kGenThreads < D) qs[r][tid + kGenThreads] = acc[r][1];
      }
      cluster.sync();
      for (int r = part; r < kGenRows; r += n_split) {   // in the order of the parts, whoever came first
        float top = kNegInf, sum = 0.f, a0 = 0.f, a1 = 0.f;
        for (int i = 0; i < n_split; ++i) {
          const float y = *cluster.map_shared_rank(&m_s[r], i);
          top = y > top || y != y ? y : top;
        }
        for (int i = 0; i < n_split; ++i) {
          const float y = *cluster.map_shared_rank(&m_s[r], i), f = y == kNegInf ? 0.f : exp2f((y - top) * post);
          sum = fmaf(*cluster.map_shared_rank(&l_s[r], i), f, sum);
          if (tid < D) a0 = fmaf(*cluster.map_shared_rank(&qs[r][tid], i), f, a0);
          if (tid + kGenThreads < D) a1 = fmaf(*cluster.map_shared_rank(&qs[r][tid + kGenThreads], i), f, a1);
        }
        finish(r, top, sum, a0, a1);
      }
      cluster.sync();   // nobody overwrites its sums, or leaves, before the others have read them
    }
    __syncthreads();
  }
}

specsteer_status check_attention(const specsteer_attention_desc* d) {
  if (!d || d->B < 0 || d->T < 0 || d->Hq <= 0 || d->Hkv <= 0 || d->Hq % d->Hkv || d->D <= 0 || d->page_size <= 0 || d->n_pages <= 0 ||
      d->table_width <= 0 || d->ld_table < d->table_width || d->window < 0)
    return SPECSTEER_ERR_INVALID_ARG;
  if (d->dtype != SPECSTEER_BF16 && d->dtype != SPECSTEER_F16) return SPECSTEER_ERR_INVALID_ARG;
  if (!(d->scale >= 0.f) || !std::isfinite(d->scale * kLog2e) || (d->flags & 0xffffu & ~(uint32_t)SPECSTEER_ATTENTION_GENERIC)) return SPECSTEER_ERR_INVALID_ARG;
  if (d->D > SPECSTEER_ATTENTION_MAX_D || d->Hkv > 65535 || d->B > kAttnMaxKv) return SPECSTEER_ERR_UNSUPPORTED;
  const long long strides[] = {d->q_tok, d->q_head, d->o_tok, d->o_head, d->kc_page, d->kc_slot, d->kc_head, d->vc_page, d->vc_slot, d->vc_head};
  for (long long x : strides)
    if (x < 0) return SPECSTEER_ERR_INVALID_ARG;
  if ((d->T > 1 && !d->o_tok) || (d->Hq > 1 && !d->o_head)) return SPECSTEER_ERR_INVALID_ARG;   // rows that overwrite one another
  if (d->B > 0 && d->T > 0 && (!d->q || !d->k_cache || !d->v_cache || !d->block_table || !d->cu_new || !d->kv_len || !d->out))
    return SPECSTEER_ERR_INVALID_ARG;
  return SPECSTEER_OK;
}

}  // namespace
}  // namespace specsteer

using namespace specsteer;

namespace {

specsteer_status run_attention(const specsteer_attention_desc* d, const TreeMask& tree, cudaStream_t s) {
  if (d->B == 0 || d->T == 0) return SPECSTEER_OK;
  const size_t need = specsteer_chunk_attention_workspace(d);
  if (need > 0 && (!d->workspace || d->workspace_bytes < (long long)need || ((uintptr_t)d->workspace & 31u))) return SPECSTEER_ERR_WORKSPACE;
  if (attention_tc_takes(d)) {
    if (launch_attention_tc(d, tree, s) != cudaSuccess) {
      cudaGetLastError();
      return SPECSTEER_ERR_CUDA;
    }
    return SPECSTEER_OK;
  }
  const long long blocks = ((long long)d->T * (d->Hq / d->Hkv) + kGenRows - 1) / kGenRows + d->B;
  const int sm = current_sm_count();
  if (sm <= 0) return SPECSTEER_ERR_CUDA;
  // A cluster of 8 a block while the blocks do not fill the SMs (kGenCtas each) four times over: 5 rows over 720 keys of
  // width 256 take 51 us (one CTA a block: 250 us), a batch of 64 single tokens of width 256 1.6 ms (2.4 ms).
  const int split = blocks * d->Hkv <= (long long)sm * kGenCtas * 4 ? kGenSplit : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)) * split, d->Hkv);
  cfg.blockDim = dim3(kGenThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const bool bf16 = d->dtype == SPECSTEER_BF16;
  const cudaError_t e = tree.bits ? (bf16 ? cudaLaunchKernelEx(&cfg, attention_generic_kernel<__nv_bfloat16, true>, *d, tree)
                                          : cudaLaunchKernelEx(&cfg, attention_generic_kernel<__half, true>, *d, tree))
                                  : (bf16 ? cudaLaunchKernelEx(&cfg, attention_generic_kernel<__nv_bfloat16, false>, *d, tree)
                                          : cudaLaunchKernelEx(&cfg, attention_generic_kernel<__half, false>, *d, tree));
  if (e != cudaSuccess) {
    cudaGetLastError();
    return SPECSTEER_ERR_CUDA;
  }
  return SPECSTEER_OK;
}

}  // namespace

extern "C" size_t specsteer_chunk_attention_workspace(const specsteer_attention_desc* d) {
  if (check_attention(d) != SPECSTEER_OK || d->B == 0 || d->T == 0) return 0;
  return attention_tc_takes(d) ? attention_tc_workspace(d) : 0;
}

extern "C" specsteer_status specsteer_chunk_attention(const specsteer_attention_desc* d, void* cuda_stream) {
  const specsteer_status st = check_attention(d);
  return st != SPECSTEER_OK ? st : run_attention(d, TreeMask{}, (cudaStream_t)cuda_stream);
}

extern "C" specsteer_status specsteer_tree_attention(const specsteer_tree_attention_desc* d, void* cuda_stream) {
  const specsteer_status st = d ? check_attention(&d->a) : SPECSTEER_ERR_INVALID_ARG;
  if (st != SPECSTEER_OK) return st;
  if (d->mask_words < 1 || d->ld_mask < d->mask_words) return SPECSTEER_ERR_INVALID_ARG;
  if (d->a.B > 0 && d->a.T > 0 && (!d->mask || (d->a.window > 0 && !d->positions))) return SPECSTEER_ERR_INVALID_ARG;
  return run_attention(&d->a, TreeMask{d->mask, d->ld_mask, d->mask_words, d->positions}, (cudaStream_t)cuda_stream);
}
