// Bookkeeping of the paged key/value cache: block tables and slot maps from request lengths, and the chunk's keys and
// values into their slots.
//
//   cache_plan_kernel    one thread-block cluster; every CTA forms the same running sums over the requests (tokens,
//                        pages taken, pages given back) in its own shared memory, then the cluster shares the page
//                        moves and the rows of the slot map.  Two cluster barriers order the three steps that touch the
//                        same memory: pages given back -> pages taken -> slots.
//   cache_append_kernel  a copy by slot, 16 bytes a thread where alignment allows.
#include <atomic>

#include "common.cuh"
#include "internal.h"
#include "specsteer.h"

namespace specsteer {
namespace {

constexpr int kPlanThreads = 1024;
// CTAs per cluster when there is much to write.  The sums are latency and are repeated by every CTA; the rows of the
// slot map (16 bytes a token) and the page moves are shared.
constexpr int kPlanCluster = 8;

typedef long long i64;

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}

// Exclusive sum of v over the threads of the block in thread order; *total receives the sum.  Ends with a barrier, so
// the scratch may be used again at once.
__device__ __forceinline__ i64 block_exclusive_sum(i64 v, i64* scratch, i64* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  i64 x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const i64 y = __shfl_up_sync(kFullMask, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) scratch[warp] = x;
  __syncthreads();
  if (warp == 0) {
    i64 w = lane < nw ? scratch[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const i64 y = __shfl_up_sync(kFullMask, w, o);
      if (lane >= o) w += y;
    }
    scratch[lane] = w;
  }
  __syncthreads();
  const i64 before = warp ? scratch[warp - 1] : 0;
  *total = scratch[31];
  __syncthreads();
  return before + x - v;
}

// The request that element i of a flattened list belongs to: the last b < B with cum[b] <= i (cum ascending, cum[0] = 0).
__device__ __forceinline__ int owner_of(const int* cum, int B, int i) {
  int lo = 0, hi = B;   // cum[lo] <= i < cum[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cum[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

// IPT: requests a thread, consecutive ones.
template <int IPT>
__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(const specsteer_cache_plan_desc p) {
  extern __shared__ int plan_smem[];
  __shared__ i64 scratch[32];
  const int B = p.B, tid = threadIdx.x;
  int* cum_tok = plan_smem;                // [B+1]
  int* cum_give = cum_tok + (B + 1);       // [B+1]
  int* cum_take = cum_give + (B + 1);      // [B+1]
  const uint32_t rank = cluster_rank(), n_cta = cluster_size();
  const int first_thread = (int)rank * blockDim.x + tid, n_threads = (int)n_cta * blockDim.x;

  const i64 head = p.ring_pos[0], tail = p.ring_pos[1], P = p.n_pages;
  const bool pool_ok = head >= 0 && tail >= head && tail - head <= P;
  const i64 capacity = (i64)p.table_width * p.page_size;

  int seq[IPT], asked[IPT], held[IPT], status[IPT];
  i64 kept[IPT];
  i64 sum = 0;
#pragma unroll
  for (int k = 0; k < IPT; ++k) {
    const int b = tid * IPT + k;
    seq[k] = asked[k] = held[k] = status[k] = 0;
    kept[k] = 0;
    if (b < B) {
      seq[k] = p.seq_len[b];
      held[k] = p.pages_held[b];
      const int n = p.new_len[b];
      kept[k] = n == -1 ? 0 : (i64)seq[k] + (p.advance ? p.advance[b] : 0);
      asked[k] = n > 0 ? n : 0;
      if (n < -1 || kept[k] < 0 || kept[k] + asked[k] > capacity || held[k] < 0 || held[k] > p.table_width || kept[k] + asked[k] > 0x7fffffff)
        status[k] = SPECSTEER_REQ_BAD_LEN;
      if (!pool_ok) status[k] |= SPECSTEER_REQ_BAD_POOL;
      if (status[k]) asked[k] = 0;
      sum += asked[k];
    }
  }
  i64 total;
  i64 run = block_exclusive_sum(sum, scratch, &total);
  // tokens beyond max_tokens are refused; then the pages each request gives back or wants
  i64 give_sum = 0, take_sum = 0;
  int target[IPT];
#pragma unroll
  for (int k = 0; k < IPT; ++k) {
    run += asked[k];
    if (asked[k] > 0 && run > p.max_tokens) { status[k] |= SPECSTEER_REQ_NO_ROOM; asked[k] = 0; }
    const bool passed_on = status[k] & (SPECSTEER_REQ_BAD_LEN | SPECSTEER_REQ_BAD_POOL);
    target[k] = passed_on ? held[k] : (int)((kept[k] + asked[k] + p.page_size - 1) / p.page_size);
    const int d = target[k] - held[k];
    if (d > 0) take_sum += d; else give_sum -= d;
  }
  i64 give_total, take_total, tok_total;
  i64 give_run = block_exclusive_sum(give_sum, scratch, &give_total);
  i64 take_run = block_exclusive_sum(take_sum, scratch, &take_total);
  const i64 room = pool_ok ? P - (tail - head) : 0;
  const int given = (int)(give_total < room ? give_total : room);   // more would mean that a page was handed out twice
  const i64 avail = pool_ok ? tail - head + given : 0;
  i64 tok_sum = 0, served_sum = 0;
#pragma unroll
  for (int k = 0; k < IPT; ++k) {
    const int b = tid * IPT + k;
    const int d = target[k] - held[k];
    if (b < B) {
      cum_give[b] = (int)(give_run < 0x7fffffff ? give_run : 0x7fffffff);
      cum_take[b] = (int)(take_run < avail ? take_run : avail);
    }
    if (d < 0) give_run -= d;
    if (d > 0) {
      take_run += d;
      // sums only grow: once a request is refused, every later one that wants pages is too, so the takers that are
      // served are a prefix and their running sum above is right
      if (take_run > avail) { status[k] |= SPECSTEER_REQ_NO_PAGES; asked[k] = 0; target[k] = held[k]; }
      else served_sum += d;
    }
    tok_sum += asked[k];
  }
  i64 tok_run = block_exclusive_sum(tok_sum, scratch, &tok_total);
  i64 served_total;
  (void)block_exclusive_sum(served_sum, scratch, &served_total);
#pragma unroll
  for (int k = 0; k < IPT; ++k) {
    const int b = tid * IPT + k;
    if (b < B) cum_tok[b] = (int)tok_run;
    tok_run += asked[k];
  }
  if (tid == 0) {
    cum_tok[B] = (int)tok_total;
    cum_give[B] = (int)(give_total < 0x7fffffff ? give_total : 0x7fffffff);
    cum_take[B] = (int)served_total;
  }
  __syncthreads();

  // pages given back: entry target + r' of the request's table to place tail + r of the ring.  The inputs held the old
  // pages_held; the first entry of a giver is its target, recovered from the lengths.
  for (int r = first_thread; r < given; r += n_threads) {
    const int b = owner_of(cum_give, B, r);
    const int n = p.new_len[b];
    const i64 kept_b = n == -1 ? 0 : (i64)p.seq_len[b] + (p.advance ? p.advance[b] : 0);
    const i64 len = kept_b + (cum_tok[b + 1] - cum_tok[b]);
    const int first = (int)((len + p.page_size - 1) / p.page_size);
    p.free_ring[(tail + r) % P] = p.block_table[(i64)b * p.ld_table + first + (r - cum_give[b])];
  }
  cluster_sync_all();   // the ring is whole, and no CTA reads pages_held, seq_len or ring_pos for the sums any more
  for (int r = first_thread; r < (int)served_total; r += n_threads) {
    const int b = owner_of(cum_take, B, r);
    const int have = p.pages_held[b];
    p.block_table[(i64)b * p.ld_table + have + (r - cum_take[b])] = __ldcg(p.free_ring + (head + r) % P);
  }
  if (rank == 0) {
#pragma unroll
    for (int k = 0; k < IPT; ++k)
      if (tid * IPT + k < B) p.req_status[tid * IPT + k] = status[k];
  }
  cluster_sync_all();   // the tables are whole; the status words are there for the slots to add to
  const int n_tok = (int)tok_total;
  for (int i = first_thread; i < p.max_tokens; i += n_threads) {
    i64 slot = -1;
    int pos = -1, b = -1;
    if (i < n_tok) {
      b = owner_of(cum_tok, B, i);
      pos = (int)((i64)p.seq_len[b] + (p.advance ? p.advance[b] : 0)) + (i - cum_tok[b]);
      const int page = __ldcg(p.block_table + (i64)b * p.ld_table + pos / p.page_size);
      if (page >= 0 && page < p.n_pages) slot = (i64)page * p.page_size + pos % p.page_size;
      else atomicOr(p.req_status + b, SPECSTEER_REQ_BAD_PAGE);
    }
    p.slot_map[i] = slot;
    if (p.positions) p.positions[i] = pos;
    if (p.token_req) p.token_req[i] = b;
  }
  cluster_sync_all();   // nobody reads an input any more: the in-place outputs may be written
  if (rank == 0) {
#pragma unroll
    for (int k = 0; k < IPT; ++k) {
      const int b = tid * IPT + k;
      if (b < B) {
        const bool passed_on = status[k] & (SPECSTEER_REQ_BAD_LEN | SPECSTEER_REQ_BAD_POOL);
        p.seq_len_out[b] = passed_on ? seq[k] : (int)kept[k];
        p.pages_held_out[b] = target[k];
        p.kv_len[b] = passed_on ? 0 : (int)(kept[k] + asked[k]);
        p.cu_new[b] = cum_tok[b];
      }
    }
    if (tid == 0) {
      p.cu_new[B] = n_tok;
      p.ring_pos_out[0] = head + served_total;
      p.ring_pos_out[1] = tail + given;
    }
  }
}

// ---- append -----------------------------------------------------------------------------------------------------
// VEC: elements a thread moves at once (16 bytes), or 1 where strides or pointers are not 16-byte multiples.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) cache_append_kernel(const specsteer_cache_append_desc p) {
  const int per_head = p.D / VEC, per_tok = per_head * p.Hkv;
  const i64 n = (i64)p.T * per_tok;
  const i64 slots = (i64)p.n_pages * p.page_size;
  for (i64 i = (i64)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (i64)gridDim.x * blockDim.x) {
    const int t = (int)(i / per_tok), r = (int)(i - (i64)t * per_tok);
    const int h = r / per_head, d = (r - h * per_head) * VEC;
    const i64 slot = p.slot_map[t];
    if (slot < 0 || slot >= slots) continue;
    const i64 page = slot / p.page_size, off = slot - page * p.page_size;
    const T* ks = (const T*)p.k + t * p.k_tok + h * p.k_head + d;
    const T* vs = (const T*)p.v + t * p.v_tok + h * p.v_head + d;
    T* kd = (T*)p.k_cache + page * p.kc_page + off * p.kc_slot + h * p.kc_head + d;
    T* vd = (T*)p.v_cache + page * p.vc_page + off * p.vc_slot + h * p.vc_head + d;
    if (VEC == 1) {
      *kd = *ks;
      *vd = *vs;
    } else {
      const uint4 a = __ldg(reinterpret_cast<const uint4*>(ks)), c = __ldg(reinterpret_cast<const uint4*>(vs));
      *reinterpret_cast<uint4*>(kd) = a;
      *reinterpret_cast<uint4*>(vd) = c;
    }
  }
}

size_t elem_size(int dtype) { return dtype == SPECSTEER_F32 ? 4 : 2; }
bool mult16(long long elems, size_t es) { return ((unsigned long long)elems * es) % 16 == 0; }

}  // namespace

// SM count of the current device, read once per device; 0 on failure.
int current_sm_count() {
  static std::atomic<int> known[64];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) { cudaGetLastError(); return 0; }
  int n = known[dev & 63].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return 0; }
    known[dev & 63].store(n, std::memory_order_relaxed);
  }
  return n;
}

}  // namespace specsteer

using namespace specsteer;

extern "C" specsteer_status specsteer_cache_plan(const specsteer_cache_plan_desc* d, void* cuda_stream) {
  if (!d || d->B < 0 || d->page_size <= 0 || d->n_pages <= 0 || d->table_width <= 0 || d->max_tokens < 0 || d->ld_table < d->table_width)
    return SPECSTEER_ERR_INVALID_ARG;
  if (!d->ring_pos || !d->ring_pos_out || !d->cu_new || !d->free_ring) return SPECSTEER_ERR_INVALID_ARG;
  if (d->B > 0 && (!d->seq_len || !d->new_len || !d->pages_held || !d->block_table || !d->seq_len_out || !d->pages_held_out ||
                   !d->kv_len || !d->req_status))
    return SPECSTEER_ERR_INVALID_ARG;
  if (d->max_tokens > 0 && !d->slot_map) return SPECSTEER_ERR_INVALID_ARG;
  if (d->B > SPECSTEER_PLAN_MAX_B) return SPECSTEER_ERR_UNSUPPORTED;
  const size_t smem = (size_t)3 * (d->B + 1) * sizeof(int);
  auto kernel = d->B <= kPlanThreads ? cache_plan_kernel<1> : cache_plan_kernel<SPECSTEER_PLAN_MAX_B / kPlanThreads>;
  if (smem > 48 * 1024 - 512) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
      cudaGetLastError();
      return SPECSTEER_ERR_CUDA;
    }
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kPlanCluster);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = (cudaStream_t)cuda_stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kPlanCluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, *d) != cudaSuccess) {
    cudaGetLastError();
    return SPECSTEER_ERR_CUDA;
  }
  return SPECSTEER_OK;
}

extern "C" specsteer_status specsteer_cache_append(const specsteer_cache_append_desc* d, void* cuda_stream) {
  if (!d || d->T < 0 || d->Hkv <= 0 || d->D <= 0 || d->page_size <= 0 || d->n_pages <= 0) return SPECSTEER_ERR_INVALID_ARG;
  if (d->dtype != SPECSTEER_F32 && d->dtype != SPECSTEER_BF16 && d->dtype != SPECSTEER_F16) return SPECSTEER_ERR_INVALID_ARG;
  if (d->T == 0) return SPECSTEER_OK;
  if (!d->k || !d->v || !d->slot_map || !d->k_cache || !d->v_cache) return SPECSTEER_ERR_INVALID_ARG;
  const long long strides[] = {d->k_tok, d->k_head, d->v_tok, d->v_head, d->kc_page, d->kc_slot, d->kc_head, d->vc_page, d->vc_slot, d->vc_head};
  for (long long x : strides)
    if (x < 0) return SPECSTEER_ERR_INVALID_ARG;
  if ((long long)d->Hkv * d->D > 0x7fffffff) return SPECSTEER_ERR_INVALID_ARG;
  const size_t es = elem_size(d->dtype);
  const int sm = current_sm_count();
  if (sm <= 0) return SPECSTEER_ERR_CUDA;
  bool vec = mult16(d->D, es);
  for (long long x : strides) vec = vec && mult16(x, es);
  const void* ptrs[] = {d->k, d->v, d->k_cache, d->v_cache};
  for (const void* x : ptrs) vec = vec && ((uintptr_t)x & 15u) == 0;
  const long long n = (long long)d->T * d->Hkv * (vec ? d->D / (16 / (int)es) : d->D);
  const long long blocks = (n + 255) / 256;
  const int grid = (int)(blocks < (long long)sm * 16 ? blocks : (long long)sm * 16);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  if (vec && es == 2) cache_append_kernel<uint16_t, 8><<<grid, 256, 0, s>>>(*d);
  else if (vec) cache_append_kernel<uint32_t, 4><<<grid, 256, 0, s>>>(*d);
  else if (es == 2) cache_append_kernel<uint16_t, 1><<<grid, 256, 0, s>>>(*d);
  else cache_append_kernel<uint32_t, 1><<<grid, 256, 0, s>>>(*d);
  if (cudaGetLastError() != cudaSuccess) return SPECSTEER_ERR_CUDA;
  return SPECSTEER_OK;
}
