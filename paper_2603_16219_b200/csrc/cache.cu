// Bookkeeping of the paged key/value cache: block tables and slot maps from request lengths, and the chunk's keys and
// values into their slots.
//
//   cache_plan_kernel    one thread-block cluster; every CTA forms the same running sums over the requests (tokens,
//                        pages taken, pages given back) in its own shared memory, then the cluster shares the page
//                        moves and the rows of the slot map.  Cluster barriers order the steps that touch the
//                        same memory: pages given back -> pages taken -> slots -> the in-place outputs.  Latency is what
//                        it costs, so a small plan gets one CTA of few threads: its barriers are cheaper.
//   cache_append_kernel  a copy by slot, 16 bytes a thread where alignment allows.  Bound by HBM: 31 thousand tokens of 8 heads
//                        of 128 (256 MB read and written) 42 us, 6.1 TB/s; 96 tokens 2 us.
#include <atomic>

#include "common.cuh"
#include "internal.h"
#include "paged.h"
#include "specsteer.h"

namespace specsteer {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanCluster = 8;      // CTAs at most: the portable cluster size

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

// Exclusive sums of a pair over the threads of the block in thread order; *total receives the sums.  One barrier: `scratch`
// ([32] pairs) must not be written again before the next one.
struct Pair { i64 a, b; };
__device__ __forceinline__ Pair block_exclusive_sums(Pair v, Pair* scratch, Pair* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  Pair x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const i64 a = __shfl_up_sync(kFullMask, x.a, o), b = __shfl_up_sync(kFullMask, x.b, o);
    if (lane >= o) { x.a += a; x.b += b; }
  }
  if (nw > 1) {
    if (lane == 31) scratch[warp] = x;
    __syncthreads();
    // every warp sums the warps' totals for itself
    Pair w = lane < nw ? scratch[lane] : Pair{0, 0};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const i64 a = __shfl_up_sync(kFullMask, w.a, o), b = __shfl_up_sync(kFullMask, w.b, o);
      if (lane >= o) { w.a += a; w.b += b; }
    }
    total->a = __shfl_sync(kFullMask, w.a, 31);
    total->b = __shfl_sync(kFullMask, w.b, 31);
    const i64 a = __shfl_sync(kFullMask, w.a, warp ? warp - 1 : 0), b = __shfl_sync(kFullMask, w.b, warp ? warp - 1 : 0);
    if (warp) { x.a += a; x.b += b; }
  } else {
    total->a = __shfl_sync(kFullMask, x.a, 31);
    total->b = __shfl_sync(kFullMask, x.b, 31);
  }
  return Pair{x.a - v.a, x.b - v.b};
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
  __shared__ Pair scratch[3][32];
  const int B = p.B, tid = threadIdx.x;
  int* cum_tok = plan_smem;                // [B+1] running sums: tokens, pages given back, pages taken
  int* cum_give = cum_tok + (B + 1);       // [B+1]
  int* cum_take = cum_give + (B + 1);      // [B+1]
  int* kept_s = cum_take + (B + 1);        // [B] tokens kept
  int* from_s = kept_s + B;                // [B] table entry where the request's pages taken or given back begin
  const uint32_t rank = cluster_rank(), n_cta = cluster_size();
  const int first_thread = (int)rank * blockDim.x + tid, n_threads = (int)n_cta * blockDim.x;

  // (a cluster barrier makes every store visible to the other SMs first, which one CTA does not need)
  auto sync_all = [&] {
    if (n_cta == 1) __syncthreads();
    else cluster_sync_all();
  };

  const i64 head = p.ring_pos[0], tail = p.ring_pos[1], P = p.n_pages;
  const bool pool_ok = head >= 0 && tail >= head && tail - head <= P;
  const i64 capacity = (i64)p.table_width * p.page_size;

  int seq[IPT], asked[IPT], held[IPT], status[IPT];
  i64 kept[IPT];
  Pair sum{0, 0}, total;
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
      sum.a += asked[k];
    }
  }
  Pair run = block_exclusive_sums(sum, scratch[0], &total);
  // tokens beyond max_tokens are refused; then the pages each request gives back or wants
  Pair pages{0, 0}, page_total;            // given back, wanted
  int target[IPT];
#pragma unroll
  for (int k = 0; k < IPT; ++k) {
    run.a += asked[k];
    if (asked[k] > 0 && run.a > p.max_tokens) { status[k] |= SPECSTEER_REQ_NO_ROOM; asked[k] = 0; }
    const bool passed_on = status[k] & (SPECSTEER_REQ_BAD_LEN | SPECSTEER_REQ_BAD_POOL);
    target[k] = passed_on ? held[k] : (int)((kept[k] + asked[k] + p.page_size - 1) / p.page_size);
    const int d = target[k] - held[k];
    if (d > 0) pages.b += d; else pages.a -= d;
  }
  Pair page_run = block_exclusive_sums(pages, scratch[1], &page_total);
  const i64 room = pool_ok ? P - (tail - head) : 0;
  const int given = (int)(page_total.a < room ? page_total.a : room);   // more would mean that a page was handed out twice
  const i64 avail = pool_ok ? tail - head + given : 0;
  Pair served{0, 0}, served_total;         // tokens, pages taken
#pragma unroll
  for (int k = 0; k < IPT; ++k) {
    const int b = tid * IPT + k;
    const int d = target[k] - held[k];
    if (b < B) {
      cum_give[b] = (int)(page_run.a < 0x7fffffff ? page_run.a : 0x7fffffff);
      cum_take[b] = (int)(page_run.b < avail ? page_run.b : avail);
      kept_s[b] = (int)kept[k];
      from_s[b] = d > 0 ? held[k] : target[k];
    }
    if (d < 0) page_run.a -= d;
    if (d > 0) {
      page_run.b += d;
      // sums only grow: once a request is refused, every later one that wants pages is too, so the takers that are
      // served are a prefix and their running sum above is right
      if (page_run.b > avail) { status[k] |= SPECSTEER_REQ_NO_PAGES; asked[k] = 0; target[k] = held[k]; }
      else served.b += d;
    }
    served.a += asked[k];
  }
  Pair tok_run = block_exclusive_sums(served, scratch[2], &served_total);
#pragma unroll
  for (int k = 0; k < IPT; ++k) {
    const int b = tid * IPT + k;
    if (b < B) cum_tok[b] = (int)tok_run.a;
    tok_run.a += asked[k];
  }
  const int n_tok = (int)served_total.a, taken = (int)served_total.b;
  if (tid == 0) {
    cum_tok[B] = n_tok;
    cum_give[B] = (int)(page_total.a < 0x7fffffff ? page_total.a : 0x7fffffff);
    cum_take[B] = taken;
  }
  __syncthreads();

  const i64 head0 = pool_ok ? head % P : 0, tail0 = pool_ok ? tail % P : 0;
  auto ring_at = [&](i64 base, int r) { return base + r < P ? base + r : base + r - P; };   // r < P
  // pages given back: entry target + i of the request's table to place tail + r of the ring (64-bit counters: a pool may have
  // 2^31 - 1 pages, and a counter steps past the last)
  for (i64 i = first_thread; i < given; i += n_threads) {
    const int r = (int)i, b = owner_of(cum_give, B, r);
    p.free_ring[ring_at(tail0, r)] = p.block_table[(i64)b * p.ld_table + from_s[b] + (r - cum_give[b])];
  }
  if (rank == 0) {
#pragma unroll
    for (int k = 0; k < IPT; ++k)
      if (tid * IPT + k < B) p.req_status[tid * IPT + k] = status[k];
  }
  sync_all();   // the ring is whole; nobody reads the inputs any more, which the outputs may be in place of
  for (i64 i = first_thread; i < taken; i += n_threads) {
    const int r = (int)i, b = owner_of(cum_take, B, r);
    p.block_table[(i64)b * p.ld_table + from_s[b] + (r - cum_take[b])] = __ldcg(p.free_ring + ring_at(head0, r));
  }
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
      p.ring_pos_out[0] = head + taken;
      p.ring_pos_out[1] = tail + given;
    }
  }
  sync_all();   // the tables are whole; the status words are there for the slots to add to
  // Four rows of the slot map a thread, their page ids on the way together.  Pages of a power of two need no division.
  const int shift = (p.page_size & (p.page_size - 1)) == 0 ? __ffs(p.page_size) - 1 : -1;
  auto page_of = [&](int pos) { return shift >= 0 ? pos >> shift : pos / p.page_size; };
  constexpr int kRows = 4;
  for (i64 i0 = first_thread; i0 < p.max_tokens; i0 += kRows * n_threads) {
    int b[kRows], pos[kRows], page[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const i64 at = i0 + (i64)k * n_threads;
      b[k] = pos[k] = -1;
      page[k] = 0;
      if (at < n_tok) {
        const int i = (int)at;
        b[k] = owner_of(cum_tok, B, i);
        pos[k] = kept_s[b[k]] + (i - cum_tok[b[k]]);
        page[k] = __ldcg(p.block_table + (i64)b[k] * p.ld_table + page_of(pos[k]));
      }
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const i64 i = i0 + (i64)k * n_threads;
      if (i >= p.max_tokens) break;
      i64 slot = -1;
      if (b[k] >= 0) {
        if (page[k] >= 0 && page[k] < p.n_pages) slot = (i64)page[k] * p.page_size + (pos[k] - page_of(pos[k]) * p.page_size);
        else atomicOr(p.req_status + b[k], SPECSTEER_REQ_BAD_PAGE);
      }
      p.slot_map[i] = slot;
      if (p.positions) p.positions[i] = pos[k];
      if (p.token_req) p.token_req[i] = b[k];
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

constexpr int kPlanIpt = SPECSTEER_PLAN_MAX_B / kPlanThreads;   // of the kernel for more requests than a CTA has threads
constexpr size_t plan_smem_bytes(int B) { return ((size_t)5 * B + 3) * sizeof(int); }

// Shared memory for the largest plan, allowed once per device.  The limit belongs to the kernel and not to a call: a call that
// set its own size would take it away under another thread that is about to launch a larger plan.
bool allow_largest_plan() {
  static std::atomic<bool> done[64];   // two threads that both find it clear set the same value
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) { cudaGetLastError(); return false; }
  if (done[dev & 63].load(std::memory_order_acquire)) return true;
  if (cudaFuncSetAttribute(cache_plan_kernel<kPlanIpt>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plan_smem_bytes(SPECSTEER_PLAN_MAX_B)) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  done[dev & 63].store(true, std::memory_order_release);
  return true;
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
  const size_t smem = plan_smem_bytes(d->B);
  auto kernel = d->B <= kPlanThreads ? cache_plan_kernel<1> : cache_plan_kernel<kPlanIpt>;
  // A plan is bound by its barriers and by the slot map's dependent steps (owner, table entry, slot), never by its bytes.
  // Up to 256 requests and 4096 rows one CTA serves: 32 threads for a handful of requests (one request and 5 rows 3.8 us,
  // with 256 threads 4.7), else 256.  Larger plans get a CTA for every 512 rows up to the cluster (512 requests and 3584
  // rows 8.1 us, in four CTAs 8.9, in one 13.6; 24 prompts with 49 thousand rows 14 us, 18 and 47), of 512 threads while
  // there is a thread a request (the first of the two with 1024: 10.4 us).
  const bool small = d->B <= 256 && d->max_tokens <= 4096;
  const int threads = !small ? (d->B <= 512 ? 512 : kPlanThreads) : d->B <= 32 && d->max_tokens <= 256 ? 32 : 256;
  const int wanted = d->max_tokens / 512 + (d->max_tokens % 512 != 0);
  const int ctas = small || wanted < 1 ? 1 : wanted < kPlanCluster ? wanted : kPlanCluster;
  if (smem > 40 * 1024 && !allow_largest_plan()) return SPECSTEER_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = (cudaStream_t)cuda_stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
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
  // slots that share memory would overwrite one another
  if ((d->n_pages > 1 && (!d->kc_page || !d->vc_page)) || (d->page_size > 1 && (!d->kc_slot || !d->vc_slot)) || (d->Hkv > 1 && (!d->kc_head || !d->vc_head)))
    return SPECSTEER_ERR_INVALID_ARG;
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
