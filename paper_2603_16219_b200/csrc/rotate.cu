// Norm by head, rotation by position, and the keys and values into their slots: what stands between a layer's projections
// and its attention, in one pass.
//
// A block takes a row (token).  Its angles are formed once, in float64, where the product of a position of 2^31 and a frequency keeps 22
// bits behind the point of a turn, and reduced to a turn before the sine; all heads of the row share them.  A warp takes a head.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "paged.h"
#include "specsteer.h"

namespace specsteer {
namespace {

typedef long long i64;
constexpr int kRotMaxD = SPECSTEER_ROTATE_MAX_D;
constexpr int kRotThreads = 256;

__device__ __forceinline__ float load_f32(const float* x) { return *x; }
__device__ __forceinline__ float load_f32(const __nv_bfloat16* x) { return __bfloat162float(*x); }
__device__ __forceinline__ float load_f32(const __half* x) { return __half2float(*x); }
__device__ __forceinline__ void store_f32(float x, float* y) { *y = x; }
__device__ __forceinline__ void store_f32(float x, __nv_bfloat16* y) { *y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void store_f32(float x, __half* y) { *y = __float2half_rn(x); }

__device__ __forceinline__ float weight_at(const void* w, int dtype, int i) {
  if (!w) return 1.f;
  if (dtype == SPECSTEER_F32) return load_f32((const float*)w + i);
  return dtype == SPECSTEER_BF16 ? load_f32((const __nv_bfloat16*)w + i) : load_f32((const __half*)w + i);
}

// Cosine and sine of pair i of row t, times the factor.
__device__ __forceinline__ float2 turn_of(const specsteer_rotate_append_desc& p, int t, int i) {
  const int axis = p.axis_of ? p.axis_of[i] : 0;
  double turns = 0.;
  if (axis >= 0 && axis < p.n_axes) turns = (double)p.positions[(i64)axis * p.T + t] * (double)p.inv_freq[i] * 0.15915494309189535;   // 1 / (2 pi)
  turns -= rint(turns);
  float s, c;
  sincospif(2.f * (float)turns, &s, &c);
  return make_float2(c * p.factor, s * p.factor);
}

// Every shape: a warp a head, lane l takes elements l, l + 32, ...
template <typename T>
__global__ void __launch_bounds__(kRotThreads) rotate_any_kernel(const specsteer_rotate_append_desc p) {
  __shared__ float2 turn_s[kRotMaxD / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int half = p.rot / 2;
  const i64 slots = (i64)p.n_pages * p.page_size;
  for (i64 t = blockIdx.x; t < p.T; t += gridDim.x) {
    __syncthreads();
    for (int i = threadIdx.x; i < half; i += kRotThreads) turn_s[i] = turn_of(p, (int)t, i);
    const i64 slot = p.Hkv > 0 ? p.slot_map[t] : -1;
    const bool stored = slot >= 0 && slot < slots;
    const i64 page = stored ? slot / p.page_size : 0, off = stored ? slot - page * p.page_size : 0;
    __syncthreads();
    for (int h = warp; h < p.Hq + p.Hkv; h += kRotThreads / 32) {
      const bool is_q = h < p.Hq;
      const int hk = h - p.Hq;
      if (!is_q && !stored) continue;
      const T* x = is_q ? (const T*)p.q + t * p.q_tok + h * p.q_head : (const T*)p.k + t * p.k_tok + hk * p.k_head;
      T* y = is_q ? (T*)p.q_out + t * p.o_tok + h * p.o_head : (T*)p.k_cache + page * p.kc_page + off * p.kc_slot + hk * p.kc_head;
      const void* weight = is_q ? p.q_weight : p.k_weight;
      float a[kRotMaxD / 32], b[kRotMaxD / 32], sum = 0.f;   // an element, the other of its pair
#pragma unroll
      for (int k = 0; k < kRotMaxD / 32; ++k) {
        const int e = lane + 32 * k;
        a[k] = b[k] = 0.f;
        if (e < p.D) {
          a[k] = load_f32(x + e);
          if (e < p.rot) b[k] = load_f32(x + (p.neighbours ? e ^ 1 : e < half ? e + half : e - half));
        }
        sum = fmaf(a[k], a[k], sum);
      }
      const float scale = p.eps >= 0.f ? 1.f / sqrtf(warp_sum(sum) / (float)p.D + p.eps) : 1.f;
      __syncwarp();   // y may be x
#pragma unroll
      for (int k = 0; k < kRotMaxD / 32; ++k) {
        const int e = lane + 32 * k;
        if (e >= p.D) continue;
        const bool normed = p.eps >= 0.f;
        float out = normed ? a[k] * scale * weight_at(weight, p.weight_dtype, e) : a[k];
        if (e < p.rot) {
          const int other = p.neighbours ? e ^ 1 : e < half ? e + half : e - half;
          const bool second = p.neighbours ? e & 1 : e >= half;
          const float2 cs = turn_s[p.neighbours ? e >> 1 : e < half ? e : e - half];
          const float partner = normed ? b[k] * scale * weight_at(weight, p.weight_dtype, other) : b[k];
          out = fmaf(out, cs.x, second ? partner * cs.y : -partner * cs.y);
        }
        store_f32(out, y + e);
      }
    }
    if (stored) {
      for (int h = warp; h < p.Hkv; h += kRotThreads / 32) {
        const T* x = (const T*)p.v + t * p.v_tok + h * p.v_head;
        T* y = (T*)p.v_cache + page * p.vc_page + off * p.vc_slot + h * p.vc_head;
        for (int e = lane; e < p.D; e += 32) y[e] = x[e];
      }
    }
  }
}

}  // namespace
}  // namespace specsteer

using namespace specsteer;

extern "C" specsteer_status specsteer_rotate_append(const specsteer_rotate_append_desc* d, void* cuda_stream) {
  if (!d || d->T < 0 || d->Hq < 0 || d->Hkv < 0 || d->D <= 0 || d->rot < 0 || d->rot > d->D || d->rot % 2) return SPECSTEER_ERR_INVALID_ARG;
  for (int dt : {d->dtype, d->weight_dtype})
    if (dt != SPECSTEER_F32 && dt != SPECSTEER_BF16 && dt != SPECSTEER_F16) return SPECSTEER_ERR_INVALID_ARG;
  if (d->eps != d->eps || d->factor != d->factor) return SPECSTEER_ERR_INVALID_ARG;
  if (d->D > SPECSTEER_ROTATE_MAX_D) return SPECSTEER_ERR_UNSUPPORTED;
  const long long strides[] = {d->q_tok, d->q_head, d->k_tok, d->k_head, d->v_tok, d->v_head, d->o_tok, d->o_head,
                               d->kc_page, d->kc_slot, d->kc_head, d->vc_page, d->vc_slot, d->vc_head};
  for (long long x : strides)
    if (x < 0) return SPECSTEER_ERR_INVALID_ARG;
  if (d->Hkv > 0) {
    if (d->page_size <= 0 || d->n_pages <= 0) return SPECSTEER_ERR_INVALID_ARG;
    if ((d->n_pages > 1 && (!d->kc_page || !d->vc_page)) || (d->page_size > 1 && (!d->kc_slot || !d->vc_slot)) || (d->Hkv > 1 && (!d->kc_head || !d->vc_head)))
      return SPECSTEER_ERR_INVALID_ARG;   // slots that share memory would overwrite one another
    if (d->T > 0 && (!d->k || !d->v || !d->slot_map || !d->k_cache || !d->v_cache)) return SPECSTEER_ERR_INVALID_ARG;
  }
  if (d->Hq > 0) {
    if ((d->T > 1 && !d->o_tok) || (d->Hq > 1 && !d->o_head)) return SPECSTEER_ERR_INVALID_ARG;
    if (d->T > 0 && (!d->q || !d->q_out)) return SPECSTEER_ERR_INVALID_ARG;
  }
  if (d->rot > 0 && (d->n_axes < 1 || (d->T > 0 && (!d->positions || !d->inv_freq)))) return SPECSTEER_ERR_INVALID_ARG;
  if ((long long)d->Hq + d->Hkv > 0x7fffffff - 64) return SPECSTEER_ERR_INVALID_ARG;
  if (d->T == 0 || d->Hq + d->Hkv == 0) return SPECSTEER_OK;
  const int sm = current_sm_count();
  if (sm <= 0) return SPECSTEER_ERR_CUDA;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  const int grid = d->T < sm * 64 ? d->T : sm * 64;
  if (d->dtype == SPECSTEER_F32) rotate_any_kernel<float><<<grid, kRotThreads, 0, s>>>(*d);
  else if (d->dtype == SPECSTEER_BF16) rotate_any_kernel<__nv_bfloat16><<<grid, kRotThreads, 0, s>>>(*d);
  else rotate_any_kernel<__half><<<grid, kRotThreads, 0, s>>>(*d);
  return cudaGetLastError() == cudaSuccess ? SPECSTEER_OK : SPECSTEER_ERR_CUDA;
}
