// Norm by head, rotation by position, and the keys and values into their slots: what stands between a layer's projections
// and its attention, in one pass.
//
// Angles are formed in float64, where the product of a position of 2^31 and a frequency keeps 24 bits behind the point of a turn, and
// reduced to a turn before the sine; all heads that a warp (rotate_kernel) or a block (rotate_any_kernel) takes of a row (token) share them.
//
//   rotate_kernel      a warp a row, or up to eight that share its heads where rows are few; each forms the row's angles for itself, and
//                      none waits for another.  A lane has a piece
//                      (16 bytes; 8 where the widths or alignments want it) of each half of a head, or two neighbouring pieces, so
//                      that the elements of a pair meet in it, and with weights w, the norm r and an element's partner x' an
//                      element becomes r (x A + x' B), A = w cos and B = -+w' sin, formed once a row and warp for the queries and
//                      once for the keys.  The words come through shared
//                      memory, by asynchronous copies several steps ahead, which takes no registers.
//                      Measured (a pass of a captured graph on changing inputs), heads of 128 with norm, bfloat16 unless said: 7671 rows of
//                      32 + 2 x 8 heads, three axes, 36.4 us (5.2 TB/s; 29.3 at the copy bandwidth), bound by the copies in flight and, at 45 % of
//                      its slots, by issue; with one axis 34.7, without norm 32.6, neighbours 46, half of each head turned 40.5; float32 (58.6
//                      at the copy bandwidth) 61, neighbours 90, half turned 70.  1280 rows of 64 + 2 x 8 heads 13.1 us (8.1): a warp's walk
//                      along its row.  5 rows of 64 + 2 x 8 heads 4.0 us, of 32 + 2 x 8 3.6.  The case with three axes took 42 us with
//                      the words in registers, 48 with pieces of 8 bytes.
//   rotate_any_kernel  every shape, alignment and width: a block a row, a warp a head, an element a lane, bound by issue (1280 and 7671 rows
//                      above: 72 and 205 us; 3000 rows of 32 + 2 x 8 heads of 33 69 us).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "f32x2.cuh"
#include "paged.h"
#include "specsteer.h"

namespace specsteer {
namespace {

typedef long long i64;
constexpr int kRotMaxD = SPECSTEER_ROTATE_MAX_D;
constexpr int kRotThreads = 128;
constexpr int kRotWarps = 16;      // on an SM

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

// A word of elements as float32 (one, or a pair of 16-bit ones).
template <int DT> struct Elem;
template <> struct Elem<SPECSTEER_F32> { static constexpr int ES = 4; };
template <> struct Elem<SPECSTEER_BF16> {
  static constexpr int ES = 2;
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(bf16lo(w), bf16hi(w)); }
  static __device__ __forceinline__ uint32_t pack(float2 x) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(x.y), "f"(x.x));
    return r;
  }
};
template <> struct Elem<SPECSTEER_F16> {
  static constexpr int ES = 2;
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
  static __device__ __forceinline__ uint32_t pack(float2 x) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(x.y), "f"(x.x));
    return r;
  }
};
// WORDS words of a head, moved at once.
template <int WORDS> struct Piece;
template <> struct Piece<2> {
  uint32_t w[2];
  __device__ __forceinline__ void get(const void* at) { const uint2 v = *(const uint2*)at; w[0] = v.x; w[1] = v.y; }
  __device__ __forceinline__ void put(void* at) const { *(uint2*)at = make_uint2(w[0], w[1]); }
  static __device__ __forceinline__ void fetch(void* to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(to)), "l"(from) : "memory"); }
};
template <> struct Piece<4> {
  uint32_t w[4];
  __device__ __forceinline__ void get(const void* at) { const uint4 v = *(const uint4*)at; w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
  __device__ __forceinline__ void put(void* at) const { *(uint4*)at = make_uint4(w[0], w[1], w[2], w[3]); }
  static __device__ __forceinline__ void fetch(void* to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory"); }
};
template <int DT, int WORDS> __device__ __forceinline__ void unpack(const Piece<WORDS>& v, float2 (&x)[WORDS * 2 / Elem<DT>::ES]) {
  if constexpr (DT == SPECSTEER_F32) {
#pragma unroll
    for (int i = 0; i < WORDS / 2; ++i) x[i] = make_float2(__uint_as_float(v.w[2 * i]), __uint_as_float(v.w[2 * i + 1]));
  } else {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) x[i] = Elem<DT>::unpack(v.w[i]);
  }
}
template <int DT, int WORDS> __device__ __forceinline__ void pack(const float2 (&x)[WORDS * 2 / Elem<DT>::ES], Piece<WORDS>& v) {
  if constexpr (DT == SPECSTEER_F32) {
#pragma unroll
    for (int i = 0; i < WORDS / 2; ++i) { v.w[2 * i] = __float_as_uint(x[i].x); v.w[2 * i + 1] = __float_as_uint(x[i].y); }
  } else {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) v.w[i] = Elem<DT>::pack(x[i]);
  }
}

constexpr int kAhead = 4;   // steps whose copies a warp has on the way
// A lane has two pieces of WORDS words.  G: lanes of a head, a power of two that covers it.  2^parts_log warps share a row; page_log:
// log2 of the page size, or -1.
template <int DT, int WORDS, int G, bool NEIGHBOURS>
__global__ void __launch_bounds__(kRotThreads, kRotWarps * 32 / kRotThreads)
rotate_kernel(const specsteer_rotate_append_desc p, const int parts_log, const int page_log) {
  __shared__ __align__(16) uint32_t ring[kRotThreads / 32][kAhead][2][32][WORDS];   // a lane's places are its own: nobody waits for anybody
  constexpr int ES = Elem<DT>::ES, H = WORDS * 4 / ES, P = H / 2, kAtOnce = 32 / G;   // elements of a piece, their pairs; heads of a warp's step
  const int lane = threadIdx.x & 31, l = lane & (G - 1), group = lane / G;
  const i64 warp = (i64)blockIdx.x * (kRotThreads / 32) + (threadIdx.x >> 5);
  const i64 t = warp >> parts_log;
  const int parts = 1 << parts_log, part = (int)warp & (parts - 1);
  if (t >= p.T) return;
  const int half = p.rot / 2;
  const bool mine = l * 2 * H < p.D;
  // the lane's two pieces: elements e0.. and e1..; their first pair, and whether they are turned
  const bool turned = NEIGHBOURS ? l * 2 * H < p.rot : l < half / H;
  const int e0 = NEIGHBOURS ? l * 2 * H : turned ? l * H : p.rot + (l - half / H) * 2 * H;
  const int e1 = !NEIGHBOURS && turned ? half + l * H : e0 + H;
  const int pair0 = l * H;
  // Steps of kAtOnce heads: of the queries, then of the keys, then of the values, in turn to the row's warps.
  const int q_steps = (p.Hq + kAtOnce - 1) / kAtOnce, k_steps = (p.Hkv + kAtOnce - 1) / kAtOnce;
  const int from_k = (part - q_steps) & (parts - 1), from_v = (from_k - k_steps) & (parts - 1);
  // A lane's way along the heads of one tensor: its two pieces of every step's head.
  struct Way {
    char *at0, *at1;
    int left;      // heads to go, this one among them (none: 0 or less)
    i64 step;
    __device__ __forceinline__ void next(int heads) { at0 += step; at1 += step; left -= heads; }
    __device__ __forceinline__ void put(const Piece<WORDS>& a, const Piece<WORDS>& b) const {
      if (left > 0) { a.put(at0); b.put(at1); }
    }
  };
  const int heads = parts * kAtOnce;   // from step to step of a warp
  auto way = [&](const void* base, i64 offset, i64 stride, int from, int n) {
    const int h = from * kAtOnce + group;
    char* at = (char*)base + (offset + h * stride) * ES;
    return Way{at + e0 * ES, at + e1 * ES, mine ? n - h : 0, heads * stride * ES};
  };
  // The warp's steps: first nq of the queries, then of the keys, then of the values; step i is fetched kAhead steps before its turn.
  const int nq = (q_steps - part + parts - 1) >> parts_log, nk = (k_steps - from_k + parts - 1) >> parts_log, nv = (k_steps - from_v + parts - 1) >> parts_log;
  const int n = nq + nk + nv;
  uint32_t (*mine_s)[2][32][WORDS] = ring[threadIdx.x >> 5];
  Way src = way(p.q, t * p.q_tok, p.q_head, part, p.Hq);
  auto fetch = [&](int i, int at) {
    if (i == nq) src = way(p.k, t * p.k_tok, p.k_head, from_k, p.Hkv);
    if (i == nq + nk) src = way(p.v, t * p.v_tok, p.v_head, from_v, p.Hkv);
    if (i < n) {
      if (src.left > 0) {
        Piece<WORDS>::fetch(mine_s[at][0][lane], src.at0);
        Piece<WORDS>::fetch(mine_s[at][1][lane], src.at1);
      }
      src.next(heads);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (!mine) {   // lanes beside a head that does not fill its group add nothing to its norm
    Piece<WORDS> zero;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) zero.w[i] = 0u;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) { zero.put(mine_s[i][0][lane]); zero.put(mine_s[i][1][lane]); }
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(i, i);
  const i64 slot = p.Hkv > 0 ? p.slot_map[t] : -1;
  float w0[H], w1[H];
  auto weights = [&](const void* weight) {
#pragma unroll
    for (int i = 0; i < H; ++i) w0[i] = w1[i] = 1.f;
    if (weight && mine && p.eps >= 0.f) {   // (weights belong to the norm)
      if (p.weight_dtype == SPECSTEER_F32) {
#pragma unroll
        for (int i = 0; i < H; ++i) { w0[i] = ((const float*)weight)[e0 + i]; w1[i] = ((const float*)weight)[e1 + i]; }
      } else {
#pragma unroll
        for (int i = 0; i < H; ++i) { w0[i] = weight_at(weight, p.weight_dtype, e0 + i); w1[i] = weight_at(weight, p.weight_dtype, e1 + i); }
      }
    }
  };
  weights(p.q_weight);
  // ---- the angles of the lane's H pairs: the warp's groups have the same ones, so each forms its share
  float2 cs[H];
#pragma unroll
  for (int i = 0; i < H; ++i) cs[i] = make_float2(1.f, 0.f);
  if (p.rot > 0) {
#pragma unroll
    for (int i = 0; i < H; i += kAtOnce) {
      float2 one = make_float2(1.f, 0.f);
      const int my = i + (kAtOnce > 1 ? group % (H < kAtOnce ? H : kAtOnce) : 0);
      if (turned) one = turn_of(p, (int)t, pair0 + my);
#pragma unroll
      for (int j = 0; j < kAtOnce && i + j < H; ++j) {
        const int from = j * G + l;
        cs[i + j] = make_float2(__shfl_sync(kFullMask, one.x, from), __shfl_sync(kFullMask, one.y, from));
      }
    }
  }
  // ---- a lane's element x with partner x' becomes r (x A + x' B)
  float2 A0[P], B0[P], A1[P], B1[P];
  auto coefficients = [&]() {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int x = 2 * i, y = x + 1;
      if (NEIGHBOURS) {
        const float2 a = cs[i], b = cs[P + i];
        A0[i] = make_float2(w0[x] * a.x, w0[y] * a.x);
        A1[i] = make_float2(w1[x] * b.x, w1[y] * b.x);
        B0[i] = make_float2(w0[y] * -a.y, w0[x] * a.y);
        B1[i] = make_float2(w1[y] * -b.y, w1[x] * b.y);
      } else {
        const float2 a = cs[x], b = cs[y];
        A0[i] = make_float2(w0[x] * a.x, w0[y] * b.x);
        A1[i] = make_float2(w1[x] * a.x, w1[y] * b.x);
        B0[i] = make_float2(w1[x] * -a.y, w1[y] * -b.y);
        B1[i] = make_float2(w0[x] * a.y, w0[y] * b.y);
      }
    }
  };
  const float inv_d = 1.f / (float)p.D;
  // one step's heads (the whole warp comes here together)
  auto turn = [&](Piece<WORDS>& v0, Piece<WORDS>& v1) {
    float2 a0[P], a1[P], b0[P], b1[P];
    unpack<DT>(v0, a0);
    unpack<DT>(v1, a1);
    float2 r2 = make_float2(1.f, 1.f);
    if (p.eps >= 0.f) {
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < P; ++i) sum = fma2(a1[i], a1[i], fma2(a0[i], a0[i], sum));
      float s = sum.x + sum.y, r;
#pragma unroll
      for (int o = G / 2; o > 0; o >>= 1) s += __shfl_xor_sync(kFullMask, s, o);
      asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(fmaf(s, inv_d, p.eps)));
      r2 = make_float2(r, r);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      b0[i] = NEIGHBOURS ? make_float2(a0[i].y, a0[i].x) : a1[i];
      b1[i] = NEIGHBOURS ? make_float2(a1[i].y, a1[i].x) : a0[i];
    }
    if (p.rot < p.D && !turned) {   // (an infinity would meet a zero)
#pragma unroll
      for (int i = 0; i < P; ++i) b0[i] = b1[i] = make_float2(0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      b0[i] = mul2(fma2(a0[i], A0[i], mul2(b0[i], B0[i])), r2);
      b1[i] = mul2(fma2(a1[i], A1[i], mul2(b1[i], B1[i])), r2);
    }
    pack<DT>(b0, v0);
    pack<DT>(b1, v1);
  };
  coefficients();
  const bool stored = slot >= 0 && slot < (i64)p.n_pages * p.page_size;
  const i64 page = !stored ? 0 : page_log >= 0 ? slot >> page_log : slot / p.page_size, off = stored ? slot - page * p.page_size : 0;
  const int last = stored ? n : nq;   // (the others are dropped)
  Way dst = way(p.q_out, t * p.o_tok, p.o_head, part, p.Hq);
#pragma unroll 1
  for (int i = 0, at = 0; i < last; ++i, at = at + 1 < kAhead ? at + 1 : 0) {
    if (i == nq) {
      weights(p.k_weight);
      coefficients();
      dst = way(p.k_cache, page * p.kc_page + off * p.kc_slot, p.kc_head, from_k, p.Hkv);
    }
    if (i == nq + nk) dst = way(p.v_cache, page * p.vc_page + off * p.vc_slot, p.vc_head, from_v, p.Hkv);
    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
    Piece<WORDS> a, b;
    a.get(mine_s[at][0][lane]);
    b.get(mine_s[at][1][lane]);
    fetch(i + kAhead, at);
    if (i < nq + nk) turn(a, b);
    dst.put(a, b);
    dst.next(heads);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
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

// Whether rotate_kernel takes a (checked) descriptor in pieces of `bytes`: whole ones everywhere, two a lane, of a pair's halves too, and
// a head in a warp.
bool takes_pieces(const specsteer_rotate_append_desc* d, int bytes) {
  const int n = bytes / (d->dtype == SPECSTEER_F32 ? 4 : 2);
  if (d->D % (2 * n) || d->D > 64 * n || d->rot % (2 * n)) return false;
  auto ok = [&](long long stride, long long extent) { return extent <= 1 || stride % n == 0; };
  auto at = [&](const void* x) { return (uintptr_t)x % bytes == 0; };
  if (d->Hq > 0 && !(at(d->q) && at(d->q_out) && ok(d->q_tok, d->T) && ok(d->q_head, d->Hq) && ok(d->o_tok, d->T) && ok(d->o_head, d->Hq))) return false;
  return d->Hkv == 0 || (at(d->k) && at(d->v) && at(d->k_cache) && at(d->v_cache) && ok(d->k_tok, d->T) && ok(d->k_head, d->Hkv) && ok(d->v_tok, d->T) && ok(d->v_head, d->Hkv) &&
                         ok(d->kc_page, d->n_pages) && ok(d->kc_slot, d->page_size) && ok(d->kc_head, d->Hkv) && ok(d->vc_page, d->n_pages) && ok(d->vc_slot, d->page_size) &&
                         ok(d->vc_head, d->Hkv));
}

template <int DT, int WORDS, int G> void launch_as(const specsteer_rotate_append_desc& d, int sm, cudaStream_t s) {
  // Warps a row: as many as the SMs hold at once (kRotWarps each), since a warp waits more than it computes, and another round of
  // warps costs more than it shares.  bfloat16, 64 + 2 x 8 heads of 128, inputs that change: 5 rows 3.8 us with 8 warps a
  // row (4: 4.5, 1: 9.5), 400 rows 6.9 with 4 (8: 8.8, 2: 7.9, 1: 10.5), 1280 rows 13.2 with 1 (2: 15.4, 8: 18.5).
  const long long steps = ((long long)d.Hq + 2 * d.Hkv) * G / 32;
  int parts_log = 0, page_log = -1;
  while (parts_log < 3 && ((long long)d.T << (parts_log + 1)) <= (long long)sm * kRotWarps && steps >= 2 << parts_log) ++parts_log;
  for (int i = 0; i < 31; ++i)
    if (d.page_size == 1 << i) page_log = i;
  const unsigned grid = (unsigned)((((long long)d.T << parts_log) + kRotThreads / 32 - 1) / (kRotThreads / 32));
  if (d.neighbours) rotate_kernel<DT, WORDS, G, true><<<grid, kRotThreads, 0, s>>>(d, parts_log, page_log);
  else rotate_kernel<DT, WORDS, G, false><<<grid, kRotThreads, 0, s>>>(d, parts_log, page_log);
}
template <int DT, int WORDS> void launch_type(const specsteer_rotate_append_desc& d, int sm, cudaStream_t s) {
  const int lanes = d.D * Elem<DT>::ES / (8 * WORDS);
  if (lanes <= 4) launch_as<DT, WORDS, 4>(d, sm, s);
  else if (lanes <= 8) launch_as<DT, WORDS, 8>(d, sm, s);
  else if (lanes <= 16) launch_as<DT, WORDS, 16>(d, sm, s);
  else launch_as<DT, WORDS, 32>(d, sm, s);
}
template <int WORDS> void launch_rotate(const specsteer_rotate_append_desc& d, int sm, cudaStream_t s) {
  if (d.dtype == SPECSTEER_F32) launch_type<SPECSTEER_F32, WORDS>(d, sm, s);
  else if (d.dtype == SPECSTEER_BF16) launch_type<SPECSTEER_BF16, WORDS>(d, sm, s);
  else launch_type<SPECSTEER_F16, WORDS>(d, sm, s);
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
  const bool by16 = takes_pieces(d, 16);
  if (by16 || takes_pieces(d, 8)) {
    if (by16) launch_rotate<4>(*d, sm, s);
    else launch_rotate<2>(*d, sm, s);
    return cudaGetLastError() == cudaSuccess ? SPECSTEER_OK : SPECSTEER_ERR_CUDA;
  }
  const int grid = d->T < sm * 64 ? d->T : sm * 64;
  if (d->dtype == SPECSTEER_F32) rotate_any_kernel<float><<<grid, kRotThreads, 0, s>>>(*d);
  else if (d->dtype == SPECSTEER_BF16) rotate_any_kernel<__nv_bfloat16><<<grid, kRotThreads, 0, s>>>(*d);
  else rotate_any_kernel<__half><<<grid, kRotThreads, 0, s>>>(*d);
  return cudaGetLastError() == cudaSuccess ? SPECSTEER_OK : SPECSTEER_ERR_CUDA;
}
