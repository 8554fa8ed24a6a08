// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits, in one read of the logits.
//
// logprobs_stream_kernel reads.  All rows' tiles of 4 KB form one list, which is cut into equal ranges, a warp each, so that few
// long rows and many short ones load the SMs alike and no warp waits for another.  With l = c x, c = log2(e)/temperature, a lane
// keeps of a row
//   S = sum 2^(l - ref),   W = sum 2^(l - ref) (l - ref)
// for a reference that follows its largest l at a distance of at most 8, so that S and W are rescaled for hardly any tile; at a row's
// or a range's end the warp brings them together and leaves a record.  The difference of logits is formed before it is
// scaled, so that entries of the type's lowest value, and rows of nothing else, stay in float32's range (see Scale).  For the likeliest tokens a lane
// leaves the largest entry of its part of a tile (a slot: 128 bytes), and the stream carries no selection at all.
//
// logprobs_end_kernel, a CTA a row, joins the records at M = max l:  lse = M + log2 S,  entropy = log2 S - W/S  (in units of log 2).
// From the slots' maxima it takes a bound that at least n_top entries reach (the least of the best few lanes' maxima of each
// warp), reads the slots that reach it again, hardly more than n_top, and ranks their entries that do by counting.  Where too
// many do (a masked vocabulary, equal entries) warps keep lists of one 64-bit key a lane instead (larger value first, then lower id)
// and pass over slots whose best possible key does not beat the list's.
//
// logprobs_few_kernel, for few rows, does both in one launch: a cluster reads a row, its warps leave records and slots in the first
// CTA's shared memory, and that CTA ends the row.  It needs no workspace, so that a call is 5 us shorter on the host.
//
// Measured (a pass among others of a captured graph on changing rows; in brackets what its bytes would take at the copy bandwidth):
//   1280 rows of 151 936, bfloat16, tempered, top 20    74 to 75 us (60), 82 to 88 in a loop of a second; without likeliest tokens 64.5 us
//   640 rows of 151 936, float32, top 20                69 us (60); without 61 us, 6.4 TB/s
//   3584 rows of 256 000, bfloat16, top 20              306 us (285)
//   5 rows of 32 000, float32, top 8                    6 us (in one launch: logprobs_few_kernel): a chain of trips to L2 and barriers
// The stream is bound by HBM with float32; with 16 bits the special-function unit (one ex2 an entry, busy for 69 % of the cycles) and the
// issue of 7 instructions an entry come up to it, and pass it at the clocks the power limit leaves.  Eight vectors a lane (two tiles, one
// ahead, are all the registers of 16 warps an SM) beat four with 24 or 32 warps: 65 us, 72 and 74 without likeliest tokens.
// A CTA a row that ends it too took 95 us for the sums alone and 140 with 20 tokens: nothing is loaded while a row ends.
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
constexpr int kThreads = 256, kCtas = 2;   // of the streaming kernel, on an SM
constexpr int kVecs = 8;                   // vectors of 16 bytes that a lane has of a tile
constexpr int kTileVecs = 32 * kVecs;      // of a tile: 4 KB, a warp's step
constexpr int kEndThreads = 128, kEndWarps = kEndThreads / 32;
// Few rows: the most CTAs of a row (a cluster), and the tiles that a CTA takes (four a warp).  No CTA waits for one of another row, so that
// all of them being on a B200's 148 SMs at once is a matter of time only; the bound is the same on a device with fewer.
constexpr int kFewCtas = 8, kFewTiles = 16;
constexpr int kFewSm = 5, kFewMax = kFewSm * 148;   // CTAs that an SM holds, and all of them
constexpr int kPicked = 512;               // slots and entries that the quick selection takes
constexpr int kMaxSms = 148;                // the workspace is laid out for as many
constexpr float kSlack = 8.f;        // how far l may be above the reference
constexpr float kLeast = 1024.f;     // and below: there a weight is zero, and its product with the distance too

// The types of logits: elements of a vector, the pair in a 32-bit word (16-bit types), -inf in every element, the largest of a vector.
template <int DT> struct Logit;
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i < 2 ? (i ? v.y : v.x) : (i == 2 ? v.z : v.w); }
template <> struct Logit<SPECSTEER_F32> {
  typedef float type;
  static constexpr int N = 4;
  static constexpr uint32_t kNone = 0xff800000u;
  static __device__ __forceinline__ float one(const float* x) { return *x; }
  static __device__ __forceinline__ float2 pair(const uint4& v, int i) {
    return i == 0 ? make_float2(__uint_as_float(v.x), __uint_as_float(v.y)) : make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  // the entries that reach tau, a bit each; the entry of a bit, and its value
  static __device__ __forceinline__ uint32_t reach(const uint4& v, float tau) {
    return (__uint_as_float(v.x) >= tau) | (__uint_as_float(v.y) >= tau) << 1 | (__uint_as_float(v.z) >= tau) << 2 | (__uint_as_float(v.w) >= tau) << 3;
  }
  static __device__ __forceinline__ int entry(int bit) { return bit; }
  static __device__ __forceinline__ float value(const uint4& v, int bit) { return __uint_as_float(word_of(v, bit)); }
  static __device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
  }
  template <int NV> static __device__ __forceinline__ float largest(const uint4 (&v)[NV]) {
    float m = __uint_as_float(v[0].x);
#pragma unroll
    for (int u = 0; u < NV; ++u) m = max3_nan(max3_nan(m, __uint_as_float(v[u].x), __uint_as_float(v[u].y)), __uint_as_float(v[u].z), __uint_as_float(v[u].w));
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
  static __device__ __forceinline__ uint32_t reach(const uint4& v, float tau) {   // bit i: low half of word i, bit 16 + i: the high one
    uint32_t got = 0;
    const uint32_t t2 = __float_as_uint(tau) | __float_as_uint(tau) >> 16;          // (tau is a number of this type)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t m;
      asm("set.ge.u32.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(word_of(v, i)), "r"(t2));
      got |= (m & 0x10001u) << i;
    }
    return got;
  }
  static __device__ __forceinline__ int entry(int bit) { return 2 * (bit & 15) + (bit >> 4); }
  static __device__ __forceinline__ float value(const uint4& v, int bit) {
    const uint32_t w = word_of(v, bit & 15);
    return bit >> 4 ? bf16hi(w) : bf16lo(w);
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  template <int NV> static __device__ __forceinline__ float largest(const uint4 (&v)[NV]) {
    uint32_t m = v[0].x;
#pragma unroll
    for (int u = 0; u < NV; ++u) m = max2(max2(m, v[u].x), max2(v[u].y, max2(v[u].z, v[u].w)));
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
  static __device__ __forceinline__ uint32_t reach(const uint4& v, float tau) {
    uint32_t got = 0;
    const uint32_t t1 = __half_as_ushort(__float2half_rn(tau)), t2 = t1 | t1 << 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t m;
      asm("set.ge.u32.f16x2 %0, %1, %2;" : "=r"(m) : "r"(word_of(v, i)), "r"(t2));
      got |= (m & 0x10001u) << i;
    }
    return got;
  }
  static __device__ __forceinline__ int entry(int bit) { return 2 * (bit & 15) + (bit >> 4); }
  static __device__ __forceinline__ float value(const uint4& v, int bit) {
    return __half2float(__ushort_as_half((unsigned short)(word_of(v, bit & 15) >> (bit & 16))));
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  template <int NV> static __device__ __forceinline__ float largest(const uint4 (&v)[NV]) {
    uint32_t m = v[0].x;
#pragma unroll
    for (int u = 0; u < NV; ++u) m = max2(max2(m, v[u].x), max2(v[u].y, max2(v[u].z, v[u].w)));
    m = max2(m, (m >> 16) | (m << 16));
    return __half2float(__ushort_as_half((unsigned short)m));
  }
};

// From logits to l: l(x) - l(y) = (x pre - y pre) c, with c pre = log2(e)/temperature and a power of two for pre, so that neither the difference
// of two logits (temperatures from 1 on: the quotient may be within float32's range where the difference is not) nor c (temperatures
// below float32's normal numbers) passes the range.  The product with pre and the subtraction are one multiply-add, which rounds once, as a
// subtraction alone would; with that one 1280 rows of 151 936 take 73.2 us, with this 73.9.
struct Scale {
  float pre, c;
};
__device__ __forceinline__ Scale scale_of(float temperature) {
  const float pre = temperature >= 1.f ? 0.25f : temperature < 0x1p-126f ? 0x1p30f : 1.f;
  return Scale{pre, kLog2e / (temperature * pre)};
}
// -y pre, or the nearest number where that is infinite: then the row's lse is none, or y is far below its largest logit and nothing as far down gets a weight.
__device__ __forceinline__ float negated(float y, Scale q) {
  constexpr float most = 3.402823466e38f;
  return fmaxf(fminf(-y * q.pre, most), -most);
}
__device__ __forceinline__ float distance(float x, float y, Scale q) { return fmaf(x, q.pre, negated(y, q)) * q.c; }

// S and W of a thread, with their reference (a logit; none yet: -inf).
struct Sums {
  float ref, s, w;
};
__device__ __forceinline__ void rescale(Sums& a, float to, Scale q) {
  if (a.ref == kNegInf) {
    a.s = a.s == a.s ? 0.f : a.s;   // NaN stays
    a.w = 0.f;
  } else {
    const float d = fmaxf(distance(a.ref, to, q), -kLeast), f = ex2(d);
    a.w = fmaf(a.s, d, a.w) * f;
    a.s *= f;
  }
  a.ref = to;
}
// Takes a chunk in; returns its largest entry.
template <int DT> __device__ __forceinline__ float take(Sums& a, const uint4 (&v)[kVecs], Scale q) {
  typedef Logit<DT> L;
  const float mx = L::largest(v);
  if (mx > kNegInf && mx < -kNegInf) {
    if (a.ref == kNegInf || distance(mx, a.ref, q) > kSlack) rescale(a, mx, q);
    const float r = negated(a.ref, q);
    const float2 c2 = make_float2(q.c, q.c), p2 = make_float2(q.pre, q.pre), r2 = make_float2(r, r);
    float2 s[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, w[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
#pragma unroll
      for (int i = 0; i < L::N / 2; ++i) {
        float2 t = mul2(fma2(L::pair(v[u], i), p2, r2), c2);
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

__device__ __forceinline__ float warp_min_redux(float v) {
  float r;
  asm volatile("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
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

struct LogParams {
  specsteer_token_logprobs_desc d;
  int tiles;                 // of a row (one of 16-byte aligned start has as many vectors as any)
  long long warps;           // that share the tiles
  double tile_inv, total_inv, warp_inv;   // 1/tiles, 1/(R tiles), 1/warps
  float4* record;            // [R + warps]: that of warp w for row r at r + w
  uint16_t* slot_max;        // [R][tiles][32], or nullptr: rounded down to bfloat16, of float16 logits as they are
};

// A row: entries before the first 16-byte boundary, whole vectors, entries behind them.
template <int DT> struct Row {
  typedef typename Logit<DT>::type T;
  static constexpr int N = Logit<DT>::N;
  const T* x;
  int head, n_vec;
  __device__ __forceinline__ Row(const specsteer_token_logprobs_desc& d, i64 r) {
    x = (const T*)d.logits + r * d.ld_row;
    const int off = (int)(((uintptr_t)x & 15u) / sizeof(T));
    head = min(d.V, off ? N - off : 0);
    n_vec = (d.V - head) / N;
  }
};
// a / b with 1/b at hand: a division of 64 bits is a hundred instructions, of a kernel that takes a few microseconds.
__device__ __forceinline__ i64 divide(i64 a, i64 b, double inv) {
  i64 q = (i64)((double)a * inv);   // off by one at most (a below 2^52: the rows lie in memory)
  if (q * b > a) --q;
  else if ((q + 1) * b <= a) ++q;
  return q;
}
// The warp whose range holds a tile: ranges are [n w / W, n (w+1) / W).
__device__ __forceinline__ i64 warp_of(const LogParams& p, i64 tile) { return divide((tile + 1) * p.warps - 1, (i64)p.d.R * p.tiles, p.total_inv); }

// A slot's maximum has 16 bits.  Rounded down it serves both ends: entries reach a bound formed from such numbers, and a slot holds
// an entry that reaches a bound of that kind just when its own number does.  Only -inf itself becomes -inf: finite numbers
// below bfloat16's lowest become that one, which as a bound stands for float32's lowest (see tau).
constexpr uint32_t kLowest = 0xff7f0000u;
template <int DT> __device__ __forceinline__ uint16_t slot_bits(float x) {
  if (DT == SPECSTEER_F16) return __half_as_ushort(__float2half_rn(x));   // (exact)
  uint32_t b = __float_as_uint(x);                                        // (NaN may become anything: its row has no result)
  if (DT == SPECSTEER_F32 && (b >> 31)) b = b >= kLowest && b < 0xff800000u ? kLowest : b + 0xffffu;
  return (uint16_t)(b >> 16);
}
// streaming loads of what is read once, which do not push what is read again out of L2
__device__ __forceinline__ uint4 load_once(const uint4* at, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(at), "l"(policy));
  return v;
}

// This lane's part of a tile.
template <int DT> __device__ __forceinline__ void load_tile(const Row<DT>& row, int tile, int lane, uint64_t policy, uint4 (&to)[kVecs]) {
  typedef Logit<DT> L;
  const uint4* at = reinterpret_cast<const uint4*>(row.x + row.head) + (i64)tile * kTileVecs + lane;
  const int left = row.n_vec - tile * kTileVecs - lane;
  if (left > 32 * (kVecs - 1)) {
#pragma unroll
    for (int u = 0; u < kVecs; ++u) to[u] = load_once(at + 32 * u, policy);
  } else {
#pragma unroll
    for (int u = 0; u < kVecs; ++u) to[u] = 32 * u < left ? load_once(at + 32 * u, policy) : make_uint4(L::kNone, L::kNone, L::kNone, L::kNone);
  }
}

template <int DT>
__global__ void __launch_bounds__(kThreads, kCtas) logprobs_stream_kernel(const LogParams p) {
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const i64 w = (i64)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), total = (i64)p.d.R * p.tiles;
  if (w >= p.warps) return;
  const i64 first = divide(total * w, p.warps, p.warp_inv), end = divide(total * (w + 1), p.warps, p.warp_inv);
  if (first >= end) return;
  const uint64_t policy = l2_policy_evict_first();
  i64 r = divide(first, p.tiles, p.tile_inv);
  int tile = (int)(first - r * p.tiles);
  // the row and tile of the loads, one tile ahead of those of the sums
  i64 next_r = r;
  int next_tile = tile;
  Row<DT> row(p.d, r);
  Scale next_q = scale_of(p.d.temperature ? p.d.temperature[r] : 1.f), q = next_q;
  uint4 v[kVecs], next[kVecs];
  load_tile(row, tile, lane, policy, v);
  Sums a{kNegInf, 0.f, 0.f};
  float top = kNegInf;
#pragma unroll 1
  for (i64 i = first; i < end; ++i) {
    const bool more = i + 1 < end;
    if (more) {
      if (++next_tile == p.tiles) {
        next_tile = 0;
        row = Row<DT>(p.d, ++next_r);
        next_q = scale_of(p.d.temperature ? p.d.temperature[next_r] : 1.f);
      }
      load_tile(row, next_tile, lane, policy, next);
    }
    const float mx = take<DT>(a, v, q);
    top = fmaxf(top, mx);
    if (p.slot_max) p.slot_max[(r * p.tiles + tile) * 32 + lane] = slot_bits<DT>(mx);
    if (!more || next_r != r) {
      const float M = warp_max(top);
      rescale(a, M == kNegInf ? 0.f : M, q);
      const float s = warp_sum(a.s), ww = warp_sum(a.w);
      if (lane == 0) p.record[r + w] = make_float4(M, s, ww, 0.f);
      a = Sums{kNegInf, 0.f, 0.f};
      top = kNegInf;
      q = next_q;
    }
    r = next_r;
    tile = next_tile;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) v[u] = next[u];
  }
}

// What no entry of a slot with (rounded) maximum x exceeds: of float32 logits the next number of bfloat16.
template <int DT> __device__ __forceinline__ float slot_bound(float x) {
  if (DT != SPECSTEER_F32 || x == kNegInf || x == -kNegInf) return x;
  const int b = __float_as_int(x);
  return x == 0.f ? __int_as_float(0x10000) : __int_as_float(b > 0 ? b + 0x10000 : b - 0x10000);
}

struct EndShared {
  float red[3][kEndWarps];
  float best[32];                  // the best few lanes' maxima of each warp
  int n_slots, n_keys;
  int slot[kPicked];
  u64 key[kPicked];
  u64 out[32];                     // the likeliest, in order
};

// Row r's end, by kEndThreads threads, from its records (n of them from `record` on) and slots; wait() returns once those are there.
// Executed once a row, so it is its latency that counts, and that of fetching its instructions: what can be is a short loop.
template <int DT, typename Wait>
__device__ __forceinline__ void end_row(const LogParams& p, i64 r, EndShared& sh, const float4* record, int n_record, const uint16_t* slot_max, Wait&& wait) {
  typedef Logit<DT> L;
  typedef Logit<DT == SPECSTEER_F16 ? SPECSTEER_F16 : SPECSTEER_BF16> S;   // of the slots' maxima
  typedef typename L::type T;
  const specsteer_token_logprobs_desc& d = p.d;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float nan = __int_as_float(0x7fc00000);
  const Row<DT> row(d, r);
  const T* x = row.x;
  const float temp = d.temperature ? d.temperature[r] : 1.f;
  const Scale sc = scale_of(temp);
  // the entries outside the vectors, one a thread
  const int rest = d.V - row.head - row.n_vec * L::N;
  float single = kNegInf;
  int single_at = -1;
  if (tid < row.head + rest) {
    single_at = tid < row.head ? tid : d.V - rest + (tid - row.head);
    single = L::one(x + single_at);
  }
  // the first of the given tokens
  auto logit_of = [&](int i, int* token) {
    *token = d.token[r * d.ld_tok + i];
    return *token >= 0 && *token < d.V ? L::one(x + *token) : 0.f;
  };
  int token = -1;
  float given = 0.f;
  if (tid < d.n_tokens) given = logit_of(tid, &token);
  if (tid == 0) sh.n_slots = sh.n_keys = 0;
  wait();
  // ---- the slots' maxima: vectors, kHeld a thread at a time; the last ones stay in registers
  const int n_slot = p.tiles * 32, n_max = d.n_top > 0 ? n_slot / S::N : 0;
  const typename S::type* slots = (const typename S::type*)slot_max;
  const uint4* maxima = reinterpret_cast<const uint4*>(slots);
  constexpr int kHeld = 4;
  const uint4 none = make_uint4(S::kNone, S::kNone, S::kNone, S::kNone);
  const int mine = lane * kEndWarps + warp;   // in turn to the warps, which then share few of them
  uint4 held[kHeld];
  auto hold = [&](int base) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      const int j = base + mine + k * kEndThreads;
      held[k] = j < n_max ? maxima[j] : none;
    }
  };
  hold(0);
  // ---- the row's records
  Sums a{kNegInf, 0.f, 0.f};
#pragma unroll 1
  for (int w = tid; w < n_record; w += kEndThreads) {
    const float4 q = record[w];
    const float M = fmaxf(a.ref, q.x);
    rescale(a, M, sc);
    Sums b{q.x, q.y, q.z};
    rescale(b, M, sc);
    a.s += b.s;
    a.w += b.w;
  }
  float top = S::largest(held);
#pragma unroll 1
  for (int base = kHeld * kEndThreads; base < n_max; base += kHeld * kEndThreads) {
    hold(base);
    top = fmaxf(top, S::largest(held));
  }
  if (single > kNegInf && single < -kNegInf) {
    const float M = fmaxf(a.ref, single);
    rescale(a, M, sc);
    const float t = fmaxf(distance(single, M, sc), -kLeast), e = ex2(t);
    a.s += e;
    a.w = fmaf(e, t, a.w);
  } else if (single != kNegInf) {
    a.s = nan;
  }
  const float warp_top = warp_max_redux(a.ref);
  if (lane == 0) sh.red[0][warp] = warp_top;
  if (d.n_top > 0) {
    const int few = (d.n_top + kEndWarps - 1) / kEndWarps;   // as many of each warp, of different lanes
    float t = top;
    if (n_slot <= kHeld * kEndThreads) {   // few vectors, which would leave lanes without a maximum: single ones
      t = kNegInf;
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        const int j = mine + k * kEndThreads;
        if (j < n_slot) t = fmaxf(t, S::one(slots + j));
      }
    }
#pragma unroll 1
    for (int i = 0; i < few; ++i) {
      const float b = warp_max_redux(t);
      const uint32_t who = __ballot_sync(kFullMask, t == b);
      if (who && lane == __ffs(who) - 1) t = kNegInf;
      if (lane == 0) sh.best[i * kEndWarps + warp] = b;
    }
  }
  __syncthreads();
  float M = sh.red[0][0];
#pragma unroll
  for (int w = 1; w < kEndWarps; ++w) M = fmaxf(M, sh.red[0][w]);
  rescale(a, M == kNegInf ? 0.f : M, sc);
  const float ws = warp_sum(a.s), ww = warp_sum(a.w);
  if (lane == 0) { sh.red[1][warp] = ws; sh.red[2][warp] = ww; }
  // ---- the bound, and the slots and single entries that reach it
  float tau = kNegInf, slot_tau = kNegInf;
  if (d.n_top > 0) {
    const int bests = (d.n_top + kEndWarps - 1) / kEndWarps * kEndWarps;
    tau = warp_min_redux(lane < bests ? sh.best[lane] : -kNegInf);
    auto pick = [&](int base) {
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        const int j = base + mine + k * kEndThreads;
        uint32_t hits = j < n_max ? S::reach(held[k], tau) : 0u;
        if (!hits) continue;
        int at = atomicAdd(&sh.n_slots, __popc(hits));
#pragma unroll 1
        for (; hits && at < kPicked; hits &= hits - 1) sh.slot[at++] = j * S::N + S::entry(__ffs(hits) - 1);
      }
    };
    if (top >= tau) {
      int base = n_max > 0 ? (n_max - 1) / (kHeld * kEndThreads) * (kHeld * kEndThreads) : 0;   // what is held
#pragma unroll 1
      for (;;) {
        pick(base);
        if ((base -= kHeld * kEndThreads) < 0) break;
        hold(base);
      }
    }
    slot_tau = tau;
    if (DT == SPECSTEER_F32 && __float_as_uint(tau) == kLowest) tau = -3.402823466e38f;   // of entries; slots have been picked
    if (single_at >= 0 && single >= tau) {
      const int at = atomicAdd(&sh.n_keys, 1);
      if (at < kPicked) sh.key[at] = entry_key(single + 0.f, single_at);
    }
  }
  __syncthreads();
  float s = 0.f, w = 0.f;
#pragma unroll
  for (int i = 0; i < kEndWarps; ++i) { s += sh.red[1][i]; w += sh.red[2][i]; }
  const float l2s = log2f(s), ln_s = l2s * kLn2, lse = ln_s + M / temp;
  const bool bad_temp = !(temp > 0.f && temp < -kNegInf);
  const bool bad = bad_temp || !(s > 0.f && s < -kNegInf) || !(fabsf(lse) < -kNegInf);
  auto from_max = [&](float y) { return fmaf(y, sc.pre, negated(M, sc)) / (temp * sc.pre); };   // (y - M) / temp
  // vector u of slot j, counted from the row's first; n_vec or more: there is none
  auto vec_of = [&](int j, int u) { return (i64)(j >> 5) * kTileVecs + (j & 31) + 32 * u; };
  const int picked = sh.n_slots;
  if (picked <= kPicked && !bad) {
    const uint4* vec = reinterpret_cast<const uint4*>(x + row.head);
    constexpr int kBatch = 3;   // vectors a thread has on the way
#pragma unroll 1
    for (int e0 = tid; e0 < picked * kVecs; e0 += kBatch * kEndThreads) {
      uint4 v[kBatch];
      int at[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int e = e0 + k * kEndThreads;
        const i64 i = e < picked * kVecs ? vec_of(sh.slot[e / kVecs], e % kVecs) : row.n_vec;
        at[k] = row.head + (int)i * L::N;
        v[k] = i < row.n_vec ? __ldg(vec + i) : make_uint4(0u, 0u, 0u, 0u);
        if (i >= row.n_vec) at[k] = -1;
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        uint32_t hits = at[k] >= 0 ? L::reach(v[k], tau) : 0u;
        if (!hits) continue;
        int n = atomicAdd(&sh.n_keys, __popc(hits));
#pragma unroll 1
        for (; hits && n < kPicked; hits &= hits - 1) {
          const int bit = __ffs(hits) - 1;
          sh.key[n++] = entry_key(L::value(v[k], bit) + 0.f, at[k] + L::entry(bit));
        }
      }
    }
  }
  if (tid == 0) {
    if (d.lse) d.lse[r] = bad ? nan : lse;
    if (d.entropy) d.entropy[r] = bad ? nan : (l2s - w / s) * kLn2;
    if (bad && d.row_status) atomicOr(d.row_status + r, bad_temp ? SPECSTEER_REQ_BAD_PARAM : SPECSTEER_REQ_NONFINITE);
  }
#pragma unroll 1
  for (int i = tid; i < d.n_tokens; i += kEndThreads) {
    if (i != tid) given = logit_of(i, &token);
    const bool outside = token < 0 || token >= d.V;
    if (outside && token != -1 && d.row_status) atomicOr(d.row_status + r, SPECSTEER_REQ_BAD_TOKEN);
    d.logprob[r * d.ld_tok + i] = bad ? nan : outside ? kNegInf : from_max(given) - ln_s;
  }
  if (d.n_top == 0) return;
  __syncthreads();
  const int keys = sh.n_keys;
  if (!bad && picked <= kPicked && keys <= kPicked) {
#pragma unroll 1
    for (int i = tid; i < keys; i += kEndThreads) {
      const u64 key = sh.key[i];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < keys; ++j) rank += sh.key[j] > key;
      if (rank < d.n_top) sh.out[rank] = key;
    }
  } else if (!bad) {
    // ---- too many: lists, a warp every kEndWarps-th tile, read again where some slot may still beat the list's last
    u64 list = 0, last = 0;
    auto offer = [&](float value, int at, bool there) {   // by the whole warp
      const u64 key = entry_key(value + 0.f, at);
      uint32_t todo = __ballot_sync(kFullMask, there && key > last);
#pragma unroll 1
      while (todo) {
        const int src = __ffs(todo) - 1;
        todo &= todo - 1;
        list_insert(list, __shfl_sync(kFullMask, key, src), lane);
      }
      last = __shfl_sync(kFullMask, list, d.n_top - 1);
    };
    if (warp == 0) offer(single, single_at, single_at >= 0);
    const uint4* vec = reinterpret_cast<const uint4*>(x + row.head);
#pragma unroll 1
    for (int tile = warp; tile < p.tiles; tile += kEndWarps) {
      const i64 from = (i64)tile * kTileVecs + lane;
      const float most = S::one(slots + tile * 32 + lane);
      const u64 bound = entry_key(slot_bound<DT>(most) + 0.f, row.head + (int)from * L::N);
      if (!__any_sync(kFullMask, from < row.n_vec && most >= slot_tau && bound > last)) continue;
      constexpr int kPart = kVecs / 2;   // (half a tile at a time: the registers are what the ordinary rows' CTAs of an SM share)
#pragma unroll 1
      for (i64 at = from; at < from + 32 * kVecs; at += 32 * kPart) {
        uint4 v[kPart];
#pragma unroll
        for (int u = 0; u < kPart; ++u) v[u] = at + 32 * u < row.n_vec ? __ldg(vec + at + 32 * u) : make_uint4(L::kNone, L::kNone, L::kNone, L::kNone);
        // (of float32 logits the slots' bounds are rounded up: once more, exactly)
        const float exact = L::largest(v);
        if (!__any_sync(kFullMask, exact >= tau && entry_key(exact + 0.f, row.head + (int)at * L::N) > last)) continue;
#pragma unroll
        for (int u = 0; u < kPart; ++u) {
          const bool there = at + 32 * u < row.n_vec;
#pragma unroll 1
          for (int i = 0; i < L::N; ++i) {
            const int bit = L::N == 8 ? (i >> 1) + 16 * (i & 1) : i;   // entry i
            const float y = L::value(v[u], bit);
            offer(y, row.head + (int)(at + 32 * u) * L::N + i, there && y >= tau);
          }
        }
      }
    }
    __syncthreads();   // (the keys are read no more)
    sh.key[tid] = list;
    __syncthreads();
    if (warp == 0) {
#pragma unroll 1
      for (int i = 1; i < kEndWarps; ++i) list = list_merge(list, sh.key[i * 32 + 31 - lane], lane);
      sh.out[lane] = list;
    }
  }
  __syncthreads();
  if (tid < d.n_top) {
    const u64 key = sh.out[tid];
    d.top_id[r * d.n_top + tid] = bad ? -1 : (int)(0xffffffffu - (uint32_t)key);
    d.top_logprob[r * d.n_top + tid] = bad ? nan : from_max(order_val((uint32_t)(key >> 32))) - ln_s;
  }
}

template <int DT>
__global__ void __launch_bounds__(kEndThreads, 10) logprobs_end_kernel(const LogParams p) {
  __shared__ EndShared sh;
  const i64 r = blockIdx.x;
  const i64 w0 = p.tiles > 0 ? warp_of(p, r * p.tiles) : 0, w1 = p.tiles > 0 ? warp_of(p, (r + 1) * p.tiles - 1) : -1;
  end_row<DT>(p, r, sh, p.record + r + w0, (int)(w1 - w0 + 1), p.slot_max + r * p.tiles * 32, [] { pdl_wait(); });
}

// Few rows of few tiles: a cluster reads a row, leaves records and slots in its first CTA's shared memory, and that one ends it.
template <int DT>
__global__ void __launch_bounds__(kEndThreads, kFewSm) logprobs_few_kernel(const LogParams p) {
  __shared__ EndShared sh;
  __shared__ __align__(16) uint16_t slot_s[kFewCtas * kFewTiles * 32];
  __shared__ float4 record_s[kFewCtas * kEndWarps];
  cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int ctas = (int)cluster.num_blocks(), warps = ctas * kEndWarps;
  const int rank = (int)cluster.block_rank(), lane = threadIdx.x & 31, w = rank * kEndWarps + (threadIdx.x >> 5);
  const i64 r = blockIdx.x / ctas;
  const Row<DT> row(p.d, r);
  const Scale q = scale_of(p.d.temperature ? p.d.temperature[r] : 1.f);
  const int first = p.tiles * w / warps, end = p.tiles * (w + 1) / warps;
  const uint64_t policy = l2_policy_evict_first();
  uint4 v[kVecs];
  if (first < end) load_tile(row, first, lane, policy, v);
  uint16_t* slots = cluster.map_shared_rank(slot_s, 0);
  float4* records = cluster.map_shared_rank(record_s, 0);
  cluster.sync();   // the first CTA is there
  Sums a{kNegInf, 0.f, 0.f};
  float top = kNegInf;
#pragma unroll 1
  for (int tile = first; tile < end; ++tile) {
    uint4 next[kVecs];
    if (tile + 1 < end) load_tile(row, tile + 1, lane, policy, next);
    const float mx = take<DT>(a, v, q);
    top = fmaxf(top, mx);
    slots[tile * 32 + lane] = slot_bits<DT>(mx);
#pragma unroll
    for (int u = 0; u < kVecs; ++u) v[u] = next[u];
  }
  const float M = warp_max(top);
  rescale(a, M == kNegInf ? 0.f : M, q);
  const float s = warp_sum(a.s), ww = warp_sum(a.w);
  if (lane == 0) records[w] = make_float4(M, s, ww, 0.f);
  auto all_written = [&] { cluster.sync(); };   // (nobody reads another's memory from there on)
  if (rank == 0) end_row<DT>(p, r, sh, record_s, warps, slot_s, all_written);
  else all_written();
}

struct LogPlan { int tiles, grid, few; long long warps; size_t record_bytes, max_bytes; };
LogPlan plan_of(const specsteer_token_logprobs_desc* d, int sm) {
  LogPlan q;
  const int es = d->dtype == SPECSTEER_F32 ? 4 : 2;
  q.tiles = (int)(((long long)d->V * es / 16 + kTileVecs - 1) / kTileVecs);
  // One launch, and no workspace, up to the CTAs that 148 SMs hold at once: clusters of as many as that leaves a row.  bfloat16, top
  // 20, device / call: 64 rows of 151 936 take 11.0 / 12.6 us, with two launches 13.7 / 16.2; 300 rows of 8000 8.4 / 10.3, 11.0 / 12.9; 740
  // rows of 16 000 12.0 / 14.4, 14.8 / 16.5; but 900 of them, in another round of CTAs, 16.9, 15.9.  With twice as many CTAs 160 rows of 32 000
  // take 13.5 instead of 9.5.
  q.few = 0;
  for (int ctas = kFewCtas; ctas > 0 && !q.few; ctas /= 2)
    if ((long long)d->R * ctas <= kFewMax && q.tiles <= ctas * kFewTiles) q.few = ctas;
  const long long total = (long long)d->R * q.tiles, most = (long long)sm * kCtas * (kThreads / 32);
  q.warps = total < most ? total : most;
  q.grid = (int)((q.warps + kThreads / 32 - 1) / (kThreads / 32));
  q.record_bytes = ((size_t)(d->R + q.warps) * sizeof(float4) + 31) & ~(size_t)31;
  q.max_bytes = d->n_top > 0 ? (size_t)total * 32 * sizeof(uint16_t) : 0;
  return q;
}

template <int DT> cudaError_t launch(const LogParams& p, const LogPlan& q, cudaStream_t s) {
  if (q.few) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.d.R * q.few);
    cfg.blockDim = dim3(kEndThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = q.few;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, logprobs_few_kernel<DT>, p);
  }
  if (q.grid > 0) {
    logprobs_stream_kernel<DT><<<q.grid, kThreads, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.d.R);
  cfg.blockDim = dim3(kEndThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = q.grid > 0 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, logprobs_end_kernel<DT>, p);
}

specsteer_status check_logprobs(const specsteer_token_logprobs_desc* d) {
  if (!d || d->R < 0 || d->V < 1 || d->n_tokens < 0 || d->n_top < 0 || d->n_top > SPECSTEER_TOP_MAX || d->n_top > d->V || d->ld_row < d->V) return SPECSTEER_ERR_INVALID_ARG;
  if (d->dtype != SPECSTEER_F32 && d->dtype != SPECSTEER_BF16 && d->dtype != SPECSTEER_F16) return SPECSTEER_ERR_INVALID_ARG;
  if (d->n_tokens > 0 && d->ld_tok < d->n_tokens) return SPECSTEER_ERR_INVALID_ARG;
  if (d->R > 0 && (!d->logits || (d->n_tokens > 0 && (!d->token || !d->logprob)) || (d->n_top > 0 && (!d->top_id || !d->top_logprob)))) return SPECSTEER_ERR_INVALID_ARG;
  return SPECSTEER_OK;
}

}  // namespace
}  // namespace specsteer

using namespace specsteer;

extern "C" size_t specsteer_token_logprobs_workspace(const specsteer_token_logprobs_desc* d) {
  if (check_logprobs(d) != SPECSTEER_OK || d->R == 0) return 0;
  const LogPlan q = plan_of(d, kMaxSms);
  return q.few ? 0 : q.record_bytes + q.max_bytes;
}

extern "C" specsteer_status specsteer_token_logprobs(const specsteer_token_logprobs_desc* d, void* cuda_stream) {
  const specsteer_status st = check_logprobs(d);
  if (st != SPECSTEER_OK || d->R == 0) return st;
  const size_t need = specsteer_token_logprobs_workspace(d);
  if (need > 0 && (!d->workspace || ((uintptr_t)d->workspace & 31u) || d->workspace_bytes < (long long)need)) return SPECSTEER_ERR_WORKSPACE;
  const int sm = current_sm_count();
  if (sm <= 0) return SPECSTEER_ERR_CUDA;
  const LogPlan q = plan_of(d, sm < kMaxSms ? sm : kMaxSms);
  LogParams p;
  p.d = *d;
  p.tiles = q.tiles;
  p.warps = q.warps;
  p.tile_inv = 1. / (q.tiles ? q.tiles : 1);
  p.total_inv = 1. / (q.tiles ? (double)d->R * q.tiles : 1.);
  p.warp_inv = 1. / (q.warps ? (double)q.warps : 1.);
  p.record = (float4*)d->workspace;
  p.slot_max = q.max_bytes ? (uint16_t*)((char*)d->workspace + q.record_bytes) : nullptr;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  const cudaError_t e = d->dtype == SPECSTEER_F32 ? launch<SPECSTEER_F32>(p, q, s)
                        : d->dtype == SPECSTEER_BF16 ? launch<SPECSTEER_BF16>(p, q, s) : launch<SPECSTEER_F16>(p, q, s);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return SPECSTEER_ERR_CUDA;
  }
  return SPECSTEER_OK;
}
