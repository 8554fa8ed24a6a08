// Attention of a chunk of new tokens over the paged cache on the tensor cores (tcgen05, TMA).
//
// Rows.  For one kv head a query tile is up to 128 rows, row r = token * G + head within the group (G = Hq/Hkv), so that
// all query heads of a kv head share every key that is loaded.  A unit of work is one or two query tiles (two when the
// request has more tokens than one tile holds) against all tiles of 128 keys that its rows see.
//
// Split.  The key tiles of all units, in order (request, kv head, unit), form one list, which is cut into equal ranges,
// one per CTA (one CTA per SM).  Ragged lengths, one long request and a large batch then load the SMs alike, and the
// cut needs nothing from the host: every CTA sums the lengths itself.  A unit that a cut goes through leaves partial
// results (unnormalised sums, maximum and sum of weights per row) that attention_join_kernel puts together.
//
// Inside a CTA: warps 8 and 9 issue the TMA loads of keys and of values, each into a ring of blocks of 64 keys (a page, or
// its part of 64 keys, is a box; one warp for both could not issue the boxes of small pages fast enough), and warp 8 also
// walks the list.  Warps 0..3 and 4..7 are two softmax groups (streams), one row a thread, and warps 10 and 11 issue the
// tcgen05.mma of one stream each (one warp for both spent its time on waits and commits).  Stream s has scores S_s (two
// blocks of 64 keys, 64 columns of tensor memory each, overwritten by the 16-bit weights P_s, which the second product
// reads from tensor memory) and sums O_s (128 columns).  The product that gives a block's next scores is issued behind the
// one that takes its weights, so while a group weighs one block the tensor cores work on the other.  With two query tiles
// each stream owns one and both use every key tile; with one query tile the streams take the key tiles in turn and are put
// together at the end.
//
// Maximum.  Weights are 2^(c s - c m + lift) with a reference m per row.  A block is weighed against the reference there
// is; only if that makes its weights sum to more than 2^15 (or there is none yet) the block's maximum is formed, the
// reference raised, O_s rescaled in tensor memory and the block weighed again.  Weights are then at most 2^15, which
// float16 holds, and after the first tile hardly any block needs its maximum, a sixth of the work.  The exponent is one fused
// multiply-add of s with the rounded lift - c m, off by half a step of c m: a common factor of the row, which cancels, as
// long as it leaves the weights in range.  From |c m| = 2^24 on (half a step: 1) it is c (s - m) + lift instead, with m the
// maximum so far, formed for every block: rare, and a branch of the warp that the other rows do not pay for.
//
// Measured (bfloat16 and D = 128 unless said; a call among others on inputs that change, on several machines; in brackets a
// pass among others of a captured graph, whose inputs stay the same):
//   3 requests of 30 to 120 thousand keys, 9 tokens of 64 heads        166 to 185 us, 5.0 to 5.6 TB/s (163 to 170): bound by HBM
//   256 requests of up to 4000 keys, 5 tokens of 64 heads              415 to 458 us, 4.8 to 5.3 TB/s (405 to 417): bound by HBM
//   a prompt of 8192 tokens of 32 heads                                0.61 to 0.63 ms, 0.88 to 0.90 PFLOP/s (0.59 to 0.60): bound by
//     the issue of the softmax warps and by the clock that the power limit leaves (tensor pipe busy for 45 % of the cycles)
//   64 single tokens, up to 4000 keys, 32 heads of 64, float16         81 to 87 us, 3.0 to 3.2 TB/s (78): the few rows of a request
//     sit in one warp of each stream, whose 2000 clocks a block of 64 keys (1500 of arithmetic and tensor-memory latency,
//     500 of handshakes) bound it
// and of trees (specsteer_tree_attention):
//   64 trees of 15 to 32 rows, up to 4000 keys, 64 heads               196 to 207 us (168 to 203), 0.5 to 0.6 PFLOP/s of useful products: bound by the
//     ends of its pieces (one every 17 tiles) and the join; without softmax and most of the products it takes 150 us
//   2 trees of 49 to 63 rows, 30 to 120 thousand keys, 32 heads        196 to 207 us (164 to 203), 0.71 to 0.75 PFLOP/s (to 0.9): bound by the chain of scores, weights
//     and sums (152 us without the arithmetic of the softmax, 119 without most of the products too)
//   48 trees of up to 25 rows, 32 heads of 64, window 1024, float16    42 to 45 us: ends of pieces
//   a tree of 1024 rows, 1100 keys, 32 heads                           73 us where a chain takes 44: masks need not be trees, so every unit of it
//     reads all of the chunk's keys, at the edge
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "attention.cuh"
#include "f32x2.cuh"

namespace specsteer {
namespace {

constexpr int kKeys = 128;          // keys per tile
constexpr int kBlock = 64;          // keys per block: half a tile, what a barrier or a box covers
constexpr int kSoftmaxWarps = 8;
constexpr int kKeyWarp = kSoftmaxWarps, kValueWarp = kSoftmaxWarps + 1, kMmaWarp = kSoftmaxWarps + 2;
constexpr int kTcThreads = 32 * (kSoftmaxWarps + 4);
constexpr uint32_t kTcCols = 512;   // S0, S1, O0, O1 of 128 columns each
constexpr int kPolyPairs = 5;       // of 32 pairs of weights, how many ex2_poly takes off the special-function unit (4 to 6 are alike)
constexpr float kMostSum = 32768.f; // of the weights of a row and block before the reference is raised
constexpr float kMostArg = 15.f;    // the exponent that no such weight exceeds
// The largest weight is 2^kLift: with float16 the weights below 2^-22 of the largest are subnormal, not those below 2^-14,
// and a whole block of largest ones still sums to less than kMostSum.
template <bool BF> constexpr float kLift = BF ? 0.f : 8.f;
constexpr float kFar = 16777216.f;  // |c m| beyond which c s - c m is not formed from the two products (see Maximum)
constexpr int kPieces = 4;          // pieces of work the producer may be ahead

template <int DP> struct TcLayout {
  static constexpr int kStageBytes = kBlock * DP * 2;
  static constexpr int kStages = DP == 128 ? 5 : 10;              // of each of the two rings
  static constexpr int kQBytes = 128 * DP * 2;
  static constexpr int kKeyRing = 2 * kQBytes;                    // offsets: two query tiles, the rings, TcShared
  static constexpr int kValueRing = kKeyRing + kStages * kStageBytes;
  static constexpr int kControl = kValueRing + kStages * kStageBytes;
};

// A piece of work: key tiles [first, first + take) of one unit (see Unit).
struct Piece {
  int b, hk;
  int row0, n, kv;             // of the request
  int tok0, tok1;              // the unit's tokens
  int two;                     // two query tiles
  int lo_first;                // where the keys of the first row begin
  int hi_first, lo_last;       // where they end, where those of the last row begin
  int first, take;             // take = 0: no more pieces
  int starts, ends;            // the piece holds the unit's first / last key tile
  int index;                   // of the pieces of this CTA
};

// Barriers of the two rings, per stage.  A block of a piece with one query tile is one stream's alone: barriers of its own
// (full 0, 1) say that it has landed, and one arrival frees it; with two query tiles both streams wait for it (full 2) and
// free it.  So every barrier is waited for each time it comes around by all that it concerns, and no phase is mistaken for
// another.  (With one set for all, each stream had to wait for the other's blocks too: contexts of 30 to 120 thousand
// keys took 162 us instead of 158.)
template <int DP> struct RingBars {
  uint64_t k_full[3][TcLayout<DP>::kStages], v_full[3][TcLayout<DP>::kStages];
  uint64_t k_empty[2][TcLayout<DP>::kStages], v_empty[2][TcLayout<DP>::kStages];   // one stream's, both streams'
};

struct TcShared {
  uint64_t q_full[2], q_empty[2];
  uint64_t s_full[2][2], p_full[2][2];   // [s][h]: scores, weights of stream s, first / last 64 keys of a tile
  uint64_t o_full[2], half_done[2];      // a piece's sums; those of the stream but for the last 64 keys
  uint64_t piece_full[kPieces], piece_empty[kPieces];
  uint64_t both, group[2], drain[2];
  uint32_t tmem_slot;
  int nonfinite;           // an infinity or NaN was taken out of a tile of values
  int start_b, start_hk, start_u, start_off;
  long long end;           // where this CTA's range ends, from the beginning of its first unit (0: it has none)
  Piece piece[kPieces];
  uint8_t bad[32];         // per block of keys (counted modulo 32): the boxes of it that lie outside the pool
  union {
    long long scan[kTcThreads / 32];
    float2 exch[2][128];   // reference and sum of each stream's rows
  };
};
template <int DP> constexpr int tc_smem_bytes() { return TcLayout<DP>::kControl + (int)(sizeof(TcShared) + sizeof(RingBars<DP>)); }
static_assert(sizeof(TcShared) % 8 == 0 && tc_smem_bytes<128>() <= 232448 && tc_smem_bytes<64>() <= 232448, "shared memory of one CTA");

struct TcParams {
  specsteer_attention_desc d;
  TreeMask tree;
  int G, box_tok, box_rows, tile_tok;  // query box: tokens and rows; tokens of a query tile
  int page_rows, boxes, page_shift;    // key box: keys, boxes per block, log2 of its keys
  int page_blocks, pb_shift;           // blocks per page (1 when a block has several pages), log2 of them or -1
  float c;                             // scale * log2(e)
  int out_vec;                         // out rows are 32-byte aligned and a multiple of 32 bytes long
  float* part;                         // [2*gridDim][256][DP] unnormalised sums
  float2* part_ml;                     // [2*gridDim][256] reference (raw score) and sum
  int* head;                           // [gridDim][8] 0: slot of the part of a unit that goes on in the next CTA (-1: none), 2..4: that
                                       // unit's first row, kv head and tokens; 1: this CTA's part of a unit that began before it (0: none,
                                       // 1: its end, 2: more)
  int* failed;                         // [gridDim] whether a bounded wait of the CTA has run out
  int stop_at;                         // blocks of keys after which a CTA loads no more (see SPECSTEER_ATTENTION_STOP)
};

// ---- PTX wrappers -------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(tm), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(tm), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void tc_alloc(uint32_t* slot) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(kTcCols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_dealloc(uint32_t addr) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(kTcCols) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// One thread of the (converged) warp issues.  The election is inside the statement: behind a branch of that thread the
// compiler moves every operand to uniform registers anew, and the issue takes longer than the product.
// D (+)= A B^T with both operands in shared memory; descriptors by their low words, the high words are alike.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 x, y;\n\telect.sync _|q, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(kDescHigh)
      : "memory");
}
// the same with A in tensor memory
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 y;\n\telect.sync _|q, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 y, {%2, %5};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(kDescHigh)
      : "memory");
}
// the barrier receives one arrival once every tcgen05.mma issued so far by the electing thread has completed
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void tm_ld32(uint32_t addr, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
        "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
        "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_ld16(uint32_t addr, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t addr, const uint32_t* u) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(u[0]),
      "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]),
      "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(addr)
      : "memory");
}
// Waits for the loads issued so far.  v, the registers of the load, are operands so that nothing that uses them moves ahead.
__device__ __forceinline__ void tm_ld_wait(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                 "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
                 "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}
// the same for further registers of the loads that tm_ld_wait waited for
__device__ __forceinline__ void tm_ld_tie(float* v) {
  asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
               "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
               "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
               "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}
__device__ __forceinline__ void tm_ld_wait16(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
               :
               : "memory");
}
// 32 bytes to a 32-byte aligned address: a whole sector a thread, a row a thread
__device__ __forceinline__ void st_256(void* at, const uint32_t* u) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]),
               "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}
__device__ __forceinline__ void tm_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory descriptors of 128-byte swizzled operands, in units of 16 bytes: low words (address, leading offset); the
// high word is the stride offset (groups of 8 rows 1024 bytes apart), the version 1 and the swizzle mode 2.  K and Q (rows
// of 64 elements along the summed axis) have no leading offset (1); of V (the summed axis, keys, runs over the rows) it is
// the distance of blocks of 64 columns, one chunk of 64 rows.
__device__ __forceinline__ uint32_t desc_rows(uint32_t addr) { return ((addr & 0x3ffffu) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_cols(uint32_t addr) { return ((addr & 0x3ffffu) >> 4) | ((uint32_t)((kBlock * 128) >> 4) << 16); }
// Instruction descriptor: float32 accumulator, operands bf16 or f16, M = 128.
__device__ __forceinline__ uint32_t instr_desc(bool bf16, int n, bool b_by_columns) {
  const uint32_t f = bf16 ? 1u : 0u;
  return (1u << 4) | (f << 7) | (f << 10) | ((b_by_columns ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN stays
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// 2^x of two numbers on the FMA and integer pipes: x = i + f with |f| <= 1/2, 2^f by the polynomial of degree 5 of least
// largest relative error (7.5e-8, 2.2e-7 with the roundings; coefficients by a Remez exchange), times 2^i.  Zero below
// 2^-126 (i = -127 makes the factor's bits zero), NaN for NaN; x up to 127.
__device__ __forceinline__ float2 ex2_poly(float2 x) {
  const float2 magic = make_float2(12582912.f, 12582912.f), unmagic = make_float2(-12582912.f, -12582912.f);
  x = make_float2(max_nan(x.x, -127.f), max_nan(x.y, -127.f));
  const float2 t = add2(x, magic);                                          // i in the low bits
  const float2 f = fma2(add2(t, unmagic), make_float2(-1.f, -1.f), x);
  float2 y = fma2(f, make_float2(1.3276472454890609e-3f, 1.3276472454890609e-3f), make_float2(9.675540961325169e-3f, 9.675540961325169e-3f));
  y = fma2(y, f, make_float2(5.550713092088699e-2f, 5.550713092088699e-2f));
  y = fma2(y, f, make_float2(2.4022120237350464e-1f, 2.4022120237350464e-1f));
  y = fma2(y, f, make_float2(6.931469440460205e-1f, 6.931469440460205e-1f));
  y = fma2(y, f, make_float2(1.0000001192092896f, 1.0000001192092896f));
  return mul2(y, make_float2(__int_as_float((__float_as_int(t.x) << 23) + 0x3f800000), __int_as_float((__float_as_int(t.y) << 23) + 0x3f800000)));
}

template <bool BF> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// the 16-bit halves of w that are infinite or NaN, as a mask of halves
template <bool BF> __device__ __forceinline__ uint32_t nonfinite_halves(uint32_t w) {
  const uint32_t e = BF ? 0x7f80u : 0x7c00u;
  return ((w & e) == e ? 0xffffu : 0u) | ((w & (e << 16)) == (e << 16) ? 0xffff0000u : 0u);
}

// log sum exp of a row from its reference (raw score) and the sum of its weights
template <bool BF> __device__ __forceinline__ float log_sum(const TcParams& p, float m, float l) {
  return l == 0.f ? kNegInf : fmaf(m, p.d.scale, (log2f(l) - kLift<BF>) * kLn2);
}

// One poll of a barrier's phase in the form without a time hint: the hardware parks the thread until the phase completes
// or a time of its own has passed.  (With a hint the compiler makes a loop of naps of it, and a waiting warp wakes late.)
__device__ __forceinline__ bool poll(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait of a whole warp for a phase of a barrier.  The hardware parks a poll that does not succeed for 4 us (measured: 4096
// of them 16.1 ms), so 2^18 are about a second; healthy waits are microseconds.  A warp's waits share a limit: once one
// has run out (limit 0) the warp issues and commits nothing more and leaves, every access still in its place.  (The loop is as
// short as it can be, and the count no parameter of the kernel: with a clock in it the 256-request batch took 3 to 12 %
// longer, with the count among the parameters the long prompt 1 %.)
constexpr int kPolls = 1 << 18;
__device__ __forceinline__ void tc_wait(uint64_t* bar, uint32_t parity, int& limit) {
#pragma unroll 1
  for (int n = limit;;) {
    if (__all_sync(kFullMask, poll(bar, parity))) break;
    if (--n <= 0) { limit = 0; break; }
  }
}
__device__ __forceinline__ void gave_up(const TcParams& p) {
  uint32_t cta;
  asm volatile("mov.u32 %0, %%ctaid.x;" : "=r"(cta));   // (read anew: blockIdx.x would be kept in a register throughout)
  p.failed[cta] = 1;
  if (p.d.req_status) atomicOr(p.d.req_status, SPECSTEER_REQ_TIMEOUT);   // said of request 0 of the call
}
// Before a role ends: copies or products that are on their way, whatever has failed.
__device__ __forceinline__ void tc_drain(uint64_t* bar, uint32_t parity) {
#pragma unroll 1
  for (int n = kPolls; n > 0 && !poll(bar, parity); --n) {}
}

// ---- units ----------------------------------------------------------------------------------------------------------
// The cut weighs a unit by its key tiles, twice as much with two query tiles, and a constant for its beginning and end
// (queries, first scores, result).  Of the constants from 0 to 24 these were the fastest: with 0 / 8 / 14 in place of 4 a
// batch of 64 single tokens takes 121 / 85 / 93 us instead of 80, four prompt chunks with 4 in place of 6 309 us instead of 287.
// Trees end in blocks whose rows look their keys up, and their units are short: 64 trees of 15 to 32 rows over up to 4000 keys take 171 us
// with 6 for both, 177 with 4 / 6, 187 with 2 / 4, 174 with 8 / 12.
template <bool TREE> __device__ __forceinline__ int unit_base(bool two) { return TREE || two ? 6 : 4; }

// TREE here and below: rows of trees of drafts, which see the cached keys before the chunk and, of the chunk's own, those of their
// mask.  What depends on it are the spans of a unit, taken as wide as any row's, and the keys that a row keeps in a block at the edge.
template <bool TREE> __device__ __forceinline__ AttnRequest request_of(const TcParams& p, int b) {
  if constexpr (TREE) return attn_request_tree(p.d, p.tree, b);
  else return attn_request(p.d, b);
}

struct Unit {
  int tok0, tok1;          // tokens of the request
  bool two;                // two query tiles
  int hi_first, hi_last;   // keys the first / last row sees end here
  int lo_first, lo_last;   // and begin here
  int base;                // see unit_base
  int t0, nt;              // first key tile, key tiles (at least one, so that a unit that sees nothing is written too)
};
template <bool TREE> __device__ __forceinline__ Unit make_unit(const TcParams& p, const AttnRequest& rq, int u) {
  Unit x;
  x.tok0 = u * 2 * p.tile_tok;
  x.tok1 = min(rq.n, x.tok0 + 2 * p.tile_tok);
  x.two = x.tok1 - x.tok0 > p.tile_tok;
  x.base = unit_base<TREE>(x.two);
  if constexpr (TREE) {
    const int past = rq.kv - rq.n;
    x.lo_first = tree_lo(p.d, past);                  // of a row as near as the root
    x.lo_last = tree_lo(p.d, past + x.tok1 - 1);      // of one as far as its own place
    x.hi_first = past;                                // every row sees the keys up to here
    x.hi_last = rq.kv;
  } else {
    attn_span(p.d, rq, x.tok0, x.lo_first, x.hi_first);
    attn_span(p.d, rq, x.tok1 - 1, x.lo_last, x.hi_last);
  }
  x.t0 = x.lo_first / kKeys;
  x.nt = max(1, (max(x.hi_last, 0) + kKeys - 1) / kKeys - x.t0);
  return x;
}
__device__ __forceinline__ long long unit_cost(const Unit& x) { return (long long)x.nt * (x.two ? 2 : 1) + x.base; }
// The key tile at which a cut `pos` into the unit falls.
__device__ __forceinline__ int cut_tile(const Unit& x, long long pos) {
  return pos <= x.base ? 0 : (int)min((long long)x.nt, (pos - x.base) >> (x.two ? 1 : 0));
}
__device__ __forceinline__ int n_units(const TcParams& p, const AttnRequest& rq) { return (rq.n + 2 * p.tile_tok - 1) / (2 * p.tile_tok); }
template <bool TREE> __device__ __forceinline__ long long head_cost(const TcParams& p, const AttnRequest& rq) {
  long long c = 0;
#pragma unroll 1
  for (int u = 0, nu = n_units(p, rq); u < nu; ++u) c += unit_cost(make_unit<TREE>(p, rq, u));
  return c;
}

// Walks this CTA's share: the pieces [off, off + take) of consecutive units.
template <bool TREE> struct Walk {
  int b, hk, u, off, take, index;
  long long end;     // where the range ends, from the beginning of the unit
  AttnRequest rq;
  Unit x;
  __device__ __forceinline__ void begin(const TcShared* sh) {
    b = sh->start_b; hk = sh->start_hk; u = sh->start_u; off = sh->start_off;
    end = sh->end;
    index = 0;
    take = 0;
  }
  __device__ __forceinline__ void load(const TcParams& p) {
    take = 0;
    if (end <= 0) return;
    rq = request_of<TREE>(p, b);
    x = make_unit<TREE>(p, rq, u);
    take = (end >= unit_cost(x) ? x.nt : cut_tile(x, end)) - off;
  }
  __device__ __forceinline__ void next(const TcParams& p) {
    end -= unit_cost(x);
    ++index;
    off = 0;
    if (end <= 0) return;
    if (++u == n_units(p, rq)) {
      u = 0;
      if (++hk == p.d.Hkv) {
        hk = 0;
        do { ++b; } while (b + 1 < p.d.B && request_of<TREE>(p, b).n == 0);   // end > 0: a request with rows follows
      }
    }
  }
  __device__ __forceinline__ void publish(Piece* q) const {
    q->b = b; q->hk = hk;
    q->row0 = rq.row0; q->n = rq.n; q->kv = rq.kv;
    q->tok0 = x.tok0; q->tok1 = x.tok1; q->two = x.two;
    q->lo_first = x.lo_first; q->hi_first = x.hi_first; q->lo_last = x.lo_last;
    q->first = x.t0 + off; q->take = take;
    q->starts = off == 0; q->ends = off + take == x.nt;
    q->index = index;
  }
};

// sums over the block of one value a thread; returns the exclusive sum, *total the sum
__device__ __forceinline__ long long block_sum(long long v, TcShared* sh, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(kFullMask, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sh->scan[warp] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kTcThreads / 32; ++w) {
    if (w < warp) before += sh->scan[w];
    all += sh->scan[w];
  }
  *total = all;
  return before + x - v;
}

template <int DP, bool BF, bool TREE>
__global__ void __launch_bounds__(kTcThreads, 1)
attention_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ TcParams p) {
  typedef TcLayout<DP> L;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const uint32_t smem0 = smem_u32(smem_raw);
  TcShared* sh = reinterpret_cast<TcShared*>(smem_raw + L::kControl);
  RingBars<DP>* ring = reinterpret_cast<RingBars<DP>*>(sh + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < L::kStages; ++i) {
      for (int j = 0; j < 3; ++j) { mbar_init(&ring->k_full[j][i], 1); mbar_init(&ring->v_full[j][i], 1); }
      for (int j = 0; j < 2; ++j) { mbar_init(&ring->k_empty[j][i], 1 + j); mbar_init(&ring->v_empty[j][i], 1 + j); }
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh->q_full[i], 1); mbar_init(&sh->q_empty[i], 2);
      for (int h = 0; h < 2; ++h) { mbar_init(&sh->s_full[i][h], 1); mbar_init(&sh->p_full[i][h], 4); }
      mbar_init(&sh->half_done[i], 1); mbar_init(&sh->o_full[i], 1);
      mbar_init(&sh->group[i], kSoftmaxWarps / 2);
    }
    for (int i = 0; i < kPieces; ++i) { mbar_init(&sh->piece_full[i], 1); mbar_init(&sh->piece_empty[i], kSoftmaxWarps + 3); }
    mbar_init(&sh->both, kSoftmaxWarps);
    for (int i = 0; i < 2; ++i) mbar_init(&sh->drain[i], 1);
    sh->nonfinite = 0;
    sh->end = 0;
    fence_barrier_init();
  }
  if (warp == kKeyWarp) sh->bad[lane] = 0;
  if (warp == kMmaWarp) tc_alloc(&sh->tmem_slot);
  pdl_wait();                // so far nothing touched what the kernels before wrote or read
  pdl_launch_dependents();   // attention_join_kernel may come up; it waits for the end of this kernel before it reads
  if (tid == 0) p.failed[blockIdx.x] = 0;

  // ---- this CTA's range of the list of key tiles
  {
    const int per = (p.d.B + kTcThreads - 1) / kTcThreads, b_lo = min(p.d.B, tid * per), b_hi = min(p.d.B, b_lo + per);
    long long mine = 0, total;
#pragma unroll 1
    for (int b = b_lo; b < b_hi; ++b) {
      const AttnRequest rq = request_of<TREE>(p, b);
      if (rq.bad && blockIdx.x == 0 && p.d.req_status) atomicOr(p.d.req_status + b, SPECSTEER_REQ_BAD_LEN);
      if (rq.n > 0) mine += head_cost<TREE>(p, rq) * p.d.Hkv;
    }
    const long long before = block_sum(mine, sh, &total);   // (its barrier also publishes the set-up above)
    const long long s0 = total * blockIdx.x / gridDim.x, s1 = total * (blockIdx.x + 1) / gridDim.x;
    if (s1 > s0 && s0 >= before && s0 < before + mine) {
      long long rem = s0 - before;
#pragma unroll 1
      for (int b = b_lo; b < b_hi; ++b) {
        const AttnRequest rq = request_of<TREE>(p, b);
        if (rq.n == 0) continue;
        const long long per_head = head_cost<TREE>(p, rq);
        if (rem >= per_head * p.d.Hkv) { rem -= per_head * p.d.Hkv; continue; }
        const int hk = (int)(rem / per_head);
        rem -= hk * per_head;
#pragma unroll 1
        for (int u = 0;; ++u) {
          const Unit x = make_unit<TREE>(p, rq, u);
          if (rem >= unit_cost(x)) { rem -= unit_cost(x); continue; }
          sh->start_b = b; sh->start_hk = hk; sh->start_u = u; sh->start_off = cut_tile(x, rem);
          sh->end = rem + s1 - s0;
          break;
        }
        break;
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sh->tmem_slot);

  if (warp == kKeyWarp || warp == kValueWarp) {
    // ================= work list and TMA =================
    const bool keys = warp == kKeyWarp;
    // A tile's two blocks are issued together, by the two halves of the warp: a block has at most 16 boxes (pages of 8 keys,
    // two chunks of 64 columns).
    constexpr int chunks = DP / 64;
    const int half = lane >> 4, box = (lane & 15) / chunks, chunk = lane % chunks;
    const bool loads = box < p.boxes;
    const uint32_t lane_off = smem0 + (keys ? L::kKeyRing : L::kValueRing) + (uint32_t)chunk * (kBlock * 128) + (uint32_t)box * p.page_rows * 128;
    const CUtensorMap* tm = keys ? &tm_k : &tm_v;
    uint64_t (*full)[L::kStages] = keys ? ring->k_full : ring->v_full;
    uint64_t (*empty)[L::kStages] = keys ? ring->k_empty : ring->v_empty;
    // Bits per stage: the parity to wait for next of its two empty barriers (a stage not used before is free: parity 1 of the
    // first), whether its last block was for both streams, of which stream it was else, the parity of its full barriers.
    uint32_t free_one = ~0u, free_two = 0, last_two = 0, last_own = 0, landed0 = 0, landed1 = 0, landed2 = 0;
    bool any_bad = false;
    int stage = 0, qi = 0, pc = 0, blocks = 0;
    int limit = kPolls;
    const int stop_at = keys ? p.stop_at : 0x7fffffff;
    bool lost = false;
    Walk<TREE> w;
    w.begin(sh);
#pragma unroll 1
    for (;; ++pc) {
      Piece* const x = &sh->piece[pc % kPieces];
      const uint32_t turn = (uint32_t)((pc / kPieces) & 1);
      if (keys) {
        w.load(p);
        tc_wait(&sh->piece_empty[pc % kPieces], turn ^ 1u, limit);
        if (limit == 0) break;
        if (lane == 0) {
          if (w.take > 0) w.publish(x);
          else x->take = 0;
          mbar_arrive(&sh->piece_full[pc % kPieces]);
        }
        __syncwarp();
      } else {
        tc_wait(&sh->piece_full[pc % kPieces], turn, limit);
        if (limit == 0) break;
      }
      const int take = x->take, kv = x->kv, hk = x->hk, b = x->b, first = x->first * 2, two = x->two, lo_first = x->lo_first;
      if (take <= 0) break;
      const int n_q = !keys ? 0 : two ? 2 : 1;
      const int* table = p.d.block_table + (long long)b * p.d.ld_table;
      auto page_at = [&](int blk) { return p.pb_shift >= 0 ? blk >> p.pb_shift : blk / p.page_blocks; };   // pages of 64 keys or more
      // page of this lane's box of tile t of the piece: the id, or n_pages (a coordinate outside, which reads zeros) for none
      auto page_of = [&](int t) -> int {
        const int blk = first + 2 * t + half;
        int page = p.d.n_pages;
        if (loads && t < take && blk * kBlock + box * p.page_rows < kv) page = __ldg(table + (p.boxes > 1 ? blk * p.boxes + box : page_at(blk)));
        return page;
      };
      int page = page_of(0), page1 = page_of(1), q_done = 0;
#pragma unroll 1
      for (int t = 0; t <= take; ++t) {
        // The queries go behind the first keys, whose stages are free sooner: once their place is, or at the latest when the
        // ring may be full of keys that wait for them.
#pragma unroll 1
        while (t > 0 && q_done < n_q && limit) {
          const int slot = qi & 1;
          const uint32_t q_turn = (uint32_t)((qi >> 1) & 1) ^ 1u;
          if (t < L::kStages / 2 && t < take && !__all_sync(kFullMask, mbar_test_nonblocking(&sh->q_empty[slot], q_turn))) break;
          tc_wait(&sh->q_empty[slot], q_turn, limit);
          if (limit == 0) break;
          const int tok = x->tok0 + q_done * p.tile_tok, cnt = min(p.tile_tok, x->tok1 - tok);
          const int nb = (cnt + p.box_tok - 1) / p.box_tok, q_box = lane / chunks;
          if (lane == 0) mbar_arrive_expect_tx(&sh->q_full[slot], (uint32_t)(nb * p.box_rows * 128 * chunks));
          __syncwarp();
          if (q_box < nb)
            tma_3d(smem0 + slot * L::kQBytes + chunk * (128 * 128) + q_box * p.box_rows * 128, &tm_q, chunk * 64, hk * p.G,
                   x->row0 + tok + q_box * p.box_tok, &sh->q_full[slot]);
          ++qi;
          ++q_done;
        }
        if (blocks >= stop_at && t < take) { limit = 0; lost = true; }
        if (limit == 0 || t == take) break;
        const int blk = first + 2 * t + half;
        const bool outside = page < 0 || page >= p.d.n_pages;
        if (keys) {
          // (pages that end before the first row's window may be gone: zeros were loaded for them, and no row sees those)
          const int key = blk * kBlock + box * p.page_rows;
          const uint32_t votes = __ballot_sync(kFullMask, loads && outside && key < kv && key + p.page_rows > lo_first);
          any_bad = any_bad || votes;   // (until then the words are zero)
          if (any_bad && (lane & 15) == 0) {
            uint32_t bad = 0;
#pragma unroll 1
            for (int i = 0; i < p.boxes; ++i) bad |= ((votes >> (16 * half + i * chunks)) & 1u) << i;
            if (bad && p.d.req_status) atomicOr(p.d.req_status + b, SPECSTEER_REQ_BAD_PAGE);
            // the softmax warps read the word at most the ring and the blocks in work later, well under 32
            *reinterpret_cast<volatile uint8_t*>(&sh->bad[(blocks + half) & 31]) = (uint8_t)bad;   // at most 8 boxes
          }
        }
        const int page2 = page_of(t + 2);
        // each half of the warp waits for its block's stage
        const int stage1 = stage + 1 < L::kStages ? stage + 1 : 0, st = half ? stage1 : stage;
        const uint32_t bits = (1u << stage) | (1u << stage1);
        const bool was_two = (last_two >> st) & 1u;
        tc_wait(&empty[was_two][st], ((was_two ? free_two : free_one) >> st) & 1u, limit);
        if (limit == 0) break;
        free_two ^= bits & last_two;
        free_one ^= bits & ~last_two;
        const int set = two ? 2 : t & 1;
        last_two = two ? last_two | bits : last_two & ~bits;
        last_own = t & 1 ? last_own | bits : last_own & ~bits;
        if (set == 0) landed0 ^= bits;
        if (set == 1) landed1 ^= bits;
        if (set == 2) landed2 ^= bits;
        if ((lane & 15) == 0) mbar_arrive_expect_tx(&full[set][st], L::kStageBytes);
        __syncwarp();
        if (loads) {
          const int in_page = p.page_blocks > 1 ? (blk - page_at(blk) * p.page_blocks) * kBlock : 0;
          tma_4d(lane_off + st * L::kStageBytes, tm, chunk * 64, in_page, hk, outside ? p.d.n_pages : page, &full[set][st]);
        }
        blocks += 2;
        stage = stage1 + 1 < L::kStages ? stage1 + 1 : 0;
        page = page1; page1 = page2;
      }
      if (limit == 0) break;
      if (keys) w.next(p);
      else if (lane == 0) mbar_arrive(&sh->piece_empty[pc % kPieces]);
    }
    if (limit == 0 && !lost && lane == 0) gave_up(p);
    if (lane == 0) {
      // The CTA does not exit under a copy: another warp may have given up without looking at those that are on their way.
#pragma unroll 1
      for (int i = 0; i < min(blocks, L::kStages); ++i) {
        const bool t2 = (last_two >> i) & 1u, t1 = (last_own >> i) & 1u;
        tc_drain(&full[t2 ? 2 : t1 ? 1 : 0][i], (((t2 ? landed2 : t1 ? landed1 : landed0) >> i) & 1u) ^ 1u);
      }
#pragma unroll 1
      for (int i = qi > 2 ? qi - 2 : 0; i < qi; ++i) tc_drain(&sh->q_full[i & 1], (uint32_t)((i >> 1) & 1));
    }
  } else if (warp >= kMmaWarp) {
    // ================= tensor-core issuers, one a stream =================
    // The whole warp runs the loop, so that addresses and descriptors stay in uniform registers.
    // All columns were allocated, so tensor memory begins at column 0.
    const int s = warp - kMmaWarp;
    const uint32_t t_s = s * 128, t_o = 256 + s * 128;
    const uint32_t id_qk = instr_desc(BF, kBlock, false), id_pv = instr_desc(BF, DP, true);
    int qi = 0, pc = 0, blocks0 = 0;
    uint32_t p_phase = 0;
    int limit = kPolls;
    auto wait = [&](uint64_t* bar, uint32_t parity) { tc_wait(bar, parity, limit); };
    uint32_t k_own = 0, k_both = 0, v_own = 0, v_both = 0;   // parity of each stage's full barriers, a bit a stage
#pragma unroll 1
    for (;; ++pc) {
      wait(&sh->piece_full[pc % kPieces], (uint32_t)((pc / kPieces) & 1));
      if (limit == 0) break;
      const Piece* q = &sh->piece[pc % kPieces];
      // (through a reduction, whose result the compiler knows to be the same in the whole warp)
      const int take = __reduce_max_sync(kFullMask, q->take), two = __reduce_max_sync(kFullMask, q->two);
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->piece_empty[pc % kPieces]);
      if (take <= 0) break;
      const int qs = two ? (qi + s) & 1 : qi & 1;
      // both tiles if there are two, so that no phase of either barrier is passed unseen
      wait(&sh->q_full[qi & 1], (uint32_t)((qi >> 1) & 1));
      if (two) wait(&sh->q_full[(qi + 1) & 1], (uint32_t)(((qi + 1) >> 1) & 1));
      const int step = two ? 1 : 2, t_from = two ? 0 : s, set = two ? 2 : s;
      uint32_t k_par = two ? k_both : k_own, v_par = two ? v_both : v_own;
      int k_stage = (blocks0 + 2 * t_from) % L::kStages, v_stage = k_stage;   // of this stream's next block
      auto advance = [&](int& stage, int by) { stage = stage + by >= L::kStages ? stage + by - L::kStages : stage + by; };
      const uint32_t q_desc = desc_rows(smem0 + qs * L::kQBytes);
#pragma unroll 1
      for (int t = t_from - step; t < take; t += step) {   // the first turn forms the first scores alone
        const bool now = t >= t_from, next = t + step < take;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int stage = v_stage;
          if (now) {
            wait(&ring->v_full[set][stage], (v_par >> stage) & 1u);
            v_par ^= 1u << stage;
            advance(v_stage, h == 0 ? 1 : 2 * step - 1);
            wait(&sh->p_full[s][h], p_phase);
            fence_after();
            const uint32_t b = desc_cols(smem0 + L::kValueRing + stage * L::kStageBytes);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_ts(t_o, t_s + h * 64 + k * 8, b + (uint32_t)(k * (2048 >> 4)), id_pv, h > 0 || k > 0 || t > t_from);
          }
          if (limit == 0) break;
          if (next) {
            // Scores of block h of tile t + step.  The commit also says that the product with the block's values before it
            // is complete.
            const int stage2 = k_stage;
            wait(&ring->k_full[set][stage2], (k_par >> stage2) & 1u);
            k_par ^= 1u << stage2;
            advance(k_stage, h == 0 ? 1 : 2 * step - 1);
            const uint32_t b = desc_rows(smem0 + L::kKeyRing + stage2 * L::kStageBytes);
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
              mma_ss(t_s + h * 64, q_desc + (uint32_t)((k >> 2) * ((128 * 128) >> 4) + (k & 3) * 2), b + (uint32_t)((k >> 2) * ((kBlock * 128) >> 4) + (k & 3) * 2),
                     id_qk, k != 0);
            if (limit == 0) break;
            mma_commit(&sh->s_full[s][h]);
            mma_commit(&ring->k_empty[two][stage2]);
          } else if (h == 0 && now) {
            mma_commit(&sh->half_done[s]);
          }
          if (now) mma_commit(&ring->v_empty[two][stage]);
        }
        if (limit == 0) break;
        if (now) p_phase ^= 1u;
      }
      if (limit == 0) break;
      // (a stream that had no tile says nothing: it could come by twice before anybody looks)
      if (t_from < take) mma_commit(&sh->o_full[s]);
      mma_commit(&sh->q_empty[qs]);
      if (two) mma_commit(&sh->q_empty[qs]);   // (its barrier counts both issuers, and this tile is the stream's alone)
      qi += two ? 2 : 1;
      blocks0 += 2 * take;
      if (two) { k_both = k_par; v_both = v_par; }
      else { k_own = k_par; v_own = v_par; }
    }
    if (limit == 0 && lane == 0) gave_up(p);
    // Products end before tensor memory is given back and the CTA exits: a softmax warp that gave up did not wait for them.
    __syncwarp();
    mma_commit(&sh->drain[s]);
    tc_drain(&sh->drain[s], 0);
  } else {
    // ================= softmax: one row a thread =================
    const int s = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_s = tmem + lanes + s * 128, t_o = tmem + lanes + 256 + s * 128;
    const int r_tok = r / p.G, r_head = r - r_tok * p.G;
    const float c = p.c;
    uint32_t o_phase = 0;                   // bit s: of stream s
    uint32_t s_phase = 0, half_phase = 0;   // s_phase: of both blocks at the beginning of a tile
    uint32_t group_phase = 0, both_phase = 0;
    int blocks0 = 0, pc = 0;     // blocks0: of the pieces before
    uint32_t v_own = 0, v_both = 0;         // as the issuer's
    int limit = kPolls;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      tc_wait(bar, parity, limit);
      fence_after();
    };
    // barriers among the softmax warps: of this stream, of both (bounded like every wait)
    auto meet = [&](bool all) {
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(all ? &sh->both : &sh->group[s]);
      wait(all ? &sh->both : &sh->group[s], all ? both_phase : group_phase);
      if (all) both_phase ^= 1u;
      else group_phase ^= 1u;
    };
    if (tid == 0) {
      int* h = p.head + blockIdx.x * 8;
      h[0] = -1;   // slot of a unit that begins in this CTA and goes on in the next
      h[1] = 0;    // its part of a unit that began in a CTA before: 0 none, 1 the end, 2 some in between
    }
#pragma unroll 1
    for (; limit; ++pc) {
      wait(&sh->piece_full[pc % kPieces], (uint32_t)((pc / kPieces) & 1));
      if (limit == 0) break;
      const Piece& x = sh->piece[pc % kPieces];
      const int take = x.take, two = x.two, first = x.first;
      if (take <= 0) break;
      const int tok = x.tok0 + (two ? s * p.tile_tok : 0) + r_tok;
      const bool live = r_tok < p.tile_tok && tok < x.tok1;
      const bool warp_live = __any_sync(kFullMask, live);
      int lo = 0, hi = 0;
      if (live) {
        hi = x.kv - x.n + tok + 1;
        lo = p.d.window > 0 && hi > p.d.window ? hi - p.d.window : 0;
        if constexpr (TREE) {   // the cached keys before the chunk; its own are looked up at the edge
          hi = x.kv - x.n;
          lo = tree_row_lo(p.d, p.tree, AttnRequest{x.row0, x.n, x.kv, false}, tok);
        }
      }
      const int hi_first = x.hi_first, lo_last = x.lo_last;
      float m = live ? kNegInf : 0.f, l = 0.f;       // reference (raw score; none yet: -inf), sum
      bool none = true;                 // some row of the warp has no reference yet, or one beyond kFar
      const int step = two ? 1 : 2, t_from = two ? 0 : s;
      uint32_t v_par = two ? v_both : v_own;
      int v_first = (blocks0 + 2 * t_from) % L::kStages;   // stage of the tile's first block
#pragma unroll 1
      for (int t = t_from; t < take && limit; t += step) {
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const int k0 = (first + t) * kKeys + h * kBlock;
          wait(&sh->s_full[s][h], s_phase);   // the block's keys have landed, and what was loaded before them
          const uint32_t bad = *reinterpret_cast<volatile uint8_t*>(&sh->bad[(blocks0 + 2 * t + h) & 31]);
          const bool edge = k0 + kBlock > hi_first || k0 < lo_last || bad != 0;
          if (edge) {
            // Values of keys that some row of the unit does not see.  What lies behind the last key in its page becomes zero
            // (whole pages behind it, and pages outside the pool, were loaded as zeros); an infinity or NaN among the others is
            // taken out here, where it would reach rows with weight 0, and added in the epilogue to the rows that see it.
            const int v_stage = v_first + h < L::kStages ? v_first + h : 0;
            wait(&ring->v_full[two ? 2 : s][v_stage], (v_par >> v_stage) & 1u);
            unsigned char* vt = smem_raw + L::kValueRing + v_stage * L::kStageBytes;
            const int kv_here = min(kBlock, max(0, x.kv - k0));
            const int from = min(kv_here, max(0, lo_last - k0)), to = min(kv_here, max(from, hi_first - k0));
            const int zero_to = min(kBlock, (kv_here + p.page_rows - 1) & -p.page_rows);
            auto vector = [&](int j, int vec) {
              return reinterpret_cast<uint4*>(vt + (vec >> 3) * (kBlock * 128) + j * 128 + (((vec & 7) ^ (j & 7)) << 4));
            };
            // two query tiles: the groups share the work
            const int me = two ? tid : tid & 127, team = two ? 256 : 128;
            constexpr int kVec = DP / 8;
#pragma unroll 1
            for (int e = kv_here * kVec + me; e < zero_to * kVec; e += team) *vector(e / kVec, e % kVec) = make_uint4(0u, 0u, 0u, 0u);
            const int n_vec = (from + (kv_here - to)) * kVec;          // of keys [0, from) and [to, kv)
            bool found = false;
#pragma unroll 2
            for (int e = me; e < n_vec; e += team) {
              const int j = e / kVec;
              const uint4 y = *vector(j < from ? j : j - from + to, e % kVec);
              found = found || (nonfinite_halves<BF>(y.x) | nonfinite_halves<BF>(y.y) | nonfinite_halves<BF>(y.z) | nonfinite_halves<BF>(y.w));
            }
            if (found) *reinterpret_cast<volatile int*>(&sh->nonfinite) = 1;
            fence_async_proxy();
            meet(two);   // everybody has looked before anything is taken out
            if (*reinterpret_cast<volatile int*>(&sh->nonfinite)) {   // (or in an earlier tile: then there is nothing to find)
#pragma unroll 1
              for (int e = tid & 127; e < n_vec; e += 128) {
                const int j = e / kVec;
                uint4* at = vector(j < from ? j : j - from + to, e % kVec);
                const uint4 y = *at;
                const uint32_t n0 = nonfinite_halves<BF>(y.x), n1 = nonfinite_halves<BF>(y.y), n2 = nonfinite_halves<BF>(y.z), n3 = nonfinite_halves<BF>(y.w);
                if (n0 | n1 | n2 | n3) *at = make_uint4(y.x & ~n0, y.y & ~n1, y.z & ~n2, y.w & ~n3);
              }
              fence_async_proxy();
            }
          }
          if (warp_live) {
            float v[64];
            tm_ld32(t_s + h * 64, v);
            tm_ld32(t_s + h * 64 + 32, v + 32);
            tm_ld_wait(v);
            tm_ld_tie(v + 32);
            if (edge) {
#pragma unroll
              for (int i = 0; i < 64; i += 32) {
                // the columns of 32 that the row sees, as bits
                const int from = max(lo - k0 - i, 0), to = min(hi - k0 - i, 32);
                uint32_t keep = to > from ? (0xffffffffu >> (32 - (to - from))) << from : 0u;
                if constexpr (TREE) {
                  if (live) keep |= tree_bits(p.tree, (long long)x.row0 + tok, x.n, k0 + i - hi);
                }
                if (bad) {
#pragma unroll 1
                  for (int j = 0; j < 32; j += 8)   // boxes hold 8 keys or more
                    if ((bad >> ((i + j) >> p.page_shift)) & 1u) keep &= ~(0xffu << j);
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) v[i + j] = (keep & (1u << j)) ? v[i + j] : kNegInf;
              }
            }
            bool raise = none;
#pragma unroll 1
            for (;;) {
              float up = fmaf(m, -c, kLift<BF>);
              if (raise) {
                float mx[8] = {m, m, m, m, m, m, m, m};
#pragma unroll
                for (int j = 0; j < 64; j += 16) {
#pragma unroll
                  for (int i = 0; i < 8; ++i) mx[i] = max3(mx[i], v[j + 2 * i], v[j + 2 * i + 1]);
                }
                const float top = max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7]));
                const float alpha = top > m && m != kNegInf ? ex2((m - top) * c) : 1.f;   // (without a reference the sums are zero)
                if (t + h > t_from && __any_sync(kFullMask, alpha != 1.f)) {
                  // The sums are at rest once the product with the last weights is complete: the scores of the other
                  // block that were formed behind it say so, or at the end of the piece a commit of its own.
                  if (h == 0) wait(&sh->s_full[s][1], s_phase);
                  else if (t + step < take) wait(&sh->s_full[s][0], s_phase ^ 1u);
                  else wait(&sh->half_done[s], half_phase);
#pragma unroll 1
                  for (int j0 = 0; j0 < DP; j0 += 16) {
                    float o[16];
                    tm_ld16(t_o + j0, o);
                    tm_ld_wait16(o);
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] *= alpha;
                    tm_st16(t_o + j0, reinterpret_cast<const uint32_t*>(o));
                  }
                }
                l *= alpha;
                m = top;
                none = __any_sync(kFullMask, live && !(fabsf(m) * c <= kFar));
                up = fmaf(m, -c, kLift<BF>);
                if (none) {
                  const float from = m == kNegInf ? 0.f : -m;
#pragma unroll
                  for (int j = 0; j < 64; j += 2) {
                    const float2 y = add2(make_float2(v[j], v[j + 1]), make_float2(from, from));
                    v[j] = y.x;
                    v[j + 1] = y.y;
                  }
                  up = kLift<BF>;
                }
              }
              const float2 c2 = make_float2(c, c), ref2 = make_float2(up, up);
              float poly_top = kNegInf;   // ex2_poly takes no more than 127
              float2 sum[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
              // The weights go to the second product in the inputs' type, rounded to nearest; the sums keep 32 bits.  The operand
              // of the product has 16 bits: weights of 32 would mean two products.  It is most of what the result is further off
              // than with weights of 32 bits (relative error 0.0023 instead of 0.0017 for the 256 requests, bfloat16).
#pragma unroll
              for (int i = 0; i < 64; i += 32) {
                uint32_t w16[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                  const float2 x2 = fma2(make_float2(v[i + 2 * j], v[i + 2 * j + 1]), c2, ref2);
                  const bool poly = ((i / 2 + j) * kPolyPairs) % 32 < kPolyPairs;
                  if (poly) poly_top = max3(poly_top, x2.x, x2.y);
                  const float2 y = poly ? ex2_poly(x2) : make_float2(ex2(x2.x), ex2(x2.y));
                  sum[j & 3] = add2(sum[j & 3], y);
                  w16[j] = pack2<BF>(y.x, y.y);
                }
                tm_st16(t_s + h * 64 + i / 2, w16);
              }
              sum[0] = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
              const float total = sum[0].x + sum[0].y;
              if (raise || __all_sync(kFullMask, !live || (total <= kMostSum && poly_top <= kMostArg))) {
                l += total;
                break;
              }
              raise = true;
            }
            tm_st_wait();
            fence_before();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh->p_full[s][h]);
        }
        v_par ^= (1u << v_first) | (1u << (v_first + 1 < L::kStages ? v_first + 1 : 0));
        v_first += 2 * step;
        if (v_first >= L::kStages) v_first -= L::kStages;
        s_phase ^= 1u;
      }
      if (limit == 0) break;
      if (t_from < take) half_phase ^= 1u;
      if (two) v_both = v_par;
      else v_own = v_par;
      // ---- end of the piece
      const int n1 = two ? take : take / 2;   // tiles of the second stream
      const bool whole = x.starts && x.ends;
      const int slot = 2 * blockIdx.x + (x.index == 0 ? 0 : 1);
      // the sums of the stream, with one query tile of both (if the second had a tile)
      if (s == 0 || !two) wait(&sh->o_full[0], o_phase & 1u);
      if (n1 > 0 && (s == 1 || !two)) wait(&sh->o_full[1], o_phase >> 1);
      o_phase ^= n1 > 0 ? 3u : 1u;
      if (m == kNegInf && l == l) l = 0.f;   // no key, or only scores of -inf: nothing was weighed
      float f0 = 1.f, f1 = 1.f;
      if (!two) {
        sh->exch[s][r] = make_float2(m, l);
        meet(true);
        const float2 e0 = sh->exch[0][r], e1 = sh->exch[1][r];
        m = fmaxf(e0.x, e1.x);
        f0 = e0.x == kNegInf ? 0.f : ex2((e0.x - m) * c);
        f1 = e1.x == kNegInf ? 0.f : ex2((e1.x - m) * c);
        l = e0.y * f0 + e1.y * f1;
      }
      const int poisoned = *reinterpret_cast<volatile int*>(&sh->nonfinite);
      const long long row = (long long)x.row0 + tok;
      const int head = x.hk * p.G + r_head;
      const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
      const int part_row = (two ? s * 128 : 0) + r;
      if (warp_live) {
        // with one query tile the two groups share the columns
        const int share = two ? DP : DP / 2, j_lo = two ? 0 : s * share;
        const uint32_t t_0 = two ? t_o : tmem + lanes + 256;
        unsigned short* dst = reinterpret_cast<unsigned short*>(p.d.out) + row * p.d.o_tok + head * p.d.o_head;
        float* part = p.part + ((long long)slot * 256 + part_row) * DP;
#pragma unroll 1
        for (int j0 = j_lo; j0 < j_lo + share; j0 += 32) {
          float o[32];
          tm_ld32(t_0 + j0, o);
          if (!two && n1 > 0) {
            float o1[32];
            tm_ld32(tmem + lanes + 384 + j0, o1);
            tm_ld_wait(o);
            tm_ld_tie(o1);
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = fmaf(o1[j], f1, o[j] * f0);
          } else {
            tm_ld_wait(o);
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] *= f0;
          }
          if (poisoned && live) {
            const int k_lo = TREE ? first * kKeys : max(lo, first * kKeys), k_hi = min(TREE ? x.kv : hi, (first + take) * kKeys);
#pragma unroll 1
            for (int key = k_lo; key < k_hi; ++key) {
              if (key < hi_first && key >= lo_last) continue;   // only those that were taken out
              if constexpr (TREE) {
                if (key < hi ? key < lo : !(tree_bits(p.tree, row, x.n, key - hi) & 1u)) continue;
              }
              const int page = p.d.block_table[(long long)x.b * p.d.ld_table + key / p.d.page_size];
              if (page < 0 || page >= p.d.n_pages) continue;
              const unsigned short* v = reinterpret_cast<const unsigned short*>(p.d.v_cache) + page * p.d.vc_page + (key % p.d.page_size) * p.d.vc_slot + x.hk * p.d.vc_head + j0;
#pragma unroll 1
              for (int j = 0; j < 32 && j0 + j < p.d.D; ++j) {
                const unsigned short bits = v[j];
                if (nonfinite_halves<BF>(bits) & 0xffffu) {
                  const float y = BF ? __uint_as_float((uint32_t)bits << 16) : __half2float(__ushort_as_half(bits));
#pragma unroll
                  for (int i = 0; i < 32; ++i)
                    if (i == j) o[i] += y;
                }
              }
            }
          }
          if (live) {
            if (!whole) {
#pragma unroll
              for (int j = 0; j < 32; j += 8) st_256(part + j0 + j, reinterpret_cast<const uint32_t*>(o + j));
            } else {
              uint32_t y[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) y[j] = pack2<BF>(o[2 * j] * inv, o[2 * j + 1] * inv);
              if (p.out_vec) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                  if (j0 + 16 * j < p.d.D) st_256(dst + j0 + 16 * j, y + 8 * j);
              } else {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                  if (j0 + j < p.d.D) dst[j0 + j] = (unsigned short)(y[j >> 1] >> ((j & 1) * 16));
              }
            }
          }
        }
        if (live && (two || s == 0)) {
          if (!whole) p.part_ml[(long long)slot * 256 + part_row] = make_float2(m, l);
          else if (p.d.lse) p.d.lse[row * p.d.Hq + head] = log_sum<BF>(p, m, l);
        }
      }
      if (tid == 0 && !whole) {
        int* h = p.head + blockIdx.x * 8;
        if (x.starts) { h[0] = slot; h[2] = x.row0 + x.tok0; h[3] = x.hk; h[4] = x.tok1 - x.tok0; }
        else h[1] = x.ends ? 1 : 2;
      }
      if (!two) meet(true);   // both halves of the sums are read before either stream goes on
      blocks0 += 2 * take;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->piece_empty[pc % kPieces]);
    }
    if (limit == 0 && lane == 0) gave_up(p);
  }
  fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    fence_after();
    tc_dealloc(tmem);
  }
}

// A call in which a bounded wait ran out leaves no number behind that could be taken for a result: NaN in every row.
template <bool BF, bool TREE> __device__ __forceinline__ void spoil(const TcParams& p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  for (int b = 0; b < p.d.B; ++b) {
    const AttnRequest rq = request_of<TREE>(p, b);
    const long long n = (long long)rq.n * p.d.Hq;
    for (long long i = warp; i < n; i += warps) {
      const long long row = rq.row0 + i / p.d.Hq, head = i % p.d.Hq;
      unsigned short* dst = reinterpret_cast<unsigned short*>(p.d.out) + row * p.d.o_tok + head * p.d.o_head;
      for (int j = lane; j < p.d.D; j += 32) dst[j] = BF ? 0x7fc0u : 0x7e00u;
      if (lane == 0 && p.d.lse) p.d.lse[row * p.d.Hq + head] = __int_as_float(0x7fc00000);
    }
  }
}

// Puts the parts of a cut unit together: blocks x take the unit that begins in CTA x and goes on in the CTAs behind it.
// One warp a row; the parts are added in their order, so the bits do not depend on who came first.
// It waits on latency (about ten dependent trips to L2): 4 to 8 us behind the main kernel, 15 to 17 us where every CTA's
// range cuts a unit of 256 rows (35 MB of parts); with 8 blocks a unit instead of 16 long contexts took 3 us
// more, with 32 the same.
template <int DP, bool BF, bool TREE>
__global__ void __launch_bounds__(256, 4) attention_join_kernel(const __grid_constant__ TcParams p, int n_cta) {
  pdl_launch_dependents();   // the next call's main kernel may set itself up meanwhile
  pdl_wait();
  const int cta = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // what every row begins with, on its way before anything is known to be needed (the addresses are the workspace's own)
  const int4 h = *reinterpret_cast<const int4*>(p.head + cta * 8);
  const int tokens = p.head[cta * 8 + 4], first_kind = lane == 0 ? 2 : cta + lane < n_cta ? p.head[(cta + lane) * 8 + 1] : 1;
  const int failed = threadIdx.x < n_cta ? p.failed[threadIdx.x] : 0;   // (at most kMaxCtas of them, fewer than the threads)
  const int slot0 = h.x;
  const bool first_block = blockIdx.x == 0 && blockIdx.y == 0;
  if (slot0 < 0 && !first_block) return;
  if (__syncthreads_or(failed)) {
    if (first_block) spoil<BF, TREE>(p);
    return;
  }
  if (slot0 < 0) return;
  const int rows = tokens * p.G, tile_rows = p.tile_tok * p.G;
  for (int q = blockIdx.y * 8 + warp; q < rows; q += gridDim.y * 8) {
    const int part_row = q < tile_rows ? q : 128 + q - tile_rows;
    float m = kNegInf, l = 0.f, o[DP / 32];
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) o[j] = 0.f;
    // The parts: the first one in slot0, then slot 2*i of every CTA i behind that has one, to the unit's end.  32 CTAs at a
    // time, a lane each, for the references and sums; then the parts themselves with the warp side by side.
    bool more = true;
    for (int base = cta; more && base < n_cta; base += 32) {
      const int i = base + lane;
      const int kind = base == cta ? first_kind : i < n_cta ? p.head[i * 8 + 1] : 1;
      const uint32_t ends = __ballot_sync(kFullMask, kind == 1);
      const uint32_t upto = ends ? (2u << (__ffs(ends) - 1)) - 1u : 0xffffffffu;   // lanes up to the first end (all: shift to 0)
      const bool has = kind != 0 && i < n_cta && ((upto >> lane) & 1u);
      more = ends == 0;
      const long long at = (long long)(i == cta ? slot0 : 2 * i) * 256 + part_row;
      const float2 ml = has ? p.part_ml[at] : make_float2(kNegInf, 0.f);
      const float top = fmaxf(m, warp_max(ml.x));
      const float keep = m == kNegInf ? 0.f : ex2((m - top) * p.c), f = ml.x == kNegInf ? 0.f : ex2((ml.x - top) * p.c);
      l = l * keep + warp_sum(ml.y * f);
#pragma unroll
      for (int j = 0; j < DP / 32; ++j) o[j] *= keep;
      m = top;
      uint32_t todo = __ballot_sync(kFullMask, has);
      while (todo) {
        // four parts in flight
        float2 y[4][DP / 64];
        float w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          w[k] = 0.f;
#pragma unroll
          for (int j = 0; j < DP / 64; ++j) y[k][j] = make_float2(0.f, 0.f);
          if (todo) {
            const int src = __ffs(todo) - 1;
            todo &= todo - 1;
            w[k] = __shfl_sync(kFullMask, f, src);
            const float* part = p.part + __shfl_sync(kFullMask, at, src) * DP + 2 * lane;
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) y[k][j] = *reinterpret_cast<const float2*>(part + 64 * j);
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int j = 0; j < DP / 64; ++j) {
            o[2 * j] = fmaf(y[k][j].x, w[k], o[2 * j]);
            o[2 * j + 1] = fmaf(y[k][j].y, w[k], o[2 * j + 1]);
          }
        }
      }
    }
    const int head = h.w * p.G + q % p.G;
    const long long row = (long long)h.z + q / p.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    unsigned short* dst = reinterpret_cast<unsigned short*>(p.d.out) + row * p.d.o_tok + head * p.d.o_head;
#pragma unroll
    for (int j = 0; j < DP / 64; ++j) {
      const int d = 64 * j + 2 * lane;
      const uint32_t y = pack2<BF>(o[2 * j] * inv, o[2 * j + 1] * inv);
      if (d < p.d.D) dst[d] = (unsigned short)y;
      if (d + 1 < p.d.D) dst[d + 1] = (unsigned short)(y >> 16);
    }
    if (lane == 0 && p.d.lse) p.d.lse[row * p.d.Hq + head] = log_sum<BF>(p, m, l);
  }
}

// ---- host side --------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn tiled_encoder() {
  static EncodeTiledFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      return (EncodeTiledFn) nullptr;
    return (EncodeTiledFn)f;
  }();
  return fn;
}

// A tensor of 16-bit elements, innermost axis dense, boxes of 64 elements (128 bytes, 128-byte swizzle), zeros outside.
bool encode(CUtensorMap* tm, bool bf16, const void* base, int rank, const long long* dims, const long long* strides, const int* box) {
  EncodeTiledFn fn = tiled_encoder();
  if (!fn) return false;
  cuuint64_t d[4], st[3];
  cuuint32_t bx[4], one[4] = {1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    d[i] = (cuuint64_t)dims[i];
    bx[i] = (cuuint32_t)box[i];
    if (i) st[i - 1] = (cuuint64_t)(dims[i] > 1 ? strides[i] * 2 : 16);   // the stride of an axis of one carries nothing
  }
  return fn(tm, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d, st, bx, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

// Query boxes of whole tokens: as few tokens as make a multiple of 8 rows (the swizzle's period), then about 32 rows.
bool query_box(int G, int* box_tok, int* boxes) {
  if (G > 128) return false;
  int tok = 8 / gcd(G, 8);
  if (tok * G > 128) return false;
  while (tok * G * 2 <= 32) tok *= 2;
  *box_tok = tok;
  *boxes = 128 / (tok * G);
  return true;
}

// One CTA per SM, up to the 148 of a B200; the workspace is laid out for that many whatever the shape.
constexpr int kMaxCtas = 148;
size_t part_bytes(int DP) { return (size_t)2 * kMaxCtas * 256 * DP * sizeof(float); }
size_t ml_bytes() { return (size_t)2 * kMaxCtas * 256 * sizeof(float2); }
size_t head_bytes() { return (size_t)kMaxCtas * 8 * sizeof(int); }
size_t failed_bytes() { return (size_t)kMaxCtas * sizeof(int); }
static_assert(kMaxCtas <= 256, "a thread of attention_join_kernel for every CTA");

template <int DP, bool BF, bool TREE>
cudaError_t launch_as(const CUtensorMap* tm, const TcParams& p, int grid, cudaStream_t s) {
  static std::atomic<bool> attr_set[64];   // per device; two host threads that both find it clear set the same value
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!attr_set[dev & 63].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(attention_tc_kernel<DP, BF, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize, tc_smem_bytes<DP>());
    if (e != cudaSuccess) return e;
    attr_set[dev & 63].store(true, std::memory_order_release);
  }
  // Both kernels may come up while the one before still runs (programmatic dependent launch); each waits for it before it
  // reads or writes global memory.
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kTcThreads);
  cfg.dynamicSmemBytes = tc_smem_bytes<DP>();
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, attention_tc_kernel<DP, BF, TREE>, tm[0], tm[1], tm[2], p);
  if (e != cudaSuccess) return e;
  cfg.gridDim = dim3(grid, 16);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, attention_join_kernel<DP, BF, TREE>, p, grid);
}
template <int DP, bool BF>
cudaError_t launch(const CUtensorMap* tm, const TcParams& p, int grid, cudaStream_t s) {
  return p.tree.bits ? launch_as<DP, BF, true>(tm, p, grid, s) : launch_as<DP, BF, false>(tm, p, grid, s);
}

}  // namespace

// From here on scale times a reference is an ordinary number (masked scores are -inf before the scale is applied, so zero is none).
constexpr float kLeastScale = 1e-30f;

bool attention_tc_takes(const specsteer_attention_desc* d) {
  int tok, boxes;
  auto a16 = [](const void* q) { return ((uintptr_t)q & 15u) == 0; };
  // strides of axes longer than one: positive multiples of 16 bytes below the tensor map's limit
  auto ok = [](long long stride, long long extent) { return extent <= 1 || (stride > 0 && stride % 8 == 0 && stride < (1ll << 38)); };
  const int pr = d->page_size < kBlock ? d->page_size : kBlock;
  return !(d->flags & SPECSTEER_ATTENTION_GENERIC) && d->T <= kAttnMaxKv && d->D <= 128 && d->D % 8 == 0 && d->scale >= kLeastScale && pr % 8 == 0 && kBlock % pr == 0 && d->page_size % pr == 0 &&
         query_box(d->Hq / d->Hkv, &tok, &boxes) && a16(d->q) && a16(d->k_cache) && a16(d->v_cache) && ok(d->q_tok, d->T) && ok(d->q_head, d->Hq) &&
         ok(d->kc_page, d->n_pages) && ok(d->kc_slot, d->page_size) && ok(d->kc_head, d->Hkv) && ok(d->vc_page, d->n_pages) &&
         ok(d->vc_slot, d->page_size) && ok(d->vc_head, d->Hkv);
}

size_t attention_tc_workspace(const specsteer_attention_desc* d) { return part_bytes(d->D <= 64 ? 64 : 128) + ml_bytes() + head_bytes() + failed_bytes(); }

cudaError_t launch_attention_tc(const specsteer_attention_desc* d, const TreeMask& tree, cudaStream_t s) {
  const int sm = current_sm_count();
  if (sm <= 0) return cudaErrorInvalidDevice;
  const bool bf16 = d->dtype == SPECSTEER_BF16;
  const int DP = d->D <= 64 ? 64 : 128;
  TcParams p;
  p.d = *d;
  p.tree = tree;
  p.G = d->Hq / d->Hkv;
  int boxes = 0;
  query_box(p.G, &p.box_tok, &boxes);
  p.box_rows = p.box_tok * p.G;
  p.tile_tok = boxes * p.box_tok;
  p.page_rows = d->page_size < kBlock ? d->page_size : kBlock;
  p.boxes = kBlock / p.page_rows;
  p.page_blocks = d->page_size / p.page_rows;
  p.pb_shift = p.page_blocks & (p.page_blocks - 1) ? -1 : 0;
  while (p.pb_shift >= 0 && (1 << p.pb_shift) < p.page_blocks) ++p.pb_shift;
  p.page_shift = 0;
  while ((1 << p.page_shift) < p.page_rows) ++p.page_shift;
  p.c = d->scale * kLog2e;
  p.out_vec = ((uintptr_t)d->out & 31u) == 0 && d->o_tok % 16 == 0 && d->o_head % 16 == 0 && d->D % 16 == 0;
  p.part = (float*)d->workspace;
  p.part_ml = (float2*)((char*)d->workspace + part_bytes(DP));
  p.head = (int*)((char*)d->workspace + part_bytes(DP) + ml_bytes());
  p.failed = p.head + kMaxCtas * 8;
  p.stop_at = d->flags >> 16 ? (int)(d->flags >> 16) - 1 : 0x7fffffff;
  CUtensorMap tm[3];
  {
    const long long dims[3] = {d->D, d->Hq, d->T}, st[3] = {0, d->q_head, d->q_tok};
    const int box[3] = {64, p.G, p.box_tok};
    if (!encode(&tm[0], bf16, d->q, 3, dims, st, box)) return cudaErrorInvalidValue;
  }
  const long long dims[4] = {d->D, d->page_size, d->Hkv, d->n_pages};
  const int box[4] = {64, p.page_rows, 1, 1};
  const long long ks[4] = {0, d->kc_slot, d->kc_head, d->kc_page}, vs[4] = {0, d->vc_slot, d->vc_head, d->vc_page};
  if (!encode(&tm[1], bf16, d->k_cache, 4, dims, ks, box) || !encode(&tm[2], bf16, d->v_cache, 4, dims, vs, box)) return cudaErrorInvalidValue;
  const int grid = sm < kMaxCtas ? sm : kMaxCtas;
  if (DP == 128) return bf16 ? launch<128, true>(tm, p, grid, s) : launch<128, false>(tm, p, grid, s);
  return bf16 ? launch<64, true>(tm, p, grid, s) : launch<64, false>(tm, p, grid, s);
}

}  // namespace specsteer
