// Attention of many new tokens per sequence (a prompt, a part of one, draft tokens) over everything cached, on the
// fifth-generation tensor cores.
//
// A token at position u - 1 sees positions i < u that are among the first `sinks` or not before
// P(u) = max(0, u - window, floor(c u)).  Its G heads of a KV head are G rows; T = 128 / G tokens (rounded down) fill the 128 rows of an
// MMA.  A CTA works on an item, 2 T tokens of a sequence and one KV head, as two subtiles of T tokens with an
// accumulator each, over tiles of 128 keys:
//   producer warp   finds this CTA's pieces of work and tells the others; Q once per piece, then K and V tiles by TMA (128-byte swizzle)
//                   into a ring of 32 KB slots
//   MMA warp        S = Q K^T (128 x 128, fp32 in tensor memory) and O += P V for the subtiles in turn, P read from tensor memory
//   8 softmax warps a thread owns a row of a subtile: reads it (tcgen05.ld), weights 2^(x - m) in bf16 back over S (tcgen05.st), their
//                   sum in fp32.  While the tensor core multiplies for one subtile, the other's weights are made
//   2 mending warps tiles that some row sees in part only: V rows behind the sequence become zero, and so do values that are not
//                   finite (noted, and added at the end for the rows that do see them): a weight of zero times an infinity in
//                   a masked place would be NaN
// The weights are taken against the reference exponent m as it stands, so that they need not wait for the tile's maximum; one vote
// of the warp, before anything is stored, finds logits beyond 2^60 of it, NaNs, masks and rows without a reference,
// which go a slower way.  m moves where a logit has exceeded it by 2^8, before the next tile; O is then rescaled in tensor memory by
// the softmax warps themselves.
// An item of at most T tokens lets its two accumulators take the even and the odd tiles instead (`halves`).
// Calls of few tokens (kFew: 64 / G rows or fewer per sequence on average; drafts, single tokens), which the stream of the cache bounds, have
// items of 64 rows cut that way, one tile of Q and six slots.  Q stands twice in its tile: rows 64 and on see the same logits, and
// put what the rounding of the weights has left over S, so that O = (row) + (row + 64) has weights of two bf16 for no more time.
//
// Work is dealt evenly whatever the lengths: the tiles of all items, laid end to end (sequence, KV head, tokens), are cut into
// runs of equal length, and every CTA (one per SM) takes as many of them, one in each round.  A piece of an item goes to a workspace as
// (m, l, O) in fp32; the last CTA to arrive merges them (a ticket, no waiting).  A run has two pieces of that kind at most.
// Several rounds keep what is looked at at a time small: 2048 tokens at 131072, all in one round, read 70 % of their
// tiles from DRAM.
//
// Weights enter the product as bf16, one rounding of 2^-8, where the MMAs are what bounds the kernel: as two bf16 they would cost half as
// many again (2^-16 in calls of few tokens, as the decode kernels have it).  Sums, references, O and what
// is merged are fp32.
#pragma once
#include <cuda.h>
#include <float.h>

#include "attn_group_umma.cuh"
#include "chunk_walk.cuh"
#include "common.cuh"
#include "score_umma.cuh"
#include "tokens.cuh"

namespace prhs {

constexpr int kCAHalfBytes = kCATile * 128;               // [128 rows][64 columns] bf16
constexpr int kCATileBytes = 2 * kCAHalfBytes;            // 32 KB
constexpr int kCATiles = 7;                               // of 32 KB: Q and the ring
constexpr int kCASlots = 6;                               // of the ring at most
constexpr int kCAMaxMended = 16;                          // tiles of a piece that a row sees in part: 3 + 3 + 1 at most
constexpr int kCAPieces = 4;                              // of a CTA that are known ahead
constexpr int kCAPieceBytes = 128;
constexpr int kCANotes = 8;                               // pieces whose mended tiles are noted: the pieces known ahead let the mending warps run four ahead at most
// What is shared beside the tiles (they leave 3 KB).
struct ChunkShared {
  unsigned char pieces[kCAPieces][kCAPieceBytes];
  // kv_full[6], kv_empty[6], v_ready[6], q_full, q_empty, s_full[2], p_full[2][2] (halves of a tile's weights), o_full[2], o_empty[2], drain,
  // piece_full[4], piece_empty[4], noted[8]
  unsigned long long bars[3 * kCASlots + 13 + 2 * kCAPieces + kCANotes];
  int mended_n[kCANotes], mended_tile[kCANotes][kCAMaxMended];      // 2 * tile + (its place in the piece, odd or even)
  uint32_t tmem;
  int abort, last;
  int fills, q_fills;              // of the ring; of Q, but for multiples of two (for the drain)
};
constexpr int kCASmemBytes = kCATiles * kCATileBytes + (int)sizeof(ChunkShared);
constexpr int kCAThreads = 12 * 32;
constexpr int kCAMmaWarp = 8, kCALoadWarp = 9, kCAMendWarp = 10;
constexpr int kCASlotFloats = 2 * kCATile * kHeadDim + 2 * kCATile * 2;      // a piece in the workspace: O [2][32][128] float4, (m, l) [2][128]
constexpr uint32_t kCAIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kCATile >> 3) << 17) | ((uint32_t)(kCATile >> 4) << 24);
constexpr uint32_t kCAIdescPV = kCAIdesc | (1u << 16);    // B = V tile read MN-major
// A row's reference moves where a logit exceeds it by 2^kCAGap; up to 2^kCAFar the weights stand (bf16 and fp32 have the range:
// 128 keys of values up to 2^50, in 592 pieces).
constexpr float kCAGap = 8.f, kCAFar = 60.f;
// ------------------------------------------------------------------------------------ instructions
__device__ __forceinline__ void tma_load_2d_plain(uint32_t dst, const CUtensorMap* tm, int c0, int c1, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(tm), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_3d_plain(uint32_t dst, const CUtensorMap* tm, int c0, int c1, int c2, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(r));
  return r != 0;
}
// lower words of the matrix descriptors (see umma_desc, umma_desc_mn); the upper one is kSUDescHi
__device__ __forceinline__ uint32_t umma_desc_lo(uint32_t smem_addr) { return ((smem_addr >> 4) & 0x3fffu) | (1u << 16); }
__device__ __forceinline__ uint32_t umma_desc_mn_lo(uint32_t smem_addr) {
  return ((smem_addr >> 4) & 0x3fffu) | ((uint32_t)(kCAHalfBytes >> 4) << 16);
}
// S = Q K^T: eight steps of 16 columns, 32 bytes apart in a row; the second 64 columns are a box of their own, 16 KB further
__device__ __forceinline__ void umma_qk(uint32_t d, uint32_t q_lo, uint32_t k_lo) {
  asm volatile(
      "{\n .reg .b32 x, y;\n .reg .b64 a, b;\n .reg .pred f, t;\n"
      " setp.ne.b32 f, 0, 0;\n setp.eq.b32 t, 0, 0;\n"
      " mov.b64 a, {%1, %3};\n mov.b64 b, {%2, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, f;\n"
      " add.u32 x, %1, 2;\n add.u32 y, %2, 2;\n mov.b64 a, {x, %3};\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, t;\n"
      " add.u32 x, %1, 4;\n add.u32 y, %2, 4;\n mov.b64 a, {x, %3};\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, t;\n"
      " add.u32 x, %1, 6;\n add.u32 y, %2, 6;\n mov.b64 a, {x, %3};\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, t;\n"
      " add.u32 x, %1, 1024;\n add.u32 y, %2, 1024;\n mov.b64 a, {x, %3};\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, t;\n"
      " add.u32 x, %1, 1026;\n add.u32 y, %2, 1026;\n mov.b64 a, {x, %3};\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, t;\n"
      " add.u32 x, %1, 1028;\n add.u32 y, %2, 1028;\n mov.b64 a, {x, %3};\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, t;\n"
      " add.u32 x, %1, 1030;\n add.u32 y, %2, 1030;\n mov.b64 a, {x, %3};\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, t;\n}"
      ::"r"(d), "r"(q_lo), "r"(k_lo), "r"(kSUDescHi), "r"(kCAIdesc)
      : "memory");
}
// O (+)= P V over 64 keys: four steps of 16 keys, 8 columns of P and 2 KB of V apart
__device__ __forceinline__ void umma_pv4(uint32_t d, uint32_t a, uint32_t v_lo, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .b32 x, y;\n .reg .b64 b;\n .reg .pred f, t;\n"
      " setp.ne.b32 f, %5, 0;\n setp.eq.b32 t, 0, 0;\n"
      " mov.b64 b, {%2, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, f;\n"
      " add.u32 x, %1, 8;\n add.u32 y, %2, 128;\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, t;\n"
      " add.u32 x, %1, 16;\n add.u32 y, %2, 256;\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, t;\n"
      " add.u32 x, %1, 24;\n add.u32 y, %2, 384;\n mov.b64 b, {y, %3};\n tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, t;\n}"
      ::"r"(d), "r"(a), "r"(v_lo), "r"(kSUDescHi), "r"(kCAIdescPV), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr));
}
// the registers are operands of the wait so that no use of them can be scheduled before it
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                 "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                 "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// the lowest n bits, none for n <= 0, all for n >= 32
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
// A bounded wait that does not end with another warp's.
__device__ __forceinline__ bool mbar_wait_through(uint32_t bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > 4 * kWaitBudgetCycles) return false;
  return true;
}
// the largest of three; NaN if one is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// (an aligned barrier, as the loads and stores of tensor memory are: all lanes of a warp at once)
__device__ __forceinline__ void softmax_bar() {
  __syncwarp();
  asm volatile("bar.sync 1, 256;" ::: "memory");
}

// Ring position: slot and the parity of its fill.
template <int kSlots>
struct RingPos {
  int slot = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void step() {
    if (++slot == kSlots) {
      slot = 0;
      parity ^= 1;
    }
  }
};

// The order in which K and V tiles go through the ring: V follows its K by one step (two where the accumulators take turns with the
// tiles, so that both have a tile under way).
#define PRHS_CHUNK_STEPS(x, k) for (int k = (x).k0, lag_ = (x).halves() ? 2 : 1, stop_ = (x).k1 > (x).k0 ? (x).k1 + lag_ : (x).k0; k < stop_; ++k)

// grid: one CTA per SM.  tm_q: q as [rows][Hq][128], box [T][G][64]; tm_k, tm_v: [rows][128], box [128][64], or [16][64] per page.
template <bool kPaged, bool kMask, bool kFew>
__global__ void __launch_bounds__(kCAThreads, 1)
chunk_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ ChunkParams p) {
  extern __shared__ __align__(1024) unsigned char ca_smem[];
  constexpr int kQTiles = kFew ? 1 : 2, kSlots = kCATiles - kQTiles;
  ChunkShared& sh = *reinterpret_cast<ChunkShared*>(ca_smem + kCATiles * kCATileBytes);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (blockIdx.x == 0) record_bad_sequences(p.row_start, p.num_rows, p.kv.seq_lens, p.max_len, p.batch, p.flags);
  const uint32_t smem0 = (uint32_t)__cvta_generic_to_shared(ca_smem);
  if (smem0 & 1023u) {                  // (the swizzle asks for it, and there is no room to round up)
    if (threadIdx.x == 0) atomicOr(p.flags, kFlagTimeout);
    return;
  }
  const uint32_t ring = smem0 + kQTiles * kCATileBytes;
  const uint32_t bar0 = (uint32_t)__cvta_generic_to_shared(sh.bars);
  const uint32_t bar_full = bar0, bar_empty = bar0 + 8 * kCASlots, bar_vready = bar0 + 16 * kCASlots;
  const uint32_t bar_qfull = bar0 + 24 * kCASlots, bar_qempty = bar_qfull + 8, bar_sfull = bar_qfull + 16, bar_pfull = bar_qfull + 32;
  const uint32_t bar_ofull = bar_qfull + 64, bar_oempty = bar_qfull + 80, bar_drain = bar_qfull + 96, bar_piece = bar_qfull + 104;
  const uint32_t bar_noted = bar_piece + 16 * kCAPieces;
  if (tid == 0) {
    for (int i = 0; i < kCASlots; ++i) {
      mbar_init(bar_full + 8 * i, 1);      // the producer's expect_tx arrive
      mbar_init(bar_empty + 8 * i, 3);     // a commit, the mending warps
      mbar_init(bar_vready + 8 * i, 2);    // the mending warps
    }
    mbar_init(bar_qfull, 1);
    mbar_init(bar_qempty, 1);              // a commit
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_sfull + 8 * i, 1);     // a commit
      mbar_init(bar_pfull + 16 * i, 4);    // the subtile's softmax warps, for each half of the columns
      mbar_init(bar_pfull + 16 * i + 8, 4);
      mbar_init(bar_ofull + 8 * i, 1);     // a commit
      mbar_init(bar_oempty + 8 * i, 4);    // the subtile's softmax warps
    }
    mbar_init(bar_drain, 1);
    for (int i = 0; i < kCAPieces; ++i) {
      mbar_init(bar_piece + 8 * i, 1);                     // the producer
      mbar_init(bar_piece + 8 * (kCAPieces + i), 11);      // all other warps
    }
    for (int i = 0; i < kCANotes; ++i) {
      mbar_init(bar_noted + 8 * i, 1);     // the mending warps' first thread, which writes the notes
      sh.mended_n[i] = 0;
    }
    sh.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  static_assert(sizeof(Piece<kMask, kFew>) <= kCAPieceBytes, "a piece has its place in shared memory");
  if (warp == kCAMmaWarp) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"((uint32_t)__cvta_generic_to_shared(&sh.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem0 = *(volatile uint32_t*)&sh.tmem;       // S0, S1, O0, O1: 128 columns each; P over the first half of S
  Piece<kMask, kFew> x;
  // The next piece, by whatever warp but the producer; false: there is none.  (Waits whatever happened: the producer tells of all pieces and
  // of the end even after an aborted wait, so that the warps of a barrier leave together.)
  int piece_at = 0;
  auto take = [&] {
    const int i = piece_at % kCAPieces;
    if (!__all_sync(0xffffffffu, mbar_wait_through(bar_piece + 8 * i, (piece_at / kCAPieces) & 1))) return false;
    x = *reinterpret_cast<const Piece<kMask, kFew>*>(sh.pieces[i]);
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_piece + 8 * (kCAPieces + i));
    __syncwarp();
    ++piece_at;
    return x.k1 >= 0;
  };
  auto gave_up = [&] {
    atomicOr(p.flags, kFlagTimeout);
    sh.abort = 1;
  };

  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // -------------------------------------------------------------------------- softmax: a thread is a row
    const int s = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t tm_s = tmem0 + s * kCATile + lanes, tm_o = tmem0 + (2 + s) * kCATile + lanes;
    const int mine = kFew ? row & 63 : row;          // (rows 64 and on repeat the others: see the top)
    const int token = mine / p.group, head = mine - token * p.group;
    const float c1 = kScale * kLog2e;
    uint32_t s_par = 0, o_par = 0;
    int buf = 0;                                     // of the mending warps' notes
    bool aborted = false;                            // a warp that gave up goes on without touching anything: barriers stay balanced
    while (take()) {
      const bool used = mine < p.tokens * p.group && token < x.e(p, s) - x.a(p, s);
      const bool warp_used = __any_sync(0xffffffffu, used);
      const int u = used ? x.uf(p, s) + token : 0;
      const int from = kMask && used ? first_visible(p, u) : 0;
      const int kb = s ? x.kb[1] : x.kb[0], ke = x.halves() ? x.k1 : min(x.k1, s ? x.ke[1] : x.ke[0]);
      const int kf = s ? x.kf[1] : x.kf[0], kd = s ? x.kd[1] : x.kd[0], sf = s ? x.sf[1] : x.sf[0];
      float m = -INFINITY, next = -INFINITY;         // the reference, and the one to go on with
      uint64_t l2 = 0ull;                            // two partial sums
      bool any = false;                              // O holds something
      bool ready = false, late = false;              // every row has a reference; one has fallen behind
      // The reference moves: what has been summed up so far is scaled down.  (S of the present tile was issued behind the
      // products of those before it, so O is at rest.)
      auto raise = [&](float mx) {
        const float mn = fmaxf(m, mx), f = mn == -INFINITY ? 1.f : exp2f(m - mn);
        l2 = fma_f32x2(l2, pack_f32x2(f, f), 0ull);
        m = mn;
        if (any) {
#pragma unroll 1
          for (int c = 0; c < 8; ++c) {
            float o[16];
            tmem_ld16(tm_o + 16 * c, o);
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] *= f;
            tmem_st16(tm_o + 16 * c, o);
          }
        }
      };
      const int step = x.halves() ? 2 : 1;
      for (int k = x.halves() ? x.k0 + s : x.k0; k < ke; k += step) {
        if (kMask && !x.halves() && k >= x.sa && k < kb) continue;
        if (!aborted) {
          aborted = !__all_sync(0xffffffffu, mbar_wait(bar_sfull + 8 * s, s_par, &sh.abort));
          if (aborted && lane == 0) gave_up();
        }
        s_par ^= 1;
        if (aborted) continue;
        if (warp_used) {
          tc_fence_after();
          uint32_t r[4][32];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32(tm_s + 32 * c, r[c]);
          if (late) {
            raise(next);
            late = false;
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_wait_ld(r[c]);
          const bool partly = !(kMask ? k < sf || (k >= kf && k < kd) : k < kd);
          float mx;
          {
            float y[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              y[c] = __uint_as_float(r[c][0]);
#pragma unroll
              for (int j = 1; j < 31; j += 2) y[c] = max3_nan(y[c], __uint_as_float(r[c][j]), __uint_as_float(r[c][j + 1]));
              y[c] = max3_nan(y[c], __uint_as_float(r[c][31]), __uint_as_float(r[c][31]));
            }
            mx = max3_nan(max3_nan(y[0], y[1], y[2]), y[3], y[3]) * c1;
          }
          // The weights are taken against the reference as it stands, so that they need not wait for the maximum; up to 2^60 they
          // are as good as any, and the reference moves before the next tile.
          const bool plain = ready && !partly && !__any_sync(0xffffffffu, used && !(mx - m <= kCAFar));
          if (plain) {
            next = mx;
            late = __any_sync(0xffffffffu, used && mx > m + kCAGap);
          } else {
            // a tile that some row sees in part, logits that are not finite, no reference yet
            mx = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if (partly) {
                const int at = x.tile(k) * kCATile + 32 * c;
                const uint32_t see = bits_below(u - at) & (kMask ? bits_below(p.sinks - at) | ~bits_below(from - at) : 0xffffffffu);
#pragma unroll
                for (int j = 0; j < 32; ++j)
                  if (!((see >> j) & 1u)) r[c][j] = 0xff800000u;
              }
#pragma unroll
              for (int j = 0; j < 32; j += 2)                        // (passes over NaNs)
                mx = fmaxf(mx, fmaxf(__uint_as_float(r[c][j]), __uint_as_float(r[c][j + 1])));
            }
            mx *= c1;
            if (__any_sync(0xffffffffu, used && mx > m + kCAGap)) raise(mx);
            ready = __all_sync(0xffffffffu, !used || m > -INFINITY);
          }
          const float ref = m == -INFINITY ? 0.f : m;
          const uint64_t cc = pack_f32x2(c1, c1), mm = pack_f32x2(-ref, -ref);
          uint64_t la = 0ull, lb = 0ull;
          // the weights (kLow: what their rounding leaves), over S, and on to the tensor core in two halves
          auto weights = [&](auto low) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t w[32];
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                const int c = 64 * h + 2 * j;
                float a, b;
                unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[c >> 5][c & 31]), __uint_as_float(r[c >> 5][(c & 31) + 1])), cc, mm), a, b);
                a = exp2_fast(a);
                b = exp2_fast(b);
                if (j & 1) la = add_f32x2(la, pack_f32x2(a, b));
                else lb = add_f32x2(lb, pack_f32x2(a, b));
                w[j] = pack_bf16x2(a, b);
                if (decltype(low)::value) w[j] = pack_bf16x2(a - bf_lo(w[j]), b - bf_hi(w[j]));
              }
              tmem_st32(tm_s + 32 * h, w);
              tmem_wait_st();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar_pfull + 16 * s + 8 * h);
              __syncwarp();
            }
          };
          if (kFew && row >= 64) weights(SlotC<1>());
          else weights(SlotC<0>());
          l2 = add_f32x2(l2, add_f32x2(la, lb));
        } else if (lane == 0) {
          mbar_arrive(bar_pfull + 16 * s);
          mbar_arrive(bar_pfull + 16 * s + 8);
        }
        any = true;
      }
      float la, lb;
      unpack_f32x2(l2, la, lb);
      const float l = la + lb;
      // ------------------------------------------------------------ the piece's result
      // (O says nothing about the mending warps: of a piece that needs no mending the tensor core does not wait for them)
      if (any && !aborted) {
        aborted = !__all_sync(0xffffffffu, mbar_wait(bar_ofull + 8 * s, o_par, &sh.abort) &&
                                               mbar_wait(bar_noted + 8 * (buf % kCANotes), (buf / kCANotes) & 1, &sh.abort));
        if (aborted && lane == 0) gave_up();
      }
      if (any) o_par ^= 1;
      const bool whole = x.first_run == x.last_run && !x.halves();
      const int slot = 2 * x.run + (x.first_run == x.run ? 1 : 0);
      float* const part = p.partials + (size_t)slot * kCASlotFloats;
      const long long out_row = ((long long)(x.row0 + x.a(p, s) + token) * p.num_q_heads + x.kvh * p.group + head);
      const int mended = any && !aborted ? sh.mended_n[buf % kCANotes] : 0;
      if (!aborted && warp_used) {
        tc_fence_after();
        const float inv = l == 0.f ? 0.f : 1.f / l;
        // (a loop, not unrolled: it is outside the tiles)
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t r[32];
          __syncwarp();                  // (rows differ in what they add and whether they write)
          if (any) {
            tmem_ld32(tm_o + 32 * c, r);
            tmem_wait_ld(r);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = 0u;
          }
          // values that are not finite and were kept out of the product: infinite or NaN whatever their weight
          for (int y = 0; y < mended; ++y) {
            const int note = sh.mended_tile[buf % kCANotes][y], at = (note >> 1) * kCATile;
            if (x.halves() && (note & 1) != s) continue;               // (the other accumulator's tile)
            for (int i = at; i < min(at + kCATile, u); ++i) {
              if (i >= p.sinks && i < from) continue;
              long long off = (long long)x.b * p.kv.stride_outer + (long long)i * kHeadDim;
              if (kPaged) {
                const int page = __ldg(p.kv.page_table + (long long)x.b * p.kv.page_table_stride + (i >> kPageShift));
                if ((unsigned)page >= (unsigned)p.kv.num_pages) continue;
                off = (long long)page * p.kv.stride_outer + (i & 15) * kHeadDim;
              }
              const __nv_bfloat16* v = p.kv.v + off + (long long)x.kvh * p.kv.stride_head + 32 * c;
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                const float f = __bfloat162float(v[j]);
                if (!isfinite(f)) r[j] = __float_as_uint(__uint_as_float(r[j]) + f);
              }
            }
          }
          if (!used) continue;
          if (whole) {
            uint4* to = reinterpret_cast<uint4*>(p.out + out_row * kHeadDim + 32 * c);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              to[j] = make_uint4(pack_bf16x2(__uint_as_float(r[8 * j]) * inv, __uint_as_float(r[8 * j + 1]) * inv),
                                 pack_bf16x2(__uint_as_float(r[8 * j + 2]) * inv, __uint_as_float(r[8 * j + 3]) * inv),
                                 pack_bf16x2(__uint_as_float(r[8 * j + 4]) * inv, __uint_as_float(r[8 * j + 5]) * inv),
                                 pack_bf16x2(__uint_as_float(r[8 * j + 6]) * inv, __uint_as_float(r[8 * j + 7]) * inv));
          } else if (any) {
            float4* to = reinterpret_cast<float4*>(part) + (s * 32 + 8 * c) * kCATile + row;
#pragma unroll
            for (int j = 0; j < 8; ++j)
              __stcg(to + j * kCATile, make_float4(__uint_as_float(r[4 * j]), __uint_as_float(r[4 * j + 1]), __uint_as_float(r[4 * j + 2]),
                                                   __uint_as_float(r[4 * j + 3])));
          }
        }
        if (used) {
          if (whole) {
            if (p.out_lse) p.out_lse[out_row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
          } else {
            __stcg(reinterpret_cast<float2*>(part + 2 * kCATile * kHeadDim) + s * kCATile + row, make_float2(m, any ? l : -1.f));
          }
        }
        tc_fence_before();
      }
      if (any) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_oempty + 8 * s);
      }
      if (x.k1 > x.k0) ++buf;
      if (!whole) {
        // ---------------------------------------------------------- the last piece of an item to arrive merges them
        __threadfence();
        softmax_bar();
        const int parts = x.last_run - x.first_run + 1;
        if (tid == 0) {
          bool last = true;
          if (parts > 1) {
            last = atomicAdd(p.tickets + x.first_run, 1u) == (unsigned)parts - 1u;
            if (last) p.tickets[x.first_run] = 0u;
          }
          sh.last = last;
        }
        softmax_bar();
        if (sh.last && !*(volatile int*)&sh.abort && used) {
          __threadfence();
          // This thread's row: its subtile's pieces, 128 columns in four goes; with `halves` those of both, and half of the columns; of few
          // tokens the rows of the weights' low parts too, and a quarter of the columns.
          const int sub0 = x.halves() ? 0 : s, subs = x.halves() ? 2 : 1, n = parts * subs;
          const int c_begin = kFew ? 64 * s + 32 * (row >> 6) : x.halves() ? 64 * s : 0, c_end = c_begin + (kFew ? 32 : x.halves() ? 64 : 128);
          float M = 0.f, L = 0.f;
#pragma unroll 1
          for (int c0 = c_begin; c0 < c_end; c0 += 32) {
            float acc[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[j] = 0.f;
            M = -FLT_MAX;                // (below or at every finite reference, so that no difference is of two infinities of one sign)
            L = 0.f;
#pragma unroll 2
            for (int i = 0; i < n; ++i) {
              const int c = x.first_run + i / subs, y = sub0 + i % subs;
              const float* from = p.partials + (size_t)(2 * c + (c == x.first_run ? 1 : 0)) * kCASlotFloats;
              const float2 v = __ldcg(reinterpret_cast<const float2*>(from + 2 * kCATile * kHeadDim) + y * kCATile + mine);
              const float4* o = reinterpret_cast<const float4*>(from) + (y * 32 + c0 / 4) * kCATile + mine;
              float4 w[8], low[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) w[j] = __ldcg(o + j * kCATile);
              if (kFew) {
#pragma unroll
                for (int j = 0; j < 8; ++j) low[j] = __ldcg(o + j * kCATile + 64);
              }
              if (v.y < 0.f) continue;                                // (no tiles, and O was not written)
              // (a piece whose logits are all -inf: v.x = -inf, g = 0, and zero times its values that are not finite)
              const float mn = fmaxf(M, v.x), f = exp2f(M - mn), g = exp2f(v.x - mn);
              M = mn;
              L = fmaf(v.y, g, L * f);
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                if (kFew) w[j] = make_float4(w[j].x + low[j].x, w[j].y + low[j].y, w[j].z + low[j].z, w[j].w + low[j].w);
                acc[4 * j] = fmaf(w[j].x, g, acc[4 * j] * f);
                acc[4 * j + 1] = fmaf(w[j].y, g, acc[4 * j + 1] * f);
                acc[4 * j + 2] = fmaf(w[j].z, g, acc[4 * j + 2] * f);
                acc[4 * j + 3] = fmaf(w[j].w, g, acc[4 * j + 3] * f);
              }
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            uint4* to = reinterpret_cast<uint4*>(p.out + out_row * kHeadDim + c0);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              to[j] = make_uint4(pack_bf16x2(acc[8 * j] * inv, acc[8 * j + 1] * inv), pack_bf16x2(acc[8 * j + 2] * inv, acc[8 * j + 3] * inv),
                                 pack_bf16x2(acc[8 * j + 4] * inv, acc[8 * j + 5] * inv), pack_bf16x2(acc[8 * j + 6] * inv, acc[8 * j + 7] * inv));
          }
          if (p.out_lse && (kFew ? s == 0 && row < 64 : !x.halves() || s == 0)) p.out_lse[out_row] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
        }
        softmax_bar();                   // the slot may be written again
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == kCALoadWarp) {
      // ------------------------------------------------------------------------ producer
      const int outer_rows = (int)(p.kv.stride_outer >> 7), head_rows = (int)(p.kv.stride_head >> 7);
      const uint32_t q_bytes = 2u * 128u * (uint32_t)(p.group * p.tokens);
      RingPos<kSlots> pos;
      uint32_t q_par = 0;
      bool ring_full = false, q_full = false;        // whether slots (Q) have been filled before
      int fills = 0;
      bool ok = true;
      ChunkWalk<kMask, kFew> walk(p);
      bool more = walk.begin();
      while (more) {
        more = walk.next(x);
        const int at = piece_at % kCAPieces;
        if (piece_at >= kCAPieces &&
            !__all_sync(0xffffffffu, mbar_wait_through(bar_piece + 8 * (kCAPieces + at), (piece_at / kCAPieces - 1) & 1))) {
          ok = false;
          break;
        }
        if (!more) break;
        if (lane == 0) {
          *reinterpret_cast<Piece<kMask, kFew>*>(sh.pieces[at]) = x;
          mbar_arrive(bar_piece + 8 * at);
        }
        ++piece_at;
        if (!ok || x.k0 == x.k1) continue;
        if (lane == 0) {
          if (q_full) {
            ok = mbar_wait(bar_qempty, q_par, &sh.abort);
            if (ok) q_par ^= 1;
          }
          if (ok) {
            mbar_expect_tx(bar_qfull, !kFew && x.halves() ? q_bytes : 2 * q_bytes);
            for (int y = 0; y < (!kFew && x.halves() ? 1 : 2); ++y)
              for (int h = 0; h < 2; ++h)
                tma_load_3d_plain(smem0 + y * (kFew ? kCAHalfBytes / 2 : kCATileBytes) + h * kCAHalfBytes, &tm_q, 64 * h, x.kvh * p.group,
                                  x.row0 + (kFew ? 0 : y * p.tokens), bar_qfull);
          }
        }
        q_full = true;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) {
          if (lane == 0) gave_up();
          continue;
        }
        // pages: lanes 0 - 15 hold the row of page (lane / 2) mod 8 of the latest three tiles
        const int page_at = (lane >> 1) & 7, half = lane & 1;
        const int* table = kPaged ? p.kv.page_table + (long long)x.b * p.kv.page_table_stride : nullptr;
        auto lookup = [&](int k) -> uint32_t {
          if (!kPaged || k >= x.k1) return p.oob_row;
          const int pg = x.tile(k) * (kCATile / kBlockRows) + page_at;
          if (pg * kBlockRows >= x.t) return p.oob_row;
          const int id = __ldg(table + pg);
          if ((unsigned)id >= (unsigned)p.kv.num_pages) {
            if (lane < 16) atomicOr(p.flags, kFlagBadPage);
            return p.oob_row;
          }
          return (uint32_t)(id * outer_rows + x.kvh * head_rows);
        };
        uint32_t next_row = lookup(x.k0), rows[2] = {p.oob_row, p.oob_row};
        auto fill = [&](const CUtensorMap* tm, int k, uint32_t page_row) {
          if (lane == 0) {
            if (ring_full) ok = mbar_wait(bar_empty + 8 * pos.slot, pos.parity ^ 1, &sh.abort);
            if (ok) mbar_expect_tx(bar_full + 8 * pos.slot, kCATileBytes);
          }
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) return;
          const uint32_t dst = ring + pos.slot * kCATileBytes, bar = bar_full + 8 * pos.slot;
          if (kPaged) {
            if (lane < 16) tma_load_2d_plain(dst + half * kCAHalfBytes + page_at * 2048, tm, 64 * half, (int)page_row, bar);
          } else if (lane == 0) {
            const int r = x.b * outer_rows + x.kvh * head_rows + x.tile(k) * kCATile;
            tma_load_2d_plain(dst, tm, 0, r, bar);
            tma_load_2d_plain(dst + kCAHalfBytes, tm, 64, r, bar);
          }
          pos.step();
          if (++fills == kSlots) ring_full = true;
        };
        PRHS_CHUNK_STEPS(x, k) {
          if (ok && k - lag_ >= x.k0) fill(&tm_v, k - lag_, rows[lag_ - 1]);
          if (ok && k < x.k1) {
            rows[1] = rows[0];
            rows[0] = next_row;
            next_row = lookup(k + 1);
            fill(&tm_k, k, rows[0]);
          } else {
            rows[1] = rows[0];
          }
        }
        if (!ok && lane == 0) gave_up();
      }
      if (walk.changed() && lane == 0) atomicOr(p.flags, kFlagBadLength);
      if (lane == 0) {                   // the end
        sh.fills = fills;
        sh.q_fills = q_full ? (int)q_par + 1 : 0;
        x.k0 = x.k1 = -1;
        *reinterpret_cast<Piece<kMask, kFew>*>(sh.pieces[piece_at % kCAPieces]) = x;
        mbar_arrive(bar_piece + 8 * (piece_at % kCAPieces));
        if (!ok) gave_up();
      }
      __syncwarp();
    } else if (warp >= kCAMendWarp) {
      // ------------------------------------------------------------------------ mending warps (they follow the ring fill by fill)
      const int t64 = tid - 32 * kCAMendWarp;
      RingPos<kSlots> pos;
      int buf = 0;
      bool ok = true;
      while (take()) {         // (a warp that gave up goes on through the barriers of the other)
        if (x.k0 == x.k1) continue;
        if (t64 == 0) sh.mended_n[buf % kCANotes] = 0;
        __syncwarp();
        asm volatile("bar.sync 2, 64;" ::: "memory");
        PRHS_CHUNK_STEPS(x, k) {
          const int prev = k - lag_;
          if (prev >= x.k0) {
            const bool mend = x.mended(prev);
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar_full + 8 * pos.slot, pos.parity, &sh.abort));
            if (mend) {
              const int at = x.tile(prev) * kCATile;
              bool odd = false;
              if (ok) {
                const uint32_t base = ring + pos.slot * kCATileBytes;
                for (int i = t64; i < kCATile * 16; i += 64) {
                  const int r = (i >> 3) & 127;
                  const uint32_t addr = base + (uint32_t)i * 16u;
                  uint32_t w[4];
                  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
                  const bool gone = at + r >= x.t;
                  bool change = gone;
#pragma unroll
                  for (int j = 0; j < 4; ++j) {
                    const uint32_t bad = gone ? 0xffffffffu : __vcmpgeu2(w[j] & 0x7fff7fffu, 0x7f807f80u);
                    change |= bad != 0u;
                    odd |= !gone && bad != 0u;
                    w[j] &= ~bad;
                  }
                  if (change)
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              }
              uint32_t any_odd;
              asm volatile("{ .reg .pred a, b; setp.ne.u32 a, %1, 0; barrier.cta.red.or.pred b, 2, 64, a; selp.u32 %0, 1, 0, b; }"
                           : "=r"(any_odd) : "r"((uint32_t)odd) : "memory");
              if (any_odd && t64 == 0) {
                const int n = sh.mended_n[buf % kCANotes];
                if (n < kCAMaxMended) {
                  sh.mended_tile[buf % kCANotes][n] = 2 * x.tile(prev) + ((prev - x.k0) & 1);
                  sh.mended_n[buf % kCANotes] = n + 1;
                }
              }
              __syncwarp();
              if (ok && lane == 0) mbar_arrive(bar_vready + 8 * pos.slot);
            }
            if (ok && lane == 0) mbar_arrive(bar_empty + 8 * pos.slot);
            pos.step();
          }
          if (k < x.k1) {
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar_full + 8 * pos.slot, pos.parity, &sh.abort));
            if (ok && lane == 0) mbar_arrive(bar_empty + 8 * pos.slot);
            pos.step();
          }
        }
        if (t64 == 0) mbar_arrive(bar_noted + 8 * (buf % kCANotes));       // (also after a wait that ran out)
        ++buf;
      }
      if (!ok && lane == 0) gave_up();
    } else if (warp == kCAMmaWarp) {
      // ------------------------------------------------------------------------ MMA issue: one thread issues, the warp waits.
      // (The control flow is the whole warp's: operands of an MMA are uniform registers, and in code that a single lane has branched
      // into each one costs about a hundred cycles to issue.)
      const bool leader = elect_one();
      RingPos<kSlots> pos;
      uint32_t q_par = 0, vr_par = 0, p_par[2] = {0, 0}, oe_par[2] = {1, 1};
      bool ok = true;
      const uint32_t q_lo = umma_desc_lo(smem0), ring_k = umma_desc_lo(ring), ring_v = umma_desc_mn_lo(ring);
      constexpr uint32_t kSlotLo = kCATileBytes >> 4;
      // (a wait that runs out leaves the later ones to return at once)
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (!mbar_try_wait(bar, parity) && !mbar_wait(bar, parity, &sh.abort)) ok = false;
      };
      while (take()) {
        if (!ok || x.k0 == x.k1) continue;
        wait(bar_qfull, q_par);
        q_par ^= 1;
        bool started[2] = {false, false};
        auto pv = [&](int s, int v_slot) {
          const uint32_t d = tmem0 + (2 + s) * kCATile, a = tmem0 + s * kCATile, v = ring_v + v_slot * kSlotLo;
          wait(bar_pfull + 16 * s, p_par[s]);
          tc_fence_after();
          if (leader && ok) umma_pv4(d, a, v, started[s] ? 1u : 0u);
          wait(bar_pfull + 16 * s + 8, p_par[s]);
          p_par[s] ^= 1;
          tc_fence_after();
          if (leader && ok) umma_pv4(d, a + 32, v + 4 * ((16 * 128) >> 4), 1u);
          started[s] = true;
        };
        auto qk = [&](int s, int k_slot) {
          if (leader && ok) {
            umma_qk(tmem0 + s * kCATile, x.halves() ? q_lo : q_lo + s * kSlotLo, ring_k + k_slot * kSlotLo);
            umma_commit(bar_sfull + 8 * s);
          }
        };
        // tiles k - 1 that both subtiles see all of, with a tile k behind them that both use: nothing to ask
        const int plain_from = max(x.k0, kMask ? max(max(x.kf[0], x.kf[1]), x.kb[1]) : 0) + 1;
        const int plain_to = x.halves() ? x.k0 : min(min(min(x.kd[0], x.kd[1]) + 1, x.k1), min(x.ke[0], x.ke[1]));       // (their last products come after)
        // the last tile of each subtile (its O is complete behind it)
        int last[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          last[s] = x.halves() ? x.k1 - 2 : min(x.k1, x.ke[s]) - 1;
          if (kMask && !x.halves() && last[s] >= x.sa && last[s] < x.kb[s]) last[s] = x.sa - 1;      // (the piece ends among tiles that it skips)
        }
        uint32_t before[2] = {0, 0};                 // what the latest two tiles ask for: bits 0, 1: the subtiles that use it; 2: mending
        auto asks = [&](int k) -> uint32_t {
          return (x.active(0, k) ? 1u : 0u) | (x.active(1, k) ? 2u : 0u) | (x.mended(k) ? 4u : 0u);
        };
        PRHS_CHUNK_STEPS(x, k) {
          if (!ok) break;
          const RingPos<kSlots> vpos = pos;
          if (k >= plain_from && k < plain_to && started[0] && started[1]) {
            pos.step();
            const RingPos<kSlots> kpos = pos;
            pos.step();
            wait(bar_full + 8 * vpos.slot, vpos.parity);
            pv(0, vpos.slot);
            wait(bar_full + 8 * kpos.slot, kpos.parity);
            qk(0, kpos.slot);
            pv(1, vpos.slot);
            if (leader && ok) umma_commit(bar_empty + 8 * vpos.slot);
            qk(1, kpos.slot);
            if (leader && ok) {
              umma_commit(bar_empty + 8 * kpos.slot);
              if (k == x.k1 - 1) umma_commit(bar_qempty);
            }
            before[0] = asks(k);
            continue;
          }
          const bool do_pv = k - lag_ >= x.k0, do_qk = k < x.k1;
          const uint32_t then = do_pv ? before[lag_ - 1] : 0u, now = do_qk ? asks(k) : 0u;
          before[1] = before[0];
          before[0] = now;
          if (do_pv) {
            pos.step();
            wait(bar_full + 8 * vpos.slot, vpos.parity);
            if (then & 4u) {
              wait(bar_vready + 8 * vpos.slot, (vr_par >> vpos.slot) & 1u);
              vr_par ^= 1u << vpos.slot;
            }
          }
          const RingPos<kSlots> kpos = pos;
          if (do_qk) pos.step();
          bool k_here = false;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if ((then >> s) & 1u) {
              if (!started[s]) {
                wait(bar_oempty + 8 * s, oe_par[s]);
                oe_par[s] ^= 1;
              }
              pv(s, vpos.slot);
              if (k - lag_ >= last[s] && leader && ok) umma_commit(bar_ofull + 8 * s);
            }
            if (s == 1 && do_pv && leader && ok) umma_commit(bar_empty + 8 * vpos.slot);
            if ((now >> s) & 1u) {
              if (!k_here) wait(bar_full + 8 * kpos.slot, kpos.parity);
              k_here = true;
              tc_fence_after();
              qk(s, kpos.slot);
            }
          }
          if (leader && ok) {
            if (do_qk) umma_commit(bar_empty + 8 * kpos.slot);
            if (k == x.k1 - 1) umma_commit(bar_qempty);
          }
        }
      }
      if (!ok) gave_up();
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (sh.abort) {
    // copies and MMAs may still be in flight: bounded waits before shared and tensor memory go back
    if (tid == kCALoadWarp * 32) {
      mbar_drain_ring(bar_full, kSlots, sh.fills);
      mbar_drain_ring(bar_qfull, 1, sh.q_fills);
    }
    if (warp == kCAMmaWarp && elect_one()) {           // (a commit is of the MMAs of the thread that makes it)
      umma_commit(bar_drain);
      const long long t0 = clock64();
      while (!mbar_try_wait(bar_drain, 0))
        if (clock64() - t0 > kWaitBudgetCycles / 8) break;
    }
    __syncthreads();
  }
  if (warp == kCAMmaWarp) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem0), "r"(512u) : "memory");
  }
}

}  // namespace prhs
