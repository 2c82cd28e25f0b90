// The 8-bit KV cache: the append that fills it and the decode attention that reads it.
//
// Layout.  A row of 128 keys (or values) is 128 bytes of e4m3 or e5m2.  Sixteen consecutive positions
// of one KV head form a block (a page of a paged cache) with one fp32 scale for its keys and one for
// its values: x ~ scale * code, scale = 2^max(ceil(log2(amax / top)), -126), top = 448 or 57344 the
// largest finite code.  Powers of two lose nothing (the codes are floating point) and make the
// quotient exact, so a code is one rounding of its element, the same on every machine.  Only whole
// blocks are quantised: the open block (the last t mod 16 positions) stays in bf16 in a tail of 16 rows
// per (sequence, KV head).  What the cache holds therefore depends on the rows alone, not on how they
// were split over calls, and nothing is ever quantised twice.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "attn.cuh"
#include "common.cuh"
#include "head_tiles.cuh"

namespace prhs {

constexpr int kE4M3 = 0, kE5M2 = 1;
constexpr int kBlockRows = 16;
constexpr int kRow8Bytes = kHeadDim;                        // 128 B per row
constexpr int kBlock8Bytes = kBlockRows * kRow8Bytes;       // 2 KB per block of keys or of values
constexpr uint32_t kFlagBadLength = 16u;
constexpr uint32_t kFlagNonFinite = 32u;

// Device-side copy of a prhs_bytekv_view.
struct ByteKvDev {
  const uint8_t* k;
  const uint8_t* v;
  const float* k_scale;
  const float* v_scale;
  const __nv_bfloat16* k_tail;      // [B][Hkv][16][128]
  const __nv_bfloat16* v_tail;
  long long stride_outer, stride_head;            // bytes
  long long scale_stride_outer, scale_stride_head;
  const int* page_table;
  int page_table_stride;
  const int* seq_lens;
  int num_pages;
};

// ---------------------------------------------------------------------------------- append
// The scale of a block whose largest magnitude has the bf16 bit pattern `amax` (sign cleared):
// top = 1.75 * 2^kTopExp, so the exponent of the quotient amax / top is that of amax less kTopExp, plus
// one where the significand of amax exceeds 1.75.  Returned as the exponent e of scale = 2^e, >= -126.
template <int kTopExp, int kTopFrac>
__device__ __forceinline__ int scale_exponent(uint32_t amax) {
  return max((int)(amax >> 7) - 127 - kTopExp + ((int)(amax & 0x7fu) > kTopFrac ? 1 : 0), -126);
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// One warp, one block of 16 rows held as rows 2i + lane / 16, 16-byte chunk lane % 16: quantised into
// `codes` (16 rows of 128 bytes) and `scale`.  Returns whether every element was finite.
template <int kFmt>
__device__ __forceinline__ bool quantise_block(const uint4 (&x)[8], uint8_t* codes, float* scale) {
  const int lane = threadIdx.x & 31;
  // the largest magnitude (two bf16 at a time: their bits order like the values)
  auto largest = [&](auto of) {
    uint32_t mx = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      mx = __vmaxu2(__vmaxu2(mx, __vmaxu2(of(x[i].x & 0x7fff7fffu), of(x[i].y & 0x7fff7fffu))),
                    __vmaxu2(of(x[i].z & 0x7fff7fffu), of(x[i].w & 0x7fff7fffu)));
    return __reduce_max_sync(0xffffffffu, max(mx & 0xffffu, mx >> 16));
  };
  uint32_t amax = largest([](uint32_t w) { return w; });
  const bool finite = amax < 0x7f80u;
  if (amax > 0x7f80u) amax = largest([](uint32_t w) { return w & ~__vcmpgtu2(w, 0x7f807f80u); });    // NaNs do not count
  const int e = kFmt == kE4M3 ? scale_exponent<8, 96>(amax) : scale_exponent<15, 96>(amax);
  const float inv = pow2i(-e);
  if (lane == 0) *scale = pow2i(e);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c[j] = __nv_cvt_float2_to_fp8x2(make_float2(bf_lo(w[j]) * inv, bf_hi(w[j]) * inv), __NV_SATFINITE,
                                      kFmt == kE4M3 ? __NV_E4M3 : __NV_E5M2);
    uint2 out = make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
    *reinterpret_cast<uint2*>(codes + (2 * i + (lane >> 4)) * kRow8Bytes + (lane & 15) * 8) = out;
  }
  return finite;
}

struct ByteKvAppendParams {
  ByteKvDev kv;
  const __nv_bfloat16* new_k;
  const __nv_bfloat16* new_v;
  long long new_stride_seq, new_stride_head, new_stride_row;     // elements
  const int* new_lens;        // [B]: rows that come in; seq_lens holds the lengths after them
  int max_new, max_len, batch, num_kv_heads;
  uint32_t* flags;
};

// One warp per (touched block, keys or values): warp pair j of a (sequence, KV head) owns block
// start / 16 + j.  The pair of the first block also writes the tail when a later block stays open: it alone
// reads the old tail, and a thread reads and writes the same 16-byte pieces of it, so program order keeps
// the two apart without a barrier.
// Bound by HBM: 512 B in and 256 B + 8 B / 16 out per position.
template <int kFmt>
__global__ void __launch_bounds__(256) bytekv_append_kernel(ByteKvAppendParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int j = blockIdx.x * (blockDim.x >> 6) + (warp >> 1), is_v = warp & 1;
  const int kvh = blockIdx.y, b = blockIdx.z;
  const int t = __ldg(p.kv.seq_lens + b), n = __ldg(p.new_lens + b);
  if (n < 0 || n > t || n > p.max_new || t > p.max_len) {
    if (threadIdx.x == 0) atomicOr(p.flags, kFlagBadLength);
    return;
  }
  const int start = t - n;
  const int blk = start / kBlockRows + j, open = t / kBlockRows;
  if (n == 0 || blk * kBlockRows >= t) return;
  const __nv_bfloat16* src = (is_v ? p.new_v : p.new_k) + (long long)b * p.new_stride_seq + (long long)kvh * p.new_stride_head;
  __nv_bfloat16* tail = const_cast<__nv_bfloat16*>(is_v ? p.kv.v_tail : p.kv.k_tail) +
                        ((long long)b * p.num_kv_heads + kvh) * (kBlockRows * kHeadDim);
  const int r0 = lane >> 4, col = (lane & 15) * 8;
  // rows of block `which` that come in now go to the tail
  auto to_tail = [&](int which) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int pos = which * kBlockRows + 2 * i + r0;
      if (pos >= start && pos < t)
        *reinterpret_cast<uint4*>(tail + (2 * i + r0) * kHeadDim + col) =
            __ldg(reinterpret_cast<const uint4*>(src + (long long)(pos - start) * p.new_stride_row + col));
    }
  };
  if (blk == open) {                     // this block stays open
    if (j == 0) to_tail(blk);            // (a later open block is the first pair's work)
    return;
  }
  bool page_ok = true;
  long long page = 0;
  if (p.kv.page_table) {
    page = __ldg(p.kv.page_table + (long long)b * p.kv.page_table_stride + blk);
    page_ok = page >= 0 && page < p.kv.num_pages;
    if (!page_ok && lane == 0) atomicOr(p.flags, kFlagBadPage);
  }
  uint4 x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int pos = blk * kBlockRows + 2 * i + r0;
    const __nv_bfloat16* from = pos < start ? tail + (2 * i + r0) * kHeadDim : src + (long long)(pos - start) * p.new_stride_row;
    x[i] = *reinterpret_cast<const uint4*>(from + col);
  }
  if (page_ok) {
    const long long outer = p.kv.page_table ? page : b;
    const long long off = outer * p.kv.stride_outer + (long long)kvh * p.kv.stride_head + (p.kv.page_table ? 0ll : (long long)blk * kBlock8Bytes);
    const long long soff = outer * p.kv.scale_stride_outer + (long long)kvh * p.kv.scale_stride_head + (p.kv.page_table ? 0 : blk);
    const bool finite = quantise_block<kFmt>(x, const_cast<uint8_t*>(is_v ? p.kv.v : p.kv.k) + off,
                                             const_cast<float*>(is_v ? p.kv.v_scale : p.kv.k_scale) + soff);
    if (!finite && lane == 0) atomicOr(p.flags, kFlagNonFinite);
  }
  if (j == 0 && open * kBlockRows < t) to_tail(open);
}

// ------------------------------------------------------------------------------- attention
// Decode attention over the 8-bit cache: every position (kList = false; a unit is a KV head of a sequence, whose query heads
// share the stream) or an explicit list per query head (kList = true).  How units are dealt to CTAs stands further down.
//
// The plumbing is that of the bf16 kernels (attn.cuh): warp-private cp.async rings of 16-row stages,
// 16-byte chunk c of row r at chunk c ^ (r & 7), parts of a unit merged by the last CTA to arrive.  What
// differs is what a row costs: half the bytes, so twice the arithmetic per byte, and that arithmetic has to
// stay cheap.  The codes become fp16 in registers (e4m3: one conversion instruction per two values; e5m2 is
// the upper byte of an fp16: one byte permute), which is exact, and the products run as mma.sync
// m16n8k16 fp16 with fp32 accumulation, keys or dimensions on the 16 rows and the heads on the 8 columns:
//   S^T = K Q^T      A = keys.  A lane's four consecutive bytes of a 16-byte chunk are dealt to the k-slots (2tg,
//                    2tg+1, 2tg+8, 2tg+9); the query's fragments are dealt the same way, and a sum does not
//                    care about the order.  No shuffles, no permutes.
//   O^T += V^T P^T   ldmatrix.trans moves byte pairs: a lane receives dimensions 2g and 2g+1 of its two keys, so
//                    tile row g is dimension 16c + 2g and row g + 8 is 16c + 2g + 1.  P^T is S^T's tile
//                    transposed 8 x 8 in registers (movmatrix).
// (The tensor cores would also take the keys' codes as they are, mma.sync m16n8k32 against the query in two e4m3
// parts, exactly and without converting the keys; that measured slower, 358 us against 333 us for 2.1 GB.)
// Sixteen MMAs per stage for up to eight heads; a lane's logits and its output columns belong to the same two
// heads, 2tg and 2tg + 1, so a new reference exponent needs no shuffle to reach the accumulators.
// (The first version had the heads on the rows: 24 MMAs, and four-lane shuffles of the factors.)
// The warps run dependent chains (copy, multiply, exponential, convert, multiply), so the stream needs many of them:
// twelve per SM with 16 KB rings.  (Eight with 24 KB rings issued 0.43 instructions per cycle and scheduler, most
// of the stalls fixed latencies: 147 us against 126 us for a ragged paged batch of 32; sixteen with 12 KB
// rings have too few bytes in flight: 341 us against 329 us for 2.1 GB.)
// Exponent bookkeeping.  The query is scaled by a power of two into [1, 2) (fp16 then keeps it to 2^-25 of its
// largest element).  A key block's scale multiplies its logits.  A value block's scale 2^e multiplies the
// weights: w = 2^(x - m) * 2^(e - R + 7), with m the running reference of the logits and R, an integer per
// head, that of the value scales; both move only when a weight would exceed 2^15 (one vote a stage).
// The largest weight stands between 2^6 (where the reference has just moved) and 2^15, so fp16 keeps weights to 2^-11 relative
// down to 2^-20 of the largest, and to 2^-31 of the largest below that.  The sum of the weights, m and the
// accumulators are fp32.
// The open block (bf16) enters the ring behind the last stage of the last warp and is one stage of the bf16 arithmetic
// (bf16_stage) into a partial of its own, merged with the warps' partials.
constexpr float k8Unscale = 0.0078125f;      // 2^-7: the weights enter the product times 2^7
constexpr int k8StageBytes = 2 * kBlock8Bytes;                          // 16 K rows + 16 V rows = 4 KB
constexpr int k8MetaBytes = 160;                                        // 16 K scales, 16 V scales, valid bits
// Lists have one CTA per unit where units are many: eight warps each, so that 256 of them keep the SMs busy.  (With four
// warps and three CTAs per SM, 188 of 444 CTA slots stay empty: 29.3 us for 256 lists of 1838 entries.)
template <bool kList, bool kWide>
struct Shape8 {
  static constexpr int kWarps = kList ? 8 : 4;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kStages = kList ? 3 : 4;
  static constexpr int kCtasPerSm = kList ? 2 : 3;
  static constexpr int kRingBytes = kWarps * kStages * k8StageBytes;
  static constexpr int kSmemBytes = kRingBytes + kWarps * kStages * k8MetaBytes;
  static_assert((kWarps + 1) * (kList ? 1 : kWide ? 16 : 8) * kHeadDim * 4 <= (kWarps - 1) * kStages * k8StageBytes,
                "the rings of all but the last warp take the partials");
};
constexpr int k8MaxCtasPerSm = 3;

struct ByteKvAttnParams {
  const __nv_bfloat16* q;   // [B][Hq][128]
  ByteKvDev kv;
  const int* idx;           // [B][Hq][idx_stride] (kList)
  const int* count;         // [B][Hq]
  int idx_stride;
  int batch, num_q_heads, group_size;
  int deal;                 // kRuns (the kernel decides), kParts, kWhole
  int max_len;              // lengths outside [0, max_len] are cut to it (and recorded)
  int sm_count;             // runs may be short while every SM has one CTA at most
  float* partials;          // [CTA][2][heads per unit][kPartStride]
  unsigned int* tickets;    // [B][Hq], zero on entry and on exit
  __nv_bfloat16* out;
  float* out_lse;
  uint32_t* flags;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same with a zero accumulator going in.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                              uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src, int src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Bytes (0, 1) and (2, 3) of w as two fp16 pairs.
template <int kFmt>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (kFmt == kE4M3) {
    asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b; }"
        : "=r"(lo), "=r"(hi) : "r"(w));
  } else {
    lo = __byte_perm(w, 0u, 0x1404);      // byte k of the result pair: (0, b0), (0, b1)
    hi = __byte_perm(w, 0u, 0x3424);
  }
}
// Bytes (0, 2) and (1, 3) of w as two fp16 pairs.
template <int kFmt>
__device__ __forceinline__ void codes_to_f16_split(uint32_t w, uint32_t& even, uint32_t& odd) {
  if (kFmt == kE4M3) {
    codes_to_f16<kFmt>(__byte_perm(w, 0u, 0x3120), even, odd);
  } else {
    even = w << 8 & 0xff00ff00u;
    odd = w & 0xff00ff00u;
  }
}

// One head's softmax bookkeeping in a lane.  R, an integer, is the reference exponent of the value scales.
struct Soft8 {
  float m = kNoLogit, l = 0.f, R = 0.f;
};

// The query of one head (g of the lane) as B fragments: this lane's elements 16c + 4tg .. + 3, scaled into [1, 2).
// Returns the factor that takes an fp32 product to the base-2 logit (without the keys' scale).
__device__ __forceinline__ float load_query_f16(const __nv_bfloat16* q, bool has, uint32_t (&lo)[8], uint32_t (&hi)[8]) {
  const int tg = threadIdx.x & 3;
  uint2 x[8];
  uint32_t mx = 0u;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    x[c] = has ? __ldg(reinterpret_cast<const uint2*>(q + 16 * c + 4 * tg)) : make_uint2(0u, 0u);
    mx = __vmaxu2(mx, __vmaxu2(x[c].x & 0x7fff7fffu, x[c].y & 0x7fff7fffu));
  }
  uint32_t amax = max(mx & 0xffffu, mx >> 16);
  amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
  amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
  const int e = min(max((int)(amax >> 7), 1), 253);          // biased exponent of the largest element
  const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    lo[c] = pack_f16x2(bf_lo(x[c].x) * inv, bf_hi(x[c].x) * inv);
    hi[c] = pack_f16x2(bf_lo(x[c].y) * inv, bf_hi(x[c].y) * inv);
  }
  return __uint_as_float((uint32_t)e << 23) * (kScale * kLog2e);
}

// Work.  A unit is a (sequence, KV head), its items the whole blocks; or (lists) a (sequence, query head), its items
// groups of sixteen entries, as many as a list can have (idx_stride: nobody has to look through all counts).
// A unit counts as at least one item (its open block, or nothing, still has to be written).  Four ways to deal
// units to CTAs:
//   runs    the blocks of all units, laid end to end, in equal runs, whatever the lengths: a run may cover the end
//           of one unit and the beginning of the next.  A CTA holds at most two parts of units that it shares with
//           its neighbours; whole units are finished on the spot.  (With an even split of every unit a ragged
//           batch waited for its longest sequence: 32 sequences of 2K to 16K, 156 us.)
//   parts   every unit in even parts, one part per CTA, where there are CTAs for that and the longest part is no
//           longer than a run and k8Crossing: a CTA that crosses into a second unit pays its start and end twice.
//           (8 KV heads of 2047 positions: 20 us in runs, 12 in parts.  32 x 8 heads of 500: 18.8 and 12.2; of 980:
//           19.9 and 18.7; of 1809: 29.3 and, with k8Crossing = 48, 31.  10 x 8 of 140 for 16 heads: 39 and 10.3.)
//   units   as runs, but a CTA takes whole units, those that begin in its run, where none is longer than k8Crossing
//           (58 x 32 heads of 300 positions: 44.9 us in runs, 41.2)
//   whole   lists, where two CTAs for each do not fit: one CTA per unit (256 lists of 1838 entries: 29 us; in runs, 34 us)
// The host's choice is runs, parts or whole; for runs the kernel, which knows the lengths, decides between the first three.
constexpr int kRuns = 0, kParts = 1, kWhole = 2, kUnits = 3;
constexpr int k8Crossing = 32;               // blocks in the time that a second start and end take
// items per CTA at least: below, a merge costs more than the shorter part saves.  Where the items are so few that
// runs of the short kind give no SM two CTAs, the short kind: nothing else would use the idle SMs
// (8 KV heads of 2047 positions: 8.5 us against 9.3; of 500, 8.1 against 9.2.  With the short kind everywhere 8192
// positions take 14.7 us, not 11.8: more than 16 parts are merged in two goes)
template <bool kList>
constexpr int k8MinRun = kList ? 32 : 16;
constexpr int k8ShortRun = 8;
// and per part, for the merge's sake: it takes `merged` parts at a time and kWarps heads, 0.6 us each, where a block costs
// a warp about 0.2; the batches that make the sum of the two smallest, rounded up.  (Without: one KV head for 16 heads, 4708
// positions 22.8 us, not 17.9, 131072 positions 116, not 49; for 4 heads 10.5, not 10.0, and 37, not 26.)
template <int kWarps>
__device__ __forceinline__ int least_part(int longest, int heads) {
  const int merged = 16 * max(1, kWarps / heads), rounds = (heads + kWarps - 1) / kWarps;
  const int batches = max(1, (int)ceilf(sqrtf((float)longest / (float)(12 * merged * rounds))));
  return (longest + merged * batches - 1) / (merged * batches);
}

// kWide: more than eight heads per KV head (two column tiles).
template <int kFmt, bool kList, bool kWide>
__global__ void __launch_bounds__(Shape8<kList, kWide>::kThreads, Shape8<kList, kWide>::kCtasPerSm)
bytekv_attn_kernel(ByteKvAttnParams p) {
  using Shape = Shape8<kList, kWide>;
  constexpr int kStages = Shape::kStages, k8Warps = Shape::kWarps;
  constexpr int kTiles = kWide ? 2 : 1;        // column tiles of eight heads
  extern __shared__ __align__(128) unsigned char g_smem[];
  __shared__ int tail_count[kBlockRows];       // kList: how often each row of the open block is listed
  __shared__ bool is_last;
  __shared__ float sm_m[k8Warps + 1][16], sm_l[k8Warps + 1][16];
  float* sm_o = reinterpret_cast<float*>(g_smem);
  const int gq = kList ? 1 : p.group_size;
  const int num_kv = p.num_q_heads / p.group_size;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, tg = lane & 3;
  const bool paged = p.kv.page_table != nullptr;
  const uint32_t smem0 = (uint32_t)__cvta_generic_to_shared(g_smem);
  const uint32_t ring = smem0 + warp * (kStages * k8StageBytes);
  const uint32_t meta = smem0 + Shape::kRingBytes + warp * (kStages * k8MetaBytes);

  // copies: a lane fills 16-byte position lane % 8 of row 2i + lane / 16 of the K (lane / 8 even) or V tile with
  // the source chunk that the swizzle wants there: the destination is the same in every stage and there are
  // four source offsets
  const uint8_t* cbase = ((lane >> 3) & 1) ? p.kv.v : p.kv.k;
  const uint32_t dst_lane = ((lane >> 3) & 1) * kBlock8Bytes + (lane >> 4) * kRow8Bytes + (lane & 7) * 16;
  uint32_t sx[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sx[i] = ((lane & 7) ^ ((2 * i + (lane >> 4)) & 7)) << 4;
  const float* sbase = lane < 16 ? p.kv.k_scale : p.kv.v_scale;
  const int lm_mi = lane >> 3, lm_r = lane & 7;
  const int vrow = (lm_mi & 1) * 8 + lm_r;

  // this CTA's work: it begins in unit `sub` of sequence `seq` (lists: unit seq), at item seg_lo
  const int max_len = p.max_len;
  auto blocks_of = [max_len](int t) { return max(1, min(t, max_len) / kBlockRows); };      // a unit's items, at least one
  const int cta = blockIdx.x, units = p.batch * (kList ? p.num_q_heads : num_kv);
  const int list_items = kList ? max(1, (p.idx_stride + kBlockRows - 1) / kBlockRows) : 0;
  int seq = cta, sub = 0, seg_lo = 0, part = 0, parts = 1;
  int run_end = 1, share = 1, unit_at = 0;
  int deal = p.deal;
  if (deal != kWhole) {
    int before = 0, longest = list_items;
    const int total = kList ? units * list_items : count_items(p.kv.seq_lens, p.batch, num_kv, blocks_of, &longest);
    // no shorter than the smallest run or a unit; parts: as many as fit with every unit rounded up
    int min_run = total <= k8ShortRun * p.sm_count ? k8ShortRun : k8MinRun<kList>;
    const int ctas = (int)gridDim.x;
    if (!kList) min_run = max(min_run, least_part<k8Warps>(longest, gq));
    auto share_of = [&](int n) { return max((total + n - 1) / n, min(min_run, (total + units - 1) / units)); };
    if (!kList) share = share_of(ctas);
    if (units <= ctas) {
      const int even = units < ctas ? share_of(ctas - units) : longest;
      if (kList || min(even, longest) <= share + k8Crossing) { deal = kParts; share = even; }
    } else if (longest <= k8Crossing) {
      deal = kUnits;
    }
    if (deal == kParts) {
      const int most = share;
      auto count = [&](int t) { return (blocks_of(t) + most - 1) / most; };
      if (kList) {
        parts = (list_items + most - 1) / most;
        if (cta >= units * parts) return;
        seq = cta / parts;
        part = cta - seq * parts;
      } else if (longest <= share) {             // one part each
        if (cta >= units) return;
        seq = cta / num_kv;
        sub = cta - seq * num_kv;
      } else {
        if (!find_item(p.kv.seq_lens, p.batch, num_kv, count, cta, &seq, &before)) return;     // more CTAs than parts
        parts = count(__ldg(p.kv.seq_lens + seq));
        sub = (cta - before) / parts;
        part = (cta - before) - sub * parts;
      }
    } else if (!kList) {
      if ((long long)cta * share >= total) return;
      const int at = cta * share;
      run_end = min(at + share, total);
      find_item(p.kv.seq_lens, p.batch, num_kv, blocks_of, at, &seq, &before);
      const int w = blocks_of(__ldg(p.kv.seq_lens + seq));
      sub = (at - before) / w;
      unit_at = before + sub * w;
      seg_lo = at - unit_at;
      if (deal == kUnits && seg_lo > 0) {        // begun by the CTA before
        unit_at += w;
        if (unit_at >= run_end) return;
        seg_lo = 0;
        if (++sub == num_kv) { sub = 0; ++seq; }
      }
    }
  }

  while (true) {                               // units of the run (one pass where the CTA has one part)
    const int b = kList ? seq / p.num_q_heads : seq;
    const int kvh = kList ? (seq - b * p.num_q_heads) / p.group_size : sub;
    const int unit0 = kList ? seq : b * p.num_q_heads + kvh * gq;
    const int given = __ldg(p.kv.seq_lens + b), t = min(max(given, 0), max_len);
    if (t != given && tid == 0) atomicOr(p.flags, kFlagBadLength);
    const int whole = t & ~(kBlockRows - 1);   // positions below are in the 8-bit cache, the rest in the tail
    const int* ptab = p.kv.page_table + (long long)b * p.kv.page_table_stride;
    const int listed = kList ? min(max(__ldg(p.count + unit0), 0), p.idx_stride) : 0;
    const int w = kList ? list_items : blocks_of(t);
    // items that have rows; parts and CTAs behind the last of them have nothing to do
    const int live = kList ? (listed + kBlockRows - 1) / kBlockRows : whole / kBlockRows;
    int first_cta = cta, seg_hi = w;
    if (deal == kParts) {
      const int per = (w + parts - 1) / parts;             // parts * per >= w > (parts - 1) * per where parts = ceil(w / share)
      seg_lo = min(part * per, w);
      seg_hi = min(seg_lo + per, w);
      first_cta = cta - part;
      if (kList) parts = max(1, (live + per - 1) / per);
    } else if (deal == kRuns) {
      seg_hi = min(w, run_end - unit_at);
      first_cta = unit_at / share;
      part = cta - first_cta;
      parts = (unit_at + w - 1) / share - first_cta + 1;
    }

    if (kList && part >= parts) return;        // behind the list's last entry

    // list entries (kList) or blocks (dense) of this warp: [start, end)
    const int seg_end = min(seg_hi, live);
    const int per_warp = (max(seg_end - seg_lo, 0) + k8Warps - 1) / k8Warps;
    int start = min(seg_lo + warp * per_warp, max(seg_end, seg_lo));
    int end = max(min(start + per_warp, seg_end), start);
    const int nstages = end - start;
    if (kList) {
      start = min(start * kBlockRows, listed);
      end = min(end * kBlockRows, listed);
    }

    // ---- the open block: belongs to the end of the unit (dense) or wherever the list names it
    const bool want_tail = t > whole && (kList ? listed > 0 : seg_hi == w);
    const int nissue = nstages + (want_tail && warp == k8Warps - 1 ? 2 : 0);      // its keys, its values
    if (kList) {
      if (tid < kBlockRows) tail_count[tid] = 0;
      __syncthreads();
    }

    float o[kTiles][8][4];
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
      for (int c = 0; c < 8; ++c) { o[hh][c][0] = 0.f; o[hh][c][1] = 0.f; o[hh][c][2] = 0.f; o[hh][c][3] = 0.f; }
    Soft8 st[kTiles][2];                       // heads 8hh + 2tg, 8hh + 2tg + 1

    // dense, paged: where 32 blocks lie, one per lane, page ids loaded a group ahead
    auto pages_of = [&](int grp) -> int {
      const int blk = start + grp * 32 + lane;
      return (paged && blk < end) ? __ldg(ptab + blk) : 0;
    };
    int pg_next = 0;
    long long off_cur = 0;
    uint32_t sid_cur = 0u, ok_cur = 0xffffffffu;
    auto place_group = [&](int page) {
      const bool ok = (unsigned)page < (unsigned)p.kv.num_pages;
      off_cur = ok ? (long long)page * p.kv.stride_outer + (long long)kvh * p.kv.stride_head : 0ll;
      sid_cur = ok ? (uint32_t)(page * p.kv.scale_stride_outer + (long long)kvh * p.kv.scale_stride_head) : 0u;
      ok_cur = __ballot_sync(0xffffffffu, ok);
    };
    // list: the row-id pipeline of the bf16 kernel (32 entries, two stages, per step)
    ListDesc ld;
    uint32_t rid_a = 0u, sid_a = 0u, valid_a = 0u;
    int pos1 = -1, pg1 = 0, pos2 = -1;
    auto check_pos = [&](int raw, int grp) -> int {
      const int pos = checked_entry(ld, raw, start + grp * 32 + lane, end, t, p.flags);
      if (pos >= whole) {                      // a row of the open block: counted, attended at the end
        atomicAdd(&tail_count[pos & (kBlockRows - 1)], 1);
        return -1;
      }
      return pos;
    };
    auto page_of = [&](int pos) -> int { return (paged && pos >= 0) ? __ldg(ptab + (pos >> kPageShift)) : 0; };
    auto resolve = [&](int pos, int page) {    // row id and scale id of this lane's entry
      bool ok = pos >= 0;
      if (ok && paged && (unsigned)page >= (unsigned)p.kv.num_pages) {
        atomicOr(p.flags, kFlagBadPage);
        ok = false;
      }
      const long long outer = paged ? page : b;
      rid_a = ok ? (uint32_t)(outer * (p.kv.stride_outer >> 7) + (long long)kvh * (p.kv.stride_head >> 7) + (paged ? (pos & 15) : pos)) : 0u;
      sid_a = ok ? (uint32_t)(outer * p.kv.scale_stride_outer + (long long)kvh * p.kv.scale_stride_head + (paged ? 0 : pos >> kPageShift)) : 0u;
      valid_a = __ballot_sync(0xffffffffu, ok);
    };
    if (kList) {
      ld.list = p.idx + (long long)unit0 * p.idx_stride;
      ld.fused = 0; ld.s0 = 0; ld.nmid = 0; ld.lo = 0; ld.wlo = 0; ld.count = listed;
      pos1 = check_pos(list_entry(ld, start + lane, end), 0);
      resolve(pos1, page_of(pos1));
      pos1 = check_pos(list_entry(ld, start + 32 + lane, end), 1);
      pg1 = page_of(pos1);
      pos2 = list_entry(ld, start + 64 + lane, end);
    } else if (paged) {
      place_group(pages_of(0));
      pg_next = pages_of(1);
    }
    const long long lin = (long long)b * p.kv.stride_outer + (long long)kvh * p.kv.stride_head;
    const long long slin = (long long)b * p.kv.scale_stride_outer + (long long)kvh * p.kv.scale_stride_head;

    int islot = 0;                             // ring slot of the next issue
    auto issue = [&](int j) {
      const uint32_t mslot = meta + (uint32_t)islot * k8MetaBytes;
      if (j < nstages) {
        const uint32_t slot = ring + (uint32_t)islot * k8StageBytes + dst_lane;
        if (kList) {
          if (j > 0 && (j & 1) == 0) {
            const int grp = j >> 1;
            resolve(pos1, pg1);
            pos1 = check_pos(pos2, grp + 1);
            pg1 = page_of(pos1);
            pos2 = list_entry(ld, start + (grp + 2) * 32 + lane, end);
          }
          const int from = (j & 1) << 4;
          const uint32_t vm = (valid_a >> from) & 0xffffu;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 2 * i + (lane >> 4);
            const uint32_t rid = __shfl_sync(0xffffffffu, rid_a, from + r);
            cp_async_16(slot + i * (2 * kRow8Bytes), cbase + (size_t)rid * kRow8Bytes + sx[i & 3], ((vm >> r) & 1u) ? 16 : 0);
          }
          const uint32_t sid = __shfl_sync(0xffffffffu, sid_a, from + (lane & 15));
          cp_async_4(mslot + lane * 4, sbase + sid, ((vm >> (lane & 15)) & 1u) ? 4 : 0);
          if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(mslot + 128u), "r"(vm) : "memory");
        } else {
          long long off = lin + (long long)(start + j) * kBlock8Bytes;
          long long sid = slin + start + j;
          bool ok = true;
          if (paged) {
            if (j > 0 && (j & 31) == 0) {
              place_group(pg_next);
              pg_next = pages_of((j >> 5) + 1);
            }
            off = __shfl_sync(0xffffffffu, off_cur, j & 31);
            sid = __shfl_sync(0xffffffffu, sid_cur, j & 31);
            ok = (ok_cur >> (j & 31)) & 1u;
            if (lane == 0) {
              if (!ok) atomicOr(p.flags, kFlagBadPage);
              asm volatile("st.shared.u32 [%0], %1;" ::"r"(mslot + 128u), "r"(ok ? 1u : 0u) : "memory");
            }
          }
          const uint8_t* src = cbase + off + (lane >> 4) * kRow8Bytes;
          if (ok) {
#pragma unroll
            for (int i = 0; i < 8; ++i) cp_async_16_full(slot + i * (2 * kRow8Bytes), src + i * (2 * kRow8Bytes) + sx[i & 3]);
            if ((lane & 15) == 0) cp_async_4(mslot + lane * 4, sbase + sid, 4);
          }
        }
      } else if (j < nissue) {                 // the open block's keys, then its values: 16 rows of 256 bytes
        const __nv_bfloat16* src = (j == nstages ? p.kv.k_tail : p.kv.v_tail) + ((long long)b * num_kv + kvh) * (kBlockRows * kHeadDim);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = 2 * i + (lane >> 4), c = lane & 15;
          cp_async_16(ring + (uint32_t)islot * k8StageBytes + r * kRowBytes + ((c ^ (r & 7)) << 4), src + r * kHeadDim + c * 8,
                      whole + r < t ? 16 : 0);
        }
      }
      cp_async_commit();
      islot = islot + 1 == kStages ? 0 : islot + 1;
    };
#pragma unroll
    for (int j = 0; j < kStages - 1; ++j) issue(j);

    // ---- query fragments (while the first copies are on their way) and logit factors
    uint32_t q0[kTiles][8], q1[kTiles][8];
    float qm[kTiles][2];
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh) {
      const float f = load_query_f16(p.q + (long long)(unit0 + 8 * hh + g) * kHeadDim, 8 * hh + g < gq, q0[hh], q1[hh]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        qm[hh][e] = __shfl_sync(0xffffffffu, f, 8 * tg + 4 * e);
      }
    }

    int slot_i = 0;
    for (int i = 0; i < nstages; ++i) {
      cp_async_wait<kStages - 2>();
      __syncwarp();
      issue(i + kStages - 1);
      const uint32_t kt = ring + (uint32_t)slot_i * k8StageBytes, vt = kt + kBlock8Bytes;
      const float* ms = reinterpret_cast<const float*>(g_smem + (meta - smem0) + slot_i * k8MetaBytes);
      slot_i = slot_i + 1 == kStages ? 0 : slot_i + 1;
      uint32_t vm = 0xffffu;
      if (kList || paged) {
        vm = reinterpret_cast<const uint32_t*>(ms)[32];
        if (vm == 0u) continue;                // warp-uniform: a block whose page id is bad, entries all elsewhere
      }
      // ---- S^T = K Q^T (two chains)
      float s[kTiles][2][4];
#pragma unroll
      for (int pp = 0; pp < 2; ++pp) {
        uint32_t b0[4], b1[4];
        ldmatrix_x4(b0, kt + lm_r * kRow8Bytes + (((4 * pp + lm_mi) ^ lm_r) << 4));
        ldmatrix_x4(b1, kt + (8 + lm_r) * kRow8Bytes + (((4 * pp + lm_mi) ^ lm_r) << 4));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t a0, a1, a2, a3;
          codes_to_f16<kFmt>(b0[c], a0, a2);
          codes_to_f16<kFmt>(b1[c], a1, a3);
#pragma unroll
          for (int hh = 0; hh < kTiles; ++hh) {
            if (pp == 0 && c < 2) mma_f16_first(s[hh][c], a0, a1, a2, a3, q0[hh][c], q1[hh][c]);
            else mma_f16(s[hh][c & 1], a0, a1, a2, a3, q0[hh][4 * pp + c], q1[hh][4 * pp + c]);
          }
        }
      }
      // ---- logits of this lane's keys g and g + 8 for its heads; value scales as exponents.  (Heads that are not there
      // have a zero query and columns that nobody reads.)
      float ks[2], ve[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        ks[n] = ms[kList ? 8 * n + g : 0];
        ve[n] = (float)((int)(__float_as_uint(ms[16 + (kList ? 8 * n + g : 0)]) >> 23) - 127);
      }
      float x[kTiles][2][2];                   // [tile][head][key]
      bool exceed = false;
#pragma unroll
      for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const Soft8& h = st[hh][e];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            x[hh][e][n] = (s[hh][0][2 * n + e] + s[hh][1][2 * n + e]) * (qm[hh][e] * ks[n]);
            if (kList && !((vm >> (8 * n + g)) & 1u)) x[hh][e][n] = -INFINITY;
          }
          // (logits are compared by their differences: a large one has no room for an exponent beside it)
          if (kList) exceed = exceed || x[hh][e][0] - h.m > 8.f - fmaxf(ve[0] - h.R, 0.f) || x[hh][e][1] - h.m > 8.f - fmaxf(ve[1] - h.R, 0.f);
          else exceed = exceed || fmaxf(x[hh][e][0], x[hh][e][1]) - h.m > 8.f - fmaxf(ve[0] - h.R, 0.f);
        }
      if (__any_sync(0xffffffffu, exceed)) {
#pragma unroll
        for (int hh = 0; hh < kTiles; ++hh) {
          float fo[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            Soft8& h = st[hh][e];
            float mx = fmaxf(x[hh][e][0], x[hh][e][1]);
#pragma unroll
            for (int off = 4; off <= 16; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float mn = fmaxf(h.m, mx);
            float my = fmaxf(x[hh][e][0] - mn + ve[0], x[hh][e][1] - mn + ve[1]);
#pragma unroll
            for (int off = 4; off <= 16; off <<= 1) my = fmaxf(my, __shfl_xor_sync(0xffffffffu, my, off));
            // m + R, the reference of the weighted values, moves up only
            const float Rn = fmaxf(ceilf(fmaxf(my, h.m - mn + h.R)), -400.f);
            fo[e] = exp2_fast(h.m - mn + h.R - Rn);
            h.l *= exp2_fast(h.m - mn);
            h.m = mn;
            h.R = Rn;
          }
#pragma unroll
          for (int c = 0; c < 8; ++c) { o[hh][c][0] *= fo[0]; o[hh][c][1] *= fo[1]; o[hh][c][2] *= fo[0]; o[hh][c][3] *= fo[1]; }
        }
      }
      uint32_t pb[kTiles][2];
#pragma unroll
      for (int hh = 0; hh < kTiles; ++hh) {
        float wgt[2][2];                       // [key][head]
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          Soft8& h = st[hh][e];
          float vf[2];                         // 2^(value scale - R + 7)
          vf[0] = exp2_fast(fminf(ve[0] - h.R + 7.f, 126.f));
          vf[1] = kList ? exp2_fast(fminf(ve[1] - h.R + 7.f, 126.f)) : vf[0];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const float pv = exp2_fast(x[hh][e][n] - h.m);
            h.l += pv;
            wgt[n][e] = pv * vf[n];
          }
        }
        pb[hh][0] = transpose_8x8(pack_f16x2(wgt[0][0], wgt[0][1]));
        pb[hh][1] = transpose_8x8(pack_f16x2(wgt[1][0], wgt[1][1]));
      }
      // ---- O^T += V^T P^T
#pragma unroll
      for (int cp = 0; cp < 4; ++cp) {
        uint32_t bv[4];
        ldmatrix_x4_trans(bv, vt + vrow * kRow8Bytes + (((2 * cp + (lm_mi >> 1)) ^ lm_r) << 4));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t a0, a1, a2, a3;
          codes_to_f16_split<kFmt>(bv[2 * k], a0, a1);
          codes_to_f16_split<kFmt>(bv[2 * k + 1], a2, a3);
#pragma unroll
          for (int hh = 0; hh < kTiles; ++hh) mma_f16(o[hh][2 * cp + k], a0, a1, a2, a3, pb[hh][0], pb[hh][1]);
        }
      }
    }
    cp_async_wait<0>();
    __syncwarp();

    // ---- partials of the warps and of the open block, in shared memory (the rings of all but the
    // last warp are free): [5][gq][128]
    __syncthreads();
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh) {
      float f[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float l = st[hh][e].l;
#pragma unroll
        for (int off = 4; off <= 16; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
        const int head = 8 * hh + 2 * tg + e;
        if (g == 0) { sm_m[warp][head] = l == 0.f ? -INFINITY : st[hh][e].m; sm_l[warp][head] = l; }
        f[e] = __uint_as_float((uint32_t)min(max((int)st[hh][e].R + 127, 0), 254) << 23);     // 2^R
        if (head < gq) {
#pragma unroll
          for (int c = 0; c < 8; ++c)
            *reinterpret_cast<float2*>(&sm_o[(warp * gq + head) * kHeadDim + 16 * c + 2 * g]) =
                make_float2(o[hh][c][e] * k8Unscale * f[e], o[hh][c][2 + e] * k8Unscale * f[e]);
        }
      }
    }
    bool tail_live = want_tail;
    if (kList && want_tail) {                  // is any row of the open block listed in this split?
      int any = 0;
      for (int r = 0; r < kBlockRows; ++r) any |= tail_count[r];
      tail_live = any != 0;
    }
    if (tail_live && warp == k8Warps - 1) {    // its rows are still in this warp's ring: the partials end before it
      constexpr int kTailHeads = kList ? 4 : kWide ? 16 : 8;
      uint32_t tq[kTiles][8][2];
      float to[kTiles][8][4];
      SoftBf ts[kTiles][2];
      load_query_bf16<kTailHeads>(p.q + (long long)unit0 * kHeadDim, gq, tq);
      clear_tiles<kTiles>(to);
      int times[2];                            // how often this lane's two keys are attended
#pragma unroll
      for (int n = 0; n < 2; ++n) times[n] = whole + 8 * n + g < t ? (kList ? tail_count[8 * n + g] : 1) : 0;
      const int passes = kList ? __reduce_max_sync(0xffffffffu, max(times[0], times[1])) : 1;
      const uint32_t kt = ring + (uint32_t)slot_i * k8StageBytes;
      const uint32_t vt = ring + (uint32_t)(slot_i + 1 == kStages ? 0 : slot_i + 1) * k8StageBytes;
      for (int d = 0; d < passes; ++d) {       // a row listed d times takes part in d passes (lists rarely repeat)
        if (kList) {                           // values of the others become zero: no weight times an infinity is NaN
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 2 * i + (lane >> 4);
            if (tail_count[r] == d)
              asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vt + r * kRowBytes + ((lane & 15u) << 4)), "r"(0u) : "memory");
          }
          __syncwarp();
        }
        bf16_stage<kTailHeads>(kt, vt, tq, times[0] > d, times[1] > d, to, ts);
        __syncwarp();
      }
      store_partial_bf16<kTailHeads>(to, ts, gq, sm_o + k8Warps * gq * kHeadDim, sm_m[k8Warps], sm_l[k8Warps]);
    }
    __syncthreads();
    // a part's place: two per CTA, the one it begins in the middle of and the other
    auto part_row = [&](int head, int i) -> float* {
      return p.partials + ((long long)(2 * (first_cta + i) + (i == 0 ? 1 : 0)) * gq + head) * kPartStride;
    };
    finish_unit<k8Warps>(sm_o, &sm_m[0][0], &sm_l[0][0], tail_live ? k8Warps + 1 : k8Warps, gq, parts, part, part_row, p.tickets,
                p.out, p.out_lse, unit0, &is_last);
    unit_at += w;
    if (kList || deal == kParts || unit_at >= run_end) return;
    seg_lo = 0;
    if (++sub == num_kv) { sub = 0; ++seq; }
    __syncthreads();                           // the ring and the partials in it are used again
  }
}

}  // namespace prhs
