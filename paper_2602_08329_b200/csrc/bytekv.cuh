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
  uint32_t mx = 0u;                                 // two bf16 magnitudes: their bits order like the values
#pragma unroll
  for (int i = 0; i < 8; ++i)
    mx = __vmaxu2(__vmaxu2(mx, __vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu)),
                  __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu));
  uint32_t amax = max(mx & 0xffffu, mx >> 16);
  amax = __reduce_max_sync(0xffffffffu, amax);
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
  return amax < 0x7f80u;
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
// Decode attention over the 8-bit cache: every position (kList = false; one CTA column per KV head, the
// group's heads share the stream) or an explicit list per query head (kList = true).
//
// The plumbing is that of the bf16 kernels (attn.cuh): warp-private cp.async rings of 16-row stages,
// 16-byte chunk c of row r at chunk c ^ (r & 7), splits merged by the last CTA to arrive.  What
// differs is what a row costs: half the bytes, so twice the arithmetic per byte, and that arithmetic has to
// stay cheap.  The codes become fp16 in registers (e4m3: one conversion instruction per two values; e5m2 is
// the upper byte of an fp16: one byte permute), which is exact, and the products run as mma.sync
// m16n8k16 fp16 with fp32 accumulation:
//   S = Q K^T   A = the heads (rows), B = keys.  A lane's four consecutive bytes of a 16-byte chunk are
//               dealt to the k-slots (2tg, 2tg+1, 2tg+8, 2tg+9); the query fragments are dealt the same way,
//               and a sum does not care about the order.  No shuffles, no permutes.
//   O^T += V^T P^T   ldmatrix.trans moves byte pairs: a lane receives dimensions 2g and 2g+1 of its two keys,
//               so tile row g is dimension 16c + 2g and row g + 8 is 16c + 2g + 1.
// Exponent bookkeeping.  The query is scaled by a power of two into [1, 2) (fp16 then keeps it to 2^-25 of its
// largest element).  A key block's scale multiplies its logits.  A value block's scale 2^e multiplies the
// weights: w = 2^(x - m) * 2^(e - R + 7), with m the running reference of the logits and R, an integer per
// head, that of the value scales; both move only when a weight would exceed 2^15 (one vote a stage).
// fp16 keeps w to 2^-12 relative down to 2^-29 of the largest weight.  The sum of the weights, m and the
// accumulators are fp32.
// The open block (bf16) is one stage of the bf16 arithmetic (group_stage) into a partial of its own, merged
// with the warps' partials.
constexpr float k8Unscale = 0.0078125f;      // 2^-7: the weights enter the product times 2^7
constexpr int k8Warps = 4;
constexpr int k8Threads = k8Warps * 32;
constexpr int k8Stages = 6;
constexpr int k8StageBytes = 2 * kBlock8Bytes;                          // 16 K rows + 16 V rows = 4 KB
constexpr int k8RingBytes = k8Warps * k8Stages * k8StageBytes;          // 96 KB
constexpr int k8MetaBytes = 160;                                        // 16 K scales, 16 V scales, valid bits
constexpr int k8TailBytes = 2 * kTTileBytes;                            // the open block in bf16: 8 KB
constexpr int k8SmemBytes = k8RingBytes + k8Warps * k8Stages * k8MetaBytes + k8TailBytes;

struct ByteKvAttnParams {
  const __nv_bfloat16* q;   // [B][Hq][128]
  ByteKvDev kv;
  const int* idx;           // [B][Hq][idx_stride] (kList)
  const int* count;         // [B][Hq]
  int idx_stride;
  int num_q_heads, group_size, splits;
  float* partials;          // [B][Hq][splits][kPartStride]
  unsigned int* tickets;    // zero on entry and on exit
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

// One head row's share of the softmax bookkeeping.
struct Soft8 {
  float m = -INFINITY, l = 0.f;
  int R = -1000;            // reference exponent of the value scales; any real exponent exceeds it
};

// The query of one head as A fragments: this lane's elements 16c + 4tg .. + 3, scaled into [1, 2).
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

// kWide: more than eight heads per KV head (both halves of the MMA's row tile carry heads).
template <int kFmt, bool kList, bool kWide>
__global__ void __launch_bounds__(k8Threads, 2) bytekv_attn_kernel(ByteKvAttnParams p) {
  extern __shared__ __align__(128) unsigned char g_smem[];
  __shared__ int tail_count[kBlockRows];       // kList: how often each row of the open block is listed
  __shared__ bool is_last;
  const int split = blockIdx.x, b = blockIdx.z;
  const int gq = kList ? 1 : p.group_size;
  const int kvh = kList ? blockIdx.y / p.group_size : blockIdx.y;
  const int unit0 = b * p.num_q_heads + (kList ? blockIdx.y : blockIdx.y * p.group_size);
  const int num_kv = p.num_q_heads / p.group_size;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, tg = lane & 3;
  const int t = __ldg(p.kv.seq_lens + b);
  const int whole = t & ~(kBlockRows - 1);     // positions below are in the 8-bit cache, the rest in the tail
  const bool paged = p.kv.page_table != nullptr;
  const int* ptab = p.kv.page_table + (long long)b * p.kv.page_table_stride;
  const uint32_t smem0 = (uint32_t)__cvta_generic_to_shared(g_smem);
  const uint32_t ring = smem0 + warp * (k8Stages * k8StageBytes);
  const uint32_t meta = smem0 + k8RingBytes + warp * (k8Stages * k8MetaBytes);
  const uint32_t tail = smem0 + k8RingBytes + k8Warps * k8Stages * k8MetaBytes;

  // list entries (kList) or blocks (dense) of this warp
  const int cnt = kList ? min(max(__ldg(p.count + unit0), 0), p.idx_stride) : whole / kBlockRows;
  constexpr int kUnit = kList ? kBlockRows : 1;               // entries or blocks per stage
  int per = (cnt + p.splits * k8Warps - 1) / (p.splits * k8Warps);
  per = (per + kUnit - 1) / kUnit * kUnit;
  const int start = min((split * k8Warps + warp) * per, cnt);
  const int end = min(start + per, cnt);
  const int nstages = (end - start + kUnit - 1) / kUnit;

  // ---- the open block: needed by the last split (dense) or wherever the list names it; fetched first, used last
  const bool want_tail = t > whole && (kList || split == p.splits - 1);
  if (kList && tid < kBlockRows) tail_count[tid] = 0;
  if (want_tail) {
    const long long off = ((long long)b * num_kv + kvh) * (kBlockRows * kHeadDim);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int piece = i * k8Threads + tid;                   // 256 K pieces, then 256 V pieces, of 16 bytes
      const int r = (piece >> 4) & 15, c = piece & 15;
      const __nv_bfloat16* src = (piece < 256 ? p.kv.k_tail : p.kv.v_tail) + off + r * kHeadDim + c * 8;
      cp_async_16(tail + (piece >> 8) * kTTileBytes + r * kRowBytes + ((c ^ (r & 7)) << 4), src, whole + r < t ? 16 : 0);
    }
  }
  if (kList) __syncthreads();                                  // tail_count is zero

  // ---- query fragments
  uint32_t qa0[8], qa2[8], qa1[8], qa3[8];
  const float qm0 = load_query_f16(p.q + (long long)(unit0 + g) * kHeadDim, g < gq, qa0, qa2);
  float qm1 = 0.f;
  if (kWide) qm1 = load_query_f16(p.q + (long long)(unit0 + g + 8) * kHeadDim, g + 8 < gq, qa1, qa3);
  const bool has0 = g < gq, has1 = kWide && g + 8 < gq;

  float o[kWide ? 2 : 1][8][4];
#pragma unroll
  for (int hh = 0; hh < (kWide ? 2 : 1); ++hh)
#pragma unroll
    for (int c = 0; c < 8; ++c) { o[hh][c][0] = 0.f; o[hh][c][1] = 0.f; o[hh][c][2] = 0.f; o[hh][c][3] = 0.f; }
  Soft8 st[kWide ? 2 : 1];

  // ---- copies.  A lane fills 16-byte position lane % 8 of row 2i + lane / 16 of the K (lane / 8 even) or V tile
  // with the source chunk that the swizzle wants there: the destination is the same in every stage and there
  // are four source offsets.
  const uint8_t* cbase = ((lane >> 3) & 1) ? p.kv.v : p.kv.k;
  const uint32_t dst_lane = ((lane >> 3) & 1) * kBlock8Bytes + (lane >> 4) * kRow8Bytes + (lane & 7) * 16;
  uint32_t sx[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sx[i] = ((lane & 7) ^ ((2 * i + (lane >> 4)) & 7)) << 4;
  const float* sbase = lane < 16 ? p.kv.k_scale : p.kv.v_scale;

  // dense: page ids of 32 blocks, one per lane, loaded a group ahead
  auto pages_of = [&](int grp) -> int {
    const int blk = start + grp * 32 + lane;
    return (paged && blk < end) ? __ldg(ptab + blk) : 0;
  };
  int pg_cur = 0, pg_next = 0;
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
    ld.fused = 0; ld.s0 = 0; ld.nmid = 0; ld.lo = 0; ld.wlo = 0; ld.count = cnt;
    pos1 = check_pos(list_entry(ld, start + lane, end), 0);
    resolve(pos1, page_of(pos1));
    pos1 = check_pos(list_entry(ld, start + 32 + lane, end), 1);
    pg1 = page_of(pos1);
    pos2 = list_entry(ld, start + 64 + lane, end);
  } else {
    pg_cur = pages_of(0);
    pg_next = pages_of(1);
  }
  const long long lin = (long long)b * p.kv.stride_outer + (long long)kvh * p.kv.stride_head;
  const long long slin = (long long)b * p.kv.scale_stride_outer + (long long)kvh * p.kv.scale_stride_head;

  auto issue = [&](int j) {
    if (j < nstages) {
      const uint32_t slot = ring + (uint32_t)(j % k8Stages) * k8StageBytes + dst_lane;
      const uint32_t mslot = meta + (uint32_t)(j % k8Stages) * k8MetaBytes;
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
        if (j > 0 && (j & 31) == 0) {
          pg_cur = pg_next;
          pg_next = pages_of((j >> 5) + 1);
        }
        long long off = lin + (long long)(start + j) * kBlock8Bytes, soff = slin + start + j;
        bool ok = true;
        if (paged) {
          const int page = __shfl_sync(0xffffffffu, pg_cur, j & 31);
          ok = (unsigned)page < (unsigned)p.kv.num_pages;
          if (!ok && lane == 0) atomicOr(p.flags, kFlagBadPage);
          off = ok ? (long long)page * p.kv.stride_outer + (long long)kvh * p.kv.stride_head : 0ll;
          soff = ok ? (long long)page * p.kv.scale_stride_outer + (long long)kvh * p.kv.scale_stride_head : 0ll;
        }
        const uint8_t* src = cbase + off + (lane >> 4) * kRow8Bytes;
#pragma unroll
        for (int i = 0; i < 8; ++i) cp_async_16(slot + i * (2 * kRow8Bytes), src + i * (2 * kRow8Bytes) + sx[i & 3], ok ? 16 : 0);
        if ((lane & 15) == 0) cp_async_4(mslot + lane * 4, sbase + soff, ok ? 4 : 0);
        if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(mslot + 128u), "r"(ok ? 0xffffu : 0u) : "memory");
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int j = 0; j < k8Stages - 1; ++j) issue(j);

  const int lm_mi = lane >> 3, lm_r = lane & 7;
  const int vrow = (lm_mi & 1) * 8 + lm_r;
  for (int i = 0; i < nstages; ++i) {
    cp_async_wait<k8Stages - 2>();
    __syncwarp();
    issue(i + k8Stages - 1);
    const uint32_t kt = ring + (uint32_t)(i % k8Stages) * k8StageBytes, vt = kt + kBlock8Bytes;
    const float* ms = reinterpret_cast<const float*>(g_smem + (meta - smem0) + (i % k8Stages) * k8MetaBytes);
    const uint32_t vm = reinterpret_cast<const uint32_t*>(ms)[32];
    if (vm == 0u) continue;                  // warp-uniform: a block whose page id is bad, entries all elsewhere
    // ---- S = Q K^T
    float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int pp = 0; pp < 2; ++pp) {
      uint32_t b0[4], b1[4];
      ldmatrix_x4(b0, kt + lm_r * kRow8Bytes + (((4 * pp + lm_mi) ^ lm_r) << 4));
      ldmatrix_x4(b1, kt + (8 + lm_r) * kRow8Bytes + (((4 * pp + lm_mi) ^ lm_r) << 4));
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t x0, x1;
        codes_to_f16<kFmt>(b0[c], x0, x1);
        mma_f16(s[0], qa0[4 * pp + c], kWide ? qa1[4 * pp + c] : 0u, qa2[4 * pp + c], kWide ? qa3[4 * pp + c] : 0u, x0, x1);
        codes_to_f16<kFmt>(b1[c], x0, x1);
        mma_f16(s[1], qa0[4 * pp + c], kWide ? qa1[4 * pp + c] : 0u, qa2[4 * pp + c], kWide ? qa3[4 * pp + c] : 0u, x0, x1);
      }
    }
    // ---- logits of this lane's keys 2tg, 2tg+1, 8+2tg, 9+2tg; value scales as exponents
    float ks[4];
    int ve[4];
    if (kList) {
      const float2 ka = *reinterpret_cast<const float2*>(ms + 2 * tg), kb = *reinterpret_cast<const float2*>(ms + 8 + 2 * tg);
      const uint2 va = *reinterpret_cast<const uint2*>(ms + 16 + 2 * tg), vb = *reinterpret_cast<const uint2*>(ms + 24 + 2 * tg);
      ks[0] = ka.x; ks[1] = ka.y; ks[2] = kb.x; ks[3] = kb.y;
      ve[0] = (int)(va.x >> 23) - 127; ve[1] = (int)(va.y >> 23) - 127;
      ve[2] = (int)(vb.x >> 23) - 127; ve[3] = (int)(vb.y >> 23) - 127;
    } else {
      const float k0 = ms[0];
      const int e = (int)(__float_as_uint(ms[16]) >> 23) - 127;
#pragma unroll
      for (int n = 0; n < 4; ++n) { ks[n] = k0; ve[n] = e; }
    }
    float x[kWide ? 2 : 1][4];
    bool exceed = false;
#pragma unroll
    for (int hh = 0; hh < (kWide ? 2 : 1); ++hh) {
      const bool has = hh ? has1 : has0;
      const float qm = hh ? qm1 : qm0;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const bool ok = has && (!kList || ((vm >> ((n >> 1) * 8 + 2 * tg + (n & 1))) & 1u));
        x[hh][n] = ok ? s[n >> 1][2 * hh + (n & 1)] * (qm * ks[n]) : -INFINITY;
        exceed = exceed || x[hh][n] + (float)max(ve[n] - st[hh].R, 0) > st[hh].m + 8.f;
      }
    }
    if (__any_sync(0xffffffffu, exceed)) {
#pragma unroll
      for (int hh = 0; hh < (kWide ? 2 : 1); ++hh) {
        float mx = fmaxf(fmaxf(x[hh][0], x[hh][1]), fmaxf(x[hh][2], x[hh][3]));
        float my = fmaxf(fmaxf(x[hh][0] + ve[0], x[hh][1] + ve[1]), fmaxf(x[hh][2] + ve[2], x[hh][3] + ve[3]));
#pragma unroll
        for (int off = 1; off <= 2; off <<= 1) {
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
          my = fmaxf(my, __shfl_xor_sync(0xffffffffu, my, off));
        }
        float fo = 1.f;
        if (mx > -INFINITY) {
          const float mn = fmaxf(st[hh].m, mx);
          // m + R, the reference of the weighted values, moves up only
          const float top = st[hh].m > -INFINITY ? fmaxf(my, st[hh].m + (float)st[hh].R) : my;
          const int Rn = (int)fmaxf(ceilf(top - mn), -400.f);
          fo = st[hh].m > -INFINITY ? exp2f(st[hh].m - mn + (float)(st[hh].R - Rn)) : 0.f;
          st[hh].l *= st[hh].m > -INFINITY ? exp2f(st[hh].m - mn) : 0.f;
          st[hh].m = mn;
          st[hh].R = Rn;
        }
        // the accumulator's columns are heads 2tg and 2tg + 1
        const float fa = __shfl_sync(0xffffffffu, fo, 8 * tg), fb = __shfl_sync(0xffffffffu, fo, 8 * tg + 4);
#pragma unroll
        for (int c = 0; c < 8; ++c) { o[hh][c][0] *= fa; o[hh][c][1] *= fb; o[hh][c][2] *= fa; o[hh][c][3] *= fb; }
      }
    }
    uint32_t pb[kWide ? 2 : 1][2];
#pragma unroll
    for (int hh = 0; hh < (kWide ? 2 : 1); ++hh) {
      float w[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float pv = x[hh][n] > -INFINITY ? exp2f(x[hh][n] - st[hh].m) : 0.f;
        st[hh].l += pv;
        w[n] = pv * __uint_as_float((uint32_t)min(max(ve[n] - st[hh].R + 134, 0), 254) << 23);
      }
      pb[hh][0] = pack_f16x2(w[0], w[1]);
      pb[hh][1] = pack_f16x2(w[2], w[3]);
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
        for (int hh = 0; hh < (kWide ? 2 : 1); ++hh) mma_f16(o[hh][2 * cp + k], a0, a1, a2, a3, pb[hh][0], pb[hh][1]);
      }
    }
  }
  cp_async_wait<0>();

  // ---- partials of the warps and of the open block, in shared memory (the ring is free): [5][gq][128]
  float* sm_o = reinterpret_cast<float*>(g_smem);
  __shared__ float sm_m[k8Warps + 1][16], sm_l[k8Warps + 1][16], sm_lt[k8Warps + 1][16];
  if (tid < 16) { sm_m[k8Warps][tid] = -INFINITY; sm_l[k8Warps][tid] = 0.f; sm_lt[k8Warps][tid] = 0.f; }
  __syncthreads();
#pragma unroll
  for (int hh = 0; hh < (kWide ? 2 : 1); ++hh) {
    float l = st[hh].l;
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (tg == 0) { sm_m[warp][8 * hh + g] = st[hh].m; sm_l[warp][8 * hh + g] = l; sm_lt[warp][8 * hh + g] = l; }
    const float f = __uint_as_float((uint32_t)min(max(st[hh].R + 127, 0), 254) << 23);     // 2^R
    const float fa = __shfl_sync(0xffffffffu, f, 8 * tg), fb = __shfl_sync(0xffffffffu, f, 8 * tg + 4);
    const int ha = 8 * hh + 2 * tg;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const int d = 16 * c + 2 * g;
      if (ha < gq) *reinterpret_cast<float2*>(&sm_o[(warp * gq + ha) * kHeadDim + d]) = make_float2(o[hh][c][0] * k8Unscale * fa, o[hh][c][2] * k8Unscale * fa);
      if (ha + 1 < gq) *reinterpret_cast<float2*>(&sm_o[(warp * gq + ha + 1) * kHeadDim + d]) = make_float2(o[hh][c][1] * k8Unscale * fb, o[hh][c][3] * k8Unscale * fb);
    }
  }
  bool tail_live = want_tail;
  if (kList && want_tail) {                    // is any row of the open block listed in this split?
    int any = 0;
    for (int r = 0; r < kBlockRows; ++r) any |= tail_count[r];
    tail_live = any != 0;
  }
  if (tail_live && warp == 0) {
    uint32_t aq[8][4];
    const uint32_t* q0 = reinterpret_cast<const uint32_t*>(p.q + (long long)(unit0 + g) * kHeadDim);
    const uint32_t* q1 = q0 + 8 * (kHeadDim / 2);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      aq[ks][0] = has0 ? __ldg(q0 + ks * 8 + tg) : 0u;
      aq[ks][1] = has1 ? __ldg(q1 + ks * 8 + tg) : 0u;
      aq[ks][2] = has0 ? __ldg(q0 + ks * 8 + 4 + tg) : 0u;
      aq[ks][3] = has1 ? __ldg(q1 + ks * 8 + 4 + tg) : 0u;
    }
    float ot[16][4];
#pragma unroll
    for (int nt = 0; nt < 16; ++nt) { ot[nt][0] = 0.f; ot[nt][1] = 0.f; ot[nt][2] = 0.f; ot[nt][3] = 0.f; }
    float m0 = -INFINITY, l0 = 0.f, m1 = -INFINITY, l1 = 0.f, lt0 = 0.f, lt1 = 0.f;
    int times[4] = {1, 1, 1, 1};               // how often this lane's four keys are attended
    int passes = 1;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int r = (n >> 1) * 8 + 2 * tg + (n & 1);
      times[n] = whole + r < t ? (kList ? tail_count[r] : 1) : 0;
    }
    if (kList) passes = __reduce_max_sync(0xffffffffu, max(max(times[0], times[1]), max(times[2], times[3])));
    for (int d = 0; d < passes; ++d)           // a row listed d times takes part in d passes (lists rarely repeat)
      group_stage(tail, tail + kTTileBytes, aq, times[0] > d, times[1] > d, times[2] > d, times[3] > d, ot, m0, l0, m1, l1, lt0, lt1);
#pragma unroll
    for (int off = 1; off <= 2; off <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, off);
      l1 += __shfl_xor_sync(0xffffffffu, l1, off);
      lt0 += __shfl_xor_sync(0xffffffffu, lt0, off);
      lt1 += __shfl_xor_sync(0xffffffffu, lt1, off);
    }
    if (tg == 0) {
      if (has0) { sm_m[k8Warps][g] = m0; sm_l[k8Warps][g] = l0; sm_lt[k8Warps][g] = lt0; }
      if (has1) { sm_m[k8Warps][g + 8] = m1; sm_l[k8Warps][g + 8] = l1; sm_lt[k8Warps][g + 8] = lt1; }
    }
#pragma unroll
    for (int nt = 0; nt < 16; ++nt) {
      if (has0) *reinterpret_cast<float2*>(&sm_o[(k8Warps * gq + g) * kHeadDim + nt * 8 + 2 * tg]) = make_float2(ot[nt][0], ot[nt][1]);
      if (has1) *reinterpret_cast<float2*>(&sm_o[(k8Warps * gq + g + 8) * kHeadDim + nt * 8 + 2 * tg]) = make_float2(ot[nt][2], ot[nt][3]);
    }
  }
  __syncthreads();
  const int slots = tail_live ? k8Warps + 1 : k8Warps;
  auto finish = [&](int unit, float acc, float M, float L, float Lt) {
    p.out[(long long)unit * kHeadDim + tid] = __float2bfloat16_rn(Lt > 0.f ? acc / Lt : 0.f);
    if (tid == 0 && p.out_lse) p.out_lse[unit] = L > 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
  };
  for (int j = 0; j < gq; ++j) {
    float M = -INFINITY;
    for (int w = 0; w < slots; ++w) M = fmaxf(M, sm_m[w][j]);
    float acc = 0.f, L = 0.f, Lt = 0.f;
    if (M != -INFINITY) {
      for (int w = 0; w < slots; ++w) {
        const float f = exp2f(sm_m[w][j] - M);
        acc = fmaf(sm_o[(w * gq + j) * kHeadDim + tid], f, acc);
        L = fmaf(sm_l[w][j], f, L);
        Lt = fmaf(sm_lt[w][j], f, Lt);
      }
    }
    if (p.splits == 1) {
      finish(unit0 + j, acc, M, L, Lt);
    } else {
      float* part = p.partials + ((long long)(unit0 + j) * p.splits + split) * kPartStride;
      part[tid] = acc;
      if (tid == 0) { part[kHeadDim] = M; part[kHeadDim + 1] = L; part[kHeadDim + 2] = Lt; }
    }
  }
  if (p.splits == 1) return;
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    const unsigned int ticket = atomicAdd(p.tickets + unit0, 1u);
    is_last = (ticket == (unsigned int)p.splits - 1u);
    if (is_last) p.tickets[unit0] = 0u;
  }
  __syncthreads();
  if (!is_last) return;
  __threadfence();
  for (int j = 0; j < gq; ++j) {
    const float* base = p.partials + (long long)(unit0 + j) * p.splits * kPartStride;
    float M = -INFINITY;
    for (int sp = 0; sp < p.splits; ++sp) M = fmaxf(M, __ldcg(base + sp * kPartStride + kHeadDim));
    float acc = 0.f, L = 0.f, Lt = 0.f;
    if (M != -INFINITY) {
      for (int sp = 0; sp < p.splits; ++sp) {
        const float f = exp2f(__ldcg(base + sp * kPartStride + kHeadDim) - M);
        acc = fmaf(__ldcg(base + sp * kPartStride + tid), f, acc);
        L = fmaf(__ldcg(base + sp * kPartStride + kHeadDim + 1), f, L);
        Lt = fmaf(__ldcg(base + sp * kPartStride + kHeadDim + 2), f, Lt);
      }
    }
    finish(unit0 + j, acc, M, L, Lt);
  }
}

}  // namespace prhs
