// Block-selected decode attention: a cheap score of every block of 16 positions against the query, the
// best blocks, and the attention over them.
//
// Bounds.  Of a block's keys the cache keeps, per KV head and coordinate, the minimum and the maximum, as
// int8 with one power-of-two scale per block: code = rint(x / s), s = 2^max(ceil(log2(amax / 127)), -126).
// 256 + 4 bytes stand for 4 KB of keys.
// Score.  q is coded the same way per head (q ~ s_q q8).  The largest value q . k can take for a key inside the
// (coded) bounds is
//   score = s_block s_q sum_d max(q8_d lo_d, q8_d hi_d) = s_block s_q (sum_d q8-_d lo_d + sum_d q8+_d hi_d),
// with q8+ = max(q8, 0), q8- = min(q8, 0): one integer product of length 256.  The sum is an integer below
// 2^24 and the scales are powers of two, so a score is exact whatever the order of the sum: equal scores are
// equal everywhere, and ties go to the lower block.
#pragma once
#include "attn.cuh"
#include "common.cuh"
#include "bytekv.cuh"

namespace prhs {

constexpr int kBoundsBytes = 2 * kHeadDim;          // minima, then maxima

// Device-side copy of a prhs_block_bounds_view: strides in blocks.
struct BoundsDev {
  int8_t* codes;
  float* scale;
  long long stride_outer, stride_head;
};

// ---------------------------------------------------------------------------------- bounds
// One warp, one block: bounds of the block's rows below `rows` (1..16) into codes / scale.  src: the block's
// first row.
__device__ __forceinline__ void bounds_of_block(const __nv_bfloat16* src, int rows, int8_t* codes, float* scale) {
  const int lane = threadIdx.x & 31;
  const int r0 = lane >> 4, col = (lane & 15) * 8;
  uint4 x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {               // rows past the end repeat row 0: no change to a minimum or maximum
    const int r = 2 * i + r0;
    x[i] = __ldg(reinterpret_cast<const uint4*>(src + (r < rows ? r : 0) * kHeadDim + col));
  }
  uint32_t lo[4], hi[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    auto word = [&](int i) { return j == 0 ? x[i].x : j == 1 ? x[i].y : j == 2 ? x[i].z : x[i].w; };
    uint32_t a = word(0), z = word(0);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      const uint32_t w = word(i);
      const __nv_bfloat162 wb = *reinterpret_cast<const __nv_bfloat162*>(&w);
      __nv_bfloat162 av = __hmin2(*reinterpret_cast<__nv_bfloat162*>(&a), wb), zv = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&z), wb);
      a = *reinterpret_cast<uint32_t*>(&av);
      z = *reinterpret_cast<uint32_t*>(&zv);
    }
    const uint32_t a2 = __shfl_xor_sync(0xffffffffu, a, 16), z2 = __shfl_xor_sync(0xffffffffu, z, 16);
    const __nv_bfloat162 av = __hmin2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&a2));
    const __nv_bfloat162 zv = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&z), *reinterpret_cast<const __nv_bfloat162*>(&z2));
    lo[j] = *reinterpret_cast<const uint32_t*>(&av);
    hi[j] = *reinterpret_cast<const uint32_t*>(&zv);
  }
  uint32_t mx = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) mx = __vmaxu2(mx, __vmaxu2(lo[j] & 0x7fff7fffu, hi[j] & 0x7fff7fffu));
  const uint32_t amax = __reduce_max_sync(0xffffffffu, max(mx & 0xffffu, mx >> 16));
  const int e = scale_exponent<6, 126>(amax);       // 127 = (1 + 126 / 128) 2^6
  const float inv = pow2i(-e);
  uint32_t c[2] = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w = lane < 16 ? lo[j] : hi[j];
    const uint32_t c0 = (uint32_t)__float2int_rn(bf_lo(w) * inv) & 0xffu, c1 = (uint32_t)__float2int_rn(bf_hi(w) * inv) & 0xffu;
    c[j >> 1] |= (c0 | (c1 << 8)) << (16 * (j & 1));
  }
  *reinterpret_cast<uint2*>(codes + lane * 8) = make_uint2(c[0], c[1]);    // lanes 0-15 the minima, 16-31 the maxima
  if (lane == 0) *scale = pow2i(e);
}

// Where block `blk` of (b, kvh) lies: rows and bounds.  false: a page id outside the pool.
__device__ __forceinline__ bool locate_block(const KvDev& kv, const BoundsDev& bd, int b, int kvh, int blk, long long& row_off,
                                             long long& bounds_idx) {
  long long outer = b, row = (long long)blk * (kBlockRows * kHeadDim), bi = blk;
  if (kv.page_table) {
    const int page = __ldg(kv.page_table + (long long)b * kv.page_table_stride + blk);
    if ((unsigned)page >= (unsigned)kv.num_pages) return false;
    outer = page; row = 0; bi = 0;
  }
  row_off = outer * kv.stride_outer + (long long)kvh * kv.stride_head + row;
  bounds_idx = outer * bd.stride_outer + (long long)kvh * bd.stride_head + bi;
  return true;
}

struct BoundsParams {
  KvDev kv;
  BoundsDev bd;
  const int* first;         // [B] or nullptr (0): bounds of the blocks that hold positions [first, t)
  int batch, num_kv_heads, blocks_max, max_len;     // blocks_max: blocks any sequence touches at most
  uint32_t* flags;
};

// One warp per block.  Bound by HBM: 4 KB of keys in, 260 B out per block.
__global__ void __launch_bounds__(256) block_bounds_kernel(BoundsParams p) {
  const long long item = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int j = (int)(item % p.blocks_max);
  const long long bh = item / p.blocks_max;
  if (bh >= (long long)p.batch * p.num_kv_heads) return;
  const int kvh = (int)(bh % p.num_kv_heads), b = (int)(bh / p.num_kv_heads);
  const int t = __ldg(p.kv.seq_lens + b);
  const int f = p.first ? __ldg(p.first + b) : 0;
  if (f < 0 || f > t || t > p.max_len || (t - f + kBlockRows - 1) / kBlockRows > p.blocks_max) {
    if ((threadIdx.x & 31) == 0) atomicOr(p.flags, kFlagBadLength);
    return;
  }
  const int blk = f / kBlockRows + j;
  if (f == t || blk * kBlockRows >= t) return;
  long long row, bi;
  if (!locate_block(p.kv, p.bd, b, kvh, blk, row, bi)) {
    if ((threadIdx.x & 31) == 0) atomicOr(p.flags, kFlagBadPage);
    return;
  }
  bounds_of_block(p.kv.k + row, min(kBlockRows, t - blk * kBlockRows), p.bd.codes + bi * kBoundsBytes, p.bd.scale + bi);
}

// ----------------------------------------------------------------------------------- score
struct BlockScoreParams {
  const __nv_bfloat16* q;   // [B][Hq][128]
  KvDev kv;
  BoundsDev bd;
  float* scores;            // [B][Hq][ld]; group_max: the row of the group's first head
  int ld, num_q_heads, group_size, group_max;
  int update_last;          // 1: the bounds of the last block are recomputed here (its score is not used)
  int max_len;
  uint32_t* flags;
};

__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The int8 codes of one head's query: this lane's words are dimensions 64h + 16tg + 4w .. + 3 (h, w in 0..1, 0..3).
// Returns the scale (0 for an absent head).
__device__ __forceinline__ float code_query(const __nv_bfloat16* q, bool has, uint32_t (&w)[2][4]) {
  const int tg = threadIdx.x & 3;
  uint4 x[2][2];
  uint32_t mx = 0u;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[h][i] = has ? __ldg(reinterpret_cast<const uint4*>(q + 64 * h + 16 * tg + 8 * i)) : make_uint4(0u, 0u, 0u, 0u);
      mx = __vmaxu2(__vmaxu2(mx, __vmaxu2(x[h][i].x & 0x7fff7fffu, x[h][i].y & 0x7fff7fffu)),
                    __vmaxu2(x[h][i].z & 0x7fff7fffu, x[h][i].w & 0x7fff7fffu));
    }
  uint32_t amax = max(mx & 0xffffu, mx >> 16);
  amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
  amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
  const int e = scale_exponent<6, 126>(amax);
  const float inv = pow2i(-e);
  auto code = [&](float v) { return (uint32_t)__float2int_rn(v * inv) & 0xffu; };
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[h][2 * i] = code(bf_lo(x[h][i].x)) | code(bf_hi(x[h][i].x)) << 8 | code(bf_lo(x[h][i].y)) << 16 | code(bf_hi(x[h][i].y)) << 24;
      w[h][2 * i + 1] = code(bf_lo(x[h][i].z)) | code(bf_hi(x[h][i].z)) << 8 | code(bf_lo(x[h][i].w)) << 16 | code(bf_hi(x[h][i].w)) << 24;
    }
  return has ? pow2i(e) : 0.f;
}

// grid (chunks of kScoreBlocks blocks, Hkv, B).  A warp takes eight blocks at a time as the columns of
// mma.sync m16n8k32 (int8 in, int32 accumulate) with the group's heads on the rows.  The B fragments come
// straight from global memory: lane (g, tg) loads the four 16-byte pieces 4i + tg of block g's 256 bytes (64
// contiguous bytes per block and instruction) and deals their words to the k-slots as they lie; the query's
// fragments are dealt the same way.  No shared memory, eight MMAs per 2 KB.  Bound by the stream of bounds.
constexpr int kScoreWarps = 4;
constexpr int kScoreTiles = 4;                                   // tiles of eight blocks per warp
constexpr int kScoreBlocks = kScoreWarps * kScoreTiles * 8;      // 128 blocks, 32 KB of bounds per CTA
__global__ void __launch_bounds__(kScoreWarps * 32) block_score_kernel(BlockScoreParams p) {
  const int kvh = blockIdx.y, b = blockIdx.z;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, tg = lane & 3;
  const int gq = p.group_size, head0 = kvh * gq;
  const int t = __ldg(p.kv.seq_lens + b);
  if (t > p.max_len || t < 0) {
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(p.flags, kFlagBadLength);
    return;
  }
  const int nb = (t + kBlockRows - 1) / kBlockRows;
  if (p.update_last && blockIdx.x == 0 && warp == kScoreWarps - 1 && nb > 0) {
    long long row, bi;
    if (locate_block(p.kv, p.bd, b, kvh, nb - 1, row, bi))
      bounds_of_block(p.kv.k + row, t - (nb - 1) * kBlockRows, p.bd.codes + bi * kBoundsBytes, p.bd.scale + bi);
    else if (lane == 0)
      atomicOr(p.flags, kFlagBadPage);
  }
  const int base = (blockIdx.x * kScoreWarps + warp) * (kScoreTiles * 8);
  if (base >= nb) return;
  // where the blocks of this warp lie: bounds index of block base + lane (32 = kScoreTiles * 8 blocks)
  static_assert(kScoreTiles * 8 == 32, "one block per lane");
  long long bi = -1;
  if (base + lane < nb) {
    long long row;
    if (!locate_block(p.kv, p.bd, b, kvh, base + lane, row, bi)) {
      atomicOr(p.flags, kFlagBadPage);
      bi = -1;
    }
  }
  const float my_scale = bi >= 0 ? p.bd.scale[bi] : 0.f;
  uint4 x[kScoreTiles][4];
#pragma unroll
  for (int n = 0; n < kScoreTiles; ++n) {
    const long long at = __shfl_sync(0xffffffffu, bi, 8 * n + g);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[n][i] = at >= 0 ? *reinterpret_cast<const uint4*>(p.bd.codes + at * kBoundsBytes + (4 * i + tg) * 16) : make_uint4(0u, 0u, 0u, 0u);
  }
  const __nv_bfloat16* q0 = p.q + ((long long)b * p.num_q_heads + head0 + g) * kHeadDim;
  const bool has0 = g < gq, has1 = g + 8 < gq;
  uint32_t w0[2][4], w1[2][4];
  const float qs0 = code_query(q0, has0, w0);
  const float qs1 = code_query(q0 + 8 * kHeadDim, has1, w1);
#pragma unroll
  for (int n = 0; n < kScoreTiles; ++n) {
    if (base + 8 * n >= nb) break;
    int d[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int h = i & 1;                       // pieces 0, 1: minima of dimensions 64h..; 2, 3: maxima
      auto part = [&](uint32_t w) { return i < 2 ? __vmins4(w, 0u) : __vmaxs4(w, 0u); };
      mma_s8(d, part(w0[h][0]), part(w1[h][0]), part(w0[h][1]), part(w1[h][1]), x[n][i].x, x[n][i].y);
      mma_s8(d, part(w0[h][2]), part(w1[h][2]), part(w0[h][3]), part(w1[h][3]), x[n][i].z, x[n][i].w);
    }
    const int blk = base + 8 * n + 2 * tg;
    const float s0 = __shfl_sync(0xffffffffu, my_scale, 8 * n + 2 * tg), s1 = __shfl_sync(0xffffffffu, my_scale, 8 * n + 2 * tg + 1);
    float v[4] = {(float)d[0] * s0 * qs0, (float)d[1] * s1 * qs0, (float)d[2] * s0 * qs1, (float)d[3] * s1 * qs1};
    if (p.group_max) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float m = fmaxf(has0 ? v[c] : -INFINITY, has1 ? v[2 + c] : -INFINITY);
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
        v[c] = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
      }
    }
    auto store = [&](int head, float a, float z) {
      float* dst = p.scores + ((long long)b * p.num_q_heads + head0 + head) * p.ld + blk;
      if (blk + 1 < nb) *reinterpret_cast<float2*>(dst) = make_float2(a, z);
      else if (blk < nb) *dst = a;
    };
    if (p.group_max ? g == 0 : has0) store(g, v[0], v[1]);
    if (!p.group_max && has1) store(g + 8, v[2], v[3]);
  }
}

// ---------------------------------------------------------------------------------- select
struct BlockSelectParams {
  const float* scores;      // [B][Hq][ld]
  int ld, num_q_heads, units_per_seq, heads_per_unit;
  const int* seq_lens;
  int top, sink, recent;
  int* out_blocks;          // [B][units_per_seq][stride], ascending, -1 past the count
  int stride;
  int* out_count;
  int max_len;
};

// One CTA per unit (a query head, or a KV head where the group shares a set).  The unit attends over blocks
// [0, lo), the `top` best of [lo, hi), and [hi, nb).  The threshold is found by narrowing an interval of keys
// (the scores' order-preserving 32-bit images): a histogram of 1024 equal bins over the interval says which
// bin the top-th key lies in; that bin is the next interval, until it is one key wide.  Scores of one unit lie
// close together, so bins over their own range spread them (bins over the leading bits would not, and the
// shared-memory atomics would serialise).  Then one ordered pass writes the list.
constexpr int kBSThreads = 512;
constexpr int kBSBins = 1024;
__global__ void __launch_bounds__(kBSThreads) block_select_kernel(BlockSelectParams p) {
  constexpr int kW = kBSThreads / 32;
  __shared__ int hist[kBSBins];
  __shared__ uint32_t red_lo[kW], red_hi[kW];
  __shared__ int warp_gt[kW], warp_eq[kW];
  __shared__ uint32_t sh_base, sh_span;
  __shared__ int sh_need;
  const int unit = blockIdx.x;
  const int b = unit / p.units_per_seq, u = unit % p.units_per_seq;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t = min(max(__ldg(p.seq_lens + b), 0), p.max_len);
  const int nb = (t + kBlockRows - 1) / kBlockRows;
  const int lo = min(p.sink, nb), hi = max(lo, nb - p.recent);
  const int need0 = min(p.top, hi - lo);
  const int total = lo + need0 + nb - hi;
  const float* s = p.scores + ((long long)b * p.num_q_heads + u * p.heads_per_unit) * p.ld;
  int* out = p.out_blocks + (long long)unit * p.stride;
  for (int i = tid; i < p.stride; i += kBSThreads) {
    if (i < lo) out[i] = i;
    else if (i >= total) out[i] = -1;
    else if (i >= lo + need0) out[i] = hi + (i - lo - need0);
  }
  if (tid == 0) p.out_count[unit] = total;
  if (need0 == 0) return;
  // the threshold: keys above `thr` are taken, and the first `need` (by position) of those equal to it
  uint32_t thr = 0u;
  int need = need0;
  if (need0 < hi - lo) {
    uint32_t kmin = 0xffffffffu, kmax = 0u;
    for (int i = lo + tid; i < hi; i += kBSThreads) {
      const uint32_t k = float_to_key(__ldg(s + i));
      kmin = min(kmin, k);
      kmax = max(kmax, k);
    }
    kmin = __reduce_min_sync(0xffffffffu, kmin);
    kmax = __reduce_max_sync(0xffffffffu, kmax);
    if (lane == 0) { red_lo[warp] = kmin; red_hi[warp] = kmax; }
    __syncthreads();
    for (int w = 0; w < kW; ++w) { kmin = min(kmin, red_lo[w]); kmax = max(kmax, red_hi[w]); }
    uint32_t base = kmin, span = kmax - kmin;        // the interval [base, base + span]
    while (span > 0u) {
      const int shift = max(0, 32 - __clz(span) - 10);   // (key - base) >> shift < 1024
      for (int i = tid; i < kBSBins; i += kBSThreads) hist[i] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += kBSThreads) {
        const uint32_t k = float_to_key(__ldg(s + i)) - base;
        if (k <= span) atomicAdd(&hist[k >> shift], 1);
      }
      __syncthreads();
      // warp 0 walks the bins from the top: lane l owns bins 1023 - 32 l .. 992 - 32 l
      if (warp == 0) {
        int sum = 0;
        for (int i = 0; i < 32; ++i) sum += hist[kBSBins - 1 - (32 * lane + i)];
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, incl, off);
          if (lane >= off) incl += v;
        }
        int above = incl - sum;
        if (above < need && incl >= need) {              // exactly one lane
          int bin = kBSBins - 1 - 32 * lane;
          while (above + hist[bin] < need) above += hist[bin--];
          sh_base = base + ((uint32_t)bin << shift);
          sh_span = min((1u << shift) - 1u, span - ((uint32_t)bin << shift));
          sh_need = need - above;
        }
      }
      __syncthreads();
      base = sh_base;
      span = sh_span;
      need = sh_need;
      __syncthreads();
    }
    thr = base;
  }
  const bool all = need0 == hi - lo;
  // ordered pass: every warp owns a run of positions; counts first, then places
  const int run = ((hi - lo + kW - 1) / kW + 31) & ~31;
  const int from = lo + warp * run, to = min(from + run, hi);
  int gt = 0, eq = 0;
  for (int i = from; i < to; i += 32) {
    const uint32_t k = i + lane < to ? float_to_key(__ldg(s + i + lane)) : 0u;
    const bool in = i + lane < to;
    gt += __popc(__ballot_sync(0xffffffffu, in && (all || k > thr)));
    eq += __popc(__ballot_sync(0xffffffffu, in && !all && k == thr));
  }
  if (lane == 0) { warp_gt[warp] = gt; warp_eq[warp] = eq; }
  __syncthreads();
  int eq_before = 0, place = lo;
  for (int w = 0; w < warp; ++w) {
    place += warp_gt[w] + max(0, min(warp_eq[w], need - eq_before));
    eq_before += warp_eq[w];
  }
  for (int i = from; i < to; i += 32) {
    const bool in = i + lane < to;
    const uint32_t k = in ? float_to_key(__ldg(s + i + lane)) : 0u;
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t eqm = __ballot_sync(0xffffffffu, in && !all && k == thr);
    const bool take = in && (all || k > thr || (k == thr && eq_before + __popc(eqm & below) < need));
    const uint32_t tm = __ballot_sync(0xffffffffu, take);
    if (take) out[place + __popc(tm & below)] = i + lane;
    place += __popc(tm);
    eq_before += __popc(eqm);
  }
}

// ------------------------------------------------------------------------------- attention
// Attention over listed blocks of a bf16 cache.  kGroup: one list per KV head, its heads on the rows of the MMA
// tile (the arithmetic of the dense kernel); else one list per query head.  grid (splits, units per
// sequence, B).  A stage of the warp-private ring is one block, whose rows are contiguous; rows past the
// end of the sequence are masked.  Partials, tickets and merge as in the dense kernel.
struct BlockAttnParams {
  AttnParams a;             // q, kv, splits, partials, tickets, out, out_lse, flags; set and idx unused
  const int* blocks;        // [B][units][stride]
  const int* count;
  int stride, units_per_seq;
};

__global__ void __launch_bounds__(kTThreads) block_attn_kernel(BlockAttnParams bp) {
  extern __shared__ __align__(128) unsigned char g_smem[];
  const AttnParams& p = bp.a;
  const int split = blockIdx.x, u = blockIdx.y, b = blockIdx.z;
  const bool shared = bp.units_per_seq * p.group_size == p.num_q_heads && p.group_size > 1;
  const int gq = shared ? p.group_size : 1;
  const int head0 = u * gq, kvh = shared ? u : u / p.group_size;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, tg = lane & 3;
  const int t = __ldg(p.kv.seq_lens + b);
  const int nb = (t + kBlockRows - 1) / kBlockRows;
  const long long unit = (long long)b * bp.units_per_seq + u;
  const int* list = bp.blocks + unit * bp.stride;
  const int cnt = min(max(__ldg(bp.count + unit), 0), bp.stride);
  const int per = (cnt + p.splits * kTWarps - 1) / (p.splits * kTWarps);
  const int start = min((split * kTWarps + warp) * per, cnt);
  const int nstages = min(start + per, cnt) - start;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(g_smem) + warp * (kTStages * kTStageBytes);
  const bool has0 = g < gq, has1 = g + 8 < gq;

  uint32_t aq[8][4];
  {
    const uint32_t* q0 = reinterpret_cast<const uint32_t*>(p.q + ((long long)b * p.num_q_heads + head0 + g) * kHeadDim);
    const uint32_t* q1 = q0 + 8 * (kHeadDim / 2);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      aq[ks][0] = has0 ? __ldg(q0 + ks * 8 + tg) : 0u;
      aq[ks][1] = has1 ? __ldg(q1 + ks * 8 + tg) : 0u;
      aq[ks][2] = has0 ? __ldg(q0 + ks * 8 + 4 + tg) : 0u;
      aq[ks][3] = has1 ? __ldg(q1 + ks * 8 + 4 + tg) : 0u;
    }
  }
  float o[16][4];
#pragma unroll
  for (int nt = 0; nt < 16; ++nt) { o[nt][0] = 0.f; o[nt][1] = 0.f; o[nt][2] = 0.f; o[nt][3] = 0.f; }
  float m0 = -INFINITY, l0 = 0.f, m1 = -INFINITY, l1 = 0.f, lt0 = 0.f, lt1 = 0.f;

  // block numbers and page ids of 32 list entries, one per lane, a group ahead of their use
  auto entry = [&](int grp) -> int {
    const int j = grp * 32 + lane;
    if (j >= nstages) return -1;
    const int blk = __ldg(list + start + j);
    if ((unsigned)blk >= (unsigned)nb) {
      atomicOr(p.flags, kFlagBadIndex);
      return -1;
    }
    return blk;
  };
  const bool paged = p.kv.page_table != nullptr;
  auto page_of = [&](int blk) -> int {
    return (paged && blk >= 0) ? __ldg(p.kv.page_table + (long long)b * p.kv.page_table_stride + blk) : 0;
  };
  int blk_cur = entry(0), pg_cur = page_of(blk_cur);
  int blk_next = entry(1), pg_next = page_of(blk_next);

  const __nv_bfloat16* src_base = (lane < 16 ? p.kv.k : p.kv.v) + (lane & 15) * 8;
  const uint32_t dst_tile = (lane < 16 ? 0u : (uint32_t)kTTileBytes);
  const long long lin = (long long)b * p.kv.stride_outer + (long long)kvh * p.kv.stride_head;
  int rows_of[kTStages];                   // real rows per ring slot (slots are compile-time below)
  auto issue = [&](int j, auto slot_c) {
    constexpr int kSlot = decltype(slot_c)::value;
    if (j < nstages) {
      if (j > 0 && (j & 31) == 0) {
        blk_cur = blk_next; pg_cur = pg_next;
        blk_next = entry((j >> 5) + 1);
        pg_next = page_of(blk_next);
      }
      const int blk = __shfl_sync(0xffffffffu, blk_cur, j & 31);
      const int page = __shfl_sync(0xffffffffu, pg_cur, j & 31);
      int rows = blk >= 0 ? min(kBlockRows, t - blk * kBlockRows) : 0;
      if (paged && rows > 0 && (unsigned)page >= (unsigned)p.kv.num_pages) {
        if (lane == 0) atomicOr(p.flags, kFlagBadPage);
        rows = 0;
      }
      const long long off = rows == 0 ? 0ll : paged ? (long long)page * p.kv.stride_outer + (long long)kvh * p.kv.stride_head
                                                    : lin + (long long)blk * (kBlockRows * kHeadDim);
      const uint32_t slot = ring + (uint32_t)kSlot * kTStageBytes + dst_tile;
#pragma unroll
      for (int r = 0; r < kTStageRows; ++r) {
        const uint32_t dst = slot + r * kRowBytes + ((((uint32_t)lane & 15u) ^ (r & 7u)) << 4);
        cp_async_16(dst, src_base + (r < rows ? off + (long long)r * kHeadDim : 0ll), r < rows ? 16 : 0);
      }
      rows_of[kSlot] = rows;
    }
    cp_async_commit();
  };
  issue(0, SlotC<0>{});
  issue(1, SlotC<1>{});
  auto stage = [&](int i, auto slot_c) {
    constexpr int kSlot = decltype(slot_c)::value;
    cp_async_wait<kTStages - 2>();
    __syncwarp();
    const int rows = rows_of[kSlot];
    issue(i + kTStages - 1, SlotC<(kSlot + kTStages - 1) % kTStages>{});
    if (rows == 0) return;
    const uint32_t kt = ring + (uint32_t)kSlot * kTStageBytes;
    group_stage(kt, kt + kTTileBytes, aq, 2 * tg < rows, 2 * tg + 1 < rows, 8 + 2 * tg < rows, 9 + 2 * tg < rows, o, m0, l0,
                m1, l1, lt0, lt1);
  };
  int i = 0;
  for (; i + 2 < nstages; i += 3) {
    stage(i, SlotC<0>{});
    stage(i + 1, SlotC<1>{});
    stage(i + 2, SlotC<2>{});
  }
  if (i < nstages) stage(i, SlotC<0>{});
  if (i + 1 < nstages) stage(i + 1, SlotC<1>{});
  cp_async_wait<0>();
  group_epilogue(p, g_smem, b, head0, gq, split, o, m0, l0, m1, l1, lt0, lt1);
}

}  // namespace prhs
