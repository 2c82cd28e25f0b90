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
#include "head_tiles.cuh"

namespace prhs {

constexpr int kBoundsBytes = 2 * kHeadDim;          // minima, then maxima

// Device-side copy of a prhs_block_bounds_view: strides in blocks.
struct BoundsDev {
  int8_t* codes;
  float* scale;
  long long stride_outer, stride_head;
};

// ---------------------------------------------------------------------------------- bounds
// The code of a number in units of its scale; infinities have the largest.
__device__ __forceinline__ int code_of(float x, float inv) { return min(max(__float2int_rn(x * inv), -127), 127); }

// One warp, one block: bounds of the block's rows below `rows` (1..16) into codes / scale.  src: the block's
// first row.  NaNs are left out (a coordinate of NaNs only counts as zero).  Returns whether every element was finite.
__device__ __forceinline__ bool bounds_of_block(const __nv_bfloat16* src, int rows, int8_t* codes, float* scale) {
  const int lane = threadIdx.x & 31;
  const int r0 = lane >> 4, col = (lane & 15) * 8;
  uint32_t lo[4], hi[4];
  // minima and maxima, and the largest magnitude of the block as bf16 bits; kNaN: one NaN makes its coordinate NaN
  auto fold = [&](auto nan_c) -> uint32_t {
    constexpr bool kNaN = decltype(nan_c)::value != 0;
    auto low = [](uint32_t a, uint32_t b) {
      const __nv_bfloat162 x = *reinterpret_cast<__nv_bfloat162*>(&a), y = *reinterpret_cast<__nv_bfloat162*>(&b);
      const __nv_bfloat162 z = kNaN ? __hmin2_nan(x, y) : __hmin2(x, y);
      return *reinterpret_cast<const uint32_t*>(&z);
    };
    auto high = [](uint32_t a, uint32_t b) {
      const __nv_bfloat162 x = *reinterpret_cast<__nv_bfloat162*>(&a), y = *reinterpret_cast<__nv_bfloat162*>(&b);
      const __nv_bfloat162 z = kNaN ? __hmax2_nan(x, y) : __hmax2(x, y);
      return *reinterpret_cast<const uint32_t*>(&z);
    };
    uint4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {             // rows past the end repeat row 0: no change to a minimum or maximum
      const int r = 2 * i + r0;
      x[i] = __ldg(reinterpret_cast<const uint4*>(src + (r < rows ? r : 0) * kHeadDim + col));
    }
    uint32_t mx = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      auto word = [&](int i) { return j == 0 ? x[i].x : j == 1 ? x[i].y : j == 2 ? x[i].z : x[i].w; };
      uint32_t a = word(0), z = word(0);
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        a = low(a, word(i));
        z = high(z, word(i));
      }
      lo[j] = low(a, __shfl_xor_sync(0xffffffffu, a, 16));
      hi[j] = high(z, __shfl_xor_sync(0xffffffffu, z, 16));
      if (!kNaN) {
        lo[j] &= ~__vcmpgtu2(lo[j] & 0x7fff7fffu, 0x7f807f80u);
        hi[j] &= ~__vcmpgtu2(hi[j] & 0x7fff7fffu, 0x7f807f80u);
      }
      mx = __vmaxu2(mx, __vmaxu2(lo[j] & 0x7fff7fffu, hi[j] & 0x7fff7fffu));
    }
    return __reduce_max_sync(0xffffffffu, max(mx & 0xffffu, mx >> 16));
  };
  uint32_t amax = fold(SlotC<1>{});
  const bool finite = amax < 0x7f80u;
  if (amax > 0x7f80u) amax = fold(SlotC<0>{});      // (read again: that is rare)
  const int e = scale_exponent<6, 126>(amax);       // 127 = (1 + 126 / 128) 2^6
  const float inv = pow2i(-e);
  uint32_t c[2] = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w = lane < 16 ? lo[j] : hi[j];
    const uint32_t c0 = (uint32_t)code_of(bf_lo(w), inv) & 0xffu, c1 = (uint32_t)code_of(bf_hi(w), inv) & 0xffu;
    c[j >> 1] |= (c0 | (c1 << 8)) << (16 * (j & 1));
  }
  *reinterpret_cast<uint2*>(codes + lane * 8) = make_uint2(c[0], c[1]);    // lanes 0-15 the minima, 16-31 the maxima
  if (lane == 0) *scale = pow2i(e);
  return finite;
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
  int max_len, max_new;     // t and t - first of any sequence at most
  uint32_t* flags;
};

// One warp per block, grid (blocks, Hkv, B).  Bound by HBM: 4 KB of keys in, 260 B out per block.
__global__ void __launch_bounds__(256) block_bounds_kernel(BoundsParams p) {
  const int j = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), kvh = blockIdx.y, b = blockIdx.z;
  const int t = __ldg(p.kv.seq_lens + b);
  const int f = p.first ? __ldg(p.first + b) : 0;
  if (f < 0 || f > t || t > p.max_len || t - f > p.max_new) {
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
  const bool finite = bounds_of_block(p.kv.k + row, min(kBlockRows, t - blk * kBlockRows), p.bd.codes + bi * kBoundsBytes, p.bd.scale + bi);
  if (!finite && (threadIdx.x & 31) == 0) atomicOr(p.flags, kFlagNonFinite);
}

// ----------------------------------------------------------------------------------- score
struct BlockScoreParams {
  const __nv_bfloat16* q;   // [B][Hq][128]
  KvDev kv;
  BoundsDev bd;
  int bounds_outer, bounds_head;   // bd's strides: a bounds index (256 bytes) fits 31 bits on any device
  float* scores;            // [B][Hq][ld]; group_max: the row of the group's first head
  int ld, batch, num_q_heads, group_size, group_max;
  int max_len;
  uint32_t* flags;
};

__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Programmatic dependent launch: a kernel of a step is launched while the one before it still runs, does what
// does not depend on it, and waits here.  Every CTA waits, those without work too, so that a kernel that has
// ended means that all before it have.
__device__ __forceinline__ void step_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void step_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// A warp takes eight blocks at a time as the columns of mma.sync m16n8k32 (int8 in, int32
// accumulate) with the group's heads on the rows (kWide: more than eight).  The bounds come through a
// warp-private cp.async ring of 16 blocks (4 KB) per stage; lane (g, tg) reads the four 16-byte pieces 4i + tg of
// block g's 256 bytes and deals their words to the k-slots as they lie, and the query's fragments are dealt the
// same way: sixteen MMAs and eight shared-memory loads per 4 KB.  The groups of 16 blocks of all units, laid end to
// end, are dealt to one wave of CTAs in equal runs (a run may cross into the next unit: then the query is coded
// again).  One CTA column per unit instead waited for the longest of ragged sequences (16 of 8K to 64K: 27 us
// for 75 MB); a dozen short CTAs per unit with register prefetch took 35 us for 137 MB against 27 us.  Bound by
// the stream of bounds.
constexpr int kScoreWarps = 4;
constexpr int kScoreRound = 16;                                  // blocks per stage
constexpr int kScoreStages = 4;
constexpr int kScoreStageBytes = kScoreRound * kBoundsBytes + kScoreRound * 4;
constexpr int kScoreSmemBytes = kScoreWarps * kScoreStages * kScoreStageBytes;      // 65 KB: three CTAs per SM
constexpr int kScoreCtasPerSm = 3;
// Registers of a thread: three CTAs leave room for one of the selection's beside them (40 x 512), which so is there when
// the scores are.  Without it selecting CTAs crowd onto the SMs that are free first: 16 ragged sequences of up to 64K,
// 128 sets, 51.9 us a step, not 49.9.
constexpr int kScoreRegs = 112;
static_assert(kScoreCtasPerSm * kScoreWarps * 32 * kScoreRegs + 40 * 512 <= 65536, "no room for a selection's CTA");
template <bool kWide>
__global__ void __launch_bounds__(kScoreWarps * 32) __maxnreg__(kWide ? 168 : kScoreRegs) block_score_kernel(BlockScoreParams p) {
  constexpr int kHeads = kWide ? 16 : 8;
  extern __shared__ __align__(128) unsigned char g_smem[];
  __shared__ __align__(16) uint8_t qcodes[kHeads][2][kHeadDim];   // negative part (meets the minima), positive part
  __shared__ float qscale[kHeads];
  step_release();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, tg = lane & 3;
  const int gq = p.group_size, num_kv = p.num_q_heads / gq;
  const bool paged = p.kv.page_table != nullptr;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(g_smem) + warp * (kScoreStages * kScoreStageBytes);

  // this CTA's run of groups and the unit it begins in; an impossible length is cut, as the selection cuts it
  const int max_len = p.max_len;
  auto length_of = [max_len](int t) { return min(max(t, 0), max_len); };
  auto groups_of = [length_of](int t) { return (length_of(t) + kScoreRound * kBlockRows - 1) / (kScoreRound * kBlockRows); };
  int b = 0, at = 0;
  const int total = count_items(p.kv.seq_lens, p.batch, num_kv, groups_of);
  const int share = max((total + (int)gridDim.x - 1) / (int)gridDim.x, kScoreWarps);
  if (blockIdx.x == 0)
    for (int i = tid; i < p.batch; i += kScoreWarps * 32)
      if (__ldg(p.kv.seq_lens + i) > max_len || __ldg(p.kv.seq_lens + i) < 0) atomicOr(p.flags, kFlagBadLength);
  if ((long long)blockIdx.x * share >= total) return;
  at = blockIdx.x * share;
  const int run_end = min(at + share, total);
  int before = 0;
  find_item(p.kv.seq_lens, p.batch, num_kv, groups_of, at, &b, &before);
  int groups = groups_of(__ldg(p.kv.seq_lens + b));
  int kvh = (at - before) / groups;
  int g_lo = at - before - kvh * groups;

  while (true) {                                       // units of the run
    const int head0 = kvh * gq;
    const int nb = (length_of(__ldg(p.kv.seq_lens + b)) + kBlockRows - 1) / kBlockRows;
    const int g_hi = min(groups, g_lo + run_end - at);
    const int rounds = max(0, (g_hi - g_lo - warp + kScoreWarps - 1) / kScoreWarps);     // groups g_lo + warp + 4r
    const int* ptab = p.kv.page_table + (long long)b * p.kv.page_table_stride;
    auto page_of = [&](int r) -> int {                   // lanes 0..15: the page of block lane of round r
      const int blk = (g_lo + warp + kScoreWarps * r) * kScoreRound + (lane & 15);
      return (paged && r < rounds && blk < nb) ? __ldg(ptab + blk) : 0;
    };
    int pg_next = page_of(0);
    const int outer = p.bounds_outer, unit_at = (paged ? 0 : b * outer) + kvh * p.bounds_head;       // bounds indexes
    // a lane copies chunk lane % 16 of every other block of the group; the swizzle depends on the block's parity
    const int c = lane & 15, half = lane >> 4;
    const uint32_t dst_lane = half * kBoundsBytes + ((c ^ (half << 2)) << 4);
    const int8_t* const src_lane = p.bd.codes + c * 16;
    auto issue = [&](int r) {
      if (r < rounds) {
        const int blk0 = (g_lo + warp + kScoreWarps * r) * kScoreRound;
        const uint32_t slot = ring + (uint32_t)(r % kScoreStages) * kScoreStageBytes;
        if (!paged && blk0 + kScoreRound <= nb) {        // 4 KB in a row
          const int8_t* src = src_lane + (long long)(unit_at + blk0 + half) * kBoundsBytes;
#pragma unroll
          for (int i = 0; i < 8; ++i) cp_async_16_full(slot + dst_lane + i * (2 * kBoundsBytes), src + i * (2 * kBoundsBytes));
          if (lane < 16) cp_async_4(slot + kScoreRound * kBoundsBytes + lane * 4, p.bd.scale + unit_at + blk0 + lane, 4);
        } else {
          int at = -1;                                   // bounds index of block lane % 16
          if (blk0 + c < nb) {
            if (!paged) at = unit_at + blk0 + c;
            else if ((unsigned)pg_next < (unsigned)p.kv.num_pages) at = pg_next * outer + unit_at;
            else atomicOr(p.flags, kFlagBadPage);
          }
          pg_next = page_of(r + 1);
          const bool all = __all_sync(0xffffffffu, at >= 0);
          if (all) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              cp_async_16_full(slot + dst_lane + i * (2 * kBoundsBytes),
                               src_lane + (long long)__shfl_sync(0xffffffffu, at, 2 * i + half) * kBoundsBytes);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int from = __shfl_sync(0xffffffffu, at, 2 * i + half);
              cp_async_16(slot + dst_lane + i * (2 * kBoundsBytes), src_lane + (long long)max(from, 0) * kBoundsBytes, from >= 0 ? 16 : 0);
            }
          }
          if (lane < 16) cp_async_4(slot + kScoreRound * kBoundsBytes + lane * 4, p.bd.scale + max(at, 0), at >= 0 ? 4 : 0);
        }
      }
      cp_async_commit();
    };
#pragma unroll
    for (int r = 0; r < kScoreStages - 1; ++r) issue(r);

    // ---- the group's query codes: sixteen threads per head, eight dimensions each
#pragma unroll
    for (int h0 = 0; h0 < kHeads; h0 += 8) {
      const int h = h0 + (tid >> 4), d = (tid & 15) * 8;
      const uint4 x = h < gq ? __ldg(reinterpret_cast<const uint4*>(p.q + ((long long)b * p.num_q_heads + head0 + h) * kHeadDim + d))
                             : make_uint4(0u, 0u, 0u, 0u);
      const uint32_t mx = __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
      uint32_t amax = max(mx & 0xffffu, mx >> 16);
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, off));
      const int e = scale_exponent<6, 126>(amax);
      const float inv = pow2i(-e);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
      uint32_t neg[2] = {0u, 0u}, pos[2] = {0u, 0u};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int code = code_of(j & 1 ? bf_hi(w[j >> 1]) : bf_lo(w[j >> 1]), inv);
        neg[j >> 2] |= ((uint32_t)min(code, 0) & 0xffu) << (8 * (j & 3));
        pos[j >> 2] |= (uint32_t)max(code, 0) << (8 * (j & 3));
      }
      *reinterpret_cast<uint2*>(&qcodes[h][0][d]) = make_uint2(neg[0], neg[1]);
      *reinterpret_cast<uint2*>(&qcodes[h][1][d]) = make_uint2(pos[0], pos[1]);
      if ((tid & 15) == 0) qscale[h] = h < gq ? pow2i(e) : 0.f;
    }
    __syncthreads();
    const bool has0 = g < gq, has1 = kWide && g + 8 < gq;
    uint4 q0[4], q1[4];                                  // heads g and g + 8: pieces 4i + tg
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q0[i] = *reinterpret_cast<const uint4*>(&qcodes[g][i >> 1][64 * (i & 1) + 16 * tg]);
      q1[i] = kWide ? *reinterpret_cast<const uint4*>(&qcodes[(g + 8) & (kHeads - 1)][i >> 1][64 * (i & 1) + 16 * tg]) : make_uint4(0u, 0u, 0u, 0u);
    }
    const float qs0 = qscale[g], qs1 = kWide ? qscale[(g + 8) & (kHeads - 1)] : 0.f;
    float* const row0 = p.scores + ((long long)b * p.num_q_heads + head0 + (p.group_max ? 0 : g)) * p.ld;

    for (int r = 0; r < rounds; ++r) {
      cp_async_wait<kScoreStages - 2>();
      __syncwarp();
      issue(r + kScoreStages - 1);
      const unsigned char* slot = g_smem + (warp * kScoreStages + r % kScoreStages) * kScoreStageBytes;
      const float* scales = reinterpret_cast<const float*>(slot + kScoreRound * kBoundsBytes);
      // four chains of four MMAs: two tiles of eight blocks, minima and maxima apart
      int d[2][2][4] = {};
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const int c = 2 * part + i;
            const uint4 x = *reinterpret_cast<const uint4*>(slot + (8 * n + g) * kBoundsBytes + (((4 * c + tg) ^ ((g & 1) << 2)) << 4));
            mma_s8(d[n][part], q0[c].x, q1[c].x, q0[c].y, q1[c].y, x.x, x.y);
            mma_s8(d[n][part], q0[c].z, q1[c].z, q0[c].w, q1[c].w, x.z, x.w);
          }
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int blk = (g_lo + warp + kScoreWarps * r) * kScoreRound + 8 * n + 2 * tg;
        const float2 s = *reinterpret_cast<const float2*>(scales + 8 * n + 2 * tg);
        auto sum = [&](int j) { return (float)(d[n][0][j] + d[n][1][j]); };
        float v[4] = {sum(0) * s.x * qs0, sum(1) * s.y * qs0, sum(2) * s.x * qs1, sum(3) * s.y * qs1};
        if (p.group_max) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float m = fmaxf(has0 ? v[c] : -INFINITY, has1 ? v[2 + c] : -INFINITY);
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            v[c] = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
          }
        }
        auto store = [&](float* row, float a, float z) {
          if (blk + 1 < nb) *reinterpret_cast<float2*>(row + blk) = make_float2(a, z);
          else if (blk < nb) row[blk] = a;
        };
        if (p.group_max ? g == 0 : has0) store(row0, v[0], v[1]);
        if (kWide && !p.group_max && has1) store(row0 + 8ll * p.ld, v[2], v[3]);
      }
    }
    cp_async_wait<0>();
    at += g_hi - g_lo;
    if (at >= run_end) return;
    g_lo = 0;
    if (++kvh == num_kv) {                               // the next sequence that has blocks
      kvh = 0;
      do groups = groups_of(__ldg(p.kv.seq_lens + ++b));
      while (groups == 0);
    }
    __syncthreads();                                     // the query's codes are written again
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

// The unit (a query head, or a KV head where the group shares a set) attends over blocks [0, lo), the `top` best of
// [lo, hi), and [hi, nb).  Selection of the middle by one CTA of kThreads: the scores are read once into registers
// (kKeys per thread; kKeys = 0 reads them again in every pass).  The threshold is found by narrowing an interval of
// keys (the scores' order-preserving 32-bit images): a histogram of 2 kThreads equal bins over the interval says which
// bin the top-th key lies in, and that bin is the next interval.  Scores of one unit lie close together, so bins over
// their own range spread them (bins over the leading bits would not, and the shared-memory atomics would serialise).
// With at most 32 keys left in the bin, a warp ranks them directly; that is usually after one histogram.  Then one
// ordered pass hands out the list, put(place, block) in ascending order.
template <int kThreads>
struct SelectSmem {
  int hist[2 * kThreads];                          // zero before and after
  uint32_t red_lo[kThreads / 32], red_hi[kThreads / 32], cand[32];
  int warp_a[kThreads / 32], warp_b[kThreads / 32];
  uint32_t base, span;
  int need, count, cands;                          // cands: zero before
};
template <int kThreads, int kKeys, typename Put>
__device__ __forceinline__ void select_middle(const float* s, int lo, int hi, int need, SelectSmem<kThreads>& sm, Put put) {
  constexpr int kWarps = kThreads / 32, kBins = 2 * kThreads, kBinBits = kThreads == 512 ? 10 : 8;
  static_assert(kBins == 1 << kBinBits, "the bins are a power of two");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (need == 0) return;
  if (need == hi - lo) {                           // every block of the middle
    for (int i = tid; i < need; i += kThreads) put(i, lo + i);
    return;
  }
  // every warp owns a run of positions, a lane every 32nd of it
  const int run = (hi - lo + kThreads - 1) / kThreads * 32;
  const int from = lo + warp * run, to = min(from + run, hi);
  uint32_t keys[kKeys > 0 ? kKeys : 1];
  auto fetch = [&](int r) -> uint32_t { return from + 32 * r + lane < to ? float_to_key(__ldcg(s + from + 32 * r + lane)) : 0u; };
  // f(r, whether the position exists, its key) over this thread's positions
  auto each = [&](auto f) {
    if constexpr (kKeys > 0) {
#pragma unroll
      for (int r = 0; r < kKeys; ++r)
        if (32 * r < run) f(r, from + 32 * r + lane < to, keys[r]);
    } else {
      for (int r = 0; 32 * r < run; ++r) f(r, from + 32 * r + lane < to, fetch(r));
    }
  };
  if constexpr (kKeys > 0) {
#pragma unroll
    for (int r = 0; r < kKeys; ++r) keys[r] = fetch(r);
  }
  uint32_t kmin = 0xffffffffu, kmax = 0u;
  each([&](int, bool in, uint32_t k) {
    if (in) { kmin = min(kmin, k); kmax = max(kmax, k); }
  });
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  if (lane == 0) { sm.red_lo[warp] = kmin; sm.red_hi[warp] = kmax; }
  __syncthreads();
  kmin = __reduce_min_sync(0xffffffffu, sm.red_lo[lane & (kWarps - 1)]);
  kmax = __reduce_max_sync(0xffffffffu, sm.red_hi[lane & (kWarps - 1)]);
  // the threshold: keys above `thr` are taken, and the first `need` (by position) of those equal to it
  uint32_t base = kmin, span = kmax - kmin;          // the interval [base, base + span]
  while (span > 0u) {
    const int shift = max(0, 32 - __clz(span) - kBinBits);   // (key - base) >> shift < kBins
    each([&](int, bool in, uint32_t k) {
      if (in && k - base <= span) atomicAdd(&sm.hist[(k - base) >> shift], 1);
    });
    __syncthreads();
    // bins from the top: thread i owns the pair kBins - 1 - 2i, kBins - 2 - 2i
    const int top_bin = kBins - 1 - 2 * tid;
    const int c0 = sm.hist[top_bin], c1 = sm.hist[top_bin - 1];
    sm.hist[top_bin] = 0;
    sm.hist[top_bin - 1] = 0;
    int incl = c0 + c1;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += v;
    }
    if (lane == 31) sm.warp_a[warp] = incl;
    __syncthreads();
    incl += __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_a[lane] : 0);
    const int above = incl - c0 - c1;
    if (above < need && incl >= need) {                // exactly one thread
      const bool second = above + c0 < need;
      const int bin = second ? top_bin - 1 : top_bin;
      sm.base = base + ((uint32_t)bin << shift);
      sm.span = min((1u << shift) - 1u, span - ((uint32_t)bin << shift));
      sm.need = need - above - (second ? c0 : 0);
      sm.count = second ? c1 : c0;
    }
    __syncthreads();
    base = sm.base;
    span = sm.span;
    need = sm.need;
    if (span > 0u && sm.count <= 32) {                 // few enough to rank directly
      each([&](int, bool in, uint32_t k) {
        if (in && k - base <= span) sm.cand[atomicAdd(&sm.cands, 1)] = k;
      });
      __syncthreads();
      const int n = sm.count;
      const uint32_t k = lane < n ? sm.cand[lane] : 0u;
      int gt = 0, ge = 0;
      for (int i = 0; i < n; ++i) {
        const uint32_t other = __shfl_sync(0xffffffffu, k, i);
        gt += other > k;
        ge += other >= k;
      }
      const uint32_t who = __ballot_sync(0xffffffffu, lane < n && gt < need && ge >= need);
      const int at = __ffs(who) - 1;                   // the threshold key (any of its equals)
      base = __shfl_sync(0xffffffffu, k, at);
      need -= __shfl_sync(0xffffffffu, gt, at);
      break;
    }
  }
  const uint32_t thr = base;
  int gt = 0, eq = 0;
  each([&](int, bool in, uint32_t k) {
    gt += __popc(__ballot_sync(0xffffffffu, in && k > thr));
    eq += __popc(__ballot_sync(0xffffffffu, in && k == thr));
  });
  __syncthreads();                                     // warp_a is read above
  if (lane == 0) { sm.warp_a[warp] = gt; sm.warp_b[warp] = eq; }
  __syncthreads();
  int eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_b[lane & (kWarps - 1)] : 0);
  int place = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_a[lane & (kWarps - 1)] : 0) + min(eq_before, need);
  each([&](int r, bool in, uint32_t k) {
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t eqm = __ballot_sync(0xffffffffu, in && k == thr);
    const bool take = in && (k > thr || (k == thr && eq_before + __popc(eqm & below) < need));
    const uint32_t tm = __ballot_sync(0xffffffffu, take);
    if (take) put(place + __popc(tm & below), from + 32 * r + lane);
    place += __popc(tm);
    eq_before += __popc(eqm);
  });
}
// What of a unit's list is known without scores: the first and the last blocks, -1 past the end, the count.
template <int kThreads>
__device__ __forceinline__ void write_known(int* out, int* count, int stride, int lo, int need, int hi, int nb) {
  const int total = lo + need + nb - hi;
  for (int i = threadIdx.x; i < stride; i += kThreads) {
    if (i < lo) out[i] = i;
    else if (i >= total) out[i] = -1;
    else if (i >= lo + need) out[i] = hi + (i - lo - need);
  }
  if (threadIdx.x == 0) *count = total;
}

// One CTA per unit.
constexpr int kBSThreads = 512;
template <int kKeys>
__global__ void __launch_bounds__(kBSThreads) block_select_kernel(BlockSelectParams p) {
  __shared__ SelectSmem<kBSThreads> sm;
  step_release();
  const int unit = blockIdx.x;
  const int b = unit / p.units_per_seq, u = unit % p.units_per_seq;
  const int tid = threadIdx.x;
  const int t = min(max(__ldg(p.seq_lens + b), 0), p.max_len);
  const int nb = (t + kBlockRows - 1) / kBlockRows;
  const int lo = min(p.sink, nb), hi = max(lo, nb - p.recent), need = min(p.top, hi - lo);
  int* out = p.out_blocks + (long long)unit * p.stride;
  write_known<kBSThreads>(out, p.out_count + unit, p.stride, lo, need, hi, nb);
  sm.hist[2 * tid] = 0;
  sm.hist[2 * tid + 1] = 0;
  if (tid == 0) sm.cands = 0;
  step_wait();
  select_middle<kBSThreads, kKeys>(p.scores + ((long long)b * p.num_q_heads + u * p.heads_per_unit) * p.ld, lo, hi, need, sm,
                                   [&](int place, int blk) { out[lo + place] = blk; });
}

// ------------------------------------------------------------------------------- attention
// Attention over listed blocks of a bf16 cache: one list per query head, or one per KV head for its whole group.
// grid (splits, units per sequence, B).  A stage of the warp-private ring is one block, whose rows are
// contiguous; rows past the end of the sequence are masked.  The arithmetic is bf16_stage for kHeads heads at most: 16 MMAs
// per block for four, 24 for eight, 48 for sixteen.  In a step, the first and the last blocks do not depend on
// the selection: they are attended over while it runs, before step_wait().
struct BlockAttnParams {
  const __nv_bfloat16* q;
  KvDev kv;
  const int* blocks;        // [B][units][stride]
  const int* count;
  int stride, units_per_seq;
  int num_q_heads, group_size, heads_per_unit, splits, units;
  int max_len;
  // a step knows without the selection that blocks [0, sink) and the last `recent` are attended over (fixed = 1): it
  // takes the lists' middle part only, `top` entries at most
  int fixed, sink, recent, top;
  BoundsDev bd;             // and it recomputes the bounds of the last block
  // kSelect: the kernel before this one is the scores', and every CTA selects for itself
  const float* scores;
  int ld;
  int* out_blocks;          // = blocks, written by the first CTA of a unit
  int* out_count;
  float* partials;          // [B][Hq][splits][kPartStride]
  unsigned int* tickets;
  __nv_bfloat16* out;
  float* out_lse;
  uint32_t* flags;
};

// kSelect (steps over at most kSelectKeys * kTThreads blocks, kSelectTop of them to select): every CTA selects for itself,
// once the scores are there, and there is no kernel for it.  32 lists, us a step: 9.0 against 9.7 with 2047 positions, 9.6 against
// 9.9 with 8191 (issued call by call: 10.3 against 12.0 and 11.3 against 12.1); 256 lists with 8191: 37.3 against 38.7.
// With 16000 positions, eight keys a thread, four warps take longer than sixteen and a launch: 11.9 against 11.2.
constexpr int kSelectKeys = 4, kSelectTop = 256;
// kOwn: a warp per unit, which it takes alone from start to end, four to a CTA; grid (units / 4).
template <int kHeads, bool kSelect, bool kOwn>
__global__ void __launch_bounds__(kTThreads, 2) block_attn_kernel(BlockAttnParams p) {
  constexpr int kTiles = kHeadTiles<kHeads>;
  static_assert(!(kSelect && kOwn), "a selection takes a CTA");
  __shared__ SelectSmem<kSelect ? kTThreads : 32> sm_select;
  __shared__ int sm_list[kSelect ? kSelectTop : 1];
  extern __shared__ __align__(128) unsigned char g_smem[];
  __shared__ float sm_m[kTWarps][16], sm_l[kTWarps][16];
  __shared__ bool is_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int own = blockIdx.x * kTWarps + warp;
  if (kOwn && own >= p.units) return;
  const int split = kOwn ? 0 : blockIdx.x, b = kOwn ? own / p.units_per_seq : blockIdx.z;
  const int u = kOwn ? own - b * p.units_per_seq : blockIdx.y;
  const int gq = p.heads_per_unit;
  const int head0 = u * gq, kvh = head0 / p.group_size;
  const int unit0 = b * p.num_q_heads + head0;
  const int g = lane >> 2;
  const int given = __ldg(p.kv.seq_lens + b), t = min(max(given, 0), p.max_len);
  if (t != given && (kOwn ? lane : tid) == 0) atomicOr(p.flags, kFlagBadLength);
  const int nb = (t + kBlockRows - 1) / kBlockRows;
  const long long unit = (long long)b * p.units_per_seq + u;
  const int* list = p.blocks + unit * p.stride;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(g_smem) + warp * (kTStages * kTStageBytes);

  uint32_t qb[kTiles][8][2];
  load_query_bf16<kHeads>(p.q + (long long)unit0 * kHeadDim, gq, qb);
  float o[kTiles][8][4];
  clear_tiles<kTiles>(o);
  SoftBf st[kTiles][2];

  // a step writes the bounds of the last block, whose score nothing reads: here and now, while the selection runs
  if (p.fixed && split == 0 && head0 % p.group_size == 0 && (kOwn || warp == kTWarps - 1) && nb > 0 && t == given) {
    long long row, bi;
    uint32_t flag = 0u;
    if (!locate_block(p.kv, p.bd, b, kvh, nb - 1, row, bi)) flag = kFlagBadPage;
    else if (!bounds_of_block(p.kv.k + row, t - (nb - 1) * kBlockRows, p.bd.codes + bi * kBoundsBytes, p.bd.scale + bi)) flag = kFlagNonFinite;
    if (flag && lane == 0) atomicOr(p.flags, flag);
  }

  // two passes over the ring: the blocks that are known (a step), then the listed ones
  const int lo = min(p.sink, nb), hi = max(lo, nb - p.recent);
  const int worker = kOwn ? 0 : split * kTWarps + warp, workers = kOwn ? 1 : p.splits * kTWarps;
  if constexpr (kSelect) {
    if (split == 0) write_known<kTThreads>(p.out_blocks + unit * p.stride, p.out_count + unit, p.stride, lo, min(p.top, hi - lo), hi, nb);
    sm_select.hist[2 * tid] = 0;
    sm_select.hist[2 * tid + 1] = 0;
    if (tid == 0) sm_select.cands = 0;
  }
  for (int pass = p.fixed ? 0 : 1; pass < 2; ++pass) {
    int cnt;
    if (pass == 0) {
      cnt = lo + nb - hi;
    } else {
      step_wait();                           // the lists may come from the kernel before this one
      if (p.fixed) {
        cnt = min(p.top, hi - lo);
        list += lo;
        if constexpr (kSelect) {
          select_middle<kTThreads, kSelectKeys>(p.scores + (long long)unit0 * p.ld, lo, hi, cnt, sm_select, [&](int place, int blk) {
            sm_list[place] = blk;
            if (split == 0) p.out_blocks[unit * p.stride + lo + place] = blk;
          });
          __syncthreads();
        }
      } else {
        cnt = min(max(__ldcg(p.count + unit), 0), p.stride);
      }
    }
    const int per = (cnt + workers - 1) / workers;
    const int start = min(worker * per, cnt);
    const int nstages = min(start + per, cnt) - start;

    // where 32 listed blocks lie (element offset and real rows), one per lane, looked up a group ahead
    const bool paged = p.kv.page_table != nullptr;
    auto entry = [&](int grp) -> int {
      const int j = grp * 32 + lane;
      if (j >= nstages) return -1;
      if (pass == 0) return start + j < lo ? start + j : hi + start + j - lo;
      const int blk = kSelect ? sm_list[start + j] : __ldcg(list + start + j);
      if ((unsigned)blk >= (unsigned)nb) {
        atomicOr(p.flags, kFlagBadIndex);
        return -1;
      }
      return blk;
    };
    auto page_of = [&](int blk) -> int {
      return (paged && blk >= 0) ? __ldg(p.kv.page_table + (long long)b * p.kv.page_table_stride + blk) : 0;
    };
    long long off_cur = 0;
    int rows_cur = 0;
    auto place_group = [&](int blk, int page) {
      rows_cur = blk >= 0 ? min(kBlockRows, t - blk * kBlockRows) : 0;
      if (paged && rows_cur > 0 && (unsigned)page >= (unsigned)p.kv.num_pages) {
        atomicOr(p.flags, kFlagBadPage);
        rows_cur = 0;
      }
      off_cur = (long long)(paged ? page : b) * p.kv.stride_outer + (long long)kvh * p.kv.stride_head +
                (paged ? 0ll : (long long)blk * (kBlockRows * kHeadDim));
      if (rows_cur == 0) off_cur = 0;
    };
    int blk_next = entry(0), pg_next = page_of(blk_next);
    place_group(blk_next, pg_next);
    blk_next = entry(1);
    pg_next = page_of(blk_next);

    // a lane copies one 16-byte chunk of every row: lanes 0-15 of K, 16-31 of V
    const __nv_bfloat16* src_base = lane < 16 ? p.kv.k : p.kv.v;
    const uint32_t dst_lane = ring + (lane < 16 ? 0u : (uint32_t)kTTileBytes) + ((lane & 15u) << 4);
    uint32_t sx[8];                          // source chunk that the swizzle wants at this lane's place, by row mod 8
#pragma unroll
    for (int k = 0; k < 8; ++k) sx[k] = (((uint32_t)lane & 15u) ^ (uint32_t)k) << 3;
    int rows_of[kTStages];                   // real rows per ring slot (slots are compile-time below)
    auto issue = [&](int j, auto slot_c) {
      constexpr int kSlot = decltype(slot_c)::value;
      if (j < nstages) {
        if (j > 0 && (j & 31) == 0) {
          place_group(blk_next, pg_next);
          blk_next = entry((j >> 5) + 1);
          pg_next = page_of(blk_next);
        }
        const __nv_bfloat16* src = src_base + __shfl_sync(0xffffffffu, off_cur, j & 31);
        const int rows = __shfl_sync(0xffffffffu, rows_cur, j & 31);
        const uint32_t dst = dst_lane + (uint32_t)kSlot * kTStageBytes;
        if (rows == kBlockRows) {
#pragma unroll
          for (int r = 0; r < kTStageRows; ++r) cp_async_16_full(dst + r * kRowBytes, src + r * kHeadDim + sx[r & 7]);
        } else {
#pragma unroll
          for (int r = 0; r < kTStageRows; ++r)
            cp_async_16(dst + r * kRowBytes, src + (r < rows ? r * kHeadDim + sx[r & 7] : 0), r < rows ? 16 : 0);
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
      bf16_stage<kHeads>(kt, kt + kTTileBytes, qb, g < rows, g + 8 < rows, o, st);
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
    __syncwarp();
  }
  if constexpr (kOwn) {                      // the warp's ring is free: it takes the unit's sums, a head in a row
    float* mine = reinterpret_cast<float*>(g_smem + warp * (kTStages * kTStageBytes));
    store_partial_bf16<kHeads>(o, st, gq, mine, sm_m[warp], sm_l[warp]);
    __syncwarp();
    for (int h = 0; h < gq; ++h) {
      Merged r;
      r.m = sm_m[warp][h];
      r.add(r.m, sm_l[warp][h], reinterpret_cast<const float4*>(mine + h * kHeadDim)[lane]);
      r.store(p.out, p.out_lse, unit0 + h);
    }
    return;
  }
  __syncthreads();                         // the ring is free: it takes the warps' partials
  float* sm_o = reinterpret_cast<float*>(g_smem);
  store_partial_bf16<kHeads>(o, st, gq, sm_o + warp * gq * kHeadDim, sm_m[warp], sm_l[warp]);
  __syncthreads();
  auto part_row = [&](int head, int part) -> float* { return p.partials + ((long long)(unit0 + head) * p.splits + part) * kPartStride; };
  finish_unit<kTWarps>(sm_o, &sm_m[0][0], &sm_l[0][0], kTWarps, gq, p.splits, split, part_row, p.tickets, p.out, p.out_lse, unit0,
              &is_last);
}

}  // namespace prhs
