// New tokens: queries and keys normalised per head and rotated by their positions, keys and values written to the cache
// (bf16 rows, or 8-bit blocks), in one pass; and rows of the 8-bit cache read back as bf16.
//
// What they move: a token's heads come in once and go out once (2 x 256 B per head and token; 256 + 128 B for the keys and values of the
// 8-bit cache).  The 64 angles of a token are computed once, in fp64, and kept in shared memory for all of its heads.  278 MB of ragged
// image prompts take 61 to 64 us (4.4 TB/s, 0.67 of measured; 49 without the arithmetic: it is the chain of shuffles, table reads and
// conversions of a head that is not hidden), 738 MB of two prompts into the 8-bit cache 158 us (0.71), 403 MB read back 65 us (0.94).
#pragma once
#include "bytekv.cuh"
#include "common.cuh"
#include "seq_rows.cuh"

namespace prhs {

struct TokenRowsDev {
  const __nv_bfloat16 *q, *k, *v;
  long long q_row, q_head, k_row, k_head, v_row, v_head;       // strides in elements
  const int* row_start;                                        // nullptr: row b is sequence b's one token
  const int* positions;
  long long positions_stride;
  int num_rows, batch, num_q_heads, num_kv_heads;
};
struct PrepDev {
  const float *q_weight, *k_weight, *inv_freq;
  float eps, rot_scale;
  int rot, norm;
  uint8_t axis_of[64];
};

// How the first `rot` values pair up.  All 128 in halves is the common case and needs no shared memory; adjacent
// pairs never leave a thread; other halves go through shared memory.
constexpr int kRotHalves = 0, kRotAdjacent = 1, kRotPartial = 2;

// ------------------------------------------------------------------------------- sequences of rows
// One CTA of a launch: records sequences that do not fit.
__device__ __forceinline__ void record_bad_sequences(const int* row_start, int num_rows, const int* seq_lens, int max_len, int batch,
                                                     uint32_t* flags) {
  bool bad = false;
  for (int b = threadIdx.x; b < batch; b += blockDim.x) bad |= !seq_rows(row_start, num_rows, seq_lens, max_len, b).ok;
  if (bad) atomicOr(flags, kFlagBadLength);
}
// Warp-collective: the last sequence that starts at or before row r (-1: none), 32 probes a round.
__device__ __forceinline__ int last_start(const int* row_start, int batch, int r) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = batch;
  for (;;) {
    const int step = (hi - lo + 31) >> 5, at = lo + lane * step;
    const int c = __popc(__ballot_sync(0xffffffffu, at < hi && __ldg(row_start + min(at, batch)) <= r));
    if (c == 0) return lo - 1;               // only in the first round, where lo = 0
    lo += (c - 1) * step;
    hi = min(hi, lo + step);
    if (step == 1) return lo;
  }
}

// ------------------------------------------------------------------------------------ heads
// cosine and sine (times scale) of pos * inv_freq radians, in fp64 until the end: the angle becomes quarter turns and the rest of one, an
// eighth of a turn at most, whose Taylor series need eight terms for 2^-49.  (64 a row, for all of its heads: fp32 would save nothing
// that shows, and its errors would move keys across the roundings of bf16 and of the 8-bit codes.)
__device__ __forceinline__ float2 rotation(int pos, float inv_freq, float scale) {
  const double turns = (double)pos * ((double)inv_freq * 0.15915494309189533577);
  const double q = rint(turns * 4.0), x = (turns - 0.25 * q) * 6.283185307179586477, y = x * x;
  double c = 1.0, s = 1.0;
#pragma unroll
  for (int n = 14; n >= 2; n -= 2) {
    c = fma(c, y * (-1.0 / (n * (n - 1))), 1.0);
    s = fma(s, y * (-1.0 / (n * (n + 1))), 1.0);
  }
  s *= x;
  const int quarter = (int)(long long)q & 3;
  const double cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
  return make_float2((float)(quarter == 1 || quarter == 2 ? -cc : cc) * scale, (float)(quarter & 2 ? -ss : ss) * scale);
}

// two fp32 at a time
__device__ __forceinline__ uint64_t pack_f32x2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t r, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// What a row's heads are rotated with: the 64 cosines and sines, or, where all 128 values turn in halves, for queries and for keys the
// products of them and the weights:  y_u = x_u (c w_u) + x_v (-s w_v),  y_v = x_v (c w_v) + x_u (s w_u).
template <int kRot>
struct RowTurns {
  float c[64], s[64];
  __device__ __forceinline__ void set(int f, float2 cs, const PrepDev&) {
    c[f] = cs.x;
    s[f] = cs.y;
  }
};
template <>
struct RowTurns<kRotHalves> {
  // [queries, keys][c w_u, -s w_v, c w_v, s w_u]: 64 of each, in the order in which eight lanes read them (lane l needs 8l .. 8l + 7), so
  // that a read of all lanes is one wavefront: these were what bounded the kernel
  float t[2][4][2][8][4];
  __device__ __forceinline__ void set(int f, float2 cs, const PrepDev& p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float* w = i ? p.k_weight : p.q_weight;
      const float wu = w ? __ldg(w + f) : 1.f, wv = w ? __ldg(w + f + 64) : 1.f;
      t[i][0][(f >> 2) & 1][f >> 3][f & 3] = __fmul_rn(cs.x, wu);
      t[i][1][(f >> 2) & 1][f >> 3][f & 3] = -__fmul_rn(cs.y, wv);
      t[i][2][(f >> 2) & 1][f >> 3][f & 3] = __fmul_rn(cs.x, wv);
      t[i][3][(f >> 2) & 1][f >> 3][f & 3] = __fmul_rn(cs.y, wu);
    }
  }
};

// Eight lanes hold a head: lane l its 16-byte chunks l and l + 8, values 8l .. 8l + 7 and 64 + 8l .. 64 + 8l + 7, two to a register pair.
// Normalises and rotates it (kind: 0 a query, else a key), every operation written out so that the kernels agree to the bit.  The
// norm's factor comes last where the rotation does not wait for it.  stage: 128 floats for this head (kRotPartial
// only).  Warp-collective.
template <int kRot>
__device__ __forceinline__ void prepare_head(uint4& a, uint4& b, const PrepDev& p, int kind, const RowTurns<kRot>& turns, float* stage) {
  const int l = threadIdx.x & 7;
  uint64_t x[8];
  {
    const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = pack_f32x2(bf_lo(u[i]), bf_hi(u[i]));
  }
  uint64_t rr = 0ull;
  if (p.norm) {
    uint64_t q = 0ull;
#pragma unroll
    for (int i = 0; i < 8; ++i) q = fma_f32x2(x[i], x[i], q);
    float ss, t;
    unpack_f32x2(q, ss, t);
    ss = __fadd_rn(ss, t);
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) ss = __fadd_rn(ss, __shfl_xor_sync(0xffffffffu, ss, off));
    // the reciprocal root, and one step of Newton's in fp64: its error would be that of all 128 values
    const float v = fmaf(ss, 1.f / kHeadDim, p.eps), r0 = rsqrtf(v);
    const float r1 = (float)fma(0.5 * r0, fma(-(double)v * r0, (double)r0, 1.0), (double)r0);
    const float r = isfinite(r1) ? r1 : r0;
    rr = pack_f32x2(r, r);
  }
  if constexpr (kRot == kRotHalves) {
    const auto& t = turns.t[kind != 0];
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      uint64_t f[4][2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 v = *reinterpret_cast<const float4*>(t[j][i >> 1][l]);
        f[j][0] = pack_f32x2(v.x, v.y);
        f[j][1] = pack_f32x2(v.z, v.w);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint64_t u = x[i + j], w = x[4 + i + j];
        x[i + j] = fma_f32x2(u, f[0][j], mul_f32x2(w, f[1][j]));
        x[4 + i + j] = fma_f32x2(w, f[2][j], mul_f32x2(u, f[3][j]));
      }
    }
    if (p.norm) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = mul_f32x2(x[i], rr);
    }
  } else if (p.norm) {
    const float* weight = kind ? p.k_weight : p.q_weight;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = mul_f32x2(x[i], rr);
    if (weight) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 w = __ldg(reinterpret_cast<const float4*>(weight + 8 * l + 4 * (i & 1) + 64 * (i >> 1)));
        x[2 * i] = mul_f32x2(x[2 * i], pack_f32x2(w.x, w.y));
        x[2 * i + 1] = mul_f32x2(x[2 * i + 1], pack_f32x2(w.z, w.w));
      }
    }
  }
  if constexpr (kRot == kRotAdjacent) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int f = 4 * l + (i < 4 ? i : 28 + i);
      if (2 * f < p.rot) {
        float u, w;
        unpack_f32x2(x[i], u, w);
        const float c = turns.c[f], n = turns.s[f];
        x[i] = pack_f32x2(fmaf(u, c, -__fmul_rn(w, n)), fmaf(w, c, __fmul_rn(u, n)));
      }
    }
  } else if constexpr (kRot == kRotPartial) {
    float y[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unpack_f32x2(x[i], y[2 * i], y[2 * i + 1]);
      *reinterpret_cast<float2*>(stage + 8 * l + 2 * (i & 3) + 64 * (i >> 2)) = make_float2(y[2 * i], y[2 * i + 1]);
    }
    __syncwarp();
    const int half = p.rot >> 1;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int d = 8 * l + (i & 7) + 64 * (i >> 3);
      if (d < half) y[i] = fmaf(y[i], turns.c[d], -__fmul_rn(stage[d + half], turns.s[d]));
      else if (d < p.rot) y[i] = fmaf(y[i], turns.c[d - half], __fmul_rn(stage[d - half], turns.s[d - half]));
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = pack_f32x2(y[2 * i], y[2 * i + 1]);
  }
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float u, w;
    unpack_f32x2(x[i], u, w);
    o[i] = pack_bf16x2(u, w);
  }
  a = make_uint4(o[0], o[1], o[2], o[3]);
  b = make_uint4(o[4], o[5], o[6], o[7]);
}

// -------------------------------------------------------------------------------- into the bf16 cache
struct QkvAppendParams {
  TokenRowsDev rows;
  PrepDev prep;
  KvDev kv;
  __nv_bfloat16* q_out;
  int max_len;
  int cta_rows;                   // rows per CTA, at most kQkvRows
  uint32_t* flags;
};
constexpr int kQkvWarps = 8, kQkvRows = 8, kQkvStages = 2;
constexpr int kQkvMaxHeads = 512;                 // (the table of heads: 16 KB)

// Where a head (queries, keys, values in this order) is read and written: bytes to add are row * src_stride and the row's offset among
// queries or in the cache.
struct HeadPlace {
  const char* src;
  long long src_stride;
  char* dst;
  int kind;                       // 0 query, 1 key, 2 value
};

// A CTA takes cta_rows rows, and every gridDim.y-th of their groups of four heads: the places of heads and rows, and the rows' angles are
// looked up and computed by all threads once, then the heads stream through, a group per warp and step, the next two on their way
// (from before the look-ups).  Eight rows: sixteen leave too few CTAs to even out (74 us for 278 MB against 67), four pay the look-ups
// twice as often (66 against 61, later).  Copies through a ring in shared memory were no faster than registers (the ring's
// wavefronts cost what its depth gains).
template <int kRot>
__global__ void __launch_bounds__(32 * kQkvWarps, 3) qkv_append_kernel(const __grid_constant__ QkvAppendParams p) {
  extern __shared__ uint4 qkv_smem[];
  HeadPlace* const sm_heads = reinterpret_cast<HeadPlace*>(qkv_smem);
  __shared__ __align__(16) RowTurns<kRot> sm_turns[kQkvRows];
  __shared__ float sm_stage[kRot == kRotPartial ? kQkvWarps : 1][kRot == kRotPartial ? 4 * kHeadDim : 1];
  __shared__ long long sm_off[kQkvRows][2];       // bytes: of the row's queries in q_out, of the token in the cache; -1: not written
  __shared__ int sm_pos[kQkvRows];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & 7;
  const TokenRowsDev& in = p.rows;
  const int nq = in.num_q_heads, nkv = in.num_kv_heads, heads = nq + 2 * nkv, groups = (heads + 3) >> 2;
  const int r0 = blockIdx.x * p.cta_rows, rows = min(p.cta_rows, in.num_rows - r0);
  if (blockIdx.x == 0 && blockIdx.y == 0)
    record_bad_sequences(in.row_start, in.num_rows, p.kv.seq_lens, p.max_len, in.batch, p.flags);
  for (int h = threadIdx.x; h < heads; h += 32 * kQkvWarps) {
    HeadPlace x;
    if (h < nq) x = {(const char*)(in.q + r0 * in.q_row + h * in.q_head), 2 * in.q_row, (char*)(p.q_out + (long long)h * kHeadDim), 0};
    else if (h < nq + nkv)
      x = {(const char*)(in.k + r0 * in.k_row + (h - nq) * in.k_head), 2 * in.k_row, (char*)(p.kv.k + (h - nq) * p.kv.stride_head), 1};
    else x = {(const char*)(in.v + r0 * in.v_row + (h - nq - nkv) * in.v_head), 2 * in.v_row, (char*)(p.kv.v + (h - nq - nkv) * p.kv.stride_head), 2};
    sm_heads[h] = x;
  }
  __syncthreads();
  // this warp's steps: every `stride`-th of the rows' groups, as (row, group) without a division
  const int stride = gridDim.y * kQkvWarps, first = blockIdx.y * kQkvWarps + warp;
  const int by_row = stride / groups, by_group = stride - by_row * groups;
  int lrow = first / groups, lgroup = first - lrow * groups;       // the next to be loaded
  uint4 a[kQkvStages], b[kQkvStages];
  auto load = [&](int i) {
    if (lrow >= rows) return;
    const HeadPlace& x = sm_heads[min(4 * lgroup + (lane >> 3), heads - 1)];
    const char* from = x.src + lrow * x.src_stride + 16 * l;
    a[i] = *reinterpret_cast<const uint4*>(from);
    b[i] = *reinterpret_cast<const uint4*>(from + 128);
    lrow += by_row;
    lgroup += by_group;
    if (lgroup >= groups) {
      lgroup -= groups;
      ++lrow;
    }
  };
  int row = lrow, group = lgroup;
#pragma unroll
  for (int i = 0; i < kQkvStages; ++i) load(i);
  for (int i = warp; i < rows; i += kQkvWarps) {
    const int r = r0 + i, seq = in.row_start ? last_start(in.row_start, in.batch, r) : r;
    long long off_q = -1, off_kv = -1;
    int pos = 0;
    if (seq >= 0) {
      const SeqRows s = seq_rows(in.row_start, in.num_rows, p.kv.seq_lens, p.max_len, seq);
      if (s.ok && r < s.r0 + s.n) {
        pos = s.t - s.n + (r - s.r0);
        off_q = (long long)r * nq * kRowBytes;
        off_kv = 2 * ((long long)seq * p.kv.stride_outer + (long long)pos * kHeadDim);
        if (p.kv.page_table) {
          const int page = __ldg(p.kv.page_table + (long long)seq * p.kv.page_table_stride + (pos >> kPageShift));
          off_kv = 2 * ((long long)page * p.kv.stride_outer + (pos & 15) * kHeadDim);
          if ((unsigned)page >= (unsigned)p.kv.num_pages) {
            off_kv = -1;
            if (lane == 0) atomicOr(p.flags, kFlagBadPage);
          }
        }
      }
    }
    if (lane == 0) {
      sm_off[i][0] = off_q;
      sm_off[i][1] = off_kv;
    }
#pragma unroll
    for (int f = lane; f < 64; f += 32)
      if (2 * f < p.prep.rot) {
        const int at = in.positions ? __ldg(in.positions + p.prep.axis_of[f] * in.positions_stride + r) : pos;
        sm_turns[i].set(f, rotation(at, __ldg(p.prep.inv_freq + f), p.prep.rot_scale), p.prep);
      }
  }
  __syncthreads();
  for (;;) {
#pragma unroll
    for (int i = 0; i < kQkvStages; ++i) {
      if (row >= rows) return;
      uint4 xa = a[i], xb = b[i];
      load(i);
      const int h = 4 * group + (lane >> 3);
      const HeadPlace& x = sm_heads[min(h, heads - 1)];
      const int kind = x.kind;
      if (!__all_sync(0xffffffffu, kind == 2)) {
        uint4 ya = xa, yb = xb;
        prepare_head<kRot>(ya, yb, p.prep, kind, sm_turns[row],
                           sm_stage[kRot == kRotPartial ? warp : 0] + (kRot == kRotPartial ? (lane >> 3) * kHeadDim : 0));
        if (kind != 2) {
          xa = ya;
          xb = yb;
        }
      }
      const long long off = sm_off[row][kind != 0];
      if (h < heads && off >= 0) {
        char* to = x.dst + off + 16 * l;
        *reinterpret_cast<uint4*>(to) = xa;
        *reinterpret_cast<uint4*>(to + 128) = xb;
      }
      row += by_row;
      group += by_group;
      if (group >= groups) {
        group -= groups;
        ++row;
      }
    }
  }
}

// --------------------------------------------------------------------------------- into the 8-bit cache
struct ByteKvQkvParams {
  TokenRowsDev rows;
  PrepDev prep;
  ByteKvDev kv;
  __nv_bfloat16* q_out;
  int max_len;
  uint32_t* flags;
};
constexpr int kQkv8Warps = 8;
template <int kRot>
constexpr int kQkv8SmemBytes = kQkv8Warps * kBlockRows * 16 * 16 + kBlockRows * (int)sizeof(RowTurns<kRot>);

// Blocks of 16 positions that a sequence's new tokens touch.
__device__ __forceinline__ int touched_blocks(const SeqRows& s) {
  return s.n ? (s.t - 1) / kBlockRows - (s.t - s.n) / kBlockRows + 1 : 0;
}

// A CTA takes a touched block (blockIdx.x) and every gridDim.y-th of its heads: 16 tokens share one table of cosines and sines, and
// the keys of a block and head meet in one warp, which quantises them (quantise_block).  The first block's CTA also writes the
// tail where a later block stays open: it alone reads the old tail, a warp does the same heads both times, and a thread reads
// and writes the same 16-byte pieces, so program order keeps the two apart.
template <int kFmt, int kRot>
__global__ void __launch_bounds__(32 * kQkv8Warps, 2) bytekv_qkv_append_kernel(const __grid_constant__ ByteKvQkvParams p) {
  extern __shared__ uint4 sm_dyn[];
  RowTurns<kRot>* const sm_turns = reinterpret_cast<RowTurns<kRot>*>(sm_dyn);
  uint4 (*const sm_rows)[kBlockRows * 16] = reinterpret_cast<uint4 (*)[kBlockRows * 16]>(sm_dyn + kBlockRows * sizeof(RowTurns<kRot>) / 16);     // a block's prepared keys on their way to quantise_block's order
  __shared__ float sm_stage[kRot == kRotPartial ? kQkv8Warps : 1][kRot == kRotPartial ? 4 * kHeadDim : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & 7;
  const TokenRowsDev& in = p.rows;
  if (blockIdx.x == 0 && blockIdx.y == 0) record_bad_sequences(in.row_start, in.num_rows, p.kv.seq_lens, p.max_len, in.batch, p.flags);
  // the sequence that holds touched block blockIdx.x (every warp finds it for itself)
  int seq = -1, j = blockIdx.x;
  for (int b0 = 0; b0 < in.batch && seq < 0; b0 += 32) {
    const int w = b0 + lane < in.batch ? touched_blocks(seq_rows(in.row_start, in.num_rows, p.kv.seq_lens, p.max_len, b0 + lane)) : 0;
    int incl = w;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += v;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, incl > j);
    if (past) {
      const int at = __ffs(past) - 1;
      seq = b0 + at;
      j -= __shfl_sync(0xffffffffu, incl - w, at);
    } else {
      j -= __shfl_sync(0xffffffffu, incl, 31);
    }
  }
  if (seq < 0) return;
  const SeqRows s = seq_rows(in.row_start, in.num_rows, p.kv.seq_lens, p.max_len, seq);
  const int start = s.t - s.n, blk = start / kBlockRows + j, open = s.t / kBlockRows;
  const int nq = in.num_q_heads, nkv = in.num_kv_heads;
  // cosines and sines of a block's new tokens
  auto angles = [&](int which) {
    for (int i = threadIdx.x; i < kBlockRows * 64; i += 32 * kQkv8Warps) {
      const int pos = which * kBlockRows + (i >> 6), f = i & 63;
      if (pos < start || pos >= s.t || 2 * f >= p.prep.rot) continue;
      const int at = in.positions ? __ldg(in.positions + p.prep.axis_of[f] * in.positions_stride + s.r0 + pos - start) : pos;
      sm_turns[i >> 6].set(f, rotation(at, __ldg(p.prep.inv_freq + f), p.prep.rot_scale), p.prep);
    }
  };
  float* const stage = sm_stage[kRot == kRotPartial ? warp : 0] + (kRot == kRotPartial ? (lane >> 3) * kHeadDim : 0);
  // head h of keys (or values) of a block's new tokens, in quantise_block's order: lane holds 16-byte piece lane % 16 of rows 2i + lane / 16
  auto fetch = [&](int which, int h, bool is_v, uint4 (&x)[8]) {
    const __nv_bfloat16* src = is_v ? in.v + (long long)h * in.v_head : in.k + (long long)h * in.k_head;
    const long long by = is_v ? in.v_row : in.k_row;
    if (is_v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int pos = which * kBlockRows + 2 * i + (lane >> 4);
        if (pos >= start && pos < s.t) x[i] = *reinterpret_cast<const uint4*>(src + (s.r0 + pos - start) * by + 8 * (lane & 15));
      }
      return;
    }
    // four rows at a time, the next four on their way
    uint4 a, b;
    auto load = [&](int i) {
      const int pos = which * kBlockRows + 4 * i + (lane >> 3);
      const __nv_bfloat16* from = src + (s.r0 + min(max(pos, start), s.t - 1) - start) * by + 8 * l;
      a = *reinterpret_cast<const uint4*>(from);
      b = *reinterpret_cast<const uint4*>(from + 64);
    };
    load(0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * i + (lane >> 3), pos = which * kBlockRows + row;
      uint4 ya = a, yb = b;
      if (i < 3) load(i + 1);
      prepare_head<kRot>(ya, yb, p.prep, 1, sm_turns[min(max(pos, start), s.t - 1) & (kBlockRows - 1)], stage);
      sm_rows[warp][row * 16 + l] = ya;
      sm_rows[warp][row * 16 + 8 + l] = yb;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = 2 * i + (lane >> 4), pos = which * kBlockRows + row;
      if (pos >= start && pos < s.t) x[i] = sm_rows[warp][row * 16 + (lane & 15)];
    }
    __syncwarp();
  };
  // keys and values of head h: tail + 16-byte piece of this lane
  auto tail_of = [&](int h, bool is_v) {
    return const_cast<__nv_bfloat16*>(is_v ? p.kv.v_tail : p.kv.k_tail) + ((long long)seq * nkv + h) * (kBlockRows * kHeadDim) + (lane >> 4) * kHeadDim +
           8 * (lane & 15);
  };
  auto to_tail = [&](int which) {
    for (int task = blockIdx.y * kQkv8Warps + warp; task < 2 * nkv; task += gridDim.y * kQkv8Warps) {
      const int h = task >> 1;
      const bool is_v = task & 1;
      uint4 x[8];
      fetch(which, h, is_v, x);
      __nv_bfloat16* tail = tail_of(h, is_v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int pos = which * kBlockRows + 2 * i + (lane >> 4);
        if (pos >= start && pos < s.t) *reinterpret_cast<uint4*>(tail + 2 * i * kHeadDim) = x[i];
      }
    }
  };
  angles(blk);
  __syncthreads();
  // queries: four heads of a row at a time
  {
    const int first = max(start, blk * kBlockRows), n = min(s.t, (blk + 1) * kBlockRows) - first, quads = (nq + 3) / 4;
    const int by = gridDim.y * kQkv8Warps;
    uint4 a[2], b[2];
    auto load = [&](int task, int i) {
      if (task >= n * quads) return;
      const int row = task / quads, hh = min((task - row * quads) * 4 + (lane >> 3), nq - 1);
      const __nv_bfloat16* from = in.q + (s.r0 + first + row - start) * in.q_row + (long long)hh * in.q_head + 8 * l;
      a[i] = *reinterpret_cast<const uint4*>(from);
      b[i] = *reinterpret_cast<const uint4*>(from + 64);
    };
    const int task0 = blockIdx.y * kQkv8Warps + warp;
    load(task0, 0);
    load(task0 + by, 1);
    for (int task1 = task0; task1 < n * quads; task1 += 2 * by) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int task = task1 + i * by;
        if (task >= n * quads) break;
        uint4 xa = a[i], xb = b[i];
        load(task + 2 * by, i);
        const int row = task / quads, h = (task - row * quads) * 4 + (lane >> 3), pos = first + row;
        prepare_head<kRot>(xa, xb, p.prep, 0, sm_turns[pos & (kBlockRows - 1)], stage);
        if (h < nq) {
          __nv_bfloat16* to = p.q_out + ((long long)(s.r0 + pos - start) * nq + h) * kHeadDim + 8 * l;
          *reinterpret_cast<uint4*>(to) = xa;
          *reinterpret_cast<uint4*>(to + 64) = xb;
        }
      }
    }
  }
  if (blk == open) {                  // this block stays open (a later open block is the first one's work)
    if (j == 0) to_tail(blk);
    return;
  }
  bool page_ok = true;
  long long page = 0;
  if (p.kv.page_table) {
    page = __ldg(p.kv.page_table + (long long)seq * p.kv.page_table_stride + blk);
    page_ok = page >= 0 && page < p.kv.num_pages;
    if (!page_ok && threadIdx.x == 0) atomicOr(p.flags, kFlagBadPage);
  }
  const long long outer = p.kv.page_table ? page : seq;
  for (int task = blockIdx.y * kQkv8Warps + warp; task < 2 * nkv; task += gridDim.y * kQkv8Warps) {
    const int h = task >> 1;
    const bool is_v = task & 1;
    uint4 x[8];
    const __nv_bfloat16* tail = tail_of(h, is_v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (blk * kBlockRows + 2 * i + (lane >> 4) < start) x[i] = *reinterpret_cast<const uint4*>(tail + 2 * i * kHeadDim);
    fetch(blk, h, is_v, x);
    if (!page_ok) continue;
    const long long off = outer * p.kv.stride_outer + (long long)h * p.kv.stride_head + (p.kv.page_table ? 0ll : (long long)blk * kBlock8Bytes);
    const long long soff = outer * p.kv.scale_stride_outer + (long long)h * p.kv.scale_stride_head + (p.kv.page_table ? 0 : blk);
    const bool finite = quantise_block<kFmt>(x, const_cast<uint8_t*>(is_v ? p.kv.v : p.kv.k) + off,
                                             const_cast<float*>(is_v ? p.kv.v_scale : p.kv.k_scale) + soff);
    if (!finite && lane == 0) atomicOr(p.flags, kFlagNonFinite);
  }
  if (j == 0 && open * kBlockRows < s.t) {
    __syncthreads();                  // the table is free
    angles(open);
    __syncthreads();
    to_tail(open);
  }
}

// ------------------------------------------------------------------------------- out of the 8-bit cache
struct ByteKvReadParams {
  ByteKvDev kv;
  KvDev out;
  const int* first;
  int max_new, max_len, num_kv_heads;
  uint32_t* flags;
};

// A warp per block of 16 positions and keys or values (grid: pairs of warps along x, KV heads, sequences): half a warp a row.
// Bound by HBM: 128 B in (and 8 B / 16) and 256 B out per row.
template <int kFmt>
__global__ void __launch_bounds__(256) bytekv_read_kernel(const __grid_constant__ ByteKvReadParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int j = blockIdx.x * (blockDim.x >> 6) + (warp >> 1), is_v = warp & 1;
  const int h = blockIdx.y, b = blockIdx.z;
  const int t = __ldg(p.kv.seq_lens + b), first = p.first ? __ldg(p.first + b) : 0;
  if (first < 0 || first > t || t - first > p.max_new || t > p.max_len) {
    if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(p.flags, kFlagBadLength);
    return;
  }
  const int blk = first / kBlockRows + j;
  if (first == t || blk * kBlockRows >= t) return;
  __nv_bfloat16* to = const_cast<__nv_bfloat16*>(is_v ? p.out.v : p.out.k) + (long long)h * p.out.stride_head;
  bool page_ok = true;
  if (p.out.page_table) {
    const int page = __ldg(p.out.page_table + (long long)b * p.out.page_table_stride + blk);
    page_ok = (unsigned)page < (unsigned)p.out.num_pages;
    to += (long long)page * p.out.stride_outer;
  } else {
    to += (long long)b * p.out.stride_outer + (long long)blk * kBlockRows * kHeadDim;
  }
  if (blk == t / kBlockRows) {        // the open block: bf16 already
    const __nv_bfloat16* tail = (is_v ? p.kv.v_tail : p.kv.k_tail) + ((long long)b * p.num_kv_heads + h) * (kBlockRows * kHeadDim);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = 2 * i + (lane >> 4), pos = blk * kBlockRows + row, at = row * kHeadDim + 8 * (lane & 15);
      if (page_ok && pos >= first && pos < t) *reinterpret_cast<uint4*>(to + at) = __ldg(reinterpret_cast<const uint4*>(tail + at));
    }
  } else {
    const uint8_t* codes = (is_v ? p.kv.v : p.kv.k) + (long long)h * p.kv.stride_head;
    const float* scale = (is_v ? p.kv.v_scale : p.kv.k_scale) + (long long)h * p.kv.scale_stride_head;
    if (p.kv.page_table) {
      const int page = __ldg(p.kv.page_table + (long long)b * p.kv.page_table_stride + blk);
      if ((unsigned)page >= (unsigned)p.kv.num_pages) page_ok = false;
      codes += (long long)page * p.kv.stride_outer;
      scale += (long long)page * p.kv.scale_stride_outer;
    } else {
      codes += (long long)b * p.kv.stride_outer + (long long)blk * kBlock8Bytes;
      scale += (long long)b * p.kv.scale_stride_outer + blk;
    }
    if (page_ok) {
      // half a warp a row, 8 codes (16 bytes of bf16) a lane: stores fill whole sectors
      uint2 c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = __ldg(reinterpret_cast<const uint2*>(codes + (2 * i + (lane >> 4)) * kRow8Bytes + 8 * (lane & 15)));
      const float z = __ldg(scale);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = 2 * i + (lane >> 4), pos = blk * kBlockRows + row;
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t w = (k < 2 ? c[i].x : c[i].y) >> (16 * (k & 1));
          const float2 x = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, kFmt == kE4M3 ? __NV_E4M3 : __NV_E5M2)));
          o[k] = pack_bf16x2(x.x * z, x.y * z);
        }
        if (pos >= first && pos < t) *reinterpret_cast<uint4*>(to + row * kHeadDim + 8 * (lane & 15)) = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
  }
  if (!page_ok && lane == 0) atomicOr(p.flags, kFlagBadPage);
}

}  // namespace prhs
