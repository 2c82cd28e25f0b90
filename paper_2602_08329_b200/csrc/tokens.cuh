// New tokens: queries and keys normalised per head and rotated by their positions, keys and values written to the cache
// (bf16 rows, or 8-bit blocks), in one pass; and rows of the 8-bit cache read back as bf16.
//
// All of it is bound by HBM: a token's heads come in once and go out once (2 x 256 B per head and token; 256 + 128 B for the
// keys and values of the 8-bit cache).  The arithmetic that could get in the way is the rotation's: 64 angles per
// token, each a product of 24 + 31 bits reduced to a turn.  They are computed once per token and head chunk, in
// fp64 (three operations and a conversion each), and kept in shared memory for all heads.
#pragma once
#include "bytekv.cuh"
#include "common.cuh"

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
// New tokens of sequence b: rows [r0, r1), positions [t - n, t).  ok: they fit together.
struct SeqRows {
  int r0, n, t;
  bool ok;
};
__device__ __forceinline__ SeqRows seq_rows(const int* row_start, int num_rows, const int* seq_lens, int max_len, int b) {
  SeqRows s;
  int r1;
  s.r0 = row_start ? __ldg(row_start + b) : b;
  r1 = row_start ? __ldg(row_start + b + 1) : b + 1;
  s.t = __ldg(seq_lens + b);
  s.ok = s.r0 >= 0 && r1 >= s.r0 && r1 <= num_rows && r1 - s.r0 <= s.t && s.t <= max_len;
  s.n = s.ok ? r1 - s.r0 : 0;
  return s;
}
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
// cosine and sine (times scale) of pos * inv_freq radians.  In fp64 the angle becomes quarter turns and the rest of one, which
// is exact to 2^-52 of the angle; the rest, an eighth of a turn at most, is what fp32 has to hold.
__device__ __forceinline__ float2 rotation(int pos, float inv_freq, float scale) {
  const double turns = (double)pos * ((double)inv_freq * 0.15915494309189533577);
  const double q = rint(turns * 4.0);
  float s, c;
  sincospif(2.f * (float)(turns - 0.25 * q), &s, &c);
  const int quarter = (int)(long long)q & 3;
  const float cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
  return make_float2((quarter == 1 || quarter == 2 ? -cc : cc) * scale, (quarter & 2 ? -ss : ss) * scale);
}

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[16], int at) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[at + 2 * i] = bf_lo(u[i]);
    x[at + 2 * i + 1] = bf_hi(u[i]);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[16], int at) {
  return make_uint4(pack_bf16x2(x[at], x[at + 1]), pack_bf16x2(x[at + 2], x[at + 3]), pack_bf16x2(x[at + 4], x[at + 5]),
                    pack_bf16x2(x[at + 6], x[at + 7]));
}

// Eight lanes hold a head: lane l its 16-byte chunks l and l + 8, values 8l .. 8l + 7 and 64 + 8l .. 64 + 8l + 7.  Normalises
// and rotates it, every operation written out so that the kernels agree to the bit.  cs: the row's 64 (cosine, sine); stage: 128 floats for this head (kRotPartial only).  Warp-collective.
template <int kRot>
__device__ __forceinline__ void prepare_head(uint4& a, uint4& b, const PrepDev& p, const float* weight, const float2* cs, float* stage) {
  const int l = threadIdx.x & 7;
  float x[16];
  unpack8(a, x, 0);
  unpack8(b, x, 8);
  if (p.norm) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
    const float r = rsqrtf(fmaf(ss, 1.f / kHeadDim, p.eps));
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= r;
    if (weight) {
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float4 w = __ldg(reinterpret_cast<const float4*>(weight + 8 * l + (i < 8 ? i : 56 + i)));
        x[i] *= w.x;
        x[i + 1] *= w.y;
        x[i + 2] *= w.z;
        x[i + 3] *= w.w;
      }
    }
  }
  if (kRot == kRotHalves) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 t = cs[8 * l + i];
      const float u = x[i], w = x[8 + i];
      x[i] = fmaf(u, t.x, -__fmul_rn(w, t.y));
      x[8 + i] = fmaf(w, t.x, __fmul_rn(u, t.y));
    }
  } else if (kRot == kRotAdjacent) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const int f = 4 * l + (i < 8 ? i / 2 : 28 + i / 2);
      if (2 * f < p.rot) {
        const float2 t = cs[f];
        const float u = x[i], w = x[i + 1];
        x[i] = fmaf(u, t.x, -__fmul_rn(w, t.y));
        x[i + 1] = fmaf(w, t.x, __fmul_rn(u, t.y));
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) stage[8 * l + (i < 8 ? i : 56 + i)] = x[i];
    __syncwarp();
    const int half = p.rot >> 1;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int d = 8 * l + (i < 8 ? i : 56 + i);
      if (d < half) {
        const float2 t = cs[d];
        x[i] = fmaf(x[i], t.x, -__fmul_rn(stage[d + half], t.y));
      } else if (d < p.rot) {
        const float2 t = cs[d - half];
        x[i] = fmaf(x[i], t.x, __fmul_rn(stage[d - half], t.y));
      }
    }
    __syncwarp();
  }
  a = pack8(x, 0);
  b = pack8(x, 8);
}

// -------------------------------------------------------------------------------- into the bf16 cache
struct QkvAppendParams {
  TokenRowsDev rows;
  PrepDev prep;
  KvDev kv;
  __nv_bfloat16* q_out;
  int max_len;
  int chunks, chunk_heads;        // a row's heads (queries, keys, values in this order) in chunks of chunk_heads, a multiple of 8
  uint32_t* flags;
};
constexpr int kQkvWarps = 4;

// A warp takes a chunk of a row's heads, eight at a time (four per step of the lanes, two steps in flight).
template <int kRot>
__global__ void __launch_bounds__(32 * kQkvWarps) qkv_append_kernel(const __grid_constant__ QkvAppendParams p) {
  __shared__ float2 sm_cs[kQkvWarps][64];
  __shared__ float sm_stage[kRot == kRotPartial ? kQkvWarps : 1][kRot == kRotPartial ? 4 * kHeadDim : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & 7;
  if (blockIdx.x == 0) record_bad_sequences(p.rows.row_start, p.rows.num_rows, p.kv.seq_lens, p.max_len, p.rows.batch, p.flags);
  const long long unit = (long long)blockIdx.x * kQkvWarps + warp;
  const int r = (int)(unit / p.chunks), h0 = (int)(unit % p.chunks) * p.chunk_heads;
  if (r >= p.rows.num_rows) return;
  const int nq = p.rows.num_q_heads, nkv = p.rows.num_kv_heads, heads = nq + 2 * nkv, h1 = min(h0 + p.chunk_heads, heads);
  const TokenRowsDev& in = p.rows;
  // where head h of this row is read
  auto source = [&](int h) {
    if (h < nq) return in.q + (long long)r * in.q_row + (long long)h * in.q_head;
    if (h < nq + nkv) return in.k + (long long)r * in.k_row + (long long)(h - nq) * in.k_head;
    return in.v + (long long)r * in.v_row + (long long)(h - nq - nkv) * in.v_head;
  };
  uint4 a[2], b[2];
  auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __nv_bfloat16* s = source(min(h + 4 * i + (lane >> 3), h1 - 1)) + 8 * l;
      a[i] = *reinterpret_cast<const uint4*>(s);
      b[i] = *reinterpret_cast<const uint4*>(s + 64);
    }
  };
  load(h0);
  const int seq = in.row_start ? last_start(in.row_start, in.batch, r) : r;
  if (seq < 0) return;
  const SeqRows s = seq_rows(in.row_start, in.num_rows, p.kv.seq_lens, p.max_len, seq);
  if (!s.ok || r >= s.r0 + s.n) return;
  const int pos = s.t - s.n + (r - s.r0);
  for (int f = lane; 2 * f < p.prep.rot; f += 32) {
    const int at = in.positions ? __ldg(in.positions + p.prep.axis_of[f] * in.positions_stride + r) : pos;
    sm_cs[warp][f] = rotation(at, __ldg(p.prep.inv_freq + f), p.prep.rot_scale);
  }
  long long row = (long long)seq * p.kv.stride_outer + (long long)pos * kHeadDim;
  bool page_ok = true;
  if (p.kv.page_table) {
    const int page = __ldg(p.kv.page_table + (long long)seq * p.kv.page_table_stride + (pos >> kPageShift));
    page_ok = (unsigned)page < (unsigned)p.kv.num_pages;
    if (!page_ok && lane == 0) atomicOr(p.flags, kFlagBadPage);
    row = (long long)page * p.kv.stride_outer + (pos & 15) * kHeadDim;
  }
  __syncwarp();
  for (int h = h0; h < h1; h += 8) {
    uint4 ca[2] = {a[0], a[1]}, cb[2] = {b[0], b[1]};
    if (h + 8 < h1) load(h + 8);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int hh = h + 4 * i + (lane >> 3);
      const bool is_v = hh >= nq + nkv;
      if (!__all_sync(0xffffffffu, is_v || hh >= h1)) {
        uint4 xa = ca[i], xb = cb[i];
        prepare_head<kRot>(xa, xb, p.prep, hh < nq ? p.prep.q_weight : p.prep.k_weight, sm_cs[warp],
                           sm_stage[kRot == kRotPartial ? warp : 0] + (kRot == kRotPartial ? (lane >> 3) * kHeadDim : 0));
        if (!is_v) {
          ca[i] = xa;
          cb[i] = xb;
        }
      }
      if (hh < h1 && (hh < nq || page_ok)) {
        __nv_bfloat16* to = hh < nq ? p.q_out + ((long long)r * nq + hh) * kHeadDim
                                    : const_cast<__nv_bfloat16*>(is_v ? p.kv.v : p.kv.k) + row +
                                          (long long)(is_v ? hh - nq - nkv : hh - nq) * p.kv.stride_head;
        *reinterpret_cast<uint4*>(to + 8 * l) = ca[i];
        *reinterpret_cast<uint4*>(to + 64 + 8 * l) = cb[i];
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

// Blocks of 16 positions that a sequence's new tokens touch.
__device__ __forceinline__ int touched_blocks(const SeqRows& s) {
  return s.n ? (s.t - 1) / kBlockRows - (s.t - s.n) / kBlockRows + 1 : 0;
}

// A CTA takes a touched block (blockIdx.x) and every gridDim.y-th of its heads: 16 tokens share one table of cosines and sines, and
// the keys of a block and head meet in one warp, which quantises them (quantise_block).  The first block's CTA also writes the
// tail where a later block stays open: it alone reads the old tail, a warp does the same heads both times, and a thread reads
// and writes the same 16-byte pieces, so program order keeps the two apart.
template <int kFmt, int kRot>
__global__ void __launch_bounds__(32 * kQkv8Warps) bytekv_qkv_append_kernel(const __grid_constant__ ByteKvQkvParams p) {
  __shared__ float2 sm_cs[kBlockRows][64];
  __shared__ uint4 sm_rows[kQkv8Warps][kBlockRows * 16];       // a block's prepared keys on their way to quantise_block's order
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
      sm_cs[i >> 6][f] = rotation(at, __ldg(p.prep.inv_freq + f), p.prep.rot_scale);
    }
  };
  float* const stage = reinterpret_cast<float*>(sm_rows[warp]) + (lane >> 3) * kHeadDim;     // (before the rows are put there)
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
    uint4 a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pos = which * kBlockRows + 4 * i + (lane >> 3);
      const __nv_bfloat16* from = src + (s.r0 + min(max(pos, start), s.t - 1) - start) * by + 8 * l;
      a[i] = *reinterpret_cast<const uint4*>(from);
      b[i] = *reinterpret_cast<const uint4*>(from + 64);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pos = which * kBlockRows + 4 * i + (lane >> 3);
      prepare_head<kRot>(a[i], b[i], p.prep, p.prep.k_weight, sm_cs[min(max(pos, start), s.t - 1) & (kBlockRows - 1)], stage);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sm_rows[warp][(4 * i + (lane >> 3)) * 16 + l] = a[i];
      sm_rows[warp][(4 * i + (lane >> 3)) * 16 + 8 + l] = b[i];
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
    for (int task = blockIdx.y * kQkv8Warps + warp; task < n * quads; task += gridDim.y * kQkv8Warps) {
      const int pos = first + task / quads, h = task % quads * 4 + (lane >> 3), hh = min(h, nq - 1);
      const long long r = s.r0 + pos - start;
      const __nv_bfloat16* from = in.q + r * in.q_row + (long long)hh * in.q_head + 8 * l;
      uint4 a = *reinterpret_cast<const uint4*>(from), b = *reinterpret_cast<const uint4*>(from + 64);
      prepare_head<kRot>(a, b, p.prep, p.prep.q_weight, sm_cs[pos & (kBlockRows - 1)], stage);
      if (h < nq) {
        __nv_bfloat16* to = p.q_out + (r * nq + h) * kHeadDim + 8 * l;
        *reinterpret_cast<uint4*>(to) = a;
        *reinterpret_cast<uint4*>(to + 64) = b;
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

// A warp per block of 16 positions and keys or values (grid: pairs of warps along x, KV heads, sequences): eight lanes a row, 16 codes each.
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
      uint4 c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = __ldg(reinterpret_cast<const uint4*>(codes + (4 * i + (lane >> 3)) * kRow8Bytes + 16 * (lane & 7)));
      const float z = __ldg(scale);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 4 * i + (lane >> 3), pos = blk * kBlockRows + row;
        const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
        uint32_t o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const __half2_raw raw = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[k >> 1] >> (16 * (k & 1))), kFmt == kE4M3 ? __NV_E4M3 : __NV_E5M2);
          const float2 x = __half22float2(__half2(raw));
          o[k] = pack_bf16x2(x.x * z, x.y * z);
        }
        if (pos >= first && pos < t) {
          __nv_bfloat16* at = to + row * kHeadDim + 16 * (lane & 7);
          *reinterpret_cast<uint4*>(at) = make_uint4(o[0], o[1], o[2], o[3]);
          *reinterpret_cast<uint4*>(at + 8) = make_uint4(o[4], o[5], o[6], o[7]);
        }
      }
    }
  }
  if (!page_ok && lane == 0) atomicOr(p.flags, kFlagBadPage);
}

}  // namespace prhs
