// Decode attention with keys or dimensions on the 16 rows of mma.sync and the heads of a unit on its 8 columns: the
// stage of 16 bf16 rows, and the end of a unit (the warps' partials combined, parts merged).
#pragma once
#include "attn.cuh"
#include "common.cuh"

namespace prhs {

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// One head's softmax bookkeeping in a lane: l sums the fp32 weights (log-sum-exp), lt the weights as rounded to bf16,
// which is what divides the output.
struct SoftBf {
  float m = -INFINITY, l = 0.f, lt = 0.f;
};

template <int kTiles>
__device__ __forceinline__ void clear_tiles(float (&o)[kTiles][8][4]) {
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
    for (int c = 0; c < 8; ++c) { o[hh][c][0] = 0.f; o[hh][c][1] = 0.f; o[hh][c][2] = 0.f; o[hh][c][3] = 0.f; }
}

// B fragments of the heads 8hh + g: 16 dimensions per k-step.  q: the unit's first head; absent heads are zero.
template <int kTiles>
__device__ __forceinline__ void load_query_bf16(const __nv_bfloat16* q, int heads, uint32_t (&qb)[kTiles][8][2]) {
  const int lane = threadIdx.x & 31, g = lane >> 2, tg = lane & 3;
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh) {
    const uint32_t* q32 = reinterpret_cast<const uint32_t*>(q + (long long)(8 * hh + g) * kHeadDim);
    const bool has = 8 * hh + g < heads;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      qb[hh][ks][0] = has ? __ldg(q32 + ks * 8 + tg) : 0u;
      qb[hh][ks][1] = has ? __ldg(q32 + ks * 8 + 4 + tg) : 0u;
    }
  }
}

// One stage of 16 rows (K tile and V tile of [16][128] bf16, 16-byte chunk c of row r at chunk c ^ (r & 7)) by a warp:
// S^T = K Q^T, online softmax, O^T += V^T P^T.  A lane owns keys g and g + 8 (real where v0, v1) for heads
// 8hh + 2tg and + 1; o[hh][c] are dimensions 16c + g (0, 1) and 16c + g + 8 (2, 3) of the same two heads.
template <int kTiles>
__device__ __forceinline__ void bf16_stage(uint32_t kt, uint32_t vt, const uint32_t (&qb)[kTiles][8][2], int heads, bool v0, bool v1,
                                           float (&o)[kTiles][8][4], SoftBf (&st)[kTiles][2]) {
  const int lane = threadIdx.x & 31, tg = lane & 3;
  const int row = (lane & 7) + 8 * ((lane >> 3) & 1), half = lane >> 4;     // ldmatrix: this lane's row, chunk of a pair
  float s[kTiles][2][4];
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
    for (int c = 0; c < 2; ++c) { s[hh][c][0] = 0.f; s[hh][c][1] = 0.f; s[hh][c][2] = 0.f; s[hh][c][3] = 0.f; }
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    uint32_t a[4];
    ldmatrix_x4(a, kt + row * kRowBytes + (((2 * ks + half) ^ (row & 7)) << 4));
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh) mma_bf16_full(s[hh][ks & 1], a[0], a[1], a[2], a[3], qb[hh][ks][0], qb[hh][ks][1]);
  }
  const float sc = kScale * kLog2e;
  float x[kTiles][2][2];                     // [tile][head][key]
  bool exceed = false;
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const bool has = 8 * hh + 2 * tg + e < heads;
      x[hh][e][0] = has && v0 ? (s[hh][0][e] + s[hh][1][e]) * sc : -INFINITY;
      x[hh][e][1] = has && v1 ? (s[hh][0][2 + e] + s[hh][1][2 + e]) * sc : -INFINITY;
      exceed = exceed || fmaxf(x[hh][e][0], x[hh][e][1]) > st[hh][e].m + 8.f;
    }
  // the reference exponent moves only when a logit exceeds it by more than 8 (weights stay below 2^8)
  if (__any_sync(0xffffffffu, exceed)) {
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh) {
      float f[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float mx = fmaxf(x[hh][e][0], x[hh][e][1]);
#pragma unroll
        for (int off = 4; off <= 16; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        const float mn = fmaxf(st[hh][e].m, mx);
        f[e] = mn > -INFINITY ? exp2f(st[hh][e].m - mn) : 1.f;
        st[hh][e].m = mn;
        st[hh][e].l *= f[e];
        st[hh][e].lt *= f[e];
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) { o[hh][c][0] *= f[0]; o[hh][c][1] *= f[1]; o[hh][c][2] *= f[0]; o[hh][c][3] *= f[1]; }
    }
  }
  uint32_t pb[kTiles][2];
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh) {
    float w[2][2];                           // [key][head]
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        w[n][e] = x[hh][e][n] > -INFINITY ? exp2f(x[hh][e][n] - st[hh][e].m) : 0.f;
        st[hh][e].l += w[n][e];
      }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint32_t pk = pack_bf16x2(w[n][0], w[n][1]);
      st[hh][0].lt += bf_lo(pk);
      st[hh][1].lt += bf_hi(pk);
      pb[hh][n] = transpose_8x8(pk);
    }
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    uint32_t bv[4];
    ldmatrix_x4_trans(bv, vt + row * kRowBytes + (((2 * c + half) ^ (row & 7)) << 4));
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh) mma_bf16_full(o[hh][c], bv[0], bv[2], bv[1], bv[3], pb[hh][0], pb[hh][1]);
  }
}

// A warp's partial into shared memory: o [heads][128], m, l, l~ [16].
template <int kTiles>
__device__ __forceinline__ void store_partial_bf16(const float (&o)[kTiles][8][4], const SoftBf (&st)[kTiles][2], int heads, float* sm_o,
                                                   float* sm_m, float* sm_l, float* sm_lt) {
  const int lane = threadIdx.x & 31, g = lane >> 2, tg = lane & 3;
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = st[hh][e].l, lt = st[hh][e].lt;
#pragma unroll
      for (int off = 4; off <= 16; off <<= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, off);
        lt += __shfl_xor_sync(0xffffffffu, lt, off);
      }
      const int head = 8 * hh + 2 * tg + e;
      if (head < heads) {
        if (g == 0) { sm_m[head] = st[hh][e].m; sm_l[head] = l; sm_lt[head] = lt; }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          sm_o[head * kHeadDim + 16 * c + g] = o[hh][c][e];
          sm_o[head * kHeadDim + 16 * c + g + 8] = o[hh][c][2 + e];
        }
      }
    }
}

// Merge of a unit's partials by the last CTA to arrive: a warp per head, a float4 of the 128 columns per lane, the
// splits' weights one per lane.  row(head, split) is the address of a partial: o[128], m, l, l~.  The loads of
// all splits are independent of one another (a merge that walked them one by one cost 20 us at 32 splits of
// four heads).
template <typename Row>
__device__ __forceinline__ void merge_partials(Row row, int splits, int heads, __nv_bfloat16* out, float* out_lse, int unit0) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  for (int h = warp; h < heads; h += warps) {
    float M = -INFINITY;
    for (int sp = lane; sp < splits; sp += 32) M = fmaxf(M, __ldcg(row(h, sp) + kHeadDim));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float L = 0.f, Lt = 0.f;
    if (M != -INFINITY) {
      for (int s0 = 0; s0 < splits; s0 += 32) {
        float f = 0.f;
        if (s0 + lane < splits) {
          const float* r = row(h, s0 + lane);
          f = exp2f(__ldcg(r + kHeadDim) - M);
          L = fmaf(__ldcg(r + kHeadDim + 1), f, L);
          Lt = fmaf(__ldcg(r + kHeadDim + 2), f, Lt);
        }
        const int n = min(32, splits - s0);
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
          const float4 x = __ldcg(reinterpret_cast<const float4*>(row(h, s0 + i)) + lane);
          const float fi = __shfl_sync(0xffffffffu, f, i);
          acc.x = fmaf(x.x, fi, acc.x); acc.y = fmaf(x.y, fi, acc.y); acc.z = fmaf(x.z, fi, acc.z); acc.w = fmaf(x.w, fi, acc.w);
        }
      }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      L += __shfl_xor_sync(0xffffffffu, L, off);
      Lt += __shfl_xor_sync(0xffffffffu, Lt, off);
    }
    const float inv = Lt > 0.f ? 1.f / Lt : 0.f;
    const uint2 y = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    *reinterpret_cast<uint2*>(out + (long long)(unit0 + h) * kHeadDim + lane * 4) = y;
    if (lane == 0 && out_lse) out_lse[unit0 + h] = L > 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
  }
}

// End of a unit's work in a CTA of 128 threads: the warps' partials in shared memory (o [slot][head][128], m, l, l~
// [slot][16]) become the result (one part) or this CTA's part in global memory; the CTA whose part arrives
// last merges them (a ticket, no waiting).
template <typename Row>
__device__ __forceinline__ void finish_unit(const float* sm_o, const float* sm_m, const float* sm_l, const float* sm_lt, int slots,
                                            int heads, int parts, int part, Row row, unsigned int* tickets, __nv_bfloat16* out,
                                            float* out_lse, int unit0, bool* is_last) {
  const int tid = threadIdx.x;
  for (int j = 0; j < heads; ++j) {
    float M = -INFINITY;
    for (int s = 0; s < slots; ++s) M = fmaxf(M, sm_m[s * 16 + j]);
    float acc = 0.f, L = 0.f, Lt = 0.f;
    if (M != -INFINITY) {
      for (int s = 0; s < slots; ++s) {
        const float f = exp2f(sm_m[s * 16 + j] - M);
        if (f > 0.f) acc = fmaf(sm_o[(s * heads + j) * kHeadDim + tid], f, acc);
        L = fmaf(sm_l[s * 16 + j], f, L);
        Lt = fmaf(sm_lt[s * 16 + j], f, Lt);
      }
    }
    if (parts == 1) {
      out[(long long)(unit0 + j) * kHeadDim + tid] = __float2bfloat16_rn(Lt > 0.f ? acc / Lt : 0.f);
      if (tid == 0 && out_lse) out_lse[unit0 + j] = L > 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
    } else {
      float* r = row(j, part);
      r[tid] = acc;
      if (tid == 0) { r[kHeadDim] = M; r[kHeadDim + 1] = L; r[kHeadDim + 2] = Lt; }
    }
  }
  if (parts == 1) return;
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    const unsigned int ticket = atomicAdd(tickets + unit0, 1u);
    *is_last = (ticket == (unsigned int)parts - 1u);
    if (*is_last) tickets[unit0] = 0u;
  }
  __syncthreads();
  if (*is_last) {
    __threadfence();
    merge_partials(row, parts, heads, out, out_lse, unit0);
  }
}

}  // namespace prhs
