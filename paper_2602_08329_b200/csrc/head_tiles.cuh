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

// Items are laid out sequence after sequence, heads * f(length) each.  Warp-collective: their number, and the largest f.
template <typename F>
__device__ __forceinline__ int count_items(const int* seq_lens, int batch, int heads, F f, int* longest = nullptr) {
  if (batch == 1) {
    const int w = f(__ldg(seq_lens));
    if (longest) *longest = w;
    return heads * w;
  }
  int sum = 0, most = 0;
#pragma unroll 4
  for (int b = threadIdx.x & 31; b < batch; b += 32) {
    const int w = f(__ldg(seq_lens + b));
    sum += w;
    most = max(most, w);
  }
  if (longest) *longest = __reduce_max_sync(0xffffffffu, most);
  return heads * __reduce_add_sync(0xffffffffu, sum);
}
// Warp-collective: the sequence that holds item x (*b) and the number of items before it; false where x lies past the end.
template <typename F>
__device__ __forceinline__ bool find_item(const int* seq_lens, int batch, int heads, F f, int x, int* b, int* before) {
  const int lane = threadIdx.x & 31;
  *b = *before = 0;
  if (batch == 1) return x < heads * f(__ldg(seq_lens));
  int sum = 0;
  for (int b0 = 0; b0 < batch; b0 += 32) {
    const int w = b0 + lane < batch ? heads * f(__ldg(seq_lens + b0 + lane)) : 0;
    int incl = w;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += v;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, sum + incl > x);
    if (past) {
      const int at = __ffs(past) - 1;
      *b = b0 + at;
      *before = sum + __shfl_sync(0xffffffffu, incl - w, at);
      return true;
    }
    sum += __shfl_sync(0xffffffffu, incl, 31);
  }
  return false;
}

// 2^x by the hardware's approximation, to 2^-22 relative; results below 2^-126 are zero.  (exp2f spends four more
// instructions on denormal results, which as weights are nothing beside the largest one.)
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The reference exponent before the first logit: below every finite logit, and finite, so that no difference is NaN.
constexpr float kNoLogit = -3.0e38f;

// One head's softmax bookkeeping in a lane: the reference exponent, and the sum of the fp32 weights.  A logit that is NaN
// or +inf makes l NaN, and it stays NaN: the maximum passes over a NaN, so it is by the sum that a row's result is known to
// be NaN, and by l = 0 alone that a row is empty.
struct SoftBf {
  float m = kNoLogit, l = 0.f;
};

// A weight enters the product with V as the sum of two bf16, to 2^-16 of itself, so that an output's error is that of its own
// rounding to bf16 (0.0017 of the norm; with one bf16, 0.0024).  Up to four heads leave four of the MMA's eight columns
// empty: the low parts go there, columns 4 to 7 being the heads 0 to 3 once more, and cost no MMA.  More heads take a second
// MMA for each tile of V.  A step, us with one bf16 and with two: one user 10.9 and 10.8 (with second MMAs there too 12.0),
// 16 ragged sequences of up to 64K with eight KV heads for 4 heads each 52.2 and 52.3, for 8 53.0 and 53.3, for 16 62.0 and 67.9.
// (An infinite value is infinite or NaN in the result: a low part is zero or negative as often as not.)
// kHeads is a unit's largest number of heads: 4, 8 or 16.
template <int kHeads>
constexpr bool kSpareColumns = kHeads == 4;
template <int kHeads>
constexpr int kHeadTiles = kHeads == 16 ? 2 : 1;

template <int kTiles>
__device__ __forceinline__ void clear_tiles(float (&o)[kTiles][8][4]) {
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
    for (int c = 0; c < 8; ++c) { o[hh][c][0] = 0.f; o[hh][c][1] = 0.f; o[hh][c][2] = 0.f; o[hh][c][3] = 0.f; }
}

// B fragments of the heads 8hh + g (g mod 4 where columns are spare): 16 dimensions per k-step.  q: the unit's first head;
// absent heads are zero.
template <int kHeads>
__device__ __forceinline__ void load_query_bf16(const __nv_bfloat16* q, int heads, uint32_t (&qb)[kHeadTiles<kHeads>][8][2]) {
  constexpr int kTiles = kHeadTiles<kHeads>;
  const int lane = threadIdx.x & 31, g = lane >> 2, tg = lane & 3;
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh) {
    const int head = kSpareColumns<kHeads> ? g & 3 : 8 * hh + g;
    const uint32_t* q32 = reinterpret_cast<const uint32_t*>(q + (long long)head * kHeadDim);
    const bool has = head < heads;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      qb[hh][ks][0] = has ? __ldg(q32 + ks * 8 + tg) : 0u;
      qb[hh][ks][1] = has ? __ldg(q32 + ks * 8 + 4 + tg) : 0u;
    }
  }
}

// One stage of 16 rows (K tile and V tile of [16][128] bf16, 16-byte chunk c of row r at chunk c ^ (r & 7)) by a warp:
// S^T = K Q^T, online softmax, O^T += V^T P^T.  A lane owns keys g and g + 8 (real where v0, v1) for heads
// 8hh + 2tg and + 1 (heads that are not there have a zero query and columns that nobody reads); o[hh][c] are dimensions 16c + g (0, 1) and 16c + g + 8 (2, 3) of the same two heads.
template <int kHeads>
__device__ __forceinline__ void bf16_stage(uint32_t kt, uint32_t vt, const uint32_t (&qb)[kHeadTiles<kHeads>][8][2], bool v0, bool v1,
                                           float (&o)[kHeadTiles<kHeads>][8][4], SoftBf (&st)[kHeadTiles<kHeads>][2]) {
  constexpr int kTiles = kHeadTiles<kHeads>;
  constexpr bool kSpare = kSpareColumns<kHeads>;
  const int lane = threadIdx.x & 31;
  const int row = (lane & 7) + 8 * ((lane >> 3) & 1), half = lane >> 4;     // ldmatrix: this lane's row, chunk of a pair
  float s[kTiles][2][4];
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    uint32_t a[4];
    ldmatrix_x4(a, kt + row * kRowBytes + (((2 * ks + half) ^ (row & 7)) << 4));
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh) {
      if (ks < 2) { s[hh][ks][0] = 0.f; s[hh][ks][1] = 0.f; s[hh][ks][2] = 0.f; s[hh][ks][3] = 0.f; }
      mma_bf16_full(s[hh][ks & 1], a[0], a[1], a[2], a[3], qb[hh][ks][0], qb[hh][ks][1]);
    }
  }
  const float sc = kScale * kLog2e;
  float x[kTiles][2][2];                     // [tile][head][key]
  bool exceed = false;
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      x[hh][e][0] = v0 ? (s[hh][0][e] + s[hh][1][e]) * sc : -INFINITY;
      x[hh][e][1] = v1 ? (s[hh][0][2 + e] + s[hh][1][2 + e]) * sc : -INFINITY;
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
        f[e] = exp2_fast(st[hh][e].m - mn);
        st[hh][e].m = mn;
        st[hh][e].l *= f[e];
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) { o[hh][c][0] *= f[0]; o[hh][c][1] *= f[1]; o[hh][c][2] *= f[0]; o[hh][c][3] *= f[1]; }
    }
  }
  uint32_t pb[kTiles][2], pc[kTiles][2];
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh) {
    float w[2][2];                           // [key][head]
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        w[n][e] = exp2_fast(x[hh][e][n] - st[hh][e].m);
        st[hh][e].l += w[n][e];
      }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint32_t high = pack_bf16x2(w[n][0], w[n][1]);
      const uint32_t low = pack_bf16x2(w[n][0] - bf_lo(high), w[n][1] - bf_hi(high));
      pb[hh][n] = transpose_8x8(kSpare && (lane & 2) ? low : high);
      if (!kSpare) pc[hh][n] = transpose_8x8(low);
    }
  }
  uint32_t bv[2][4];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    ldmatrix_x4_trans(bv[c & 1], vt + row * kRowBytes + (((2 * c + half) ^ (row & 7)) << 4));
    const uint32_t(&b)[4] = bv[c & 1];
    const uint32_t(&a)[4] = bv[(c + 1) & 1];                   // those of c - 1: two products into one tile are kept apart
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh) {
      mma_bf16_full(o[hh][c], b[0], b[2], b[1], b[3], pb[hh][0], pb[hh][1]);
      if (!kSpare && c > 0) mma_bf16_full(o[hh][c - 1], a[0], a[2], a[1], a[3], pc[hh][0], pc[hh][1]);
    }
  }
  if (!kSpare) {
#pragma unroll
    for (int hh = 0; hh < kTiles; ++hh) mma_bf16_full(o[hh][7], bv[1][0], bv[1][2], bv[1][1], bv[1][3], pc[hh][0], pc[hh][1]);
  }
}

// A warp's partial into shared memory: o [heads][128], m, l [16].
template <int kHeads>
__device__ __forceinline__ void store_partial_bf16(const float (&o)[kHeadTiles<kHeads>][8][4], const SoftBf (&st)[kHeadTiles<kHeads>][2],
                                                   int heads, float* sm_o, float* sm_m, float* sm_l) {
  constexpr int kTiles = kHeadTiles<kHeads>;
  const int lane = threadIdx.x & 31, g = lane >> 2, tg = lane & 3;
#pragma unroll
  for (int hh = 0; hh < kTiles; ++hh)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = st[hh][e].l;
#pragma unroll
      for (int off = 4; off <= 16; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
      const int head = 8 * hh + 2 * tg + e;
      const bool has = head < heads;
      if (has && g == 0) { sm_m[head] = l == 0.f ? -INFINITY : st[hh][e].m; sm_l[head] = l; }
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        float a = o[hh][c][e], z = o[hh][c][2 + e];
        if (kSpareColumns<kHeads>) {         // the low parts, four columns further
          a += __shfl_xor_sync(0xffffffffu, a, 2);
          z += __shfl_xor_sync(0xffffffffu, z, 2);
        }
        if (has) {
          sm_o[head * kHeadDim + 16 * c + g] = a;
          sm_o[head * kHeadDim + 16 * c + g + 8] = z;
        }
      }
    }
}

// Running combination of partials (m, l and four of the 128 columns per lane).
struct Merged {
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void rescale(float mn) {
    const float f = mn > -INFINITY ? exp2f(m - mn) : 0.f;
    l *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
    m = mn;
  }
  __device__ __forceinline__ void add(float m2, float l2, float4 x) {      // m2 <= m
    const float f = m2 > -INFINITY ? exp2f(m2 - m) : 0.f;
    l = fmaf(l2, f, l);                                  // a NaN passes a factor of zero
    o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* out, float* out_lse, long long unit) const {
    const int lane = threadIdx.x & 31;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint2*>(out + unit * kHeadDim + lane * 4) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
    if (lane == 0 && out_lse) out_lse[unit] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
};

// End of a unit's work in a CTA of kWarps warps: the warps' partials in shared memory (o [slot][head][128], m, l
// [slot][16]; at most one slot more than warps) become the result (one part) or this CTA's part in global memory, row(head, part)
// = o[128], m, l; the CTA whose part arrives last merges them (a ticket, no waiting).  A warp per head, or
// several warps per head where there are fewer than kWarps; a lane has four columns, and the loads of sixteen parts
// are in flight at once.  (Heads one after the other, a column per thread, cost 5000 cycles for four heads in the
// first half and 20 us for a merge of 32 parts.)
template <int kWarps, typename Row>
__device__ __forceinline__ void finish_unit(float* sm_o, float* sm_m, float* sm_l, int slots, int heads, int parts, int part,
                                            Row row, unsigned int* tickets, __nv_bfloat16* out, float* out_lse, int unit0, bool* is_last) {
  constexpr int kMaxSlots = kWarps + 1, kBatch = 16;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int h = warp; h < heads; h += kWarps) {
    Merged r;
    float m[kMaxSlots];
    float mx = -INFINITY;
#pragma unroll
    for (int s = 0; s < kMaxSlots; ++s) {
      m[s] = s < slots ? sm_m[s * 16 + h] : -INFINITY;
      mx = fmaxf(mx, m[s]);
    }
    r.m = mx;
#pragma unroll
    for (int s = 0; s < kMaxSlots; ++s)
      if (m[s] > -INFINITY) r.add(m[s], sm_l[s * 16 + h], reinterpret_cast<const float4*>(sm_o + (s * heads + h) * kHeadDim)[lane]);
    if (parts == 1) {
      r.store(out, out_lse, unit0 + h);
    } else {
      float4* dst = reinterpret_cast<float4*>(row(h, part));
      __stcg(dst + lane, r.o);
      if (lane == 0) __stcg(dst + 32, make_float4(r.m, r.l, 0.f, 0.f));
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
  if (!*is_last) return;
  __threadfence();
  const int slices = heads >= kWarps ? 1 : kWarps / heads;            // warps per head
  const int slice = slices == 1 ? 0 : warp % slices;
  for (int h = warp / slices; h < heads; h += kWarps / slices) {
    Merged r;
    for (int p0 = slice; p0 < parts; p0 += slices * kBatch) {
      // m, l of sixteen parts, one per lane; their columns
      const int mine = p0 + lane * slices;
      float2 st = make_float2(-INFINITY, 0.f);
      float4 x[kBatch];
      if (lane < kBatch && mine < parts) st = __ldcg(reinterpret_cast<const float2*>(row(h, mine)) + 64);
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (p0 + i * slices < parts) x[i] = __ldcg(reinterpret_cast<const float4*>(row(h, p0 + i * slices)) + lane);
      }
      float mn = st.x;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, off));
      r.rescale(fmaxf(mn, r.m));
      const float f = st.x > -INFINITY ? exp2f(st.x - r.m) : 0.f;
      r.l = fmaf(st.y, f, r.l);                // per lane until the end
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const float fi = __shfl_sync(0xffffffffu, f, i);
        r.o.x = fmaf(x[i].x, fi, r.o.x); r.o.y = fmaf(x[i].y, fi, r.o.y);
        r.o.z = fmaf(x[i].z, fi, r.o.z); r.o.w = fmaf(x[i].w, fi, r.o.w);
      }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) r.l += __shfl_xor_sync(0xffffffffu, r.l, off);
    if (slices == 1) {
      r.store(out, out_lse, unit0 + h);
    } else {
      reinterpret_cast<float4*>(sm_o + warp * kHeadDim)[lane] = r.o;
      if (lane == 0) { sm_m[warp] = r.m; sm_l[warp] = r.l; }
    }
  }
  if (slices == 1) return;
  __syncthreads();
  if (warp < heads) {
    Merged r;
    for (int s = 0; s < slices; ++s) r.m = fmaxf(r.m, sm_m[warp * slices + s]);
    for (int s = 0; s < slices; ++s)
      r.add(sm_m[warp * slices + s], sm_l[warp * slices + s],
            reinterpret_cast<const float4*>(sm_o + (warp * slices + s) * kHeadDim)[lane]);
    r.store(out, out_lse, unit0 + warp);
  }
}

}  // namespace prhs
