// What the CTAs of the chunk attention work on: items, pieces of items and runs (chunk_attn.cuh says why).  Index arithmetic and warp votes
// alone, so that it can be run without a GPU.
#pragma once
#include "common.cuh"
#include "seq_rows.cuh"

namespace prhs {

constexpr int kCATile = 128;                              // keys per tile, rows per subtile
// An item's Q, merge and output cost about as much as two tiles; a run of fewer than kCAMinRun tiles is not worth its merge (four drafts
// of one user over 2047 positions: 24 us with runs of 3, 23 with 4, 26 with 8).
constexpr int kCAItemCost = 2;
constexpr int kCAMinRun = 4;
// What the CTAs work on at a time should stay in L2: a round for every 1024 tiles that are looked at (64 MB), of runs of at least 192
// (2048 tokens at 131072: 4407 us in one round, 4234 in four, 4190 in eight, for twice the workspace; runs of 48, in which the pieces'
// merges show, made 16384 with a window 1063 us instead of 884).
constexpr int kCARoundTiles = 1024, kCARoundRun = 192, kCAMaxRounds = 4;

struct ChunkParams {
  KvDev kv;
  const int* row_start;
  __nv_bfloat16* out;
  float* out_lse;
  float* partials;               // [2 gridDim.x max_rounds][kCASlotFloats]
  unsigned int* tickets;         // [gridDim.x max_rounds], zero between launches
  uint32_t* flags;
  double psaw_c;
  int num_rows, batch, num_q_heads, num_kv_heads, group, tokens;     // tokens = T
  int max_rounds;
  int sinks, window, max_len;
  unsigned int oob_row;          // a row outside the K and V tensors: zeros
};

// ---------------------------------------------------------------------------------------- the work
__device__ __forceinline__ int first_visible(const ChunkParams& p, int u) {
  int lo = p.psaw_c > 0.0 ? psaw_start(p.psaw_c, u) : 0;
  if (p.window > 0) lo = max(lo, u - p.window);
  return lo;
}
// A piece of an item: tiles k0 .. k1 - 1 of those its tokens see.
template <bool kMask, bool kFew>
struct Piece {
  int b, kvh, row0, ntok, u0;    // u0: visible length of the first token
  int k0, k1, st, lo;            // tile k is k for k < st, else lo + k - st
  int run, first_run, last_run;  // this one, and those that have pieces of the item
  int t;
  int short_item;
  __device__ __forceinline__ bool halves() const { return kFew || short_item; }
  // Subtile s uses tile k if k < sa or kb <= k < ke, and every one of its rows sees all of it if k < sf or kf <= k < kd.  (The first
  // positions may reach beyond `lo`: all tiles are listed then, and st = lo.)
  int sa, kb[2], ke[2], kf[2], kd[2], sf[2];
  __device__ __forceinline__ int tile(int k) const { return !kMask || k < st ? k : lo + k - st; }
  // subtile s: tokens [a, e) of the item, visible lengths of its first and its last
  __device__ __forceinline__ int a(const ChunkParams& p, int s) const { return halves() || s == 0 ? 0 : p.tokens; }
  __device__ __forceinline__ int e(const ChunkParams& p, int s) const { return halves() || s == 1 ? ntok : min(ntok, p.tokens); }
  __device__ __forceinline__ int uf(const ChunkParams& p, int s) const { return u0 + a(p, s); }
  __device__ __forceinline__ int ul(const ChunkParams& p, int s) const { return u0 + e(p, s) - 1; }
  __device__ __forceinline__ void ranges(const ChunkParams& p) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int first = uf(p, s), last = ul(p, s);
      ke[s] = (last + kCATile - 1) / kCATile;
      kd[s] = first / kCATile;
      kb[s] = kf[s] = sf[s] = 0;
      if (kMask) {
        const int shift = st - lo, all = min(p.sinks, ul(p, 1));
        sa = shift ? st : (all + kCATile - 1) / kCATile;
        kb[s] = first_visible(p, first) / kCATile + shift;
        kf[s] = max((first_visible(p, last) + kCATile - 1) / kCATile + shift, st);
        sf[s] = shift ? min(min(p.sinks, first) / kCATile, st) : min(p.sinks, first) / kCATile;
        ke[s] += shift;
        kd[s] += shift;
      }
    }
  }
  __device__ __forceinline__ bool active(int s, int k) const {
    return halves() ? ((k - k0) & 1) == s : k < ke[s] && (!kMask || k < sa || k >= kb[s]);
  }
  // some row of the subtile does not see all of the tile
  __device__ __forceinline__ bool partly(int s, int k) const { return !(kMask ? k < sf[s] || (k >= kf[s] && k < kd[s]) : k < kd[s]); }
  __device__ __forceinline__ bool mended(int k) const { return (active(0, k) && partly(0, k)) || (active(1, k) && partly(1, k)); }
};
// Walks this CTA's runs: one warp, all lanes hold the same values.  Lengths and starts are read more than once; where they have changed in
// between (by work on another stream), the walk ends early and says so: every loop is bounded by the batch, not by the sums.
template <bool kMask, bool kFew>
struct ChunkWalk {
  const ChunkParams& p;
  long long at = 0, end = 0, total = 0, item_at = 0;
  int ctas = 0, runs = 0, run = 0, b = 0, kvh = 0, i = 0, items = 0;
  SeqRows s;

  __device__ __forceinline__ explicit ChunkWalk(const ChunkParams& params) : p(params) {}
  // The lengths are not those that the work was counted from.
  __device__ __forceinline__ bool changed() const { return total < 0; }
  __device__ __forceinline__ bool give_up() {
    total = -1;
    return false;
  }
  // tiles that item i's tokens see, as (st, lo, hi)
  __device__ __forceinline__ void range(const SeqRows& q, int item, int* st, int* lo, int* hi) const {
    const int a = item * per_item(), e = min(q.n, a + per_item());
    const int uf = q.t - q.n + a + 1, ul = q.t - q.n + e;
    *hi = (ul + kCATile - 1) / kCATile;
    *lo = kMask ? first_visible(p, uf) / kCATile : 0;
    *st = kMask ? min((min(p.sinks, ul) + kCATile - 1) / kCATile, *lo) : 0;
  }
  __device__ __forceinline__ int cost(const SeqRows& q, int item) const {
    int st, lo, hi;
    range(q, item, &st, &lo, &hi);
    return st + hi - lo + kCAItemCost;
  }
  __device__ __forceinline__ int per_item() const { return kFew ? p.tokens : 2 * p.tokens; }
  __device__ __forceinline__ int items_of(const SeqRows& q) const { return (q.n + per_item() - 1) / per_item(); }
  __device__ __forceinline__ SeqRows seq(int at_b) const { return seq_rows(p.row_start, p.num_rows, p.kv.seq_lens, p.max_len, at_b); }
  // Sequence b0 + lane; none: no rows
  __device__ __forceinline__ SeqRows lane_seq(int b0) const {
    const int at_b = b0 + (int)(threadIdx.x & 31);
    SeqRows q{0, 0, 0, true};
    if (at_b < p.batch) q = seq(at_b);
    return q;
  }
  // Warp-collective: cost of all items of the lane's sequence (one KV head)
  __device__ __forceinline__ long long costs(const SeqRows& q) const {
    const int lane = threadIdx.x & 31;
    const int m = items_of(q);
    long long sum = 0;
    if (m <= 2)
      for (int x = 0; x < m; ++x) sum += cost(q, x);
    uint32_t many = __ballot_sync(0xffffffffu, m > 2);
    while (many) {
      const int src = __ffs(many) - 1;
      many &= many - 1;
      SeqRows r;
      r.n = __shfl_sync(0xffffffffu, q.n, src);
      r.t = __shfl_sync(0xffffffffu, q.t, src);
      const int mm = items_of(r);
      long long part = 0;
      for (int x = lane; x < mm; x += 32) part += cost(r, x);
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) part += __shfl_xor_sync(0xffffffffu, part, off);
      if (lane == src) sum = part;
    }
    return sum;
  }
  // The run that holds place x.
  __device__ __forceinline__ int run_of(long long x) const { return (int)(((x + 1) * runs - 1) / total); }

  // Warp-collective.  false: nothing for this CTA
  __device__ __forceinline__ bool begin() {
    long long seen = 0;           // tiles that are looked at, each once
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      const SeqRows q = lane_seq(b0);
      long long w = costs(q), v = 0;
      if (q.n > 0) {
        int st, lo, hi;
        range(q, 0, &st, &lo, &hi);
        v = st + (q.t + kCATile - 1) / kCATile - lo;
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) {
        w += __shfl_xor_sync(0xffffffffu, w, off);
        v += __shfl_xor_sync(0xffffffffu, v, off);
      }
      total += w;
      seen += v;
    }
    total *= p.num_kv_heads;
    seen *= p.num_kv_heads;
    if (total == 0) return false;
    ctas = (int)min((long long)gridDim.x, max(1ll, total / kCAMinRun));
    const long long rounds = min(min((seen + kCARoundTiles - 1) / kCARoundTiles, total / ((long long)ctas * kCARoundRun)), (long long)p.max_rounds);
    runs = ctas * (int)max(rounds, 1ll);
    run = (int)blockIdx.x;
    return run < ctas && seek();
  }
  // Warp-collective: to the beginning of run `run`.
  __device__ __forceinline__ bool seek() {
    const int lane = threadIdx.x & 31;
    if (run >= runs) return false;
    at = total * run / runs;
    end = total * (run + 1) / runs;
    // the sequence
    long long before = 0, one = 0;
    int b0 = 0;
    for (; b0 < p.batch; b0 += 32) {
      const SeqRows q = lane_seq(b0);
      const long long w = costs(q);
      long long incl = w * p.num_kv_heads;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += v;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + incl > at);
      if (past) {
        const int l = __ffs(past) - 1;
        b = b0 + l;
        one = __shfl_sync(0xffffffffu, w, l);
        s.r0 = __shfl_sync(0xffffffffu, q.r0, l);
        s.n = __shfl_sync(0xffffffffu, q.n, l);
        s.t = __shfl_sync(0xffffffffu, q.t, l);
        before += __shfl_sync(0xffffffffu, incl, l) - one * p.num_kv_heads;
        break;
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (b0 >= p.batch) return give_up();
    items = items_of(s);
    kvh = (int)((at - before) / one);
    before += one * kvh;
    // the item (of the lengths that its sequence was found with)
    int x0 = 0;
    for (; x0 < items; x0 += 32) {
      const int w = x0 + lane < items ? cost(s, x0 + lane) : 0;
      int incl = w;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += v;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + incl > at);
      if (past) {
        const int l = __ffs(past) - 1;
        i = x0 + l;
        item_at = before + __shfl_sync(0xffffffffu, incl - w, l);
        break;
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
    return x0 < items || give_up();
  }
  // Warp-collective.
  __device__ __forceinline__ bool next(Piece<kMask, kFew>& x) {
    if (at >= end) {
      run += ctas;
      if (!seek()) return false;
    }
    x.run = run;
    if (i == items) {
      i = 0;
      if (++kvh == p.num_kv_heads) {
        kvh = 0;
        do {
          if (++b >= p.batch) return give_up();
          s = seq(b);
        } while (s.n == 0);
        items = items_of(s);
      }
    }
    int hi;
    range(s, i, &x.st, &x.lo, &hi);
    const int w = x.st + hi - x.lo + kCAItemCost;
    const long long to = min(item_at + w, end);
    x.k0 = max((int)(at - item_at) - kCAItemCost, 0);
    x.k1 = max((int)(to - item_at) - kCAItemCost, 0);
    x.first_run = run_of(item_at);
    x.last_run = run_of(item_at + w - 1);
    if (x.last_run >= runs) return give_up();        // (there is no such run)
    x.b = b;
    x.kvh = kvh;
    x.row0 = s.r0 + i * per_item();
    x.ntok = min(s.n - i * per_item(), per_item());
    x.u0 = s.t - s.n + i * per_item() + 1;
    x.t = s.t;
    x.short_item = x.ntok <= p.tokens;
    x.ranges(p);
    at = to;
    if (to == item_at + w) {
      item_at = to;
      ++i;
    }
    return true;
  }
};

}  // namespace prhs
