// The chunk attention's division of work, lane by lane on the host.
//   chunk_walk whole    every tile of every item is taken exactly once, and pieces, runs, slots and arrivals fit together
//   chunk_walk changed  lengths and starts that change while the work is being counted: the walk ends, in range, and says so
#include "warp.h"

#include "chunk_walk.cuh"

#include <map>
#include <random>
#include <set>
#include <tuple>

using namespace prhs;

struct Call {
  std::vector<int> lens, starts;
  int kv_heads, group, sinks = 0, window = 0, rounds = 4;
  double c = 0.0;
};

template <bool kFew>
ChunkParams params(const Call& x) {
  ChunkParams p{};
  p.kv.seq_lens = x.lens.data();
  p.row_start = x.starts.data();
  p.psaw_c = x.c;
  p.batch = (int)x.lens.size();
  p.num_rows = x.starts.back();
  p.num_kv_heads = x.kv_heads;
  p.num_q_heads = x.kv_heads * x.group;
  p.group = x.group;
  p.tokens = (kFew ? kCATile / 2 : kCATile) / x.group;
  p.max_rounds = x.rounds;
  p.sinks = x.sinks;
  p.window = x.window;
  p.max_len = 1 << 20;
  return p;
}

#define EXPECT(c) \
  if (!(c)) die(#c)

// What a walk gave: the pieces of one CTA, and what it says of lengths that have changed.
template <bool kMask, bool kFew>
std::vector<Piece<kMask, kFew>> walk_of(const ChunkParams& p, int cta, int* runs, bool* changed) {
  std::vector<Piece<kMask, kFew>> out;
  blockIdx.x = cta;
  warp.run([&] {
    ChunkWalk<kMask, kFew> w(p);
    Piece<kMask, kFew> x{};
    bool more = w.begin();
    while (more) {
      more = w.next(x);
      if (more && threadIdx.x == 0) out.push_back(x);
      if (out.size() > 200000) die("pieces without end");
    }
    if (threadIdx.x == 0) {
      *runs = w.runs;
      *changed = w.changed();
    }
  }, 2000000);
  return out;
}

// How many positions of tile k the token of visible length u sees.
template <bool kMask>
int sees(const ChunkParams& p, int u, int k) {
  const int lo = kMask ? first_visible(p, u) : 0;
  int n = 0;
  for (int i = k * kCATile; i < std::min(u, (k + 1) * kCATile); ++i) n += i >= lo || (kMask && i < p.sinks);
  return n;
}

template <bool kMask, bool kFew>
int whole(const Call& x, int sms) {
  const ChunkParams p = params<kFew>(x);
  gridDim.x = sms;
  typedef std::tuple<int, int, int> Item;                          // sequence, KV head, first row
  std::map<Item, std::set<int>> tiles, from;                       // tiles that were taken; the runs that have pieces of the item
  std::map<int, Item> slot_of, ticket_of;
  std::map<Item, int> parts;
  int runs = 0;
  for (int cta = 0; cta < sms; ++cta) {
    bool changed = false;
    int r = 0, last = -1;
    for (const auto& q : walk_of<kMask, kFew>(p, cta, &r, &changed)) {
      const Item item(q.b, q.kvh, q.row0);
      runs = std::max(runs, r);
      EXPECT(q.run % std::min(sms, r) == cta && q.run >= last && q.run < r);
      last = q.run;
      EXPECT(q.first_run >= 0 && q.first_run <= q.run && q.run <= q.last_run && q.last_run < r);
      EXPECT(q.k0 >= 0 && q.k0 <= q.k1);
      EXPECT(from[item].insert(q.run).second);
      EXPECT(parts.emplace(item, q.last_run - q.first_run + 1).first->second == q.last_run - q.first_run + 1);
      int odd = 0;
      for (int k = q.k0; k < q.k1; ++k) {
        EXPECT(tiles[item].insert(q.tile(k)).second);
        odd += q.mended(k);
        for (int s = 0; s < 2; ++s) {
          // the subtile's first and last token stand for those between: what a token sees begins and ends no earlier than before it
          bool any = false, all = true;
          for (int j = q.a(p, s); j < q.e(p, s); j += std::max(1, std::min(q.e(p, s) - 1 - j, 13))) {
            const int n = sees<kMask>(p, q.u0 + j, q.tile(k));
            any |= n > 0;
            all &= n == kCATile;
          }
          if (!q.halves()) EXPECT(q.active(s, k) || !any);
          if (!q.partly(s, k)) EXPECT(all);
        }
        if (q.halves()) EXPECT(q.active(0, k) != q.active(1, k));
      }
      EXPECT(odd <= 7);
      if (q.first_run != q.last_run) {
        EXPECT(slot_of.emplace(2 * q.run + (q.first_run == q.run ? 1 : 0), item).second);        // nobody else's
        EXPECT(ticket_of.emplace(q.first_run, item).first->second == item);
      }
    }
    EXPECT(!changed);
  }
  size_t items = 0;
  for (int b = 0; b < p.batch; ++b) {
    const int n = x.starts[b + 1] - x.starts[b], t = x.lens[b], per = kFew ? p.tokens : 2 * p.tokens;
    for (int a = 0; a < n; a += per)
      for (int h = 0; h < x.kv_heads; ++h) {
        const Item item(b, h, x.starts[b] + a);
        ++items;
        EXPECT(from.count(item) && (int)from[item].size() == parts[item]);                       // all of them arrive
        for (int j = a; j < std::min(n, a + per); j += std::max(1, std::min(std::min(n, a + per) - 1 - j, 13)))
          for (int k = 0; k * kCATile < t; ++k)
            if (sees<kMask>(p, t - n + j + 1, k)) EXPECT(tiles[item].count(k));
      }
  }
  EXPECT(items == from.size());
  return runs;
}

std::vector<int> sums(const std::vector<int>& n) {
  std::vector<int> s{0};
  for (int x : n) s.push_back(s.back() + x);
  return s;
}

template <bool kMask, bool kFew>
void changed_lengths(Call x, int sms, std::mt19937& rng) {
  const Call keep = x;
  ChunkParams p = params<kFew>(x);
  gridDim.x = sms;
  const int* lens0 = x.lens.data();
  const int* starts0 = x.starts.data();
  const int batch = p.batch;
  long long reads = 0, from = 0;
  int kind = 0;
  ldg_hook = [&](const int* a) {
    const bool is_len = a >= lens0 && a < lens0 + batch, is_start = a >= starts0 && a <= starts0 + batch;
    if (!is_len && !is_start) die("a read out of range");
    if (++reads <= from) return *a;
    if (kind == 0) return is_len ? 0 : *a;                                       // nothing fits any more
    if (kind == 1) return is_len ? std::max(1, *a / 2) : *a;                     // shorter
    if (kind == 2) return is_len ? std::min(p.max_len, 3 * *a + 500) : *a;       // longer
    return is_start ? (int)(a - starts0) : *a;                                   // a row each
  };
  int noticed = 0;
  for (kind = 0; kind < 4; ++kind)
    for (int tries = 0; tries < 12; ++tries) {
      reads = 0;
      from = 1ll << 60;
      int r = 0;
      bool changed = false;
      const int cta = (int)(rng() % (unsigned)sms);
      walk_of<kMask, kFew>(p, cta, &r, &changed);
      EXPECT(!changed);
      const long long all = reads;
      reads = 0;
      from = (long long)(rng() % (unsigned long long)std::max(all, 1ll));
      const auto got = walk_of<kMask, kFew>(p, cta, &r, &changed);
      noticed += changed;
      for (const auto& q : got) {
        EXPECT(q.b >= 0 && q.b < batch && q.kvh >= 0 && q.kvh < p.num_kv_heads && q.row0 >= 0 && q.ntok >= 1 && q.row0 + q.ntok <= p.num_rows);
        EXPECT(q.first_run >= 0 && q.first_run <= q.run && q.run <= q.last_run && q.last_run < r);
        EXPECT(q.k0 >= 0 && q.k0 <= q.k1 && (q.k1 == 0 || q.tile(q.k1 - 1) * kCATile < q.t) && q.t <= p.max_len);
      }
    }
  ldg_hook = nullptr;
  EXPECT(noticed > 0);
}

int main(int argc, char** argv) {
  std::mt19937 rng(argc > 2 ? atoi(argv[2]) : 1);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  auto any = [&](int most, int batch) {
    Call x;
    std::vector<int> n;
    for (int b = 0; b < batch; ++b) {
      x.lens.push_back(pick(0, most));
      n.push_back(std::min(x.lens.back(), pick(0, 3) ? pick(0, 9) : pick(0, 900)));
    }
    x.lens.push_back(most);
    n.push_back(std::min(most, 5));
    x.starts = sums(n);
    const int groups[] = {1, 2, 4, 7, 16};
    x.kv_heads = pick(1, 4);
    x.group = groups[pick(0, 4)];
    x.rounds = pick(1, 4);
    return x;
  };
  auto masked = [&](Call x) {
    const int sinks[] = {0, 4, 130, 5000}, windows[] = {0, 1, 100, 700, 4096};
    x.sinks = sinks[pick(0, 3)];
    x.window = windows[pick(0, 4)];
    x.c = pick(0, 1) ? 0.3 : x.window ? 0.0 : 1.0;
    return x;
  };
  if (argc > 1 && !strcmp(argv[1], "changed")) {
    for (int i = 0; i < 6; ++i) {
      changed_lengths<false, false>(any(3000, pick(1, 70)), pick(3, 148), rng);
      changed_lengths<true, false>(masked(any(3000, pick(1, 70))), pick(3, 148), rng);
      changed_lengths<false, true>(any(3000, pick(1, 70)), pick(3, 148), rng);
    }
    // several rounds: each begins with a look at the lengths
    Call x;
    x.lens = {40000, 9000};
    x.starts = sums({900, 300});
    x.kv_heads = 4;
    x.group = 4;
    changed_lengths<false, true>(x, 8, rng);
    return 0;
  }
  int most = 0;
  for (int i = 0; i < 12; ++i) {
    const int sms = pick(1, 148);
    whole<false, false>(any(pick(1, 2500), pick(0, 70)), sms);
    whole<true, false>(masked(any(pick(1, 2500), pick(0, 70))), sms);
    whole<false, true>(any(pick(1, 2500), pick(0, 70)), sms);
    whole<true, true>(masked(any(pick(1, 2500), pick(0, 70))), sms);
  }
  // more work than one round takes: items that go on from the last run of a round to the first of the next
  for (int rounds = 1; rounds <= 4; ++rounds) {
    Call x;
    x.lens = {33000, 700, 20000, 26001};
    x.starts = sums({700, 33, 0, 1400});
    x.kv_heads = 8;
    x.group = 4;
    x.rounds = rounds;
    const int got = whole<false, false>(x, 13);
    EXPECT(got == 13 * rounds);
    x.sinks = 130;
    x.window = 9000;
    whole<true, false>(x, 7);
    most = std::max(most, got);
  }
  printf("%d runs\n", most);
  return 0;
}
