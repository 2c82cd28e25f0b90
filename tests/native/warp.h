// One warp of 32 lanes on the host, for code that is index arithmetic and warp votes alone: each lane is a fiber, and a vote or shuffle hands its
// value in and waits for the other lanes.  Loads (__ldg) go through a hook that may check their address or change what they give.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>
#include <unistd.h>

#include <algorithm>
#include <cmath>
#include <functional>
#include <vector>

using std::floor;
using std::max;
using std::min;

struct Dim {
  int x = 0, y = 0, z = 0;
};
static Dim threadIdx, blockIdx, gridDim;

[[noreturn]] static void die(const char* what) {
  fprintf(stderr, "FAILED: %s\n", what);
  _exit(1);               // (maybe on a fiber)
}

struct Warp {
  static constexpr size_t kStack = 256 * 1024;
  ucontext_t home, lane[32];
  std::vector<char> stacks = std::vector<char>(32 * kStack);
  bool done[32];
  uint64_t slot[2][32];
  int phase[32], at = 0;                // collectives that a lane has entered
  long long steps = 0, limit = 0;       // collectives; more than `limit` of them: it does not end
  std::function<void()> body;

  void to_next() {
    const int from = at;
    for (int i = 1; i <= 32; ++i) {
      const int n = (from + i) % 32;
      if (done[n]) continue;
      if (n == from) return;
      at = n;
      threadIdx.x = n;
      swapcontext(&lane[from], &lane[n]);
      return;
    }
  }
  // All lanes' values, in the order of lanes.
  const uint64_t* exchange(uint64_t v) {
    const int me = at, ph = phase[me]++;
    if (me == 0 && ++steps > limit) die("the walk does not end");
    slot[ph & 1][me] = v;
    for (int i = 0; i < 32; ++i)
      if (done[i]) die("a lane has left while others vote");
    for (;;) {
      bool all = true;
      for (int i = 0; i < 32; ++i) all &= phase[i] > ph;
      if (all) return slot[ph & 1];
      to_next();
    }
  }
  static void entry();
  void run(std::function<void()> f, long long most) {
    body = std::move(f);
    steps = 0;
    limit = most;
    for (int i = 0; i < 32; ++i) {
      done[i] = false;
      phase[i] = 0;
      getcontext(&lane[i]);
      lane[i].uc_stack.ss_sp = stacks.data() + i * kStack;
      lane[i].uc_stack.ss_size = kStack;
      lane[i].uc_link = &home;
      makecontext(&lane[i], &Warp::entry, 0);
    }
    for (int i = 0; i < 32; ++i) {
      if (done[i]) continue;
      at = i;
      threadIdx.x = i;
      swapcontext(&home, &lane[i]);
      i = -1;                           // (a lane that ends comes back here: on with the first that has not)
      bool any = false;
      for (int k = 0; k < 32; ++k) any |= !done[k];
      if (!any) return;
    }
  }
};
static Warp warp;
inline void Warp::entry() {
  warp.body();
  warp.done[warp.at] = true;
}

static std::function<int(const int*)> ldg_hook;
static inline int __ldg(const int* p) { return ldg_hook ? ldg_hook(p) : *p; }
static inline uint32_t __ballot_sync(uint32_t, bool v) {
  const uint64_t* s = warp.exchange(v);
  uint32_t m = 0;
  for (int i = 0; i < 32; ++i) m |= (uint32_t)(s[i] & 1) << i;
  return m;
}
template <typename T>
static inline T from_lane(T v, int src) {
  uint64_t raw = 0;
  memcpy(&raw, &v, sizeof v);
  const int me = warp.at;
  const uint64_t* s = warp.exchange(raw);
  T out;
  memcpy(&out, &s[src >= 0 && src < 32 ? src : me], sizeof out);
  return out;
}
template <typename T>
static inline T __shfl_sync(uint32_t, T v, int src) { return from_lane(v, src & 31); }
template <typename T>
static inline T __shfl_up_sync(uint32_t, T v, int by) { return from_lane(v, warp.at - by); }
template <typename T>
static inline T __shfl_xor_sync(uint32_t, T v, int by) { return from_lane(v, warp.at ^ by); }
static inline int __popc(uint32_t x) { return __builtin_popcount(x); }
static inline int __ffs(uint32_t x) { return __builtin_ffs((int)x); }
static inline float __uint_as_float(uint32_t x) {
  float f;
  memcpy(&f, &x, 4);
  return f;
}
static inline uint32_t __float_as_uint(float f) {
  uint32_t x;
  memcpy(&x, &f, 4);
  return x;
}
