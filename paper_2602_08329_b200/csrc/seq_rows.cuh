// The packed rows of a sequence's new tokens.  Index arithmetic alone, with nothing that only a GPU has but the loads.
#pragma once

namespace prhs {

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

}  // namespace prhs
