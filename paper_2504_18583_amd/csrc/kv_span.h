// Keys that a tile of attention's rows see, in stages.  Plain C++: the kernels
// and the test of its bounds share it.
#pragma once

namespace pard {

constexpr int kv_min(int a, int b) { return a < b ? a : b; }
constexpr int kv_max(int a, int b) { return a > b ? a : b; }

// Keys key .. of one run, low .. high; those outside the run repeat its ends.
struct KvRun { int key, low, high; };

// The rows at positions pos_lo .. pos_hi see between them the first tokens 0 ..
// a_last (-1: none beside the others), then lo .. last, which has a page: the
// table names positions below cap.
struct KvSpan { int lo, last, a_last; };
constexpr KvSpan kv_span(int pos_lo, int pos_hi, int cap, int window, int sinks) {
  const int last = kv_min(pos_hi, cap - 1), lo = window ? kv_max(pos_lo - window + 1, 0) : 0;
  if (pos_lo >= cap) return KvSpan{0, -1, -1};         // (such rows are NaN whatever they see)
  return sinks >= lo ? KvSpan{0, last, -1} : KvSpan{lo, last, sinks - 1};
}

// Stages of `stage` keys: n_a of the first tokens, the others from key `from`,
// n_all together.
constexpr int kv_from(const KvSpan& s) { return s.lo & ~15; }
constexpr int kv_first_stages(const KvSpan& s, int stage) { return (s.a_last + stage) / stage; }
constexpr int kv_stages(const KvSpan& s, int stage) {
  return s.last < 0 ? 0 : kv_first_stages(s, stage) + (s.last - kv_from(s)) / stage + 1;
}

// Stage st (any, those behind the last too) from its key `at` on.
constexpr KvRun kv_run(const KvSpan& s, int stage, int st, int at) {
  const int n_a = kv_first_stages(s, stage);
  const bool in_a = st < n_a;
  return KvRun{(in_a ? st * stage : kv_from(s) + (st - n_a) * stage) + at, in_a ? 0 : s.lo, in_a ? s.a_last : s.last};
}

}  // namespace pard
