// Keys that a tile of attention's rows see, in stages.  Plain C++: the kernels
// and the test of its bounds share it.
#pragma once

namespace pard {

// Keys key .. of one run, low .. high; those outside the run repeat its ends.
struct KvRun { int key, low, high; };

// The rows at positions pos_lo .. pos_hi see between them the first tokens 0 ..
// a_last (-1: none beside the others), then lo .. last, which has a page: the
// table names positions below cap.  Stages of `stage` keys: n_a of the first
// tokens, the others from key `from`, n_all together.  (Its form is the compiler's:
// with an early return for rows past the table 1000 rows of 64 dims over 9000
// keys took 197 us for 193.)
struct KvSpan { int lo, last, a_last, from, n_a, n_all; };
constexpr KvSpan kv_span(int pos_lo, int pos_hi, int cap, int window, int sinks, int stage) {
  const int last = pos_hi < cap - 1 ? pos_hi : cap - 1;
  int lo = window && pos_lo - window + 1 > 0 ? pos_lo - window + 1 : 0;
  int a_last = (sinks < lo ? sinks : lo) - 1;
  if (sinks >= lo) lo = 0, a_last = -1;                // one run of keys
  const int from = lo & ~15, n_a = (a_last + stage) / stage;
  // (rows all past the table are NaN whatever they see: without stages, since
  // neither run need end within the table then)
  return KvSpan{lo, last, a_last, from, n_a, last < 0 || pos_lo >= cap ? 0 : n_a + (last - from) / stage + 1};
}

// Stage st (any, those behind the last too) from its key `at` on.
constexpr KvRun kv_run(const KvSpan& s, int stage, int st, int at) {
  const bool in_a = st < s.n_a;
  return KvRun{(in_a ? st * stage : s.from + (st - s.n_a) * stage) + at, in_a ? 0 : s.lo, in_a ? s.a_last : s.last};
}

}  // namespace pard
