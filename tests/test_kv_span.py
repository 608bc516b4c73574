"""Keys that a tile of attention's rows see over a paged cache (csrc/kv_span.h,
plain C++), compiled for the host: no stage leads past what the page table names,
whatever the lengths, windows and first tokens, and every key that a row sees
lies in one stage."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_18583_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "kv_span.h"
using namespace pard;

static int bad = 0;
static void say(const char* what, int stage, int lo, int hi, int cap, int window, int sinks, long long key) {
  if (++bad <= 20) printf("%s: stages of %d, positions %d .. %d, table %d, window %d, first %d: key %lld\n", what, stage, lo, hi, cap, window, sinks, key);
}

template <int STAGE>
static void check(int pos_lo, int pos_hi, int cap, int window, int sinks) {
  const KvSpan s = kv_span(pos_lo, pos_hi, cap, window, sinks, STAGE);
  // table entries are read for these stages, ahead of the last one too
  const int n = s.n_all;
  for (int st = 0; n > 0 && st <= n + 4; ++st) {
    if (st == 40 && n > 50) st = n - 4;
    for (int at = 0; at < STAGE; at += 16) {
      const KvRun k = kv_run(s, STAGE, st, at);
      const long long key = k.key < k.high ? k.key : k.high;
      if (key < 0 || key >= cap) say("read past the table", STAGE, pos_lo, pos_hi, cap, window, sinks, key);
    }
  }
  if (pos_hi > 4000 || pos_lo >= cap) return;          // (rows past the table are NaN whatever they read)
  std::vector<int> times(pos_hi + 1 > 0 ? pos_hi + 1 : 0);
  for (int st = 0; st < n; ++st) {
    const KvRun k = kv_run(s, STAGE, st, 0);
    for (int j = k.key > k.low ? k.key : k.low; j <= k.high && j < k.key + STAGE; ++j) ++times[j];
  }
  for (int j = 0; j <= pos_hi && j < cap; ++j) {
    bool seen = false;
    for (int p = pos_lo; p <= pos_hi; ++p) seen |= j <= p && (!window || j > p - window || j < sinks);
    if (times[j] > 1 || (seen && !times[j])) say(seen ? "times seen" : "twice", STAGE, pos_lo, pos_hi, cap, window, sinks, j);
  }
}

int main() {
  const int past[] = {-70, -1, 0, 1, 15, 16, 63, 64, 65, 255, 640, 1000, 1023, 1024, 1101, 2199, 3000, 1 << 20, 1 << 30, 2147483500};
  const int caps[] = {16, 64, 640, 1024, 1 << 30}, windows[] = {0, 1, 4, 16, 17, 100, 1000, 1 << 30};
  const int firsts[] = {0, 1, 4, 17, 64, 100, 300, 1000, 1025, 2048, 100000, 1 << 30};
  for (int lo : past)
    for (int more : {0, 1, 15, 16, 66, 130})
      for (int cap : caps)
        for (int window : windows)
          for (int sinks : firsts) {
            check<64>(lo, lo + more, cap, window, sinks);
            check<128>(lo, lo + more, cap, window, sinks);
          }
  printf("%d bad\n", bad);
  return bad != 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")
def test_stages_stay_within_the_table_and_hold_what_rows_see(tmp_path):
    src, exe = tmp_path / "spans.cpp", tmp_path / "spans"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, f"wrong stages:\n{res.stdout[:3000]}"
