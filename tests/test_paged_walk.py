"""The walk of a block of rows over windows (csrc/paged_walk.h), compiled for the CPU with
overflow checks: what its page lookups ask for lies in the sequence, wherever rows stand,
and its tiles are those that hold what the rows see."""
import os
import shutil
import subprocess

import pytest

from paper_2506_12035_amd import build

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>
#include "paged_walk.h"
using namespace marche;
static const long long BIG = 2147483647;
static long long checked = 0;
[[noreturn]] static void fail(const char *what, long long len, long long t, long long w, long long s, long long x) {
  std::printf("%s: len %lld, token %lld, window %lld, sinks %lld: %lld\n", what, len, t, w, s, x);
  std::exit(1);
}
struct Rows {
  int lo, hi;
};
// earliest start (of rows that see any token) and latest end of rows at tokens t0 .. t1, in 64 bits
static Rows rows_of(long long len, long long t0, long long t1, long long window) {
  Rows r{(int)BIG, 0};
  for (long long t : {std::min(std::max(t0, 0LL), t1), t1}) {
    const long long hi = t < 0 ? 0 : std::min(t + 1, len), lo = std::max(t - (window - 1), 0LL);
    if (hi > 0) r.lo = std::min<int>(r.lo, (int)lo);
    r.hi = std::max<int>(r.hi, (int)hi);
  }
  return r;
}
template <int TK>
static void lookups(long long len, long long t0, long long t1, long long window, long long sinks) {
  const Rows r = rows_of(len, t0, t1, window);
  const auto walk = WindowWalk<TK>::of(r.lo, r.hi, (int)sinks);
  if (walk.tiles < 0 || walk.tiles > (len + TK - 1) / TK) fail("tiles", len, t1, window, sinks, walk.tiles);
  const auto key = [&](int place) { return walk.key(place); };
  for (int splits : {1, 3, 64}) {
    const int chunk = (walk.tiles + splits - 1) / splits;
    for (int i = 0; i < splits; ++i) {
      const int first = i * chunk, stop = std::min(first + chunk, walk.tiles);
      // a lookup of 16 tiles at the range's first ones and at its last ones
      for (int base : {first, first + 1, stop - 17, stop - 2, stop - 1}) {
        if (base < first || base >= stop) continue;
        for (int ahead = 0; ahead < 16; ++ahead)
          for (int part = 0; part < TK / 16; ++part) {
            const int token = token_of(key, base + ahead, stop, part, r.hi);
            ++checked;
            if (token < -1 || token >= len) fail("lookup", len, t1, window, sinks, token);
            if (base + ahead < stop && token < 0 && key(base + ahead) + 16LL * part < r.hi)
              fail("lookup left out", len, t1, window, sinks, base + ahead);
          }
      }
    }
  }
}
template <int TK>
static void tiles(int len, int t0, int t1, int window, int sinks) {
  const Rows r = rows_of(len, t0, t1, window);
  const auto walk = WindowWalk<TK>::of(r.lo, r.hi, sinks);
  std::set<int> in;
  for (int p = 0; p < walk.tiles; ++p) {
    if (walk.key(p) % TK || walk.key(p) >= r.hi) fail("tile", len, t1, window, sinks, walk.key(p));
    if (!in.insert(walk.key(p)).second) fail("tile twice", len, t1, window, sinks, walk.key(p));
  }
  for (int t = std::max(t0, 0); t <= t1; ++t)
    for (int j = 0; j < len && j <= t; ++j)
      if ((j > (long long)t - window || j < sinks) && !in.count(j / TK * TK)) fail("token left out", len, t, window, sinks, j);
}
int main() {
  const std::vector<long long> lens = {0, 1, 15, 16, 63, 64, 65, 1000, 4097, 1 << 20, BIG - 65535};
  const std::vector<long long> windows = {1, 2, 64, 256, 960, 1024, 100000, 1 << 30, BIG - 1, BIG};
  const std::vector<long long> sinks = {0, 1, 4, 64, 100, 1 << 20, BIG};
  std::vector<long long> tokens = {-BIG - 1, -1, 0, 1, 63, 64, 500, 999, 1000, 1 << 20, 1 << 30};
  for (long long w : windows)
    for (long long d : {0LL, 1LL, 63LL, 64LL, 900LL, 960LL, 1024LL, 5000LL})
      for (long long t : {BIG - d, BIG - w - d, BIG - w + d})
        if (t >= 0 && t <= BIG) tokens.push_back(t);
  for (long long len : lens)
    for (long long w : windows)
      for (long long s : sinks)
        for (long long t : tokens)
          for (long long before : {0LL, 1LL, 127LL}) {
            const long long t0 = std::max(t - before, -BIG - 1);
            lookups<64>(len, t0, t, w, s);
            lookups<32>(len, t0, t, w, s);
          }
  for (int len : {0, 1, 31, 32, 33, 64, 130, 200})
    for (int w : {1, 2, 31, 32, 33, 64, 65, 150, 300})
      for (int s : {0, 1, 31, 32, 33, 65, 129, 400})
        for (int t : {-3, 0, 1, 31, 32, 63, 64, 100, 199, 260, 500})
          for (int before : {0, 1, 20, 90}) {
            tiles<64>(len, t - before, t, w, s);
            tiles<32>(len, t - before, t, w, s);
          }
  std::printf("checked %lld lookups\n", checked);
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not installed")
def test_lookups_of_a_window_stay_in_its_sequence(tmp_path):
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(PROGRAM)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                        "-I", os.path.join(build.CSRC), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr
    assert int(r.stdout.split()[1]) > 100000
