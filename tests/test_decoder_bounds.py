"""Who sees what at the borders of 32 bits, on the host: the window and prefix arithmetic of csrc/kv_cache.h against its definition in 64 bits."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# For rows at positions first .. first + rows - 1 of `len` tokens, where a table holds `tokens`: steps must hold every token that some row sees; where "all see" says so, all rows
# must see all 32 tokens; where "some see" denies it, none may see any; the lane's own rule must be the definition.
PROBE = r'''
#include "kv_cache.h"
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <cstring>
using namespace moqe;
static bool sees(long long p, long long t, long long len, long long window, long long prefix) {
  return t < len && (t < prefix || (t <= p && (window <= 0 || p - t < window)));
}
int main(int argc, char** argv) {
  const long long asked = atoll(argv[1]), prefix = atoll(argv[2]), tokens = atoll(argv[3]);
  long bad = 0, n = 0;
  for (int len = 0; len <= tokens && len <= 200; len += 9) for (int first = -40; first <= len; first += 3) for (int rows = 1; rows <= 45; rows += 11) {
    if (first + rows > len) continue;                       // rows are the last tokens
    const int last = first + rows - 1, window = kv_window(int(asked), tokens);
    const int pre = kv_prefix(int(prefix), len);
    int seen = last + 1 > pre ? last + 1 : pre;
    seen = seen < 0 ? 0 : seen > len ? len : seen;
    const KvSteps k = kv_steps(len, seen, first, window, pre);
    static char got[64];
    memset(got, 0, sizeof(got));
    for (int j = 0; j < k.count; ++j) { const int s = k.step(j); if (s < 0 || s * 32 >= len) ++bad; else got[s] = 1; }
    const KvRange all = kv_all_see(first, last, pre, window), some = kv_some_see(first, last, pre, window);
    for (int t0 = 0; t0 < len; t0 += 32) {
      bool every = true, any = false;
      for (int p = first; p <= last; ++p) {
        const KvSight lane = kv_sight(p, len, window);
        for (int t = t0; t < t0 + 32; ++t) {
          const bool is = sees(p, t, len, asked, prefix);
          every &= is;
          any |= is;
          if (t < len && lane.sees(t, pre) != is) ++bad;
        }
      }
      if (all.has(t0) && !every) ++bad;
      if (any && (!some.has(t0) || !got[t0 / 32])) ++bad;
      ++n;
    }
  }
  printf("%ld bad of %ld\n", bad, n);
  return 0;
}
'''


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    d = tmp_path_factory.mktemp("bounds")
    src, exe = d / "probe.cpp", d / "probe"
    src.write_text(PROBE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fwrapv", "-I", os.path.join(ROOT, "paper_2508_09204_amd", "csrc"), "-o", str(exe), str(src)], check=True)

    def run(*a):
        bad, n = subprocess.run([str(exe)] + [str(x) for x in a], check=True, capture_output=True, text=True).stdout.split(" bad of ")
        assert int(n) > 0 or a[2] == 0
        return int(bad)
    return run


@pytest.mark.parametrize("tokens", [32, 192, 1 << 30])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 30, 2 ** 31 - 31, 2 ** 30, 2 ** 30 - 1, 193, 192, 191, 33, 32, 31, 1, 0, -1, -2 ** 31])
def test_windows_of_any_size(probe, window, tokens):
    assert probe(window, 0, tokens) == 0
    assert probe(window, 40, tokens) == 0


@pytest.mark.parametrize("prefix", [-2 ** 31, -2 ** 31 + 30, -2 ** 31 + 31, -1, 0, 1, 31, 32, 100, 2 ** 30, 2 ** 31 - 1])
@pytest.mark.parametrize("window", [0, 50])
def test_prefixes_of_any_size(probe, prefix, window):
    assert probe(window, prefix, 192) == 0
