"""f8_shape() of csrc/dispatch_rules.h, compiled for the host: the tiles that tests/test_gpu_f8_shapes.py runs, sizes where one side was measured to be faster, and what any size gets."""
import os
import subprocess

import pytest

from tests.f8_shapes import SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROBE = r'''
#include "dispatch_rules.h"
#include <initializer_list>
#include <cstdio>
#include <cstdlib>
#include <cstring>
int main(int argc, char** argv) {
  if (argc == 6) {
    const moqe::F8Shape s = moqe::f8_shape(atoll(argv[1]), atoi(argv[2]), atoi(argv[3]), atoi(argv[4]) != 0, atoi(argv[5]) != 0);
    printf("%d %d %d %d\n", s.rows, s.cols, s.parts, s.blocks);
    return 0;
  }
  for (long long M : {1, 2, 9, 16, 17, 32, 33, 64, 65, 100, 128, 129, 500, 1000, 10000, 1000000})
    for (int K : {1, 2, 3, 8, 16})
      for (int tiles : {1, 2, 8, 40, 160, 500, 2000, 60000})
        for (int gated = 0; gated < 2; ++gated)
          for (int exact = 0; exact < 2; ++exact) {
            const moqe::F8Shape s = moqe::f8_shape(M, K, gated ? 2 * tiles : tiles, gated, exact);
            const bool tile = s.blocks == 0 && ((s.rows == 128 && s.cols == 16 && s.parts == 1 && !exact) || (s.rows == 64 && (s.cols == 16 || s.cols == 8) && s.parts == 1) ||
                                                (s.rows == 32 && s.cols == 8 && s.parts == 1) || (gated && s.rows == 32 && s.cols == 8 && s.parts == 2) ||
                                                (!gated && s.rows == 64 && s.cols == 4 && s.parts == 2) || (!gated && s.rows == 32 && s.cols == 4 && s.parts == 4));
            const bool few = s.rows == 0 && ((s.blocks == 1 && (s.cols == 2 || (s.cols == 1 && !gated))) || (s.blocks == 2 && s.cols == 2 && !gated));
            if (!tile && !few) { printf("none: %lld %d %d %d %d\n", M, K, tiles, gated, exact); return 1; }
          }
  printf("all\n");
  return 0;
}
'''


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("f8rules")
    src, exe = d / "probe.cpp", d / "probe"
    src.write_text(PROBE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2508_09204_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    return lambda *a: subprocess.run([str(exe)] + [str(int(x)) for x in a], check=True, capture_output=True, text=True).stdout.strip()


def _shape(rule, M, K, n, gated, exact):
    return tuple(map(int, rule(M, K, -(-n // 16) * (2 if gated else 1), gated, exact).split()))


@pytest.mark.parametrize("shape,case", SHAPES)
def test_calls_take_the_tiles_they_are_meant_for(rule, shape, case):
    S, T, K, n, k, gated, exact = case
    assert _shape(rule, S * T, K, n, gated, exact) == shape


def test_any_size_has_a_kernel(rule):
    assert rule() == "all"


@pytest.mark.parametrize("args,shape", [
    ((64, 1, 32000, False, False), (64, 8, 1, 0)), ((128, 1, 32000, False, False), (64, 16, 1, 0)), ((512, 1, 32000, False, False), (128, 16, 1, 0)), ((512, 1, 4096, False, False), (64, 8, 1, 0)),
    ((256, 1, 4096, False, False), (64, 4, 2, 0)), ((128, 1, 4096, False, False), (32, 4, 4, 0)), ((128, 1, 32000, False, True), (64, 8, 1, 0)), ((1, 1, 32000, False, True), (0, 1, 1, 1)),
    ((16, 1, 32000, False, True), (32, 8, 1, 0)), ((16, 1, 4096, False, False), (0, 1, 1, 1)), ((64, 1, 4096, False, False), (0, 2, 1, 2)), ((16, 4, 11008, True, False), (0, 2, 1, 1)),
    ((64, 4, 11008, True, False), (32, 8, 1, 0)), ((8192, 1, 4096, False, False), (128, 16, 1, 0)), ((8192, 4, 11008, True, True), (64, 16, 1, 0)),
])
def test_the_faster_side(rule, args, shape):
    M, K, n, gated, exact = args
    assert _shape(rule, M, K, n, gated, exact) == shape
