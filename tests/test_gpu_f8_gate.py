"""The gate's function silu(g) u of 8-bit products by itself: products of one row whose gates and ups are exact in fp32.

Roundings on the way, relative to the result, in half steps of 2^-24: exponential and reciprocal two each (one step), the exponential's correction and its product, the sum in the denominator and
two products one each: nine, 2^-20.8.  Below g = -87.3 the reciprocal is under 2^-126 and may be 0: that loses |g| 2^-126, up to 2^-119 of u for g down to -128."""
import numpy as np
import pytest
import torch

from paper_2508_09204_amd import binding as mq
from tests.test_gpu_f8 import f64, result, rows_of, sync

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.mark.parametrize("M", [1, 3, 70, 300])
def test_silu_over_its_range(M):
    n, k = 4096, 64
    rng = np.random.default_rng(M)
    gate, up = np.zeros((n, k)), np.zeros((n, k))
    gate[:, 0] = rng.uniform(-104, 88, size=n) * rng.choice([1.0, 0.1, 1e-3], size=n)
    gate[:, 1] = rng.normal(size=n)                         # a second summand: gates of more digits than a code has
    up[:, 0] = rng.choice([1.0, 1.0, -1.5, 0.25], size=n)
    row = np.zeros((M, k))
    row[:, :2] = 1.0
    a, av = rows_of(row)
    (g, gv), (u, uv) = rows_of(gate), rows_of(up)
    y = result(M, n, F32)
    mq.moqe_f8_gemm(a, [mq.F8Mat.pack(g, u)], y)
    sync()
    x, v = gv.sum(1), uv[:, 0]
    assert np.array_equal(x.astype(np.float32), x) and (np.abs(x) > 40).sum() > 500 and np.array_equal(av, row)
    want = x / (1 + np.exp(-x)) * v
    got = f64(y)
    assert (got == got[0]).all()
    off = np.abs(got[0] - want)
    bad = off > np.where(x > -87, 2.0 ** -20.8 * np.abs(want), 2.0 ** -119 * np.abs(v))
    assert not bad.any(), (x[bad][:5], got[0][bad][:5], want[bad][:5])


def test_gates_without_end():
    """Infinite and huge gates, and NaN: g u for plus infinity, nothing for huge negative ones."""
    n, k = 16, 16
    gate, up = np.zeros((n, k)), np.zeros((n, k))
    gate[:6, 0] = [448 * 2.0 ** 100, -448 * 2.0 ** 100, 2.0 ** 60, -2.0 ** 60, 144.0, -144.0]
    up[:, 0] = 2.0
    row = np.zeros((2, k))
    row[0, 0], row[1, 0] = 1.0, 2.0 ** 26
    a, _ = rows_of(row)
    y = result(2, n, F32)
    mq.moqe_f8_gemm(a, [mq.F8Mat.pack(rows_of(gate)[0], rows_of(up)[0])], y)
    sync()
    got = f64(y)
    assert (got[0, :6] == [896 * 2.0 ** 100, 0, 2.0 ** 61, 0, 288, 0]).all() and (got[0, 6:] == 0).all()
    assert got[1, 0] == np.inf and got[1, 2] == 2.0 ** 113 and got[1, 3] == 0 and got[1, 4] == 288 * 2.0 ** 52
