"""8-bit rows and results at the end of fp32's range, against the 64-bit oracle bit for bit."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from oracle import f8_oracle as fo
from paper_2508_09204_amd import binding as mq
from tests.test_gpu_f8 import dev, empty_rows, f64, rows_of, sync

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_infinities_beside_the_largest_values(t):
    """The scale is 2^120 there, and 448 times it more than fp32 holds: infinities become the largest code of their sign all the same, and finite values keep theirs, bit for bit."""
    x = torch.zeros((7, 300), device=DEV)
    x[0, 3], x[0, 4], x[0, 5] = 3e38, INF, -INF
    x[1, :128] = torch.linspace(-1, 1, 128, device=DEV) * 3.3e38
    x[1, 40], x[1, 90] = INF, -INF
    x[2, 200], x[2, 201], x[2, 202], x[2, 203] = -3.3e38, -INF, float("nan"), 1e30
    x[3, 299], x[3, 298], x[3, 297] = 2.9e38, INF, 1.0                  # 2^119, the scale below
    x[4] = torch.exp2(torch.linspace(100, 127.9, 300, device=DEV))      # down to the smallest codes of 2^120 and zeros
    x[5, 0], x[5, 1], x[5, 2], x[5, 3] = 3e38, 2.0 ** 110, 2.0 ** 109 * 1.0000001, 1e-45
    x[6] = INF
    x = x.to(t)
    assert x[torch.arange(6), torch.tensor([3, 0, 200, 299, 299, 0])].isfinite().all()
    got = empty_rows(7, 300)
    mq.moqe_residual_norm_f8(None, x, got)
    sync()
    codes, scales = fo.quantize_rows(f64(x))
    assert scales[0, 0] == scales[1, 0] == scales[2, 1] == 127 + 120 and scales[3, 2] == 127 + 119 and codes[0, 4] == 0x7e and codes[0, 5] == 0xfe
    assert np.array_equal(got.scales[:, :3].cpu().numpy(), scales)
    ours, nan = got.codes.cpu().numpy(), (codes & 0x7f) == 0x7f
    assert np.array_equal(ours[~nan], codes[~nan]) and ((ours[nan] & 0x7f) == 0x7f).all()


@pytest.mark.parametrize("M,n,fast", [(3, 128, False), (70, 260, True), (1000, 3250, False), (1290, 2050, True)])
def test_gated_results_beside_infinities(M, n, fast):
    """Results of 1.875 * 2^127 and of plus and minus infinity in one block, through the workspace and from either tile: gates of 2^60, whose silu is themselves, times ups of 240 * 2^60, and of
    2^72 where results are infinite."""
    k = 128
    one = np.zeros((M, k))
    one[:, 0] = 2.0 ** 60
    gate, up = np.zeros((n, k)), np.zeros((n, k))
    gate[:, 0], up[:, 0] = 1.0, 240.0
    up[3::60, 0], up[4::60, 0], up[5::60, 0] = 2.0 ** 12, -2.0 ** 12, 2.0 ** 6
    a, av = rows_of(one)
    (g, gv), (u, uv) = rows_of(gate), rows_of(up)
    assert np.array_equal(av, one) and np.array_equal(gv, gate) and np.array_equal(uv, up)
    y = empty_rows(M, n)
    mq.moqe_f8_gemm(a, [mq.F8Mat.pack(g, u)], y, fast=fast)
    sync()
    want = 2.0 ** 120 * up[:, 0]
    want[np.abs(want) >= 2.0 ** 128] *= np.inf
    codes, scales = fo.quantize_rows(want[None])
    assert scales[0, 0] == 127 + 120 and codes[0, 3] == 0x7e and codes[0, 4] == 0xfe
    b = y.blocks
    assert (y.scales[:, :b].cpu().numpy() == scales).all() and (y.codes[:, : b * 128].cpu().numpy() == codes).all()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dh", [64, 128])
def test_infinities_beside_the_largest_keys_and_values(t, dh):
    """The same of the cache's blocks, whose tokens come 32 at a time and one by one."""
    rng = np.random.default_rng(dh)
    rows, bt = 40, 32
    x = np.where(rng.random((rows, 3 * dh)) < 0.5, 1.0, -1.0) * 2.0 ** 127 * rng.uniform(0.01, 1.99, size=(rows, 3 * dh))
    x[:, :dh] = 1.0
    x[3, dh + 7], x[35, dh + 1], x[20, 2 * dh + 9], x[9, 2 * dh + 8], x[39, 3 * dh - 1] = INF, -INF, INF, -INF, INF
    x = dev(x, torch.float32).to(t)
    cache = mq.KvCache.empty(2, 1, bt, dh, DEV)
    q = torch.empty((rows, dh), dtype=torch.bfloat16, device=DEV)
    mq.moqe_kv_append(x, 1, mq.Rope(None, 0), mq.KvBatch(dev(np.array([[1, 0]], np.int32)), dev(np.array([rows], np.int32)), 1, rows, rows), cache, q)
    sync()
    want = f64(x)
    tok, d = np.meshgrid(np.arange(bt), np.arange(dh), indexing="ij")
    for codes, scales, at, first in ((cache.k, cache.k_scale, do.key_at(tok, d, dh), dh), (cache.v, cache.v_scale, do.value_at(tok, d, dh), 2 * dh)):
        for n, block in enumerate((1, 0)):
            part = want[n * bt : (n + 1) * bt, first : first + dh]
            s = do.scale_for(np.abs(part[np.isfinite(part)]).max())
            assert s == 2.0 ** 120 == float(scales[block, 0]) and np.isinf(part).any()
            assert np.array_equal(codes[block, 0].cpu().numpy()[at][: len(part)], do.e4m3_code(part / s))
