"""Every kernel and tile of the 8-bit products on the GPU, in every type of result, against 64-bit products of the same values on the GPU.  Tolerances as in tests/test_gpu_f8.py."""
import numpy as np
import pytest
import torch

from paper_2508_09204_amd import binding as mq
from paper_2508_09204_amd import experts as ex
from tests.f8_shapes import SHAPES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _cut(a, w):
    pad = lambda x: torch.nn.functional.pad(x.abs(), (0, -x.shape[1] % 8)).view(len(x), -1, 8).amax(2)
    return 7 * 2.0 ** -13 * pad(a) @ pad(w).T


def _check(got, a, w, t, fast):
    rel = 2.0 ** -24 * (-(-a.shape[1] // 128) + 128)
    off = lambda m: rel * (a.abs() @ m.abs().T) + (_cut(a, m) if fast else 0)
    y = [a @ m.T for m in w]
    if len(w) == 1:
        want, tol = y[0], off(w[0])
    else:
        silu = y[0] / (1 + torch.exp(-y[0]))
        want = silu * y[1]
        tol = 1.1 * off(w[0]) * y[1].abs() + off(w[1]) * (silu.abs() + 1.1 * off(w[0])) + 2.0 ** -20 * want.abs() + 1e-37
    if t == "f8":
        b = got.blocks
        scale = torch.exp2(got.scales[:, :b].double() - 127).repeat_interleave(128, 1)[:, : got.d]
        v = got.float().double()
        near = tol.amax(1, keepdim=True)
        assert (v.abs() <= 448 * scale).all()
        assert ((v - want).abs() <= torch.maximum(2.0 ** -4 * want.abs(), scale * 2.0 ** -10) + 2.07 * near).all()
        top = torch.nn.functional.pad(want.abs(), (0, b * 128 - got.d)).view(len(want), b, 128).amax(2)
        s = torch.exp2(got.scales[:, :b].double() - 127)
        assert (top <= 448 * s + near).all() and ((top > 224 * s - near) | (got.scales[:, :b] == 7)).all()
        assert not got.codes[:, got.d : b * 128].any()
    else:
        assert ((got.double() - want).abs() <= tol + (2.0 ** -8 * (want.abs() + tol) if t == BF else 2.0 ** -24 * want.abs())).all()


@pytest.mark.parametrize("shape,case", SHAPES)
@pytest.mark.parametrize("scatter", [False, True])
def test_shape(shape, case, scatter):
    S, T, K, n, k, gated, exact = case
    g = torch.Generator(device=DEV).manual_seed(S + n + k)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV)
    M = S * T
    a = ex.quantize_rows_f8(rand(M, k) * torch.exp2(torch.randint(-4, 4, (M, 1), generator=g, device=DEV).float()))
    w = [[ex.quantize_rows_f8(rand(n, k) * k ** -0.5) for _ in range(2 if gated else 1)] for _ in range(K)]
    mats = [mq.F8Mat.pack(*x) for x in w]
    e = torch.randint(0, K, (S,), generator=g, device=DEV)
    perm = torch.argsort(e, stable=True).to(torch.int32)
    offsets = torch.cat([torch.zeros(1, device=DEV), torch.bincount(e, minlength=K).cumsum(0)]).to(torch.int32)
    for t in ([F32] if exact else [BF]) + (["f8"] if gated else []) + ([] if exact else [F32]):
        fast = t == BF or not exact
        y = mq.F8Rows.empty(M, n, DEV) if t == "f8" else torch.full((M, n), float("nan"), dtype=t, device=DEV)
        if K == 1 and not scatter:
            mq.moqe_f8_gemm(a, mats, y, fast=fast)
        else:
            mq.moqe_f8_gemm(a, mats, y, offsets, perm, S, T, scatter=scatter, fast=fast)
        torch.cuda.synchronize()
        order = (perm.long()[:, None] * T + torch.arange(T, device=DEV)).flatten()
        av, at = a.float().double()[order], 0
        for x in range(K):
            rows = int((e == x).sum()) * T
            if rows:
                here = slice(at, at + rows)
                pick = order[here] if K > 1 and scatter or K == 1 and scatter else torch.arange(M, device=DEV)[here]
                part = mq.F8Rows(y.codes[pick], y.scales[pick], rows, n) if t == "f8" else y[pick]
                _check(part, av[here], [m.float().double() for m in w[x]], t, fast)
            at += rows
