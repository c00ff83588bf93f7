"""Which sums 8-bit products have: results in bf16 are those in fp32 of the same sums, rounded once, and fast sums are had on request only, from every kernel and through the decoder."""
import pytest
import torch

from paper_2508_09204_amd import binding as mq
from paper_2508_09204_amd import decoder as dec
from paper_2508_09204_amd import experts as ex

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("M,n,k", [(1, 3000, 2000), (5, 9000, 900), (30, 700, 1700), (50, 700, 1700), (90, 1000, 2300), (250, 3000, 1500), (20, 20500, 700), (300, 4100, 513), (1000, 6500, 640),
                                   (1290, 4100, 300)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("fast", [False, True])
def test_bf16_results_are_fp32_ones_rounded(M, n, k, gated, fast):
    g = torch.Generator(device=DEV).manual_seed(M + n)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    a = ex.quantize_rows_f8(rand(M, k))
    mat = ex.quantize_f8(rand(n, k), rand(n, k) if gated else None)
    wide, narrow = torch.empty((M, n), dtype=F32, device=DEV), torch.empty((M, n), dtype=BF, device=DEV)
    mq.moqe_f8_gemm(a, [mat], wide, fast=fast)
    mq.moqe_f8_gemm(a, [mat], narrow, fast=fast)
    torch.cuda.synchronize()
    assert torch.equal(narrow, wide.to(BF))


def test_small_results_beside_large_ones():
    """Sums that cancel: 2^-12 of the others' size and less.  A rounding to bf16 is 2^-20 of that size at most, fp32 sums of 512 terms 2^-24 sqrt(4 + 128) of sum |a w|, 14.5 of the size, in the mean
    square: 1.1e-5 together, and under 1e-6 measured; sums of cut products are 1.8e-5 off."""
    M, n, k = 2000, 4096, 512
    g = torch.Generator(device=DEV).manual_seed(1)
    a, w = (ex.quantize_rows_f8(torch.randn((m, k), generator=g, device=DEV)) for m in (M, n))
    y = torch.empty((M, n), dtype=BF, device=DEV)
    mq.moqe_f8_gemm(a, [mq.F8Mat.pack(w)], y)
    want = a.float().double() @ w.float().double().T
    size = float(want.pow(2).mean().sqrt())
    small = want.abs() < 2.0 ** -12 * size
    assert int(small.sum()) > 1000
    assert float((y.double() - want)[small].pow(2).mean().sqrt()) / size < 1.1e-5


@pytest.mark.parametrize("fast", [False, True])
def test_a_decoders_products_have_the_sums_that_are_asked_for(fast):
    """Every 8-bit product of a layer again, by itself, on the rows that the layer gave it."""
    S, T, d, f = 4, 70, 256, 384
    model = dec.synthetic(1, d, f, 4, 2, 64, 3, seed=5, vocabulary=300, fast=True) if fast else dec.synthetic(1, d, f, 4, 2, 64, 3, seed=5, vocabulary=300)
    layer = model.layers[0]
    assert layer.fast == layer.mlp.fast == fast
    seqs = dec.Sequences(model, S, 128, 32, DEV)
    x = torch.randn((S * T, d), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
    seqs.route(model, x.to(BF), T)
    step = dec.Step(model, seqs, T)
    step.x.copy_(x)
    step()
    per_expert = dict(offsets=seqs.offsets, perm=seqs.perm, S=S, T=T, scatter=True)
    differ = 0
    for flag in (fast, not fast):
        h = mq.F8Rows.empty(S * T, f, DEV)
        y = torch.empty_like(step.y16)
        mq.moqe_f8_gemm(step.normed8, layer.mlp.gate_up, h, fast=flag, **per_expert)
        mq.moqe_f8_gemm(step.h8, layer.mlp.down, y, fast=flag, **per_expert)
        torch.cuda.synchronize()
        same = torch.equal(h.codes, step.h8.codes) and torch.equal(y, step.y16)
        assert same == (flag == fast)
        differ += not same
    assert differ == 1
