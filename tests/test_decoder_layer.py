"""The decoder of decoder.py without a GPU: its frequencies, what a step refuses, and all of its calls with their arguments checked (dry-run mode)."""
import math

import pytest
import torch

from paper_2508_09204_amd import decoder as dec


@pytest.fixture(scope="module")
def mq():
    from paper_2508_09204_amd import binding
    binding.moqe_set_dry_run(True)
    yield binding
    binding.moqe_set_dry_run(False)


def test_rope_frequencies():
    f = dec.rope_frequencies(64, 1e4, device="cpu")
    assert f.dtype == torch.float64 and f.shape == (32,) and float(f[0]) == 1.0 and math.isclose(float(f[16]), 1e-2, rel_tol=1e-12)
    assert torch.equal(dec.rope_frequencies(64, 1e4, stretch=4.0, device="cpu"), f / 4)
    parts = dec.rope_frequencies(64, 1e4, stretch=4.0, by_parts=(4096, 32.0, 1.0), device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(parts[turns > 32], f[turns > 32]) and torch.allclose(parts[turns < 1], f[turns < 1] / 4, rtol=1e-12)
    between = (turns < 32) & (turns > 1)
    assert between.any() and (parts[between] < f[between]).all() and (parts[between] > f[between] / 4).all()


def _aligned(nbytes):
    t = torch.zeros(nbytes + 256, dtype=torch.uint8)
    at = -t.data_ptr() % 256
    return t[at:at + nbytes]


def _model(mq, layers=2, d=256, f=512, heads=4, kv=2, dh=64, K=3):
    def matrix(n, k):
        return [mq.QMat(_aligned(mq.moqe_packed_bytes(n, k, 4, 128, False)), None, None, n, k, 4, 128, False, 0, mq.LAYOUT_PACKED) for _ in range(K)]
    router = mq.Router(None, None, torch.zeros(K, d), None, d, 0, K)
    norm = lambda: mq.Norm("rms", 1e-6, torch.ones(d))
    made = [dec.Layer(norm(), matrix((heads + 2 * kv) * dh, d), matrix(d, heads * dh), norm(),
                      mq.Block(kind=mq.KIND_SILU_MLP, router=router, w0=matrix(f, d), w1=matrix(f, d), w2=matrix(d, f))) for _ in range(layers)]
    return dec.Decoder(made, norm(), router, mq.Rope(dec.rope_frequencies(dh, device="cpu"), dh), heads, kv, dh)


def test_a_step_passes_every_check(mq):
    model = _model(mq)
    seqs = dec.Sequences(model, 3, 100, 32, device="cpu")
    assert seqs.block_table.shape == (3, 4) and len(seqs.caches) == 2
    prompt, token = dec.Step(model, seqs, 97, _aligned(1 << 24)), dec.Step(model, seqs, 1, _aligned(1 << 24))
    assert prompt().shape == (3 * 97, 256) and int(seqs.kv_len[0]) == 97
    for _ in range(3):
        token()
    assert int(seqs.kv_len[2]) == 100
    with pytest.raises(ValueError):
        token()
    seqs.clear()
    assert int(seqs.kv_len.sum()) == 0 and token().shape == (3, 256)


def test_a_step_refuses_a_short_workspace(mq):
    model = _model(mq, layers=1)
    with pytest.raises(ValueError):
        dec.Step(model, dec.Sequences(model, 2, 100, 32, device="cpu"), 1, _aligned(256))


@pytest.mark.parametrize("T", [0, 101])
def test_a_step_refuses_rows(mq, T):
    model = _model(mq, layers=1)
    with pytest.raises(ValueError):
        dec.Step(model, dec.Sequences(model, 2, 100, 32, device="cpu"), T)


def test_a_step_refuses_vectors_of_another_width(mq):
    model = _model(mq, layers=1)
    model.final_norm = mq.Norm("rms", 1e-6, torch.ones(8))
    with pytest.raises(ValueError):
        dec.Step(model, dec.Sequences(model, 2, 100, 32, device="cpu"), 1)
