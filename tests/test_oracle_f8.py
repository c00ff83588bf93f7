"""The oracle of 8-bit rows and sampling against independent statements of the same definitions."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo


def test_rows_against_torch_conversion():
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(5, 300)) * np.exp2(rng.integers(-20, 20, size=(5, 1)))).astype(np.float32)
    codes, scales = fo.quantize_rows(x)
    t = torch.nn.functional.pad(torch.from_numpy(x), (0, 84)).view(5, 3, 128)
    e = torch.from_numpy(scales.astype(np.int32)) - 127
    assert (t.abs().amax(2) <= 448 * torch.exp2(e.double())).all() and (t.abs().amax(2) > 448 * torch.exp2(e.double() - 1)).all()
    want = torch.ldexp(t, -e[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(torch.from_numpy(codes).view(5, 3, 128), want)
    assert np.array_equal(fo.rows_value(codes, scales, 300), (want.view(torch.float8_e4m3fn).double() * torch.exp2(e.double())[:, :, None]).view(5, -1)[:, :300].numpy())


def test_rows_of_zeros_infinities_and_nan():
    x = np.zeros((1, 256))
    x[0, 130:134] = np.inf, -np.inf, np.nan, 3.0
    codes, scales = fo.quantize_rows(x)
    assert scales.tolist() == [[7, 127 - 7]] and not codes[0, :128].any()
    assert codes[0, 130] == 0x7e and codes[0, 131] == 0xfe and codes[0, 132] & 0x7f == 0x7f and fo.rows_value(codes, scales, 256)[0, 133] == 3.0


@pytest.mark.parametrize("filters", [{}, {"top_k": 5}, {"top_p": 0.7}, {"min_p": 0.2}, {"top_k": 6, "top_p": 0.8, "min_p": 0.1, "temperature": 0.7}])
def test_tokens_come_out_with_their_probability(filters):
    """Over a fine grid of u each token's share is its filtered probability, and its log probability says so."""
    x = np.array([0.3, -1.0, 2.0, 2.0, -np.inf, 1.1, 0.0, np.nan, 1.7, -3.0])
    n = 20000
    tokens = [fo.sample(x, (i + 0.5) / n, **filters)[:2] for i in range(n)]
    for t in range(10):
        got = [lp for tok, lp in tokens if tok == t]
        if got:
            assert abs(len(got) / n - np.exp(got[0])) < 2 / n
    assert all(a[0] <= b[0] for a, b in zip(tokens, tokens[1:])) and not any(tok in (4, 7) for tok, _ in tokens)


def test_filters_by_hand():
    x = np.log([0.4, 0.1, 0.3, 0.2])
    kept = lambda **f: {fo.sample(x, u, **f)[0] for u in np.linspace(0, 0.999, 400)}
    assert kept(top_k=2) == {0, 2} and kept(top_p=0.5) == {0, 2} and kept(top_p=0.39) == {0} and kept(top_p=0.0) == {0}
    assert kept(min_p=0.45) == {0, 2, 3} and kept(min_p=2.0) == {0} and kept(temperature=0.0) == {0} and kept(top_k=3, top_p=0.8) == {0, 2, 3}
    assert kept(top_k=3, top_p=0.77) == {0, 2}
    tie = np.zeros(6)
    assert {fo.sample(tie, u, top_k=2)[0] for u in np.linspace(0, 0.999, 50)} == {0, 1} and {fo.sample(tie, u, top_p=0.4)[0] for u in np.linspace(0, 0.999, 50)} == {0, 1, 2}
    assert fo.sample([-np.inf, np.nan], 0.5)[0] == -1 and fo.sample([1.0, np.inf, np.inf], 0.9)[:2] == (2, np.log(0.5))
    assert fo.sample(tie, 1.0)[0] == 5 and fo.sample(tie, float("nan"))[0] == 0
