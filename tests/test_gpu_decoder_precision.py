"""How far attention is from 64 bits in the mean, beside the worst case of the other tests: on long contexts outputs are small beside sum w |v|, and a bound by that alone would
let errors of some per cent of the outputs pass.

Roundings counted: the result's to bf16, uniform over a step 2^(e - 7), so step^2 / 12 in the mean square; the weights' to bf16 where a kernel has it (more than eight columns of row x query
head of a key head), as large again for values of one size: together at most 2^(1/2) 2^-7 / 12^(1/2) = 0.0032 of the outputs, 2^-8 allowed.  Up to eight columns weights are carried
in two pieces, 2^-17 of them: what is left is the error of the oracle itself when it is rounded to bf16, and 2 % for scores in fp32."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from paper_2508_09204_amd import binding as mq
from tests import test_gpu_decoder as tg

pytestmark = pytest.mark.gpu


def _errors(rows, lens, heads, kv, dh, bt, cap, slopes, window, seed):
    rng = np.random.default_rng(seed)
    table, n_blocks = tg._lay_out(rng, lens, bt)
    cache = tg._random_cache(rng, n_blocks, kv, bt, dh)
    tg._poison(cache, table, lens)
    batch, seqs, T = tg._batch(table, lens, rows)
    q = tg.dev(rng.normal(size=(batch.M, heads * dh)), torch.bfloat16)
    out = torch.empty_like(q)
    sl = 2.0 ** -(3 + np.arange(heads) % 5.0) if slopes else None
    mq.moqe_kv_attention(q, mq.Attention(heads, dh ** -0.5, cap, window, None if sl is None else tg.dev(sl, torch.float32)), batch, tg._on_device(cache), out)
    tg.sync()
    want, size = do.kv_attention(tg.f64(q), heads, cache, table, seqs, T, dh ** -0.5, cap, window, sl)
    want, size, got = want.reshape(batch.M, -1), size.reshape(batch.M, -1), tg.f64(out)
    return got - want, want, size


EXTRAS = [dict(cap=0.0, slopes=False, window=0), dict(cap=9.0, slopes=False, window=0), dict(cap=0.0, slopes=True, window=0), dict(cap=9.0, slopes=True, window=600)]


@pytest.mark.parametrize("extra", range(len(EXTRAS)))
@pytest.mark.parametrize("dh", [64, 128, 256])
@pytest.mark.parametrize("rows,heads,kv", [([1] * 12, 7, 1), ([1] * 12, 8, 4), ([4] * 5, 4, 2)])
def test_up_to_eight_columns_round_the_result_only(rows, heads, kv, dh, extra):
    lens = [40 + 211 * s for s in range(len(rows))]
    err, want, size = _errors(rows, lens, heads, kv, dh, 64, seed=dh + extra, **EXTRAS[extra])
    rounding = torch.from_numpy(want).to(torch.bfloat16).double().numpy() - want
    assert np.sqrt((err * err).sum()) <= 1.02 * np.sqrt((rounding * rounding).sum())
    assert (np.abs(err) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * size).all()


@pytest.mark.parametrize("extra", range(len(EXTRAS)))
@pytest.mark.parametrize("dh", [64, 128, 256])
@pytest.mark.parametrize("rows,heads,kv", [([4] * 4, 16, 4), ([5] * 4, 6, 1), ([40, 33, 70], 4, 2)])
def test_more_columns_round_the_weights_too(rows, heads, kv, dh, extra):
    lens = [100 + 450 * s for s in range(len(rows))]
    err, want, size = _errors(rows, lens, heads, kv, dh, 64, seed=dh + extra, **EXTRAS[extra])
    assert np.sqrt((err * err).sum()) <= 2.0 ** -8 * np.sqrt((want * want).sum())
    assert (np.abs(err) <= tg._attention_tol(want, size)).all()
