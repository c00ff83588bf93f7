"""Every kernel of the attention at least once: head widths, what scores need beyond their scale, and column counts (rows x query heads of a key head) on either side of each border,
on short contexts and on such as are divided over work-groups, with masks that leave rows empty.  Tolerances as in test_gpu_decoder.py."""
import numpy as np
import pytest

from oracle import decoder_oracle as do
from paper_2508_09204_amd import binding as mq
from tests import test_gpu_decoder as tg

pytestmark = pytest.mark.gpu

SCORES = {"plain": {}, "cap": dict(cap=6.0), "bias": dict(slopes=True), "both": dict(cap=6.0, slopes=True), "far": dict(cap=5000.0), "far_bias": dict(cap=5000.0, slopes=True)}
COLUMNS = {  # rows, heads, key heads: form of the kernel by the largest number of columns
    8: ([2, 1, 2], 8, 2), 9: ([3, 0, 1], 6, 2), 16: ([4, 2, 1], 4, 1), 17: ([17, 3, 0], 2, 2), 32: ([8, 1, 5], 8, 2), 33: ([33, 2, 1], 1, 1), 130: ([65, 1, 40], 4, 2),
}


def form(columns, dh):
    """csrc/dispatch_rules.h: up to 32 columns in registers, 16 where the head is 256 wide."""
    if columns > (16 if dh == 256 else 32):
        return "many"
    return "pair" if columns <= 8 else "sixteen" if columns <= 16 else "thirty-two"


def test_every_form_is_here():
    for dh, forms in ((64, 4), (128, 4), (256, 3)):
        assert len({form(c, dh) for c in COLUMNS}) == forms
    for c, (rows, heads, kv) in COLUMNS.items():
        assert max(rows) * heads // kv == c


@pytest.mark.parametrize("columns", COLUMNS)
@pytest.mark.parametrize("scores", SCORES)
@pytest.mark.parametrize("dh", [64, 128, 256])
def test_attention_in_every_form(dh, scores, columns):
    rows, heads, kv = COLUMNS[columns]
    tg._check_attention(rows, [150, 40, 97], heads, kv, dh, 32, seed=900, **SCORES[scores])
    tg._check_attention(rows, [2700, 70, 1300], heads, kv, dh, 64, seed=901, window=1200, prefix=[40, -1, 0], absent=[(0, 0), (0, 25), (2, 20)], **SCORES[scores])


@pytest.mark.parametrize("rows,heads,kv", [([2], 4, 1), ([4], 4, 1), ([8], 4, 1), ([8], 2, 1), ([16], 2, 1)])
@pytest.mark.parametrize("dh,L", [(64, 180), (128, 180), (128, 2600), (256, 180), (64, 2600)])
@pytest.mark.parametrize("window", [0, 100])
def test_nan_in_the_cache_in_every_form_of_few_rows(rows, heads, kv, dh, L, window):
    """Values of two tokens are NaN in one dim each, one of them between the call's rows, one at the window's lower edge: rows that see them, and no others, have NaN there."""
    rng = np.random.default_rng(dh + L)
    bt, n = 32, rows[0]
    table, n_blocks = tg._lay_out(rng, [L], bt)
    cache = tg._random_cache(rng, n_blocks, kv, bt, dh)
    clean = do.Cache(n_blocks, kv, bt, dh)
    clean.k, clean.v, clean.k_scale, clean.v_scale = cache.k.copy(), cache.v.copy(), cache.k_scale, cache.v_scale
    bad = [(L - 1 - n // 2, 7), (L - 100 - n // 2, dh - 3)]
    for tok, dim in bad:
        cache.v[table[0, tok // bt], 0][cache.at["v"][tok % bt, dim]] = 0xff
        clean.v[table[0, tok // bt], 0][cache.at["v"][tok % bt, dim]] = 0
    batch, seqs, T = tg._batch(table, [L], rows)
    q = tg.dev(rng.normal(size=(n, heads * dh)), tg.BF)
    out = q.clone()
    mq.moqe_kv_attention(q, mq.Attention(heads, dh ** -0.5, window=window), batch, tg._on_device(cache), out)
    tg.sync()
    want, size = do.kv_attention(tg.f64(q), heads, clean, table, seqs, T, dh ** -0.5, 0.0, window)
    got, p = tg.f64(out).reshape(n, heads, dh), np.arange(L - n, L)
    hit = np.zeros(got.shape, bool)
    for tok, dim in bad:
        hit[:, :, dim] |= ((tok <= p) & ((p - tok < window) if window else True))[:, None]
    assert np.array_equal(np.isnan(got), hit)
    assert (np.abs(got - want)[~hit] <= tg._attention_tol(want, size)[~hit]).all()


@pytest.mark.parametrize("bt", [32, 64, 128])
@pytest.mark.parametrize("dh", [64, 128, 256])
@pytest.mark.parametrize("t", [tg.F32, tg.BF])
def test_append_in_every_form(t, dh, bt):
    """Head widths, types and block sizes; one row a sequence and as many as fill blocks, scales that grow, with and without head norms."""
    for inter in (False, True):
        c = dict(heads=4, kv=2, dh=dh, bt=bt, t=t, rot=dh if inter else dh // 2, inter=inter, norm=inter)
        tg._check_append(dict(c, rows=[1, 1, 1], lens=[1, bt + 1, 3 * bt]), seed=910)
        tg._check_append(dict(c, rows=[bt + 5, 2, 2 * bt], lens=[2 * bt + 9, bt + 1, 2 * bt]), seed=911)
