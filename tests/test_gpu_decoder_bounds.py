"""Arguments at the ends of their ranges, on the GPU against the 64-bit oracle.  Tolerances as in test_gpu_decoder.py."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from paper_2508_09204_amd import binding as mq
from tests import test_gpu_decoder as tg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 30, 2 ** 30, 300])
@pytest.mark.parametrize("rows,lens", [([130, 33, 80], [130, 33, 200]), ([100, 60], [50, 61]), ([1, 1], [1, 300]), ([3, 8], [3, 5])])
def test_windows_that_hide_nothing(window, rows, lens):
    """Fresh prompts, prompts with rows below position 0 and single rows: the window of any length is as none."""
    got = tg._check_attention(rows, lens, 4, 2, 64, 32, window=window, seed=800)
    none = tg._check_attention(rows, lens, 4, 2, 64, 32, window=0, seed=800)
    assert (got == none).all()


@pytest.mark.parametrize("rows,lens", [([130, 40], [130, 200]), ([2, 1], [40, 300])])
def test_prefixes_at_the_ends_of_their_range(rows, lens):
    """A prefix below 0 is none, one past the last token is all of them."""
    for window in (0, 20):
        for prefix in (-2 ** 31, -2 ** 31 + 20, -1, 2 ** 31 - 1):
            tg._check_attention(rows, lens, 4, 2, 64, 32, window=window, prefix=[prefix] * 2, seed=801)


@pytest.mark.parametrize("dh,rot", [(64, 16), (64, 32), (128, 64), (256, 16), (64, 0)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_rotation_leaves_the_other_dims_alone(dh, rot, inter, t):
    """Infinities and NaN in every dim in turn, past the rotation among them: a turned pair spoils itself, what is not turned keeps its value, queries and keys alike.
    Keys that are not turned have the code of the value itself; the turned ones that are finite may have a neighbour's."""
    bt, rows = 32, 32
    rng = np.random.default_rng(dh + rot)
    host = rng.normal(size=(rows, 3 * dh))
    for i in range(rows):
        host[i, i * 7 % dh] = host[i, dh + i * 5 % dh] = (np.inf, -np.inf, np.nan)[i % 3]
    for i in range(12):                                      # a row each for the dims around the rotation's end
        host[i, :2 * dh] = rng.normal(size=2 * dh)
        host[i, (rot - 2 + i) % dh] = host[i, dh + (rot - 2 + i) % dh] = (np.inf, np.nan)[i % 2]
    x = torch.from_numpy(host).to(tg.DEV, t)
    f = 100.0 ** (-2.0 * np.arange(rot // 2) / max(1, rot))
    i32 = dict(dtype=torch.int32, device=tg.DEV)
    cache, batch = do.Cache(1, 1, bt, dh), mq.KvBatch(torch.zeros((1, 1), **i32), torch.full((1,), rows, **i32), 1, rows, rows)
    d, q = tg._on_device(cache), torch.empty((rows, dh), dtype=torch.bfloat16, device=tg.DEV)
    mq.moqe_kv_append(x, 1, mq.Rope(tg.dev(f) if rot else None, rot, inter, 1.125), batch, d, q)
    tg.sync()
    with np.errstate(invalid="ignore"):
        want = do.kv_append(tg.f64(x), 1, cache, np.zeros((1, 1), int), do.sequences(1, rows, rows, [rows], 1, bt), rows, f, rot, inter, 1.125).reshape(rows, dh)
    got = tg.f64(q)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    size = np.abs(np.where(np.isfinite(host), host, 0.0)).max()
    assert (np.abs(got[fine] - want[fine]) <= 2.0 ** -8 * np.abs(want[fine]) + 2.0 ** -19 * 2.5 * size).all()
    at = cache.at["k"][:rows]
    code, right = d.k.cpu().numpy()[0, 0][at], cache.k[0, 0][at]
    gv, wv = do.e4m3_value(code), do.e4m3_value(right)
    same = (code == right) | (np.isnan(gv) & np.isnan(wv)) | ((gv == 0) & (wv == 0))
    assert float(d.k_scale[0, 0]) == cache.k_scale[0, 0] and np.array_equal(np.isnan(gv), np.isnan(wv))
    assert same[:, rot:].all() and (np.abs(code.astype(int) - right.astype(int))[~same] == 1).all() and (~same).mean() < 2e-3


@pytest.mark.parametrize("cap", [1e-3, 0.5, 30.0, 1e3, 1e4, 1e6, 1e12, 3e38, 1e300])
@pytest.mark.parametrize("rows,dh", [([1, 1], 128), ([9, 4], 64), ([70, 40], 128), ([40, 70], 256)])
def test_caps_of_any_size(cap, rows, dh):
    """Scores far below the cap are the scores, those far above are the cap; past the largest fp32 (1e300) it is infinite, so none."""
    for q_by in (0.2, 3.0):
        tg._check_attention(rows, [90, 200], 4, 2, dh, 32, cap=cap, q_by=q_by, seed=802)
    tg._check_attention(rows, [90, 200], 4, 2, dh, 32, cap=cap, slopes=True, seed=803)


@pytest.mark.parametrize("T,heads,dh", [(1, 4, 64), (4, 4, 128), (8, 8, 64), (3, 4, 256), (40, 4, 64)])
@pytest.mark.parametrize("prefix", [None, 20])
def test_rows_past_the_call_s_own_and_their_tokens(T, heads, dh, prefix):
    """Sequences with more rows than the call computes: the tokens of the others, never stored, have no influence, whatever their blocks hold."""
    rng = np.random.default_rng(T)
    bt, H, rows, lens = 32, 2, [T + 150, 1, T + 40], [700, 90, T + 40]
    table, n_blocks = tg._lay_out(rng, lens, bt)
    cache = tg._random_cache(rng, n_blocks, H, bt, dh)
    for s, (n, L) in enumerate(zip(rows, lens)):
        stored = L - n + min(n, T)
        for b in range(-(-stored // bt), -(-L // bt)):
            for which in ("k", "v"):
                cache.codes(which)[table[s, b]] = 0x7f if b % 2 else 0x55
                cache.scales(which)[table[s, b]] = (np.nan, np.inf)[s % 2]
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    M = int(cu[-1])
    seqs = do.sequences(len(rows), T, M, lens, table.shape[1], bt, cu)
    batch = mq.KvBatch(tg.dev(table), tg.dev(np.array(lens, dtype=np.int32)), len(rows), T, M, tg.dev(cu))
    q = tg.dev(rng.normal(size=(M, heads * dh)), torch.bfloat16)
    out = torch.full_like(q, 7.0)
    pre = None if prefix is None else np.full(len(rows), prefix, dtype=np.int32)
    mq.moqe_kv_attention(q, mq.Attention(heads, dh ** -0.5, prefix=None if pre is None else tg.dev(pre)), batch, tg._on_device(cache), out)
    tg.sync()
    want, size = do.kv_attention(tg.f64(q), heads, cache, table, seqs, T, dh ** -0.5, prefix=pre)
    want, size, got = want.reshape(M, -1), size.reshape(M, -1), tg.f64(out)
    done = ~np.isnan(want)
    assert done.any() and (np.abs(got[done] - want[done]) <= tg._attention_tol(want, size)[done]).all() and (got[~done] == 7.0).all()


def _attend(q, heads, kv, dh, bt, rows, lens, scale, slopes=None, seed=810, prefix=None):
    """Outputs and the oracle's, with the sums over |v|."""
    rng = np.random.default_rng(seed)
    table, n_blocks = tg._lay_out(rng, lens, bt)
    cache = tg._random_cache(rng, n_blocks, kv, bt, dh)
    tg._poison(cache, table, lens)
    batch, seqs, T = tg._batch(table, lens, rows)
    x = tg.dev(q, torch.bfloat16)
    out = torch.full_like(x, 7.0)
    mq.moqe_kv_attention(x, mq.Attention(heads, scale, slopes=None if slopes is None else tg.dev(slopes, torch.float32)), batch, tg._on_device(cache), out)
    tg.sync()
    with np.errstate(invalid="ignore", over="ignore"):
        want, size = do.kv_attention(tg.f64(x), heads, cache, table, seqs, T, scale, slopes=slopes)
    return tg.f64(out), want.reshape(batch.M, -1), size.reshape(batch.M, -1)


FORMS = [([1, 1], 4, 2), ([4, 3], 8, 2), ([9, 4], 4, 2), ([70, 40], 4, 2)]


@pytest.mark.parametrize("scale", [0.0, -0.125, 1e-30, 1e6])
@pytest.mark.parametrize("rows,heads,kv", FORMS)
def test_scales_of_any_sign_and_size(rows, heads, kv, scale):
    """Scale 0 is the mean of what a row sees, a negative one prefers the smallest products, a large one leaves the largest alone (here by a score of thousands)."""
    q = np.random.default_rng(5).normal(size=(sum(rows), heads * 64))
    got, want, size = _attend(q, heads, kv, 64, 32, rows, [90, 200], scale)
    assert (np.abs(got - want) <= tg._attention_tol(want, size)).all()


@pytest.mark.parametrize("by", [-0.25, 40.0])
@pytest.mark.parametrize("rows,heads,kv", FORMS)
def test_slopes_of_any_sign_and_size(rows, heads, kv, by):
    """Negative slopes prefer far tokens, large ones leave a row its own token alone."""
    q = np.random.default_rng(6).normal(size=(sum(rows), heads * 64))
    got, want, size = _attend(q, heads, kv, 64, 32, rows, [90, 200], 0.125, slopes=by * (1 + np.arange(heads)))
    assert (np.abs(got - want) <= tg._attention_tol(want, size)).all()


@pytest.mark.parametrize("rows,heads,kv", [([3, 3], 2, 1), ([4, 4], 4, 1), ([8, 8], 4, 1), ([70, 40], 4, 2)])
def test_rows_of_nan_and_infinities_keep_apart(rows, heads, kv):
    q = np.random.default_rng(7).normal(size=(sum(rows), heads * 64))
    q[1, 5], q[rows[0], 64 + 3], q[-1, 0] = np.nan, np.inf, -np.inf
    got, want, size = _attend(q, heads, kv, 64, 32, rows, [90, 200], 0.125)
    fine = np.ones(got.shape, bool)
    for r, h in ((1, 0), (rows[0], 1), (len(q) - 1, 0)):
        fine[r, h * 64:(h + 1) * 64] = False
    assert np.isnan(got[1, :64]).all() and (np.abs(got - want)[fine] <= tg._attention_tol(want, size)[fine]).all()


@pytest.mark.parametrize("rows,heads,kv,lens", [([1, 1], 150, 1, [300, 40]), ([3, 2], 150, 1, [90, 700]), ([1] * 3, 96, 96, [40, 1, 90]), ([1, 2], 640, 640, [33, 40])])
def test_many_heads(rows, heads, kv, lens):
    """More query heads to a key head than a tile has columns, and more key heads than work-groups run at once."""
    tg._check_attention(rows, lens, heads, kv, 64, 32, seed=820)


def test_six_hundred_sequences():
    n = 600
    tg._check_attention([1] * n, [1 + (s * 131) % 300 + (2300 if s % 97 == 5 else 0) for s in range(n)], 2, 1, 64, 32, seed=821)
    tg._check_attention([1 + s % 3 * 20 for s in range(n)], [61 + (s * 131) % 90 for s in range(n)], 1, 1, 64, 32, seed=822)


def test_norms_of_four_million_rows():
    """More work-groups than a launch takes along x, and elements past 2^31: every row against torch's fp32, half a bf16 step and 2^-18 of the row's largest value."""
    M, d = (1 << 22) + 9, 520
    r = torch.randn((M, d), generator=torch.Generator(device=tg.DEV).manual_seed(3), device=tg.DEV, dtype=torch.bfloat16)
    out = torch.empty_like(r)
    mq.moqe_residual_norm(None, r, out, pre=mq.Norm("rms", 1e-5))
    for lo in range(0, M, 1 << 19):
        x = r[lo:lo + (1 << 19)].float()
        want = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        assert ((out[lo:lo + (1 << 19)].float() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True)).all()


def test_rows_past_two_to_the_31_elements():
    """140000 sequences of one token: the last rows of a call are those of a call of their own, and attention over one token is its value."""
    S, heads, dh, bt, few = 140000, 62, 256, 32, 500
    gen = torch.Generator(device=tg.DEV).manual_seed(4)
    qkv = torch.randn((S, (heads + 2) * dh), generator=gen, device=tg.DEV, dtype=torch.bfloat16)
    assert qkv.numel() > 2 ** 31
    rope = mq.Rope(tg.dev(100.0 ** (-2.0 * np.arange(128) / 256)), 256)
    i32 = dict(dtype=torch.int32, device=tg.DEV)

    def run(x):
        n = len(x)
        cache = mq.KvCache.empty(n, 1, bt, dh, tg.DEV)
        batch = mq.KvBatch(torch.arange(n, **i32).view(n, 1), torch.ones(n, **i32), n, 1, n)
        q, out = (torch.empty((n, heads * dh), dtype=torch.bfloat16, device=tg.DEV) for _ in range(2))
        mq.moqe_kv_append(x, heads, rope, batch, cache, q)
        mq.moqe_kv_attention(q, mq.Attention(heads, 1 / 16), batch, cache, out)
        tg.sync()
        return q, out, cache
    q, out, cache = run(qkv)
    q2, out2, cache2 = run(qkv[-few:])
    assert torch.equal(q[-few:], q2) and torch.equal(out[-few:], out2) and torch.equal(cache.v_scale[-few:], cache2.v_scale)
    at = torch.from_numpy(do.value_at(np.zeros(dh, dtype=np.int64), np.arange(dh), dh)).to(tg.DEV)
    v = cache.v[-few:, 0][:, at].view(torch.float8_e4m3fn).float() * cache.v_scale[-few:]
    assert torch.equal(out2.view(few, heads, dh).float(), v[:, None].expand(few, heads, dh))
