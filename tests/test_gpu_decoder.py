"""The decoder layer's operators on the GPU against the 64-bit oracle, at the sizes and masks where they can go wrong.

Tolerances, from the roundings of each path (half a step: bf16 2^-8 of a value, fp32 2^-24, e4m3 2^-4 or half the smallest step):
  norms      fp32 sums of d terms: 2^-18 of the row's largest value covers d <= 32768 in their order; bf16 results half a step more
  queries    bf16: half a step, plus 2^-19 of the pair's length for the angle (2^-24 of a turn) and the fp32 products
  codes      bit-equal where the value is exact in fp32 (values; keys without rotation); else the code of a neighbour within 2^-19
  attention  out half a bf16 step; weights half a bf16 step each: 2^-8 of sum w |v|; scores in fp32: 2^-12 of it
"""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from paper_2508_09204_amd import binding as mq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def f64(t):
    return t.detach().double().cpu().numpy()


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def sync():
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------------------------ norms
def _norm_case(M, d, y_t, r_t, post, pre, gate, seed=0, pad=0, lead=0):
    """Rows with `pad` spare elements between them and `lead` before the first."""
    rng = np.random.default_rng(seed + M * 7 + d)
    def rows(t):
        buf = torch.zeros(lead + M * (d + pad), dtype=t, device=DEV)
        v = buf[lead:].view(M, d + pad)[:, :d]
        v.copy_(dev(rng.normal(size=(M, d)) + 0.5))
        return v
    y, r = rows(y_t) if y_t else None, rows(r_t)
    out, res = rows(BF), rows(r_t)
    gate_rows = 3 if gate == "sample" else 0
    g = None if not gate else dev(rng.normal(size=(-(-M // 3), d) if gate == "sample" else d).astype(np.float32))
    vec = lambda on: dev(rng.normal(size=d).astype(np.float32)) if on else None
    norms = {n: None if not k else mq.Norm(k, 1e-5, vec(n == "pre" or k == "rms"), vec(k == "layer")) for n, k in (("post", post), ("pre", pre))}
    args = {n: None if v is None else (v.kind, 1e-5, None if v.gain is None else f64(v.gain), None if v.offset is None else f64(v.offset))
            for n, v in norms.items()}
    want_t, want_o = do.residual_norm(None if y is None else f64(y), f64(r), None if g is None else f64(g), gate_rows, 0.75, args["post"], args["pre"])
    mq.moqe_residual_norm(y, r, out, res, g, gate_rows, 0.75, norms["post"], norms["pre"])
    sync()
    for got, want, t in ((res, want_t, r_t), (out, want_o, BF)):
        tol = 2.0 ** -18 * np.abs(want).max(1, keepdims=True) + (2.0 ** -8 * np.abs(want) if t == BF else 0.0)
        assert (np.abs(f64(got) - want) <= tol).all()
    return y, r, out, res


F32 = torch.float32


@pytest.mark.parametrize("M,d", [(1, 1), (1, 64), (3, 7), (5, 8), (4, 255), (2, 2047), (2, 2048), (9, 2056), (3, 4096), (2, 5003), (2, 8192), (2, 8200),
                                 (1, 16384), (2, 32760), (1, 32767), (1, 32768), (130, 96)])
@pytest.mark.parametrize("pre", ["rms", "layer"])
def test_norm_sizes(M, d, pre):
    _norm_case(M, d, F32, BF, "", pre, "")
    _norm_case(M, d, BF, F32, "layer" if pre == "rms" else "rms", pre, "sample")


@pytest.mark.parametrize("y_t,r_t", [(F32, F32), (F32, BF), (BF, F32), (BF, BF), (None, F32)])
@pytest.mark.parametrize("post,gate", [("", ""), ("rms", "all"), ("layer", "sample")])
def test_norm_types(y_t, r_t, post, gate):
    _norm_case(7, 200, y_t, r_t, post, "", gate)
    _norm_case(7, 200, y_t, r_t, post, "rms", gate)


@pytest.mark.parametrize("pad,lead", [(8, 0), (1, 0), (5, 3), (0, 1), (0, 2)])
def test_norm_strides_and_alignment(pad, lead):
    for d in (64, 100, 5000):
        _norm_case(6, d, BF, F32, "rms", "layer", "all", pad=pad, lead=lead)


def test_norm_in_place_and_single_outputs():
    rng = np.random.default_rng(5)
    y, r = dev(rng.normal(size=(9, 520)), F32), dev(rng.normal(size=(9, 520)), BF)
    out, res = torch.empty((9, 520), dtype=BF, device=DEV), torch.empty_like(r)
    norm = mq.Norm("rms", 1e-6, torch.ones(520, device=DEV))
    mq.moqe_residual_norm(y, r, out, res, pre=norm)
    only, same = torch.empty_like(out), r.clone()
    mq.moqe_residual_norm(y, r, only, None, pre=norm)
    mq.moqe_residual_norm(y, same, None, same)
    sync()
    assert torch.equal(only, out) and torch.equal(same, res)


def test_norm_rows_keep_apart():
    """A row of infinities or NaN spoils itself only; a row of zeros is zeros."""
    r = torch.ones((8, 300), device=DEV)
    r[2, 7], r[4, 0], r[5] = float("inf"), float("nan"), 0.0
    out = torch.empty((8, 300), dtype=BF, device=DEV)
    mq.moqe_residual_norm(None, r, out, pre=mq.Norm("rms", 1e-6))
    sync()
    fine = [0, 1, 3, 6, 7]
    assert (out[fine] == 1.0).all() and (out[5] == 0.0).all() and out[4].isnan().all() and out[2, 7].isnan() and (out[2, :7] == 0.0).all()


# ------------------------------------------------------------------------------------------------------------------ cache
def _lay_out(rng, lens, bt, spare=2, absent=()):
    """A block table in random order with -1 past every sequence's tokens; absent: (sequence, block) without a block."""
    need = [-(-n // bt) for n in lens]
    width = max(1, max(need))
    ids = rng.permutation(sum(need) + spare)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n]
        at += n
    for s, b in absent:
        table[s, b] = -1 if (s + b) % 2 else len(ids) + 5            # below and above the range
    return table, len(ids)


def _on_device(cache):
    return mq.KvCache(dev(cache.k), dev(cache.v), dev(cache.k_scale, F32), dev(cache.v_scale, F32), cache.bt, cache.dh)


def _batch(table, lens, rows, uniform=False):
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    S, T, M = len(rows), max(1, max(rows)), int(cu[-1])
    b = mq.KvBatch(dev(table), dev(np.array(lens, dtype=np.int32)), S, T, M, None if uniform else dev(cu))
    return b, do.sequences(S, T, M, lens, table.shape[1], 1 << 30, None if uniform else cu), T


APPEND = [  # rows, tokens with them, heads, key heads, dims, block, type, rot, interleaved, norms
    dict(rows=[1], lens=[1], heads=1, kv=1, dh=64, bt=32, t=BF, rot=64, inter=False, norm=False),
    dict(rows=[1, 1, 1, 1], lens=[1, 32, 33, 200], heads=7, kv=1, dh=128, bt=32, t=BF, rot=128, inter=False, norm=False),
    dict(rows=[5, 0, 31, 33, 64, 100], lens=[5, 40, 31, 90, 128, 177], heads=6, kv=2, dh=64, bt=64, t=F32, rot=32, inter=True, norm=True),
    dict(rows=[130, 3], lens=[300, 2], heads=4, kv=4, dh=128, bt=128, t=BF, rot=64, inter=False, norm=True),      # more rows than tokens: positions below 0
    dict(rows=[2, 70], lens=[129, 70], heads=3, kv=3, dh=256, bt=128, t=F32, rot=240, inter=False, norm=False),
    dict(rows=[40, 40], lens=[40, 100], heads=8, kv=2, dh=256, bt=32, t=BF, rot=16, inter=True, norm=False),
    dict(rows=[129], lens=[1000], heads=2, kv=1, dh=64, bt=128, t=F32, rot=0, inter=False, norm=False),
    dict(rows=[256], lens=[256], heads=2, kv=2, dh=256, bt=128, t=BF, rot=256, inter=False, norm=False),
]


def _append_args(c, rng, M):
    qkv = rng.normal(size=(M, (c["heads"] + 2 * c["kv"]) * c["dh"])) * np.exp(rng.normal(size=(M, 1)))
    x = dev(qkv, c["t"])
    f = 10000.0 ** (-2.0 * np.arange(c["rot"] // 2) / max(1, c["rot"]))
    gains = [rng.normal(size=c["dh"]).astype(np.float32) if c["norm"] else None for _ in range(2)]
    rope = mq.Rope(dev(f) if c["rot"] else None, c["rot"], c["inter"], 1.125, *(None if g is None else dev(g) for g in gains), eps=1e-6)
    return x, f, gains, rope


def _check_append(c, seed, absent=(), uniform=False, grow=True):
    rng = np.random.default_rng(seed)
    rows, lens, H, dh, bt = c["rows"], c["lens"], c["kv"], c["dh"], c["bt"]
    table, n_blocks = _lay_out(rng, lens, bt, absent=absent)
    cache = do.Cache(n_blocks, H, bt, dh)
    for which in ("k", "v"):                                         # earlier tokens: any codes (NaN among them), small scales so that some grow
        cache.codes(which)[:] = rng.integers(0, 256, cache.codes(which).shape)
        cache.scales(which)[:] = 2.0 ** rng.integers(-12, -4 if grow else -8, (n_blocks, H))
    d = _on_device(cache)
    batch, seqs, T = _batch(table, lens, rows, uniform)
    x, f, gains, rope = _append_args(c, rng, batch.M)
    q = torch.full((batch.M, c["heads"] * dh), 7.0, dtype=BF, device=DEV)
    mq.moqe_kv_append(x, c["heads"], rope, batch, d, q)
    sync()
    before = {w: cache.codes(w).copy() for w in ("k", "v")}
    want = do.kv_append(f64(x), c["heads"], cache, table, seqs, T, f, c["rot"], c["inter"], 1.125, *gains, 1e-6)
    want = want.reshape(batch.M, -1)
    got = f64(q)
    done = ~np.isnan(want)
    heads = f64(x)[:, :c["heads"] * dh].reshape(batch.M, c["heads"], dh)
    size = np.abs(heads).max(-1, keepdims=True) if not c["norm"] else np.full((batch.M, c["heads"], 1), np.abs(gains[0]).max() * dh ** 0.5)
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * 2.5 * np.broadcast_to(size, heads.shape).reshape(batch.M, -1)
    assert (np.abs(got - want)[done] <= tol[done]).all() and (got[~done] == 7.0).all()
    exact = {"v": True, "k": c["rot"] == 0 and not c["norm"]}
    for which, dt, ds in (("k", d.k, d.k_scale), ("v", d.v, d.v_scale)):
        g, w = dt.cpu().numpy(), cache.codes(which)
        assert np.array_equal(f64(ds), cache.scales(which))
        gv, wv = do.e4m3_value(g), do.e4m3_value(w)
        same = (g == w) | (np.isnan(gv) & np.isnan(wv)) | ((gv == 0) & (wv == 0))
        if exact[which]:
            assert same.all()
        else:
            assert (np.abs(g.astype(int) - w.astype(int))[~same] == 1).all() and (~same).mean() < 1e-3
        untouched = before[which] == w
        assert (same[untouched]).all()


@pytest.mark.parametrize("i", range(len(APPEND)))
def test_append(i):
    _check_append(APPEND[i], seed=10 + i)


def test_append_absent_blocks_are_left_out():
    c = dict(APPEND[2], rows=[50, 20, 90], lens=[100, 80, 190])
    _check_append(c, seed=40, absent=[(0, 1), (1, 1), (2, 2)])


def test_append_uniform_rows():
    _check_append(dict(APPEND[3], rows=[33, 33, 33], lens=[33, 70, 500]), seed=41, uniform=True)


def test_append_far_positions_keep_their_angles():
    """Positions near 2^20: angles of up to a million radians, which 32 bits would know to some hundredths."""
    bt, lens, rows = 64, [1 << 20, 999999], [3, 1]
    table = np.full((2, (1 << 20) // bt), -1, dtype=np.int32)
    cache = do.Cache(4, 1, bt, 64)
    table[0, (1 << 20) // bt - 1], table[1, 999998 // bt] = 2, 0
    batch, seqs, T = _batch(table, lens, rows)
    c = dict(APPEND[0], heads=2, rot=64, t=F32)
    x, f, _, rope = _append_args(c, np.random.default_rng(3), batch.M)
    d, q = _on_device(cache), torch.empty((4, 128), dtype=BF, device=DEV)
    mq.moqe_kv_append(x, 2, rope, batch, d, q)
    sync()
    want = do.kv_append(f64(x), 2, cache, table, seqs, T, f, 64, False, 1.125).reshape(4, -1)
    size = np.abs(f64(x)).max()
    assert (np.abs(f64(q) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * 2.5 * size).all()
    assert np.array_equal(f64(d.k_scale), cache.k_scale)


@pytest.mark.parametrize("dh,bt", [(64, 32), (128, 64), (256, 128)])
def test_append_token_by_token_is_append_at_once(dh, bt):
    """Values grow, so that scales do: the codes of power-of-two scales end up the same, but for those that pass through subnormals."""
    rng = np.random.default_rng(8)
    L, H, Hq = bt + 9, 2, 4
    x = dev(rng.normal(size=(L, (Hq + 2 * H) * dh)) * 1.5 ** (np.arange(L) % 13)[:, None], F32)
    rope = mq.Rope(dev(1000.0 ** (-2.0 * np.arange(16) / 32)), 32)
    table = dev(np.array([[1, 3]], dtype=np.int32))
    many, once = (mq.KvCache.empty(4, H, bt, dh, DEV) for _ in range(2))
    for c in (many, once):
        c.k.zero_(), c.v.zero_()
    q1, q2 = (torch.empty((L, Hq * dh), dtype=BF, device=DEV) for _ in range(2))
    length = torch.zeros(1, dtype=torch.int32, device=DEV)
    for p in range(L):
        length.fill_(p + 1)
        mq.moqe_kv_append(x[p:p + 1], Hq, rope, mq.KvBatch(table, length, 1, 1, 1), many, q1[p:p + 1])
    mq.moqe_kv_append(x, Hq, rope, mq.KvBatch(table, length, 1, L, L), once, q2)
    sync()
    assert torch.equal(q1, q2)
    for a, b, sa, sb in ((many.k, once.k, many.k_scale, once.k_scale), (many.v, once.v, many.v_scale, once.v_scale)):
        assert torch.equal(sa[[1, 3]], sb[[1, 3]])
        va, vb = do.e4m3_value(a[[1, 3]].cpu().numpy()), do.e4m3_value(b[[1, 3]].cpu().numpy())
        assert (np.abs(va - vb) <= 2.0 ** -9).all() and (va[np.abs(vb) >= 2.0 ** -5] == vb[np.abs(vb) >= 2.0 ** -5]).all()


def test_append_infinities_and_nan():
    dh, bt = 64, 32
    x = torch.ones((3, 3 * dh), device=DEV)
    x[1, dh + 5], x[1, 2 * dh + 6], x[2, 2 * dh + 7] = float("nan"), float("inf"), float("-inf")
    cache = mq.KvCache.empty(1, 1, bt, dh, DEV)
    q = torch.empty((3, dh), dtype=BF, device=DEV)
    mq.moqe_kv_append(x, 1, mq.Rope(None, 0), mq.KvBatch(torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.full((1,), 3, dtype=torch.int32, device=DEV), 1, 3, 3), cache, q)
    sync()
    t, d = np.meshgrid(np.arange(3), np.arange(dh), indexing="ij")
    k = do.e4m3_value(cache.k[0, 0].cpu().numpy()[do.key_at(t, d, dh)]) * float(cache.k_scale[0, 0])
    v = do.e4m3_value(cache.v[0, 0].cpu().numpy()[do.value_at(t, d, dh)]) * float(cache.v_scale[0, 0])
    assert np.isnan(k[1, 5]) and np.nansum(k) == 3 * dh - 1 and float(cache.v_scale[0, 0]) == 2.0 ** -8
    assert v[1, 6] == 448 / 256 and v[2, 7] == -448 / 256 and (np.delete(v.ravel(), [dh + 6, 2 * dh + 7]) == 1.0).all()


# -------------------------------------------------------------------------------------------------------------- attention
def _random_cache(rng, n_blocks, H, bt, dh):
    cache = do.Cache(n_blocks, H, bt, dh)
    for which in ("k", "v"):
        cache.codes(which)[:] = do.e4m3_code(rng.normal(size=cache.codes(which).shape) * 60)
        cache.scales(which)[:] = 2.0 ** rng.integers(-8, -4, (n_blocks, H))
    return cache


def _poison(cache, table, lens):
    """NaN codes past every sequence's tokens, NaN scales and codes in blocks that nobody has."""
    for s, n in enumerate(lens):
        b = n // cache.bt
        if n % cache.bt and 0 <= table[s, b] < cache.n_blocks:
            for which in ("k", "v"):
                for h in range(cache.n_heads):
                    cache.codes(which)[table[s, b], h][cache.at[which][n % cache.bt:]] = 0xff if h % 2 else 0x7f
    free = np.setdiff1d(np.arange(cache.n_blocks), table)
    for which in ("k", "v"):
        cache.codes(which)[free] = 0x7f
        cache.scales(which)[free] = np.nan


def _attention_tol(want, size):
    return 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * size


def _check_attention(rows, lens, heads, kv, dh, bt, cap=0.0, window=0, slopes=False, prefix=None, seed=0, absent=(), uniform=False, pad=0, q_by=1.0):
    rng = np.random.default_rng(seed)
    table, n_blocks = _lay_out(rng, lens, bt, absent=absent)
    cache = _random_cache(rng, n_blocks, kv, bt, dh)
    _poison(cache, table, lens)
    batch, seqs, T = _batch(table, lens, rows, uniform)
    M = batch.M
    q = torch.zeros((M, heads * dh + pad), dtype=BF, device=DEV)[:, :heads * dh]
    q.copy_(dev(rng.normal(size=(M, heads * dh)) * q_by))
    out = torch.full((M, heads * dh + pad), 7.0, dtype=BF, device=DEV)
    sl = 2.0 ** -(1 + np.arange(heads) % 7.0) if slopes else None
    pre = None if prefix is None else np.array(prefix, dtype=np.int32)
    scale = dh ** -0.5
    attn = mq.Attention(heads, scale, cap, window, None if sl is None else dev(sl, F32), None if pre is None else dev(pre))
    mq.moqe_kv_attention(q, attn, batch, _on_device(cache), out[:, :heads * dh])
    sync()
    want, size = do.kv_attention(f64(q), heads, cache, table, seqs, T, scale, cap, window, sl, pre)
    want, size, got = want.reshape(M, -1), size.reshape(M, -1), f64(out)
    done = ~np.isnan(want)
    bad = np.abs(got[:, :heads * dh] - want) > _attention_tol(want, size)
    assert not bad[done].any(), (np.argwhere(bad & done)[:5], np.abs(got[:, :heads * dh] - want)[done].max())
    assert np.isfinite(got[:, :heads * dh][done]).all() and (got[:, heads * dh:] == 7.0).all()
    return got


FEW = [  # rows, tokens, heads, key heads, dims, block
    ([1], [1], 1, 1, 64, 32), ([1], [31], 8, 8, 64, 32), ([1], [32], 7, 1, 128, 64), ([1], [33], 4, 2, 256, 128), ([1], [256], 8, 1, 128, 32),
    ([1], [257], 16, 1, 128, 32), ([1], [3000], 3, 1, 128, 64), ([1], [9001], 2, 2, 64, 128), ([1, 1, 1, 1, 1], [1, 700, 0, 64, 2001], 14, 2, 128, 64),
    ([2, 1, 3, 0], [2, 900, 1, 50], 8, 2, 128, 32), ([4, 4], [500, 4], 28, 4, 128, 64), ([5], [777], 12, 1, 128, 64), ([8], [600], 8, 1, 64, 32),
    ([4], [300], 8, 1, 256, 64), ([16], [400], 4, 1, 128, 64), ([64], [64], 1, 1, 64, 64),
]


@pytest.mark.parametrize("i", range(len(FEW)))
def test_attention_few_rows(i):
    _check_attention(*FEW[i], seed=100 + i)


MANY = [
    ([65], [65], 1, 1, 64, 32), ([17], [17], 4, 1, 128, 64), ([129], [129], 1, 1, 128, 64), ([70, 1, 33], [70, 400, 500], 7, 1, 128, 64),
    ([128], [1000], 2, 2, 64, 128), ([40], [90], 4, 2, 256, 128), ([100, 0, 31], [50, 7, 300], 6, 2, 64, 32), ([33], [1], 2, 1, 256, 32),
    ([200], [201], 3, 1, 128, 32),
]


@pytest.mark.parametrize("i", range(len(MANY)))
def test_attention_many_rows(i):
    _check_attention(*MANY[i], seed=200 + i)


MASKS = [
    dict(window=1), dict(window=17), dict(window=64), dict(window=1000), dict(prefix=[0, 40, 500]), dict(prefix=[-3, 1, 33], window=20),
    dict(cap=5.0), dict(slopes=True), dict(cap=20.0, slopes=True, window=50, prefix=[5, 64, 100]), dict(window=40, prefix=[90, 90, 90], q_by=8.0),
]


@pytest.mark.parametrize("i", range(len(MASKS)))
@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 2, 4], [40, 70, 33]])
def test_attention_masks(i, rows):
    _check_attention(rows, [90, 333, 150], 8, 2, 64 if i % 2 else 128, 32, seed=300 + i, **MASKS[i])


LONG = [  # contexts so long that the tokens of a column tile are divided over work-groups
    dict(rows=[70], lens=[3000], heads=2, kv=1, dh=128, bt=64), dict(rows=[100, 30], lens=[2500, 6000], heads=4, kv=2, dh=64, bt=32),
    dict(rows=[17, 0, 90], lens=[5000, 100, 95], heads=8, kv=2, dh=256, bt=128), dict(rows=[100, 70], lens=[4000, 1500], heads=3, kv=1, dh=128, bt=64, window=700, prefix=[90, 1200]),
    dict(rows=[66], lens=[2100], heads=2, kv=2, dh=64, bt=64, cap=9.0, slopes=True), dict(rows=[80, 80], lens=[3000, 1100], heads=2, kv=1, dh=128, bt=128, absent=[(0, 3), (0, 23), (1, 8)]),
    dict(rows=[130], lens=[2049], heads=5, kv=1, dh=128, bt=32, window=3),
]


@pytest.mark.parametrize("i", range(len(LONG)))
def test_attention_many_rows_on_long_contexts(i):
    _check_attention(seed=700 + i, **LONG[i])


@pytest.mark.parametrize("rows", [[1, 1, 1], [80, 80, 80]])
def test_attention_absent_blocks(rows):
    """Blocks given back are not seen; a sequence that has none gives zeros, also where the window leaves it only absent ones."""
    got = _check_attention(rows, [200, 100, 300], 4, 2, 128, 64, seed=400, absent=[(0, 0), (0, 2), (1, 0), (1, 1), (2, 4)])
    assert (got[rows[0]:rows[0] + rows[1]] == 0.0).all()
    _check_attention(rows, [200, 100, 300], 4, 2, 128, 64, seed=401, window=20, absent=[(0, 3), (0, 2), (1, 1), (2, 4), (2, 3)])


@pytest.mark.parametrize("rows", [1, 70])
def test_attention_strides_and_uniform_rows(rows):
    _check_attention([rows] * 3, [rows + 5, rows, rows + 200], 4, 2, 64, 64, seed=500, uniform=True, pad=24)


@pytest.mark.parametrize("rows", [1, 90])
def test_attention_of_many_sequences(rows):
    """More sequences than a wave has lanes, of all lengths."""
    n = 70
    _check_attention([1 + (s * 7) % rows for s in range(n)], [1 + (s * 37) % 400 + rows for s in range(n)], 2, 1, 64, 32, seed=600)


@pytest.mark.parametrize("rows,window,L", [([1], 100, 180), ([4], 0, 180), ([90], 0, 180), ([90], 30, 180), ([90], 0, 2100), ([3], 0, 2100)])
def test_nan_in_the_cache_reaches_those_who_see_it(rows, window, L):
    """The 30th token from the end is NaN in one dim of its values, the 80th in one of its keys: only rows that see them have NaN, in the dims concerned."""
    rng = np.random.default_rng(9)
    dh, bt, H = 64, 32, 2
    lens = [L if rows[0] > 1 else L - 30]
    for bad_key in (False, True):
        table, n_blocks = _lay_out(rng, [L], bt)
        cache = _random_cache(rng, n_blocks, H, bt, dh)
        tok, dim = (L - 80, 3) if bad_key else (L - 30, 40)
        which = "k" if bad_key else "v"
        cache.codes(which)[table[0, tok // bt], 1][cache.at[which][tok % bt, dim]] = 0x7f
        batch, seqs, T = _batch(table, lens, rows)
        q = dev(rng.normal(size=(batch.M, 4 * dh)), BF)
        out = torch.empty_like(q)
        mq.moqe_kv_attention(q, mq.Attention(4, 0.125, window=window), batch, _on_device(cache), out)
        sync()
        clean = do.Cache(n_blocks, H, bt, dh)
        clean.k, clean.v, clean.k_scale, clean.v_scale = cache.k.copy(), cache.v.copy(), cache.k_scale, cache.v_scale
        clean.codes(which)[table[0, tok // bt], 1][cache.at[which][tok % bt, dim]] = 0
        want, size = do.kv_attention(f64(q), 4, clean, table, seqs, T, 0.125, 0.0, window)
        got = f64(out).reshape(batch.M, 4, dh)
        p = np.arange(lens[0] - rows[0], lens[0])
        sees = (tok <= p) & ((p - tok < window) if window else True)
        hit = np.zeros(got.shape, bool)
        hit[np.ix_(sees, [2, 3], np.arange(dh) if bad_key else [dim])] = True
        assert np.isnan(got[hit]).all()
        assert (np.abs(got - want) <= _attention_tol(want, size))[~hit].all()


def test_attention_of_blocks_past_4_gib():
    """The same tokens in blocks at the start of a cache and in blocks whose bytes lie past 2^32: the same results, bit for bit."""
    H, bt, dh, n_blocks = 8, 128, 256, 17000                              # 256 KiB a block: 4.4 GB of keys, as many of values
    c = mq.KvCache.empty(n_blocks, H, bt, dh, DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    rows = 150
    qkv = torch.randn((rows, (16 + 2 * H) * dh), generator=gen, device=DEV, dtype=BF)
    rope = mq.Rope(dev(100.0 ** (-2.0 * np.arange(128) / 256)), 256)
    outs = []
    for ids in ((0, 1), (n_blocks - 2, n_blocks - 1)):
        table, length = torch.tensor([ids], dtype=torch.int32, device=DEV), torch.tensor([rows], dtype=torch.int32, device=DEV)
        q = torch.empty((rows, 16 * dh), dtype=BF, device=DEV)
        batch = mq.KvBatch(table, length, 1, rows, rows)
        mq.moqe_kv_append(qkv, 16, rope, batch, c, q)
        many, few = torch.empty_like(q), torch.empty_like(q[-1:])
        mq.moqe_kv_attention(q, mq.Attention(16, 1 / 16), batch, c, many)
        mq.moqe_kv_attention(q[-1:], mq.Attention(16, 1 / 16), mq.KvBatch(table, length, 1, 1, 1), c, few)
        sync()
        outs.append((q, many, few))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert (outs[0][1][-1].double() - outs[0][2][0].double()).abs().max() < 2.0 ** -6 * outs[0][1][-1].double().abs().max()


def test_values_on_the_device_are_taken_into_their_ranges():
    """Lengths, rows and blocks outside what the buffers hold: nothing outside is read, rows of other sequences stay right."""
    rng = np.random.default_rng(12)
    dh, bt, H = 64, 32, 1
    cache = _random_cache(rng, 6, H, bt, dh)
    table = np.array([[0, 1], [2, 3], [4, 99]], dtype=np.int32)
    for rows, T in (([1, 1, 1], 1), ([40, 40, 40], 40)):
        M = sum(rows)
        q = dev(rng.normal(size=(M, 2 * dh)), BF)
        cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        for lens, cu2 in (([64, 1 << 20, -7], cu), ([64, 60, 50], np.array([0, rows[0], 5 * M, -3], dtype=np.int32))):
            batch = mq.KvBatch(dev(table), dev(np.array(lens, dtype=np.int32)), 3, T, M, dev(cu2))
            seqs = do.sequences(3, T, M, lens, 2, bt, cu2)
            out = torch.full_like(q, 7.0)
            mq.moqe_kv_attention(q, mq.Attention(2, 0.125), batch, _on_device(cache), out)
            sync()
            want, size = do.kv_attention(f64(q), 2, cache, table, seqs, T, 0.125)
            want, size = want.reshape(M, -1), size.reshape(M, -1)
            done = ~np.isnan(want)
            assert (np.abs(f64(out) - want) <= _attention_tol(want, size))[done].all() and (f64(out)[~done] == 7.0).all()


@pytest.mark.parametrize("rows", [1, 80])
def test_other_streams_and_graphs(rows):
    """The whole step on a stream of its own, then as a graph replayed with lengths that grow on the device."""
    rng = np.random.default_rng(20)
    S, H, Hq, dh, bt, L0 = 3, 2, 8, 64, 32, 300
    table = dev(np.arange(S * 40, dtype=np.int32).reshape(S, 40))
    length = torch.full((S,), L0 + rows, dtype=torch.int32, device=DEV)
    cache = _on_device(_random_cache(rng, S * 40, H, bt, dh))
    start = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    batch = mq.KvBatch(table, length, S, rows, S * rows)
    res, y = dev(rng.normal(size=(S * rows, 128)), F32), dev(rng.normal(size=(S * rows, 128)), F32)
    qkv = dev(rng.normal(size=(S * rows, (Hq + 2 * H) * dh)), BF)
    q, out = (torch.empty((S * rows, Hq * dh), dtype=BF, device=DEV) for _ in range(2))
    normed, kept = torch.empty((S * rows, 128), dtype=BF, device=DEV), torch.empty_like(res)
    calls = [mq.ResidualNormCall(y, res, normed, kept, pre=mq.Norm("rms", 1e-6)),
             mq.KvAppendCall(qkv, Hq, mq.Rope(dev(100.0 ** (-np.arange(32) / 32.0)), 64), batch, cache, q),
             mq.KvAttentionCall(q, mq.Attention(Hq, 0.125), batch, cache, out)]

    def reset():
        for t, s in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), start):
            t.copy_(s)
        length.fill_(L0 + rows)

    def steps(n, once):
        got = []
        for _ in range(n):
            once()
            sync()
            got.append((out.clone(), q.clone(), normed.clone()))
            length.add_(rows)
            sync()
        return got

    def eager():
        for c in calls:
            c()

    reset()
    want = steps(3, eager)
    side = torch.cuda.Stream()
    reset()
    sync()
    with torch.cuda.stream(side):
        got = steps(3, eager)
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eager()
    reset()
    sync()
    replayed = steps(3, graph.replay)
    for a, b, c in zip(want, got, replayed):
        assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(a, b, c))


def test_append_turns_infinities():
    """An infinite key value makes its pair infinite, hence the largest codes; NaN makes its pair NaN; the others are the oracle's codes."""
    dh, bt, rows = 64, 32, 5
    rng = np.random.default_rng(31)
    host = rng.normal(size=(rows, 3 * dh))
    host[1, dh + 5], host[2, dh + 40], host[3, dh + 7], host[4, dh + 33] = np.inf, -np.inf, np.nan, np.inf
    x = dev(host, F32)
    for inter in (False, True):
        for t in (F32, BF):
            f = 100.0 ** (-2.0 * np.arange(32) / 64)
            cache, batch = do.Cache(1, 1, bt, dh), mq.KvBatch(dev(np.zeros((1, 1), np.int32)), dev(np.array([rows], np.int32)), 1, rows, rows)
            d, q = _on_device(cache), torch.empty((rows, dh), dtype=BF, device=DEV)
            mq.moqe_kv_append(x.to(t), 1, mq.Rope(dev(f), 64, inter), batch, d, q)
            sync()
            with np.errstate(invalid="ignore"):
                do.kv_append(f64(x.to(t)), 1, cache, np.zeros((1, 1), int), do.sequences(1, rows, rows, [rows], 1, bt), rows, f, 64, inter)
            at = cache.at["k"][:rows]
            got, want = do.e4m3_value(d.k.cpu().numpy()[0, 0][at]), do.e4m3_value(cache.k[0, 0][at])
            assert float(d.k_scale[0, 0]) == cache.k_scale[0, 0]
            assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).sum() == 2 and (np.abs(want) == 448).sum() >= 6
            assert (got == want)[~np.isnan(want)].mean() > 0.98 and np.array_equal(np.abs(got) == 448, np.abs(want) == 448)


def test_attention_of_many_sequences_in_chunks():
    """More sequences than a wave has lanes, of 1 to 40 chunks, some without rows and one without tokens."""
    n = 70
    lens = [1 + (s * 977) % 2600 for s in range(n)]
    lens[5], lens[66] = 0, 41000
    _check_attention([0 if s % 9 == 4 else 1 for s in range(n)], lens, 2, 1, 64, 32, seed=610)


@pytest.mark.parametrize("rows,lens,heads,kv,dh,bt,masks", [
    ([8, 3], [3000, 3], 4, 1, 128, 64, {}), ([5], [5000], 6, 1, 64, 128, dict(window=2100, prefix=[700])), ([4, 1, 2], [2500, 1100, 40], 4, 1, 256, 32, dict(cap=8.0)),
    ([8, 8], [2049, 1056], 4, 1, 128, 32, dict(slopes=True)), ([32], [4100], 1, 1, 128, 64, dict(absent=[(0, 0), (0, 30), (0, 64)])),
    ([33], [4100], 1, 1, 128, 64, {}), ([17], [1500], 1, 1, 256, 64, {}),
])
def test_attention_few_rows_in_chunks(rows, lens, heads, kv, dh, bt, masks):
    """Up to 32 columns (16 where heads are 256 wide), and one more, on contexts that are cut into chunks."""
    _check_attention(rows, lens, heads, kv, dh, bt, seed=620, **masks)
