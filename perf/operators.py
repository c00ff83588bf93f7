"""Performance cases of the operators that surround the routed MLP in a decoder layer.

`listed()` names the cases, `draw(rng)` gives further ones of the same ranges, `prepare` builds what a serving program holds before
the call, `run` makes one call, `work` states the bytes and operations the call cannot do without, `exact` is the same call in
64-bit arithmetic.  With `own` false `run` computes the operators from elementary torch operations in 32 bits.

Kinds of calls:
  norm    moqe_residual_norm: r' = r + scale * gate * post(y), out = pre(r')
  append  moqe_kv_append: rotary positions (and norms) of the heads of a fused projection, keys and values into the 8-bit paged cache
  attend  moqe_kv_attention: attention of new rows over that cache

The cache holds e4m3 codes with a power-of-two scale for each block of tokens and head.  Codes of one block and head:
  keys    [tokens / 16][dims / 64][64 lanes][16]  lane 16 kq + r, byte 8 st + i: token r, dim 32 st + 8 kq + i
  values  [tokens / 32][dims / 32][64 lanes][16]  lane 16 kq + r, byte 8 dt + i: dim 16 dt + r, token 4 kq + i (i < 4) or 12 + 4 kq + i
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
GOLDEN = 0.6180339887498949


def listed():
    return [
        # ---- norms around a block
        # decode of 64 requests at width 4096: the MLP's fp32 rows onto a bf16 residual, normed for the next projection
        dict(name="norm_decode", kind="norm", M=64, d=4096, y="fp32", res="bf16", post="", pre="rms", gate="", gate_rows=0, scale=1.0),
        # prefill of 128 sequences of 256 tokens at width 3584, norms before and after the block, a learned gate for each feature
        dict(name="norm_prefill", kind="norm", M=32768, d=3584, y="bf16", res="fp32", post="rms", pre="rms", gate="all", gate_rows=0,
             scale=0.5),
        # an odd width in layer norms with a gate vector for each sample: nothing is aligned, rows do not fill a wave
        dict(name="norm_odd", kind="norm", M=1500, d=1003, y="fp32", res="fp32", post="layer", pre="layer", gate="sample",
             gate_rows=196, scale=1.0),
        # ---- positions and cache
        # a decode step of 64 requests, 28 query heads on 4 key heads: one token each, mostly in the middle of a block
        dict(name="append_decode", kind="append", S=64, rows_lo=1, rows_hi=1, past_lo=0, past_hi=8000, heads=28, kv=4, dh=128, bt=64,
             qkv="bf16", rot=128, inter=False, norm=False, theta=1e4, stretch=1.0),
        # 16 fresh prompts of 512 tokens, 32 heads of their own keys (width 4096)
        dict(name="append_prefill", kind="append", S=16, rows_lo=512, rows_hi=512, past_lo=0, past_hi=0, heads=32, kv=32, dh=128, bt=64,
             qkv="bf16", rot=128, inter=False, norm=False, theta=1e4, stretch=1.0),
        # follow-ups of mixed lengths deep in long contexts: fp32 rows, neighbouring pairs of half the head, stretched positions, head norms
        dict(name="append_ragged", kind="append", S=40, rows_lo=1, rows_hi=900, past_lo=0, past_hi=100000, heads=28, kv=4, dh=128, bt=32,
             qkv="fp32", rot=64, inter=True, norm=True, theta=1e6, stretch=4.0),
        # ---- attention over the cache
        # one request being decoded: the smallest call
        dict(name="attend_one", kind="attend", S=1, rows_lo=1, rows_hi=1, past_lo=600, past_hi=600, heads=32, kv=32, dh=128, bt=64,
             cap=0.0, window=0, slopes=False, prefix=0),
        # a decode step of 64 requests whose contexts differ, 7 query heads to a key head
        dict(name="attend_decode", kind="attend", S=64, rows_lo=1, rows_hi=1, past_lo=0, past_hi=8000, heads=28, kv=4, dh=128, bt=64,
             cap=0.0, window=0, slopes=False, prefix=0),
        # two requests with long documents behind them
        dict(name="attend_long", kind="attend", S=2, rows_lo=1, rows_hi=1, past_lo=131000, past_hi=131000, heads=32, kv=8, dh=128, bt=64,
             cap=0.0, window=0, slopes=False, prefix=0),
        # 16 fresh prompts of 512 tokens
        dict(name="attend_prefill", kind="attend", S=16, rows_lo=512, rows_hi=512, past_lo=0, past_hi=0, heads=32, kv=32, dh=128, bt=64,
             cap=0.0, window=0, slopes=False, prefix=0),
        # the largest: chunks of 2048 tokens of two documents, 14336 tokens in the cache already
        dict(name="attend_chunk", kind="attend", S=2, rows_lo=2048, rows_hi=2048, past_lo=14336, past_hi=14336, heads=28, kv=4, dh=128,
             bt=64, cap=0.0, window=0, slopes=False, prefix=0),
        # prompts of mixed lengths with everything on: capped scores, a bias by distance, a window, a prefix that all rows see
        dict(name="attend_masks", kind="attend", S=24, rows_lo=1, rows_hi=700, past_lo=0, past_hi=1500, heads=16, kv=4, dh=64, bt=32,
             cap=30.0, window=500, slopes=True, prefix=100),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "append", "append", "attend", "attend", "attend"))
    if kind == "norm":
        d = _log(rng, 64, 16384)
        if rng.random() < 0.5:
            d = max(64, d // 64 * 64)
        M = _log(rng, 1, min(32768, 32768 * 3584 // d))
        gate = rng.choice(("", "all", "sample"))
        return dict(kind="norm", M=M, d=d, y=rng.choice(("fp32", "bf16")), res=rng.choice(("fp32", "bf16")),
                    post=rng.choice(("", "rms", "layer")), pre=rng.choice(("rms", "layer")), gate=gate,
                    gate_rows=rng.randint(1, 300) if gate == "sample" else 0, scale=rng.choice((1.0, 0.5, 0.25)))
    dh = rng.choice((64, 128, 128, 256))
    kv = rng.choice((1, 2, 4, 8))
    heads = kv * rng.choice((1, 3, 4, 7, 8))
    bt = rng.choice((32, 64, 128))
    if kind == "append":
        S, most = _log(rng, 1, 96), 8192 * 32 * 128
        rows_hi = _log(rng, 1, max(1, min(4096, most // (S * heads * dh))))
        return dict(kind="append", S=S, rows_lo=rng.randint(1, rows_hi), rows_hi=rows_hi, past_lo=0, past_hi=_log(rng, 1, 100000), heads=heads,
                    kv=kv, dh=dh, bt=bt, qkv=rng.choice(("bf16", "fp32")), rot=rng.choice((dh, dh, dh // 2, dh // 4)),
                    inter=rng.random() < 0.5, norm=rng.random() < 0.5, theta=rng.choice((1e4, 1e6)), stretch=rng.choice((1.0, 8.0)))
    form = rng.choice(("decode", "decode", "rows", "prompt"))
    S = _log(rng, 1, 96)
    rows_hi = 1 if form == "decode" else _log(rng, 2, 12) if form == "rows" else _log(rng, 16, 1500)
    # what the listed cases cost at most: elements of the cache, pairs of rows and tokens
    most = min(131072, 2 * 131072 * 8 * 128 // (S * kv * dh), 2 * 28 * 2048 * 15000 * 128 // (S * heads * rows_hi * dh))
    length = _log(rng, 32, max(32, most))
    rows_hi = min(rows_hi, length)
    past_hi = length - rows_hi
    return dict(kind="attend", S=S, rows_lo=rng.randint(1, rows_hi), rows_hi=rows_hi, past_lo=rng.randint(0, past_hi), past_hi=past_hi,
                heads=heads, kv=kv, dh=dh, bt=bt, cap=rng.choice((0.0, 0.0, 20.0, 50.0)), window=rng.choice((0, 0, 100, 1024)),
                slopes=rng.random() < 0.3, prefix=rng.choice((0, 0, 64)))


def _lengths(c):
    """Rows and tokens already cached of every sequence: spread over their ranges by the case alone."""
    at = [((s + 1) * GOLDEN) % 1.0 for s in range(c["S"])]
    past = [((s + 1) * GOLDEN * GOLDEN * 3) % 1.0 for s in range(c["S"])]
    rows = [c["rows_lo"] + int((c["rows_hi"] - c["rows_lo"]) * a + 0.5) for a in at]
    return rows, [c["past_lo"] + int((c["past_hi"] - c["past_lo"]) * a + 0.5) for a in past]


def _type(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


# ------------------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    st = {"case": c}
    if c["kind"] == "norm":
        M, d = c["M"], c["d"]
        wide = 1.0 + 3.0 * (torch.rand((d,), generator=g, device=DEV) < 0.01)          # a few features are larger, as in trained models
        st["y"] = (rand(M, d) * 0.5 * wide).to(_type(c["y"]))
        st["r"] = (rand(M, d) * wide + 0.1).to(_type(c["res"]))
        st["gate"] = None if not c["gate"] else 1.0 + 0.3 * rand(d) if c["gate"] == "all" else 1.0 + 0.3 * rand(-(-M // c["gate_rows"]), d)
        for n in ("post", "pre"):
            st[n + "_gain"] = 1.0 + 0.2 * rand(d) if c[n] else None
            st[n + "_offset"] = 0.1 * rand(d) if c[n] == "layer" else None
        return st
    rows, past = _lengths(c)
    S, H, dh, bt = c["S"], c["kv"], c["dh"], c["bt"]
    lens = [a + b for a, b in zip(rows, past)]
    first = [b // bt for b in past] if c["kind"] == "append" else [0] * S              # blocks that the call touches
    last = [-(-n // bt) for n in lens]
    width = max(last)
    pairs = [(s, b) for s in range(S) for b in range(first[s], last[s])]
    n_blocks = len(pairs) + 3
    perm = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(seed))[: len(pairs)]
    table = torch.full((S, width), -1, dtype=torch.int32)
    table[[s for s, _ in pairs], [b for _, b in pairs]] = perm.to(torch.int32)
    st["table"] = table.to(DEV)
    st["pairs"] = torch.tensor(pairs, dtype=torch.int64).to(DEV)
    st["kv_len"] = torch.tensor(lens, dtype=torch.int32).to(DEV)
    cu = [0]
    for n in rows:
        cu.append(cu[-1] + n)
    st["cu"] = torch.tensor(cu, dtype=torch.int32).to(DEV)
    st["M"], st["rows"], st["lens"] = cu[-1], rows, lens
    # what earlier calls left in the cache: keys with a few strong dims, values of size 1, codes by the block's largest value
    strong = 1.0 + 4.0 * (torch.rand((H, 1, dh), generator=g, device=DEV) < 0.03)
    for n in ("k", "v"):
        x = torch.randn((n_blocks, H, bt, dh), generator=g, device=DEV)
        x = x * strong if n == "k" else x
        s = torch.exp2(torch.ceil(torch.log2(x.abs().amax((2, 3)) / 448)))
        st[n] = (_to_tiles_k if n == "k" else _to_tiles_v)((x / s[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)).contiguous()
        st[n + "_scale"] = s
        del x
    if c["kind"] == "append":
        wide = 1.0 + 4.0 * (torch.rand(((c["heads"] + 2 * H) * dh,), generator=g, device=DEV) < 0.03)
        st["qkv"] = (rand(st["M"], (c["heads"] + 2 * H) * dh) * wide).to(_type(c["qkv"]))
        j = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV)
        st["inv_freq"] = c["theta"] ** (-2.0 * j / c["rot"]) / c["stretch"]
        st["gains"] = [1.0 + 0.2 * rand(dh) for _ in range(2)] if c["norm"] else [None, None]
    else:
        st["q"] = rand(st["M"], c["heads"], dh).to(torch.bfloat16)
        st["slopes"] = 2.0 ** (-8.0 * (1 + torch.arange(c["heads"], device=DEV)) / c["heads"]) if c["slopes"] else None
        st["prefix"] = torch.full((S,), c["prefix"], dtype=torch.int32, device=DEV) if c["prefix"] else None
    return st


# --------------------------------------------------------------------------------------------------------- the plain forms
def _to_tiles_k(u):
    """[blocks, heads, tokens, dims] -> the order of the keys' codes."""
    b, h, t, d = u.shape
    return u.view(b, h, t // 16, 16, d // 64, 2, 4, 8).permute(0, 1, 2, 4, 6, 3, 5, 7).reshape(b, h, t * d)


def _to_tiles_v(u):
    b, h, t, d = u.shape
    return u.view(b, h, t // 32, 2, 4, 4, d // 32, 2, 16).permute(0, 1, 2, 6, 4, 8, 7, 3, 5).reshape(b, h, t * d)


def _from_tiles_k(u, t, d):
    b, h = u.shape[:2]
    return u.view(b, h, t // 16, d // 64, 4, 16, 2, 8).permute(0, 1, 2, 5, 3, 6, 4, 7).reshape(b, h, t, d)


def _from_tiles_v(u, t, d):
    b, h = u.shape[:2]
    return u.view(b, h, t // 32, d // 32, 4, 16, 2, 2, 4).permute(0, 1, 2, 7, 4, 8, 3, 6, 5).reshape(b, h, t, d)


def _normed(x, kind, gain, offset):
    if kind == "rms":
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain + offset


def _plain_norm(st):
    c = st["case"]
    u, r = st["y"].float(), st["r"].float()
    if c["post"]:
        u = _normed(u, c["post"], st["post_gain"], st["post_offset"])
    if c["gate"]:
        u = u * (st["gate"] if c["gate"] == "all" else st["gate"].repeat_interleave(c["gate_rows"], 0)[: c["M"]])
    t = r + c["scale"] * u
    return {"residual": t.to(st["r"].dtype), "out": _normed(t, c["pre"], st["pre_gain"], st["pre_offset"]).to(torch.bfloat16)}


def _row_places(st):
    """Of every row: its sequence, its number in it, its position."""
    m = torch.arange(st["M"], device=DEV)
    seq = torch.searchsorted(st["cu"], m.to(torch.int32), right=True) - 1
    i = m - st["cu"][seq]
    return seq, i, st["kv_len"][seq] - (st["cu"][seq + 1] - st["cu"][seq]) + i


def _turned(x, c, cos, sin):
    """x [rows, heads, dims] with the pairs of its first `rot` dims turned."""
    r = c["rot"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["inter"] else (x[..., : r // 2], x[..., r // 2 : r])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if c["inter"] else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _into_cache(st, name, x, seq, pos, to, back):
    """Rows x [rows, heads, dims] into their blocks: the blocks' new scales, old codes brought to them, new codes."""
    c, bt, dh = st["case"], st["case"]["bt"], st["case"]["dh"]
    ps, pb = st["pairs"][:, 0], st["pairs"][:, 1]
    block = st["table"][ps, pb].long()
    start = torch.full_like(st["kv_len"], 1 << 30).scatter_reduce(0, seq, pos.to(torch.int32), "amin")[ps]
    token = pb[:, None] * bt + torch.arange(bt, device=DEV)
    held, live = ((token < n[:, None])[:, None, :, None] for n in (start, st["kv_len"][ps]))
    scale = st[name + "_scale"]
    old = scale[block] * (pb * bt < start)[:, None]
    place = torch.full(st["table"].shape, -1, dtype=torch.long, device=DEV).index_put((ps, pb), torch.arange(len(ps), device=DEV))
    new = torch.zeros((len(ps), bt, c["kv"], dh), device=DEV).index_put((place[seq, pos // bt], pos % bt), x).transpose(1, 2)
    codes = back(st[name][block], bt, dh)
    was = codes.view(torch.float8_e4m3fn).float() * scale[block][:, :, None, None]
    need = torch.exp2(torch.ceil(torch.log2(new.double().abs().amax((2, 3)) / 448)).clamp(-120, 120)).float()
    s = torch.maximum(need, old)
    value = (torch.where(held, was, new) / s[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    st[name][block] = to(torch.where(live, value, codes))                                      # places past the last token keep what they hold
    scale[block] = s


def _plain_append(st):
    c = st["case"]
    seq, _, pos = _row_places(st)
    x = st["qkv"].float().view(st["M"], c["heads"] + 2 * c["kv"], c["dh"])
    q, k, v = x.split((c["heads"], c["kv"], c["kv"]), 1)
    if c["norm"]:
        q, k = (_normed(a, "rms", gain, None) for a, gain in zip((q, k), st["gains"]))
    angle = (pos.double()[:, None] * st["inv_freq"])[:, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    q, k = _turned(q, c, cos, sin), _turned(k, c, cos, sin)
    _into_cache(st, "k", k, seq, pos, _to_tiles_k, _from_tiles_k)
    _into_cache(st, "v", v, seq, pos, _to_tiles_v, _from_tiles_v)
    return {"q": q.to(torch.bfloat16), **_cache_values(st)}


def _cache_values(st):
    return {"k": st["k"].view(torch.float8_e4m3fn), "v": st["v"].view(torch.float8_e4m3fn), "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _plain_attend(st):
    c = st["case"]
    S, H, G, dh, bt, T = c["S"], c["kv"], c["heads"] // c["kv"], c["dh"], c["bt"], max(st["rows"])
    table = st["table"].long()
    k, v = ((back(st[n], bt, dh).view(torch.float8_e4m3fn).float() * st[n + "_scale"][:, :, None, None])[table].transpose(1, 2).reshape(S, H, -1, dh)
            for n, back in (("k", _from_tiles_k), ("v", _from_tiles_v)))
    i = torch.arange(T, device=DEV)
    n = (st["cu"][1:] - st["cu"][:-1])[:, None]
    q = st["q"][(st["cu"][:-1, None] + i).clamp(max=st["M"] - 1).long()].float()               # [S, T, heads, dims], rows past a sequence's own unused
    a = torch.matmul(q.view(S, T, H, G, dh).permute(0, 2, 3, 1, 4).reshape(S, H, G * T, dh), k.transpose(2, 3)).view(S, H, G, T, -1) * dh ** -0.5
    if c["cap"]:
        a = c["cap"] * torch.tanh(a / c["cap"])
    p = (st["kv_len"][:, None] - n + i)[:, :, None]
    t = torch.arange(table.shape[1] * bt, device=DEV)
    if c["slopes"]:
        a = a - st["slopes"].view(H, G, 1, 1) * (p - t).abs()[:, None, None]
    sees = t <= p
    if c["window"]:
        sees = sees & (p - t < c["window"])
    if c["prefix"]:
        sees = sees | (t < st["prefix"][:, None, None])
    sees = sees & (t < st["kv_len"][:, None, None]) & (table >= 0).repeat_interleave(bt, 1)[:, None]
    a = a.masked_fill(~sees[:, None, None], -math.inf)
    a = torch.exp(a - a.amax(-1, keepdim=True).clamp(min=-3e38))
    o = torch.matmul(a.view(S, H, G * T, -1), v) / a.sum(-1).view(S, H, G * T, 1).clamp(min=1e-30)
    seq, i, _ = _row_places(st)
    return o.view(S, H, G, T, dh).permute(0, 3, 1, 2, 4).reshape(S, T, c["heads"] * dh)[seq, i].to(torch.bfloat16)


# -------------------------------------------------------------------------------------------------- the framework's operators
def _call(st):
    """The call with its arguments marshalled once, as a serving loop keeps it, and its outputs."""
    from paper_2508_09204_amd import binding as mq
    c = st["case"]
    if c["kind"] == "norm":
        norm = lambda n: mq.Norm(c[n], EPS, st[n + "_gain"], st[n + "_offset"]) if c[n] else None  # noqa: E731
        out = {"residual": torch.empty_like(st["r"]), "out": torch.empty((c["M"], c["d"]), dtype=torch.bfloat16, device=DEV)}
        return mq.ResidualNormCall(st["y"], st["r"], out["out"], residual_out=out["residual"], gate=st["gate"], gate_rows=c["gate_rows"],
                                   scale=c["scale"], post=norm("post"), pre=norm("pre")), out
    cache = mq.KvCache(st["k"], st["v"], st["k_scale"], st["v_scale"], c["bt"], c["dh"])
    batch = mq.KvBatch(st["table"], st["kv_len"], S=c["S"], T=max(st["rows"]), M=st["M"], cu_rows=st["cu"])
    if c["kind"] == "append":
        rope = mq.Rope(st["inv_freq"], c["rot"], interleaved=c["inter"], q_gain=st["gains"][0], k_gain=st["gains"][1], eps=EPS)
        q = torch.empty((st["M"], c["heads"], c["dh"]), dtype=torch.bfloat16, device=DEV)
        return mq.KvAppendCall(st["qkv"], c["heads"], rope, batch, cache, q), {"q": q, **_cache_values(st)}
    out = torch.empty((st["M"], c["heads"] * c["dh"]), dtype=torch.bfloat16, device=DEV)
    attn = mq.Attention(c["heads"], c["dh"] ** -0.5, cap=c["cap"], window=c["window"], slopes=st["slopes"], prefix=st["prefix"])
    return mq.KvAttentionCall(st["q"], attn, batch, cache, out), out


def run(st):
    if own:
        if "call" not in st:
            st["call"] = _call(st)
        call, out = st["call"]
        call()
        return out
    return {"norm": _plain_norm, "append": _plain_append, "attend": _plain_attend}[st["case"]["kind"]](st)


# ------------------------------------------------------------------------------------------------------------- bytes, operations
def _pairs_seen(c, rows, lens):
    """Pairs of a row and a token that it sees, and tokens that any row of their sequence sees."""
    seen, tokens = 0, 0
    for n, L in zip(rows, lens):
        pre, w = min(c["prefix"], L), c["window"]
        for p in range(L - n, L):
            lo = max(0, p + 1 - w) if w else 0
            seen += p + 1 - lo + max(0, pre - (p + 1)) + min(lo, pre)
        lo = max(0, L - n + 1 - w) if w else 0
        tokens += L - lo + min(lo, pre)
    return seen, tokens


def work(c):
    if c["kind"] == "norm":
        size = {"fp32": 4, "bf16": 2}
        vectors = (c["post"] == "rms") + 2 * (c["post"] == "layer") + (c["pre"] == "rms") + 2 * (c["pre"] == "layer")
        gates = 0 if not c["gate"] else 1 if c["gate"] == "all" else -(-c["M"] // c["gate_rows"])
        return {"bytes": c["M"] * c["d"] * (size[c["y"]] + 2 * size[c["res"]] + 2) + 4 * c["d"] * (vectors + gates), "flops": 10 * c["M"] * c["d"]}
    rows, past = _lengths(c)
    M, lens = sum(rows), [a + b for a, b in zip(rows, past)]
    H, dh = c["kv"], c["dh"]
    if c["kind"] == "append":
        size = 4 if c["qkv"] == "fp32" else 2
        blocks = sum(-(-n // c["bt"]) - b // c["bt"] for n, b in zip(lens, past))
        return {"bytes": M * (c["heads"] + 2 * H) * dh * size + M * c["heads"] * dh * 2 + 2 * M * H * dh + 8 * blocks * H,
                "flops": 6 * M * (c["heads"] + 2 * H) * dh}
    seen, tokens = _pairs_seen(c, rows, lens)
    return {"bytes": 2 * tokens * H * dh + 4 * M * c["heads"] * dh, "flops": 4 * seen * c["heads"] * dh}


# ------------------------------------------------------------------------------------------------------------------ in 64 bits
def _e4m3_table():
    """What the 256 codes stand for: sign, four bits of exponent (bias 7), three of mantissa."""
    u = torch.arange(256, dtype=torch.float64)
    e, m = torch.div(u % 128, 8, rounding_mode="floor"), u % 8
    x = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7))
    return torch.where(u < 128, x, -x).to(DEV)


def _e4m3_nearest(x):
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _address(c, name, block, head, token, dim):
    """Where the code of a token's dim lies: `block`, `head`, `token` (in its block) and `dim` broadcast."""
    bt, dh = c["bt"], c["dh"]
    base = (block * c["kv"] + head) * (bt * dh)
    if name == "k":
        lane = (dim % 32) // 8 * 16 + token % 16
        return base + token // 16 * (16 * dh) + dim // 64 * 1024 + lane * 16 + dim % 64 // 32 * 8 + dim % 8
    u = token % 32
    lane = u % 16 // 4 * 16 + dim % 16
    return base + token // 32 * (32 * dh) + dim // 32 * 1024 + lane * 16 + dim % 32 // 16 * 8 + u // 16 * 4 + u % 4


def _exact_norm(st):
    c = st["case"]

    def norm(x, n):
        if c[n] == "layer":
            return torch.nn.functional.layer_norm(x, (c["d"],), st[n + "_gain"].double(), st[n + "_offset"].double(), EPS)
        return x / (x.pow(2).sum(1, keepdim=True) / c["d"] + EPS).sqrt() * st[n + "_gain"].double()

    u = norm(st["y"].double(), "post") if c["post"] else st["y"].double()
    if c["gate"]:
        row = torch.arange(c["M"], device=DEV) // max(1, c["gate_rows"])
        u = u * (st["gate"].double() if c["gate"] == "all" else st["gate"].double()[row])
    t = st["r"].double() + c["scale"] * u
    return {"residual": t, "out": norm(t, "pre")}


def _exact_append(st):
    c = st["case"]
    H, Hq, dh, bt, half = c["kv"], c["heads"], c["dh"], c["bt"], c["rot"] // 2
    x = st["qkv"].double().view(st["M"], -1, dh)
    if c["norm"]:
        gain = torch.ones((Hq + 2 * H, dh), dtype=torch.float64, device=DEV)
        gain[:Hq], gain[Hq : Hq + H] = st["gains"][0].double(), st["gains"][1].double()
        size = (x.pow(2).sum(-1, keepdim=True) / dh + EPS).sqrt()
        size[:, Hq + H :] = 1
        x = x / size * gain
    pos = torch.cat([torch.arange(n - r, n, device=DEV) for r, n in zip(st["rows"], st["lens"])])
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.double()[:, None] * st["inv_freq"])[:, None]
    j = torch.arange(half, device=DEV)
    a, b = (2 * j, 2 * j + 1) if c["inter"] else (j, j + half)
    z = torch.complex(x[:, : Hq + H, a], x[:, : Hq + H, b]) * turn
    x[:, : Hq + H, a], x[:, : Hq + H, b] = z.real, z.imag
    table, got = _e4m3_table(), {"q": x[:, :Hq]}
    dims, heads = torch.arange(dh, device=DEV), torch.arange(H, device=DEV)[:, None, None]
    for name, at in (("k", Hq), ("v", Hq + H)):
        values, scales = table[st[name].long()].reshape(-1), st[name + "_scale"].double()
        row = 0
        for s in range(c["S"]):
            n, L = st["rows"][s], st["lens"][s]
            mine = x[row : row + n, at : at + H].transpose(0, 1)                          # [heads, rows, dims]
            row += n
            ids = st["table"][s].tolist()
            for b in range((L - n) // bt, -(-L // bt)):
                lo, hi = max(L - n, b * bt), min(L, (b + 1) * bt)
                new = mine[:, lo - (L - n) : hi - (L - n)]
                scale = torch.exp2(torch.ceil(torch.log2(new.abs().flatten(1).amax(1) / 448)).clamp(-120, 120))
                if lo > b * bt:
                    scale = torch.maximum(scale, scales[ids[b]])
                old = _address(c, name, ids[b], heads, torch.arange(b * bt, lo, device=DEV)[:, None] % bt, dims)
                values[old] = _e4m3_nearest(values[old] * (scales[ids[b]] / scale)[:, None, None])
                values[_address(c, name, ids[b], heads, torch.arange(lo, hi, device=DEV)[:, None] % bt, dims)] = _e4m3_nearest(new / scale[:, None, None])
                scales[ids[b]] = scale
        got[name], got[name + "_scale"] = values.view(st[name].shape), scales
    return got


def _exact_attend(st):
    c = st["case"]
    H, G, dh, bt = c["kv"], c["heads"] // c["kv"], c["dh"], c["bt"]
    table, dims = _e4m3_table(), torch.arange(dh, device=DEV)
    out = torch.zeros((st["M"], c["heads"], dh), dtype=torch.float64, device=DEV)
    row = 0
    for s in range(c["S"]):
        n, L = st["rows"][s], st["lens"][s]
        t, p = torch.arange(L, device=DEV), torch.arange(L - n, L, device=DEV)[:, None]
        block = st["table"][s, t // bt].long()
        far = (p - t).abs()
        hidden = t > p
        if c["window"]:
            hidden = hidden | (p - t >= c["window"])
        hidden = hidden & (t >= c["prefix"])
        for h in range(H):
            k, v = (table[st[m].view(-1)[_address(c, m, block[:, None], h, t[:, None] % bt, dims)].long()] * st[m + "_scale"][block, h].double()[:, None]
                    for m in ("k", "v"))
            for g in range(h * G, (h + 1) * G):
                a = st["q"][row : row + n, g].double() @ k.T / math.sqrt(dh)
                a = c["cap"] * torch.tanh(a / c["cap"]) if c["cap"] else a
                a = a - st["slopes"][g].double() * far if c["slopes"] else a
                out[row : row + n, g] = torch.softmax(a.masked_fill(hidden, -math.inf), 1) @ v
        row += n
    return out.view(st["M"], -1)


def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _exact_norm, "append": _exact_append, "attend": _exact_attend}[case["kind"]](st)
