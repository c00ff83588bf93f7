"""Performance cases of the 8-bit floating-point path and of the step from a decoder's last rows to its next tokens.

`listed()` names the cases, `draw(rng)` gives further ones of the same ranges, `prepare` builds what a serving program holds before
the call, `run` makes one call, `work` states the bytes and operations the call cannot do without, `exact` is the same call in
64-bit arithmetic.  With `own` false `run` computes the operators from elementary torch operations, in 32 bits and in 64 where
values next to a border decide.

Kinds of calls:
  norm     moqe_residual_norm_f8: r' = r + scale * gate * post(y), out = pre(r') in e4m3 with a power-of-two scale for each 128 features
  product  moqe_f8_gemm: rows times matrices, both in e4m3 with a power-of-two scale for each 128 values of a row; dense or by expert,
           plain or gated (silu(g) * u)
  sample   moqe_sample: one token a row by temperature, top-k, top-p and min-p from a given uniform number

8-bit rows: codes uint8 [rows, features padded to 128], scales uint8 [rows, blocks padded to 4], 127 + the power of two.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
BLOCK = 128


def listed():
    return [
        # ---- norms whose rows go into an 8-bit product
        # decode of 64 requests at width 4096: the block's fp32 rows onto a bf16 residual, normed for the next projection
        dict(name="norm_decode", kind="norm", M=64, d=4096, y="fp32", res="bf16", post="", pre="rms", gate="", gate_rows=0, scale=1.0),
        # prefill of 128 sequences of 256 tokens at width 3584, norms before and after the block, a learned gate for each feature
        dict(name="norm_prefill", kind="norm", M=32768, d=3584, y="bf16", res="fp32", post="rms", pre="rms", gate="all", gate_rows=0,
             scale=0.5),
        # an odd width in layer norms with a gate vector for each sample: unaligned rows, a last block of 107 features
        dict(name="norm_odd", kind="norm", M=1500, d=1003, y="fp32", res="fp32", post="layer", pre="layer", gate="sample",
             gate_rows=196, scale=1.0),
        # ---- products
        # one request being decoded, its row onto a vocabulary of 32000: the smallest product
        dict(name="product_one", kind="product", K=1, S=1, T=1, k=4096, n=32000, gated=False, out="fp32", skew=0.0),
        # a decode step of 64 requests on four experts: gate and up of an MLP 4096 / 11008, the result again in 8 bits
        dict(name="product_decode", kind="product", K=4, S=64, T=1, k=4096, n=11008, gated=True, out="f8", skew=0.3),
        # rows of a padded width onto an odd vocabulary: nothing divides by a tile
        dict(name="product_odd", kind="product", K=1, S=777, T=1, k=1000, n=50257, gated=False, out="fp32", skew=0.0),
        # 16 prompts of 512 tokens, the way down of an MLP 4096 / 11008, one matrix for all
        dict(name="product_prefill", kind="product", K=1, S=16, T=512, k=11008, n=4096, gated=False, out="bf16", skew=0.0),
        # the largest: the same prompts on four experts, gate and up, the result again in 8 bits
        dict(name="product_gated", kind="product", K=4, S=16, T=512, k=4096, n=11008, gated=True, out="f8", skew=0.3),
        # ---- tokens
        # one request, a vocabulary of 32000, every filter on
        dict(name="sample_one", kind="sample", S=1, V=32000, logits="fp32", sharp=2.5, filters="all"),
        # 64 requests with settings of their own on a vocabulary of 128000
        dict(name="sample_batch", kind="sample", S=64, V=128000, logits="fp32", sharp=2.5, filters="mixed"),
        # bf16 logits (equal values among them) of an odd vocabulary, flat distributions
        dict(name="sample_odd", kind="sample", S=200, V=50257, logits="bf16", sharp=1.0, filters="mixed"),
        # 256 requests, temperature alone
        dict(name="sample_plain", kind="sample", S=256, V=32000, logits="fp32", sharp=2.5, filters="none"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "product", "product", "product", "sample", "sample"))
    if kind == "norm":
        d = _log(rng, 64, 16384)
        if rng.random() < 0.5:
            d = max(64, d // 64 * 64)
        gate = rng.choice(("", "all", "sample"))
        return dict(kind="norm", M=_log(rng, 1, min(32768, 32768 * 3584 // d)), d=d, y=rng.choice(("fp32", "bf16")), res=rng.choice(("fp32", "bf16")),
                    post=rng.choice(("", "rms", "layer")), pre=rng.choice(("rms", "layer")), gate=gate,
                    gate_rows=rng.randint(1, 300) if gate == "sample" else 0, scale=rng.choice((1.0, 0.5, 0.25)))
    if kind == "product":
        K, gated = rng.choice((1, 1, 2, 4, 8)), rng.random() < 0.4
        k, n = _log(rng, 128, 16384), _log(rng, 16, 32768)
        if rng.random() < 0.6:
            k, n = max(128, k // 128 * 128), max(16, n // 16 * 16)
        n = min(n, 2 ** 29 // (k * K))                                                  # experts of at most half a gigabyte, a gigabyte gated
        S = _log(rng, 1, max(1, min(8192, 8192 * 4096 * 11008 // (k * n))))
        T = _log(rng, 1, max(1, min(8192, 8192 * 4096 * 11008 // (k * n)) // S))
        return dict(kind="product", K=K, S=S, T=T, k=k, n=n, gated=gated, out=rng.choice(("fp32", "bf16", "f8") if gated else ("fp32", "bf16")),
                    skew=rng.choice((0.0, 0.3, 1.0)) if K > 1 else 0.0)
    V = _log(rng, 1000, 160000)
    return dict(kind="sample", S=_log(rng, 1, min(256, 256 * 50257 // V)), V=V, logits=rng.choice(("fp32", "bf16")), sharp=rng.choice((0.5, 1.0, 2.5, 4.0)),
                filters=rng.choice(("none", "all", "mixed", "mixed")))


def _type(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


# ------------------------------------------------------------------------------------------------------------------- inputs
def _counts(c):
    """Samples of every expert: shares 1 / (1 + expert)^skew, in an order of the case's own."""
    share = [(1 + e) ** -c["skew"] for e in range(c["K"])]
    edges = [int(c["S"] * sum(share[:e]) / sum(share) + 0.5) for e in range(c["K"] + 1)]
    return [b - a for a, b in zip(edges, edges[1:])]


def _rows(x):
    """8-bit rows of fp32 rows x [M, d]: codes [M, blocks * 128], scale bytes [M, blocks]."""
    M, d = x.shape
    blocks = -(-d // BLOCK)
    x = torch.nn.functional.pad(x, (0, blocks * BLOCK - d)).view(M, blocks, BLOCK)
    m, e = torch.frexp(x.abs().amax(2))
    e = torch.where(m == 0, -120, (e - 9 + (m > 0.875)).clamp(-120, 120))               # 448 is 0.875 * 2 ** 9
    codes = torch.ldexp(x, -e[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.view(M, blocks * BLOCK), (e + 127).to(torch.uint8)


def _padded(scales):
    return torch.nn.functional.pad(scales, (0, -scales.shape[1] % 4)).contiguous()


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
    elif c["kind"] == "product":
        M, k = c["S"] * c["T"], c["k"]
        wide = 1.0 + 3.0 * (torch.rand((k,), generator=g, device=DEV) < 0.01)
        codes, scales = _rows(rand(M, k) * wide)
        st["a"] = codes.contiguous(), _padded(scales)
        st["w"] = []
        for _ in range(c["K"] * (2 if c["gated"] else 1)):
            codes, scales = _rows(rand(c["n"], k) * k ** -0.5)
            st["w"].append((codes.contiguous(), _padded(scales)))
        st["counts"] = _counts(c)
        at = [0]
        for n in st["counts"]:
            at.append(at[-1] + n)
        st["offsets"] = torch.tensor(at, dtype=torch.int32).to(DEV)
        st["perm"] = torch.randperm(c["S"], generator=torch.Generator().manual_seed(seed)).to(torch.int32).to(DEV)
    else:
        S, V = c["S"], c["V"]
        x = rand(S, V) * c["sharp"]
        x += 4.0 * c["sharp"] * (torch.rand((S, V), generator=g, device=DEV) < 8.0 / V)     # a few likely tokens
        st["logits"] = x.to(_type(c["logits"]))
        st["u"] = torch.rand((S,), generator=g, device=DEV)
        pick = lambda *v: torch.tensor(v, device=DEV)[torch.randint(0, len(v), (S,), generator=g, device=DEV)]  # noqa: E731
        mixed = c["filters"] == "mixed"
        st["temperature"] = 0.6 + 0.6 * torch.rand((S,), generator=g, device=DEV)
        if mixed:
            st["temperature"][torch.rand((S,), generator=g, device=DEV) < 0.1] = 0.0
        st["top_k"] = st["top_p"] = st["min_p"] = None
        if c["filters"] != "none":                                                          # 0 and 1 leave a filter out
            st["top_k"] = pick(*((0, 0, 1, 20, 50, 500) if mixed else (40, 50, 100))).to(torch.int32)
            st["top_p"] = pick(*((1.0, 0.5, 0.9, 0.95) if mixed else (0.9, 0.95)))
            st["min_p"] = pick(*((0.0, 0.0, 0.02, 0.1) if mixed else (0.01, 0.05)))
    return st


# --------------------------------------------------------------------------------------------------------- the plain forms
def _normed(x, kind, gain, offset):
    if kind == "rms":
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain + offset


def _values(codes, scales):
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}


def _plain_norm(st):
    c = st["case"]
    u, r = st["y"].float(), st["r"].float()
    if c["post"]:
        u = _normed(u, c["post"], st["post_gain"], st["post_offset"])
    if c["gate"]:
        u = u * (st["gate"] if c["gate"] == "all" else st["gate"].repeat_interleave(c["gate_rows"], 0)[: c["M"]])
    t = r + c["scale"] * u
    return {"residual": t.to(st["r"].dtype), **_values(*_rows(_normed(t, c["pre"], st["pre_gain"], st["pre_offset"])))}


def _floats(rows, d):
    codes, scales = rows
    n = codes.shape[1] // BLOCK
    return (codes.view(torch.float8_e4m3fn).float().view(-1, n, BLOCK) * scales[:, :n].view(torch.float8_e8m0fnu).float()[:, :, None]).flatten(1)[:, :d]


def _bucket_rows(st, at, n):
    """Numbers of the rows of n samples in bucket order from `at` on."""
    T = st["case"]["T"]
    return (st["perm"][at : at + n].long()[:, None] * T + torch.arange(T, device=DEV)).flatten()


def _plain_product(st):
    c = st["case"]
    a = _floats(st["a"], c["k"])
    y = torch.empty((a.shape[0], c["n"]), device=DEV)
    at = 0
    for e, n in enumerate(st["counts"]):
        rows = _bucket_rows(st, at, n)
        at += n
        x = a[rows]
        if c["gated"]:
            gate, up = (torch.matmul(x, _floats(w, c["k"]).T) for w in st["w"][2 * e : 2 * e + 2])
            y[rows] = gate / (1.0 + torch.exp(-gate)) * up
        else:
            y[rows] = torch.matmul(x, _floats(st["w"][e], c["k"]).T)
    return _values(*_rows(y)) if c["out"] == "f8" else y.to(_type(c["out"]))


def _plain_sample(st):
    logits = st["logits"].double()
    S, V = logits.shape
    T = st["temperature"].double()[:, None]
    greedy = T <= 0
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices
    x = logits / torch.where(greedy, 1.0, T)
    w = torch.exp(x - x.amax(1, keepdim=True)).gather(1, order)
    place = torch.arange(V, device=DEV)
    kept = place < torch.where(greedy, 1, V)
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        kept &= (k <= 0) | (place < k)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        run = (w * kept).cumsum(1)
        kept &= (p >= 1) | (run - w * kept < p * run[:, -1:])
    if st["min_p"] is not None:
        kept &= w >= st["min_p"].double()[:, None]
    kept = torch.zeros_like(kept).scatter(1, order, kept)
    w = torch.zeros_like(w).scatter(1, order, w) * kept
    run = w.cumsum(1)
    token = (run <= st["u"].double()[:, None] * run[:, -1:]).sum(1).clamp(max=V - 1)
    return {"tokens": token.to(torch.int32), "logprobs": torch.log(w.gather(1, token[:, None])[:, 0] / run[:, -1]).float()}


# -------------------------------------------------------------------------------------------------- the framework's operators
def _call(st):
    """The call with its arguments marshalled once, as a serving loop keeps it, and its outputs."""
    from paper_2508_09204_amd import binding as mq
    c = st["case"]
    if c["kind"] == "norm":
        norm = lambda n: mq.Norm(c[n], EPS, st[n + "_gain"], st[n + "_offset"]) if c[n] else None  # noqa: E731
        rows, residual = mq.F8Rows.empty(c["M"], c["d"], DEV), torch.empty_like(st["r"])
        call = mq.ResidualNormF8Call(st["y"], st["r"], rows, residual_out=residual, gate=st["gate"], gate_rows=c["gate_rows"], scale=c["scale"],
                                     post=norm("post"), pre=norm("pre"))
        return call, {"residual": residual, **_values(rows.codes, rows.scales[:, : rows.blocks])}
    if c["kind"] == "product":
        M = c["S"] * c["T"]
        rows = lambda w, m: mq.F8Rows(w[0], w[1], m, c["k"])  # noqa: E731
        w = [rows(x, c["n"]) for x in st["w"]]
        mats = [mq.F8Mat.pack(*w[e * len(w) // c["K"] : (e + 1) * len(w) // c["K"]]) for e in range(c["K"])]
        if c["out"] == "f8":
            y = mq.F8Rows.empty(M, c["n"], DEV)
            out = _values(y.codes, y.scales[:, : y.blocks])
        else:
            y = out = torch.empty((M, c["n"]), dtype=_type(c["out"]), device=DEV)
        if c["K"] == 1:
            return mq.F8GemmCall(rows(st["a"], M), mats, y), out
        return mq.F8GemmCall(rows(st["a"], M), mats, y, offsets=st["offsets"], perm=st["perm"], S=c["S"], T=c["T"], scatter=True), out
    tokens, logprobs = torch.empty((c["S"],), dtype=torch.int32, device=DEV), torch.empty((c["S"],), device=DEV)
    call = mq.SampleCall(st["logits"], st["u"], tokens, temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"],
                         logprobs=logprobs)
    return call, {"tokens": tokens, "logprobs": logprobs}


def run(st):
    if own:
        if "call" not in st:
            st["call"] = _call(st)
        call, out = st["call"]
        call()
        return out
    return {"norm": _plain_norm, "product": _plain_product, "sample": _plain_sample}[st["case"]["kind"]](st)


# ------------------------------------------------------------------------------------------------------------- bytes, operations
def work(c):
    size = {"fp32": 4, "bf16": 2}
    if c["kind"] == "norm":
        vectors = (c["post"] == "rms") + 2 * (c["post"] == "layer") + (c["pre"] == "rms") + 2 * (c["pre"] == "layer")
        gates = 0 if not c["gate"] else 1 if c["gate"] == "all" else -(-c["M"] // c["gate_rows"])
        return {"bytes": c["M"] * (c["d"] * (size[c["y"]] + 2 * size[c["res"]] + 1) + -(-c["d"] // BLOCK)) + 4 * c["d"] * (vectors + gates),
                "flops": 12 * c["M"] * c["d"]}
    if c["kind"] == "product":
        M, k, n, mats = c["S"] * c["T"], c["k"], c["n"], sum(x > 0 for x in _counts(c)) * (2 if c["gated"] else 1)
        blocks = -(-k // BLOCK)
        out = n + -(-n // BLOCK) if c["out"] == "f8" else n * size[c["out"]]
        return {"bytes": (M + mats * n) * (k + blocks) + M * out, "flops": 2 * M * n * k * (2 if c["gated"] else 1)}
    return {"bytes": c["S"] * (c["V"] * size[c["logits"]] + 28), "flops": 8 * c["S"] * c["V"]}


# ------------------------------------------------------------------------------------------------------------------ in 64 bits
def _e4m3_table():
    """What the 256 codes stand for: sign, four bits of exponent (bias 7), three of mantissa."""
    u = torch.arange(256, dtype=torch.float64)
    e, m = torch.div(u % 128, 8, rounding_mode="floor"), u % 8
    x = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7))
    return torch.where(u < 128, x, -x).to(DEV)


def _exact_rows(x):
    """Codes' values and scales of rows in 64 bits."""
    M, d = x.shape
    blocks = -(-d // BLOCK)
    x = torch.cat((x, x.new_zeros(M, blocks * BLOCK - d)), 1).unflatten(1, (blocks, BLOCK))
    scale = torch.exp2(torch.ceil(torch.log2(x.abs().amax(2) / 448)).clamp(-120, 120))
    x = x / scale[:, :, None]
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return {"codes": (torch.round(x / step) * step).clamp(-448, 448).flatten(1), "scales": scale}


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
    return {"residual": t, **_exact_rows(norm(t, "pre"))}


def _exact_product(st):
    c = st["case"]
    table = _e4m3_table()

    def matrix(rows):
        codes, scales = rows
        return table[codes.long()] * torch.exp2(scales.double() - 127)[:, torch.arange(codes.shape[1], device=DEV) // BLOCK]

    a, out, first = matrix(st["a"]), [], 0
    for e in range(c["K"]):
        x = a.unflatten(0, (c["S"], c["T"]))[st["perm"][first : first + st["counts"][e]].long()].flatten(0, 1)
        first += st["counts"][e]
        if c["gated"]:
            gate = x @ matrix(st["w"][2 * e]).T
            out.append(torch.nn.functional.silu(gate) * (x @ matrix(st["w"][2 * e + 1]).T))
        else:
            out.append(x @ matrix(st["w"][e]).T)
    y = torch.empty((c["S"], c["T"], c["n"]), dtype=torch.float64, device=DEV)
    y[st["perm"].long()] = torch.cat(out).unflatten(0, (c["S"], c["T"]))
    return _exact_rows(y.flatten(0, 1)) if c["out"] == "f8" else y.flatten(0, 1)


def _exact_sample(st):
    """Row by row, the kept set grown from the most likely token down."""
    c, tokens, logprobs = st["case"], [], []
    for s in range(c["S"]):
        x, T = st["logits"][s].double(), float(st["temperature"][s])
        order = torch.argsort(x, dim=0, descending=True, stable=True)
        x = x[order] / (T if T > 0 else 1.0)
        n = 1 if T <= 0 else c["V"]
        if st["top_k"] is not None and int(st["top_k"][s]) > 0:
            n = min(n, int(st["top_k"][s]))
        w = torch.exp(x[:n] - x[0])
        if st["top_p"] is not None and float(st["top_p"][s]) < 1:
            n = int(torch.searchsorted(torch.cumsum(w, 0), float(st["top_p"][s]) * w.sum())) + 1
            w = w[:n]
        if st["min_p"] is not None:
            w = w[w >= float(st["min_p"][s])]
        at = torch.argsort(order[: len(w)])
        run = torch.cumsum(w[at], 0)
        i = min(int(torch.searchsorted(run, float(st["u"][s]) * run[-1], right=True)), len(w) - 1)
        tokens.append(order[at[i]])
        logprobs.append(torch.log(w[at[i]] / run[-1]))
    return {"tokens": torch.stack(tokens).to(torch.int32), "logprobs": torch.stack(logprobs)}


def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _exact_norm, "product": _exact_product, "sample": _exact_sample}[case["kind"]](st)
