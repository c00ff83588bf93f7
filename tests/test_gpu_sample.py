"""moqe_sample on the GPU against the 64-bit oracle.

Tokens have to be equal.  Sums on the GPU are of weights cut to 2^-42 of the largest, V of them, once for the share that top-p asks for and once for the draw: a choice that lies nearer to another
one than V 2^-40 of the largest weight (the oracle's gap) could come out either way and is passed over.  logprobs: fp32, half a step, and 2^-20 absolute for the weights' sums (V 2^-42 for the
largest V, times four)."""
import math

import numpy as np
import pytest
import torch

from oracle import f8_oracle as fo
from paper_2508_09204_amd import binding as mq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def run(logits, u, stride=None, **how):
    """logits: tensor [S, V] on the GPU; how: lists of a value per row."""
    S, V = logits.shape
    kinds = {"temperature": F32, "top_k": torch.int32, "top_p": F32, "min_p": F32}
    args = {k: torch.tensor(v, dtype=kinds[k], device=DEV) for k, v in how.items()}
    tokens, lp = torch.full((S,), -9, dtype=torch.int32, device=DEV), torch.full((S,), 7.0, device=DEV)
    mq.moqe_sample(logits, torch.tensor(u, dtype=F32, device=DEV), tokens, logprobs=lp, **args)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), lp.double().cpu().numpy(), {k: t.double().cpu().numpy() for k, t in args.items()}


def check(logits, u, **how):
    tokens, lp, args = run(logits, u, **how)
    x = logits.double().cpu().numpy()
    u32 = torch.tensor(u, dtype=F32).double().numpy()
    near = 0
    for s in range(len(x)):
        row = {k: (int(v[s]) if k == "top_k" else float(v[s])) for k, v in args.items()}
        want, want_lp, gap = fo.sample(x[s], u32[s], **row)
        if gap <= x.shape[1] * 2.0 ** -40:
            near += 1
            continue
        assert tokens[s] == want, (s, row, u32[s], tokens[s], want, gap)
        assert lp[s] == want_lp or abs(lp[s] - want_lp) <= 2.0 ** -24 * abs(want_lp) + 2.0 ** -20, (s, lp[s], want_lp)
    assert near <= 1 + len(x) // 8                                  # such rows are rare
    return tokens


def logits_of(S, V, t=F32, sharp=2.0, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + V)
    return (torch.randn((S, V), generator=g, device=DEV) * sharp).to(t)


def uniform(S, seed=0):
    return np.random.default_rng(seed).random(S).astype(np.float32).tolist()


SIZES = [1, 2, 3, 63, 64, 65, 255, 1000, 1024, 1025, 4096, 4097, 8191, 16384, 16385, 32000, 50257, 131072, 262145]


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("t", [F32, BF])
def test_sizes(V, t):
    S = 6
    x = logits_of(S, V, t)
    u = uniform(S, V)
    check(x, u)
    check(x, u, temperature=[0.7, 1.0, 0.0, 1.3, 0.2, 5.0])
    check(x, u, top_k=[1, 0, 5, 40, V, -1], top_p=[0.9, 0.5, 1.0, 0.95, 0.3, 0.8], min_p=[0.0, 0.01, 0.1, 0.0, 0.0, 0.3], temperature=[1.0, 0.8, 1.1, 0.6, 1.0, 2.0])


@pytest.mark.parametrize("t", [F32, BF])
@pytest.mark.parametrize("sharp", [0.05, 1.0, 8.0])
def test_each_filter(t, sharp):
    S, V = 24, 3001
    x, u = logits_of(S, V, t, sharp, 5), uniform(S, 3)
    check(x, u, top_k=[1, 2, 3, 4, 7, 15, 16, 17, 63, 64, 65, 100, 255, 256, 257, 500, 1000, 1023, 1024, 1025, 2000, 3000, 3001, 3002])
    check(x, u, top_p=np.linspace(0.0, 1.05, S).tolist())
    check(x, u, min_p=[0.0, 1e-6, 1e-4, 1e-3, 0.003, 0.01, 0.02, 0.05, 0.1, 0.15, 0.2, 0.3, 0.4, 0.5, 0.6, 0.7, 0.8, 0.9, 0.99, 1.0, 1.5, -1.0, float("nan"), 0.25])
    check(x, u, temperature=[0.0, -1.0, float("nan"), 0.01, 0.1, 0.2, 0.3, 0.5, 0.7, 0.9, 1.0, 1.1, 1.5, 2.0, 3.0, 5.0, 10.0, 100.0, 1e4, float("inf"), 1e-6, 1e-30, 0.6, 0.8])


def test_equal_logits_go_by_index():
    """All equal, two values, and bf16 steps: cuts fall inside runs of equal values."""
    S, V = 16, 5000
    u = np.linspace(0.01, 0.99, S).tolist()
    flat = torch.zeros((S, V), device=DEV)
    check(flat, u)
    check(flat, u, top_k=[1, 2, 3, 10, 64, 100, 1000, 1024, 2000, 3333, 4096, 4999, 5000, 7, 65, 257])
    check(flat, u, top_p=(np.arange(1, S + 1) / S * 0.999 + 1e-4).tolist())
    two = (torch.arange(V, device=DEV) % 7 == 3).float().repeat(S, 1)
    check(two, u, top_k=[5, 700, 714, 715, 716, 1000, 4000, 5000] * 2, top_p=[0.9] * 8 + [0.31234] * 8)
    check(two, u, top_p=(np.arange(1, S + 1) / S * 0.999 + 1e-4).tolist(), min_p=[0.2, 0.5] * 8)
    steps = torch.round(logits_of(S, V, F32, 1.0, 9) * 2) / 2
    check(steps, u, top_k=[50, 300, 1000, 2500] * 4, top_p=[0.2, 0.6, 0.9, 1.0] * 4)


@pytest.mark.parametrize("t", [F32, BF])
@pytest.mark.parametrize("V,sharp", [(20000, 0.02), (60000, 0.3), (110000, 1.0), (300000, 0.4), (1 << 20, 0.5)])
def test_cuts_among_many(V, sharp, t):
    """Cuts fall where thousands to hundreds of thousands of logits lie within a quarter of an octave."""
    S = 4
    x, u = logits_of(S, V, t, sharp, 11), uniform(S, V)
    check(x, u, top_k=[V // 2, V // 7, V - 100, 0], top_p=[1.0, 0.3, 0.9, 0.5])
    check(x, u, top_p=[0.1, 0.5, 0.9, 0.99], temperature=[0.7, 1.0, 1.5, 1.0], min_p=[0.0, 0.5, 0.0, 0.3])


def test_special_values():
    inf, nan = float("inf"), float("nan")
    V = 700
    x = logits_of(12, V)
    x[0] = -inf
    x[1] = nan
    x[2, :] = -inf
    x[2, 699] = -50.0
    x[3, 5], x[3, 600] = inf, inf
    x[4, ::2] = -inf
    x[5, 1::2] = nan
    x[6, 100] = 3e38
    x[7] = -3e38
    x[8] = torch.where(torch.arange(V, device=DEV) % 2 == 0, 0.0, -0.0)
    x[9, :350], x[9, 350:] = 1e-40, -1e-40
    x[10], x[10, 17] = -inf, nan
    x[11], x[11, 3], x[11, 4] = nan, inf, -inf
    tokens = check(x, uniform(12, 8))
    assert tokens[0] == -1 and tokens[1] == -1 and tokens[2] == 699 and tokens[10] == -1 and tokens[11] == 3 and tokens[6] == 100
    check(x, uniform(12, 9), top_k=[3] * 12, top_p=[0.8] * 12, min_p=[0.01] * 12, temperature=[0.5] * 12)
    assert check(x, uniform(12, 9), temperature=[0.0] * 12)[3] == 5


@pytest.mark.parametrize("t", [F32, BF])
def test_every_kind_of_nan_is_passed_over(t):
    x = logits_of(3, 900, t)
    bits = x.view(torch.int16 if t == BF else torch.int32)
    kinds = [0x7fc0, 0x7f81, 0xffc0 - 65536, 0xff81 - 65536] if t == BF else [0x7fc00000, 0x7f800001, 0xffc00000 - (1 << 32), 0xff800001 - (1 << 32)]
    for i, b in enumerate(kinds):
        bits[:, i::7] = b
    assert int(x.isnan().sum()) == 3 * sum(len(range(i, 900, 7)) for i in range(4))
    check(x, uniform(3))
    check(x, uniform(3), top_k=[5, 0, 100], top_p=[0.9, 0.5, 1.0])
    check(x, uniform(3), temperature=[0.0] * 3)


def test_u_at_its_ends():
    x = logits_of(4, 2000)
    x[:, -300:] = -float("inf")
    x[:, :10] = -float("inf")
    tokens, _, _ = run(x, [0.0, 1.0, float("nan"), 5.0])
    assert tokens.tolist() == [10, 1699, 10, 1699]
    tokens, _, _ = run(x, [0.0, 1.0, -3.0, 1.0], top_k=[3] * 4)
    top = torch.topk(x, 3, 1).indices.sort(1).values.cpu().numpy()
    assert tokens.tolist() == [top[0, 0], top[1, 2], top[2, 0], top[3, 2]]


def test_every_token_has_its_share():
    """2^14 rows of one distribution with evenly spread u: each kept token comes up as often as its probability says, within one count at each end of its interval."""
    S, V = 1 << 14, 97
    row = logits_of(1, V, F32, 1.5, 2)
    u = ((np.arange(S) + 0.5) / S).astype(np.float32)
    tokens, lp, _ = run(row.expand(S, V).contiguous(), u.tolist(), top_p=[0.9] * S, temperature=[1.2] * S)
    count = np.bincount(tokens, minlength=V)
    seen = {t: l for t, l in zip(tokens, lp)}
    assert abs(sum(math.exp(l) for l in seen.values()) - 1) < 1e-5
    for t, l in seen.items():
        assert abs(count[t] - S * math.exp(l)) <= 2
    assert (np.diff(tokens) >= 0).all()


@pytest.mark.parametrize("t", [F32, BF])
@pytest.mark.parametrize("pad,lead", [(0, 0), (1, 0), (3, 1), (8, 2), (5, 3)])
def test_strides_and_alignment(t, pad, lead):
    S, V = 5, 1237
    buf = torch.full((lead + S * (V + pad),), float("nan"), dtype=t, device=DEV)
    buf.fill_(1e4)
    x = buf[lead:].view(S, V + pad)[:, :V]
    x.copy_(logits_of(S, V, t))
    check(x, uniform(S), top_k=[0, 10, 50, 0, 3], top_p=[0.9, 1.0, 0.7, 1.0, 0.5])


def test_many_rows_and_none():
    x = logits_of(700, 513, BF, 2.0)
    check(x, uniform(700), temperature=[0.9] * 700, top_p=[0.95] * 700)
    mq.moqe_sample(torch.empty((0, 10), device=DEV), torch.empty(0, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV))


def test_the_same_every_time_on_streams_and_captured():
    S, V = 9, 40000
    x = logits_of(S, V, F32, 3.0, 4)
    u, tokens, lp = torch.rand(S, device=DEV), torch.empty(S, dtype=torch.int32, device=DEV), torch.empty(S, device=DEV)
    top_p, k = torch.full((S,), 0.9, device=DEV), torch.tensor([0, 1, 50] * 3, dtype=torch.int32, device=DEV)
    call = mq.SampleCall(x, u, tokens, top_k=k, top_p=top_p, logprobs=lp)
    call()
    torch.cuda.synchronize()
    want = tokens.clone(), lp.clone()
    side = torch.cuda.Stream()
    for _ in range(3):
        tokens.fill_(-5)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        assert torch.equal(tokens, want[0]) and torch.equal(lp, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    keep = x.clone()
    for i in range(4):
        x.copy_(logits_of(S, V, F32, 3.0, 40 + i))
        graph.replay()
        torch.cuda.synchronize()
        replayed = tokens.clone(), lp.clone()
        tokens.fill_(-5)
        torch.randn(1000, device=DEV).sum().item()
        call()
        torch.cuda.synchronize()
        assert torch.equal(tokens, replayed[0]) and torch.equal(lp, replayed[1])
    x.copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(tokens, want[0]) and torch.equal(lp, want[1])
