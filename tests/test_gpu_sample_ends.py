"""moqe_sample where single weights are far below what a row's sums are counted in: tokens at the ends of u on rows with faint neighbourhoods, the same token whatever else a call has, and log
probabilities next to 0.

Without filters, weights are rounded to 2^-43 of the power of two above the largest of their 256 neighbours, whose sums are cut to whole units of the row: of a largest weight of 1, V 2^-42 for
roundings and for the table and cubic (2^-42 of a weight) each, and V / 256 units of 2^-42, together less than V 2^-40.  So a token is right if u W lies within V 2^-40 of its part of the running weight.
Log probabilities: fp32, half a step, and 2^-20 absolute for the sums."""
import math

import numpy as np
import pytest
import torch

from paper_2508_09204_amd import binding as mq
from tests.test_gpu_sample import logits_of, run, uniform

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
NAN = float("nan")
ENDS = [0.0, NAN, 1e-45, 1e-30, 2.0 ** -24, 1.0 - 2.0 ** -24, 1.0, 7.0]


def check_token(x, u, token, lp, T=1.0):
    """x: a row's logits in 64 bits."""
    w = np.exp((x - x.max()) / T)
    upto = np.cumsum(w)
    goal = min(max(u, 0.0), 1.0) * upto[-1] if u == u else 0.0
    tol = len(x) * 2.0 ** -40
    assert 0 <= token < len(x), (u, token)
    assert w[token] > 0 and upto[token] - w[token] <= goal + tol and upto[token] >= goal - tol, (u, token, goal, upto[token])
    want = math.log(w[token] / upto[-1])
    assert lp <= 0 and abs(lp - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -20, (lp, want)


def check_all(x, u, T=None, **how):
    tokens, lp, args = run(x, u, **how, **({} if T is None else {"temperature": T}))
    rows, u32 = x.double().cpu().numpy(), torch.tensor(u, dtype=F32).double().numpy()
    for s in range(len(rows)):
        check_token(rows[s], u32[s], tokens[s], lp[s], 1.0 if T is None else args["temperature"][s])


@pytest.mark.parametrize("V", [512, 4096, 32000, 50257, 262145, 1 << 20])
@pytest.mark.parametrize("faint", [-29.3, -30.3, -30.6, -31.0, -33.0, -36.0, -60.0])
def test_one_logit_above_faint_ones(V, faint):
    """The largest in the first, a middle and the last place, the others 42 to 87 octaves below: both ends of u fall among faint neighbourhoods."""
    x = torch.full((3 * len(ENDS), V), faint, device=DEV)
    for i, at in enumerate((0, V // 2, V - 1)):
        x[i::3, at] = 0.0
    check_all(x, [u for u in ENDS for _ in range(3)])


@pytest.mark.parametrize("none", [-float("inf"), NAN])
@pytest.mark.parametrize("V,S", [(5003, 16), (40000, 16), (40000, 64), (300000, 16)])
def test_places_without_anything(none, V, S):
    """Rows of which whole stretches, of thousands of logits and of 256, hold nothing that can be taken; a workspace that held other numbers."""
    x = torch.full((S, V), none, device=DEV)
    for i in range(S):
        x[i, (i * 2711) % V :: 997 if i % 2 else V] = float(i % 5)
        x[i, (i * 1301) % V] = 3.0
    u = [ENDS[i % len(ENDS)] if i < 8 else i / S for i in range(S)]
    tokens, lp = torch.full((S,), -9, dtype=torch.int32, device=DEV), torch.full((S,), 7.0, device=DEV)
    for fill in (0, 0x3f, 0xff):
        ws = torch.full((mq.moqe_sample_workspace_bytes(S, V),), fill, dtype=torch.uint8, device=DEV)
        mq.moqe_sample(x, torch.tensor(u, dtype=F32, device=DEV), tokens.fill_(-9), logprobs=lp, workspace=ws)
        torch.cuda.synchronize()
        rows, u32 = torch.where(x.isnan(), -float("inf"), x).double().cpu().numpy(), torch.tensor(u, dtype=F32).double().numpy()
        for s in range(S):
            check_token(rows[s], u32[s], int(tokens[s]), float(lp[s]))


@pytest.mark.parametrize("t", [F32, BF])
def test_a_confident_models_rows(t):
    """Normal logits and one winner far above them, by temperatures below 1, at both ends of u."""
    S, V = 96, 32000
    x = logits_of(S, V, F32, 2.0, 3)
    g = torch.Generator(device=DEV).manual_seed(7)
    x[torch.arange(S, device=DEV), torch.randint(0, V, (S,), generator=g, device=DEV)] = 30.0 + 1.5 * torch.randn(S, generator=g, device=DEV)
    check_all(x.to(t), [ENDS[i % len(ENDS)] for i in range(S)], T=[0.8] * S)


def test_a_generators_first_numbers():
    """u as Draw has it before any is given: zeros; every row gets a token of its own."""
    x = torch.full((4, 3000), -32.0, device=DEV)
    x[:, 2900] = 0.0
    tokens, lp, _ = run(x, [0.0] * 4)
    assert (tokens >= 0).all() and (tokens < 3000).all() and (lp <= 0).all()


@pytest.mark.parametrize("how", [{}, {"temperature": 0.7}, {"top_p": 0.9}, {"top_p": 0.999999, "temperature": 0.8}, {"top_k": 40, "top_p": 0.9}, {"top_k": 20000, "top_p": 0.97}, {"min_p": 1e-12},
                                 {"top_p": 0.5, "min_p": 0.001, "temperature": 1.3}])
@pytest.mark.parametrize("t", [F32, BF])
@pytest.mark.parametrize("sharp,above", [(2.5, 20.0), (1.0, 0.0), (6.0, 35.0)])
def test_a_row_draws_the_same_alone_and_in_a_batch(how, t, sharp, above):
    """A few rows and hundreds are divided differently over work-groups."""
    V, S = 32000, 130
    x = logits_of(S, V, F32, sharp, 21)
    x[:, 777] += above
    x = x.to(t)
    u = uniform(S, 5)
    u[:8] = ENDS
    many = run(x, u, **{k: [v] * S for k, v in how.items()})
    for at in (slice(0, 3), slice(3, 8), slice(60, 61), slice(100, 130)):
        few = run(x[at].contiguous(), u[at], **{k: [v] * (at.stop - at.start) for k, v in how.items()})
        assert np.array_equal(few[0], many[0][at]) and np.array_equal(few[1], many[1][at])


def kept(x, T, k, p, least, slack):
    """What the filters leave, with the borders of top-p and min-p moved by `slack` of the largest weight: outwards where it is positive."""
    w = np.exp((x - x.max()) / T)
    order = np.lexsort((np.arange(len(x)), -x))
    n = min(len(x), k) if k >= 1 else len(x)
    if p < 1:
        run = np.cumsum(w[order[:n]])
        n = max(1, int((run - w[order[:n]] < p * run[-1] + slack).sum()))
    keep = np.zeros(len(x), bool)
    keep[order[:n]] = True
    if least > 0:
        keep &= w >= min(least, 1.0) - slack
    keep[order[0]] = True
    return w * keep, keep


@pytest.mark.parametrize("t", [F32, BF])
@pytest.mark.parametrize("above", [0.0, 12.0, 28.0])
@pytest.mark.parametrize("V", [600, 40000])
def test_filters_at_the_ends_of_u(t, above, V):
    """Every row has a token of those that are kept, however near u or a border of the filters is to a choice."""
    how = [(1, 1.0, 0.0), (2, 0.9, 0.0), (50, 0.95, 0.01), (0, 0.9, 0.0), (0, 0.999999, 0.0), (0, 0.0, 0.0), (0, 1.0, 1.0), (0, 1.0, 1e-13), (V // 2, 1.0, 0.0), (V - 1, 0.5, 0.2)]
    S = len(how) * len(ENDS)
    x = logits_of(S, V, F32, 2.5, 31)
    x[:, V // 3] += above
    x = x.to(t)
    u, T = [ENDS[i // len(how)] for i in range(S)], [(0.6, 1.0, 1.4)[i % 3] for i in range(S)]
    tokens, lp, args = run(x, u, temperature=T, top_k=[how[i % len(how)][0] for i in range(S)], top_p=[how[i % len(how)][1] for i in range(S)], min_p=[how[i % len(how)][2] for i in range(S)])
    rows, u32, tol = x.double().cpu().numpy(), torch.tensor(u, dtype=F32).double().numpy(), V * 2.0 ** -40
    for s in range(S):
        settings = (args["temperature"][s], int(args["top_k"][s]), args["top_p"][s], args["min_p"][s])
        (few, sure), (many, may) = kept(rows[s], *settings, -tol), kept(rows[s], *settings, tol)
        end = min(max(u32[s], 0.0), 1.0) if u32[s] == u32[s] else 0.0
        at = tokens[s]
        assert 0 <= at < V and may[at], (settings, u[s], at)
        assert few[:at].sum() <= end * many.sum() + tol and many[: at + 1].sum() >= end * few.sum() - tol, (settings, u[s], at)
        most, least = math.log(many[at] / few.sum()), math.log(many[at] / many.sum())
        assert lp[s] <= 0 and least - 2.0 ** -24 * abs(least) - 2.0 ** -20 <= lp[s] <= most + 2.0 ** -24 * abs(most) + 2.0 ** -20, (settings, u[s], lp[s])


@pytest.mark.parametrize("t", [F32, BF])
def test_the_only_token_kept_has_log_probability_0(t):
    S, V = 64, 5003
    x, u = logits_of(S, V, t, 2.0, 2), uniform(S, 4)
    top = x.double().cpu().numpy().argmax(1)
    T = (0.3 + 0.05 * np.arange(S)).tolist()
    peaked = x.clone()
    peaked[torch.arange(S, device=DEV), torch.from_numpy(top).to(DEV)] = 40.0
    alone = torch.full_like(x, -float("inf"))
    alone[torch.arange(S, device=DEV), torch.from_numpy(top).to(DEV)] = x.amax(1)
    for logits, how in ((x, dict(top_k=[1] * S)), (x, dict(top_k=[1] * S, top_p=[0.9] * S, min_p=[0.1] * S)), (x.float() + torch.arange(V, device=DEV) * 1e-6, dict(min_p=[1.0] * S)),
                        (peaked, dict(top_p=[0.9] * S)), (peaked, dict(min_p=[0.5] * S)), (x, dict(top_p=[0.0] * S)), (alone, {}), (alone, dict(top_p=[0.9] * S))):
        best = logits.double().cpu().numpy().argmax(1)
        for temperature in ({}, {"temperature": T}):
            tokens, lp, _ = run(logits, u, **how, **temperature)
            assert np.array_equal(tokens, best) and (lp == 0).all(), (how.keys(), lp[lp != 0][:4])


@pytest.mark.parametrize("gap", [1e-3, 0.1, 1.0, 5.0, 10.0, 20.0, 30.0, 60.0])
def test_log_probabilities_are_at_most_0(gap):
    """Two tokens, and two above faint ones: next to 0 the log probability is as near as the sums' units let it be, 2^-40, and never above."""
    S, V = 40, 4000
    for rest in (-float("inf"), -60.0):
        x = torch.full((S, V), rest, device=DEV)
        x[:, 5] = torch.linspace(-3.0, 17.0, S, device=DEV)
        x[:, 3005] = x[:, 5] - gap
        u = uniform(S, 8)
        for how in ({}, {"top_k": [2] * S}):
            tokens, lp, _ = run(x, u, **how)
            v = x.double().cpu().numpy()
            for s in range(S):
                w = np.exp(v[s] - v[s].max())
                want = math.log(w[tokens[s]] / w.sum())
                assert tokens[s] in (5, 3005) and lp[s] <= 0 and abs(lp[s] - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -40, (rest, how, lp[s], want)
