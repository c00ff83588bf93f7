"""The decoder in 8-bit floating point on the GPU, from tokens to tokens: stages of a layer against the oracle, each on what the GPU gave it, tokens against the oracle's from the GPU's own
logits, graphs against eager runs.

Tolerances: as in the operators' own tests; where an e4m3 rounding between two stages may fall on the other side, the next stage is checked on the GPU's own rows."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from oracle import f8_oracle as fo
from paper_2508_09204_amd import binding as mq
from paper_2508_09204_amd import decoder as dec
from paper_2508_09204_amd import experts as ex
from tests.test_gpu_f8 import check_product, check_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def f64(t):
    return t.detach().double().cpu().numpy()


def _model(layers=1, d=256, f=384, heads=4, kv=2, dh=64, K=3, V=1000, seed=0):
    return dec.synthetic(layers, d, f, heads, kv, dh, K, seed=seed, vocabulary=V, head_norms=True)


def _values(mat):
    rows = [mq.F8Rows.empty(mat.n, mat.k, DEV) for _ in range(2 if mat.gated else 1)]
    mq.moqe_f8_unpack(mat, *rows)
    return [f64(r.float()) for r in rows]


@pytest.mark.parametrize("T", [1, 30])
def test_stages_of_a_layer(T):
    S, d = 5, 256
    model = _model(seed=T)
    seqs = dec.Sequences(model, S, 64, 32, DEV)
    x = torch.randn((S * T, d), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
    seqs.route(model, x.to(BF), T)
    step = dec.Step(model, seqs, T)
    step.x.copy_(x)
    layer = model.layers[0]
    # the first norm and projection, stopped before the buffers are used again
    step._calls[0]()
    step._calls[1]()
    torch.cuda.synchronize()
    want = do.norm(f64(x), "rms", 1e-6, f64(layer.attn_norm.gain))
    check_rows(step.normed8, want, 2.0 ** -18 * np.abs(want).max(1, keepdims=True))
    check_product(step.qkv, f64(step.normed8.float()), _values(layer.qkv[0])[0], None, BF)
    step()
    torch.cuda.synchronize()
    att = f64(step.att)
    codes, scales = fo.quantize_rows(att)
    assert np.array_equal(step.att8.codes.cpu().numpy(), codes) and np.array_equal(step.att8.scales[:, : scales.shape[1]].cpu().numpy(), scales)
    # MLP: rows of each sequence on its own expert
    e = seqs.expert_idx.cpu().numpy()
    h_in, h = f64(step.normed8.float()), f64(step.h8.float())
    for s in range(S):
        at = slice(s * T, (s + 1) * T)
        gate, up = _values(layer.mlp.gate_up[e[s]])
        check_product(mq.F8Rows(step.h8.codes[at], step.h8.scales[at], T, step.h8.d), h_in[at], gate, up, "f8", fast=layer.mlp.fast)
        check_product(step.y16[at], h[at], _values(layer.mlp.down[e[s]])[0], None, BF)
    want = do.norm(f64(step.x), "rms", 1e-6, f64(model.final_norm.gain))
    near = 2.0 ** -18 * np.abs(want).max(1, keepdims=True)
    check_rows(step.out8, want, near)
    assert (np.abs(f64(step.out) - want) <= near + 2.0 ** -8 * np.abs(want)).all()


def _how(S):
    full = lambda v, t=torch.float32: torch.full((S,), v, dtype=t, device=DEV)
    return dict(temperature=full(0.9), top_k=full(200, torch.int32), top_p=full(0.9), min_p=full(0.01))


def _uniform(n, S):
    return torch.rand((n, S), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)


def test_tokens_are_drawn_from_the_heads_logits():
    S, T, V = 4, 9, 1000
    model = _model(layers=2, V=V, seed=3)
    g = dec.Generator(model, S, T, 8, 32, **_how(S))
    prompt = torch.randint(0, V, (S, T), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    u = _uniform(9, S)
    head = _values(model.head)[0]
    for i in range(6):
        tokens = g.start(prompt, u[0]) if i == 0 else g.next(u[i])
        torch.cuda.synchronize()
        draw, step = (g.first, g.prompt) if i == 0 else (g.draw, g.token)
        last = f64(step.out8.float()).reshape(S, -1, 256)[:, -1]
        check_product(draw.logits, last, head, None, torch.float32)
        logits = f64(draw.logits)
        for s in range(S):
            want, lp, gap = fo.sample(logits[s], float(u[i, s]), float(np.float32(0.9)), 200, float(np.float32(0.9)), float(np.float32(0.01)))
            assert gap > V * 2.0 ** -40 and int(tokens[s]) == want and abs(float(draw.logprobs[s]) - lp) <= 2.0 ** -20 * (1 + abs(lp))
    assert (g.seqs.kv_len == T + 5).all() and g.seqs.tokens == T + 5


def test_a_replayed_generator_is_the_eager_one():
    """Tokens, log probabilities and rows of a generator that replays its graph, with other work between, against one whose steps are enqueued each time; two generators at once on streams of
    their own."""
    S, T, V, n = 3, 20, 777, 7
    model = _model(layers=2, V=V, seed=4)
    prompt = torch.randint(0, V, (S, T), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    u = _uniform(n + 1, S)
    eager = dec.Generator(model, S, T, n, 32, **_how(S))
    want = [eager.start(prompt, u[0]).clone()]
    for i in range(n):
        eager.draw.u.copy_(u[1 + i])
        eager.seqs.tokens += 1
        eager._enqueue()
        want.append(torch.stack([eager.draw.tokens.float(), eager.draw.logprobs]).clone())
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        eager.next(u[0])
    pair = [dec.Generator(model, S, T, n, 32, **_how(S)) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in pair]
    got = [[] for _ in pair]
    for i in range(n + 1):
        for k, g in enumerate(pair):
            if i > 1:
                streams[k].wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(streams[k]):
                    g.next(u[i])
                    got[k].append(torch.stack([g.draw.tokens.float(), g.draw.logprobs]))
            else:                                                      # captures and first launches one after the other
                (g.start(prompt, u[0]) if i == 0 else g.next(u[i]))
                got[k].append(g.draw.tokens.clone() if i == 0 else torch.stack([g.draw.tokens.float(), g.draw.logprobs]).clone())
                torch.cuda.synchronize()
        torch.randn(5000, device=DEV).sum()
    torch.cuda.synchronize()
    for mine in got:
        assert all(torch.equal(a, b) for a, b in zip(want, mine))


def test_integer_and_8_bit_matrices_in_one_layer():
    """Projections and MLP of either kind, shared or by expert, go together: one step of each mixture is finite and near the same in all roundings' sense."""
    S, T, d, heads, kv, dh, f = 6, 16, 256, 4, 2, 64, 384
    g = torch.Generator(device=DEV).manual_seed(6)
    rand = lambda n, k: torch.randn((n, k), generator=g, device=DEV) * k ** -0.5
    w = {"qkv": rand((heads + 2 * kv) * dh, d), "out": rand(d, heads * dh), "gate": rand(f, d), "up": rand(f, d), "down": rand(d, f)}
    router = mq.Router(None, None, torch.randn((2, d), generator=g, device=DEV), None, d, 0, 2)
    ints = lambda n: [ex.quantize_and_pack(w[n], 8, 0, True) for _ in range(2)]
    norm = lambda: mq.Norm("rms", 1e-6, torch.ones(d, device=DEV))
    x = torch.randn((S * T, d), generator=g, device=DEV)
    outs = []
    for qkv8, out8, mlp8 in ((0, 0, 0), (1, 0, 0), (0, 2, 0), (0, 0, 1), (1, 2, 1), (2, 1, 2)):
        f8 = lambda n, k: [ex.quantize_f8(w[n])] * k
        layer = dec.Layer(norm(), f8("qkv", qkv8) if qkv8 else ints("qkv"), f8("out", out8) if out8 else ints("out"), norm(),
                          dec.F8Mlp([ex.quantize_f8(w["gate"], w["up"])] * mlp8, f8("down", mlp8)) if mlp8 else
                          mq.Block(kind=mq.KIND_SILU_MLP, router=router, w0=ints("gate"), w1=ints("up"), w2=ints("down")))
        model = dec.Decoder([layer, layer], norm(), router, mq.Rope(dec.rope_frequencies(dh, device=DEV), dh), heads, kv, dh, residual_scale=0.5)
        seqs = dec.Sequences(model, S, 32, 32, DEV)
        seqs.route(model, x.to(BF), T)
        step = dec.Step(model, seqs, T)
        step.x.copy_(x)
        outs.append(step().double().clone())
    torch.cuda.synchronize()
    for o in outs[1:]:
        err = (o - outs[0]).pow(2).mean().sqrt() / outs[0].pow(2).mean().sqrt()
        # e4m3 rounds by 2^-4 / sqrt(3) = 0.036 of a value at most in the mean square, for both operands of three products in a row and two layers: 0.036 * sqrt(12)
        assert o.isfinite().all() and float(err) < 0.036 * 12 ** 0.5


def test_a_sequence_without_a_token_goes_on():
    """Token -1 (a row of logits that are all NaN or minus infinity) is looked up as token 0, in the first launch and in the replayed graph; the other sequences see nothing of it."""
    S, T, V, n = 3, 5, 500, 4
    model = _model(layers=1, V=V, seed=9)
    prompt = torch.randint(0, V, (S, T), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    u = _uniform(n + 1, S)
    seen = []
    for none in (-1, 0):
        g = dec.Generator(model, S, T, n, 32, **_how(S))
        g.start(prompt, u[0])
        got = []
        for i in range(n):
            g.draw.tokens[1] = none
            got.append(torch.cat([g.next(u[1 + i]).float(), g.draw.logprobs]))
        torch.cuda.synchronize()
        seen.append(torch.stack(got))
    assert torch.equal(*seen)
    with pytest.raises(ValueError, match="tokens"):
        g.start(prompt[:, 1:], u[0])
    with pytest.raises(ValueError, match="tokens"):
        g.start(prompt + V, u[0])
