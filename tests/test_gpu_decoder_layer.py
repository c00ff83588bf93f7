"""The decoder of decoder.py on the GPU: its operators together against the oracle, prompts against single tokens, graphs.

Tolerances: a layer's buffers are compared stage by stage, each on what the GPU gave the stage, with the stage's own roundings (as in the operators' tests, and
2e-3 for the grouped products).  Where a bf16 rounding between two stages may fall on the other side, 2^-8 of the stage's input goes through the next product."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do
from oracle import moqe_oracle as oc
from paper_2508_09204_amd import binding as mq
from paper_2508_09204_amd import decoder as dec
from tests import oracle_blocks as ob

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def f64(t):
    return t.detach().double().cpu().numpy()


def _experts(rng, n, k):
    from tests import gpu_blocks as gb
    w = (rng.normal(size=(n, k)) * k ** -0.5).astype(np.float32)
    host = [oc.quantize(w, *spec) for spec in ((4, 128, False, 1.0, 0), (8, 0, True, 1.0, 0), (3, 64, False, 1.0, 0))]
    return host, [gb.packed_dev(q) for q in host]


def _model(layers, d=256, f=384, heads=4, kv=2, dh=64, cap=0.0, window=0, seed=0):
    rng = np.random.default_rng(seed)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    gain = lambda n: (1.0 + 0.1 * rng.normal(size=n)).astype(np.float32)
    router = mq.Router(None, None, dev((rng.normal(size=(3, d)) * 0.3).astype(np.float32)), None, d, 0, 3)
    host, made = [], []
    for _ in range(layers):
        h = {"attn_norm": gain(d), "mlp_norm": gain(d)}
        m = {}
        for name, n, k in (("qkv", (heads + 2 * kv) * dh, d), ("out", d, heads * dh), ("gate", f, d), ("up", f, d), ("down", d, f)):
            h[name], m[name] = _experts(rng, n, k)
        made.append(dec.Layer(mq.Norm("rms", 1e-6, dev(h["attn_norm"])), m["qkv"], m["out"], mq.Norm("rms", 1e-6, dev(h["mlp_norm"])),
                              mq.Block(kind=mq.KIND_SILU_MLP, router=router, w0=m["gate"], w1=m["up"], w2=m["down"])))
        host.append(h)
    final = gain(d)
    rope = mq.Rope(dec.rope_frequencies(dh, 1000.0, device=DEV), dh, q_gain=dev(gain(dh)), k_gain=dev(gain(dh)))
    return dec.Decoder(made, mq.Norm("rms", 1e-6, dev(final)), router, rope, heads, kv, dh, cap, window, 0.5), host, final


def _cache_of(c, S):
    o = do.Cache(c.k_scale.shape[0], c.k_scale.shape[1], c.block_tokens, c.head_dim)
    o.k, o.v, o.k_scale, o.v_scale = c.k.cpu().numpy().copy(), c.v.cpu().numpy().copy(), f64(c.k_scale), f64(c.v_scale)
    return o


@pytest.mark.parametrize("T,cap,window", [(37, 0.0, 0), (70, 20.0, 30), (1, 0.0, 0)])
def test_one_layer_stage_by_stage(T, cap, window):
    S, d, heads, kv, dh = 5, 256, 4, 2, 64
    model, host, final = _model(1, cap=cap, window=window, seed=T)
    seqs = dec.Sequences(model, S, 150, 32, DEV)
    x0 = torch.randn((S * 60, d), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
    seqs.route(model, x0.bfloat16(), 60)
    warm = dec.Step(model, seqs, 60)
    warm.x.copy_(x0)
    warm()                                                       # 60 tokens are in the cache already
    step = dec.Step(model, seqs, T)
    x = torch.randn((S * T, d), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV)
    step.x.copy_(x)
    torch.cuda.synchronize()
    before = _cache_of(seqs.caches[0], S)
    out = step()
    torch.cuda.synchronize()
    e = seqs.expert_idx.cpu().numpy()
    h, layer = host[0], model.layers[0]
    ref_idx = oc.bucket(e, 3)
    assert np.array_equal(seqs.perm.cpu().numpy(), ref_idx[2]) and (seqs.kv_len.cpu().numpy() == 60 + T).all()
    by_expert = lambda rows, mats: np.concatenate([oc.qlinear(rows[s * T:(s + 1) * T], mats[e[s]]) for s in range(S)])
    round16 = lambda a: f64(torch.from_numpy(a).to(torch.bfloat16))
    # norm and fused projection
    n0 = round16(do.norm(f64(x), "rms", 1e-6, h["attn_norm"]))
    want = by_expert(n0, h["qkv"])
    got = f64(step.qkv)
    rms = np.sqrt((want * want).mean())
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (2e-3 + 2.0 ** -8) * rms).all()
    # positions and cache
    seq = do.sequences(S, T, S * T, seqs.kv_len.cpu().numpy(), seqs.block_table.shape[1], 32)
    table = seqs.block_table.cpu().numpy()
    q = do.kv_append(got, heads, before, table, seq, T, f64(model.rope.inv_freq), dh, False, 1.0, f64(model.rope.q_gain), f64(model.rope.k_gain), 1e-6)
    after = _cache_of(seqs.caches[0], S)
    assert np.array_equal(after.k_scale, before.k_scale) and np.array_equal(after.v_scale, before.v_scale)
    size = np.abs(f64(model.rope.q_gain)).max() * dh ** 0.5
    q = q.reshape(S * T, -1)
    assert (np.abs(f64(step.q) - q) <= 2.0 ** -8 * np.abs(q) + 2.0 ** -19 * 2.5 * size).all()
    # attention over the GPU's own cache
    att, of = do.kv_attention(f64(step.q), heads, after, table, seq, T, dh ** -0.5, cap, window)
    att, of = att.reshape(S * T, -1), of.reshape(S * T, -1)
    assert (np.abs(f64(step.att) - att) <= 2.0 ** -8 * np.abs(att) + (2.0 ** -8 + 2.0 ** -12) * of).all()
    # output projection, residual, MLP, residual, final norm
    t1 = f64(x) + 0.5 * by_expert(f64(step.att), h["out"])
    n1 = round16(do.norm(t1, "rms", 1e-6, h["mlp_norm"]))
    y2 = np.concatenate([oc.silu_mlp(n1[s * T:(s + 1) * T], h["gate"][e[s]], h["up"][e[s]], h["down"][e[s]])[0] for s in range(S)])
    t2 = t1 + 0.5 * y2
    rms = np.sqrt((y2 * y2).mean())
    assert (np.abs(f64(step.x) - t2) <= 0.5 * (2e-3 * np.abs(y2) + 4 * 2.0 ** -8 * rms) + 2e-3 * np.abs(t1 - f64(x)) + 1e-3).all()
    o = do.norm(f64(step.x), "rms", 1e-6, final)
    assert (np.abs(f64(out) - o) <= 2.0 ** -8 * np.abs(o) + 2.0 ** -18 * np.abs(o).max(1, keepdims=True)).all()


def test_single_tokens_follow_a_prompt_as_one_prompt_would():
    """Two layers: 48 tokens at once, against 40 and then eight single ones.  Scales end up the same; what differs are codes that were rounded to a smaller scale first, and
    roundings to bf16 between the stages: less than 3 % of the rows' size."""
    S, d = 4, 256
    model, _, _ = _model(2, seed=9)
    x = torch.randn((S, 48, d), generator=torch.Generator(device=DEV).manual_seed(7), device=DEV)
    a, b = dec.Sequences(model, S, 64, 32, DEV), dec.Sequences(model, S, 64, 32, DEV)
    for s in (a, b):
        s.route(model, x.bfloat16().view(S * 48, d), 48)
    whole = dec.Step(model, a, 48)
    whole.x.copy_(x.view(S * 48, d))
    want = whole().view(S, 48, d).double()
    prompt, token = dec.Step(model, b, 40), dec.Step(model, b, 1)
    prompt.x.copy_(x[:, :40].reshape(S * 40, d))
    got = [prompt().view(S, 40, d).double()]
    for t in range(40, 48):
        token.x.copy_(x[:, t])
        got.append(token().view(S, 1, d).double())
    got = torch.cat(got, 1)
    torch.cuda.synchronize()
    assert torch.equal(a.expert_idx, b.expert_idx) and torch.equal(a.kv_len, b.kv_len)
    err = (got - want).pow(2).mean(-1).sqrt() / want.pow(2).mean(-1).sqrt()
    assert float(err.max()) < 0.03


def test_a_captured_step_is_the_step():
    """Replays with eager work between them give the eager results bit for bit, every time."""
    S, d = 3, 256
    model, _, _ = _model(2, seed=11)
    x = torch.randn((6, S, d), generator=torch.Generator(device=DEV).manual_seed(8), device=DEV)
    results = []
    for captured in (False, True):
        seqs = dec.Sequences(model, S, 40, 32, DEV)
        seqs.route(model, x.bfloat16().view(6 * S, d)[:S], 1)
        step = dec.Step(model, seqs, 1)
        got = []
        for t in range(6):
            if captured and t == 1:
                step.capture()
            step.x.copy_(x[t])
            got.append((step().clone(), step.att.clone(), step.x.clone()))
            torch.cuda.synchronize()
        results.append(got)
    for eager, replayed in zip(*results):
        assert all(torch.equal(u, v) for u, v in zip(eager, replayed))
