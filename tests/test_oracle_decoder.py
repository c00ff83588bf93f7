"""The oracle of the decoder layer's operators, pinned against torch's own and against values worked by hand."""
import math

import numpy as np
import torch

from oracle import decoder_oracle as do


def test_e4m3_values_and_codes_agree_with_torch():
    codes = np.arange(256, dtype=np.uint8)
    mine, theirs = do.e4m3_value(codes), torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(mine), np.isnan(theirs)) and np.array_equal(mine[~np.isnan(mine)], theirs[~np.isnan(theirs)])
    v = np.sort(theirs[np.isfinite(theirs)])
    x = np.concatenate([v, (v[:-1] + v[1:]) / 2, (v[:-1] + v[1:]) / 2 * (1 + 1e-6), np.random.default_rng(0).normal(0, 30, 20000)])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = do.e4m3_code(x)
    same = (got == want) | ((x == 0) & (got & 127 == 0) & (want & 127 == 0))
    assert same.all()
    assert do.e4m3_code(np.array([np.inf, -np.inf, 1e9])).tolist() == [0x7e, 0xfe, 0x7e] and do.e4m3_code(np.array([np.nan]))[0] == 0x7f


def test_scales_are_the_smallest_powers_of_two():
    for a in (448.0, 448.0 * (1 + 2 ** -20), 447.9, 1.0, 1.75, 1.7500001, 3e-5, 1e30):
        s = do.scale_for(a)
        assert math.log2(s) == int(math.log2(s)) and a <= 448 * s and a > 448 * s / 2
    assert do.scale_for(0.0) == 2.0 ** -120 and do.scale_for(1e-40) == 2.0 ** -120 and do.scale_for(1e39) == 2.0 ** 120


def test_places_are_a_bijection():
    for dh in (64, 128, 256):
        for bt in (32, 64, 128):
            c = do.Cache(1, 1, bt, dh)
            for which in ("k", "v"):
                assert np.array_equal(np.sort(c.at[which].ravel()), np.arange(bt * dh))


def test_norms_agree_with_torch():
    rng = np.random.default_rng(1)
    x, g, o = rng.normal(size=(5, 37)), rng.normal(size=37), rng.normal(size=37)
    t = torch.from_numpy
    assert np.allclose(do.norm(x, "layer", 1e-5, g, o), torch.nn.functional.layer_norm(t(x), (37,), t(g), t(o), 1e-5).numpy(), atol=1e-12)
    assert np.allclose(do.norm(x, "rms", 1e-5, g), torch.nn.functional.rms_norm(t(x), (37,), t(g), 1e-5).numpy(), atol=1e-12)


def test_rotation_keeps_lengths_and_depends_on_distance_only():
    rng = np.random.default_rng(2)
    q, k, f = rng.normal(size=64), rng.normal(size=64), 10000.0 ** (-2 * np.arange(24) / 48)
    for inter in (False, True):
        a = do.rotated(q, 11, f, 48, inter) @ do.rotated(k, 4, f, 48, inter)
        b = do.rotated(q, 100007, f, 48, inter) @ do.rotated(k, 100000, f, 48, inter)
        assert abs(a - b) < 1e-8 and abs(np.linalg.norm(do.rotated(q, 9, f, 48, inter)) - np.linalg.norm(q)) < 1e-12
        assert np.array_equal(do.rotated(q, 9, f, 48, inter)[48:], q[48:])
    x = np.zeros(64)
    x[1] = 1.0
    assert do.rotated(x, 1, [0.0, math.pi / 2] + [0.0] * 22, 48, False)[1 + 24] == 1.0       # pair 1 of the half layout: dims 1 and 25


def test_attention_agrees_with_torch_on_a_growing_sequence():
    rng = np.random.default_rng(3)
    H, G, dh, bt, L, n = 2, 3, 64, 32, 75, 11
    cache, table = do.Cache(5, H, bt, dh, fill=0x7f), np.array([[4, 1, 2, -1]])
    qkv = rng.normal(size=(L, (H * G + 2 * H) * dh))
    f = 10000.0 ** (-2 * np.arange(32) / 64)
    for lo, hi in ((0, 40), (40, 41), (41, 64), (64, L)):
        do.kv_append(qkv[lo:hi], H * G, cache, table, [(0, hi - lo, hi)], hi - lo, f, 64)
    K, V = (np.concatenate([np.stack([cache.read(m, b, h) for h in range(H)], 1) for b in (4, 1, 2)])[:L] for m in ("k", "v"))
    x = qkv.reshape(L, -1, dh)
    true_k = np.stack([do.rotated(x[p, H * G:H * G + H], p, f, 64, False) for p in range(L)])
    assert np.abs(V - x[:, H * G + H:]).max() < 0.3 and np.linalg.norm(K - true_k) < 0.04 * np.linalg.norm(true_k)
    q = rng.normal(size=(n, H * G, dh))
    got, _ = do.kv_attention(q, H * G, cache, table, [(0, n, L)], n, dh ** -0.5, window=30, prefix=[7])
    p, t = np.arange(L - n, L)[:, None], np.arange(L)
    mask = (t < 7) | ((t <= p) & (p - t < 30))
    rep = lambda a: torch.from_numpy(a).transpose(0, 1).repeat_interleave(G, 0)
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1), rep(K), rep(V), torch.from_numpy(mask))
    assert np.allclose(got, want.transpose(0, 1).numpy(), atol=1e-12)


def test_a_growing_scale_moves_earlier_codes_by_powers_of_two():
    cache = do.Cache(1, 1, 32, 64)
    a = np.full((3, 64), 1.25)
    cache.write("v", 0, 0, 0, a, False)
    assert cache.v_scale[0, 0] == 2.0 ** -8 and np.array_equal(cache.read("v", 0, 0)[:3], a)
    cache.write("v", 0, 0, 3, np.full((2, 64), 300.0), True)
    assert cache.v_scale[0, 0] == 1.0 and np.array_equal(cache.read("v", 0, 0)[:3], a)
    assert cache.read("v", 0, 0)[3, 0] in (288.0, 320.0)                     # 300 lies between two codes
    cache.write("v", 0, 0, 5, np.full((1, 64), 0.01), True)                  # a small one keeps the scale
    assert cache.v_scale[0, 0] == 1.0 and cache.read("v", 0, 0)[5, 0] == 0.009765625
