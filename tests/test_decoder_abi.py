"""The decoder layer's entry points without a GPU: refusals (dry-run mode: nothing is enqueued), the cache's places, scales and steps of
csrc/kv_cache.h compiled for the host, and what the binding checks of its tensors."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import decoder_oracle as do

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # a non-NULL, 256-byte aligned address; never dereferenced in dry-run mode


@pytest.fixture(scope="module")
def mq():
    from paper_2508_09204_amd import binding
    binding.moqe_set_dry_run(True)
    yield binding
    binding.moqe_set_dry_run(False)


def _step(mq, **kw):
    s = mq._ResidualStep()
    s.y = s.residual = s.residual_out = s.out = s.gate = FAKE
    s.y_stride = s.residual_stride = s.residual_out_stride = s.out_stride = 64
    s.post, s.pre = mq._Norm(FAKE, None, 1, 1e-5), mq._Norm(FAKE, FAKE, 2, 1e-5)
    s.M, s.d, s.y_type, s.residual_type, s.gate_rows, s.scale = 4, 64, 0, 1, 0, 1.0
    for k, v in kw.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("change,code", [
    ({}, 0), ({"M": 0, "residual": None}, 0), ({"y": None}, 0), ({"out": None}, 0), ({"residual_out": None}, 0), ({"gate": None}, 0),
    ({"d": 0}, -2), ({"d": 32769}, -2), ({"M": -1}, -2), ({"y_type": 2}, -3), ({"residual_type": -1}, -3), ({"gate_rows": -1}, -2),
    ({"residual": None}, -1), ({"residual_out": None, "out": None}, -1), ({"y_stride": 63}, -2), ({"out_stride": 8}, -2),
    ({"residual_out_stride": 72, "residual": FAKE}, -2), ({"y": FAKE + 2}, -2), ({"residual": FAKE + 1}, -2), ({"gate": FAKE + 2}, -2),
])
def test_residual_norm_refusals(mq, change, code):
    s = _step(mq, **change)
    assert mq.lib.moqe_residual_norm(C.byref(s), None) == code


def test_residual_norm_refuses_norms(mq):
    call = lambda **kw: mq.lib.moqe_residual_norm(C.byref(_step(mq, **kw)), None)
    assert call(pre=mq._Norm(FAKE, None, 3, 1e-5)) == -3 and call(post=mq._Norm(FAKE, None, -1, 1e-5)) == -3
    assert call(pre=mq._Norm(FAKE, None, 1, -1.0)) == -2 and call(pre=mq._Norm(FAKE, None, 1, float("nan"))) == -2
    assert call(pre=mq._Norm(FAKE, FAKE, 1, 0.0)) == -3                     # an offset belongs to layer norms
    assert call(pre=mq._Norm(FAKE + 2, None, 1, 0.0)) == -2 and call(pre=mq._Norm(None, None, 1, 0.0)) == 0
    assert mq.lib.moqe_residual_norm(None, None) == -1


def _parts(mq, cache={}, batch={}, rope={}, attn={}):
    c = mq._KvCache(FAKE, FAKE, FAKE, FAKE, 10, 64, 4, 128)
    b = mq._KvBatch(FAKE, FAKE, FAKE, 3, 5, 11, 20)
    r = mq._Rope(FAKE, None, None, 1e-6, 1.0, 128, 0)
    a = mq._Attention(None, None, 0.1, 0.0, 28, 0)
    for o, kw in ((c, cache), (b, batch), (r, rope), (a, attn)):
        for k, v in kw.items():
            setattr(o, k, v)
    return c, b, r, a


def _append(mq, qkv=FAKE, typ=1, stride=36 * 128, heads=28, q=FAKE, q_stride=28 * 128, **kw):
    c, b, r, _ = _parts(mq, **kw)
    return mq.lib.moqe_kv_append(qkv, typ, stride, heads, C.byref(r), C.byref(b), C.byref(c), q, q_stride, None)


def _attend(mq, q=FAKE, stride=28 * 128, out=FAKE, out_stride=28 * 128, ws=FAKE, short=0, **kw):
    c, b, _, a = _parts(mq, **kw)
    need = mq.lib.moqe_kv_attention_workspace_bytes(C.byref(a), C.byref(b), C.byref(c))
    return mq.lib.moqe_kv_attention(q, stride, C.byref(a), C.byref(b), C.byref(c), out, out_stride, ws, max(0, need - short), None)


CACHE_BATCH = [
    ({"cache": {"head_dim": 96}}, -2), ({"cache": {"block_tokens": 48}}, -2), ({"cache": {"n_blocks": 0}}, -2), ({"cache": {"n_heads": 0}}, -2),
    ({"cache": {"n_heads": 3}}, -2), ({"cache": {"k": None}}, -1), ({"cache": {"v_scale": None}}, -1), ({"cache": {"v": FAKE + 8}}, -2),
    ({"cache": {"k_scale": FAKE + 2}}, -2), ({"batch": {"S": -1}}, -2), ({"batch": {"T": 0}}, -2), ({"batch": {"M": -1}}, -2),
    ({"batch": {"table_width": 0}}, -2), ({"batch": {"table_width": 1 << 25}}, -2), ({"batch": {"block_table": None}}, -1),
    ({"batch": {"kv_len": None}}, -1), ({"batch": {"cu_rows": None}}, -2), ({"batch": {"cu_rows": None, "M": 15}}, 0),
    ({"batch": {"cu_rows": FAKE + 2}}, -2), ({"batch": {"S": 1 << 20, "T": 1 << 12}}, -2), ({"batch": {"S": 0, "block_table": None, "kv_len": None}}, 0),
    ({"batch": {"M": 0}}, 0), ({}, 0),
]


@pytest.mark.parametrize("kw,code", CACHE_BATCH + [
    ({"typ": 2}, -3), ({"qkv": None}, -1), ({"q": None}, -1), ({"qkv": FAKE + 8}, -2), ({"stride": 36 * 128 - 8}, -2), ({"stride": 36 * 128 + 4}, -2),
    ({"q_stride": 27 * 128}, -2), ({"heads": 30}, -2), ({"heads": 0}, -2), ({"rope": {"rot_dim": 8}}, -2), ({"rope": {"rot_dim": 144}}, -2),
    ({"rope": {"rot_dim": -16}}, -2), ({"rope": {"inv_freq": None}}, -1), ({"rope": {"inv_freq": None, "rot_dim": 0}}, 0), ({"rope": {"inv_freq": FAKE + 4}}, -2),
    ({"rope": {"q_gain": FAKE, "eps": -1.0}}, -2), ({"rope": {"k_gain": FAKE + 1}}, -2),
])
def test_append_refusals(mq, kw, code):
    assert _append(mq, **kw) == code


@pytest.mark.parametrize("kw,code", CACHE_BATCH + [
    ({"q": None}, -1), ({"out": None}, -1), ({"out": FAKE + 2}, -2), ({"stride": 100}, -2), ({"out_stride": 28 * 128 + 2}, -2), ({"attn": {"n_heads": 27}}, -2),
    ({"attn": {"cap": -1.0}}, -2), ({"attn": {"cap": float("nan")}}, -2), ({"attn": {"scale": float("nan")}}, -2), ({"attn": {"slopes": FAKE + 1}}, -2),
    ({"attn": {"prefix": FAKE + 2}}, -2), ({"attn": {"slopes": FAKE, "prefix": FAKE, "window": 5, "cap": 3.0}}, 0),
    ({"ws": None}, -4), ({"ws": FAKE + 8}, -4), ({"short": 1}, -4),
])
def test_attention_refusals(mq, kw, code):
    assert _attend(mq, **kw) == code
    if code:
        assert mq.lib.moqe_last_error_string().startswith(b"moqe_kv_attention")


def test_descriptors_that_are_missing(mq):
    c, b, r, a = (C.byref(x) for x in _parts(mq))
    lib = mq.lib
    assert lib.moqe_kv_append(FAKE, 1, 4608, 28, None, b, c, FAKE, 3584, None) == -1
    assert lib.moqe_kv_append(FAKE, 1, 4608, 28, r, None, c, FAKE, 3584, None) == -1
    assert lib.moqe_kv_append(FAKE, 1, 4608, 28, r, b, None, FAKE, 3584, None) == -1
    for bad in ((None, b, c), (a, None, c), (a, b, None)):
        assert lib.moqe_kv_attention(FAKE, 3584, *bad, FAKE, 3584, FAKE, 1 << 30, None) == -1
        assert lib.moqe_kv_attention_workspace_bytes(*bad) == 0
    assert lib.moqe_kv_codes_bytes(c) == 10 * 4 * 64 * 128 and lib.moqe_kv_codes_bytes(None) == 0


def test_many_rows_and_short_contexts_need_no_workspace(mq):
    def need(**kw):
        c, b, _, a = _parts(mq, **kw)
        return mq.lib.moqe_kv_attention_workspace_bytes(C.byref(a), C.byref(b), C.byref(c))
    assert need() > 0 and need(batch={"T": 1}) > 0
    assert need(batch={"T": 1, "table_width": 4}) == 0                     # a sequence is one chunk


def test_binding_checks_tensors(mq):
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)
    bf, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
    with pytest.raises(TypeError):
        mq.ResidualNormCall(z(2, 8, t=torch.float16), z(2, 8), z(2, 8, t=bf))
    with pytest.raises(ValueError):
        mq.ResidualNormCall(z(2, 7), z(2, 8), z(2, 8, t=bf))
    with pytest.raises(TypeError):
        mq.ResidualNormCall(z(2, 8), z(2, 8), z(2, 8))
    with pytest.raises(ValueError):
        mq.ResidualNormCall(z(2, 8), z(2, 8), z(2, 8, t=bf), gate=z(8), gate_rows=1)
    with pytest.raises(ValueError):
        mq.ResidualNormCall(z(8, 2).t(), z(2, 8), z(2, 8, t=bf))               # rows are not dense
    with pytest.raises(ValueError):
        mq.ResidualNormCall(z(2, 8), z(2, 8), z(2, 8, t=bf), pre=mq.Norm("rms", 1e-5, z(4)))
    mq.ResidualNormCall(z(2, 16)[:, :8], z(2, 8), z(2, 8, t=bf))
    cache = mq.KvCache.empty(3, 2, 32, 64, "cpu")
    batch = mq.KvBatch(z(2, 4, t=i32), z(2, t=i32), 2, 1, 2)
    attn = mq.Attention(4, 0.1)
    mq.KvAttentionCall(z(2, 256, t=bf), attn, batch, cache, z(2, 4, 64, t=bf))
    with pytest.raises(ValueError):
        mq.KvAttentionCall(z(2, 128, t=bf), attn, batch, cache, z(2, 256, t=bf))
    with pytest.raises(ValueError):
        mq.KvAttentionCall(z(2, 256, t=bf), mq.Attention(4, 0.1, slopes=z(3)), batch, cache, z(2, 256, t=bf))
    with pytest.raises(ValueError):
        mq.KvBatch(z(2, 4, t=torch.int64), z(2, t=i32), 2, 1, 2).c()
    with pytest.raises(ValueError):
        mq.KvCache(cache.k[:2], cache.v, cache.k_scale, cache.v_scale, 32, 64).c()
    with pytest.raises(ValueError):
        mq.KvAppendCall(z(2, 512), 4, mq.Rope(z(32), 64), batch, cache, z(2, 256, t=bf))          # inv_freq is float64


PROBE = r'''
#include "kv_cache.h"
#include <cstdio>
#include <cstring>
#include <cstdlib>
#include <cmath>
using namespace moqe;
int main(int argc, char** argv) {
  if (!strcmp(argv[1], "at")) {
    const unsigned bt = atoi(argv[2]), dh = atoi(argv[3]);
    for (unsigned t = 0; t < bt; ++t) for (unsigned d = 0; d < dh; ++d) printf("%u %u\n", kv_key_at(t, d, dh), kv_value_at(t, d, dh));
  } else if (!strcmp(argv[1], "scale")) {
    for (int i = 2; i < argc; ++i) { float f = strtof(argv[i], nullptr); uint32_t b; memcpy(&b, &f, 4); printf("%d\n", kv_scale_exponent(b)); }
  } else {
    // every step list against the definition: steps in order, none twice, all that some row sees
    long bad = 0, n = 0;
    for (int len = 0; len <= 200; len += 7) for (int first = -40; first <= len; first += 5) for (int rows = 1; rows <= 60; rows += 13)
      for (int window = 0; window <= 120; window += 17) for (int prefix = -5; prefix <= 230; prefix += 23) {
        const int pre = prefix < len ? prefix : len, last = first + rows - 1;
        int seen = last + 1 > pre ? last + 1 : pre;
        seen = seen < 0 ? 0 : seen > len ? len : seen;
        const KvSteps k = kv_steps(len, seen, first, window, prefix);
        static char got[64];
        memset(got, 0, sizeof(got));
        int prev = -1;
        for (int j = 0; j < k.count; ++j) { const int s = k.step(j); if (s <= prev || s * 32 >= len) ++bad; prev = s; if (s >= 0 && s < 64) got[s] = 1; }
        for (int p = first; p <= last; ++p) for (int t = 0; t < len; ++t)
          if ((t < pre || (t <= p && (window <= 0 || p - t < window))) && !got[t / 32]) ++bad;
        ++n;
      }
    printf("%ld bad of %ld\n", bad, n);
  }
  return 0;
}
'''


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv")
    src, exe = d / "probe.cpp", d / "probe"
    src.write_text(PROBE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2508_09204_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    return lambda *a: subprocess.run([str(exe)] + [str(x) for x in a], check=True, capture_output=True, text=True).stdout


@pytest.mark.parametrize("bt,dh", [(32, 64), (64, 128), (128, 256)])
def test_places_of_codes(probe, bt, dh):
    got = np.array([[int(x) for x in line.split()] for line in probe("at", bt, dh).splitlines()])
    t, d = np.meshgrid(np.arange(bt), np.arange(dh), indexing="ij")
    assert np.array_equal(got[:, 0], do.key_at(t, d, dh).ravel()) and np.array_equal(got[:, 1], do.value_at(t, d, dh).ravel())


def test_scale_exponents(probe):
    x = np.array([0.0, 1e-45, 1e-38, 1.0, 448.0, np.nextafter(np.float32(448), np.float32(500)), 447.0, 1.75, 1.7500001, 3.4e38, 5e-7, 896.0, 897.0], dtype=np.float32)
    got = [int(v) for v in probe("scale", *[repr(float(v)) for v in x]).split()]
    assert [2.0 ** e for e in got] == [do.scale_for(float(v)) for v in x]


def test_steps_cover_what_rows_see(probe):
    assert probe("steps").startswith("0 bad of ")


def test_sizes_that_the_launches_do_not_hold_are_refused(mq):
    assert _attend(mq, batch={"S": 1 << 16, "T": 1, "M": 1 << 16, "table_width": 1 << 13}) == 0
    assert _attend(mq, batch={"S": 1 << 16, "T": 1, "M": 1 << 16, "table_width": 1 << 14}) == -2        # 2^36 places for tokens
    assert _append(mq, batch={"S": 1 << 16, "T": 1, "M": 1 << 16, "table_width": 1 << 14}) == -2
