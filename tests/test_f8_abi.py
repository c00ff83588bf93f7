"""8-bit rows, products and sampling without a GPU: refusals (dry-run mode: nothing is enqueued), the places of csrc/f8_rows.h compiled for the host, and what the binding
checks of its tensors."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # a non-NULL, 256-byte aligned address; never dereferenced in dry-run mode


@pytest.fixture(scope="module")
def mq():
    from paper_2508_09204_amd import binding
    binding.moqe_set_dry_run(True)
    yield binding
    binding.moqe_set_dry_run(False)


def _rows(mq, d=300, **kw):
    b = -(-d // 128)
    r = mq._F8Rows(FAKE, FAKE, b * 128, (b + 3) // 4 * 4)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


BAD_ROWS = [({"codes": None}, -1), ({"scales": None}, -1), ({"codes": FAKE + 8}, -2), ({"scales": FAKE + 2}, -2), ({"code_stride": 383}, -2), ({"code_stride": 368}, -2),
            ({"code_stride": 392}, -2), ({"scale_stride": 3}, -2), ({"scale_stride": 0}, -2), ({"scale_stride": 6}, -2), ({"code_stride": (1 << 32) + 16}, -2)]


def _step(mq, **kw):
    s = mq._ResidualStep()
    s.residual, s.residual_stride, s.M, s.d, s.residual_type, s.scale = FAKE, 300, 4, 300, 1, 1.0
    for k, v in kw.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("change,code", [({}, 0), ({"code_stride": 400}, 0), ({"scale_stride": 8}, 0)] + BAD_ROWS)
def test_norm_refuses_rows(mq, change, code):
    assert mq.lib.moqe_residual_norm_f8(C.byref(_step(mq)), C.byref(_rows(mq, **change)), None) == code


def test_norm_refuses_what_the_norm_in_bf16_does(mq):
    call = lambda **kw: mq.lib.moqe_residual_norm_f8(C.byref(_step(mq, **kw)), C.byref(_rows(mq)), None)
    assert call() == 0 and call(M=0, residual=None) == 0 and call(out=FAKE, out_stride=300) == 0
    assert call(d=0) == -2 and call(M=-1) == -2 and call(residual=None) == -1 and call(out=FAKE, out_stride=299) == -2 and call(residual_type=2) == -3
    assert call(pre=mq._Norm(FAKE, None, 3, 1e-5)) == -3 and call(gate_rows=-1) == -2
    assert mq.lib.moqe_residual_norm_f8(None, C.byref(_rows(mq)), None) == -1 and mq.lib.moqe_residual_norm_f8(C.byref(_step(mq)), None, None) == -1


def test_packed_sizes(mq):
    f = mq.lib.moqe_f8_packed_bytes
    assert f(16, 128, 0) == 2048 + 256 and f(1, 1, 0) == 2048 + 256 and f(17, 129, 0) == 4 * 2048 + 256 and f(17, 129, 1) == 8 * 2048 + 256
    assert f(0, 128, 0) == 0 and f(16, 0, 0) == 0 and f(-16, 128, 0) == 0 and f(1 << 30, 1 << 30, 0) == 0 and f(2 ** 31 - 1, 2 ** 31 - 1, 1) == 0
    assert f(32768, 100000, 0) > 0 and f(32768, 131072, 0) == 0 and f(32768, 65536, 1) == 0                        # 4 GiB


@pytest.mark.parametrize("change,code", [({}, 0)] + BAD_ROWS)
@pytest.mark.parametrize("which", [0, 1])
def test_pack_refuses_rows(mq, change, code, which):
    r = [_rows(mq), _rows(mq)]
    r[which] = _rows(mq, **change)
    assert mq.lib.moqe_f8_pack(C.byref(r[0]), C.byref(r[1]), 20, 300, FAKE, 1 << 20, None) == code
    mat = mq._F8Mat(FAKE, 20, 300, 1)
    assert mq.lib.moqe_f8_unpack(C.byref(mat), C.byref(r[0]), C.byref(r[1]), None) == code


def test_pack_refusals(mq):
    r = _rows(mq)
    need = mq.lib.moqe_f8_packed_bytes(20, 300, 0)
    pack = lambda n=20, k=300, out=FAKE, size=need: mq.lib.moqe_f8_pack(C.byref(r), None, n, k, out, size, None)
    assert pack() == 0 and pack(n=0) == -2 and pack(k=0) == -2 and pack(out=None) == -1 and pack(out=FAKE + 128) == -2 and pack(size=need - 1) == -2
    assert mq.lib.moqe_f8_pack(None, None, 20, 300, FAKE, need, None) == -1
    unpack = lambda m, up=None: mq.lib.moqe_f8_unpack(C.byref(mq._F8Mat(*m)), C.byref(r), up, None)
    assert unpack((FAKE, 20, 300, 0)) == 0 and unpack((None, 20, 300, 0)) == -1 and unpack((FAKE + 64, 20, 300, 0)) == -2 and unpack((FAKE, 20, 300, 1)) == -3
    assert unpack((FAKE, 20, 300, 0), C.byref(r)) == -3 and mq.lib.moqe_f8_unpack(None, C.byref(r), None, None) == -1


def _gemm(mq, a=None, offsets=FAKE, perm=FAKE, S=6, T=5, mats=None, K=2, y=None, flags=1, ws=FAKE, ws_bytes=1 << 40, n=40, k=300, gated=0):
    mats = mats if mats is not None else [(FAKE, n, k, gated)] * K
    arr = (mq._F8Mat * len(mats))(*(mq._F8Mat(*m) for m in mats))
    y = y if y is not None else mq._F8Result(FAKE, n, 0, mq._F8Rows())
    a = _rows(mq, k) if a is None else a
    return mq.lib.moqe_f8_gemm(C.byref(a), offsets, perm, S, T, arr, K, C.byref(y), flags, ws, ws_bytes, None)


@pytest.mark.parametrize("change,code", [
    ({}, 0), ({"S": 0}, 0), ({"flags": 3}, 0), ({"flags": 0, "perm": None}, 0), ({"offsets": None, "perm": None, "K": 1, "flags": 0}, 0), ({"K": 16}, 0),
    ({"S": -1}, -2), ({"T": 0}, -2), ({"S": 1 << 20, "T": 1 << 11}, -2), ({"K": 17}, -2), ({"K": 0, "mats": [(FAKE, 40, 300, 0)]}, -2), ({"flags": 9}, 0), ({"flags": 4}, -3), ({"flags": 17}, -3),
    ({"offsets": None}, -1), ({"perm": None}, -1), ({"offsets": FAKE + 2}, -2), ({"perm": FAKE + 1}, -2),
    ({"mats": [(FAKE, 40, 300, 0), (None, 40, 300, 0)]}, -1), ({"mats": [(FAKE, 40, 300, 0), (FAKE + 16, 40, 300, 0)]}, -2), ({"mats": [(FAKE, 40, 300, 0), (FAKE, 41, 300, 0)]}, -2),
    ({"mats": [(FAKE, 40, 300, 0), (FAKE, 40, 300, 1)]}, -2), ({"mats": [(FAKE, 40, 300, 0), (FAKE, 40, 301, 0)]}, -2), ({"n": 0}, -2), ({"k": 0}, -2),
    ({"S": 12000000, "T": 1}, -2),                                                        # 4.6 GB of codes
])
def test_product_refusals(mq, change, code):
    assert _gemm(mq, **change) == code


def test_product_refuses_results_and_workspaces(mq):
    res = lambda **kw: _gemm(mq, y=mq._F8Result(**{"data": FAKE, "stride": 40, "type": 0, **kw}))
    assert res() == 0 and res(type=1) == 0 and res(stride=41) == 0 and res(data=FAKE + 4) == 0 and res(data=FAKE + 2, type=1) == 0
    assert res(data=None) == -1 and res(stride=39) == -2 and res(data=FAKE + 2) == -2 and res(data=FAKE + 1, type=1) == -2 and res(type=3) == -3 and res(type=-1) == -3
    assert res(type=2, rows8=_rows(mq, 40)) == -3                                          # only gated pairs give 8 bits
    rows8 = lambda r, **kw: _gemm(mq, gated=1, y=mq._F8Result(None, 0, 2, r), **kw)
    assert rows8(_rows(mq, 40)) == 0 and rows8(_rows(mq, 40, codes=None)) == -1 and rows8(_rows(mq, 40, code_stride=112)) == -2
    assert rows8(_rows(mq, 32768), n=32768) == 0 and rows8(_rows(mq, 32769), n=32769) == -2
    mats = (mq._F8Mat * 2)(*[mq._F8Mat(FAKE, 40, 300, 1)] * 2)
    need = mq.lib.moqe_f8_gemm_workspace_bytes(mats, 2, 6, 5, 2)
    if need:
        assert rows8(_rows(mq, 40), ws=None) == -4 and rows8(_rows(mq, 40), ws_bytes=need - 1) == -4 and rows8(_rows(mq, 40), ws=FAKE + 16) == -4
    assert rows8(_rows(mq, 40), ws_bytes=need) == 0 and _gemm(mq, ws=None, ws_bytes=0) == 0
    assert mq.lib.moqe_f8_gemm_workspace_bytes(mats, 2, 6, 5, 3) == 0 and mq.lib.moqe_f8_gemm_workspace_bytes(None, 2, 6, 5, 0) == 0


@pytest.mark.parametrize("change,code", BAD_ROWS)
def test_product_refuses_rows(mq, change, code):
    assert _gemm(mq, a=_rows(mq, **change)) == code


def _sample(mq, logits=FAKE, typ=0, stride=1000, S=5, V=1000, how=(FAKE, FAKE, FAKE, FAKE), u=FAKE, tokens=FAKE, lp=FAKE, ws=FAKE, short=0):
    need = mq.lib.moqe_sample_workspace_bytes(S, V)
    return mq.lib.moqe_sample(logits, typ, stride, S, V, C.byref(mq._Sampling(*how)) if how is not None else None, u, tokens, lp, ws, max(0, need - short), None)


@pytest.mark.parametrize("change,code", [
    ({}, 0), ({"S": 0, "logits": None}, 0), ({"typ": 1}, 0), ({"how": (None,) * 4}, 0), ({"lp": None}, 0), ({"stride": 1001}, 0), ({"logits": FAKE + 2, "typ": 1}, 0), ({"V": 1 << 20, "stride": 1 << 20}, 0),
    ({"S": -1}, -2), ({"V": 0}, -2), ({"V": (1 << 20) + 1, "stride": 1 << 21}, -2), ({"typ": 2}, -3), ({"how": None}, -1), ({"logits": None}, -1), ({"u": None}, -1), ({"tokens": None}, -1),
    ({"stride": 999}, -2), ({"logits": FAKE + 2}, -2), ({"logits": FAKE + 1, "typ": 1}, -2), ({"u": FAKE + 1}, -2), ({"tokens": FAKE + 2}, -2), ({"lp": FAKE + 3}, -2),
    ({"how": (FAKE + 1, None, None, None)}, -2), ({"how": (None, FAKE + 2, None, None)}, -2), ({"how": (None, None, FAKE + 3, None)}, -2), ({"how": (None, None, None, FAKE + 1)}, -2),
])
def test_sample_refusals(mq, change, code):
    assert _sample(mq, **change) == code


def test_sample_workspace(mq):
    need = mq.lib.moqe_sample_workspace_bytes(5, 1000)
    if need:
        assert _sample(mq, ws=None) == -4 and _sample(mq, ws=FAKE + 128) == -4 and _sample(mq, short=1) == -4
    assert mq.lib.moqe_sample_workspace_bytes(0, 1000) == 0 and mq.lib.moqe_sample_workspace_bytes(5, 0) == 0 and mq.lib.moqe_sample_workspace_bytes(5, (1 << 20) + 1) == 0


# ------------------------------------------------------------------------------------------------------------------ places
def test_places_are_a_bijection(tmp_path):
    src = tmp_path / "places.cpp"
    src.write_text('''
#include "f8_rows.h"
#include <cstdio>
#include <vector>
using namespace moqe;
int main() {
  std::vector<int> seen(2048, 0);
  for (int r = 0; r < 16; ++r)
    for (int c = 0; c < 128; ++c) {
      const uint32_t at = f8_code_at(r, c);
      if (at >= 2048 || seen[at]++) { printf("code %d %d\\n", r, c); return 1; }
      const int lane = at % 1024 / 16;                       // a lane has one row, and 16 neighbouring columns to a kilobyte
      if (lane % 16 != r || lane / 16 != c % 64 / 16 || int(at / 1024) != c / 64) { printf("lane %d %d\\n", r, c); return 1; }
    }
  for (int n : {1, 16, 17, 300})
    for (int k : {1, 128, 129, 640, 5000})
      for (int gated = 0; gated < 2; ++gated) {
        const F8Packed p = f8_packed(n, k, gated);
        std::vector<int> s(p.total - p.scale_off, 0);
        if (p.tiles < (n + 15) / 16 * (gated + 1) || p.blocks != (k + 127) / 128 || p.scale_off != size_t(p.tiles) * p.blocks * 2048 || p.total % 256) return 1;
        for (int t = 0; t < p.tiles; ++t)
          for (int r = 0; r < 16; ++r)
            for (int b = 0; b < p.blocks; ++b) {
              const size_t at = f8_scale_at(p, t, r, b);
              if (at < p.scale_off || at >= p.total || s[at - p.scale_off]++) { printf("scale %d %d %d\\n", t, r, b); return 1; }
            }
      }
  printf("ok\\n");
}
''')
    exe = tmp_path / "places"
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2508_09204_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout == "ok\n"


# ------------------------------------------------------------------------------------------------------------------ the binding
def _aligned(nbytes):
    t = torch.zeros(nbytes + 256, dtype=torch.uint8)
    at = -t.data_ptr() % 256
    return t[at:at + nbytes]


def _host_rows(mq, M, d):
    b = -(-d // 128)
    return mq.F8Rows(_aligned(M * b * 128).view(M, b * 128), _aligned(M * ((b + 3) // 4 * 4)).view(M, -1), M, d)


def _mat(mq, n, k, gated=False):
    return mq.F8Mat(_aligned(mq.moqe_f8_packed_bytes(n, k, gated)), n, k, gated)


def test_binding_passes_good_calls(mq):
    a = _host_rows(mq, 12, 300)
    mq.F8GemmCall(a, [_mat(mq, 40, 300)], torch.zeros(12, 40))()
    mq.F8GemmCall(a, [_mat(mq, 40, 300, True)], _host_rows(mq, 12, 40), workspace=_aligned(1 << 20))()
    mq.F8GemmCall(a, [_mat(mq, 40, 300)] * 2, torch.zeros(12, 40, dtype=torch.bfloat16), offsets=torch.zeros(3, dtype=torch.int32), perm=torch.zeros(4, dtype=torch.int32), S=4, T=3,
                  scatter=True)()
    mq.ResidualNormF8Call(None, torch.zeros(12, 300), a)()
    mq.moqe_f8_pack(_host_rows(mq, 40, 300), None, _mat(mq, 40, 300).packed)
    mq.SampleCall(torch.zeros(3, 50), torch.zeros(3), torch.zeros(3, dtype=torch.int32), workspace=_aligned(1 << 20))()


@pytest.mark.parametrize("call", [
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 301)], torch.zeros(12, 40)),
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 300)], torch.zeros(11, 40)),
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 300)], torch.zeros(12, 41)),
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 300)], torch.zeros(12, 40, dtype=torch.float16)),
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 300)], torch.zeros(12, 40), S=5, T=2),
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 300)], torch.zeros(12, 40), perm=torch.zeros(12, dtype=torch.int32)),
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 300)] * 2, torch.zeros(12, 40), offsets=torch.zeros(2, dtype=torch.int32)),
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 300)], torch.zeros(12, 40), offsets=torch.zeros(2, dtype=torch.int64)),
    lambda mq, a: mq.F8GemmCall(a, [mq.F8Mat(_aligned(1000), 40, 300)], torch.zeros(12, 40)),
    lambda mq, a: mq.F8GemmCall(a, [_mat(mq, 40, 300, True)], _host_rows(mq, 12, 41)),
    lambda mq, a: mq.F8GemmCall(mq.F8Rows(a.codes.t(), a.scales, 12, 300), [_mat(mq, 40, 300)], torch.zeros(12, 40)),
    lambda mq, a: mq.F8GemmCall(mq.F8Rows(a.codes, a.scales, 12, 600), [_mat(mq, 40, 600)], torch.zeros(12, 40)),
    lambda mq, a: mq.F8GemmCall(mq.F8Rows(a.codes.to(torch.int8), a.scales, 12, 300), [_mat(mq, 40, 300)], torch.zeros(12, 40)),
    lambda mq, a: mq.ResidualNormF8Call(None, torch.zeros(12, 299), a),
    lambda mq, a: mq.F8Mat.pack(_host_rows(mq, 40, 300), _host_rows(mq, 40, 301)),
    lambda mq, a: mq.moqe_f8_unpack(_mat(mq, 40, 300), _host_rows(mq, 41, 300)),
    lambda mq, a: mq.SampleCall(torch.zeros(3, 50), torch.zeros(2), torch.zeros(3, dtype=torch.int32)),
    lambda mq, a: mq.SampleCall(torch.zeros(3, 50), torch.zeros(3), torch.zeros(3, dtype=torch.int64)),
    lambda mq, a: mq.SampleCall(torch.zeros(3, 50), torch.zeros(3), torch.zeros(3, dtype=torch.int32), top_k=torch.zeros(3)),
    lambda mq, a: mq.SampleCall(torch.zeros(3, 50).double(), torch.zeros(3), torch.zeros(3, dtype=torch.int32)),
    lambda mq, a: mq.SampleCall(torch.zeros(150), torch.zeros(3), torch.zeros(3, dtype=torch.int32)),
    lambda mq, a: mq.moqe_f8_packed_bytes(1 << 32, 128),
])
def test_binding_refuses(mq, call):
    with pytest.raises((ValueError, TypeError)):
        call(mq, _host_rows(mq, 12, 300))


def test_tensors_of_another_gpu_are_refused(mq, monkeypatch):
    call = mq.SampleCall(torch.zeros(3, 50), torch.zeros(3), torch.zeros(3, dtype=torch.int32), workspace=_aligned(1 << 20))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    call._device = 0
    call()
    call._device = 1
    with pytest.raises(ValueError):
        call()


def test_scales_end_at_a_multiple_of_four(mq):
    a = _host_rows(mq, 12, 300)
    with pytest.raises(ValueError):
        mq.F8GemmCall(mq.F8Rows(a.codes, a.scales[:, :3], 12, 300), [_mat(mq, 40, 300)], torch.zeros(12, 40))


def test_host_memory_is_for_dry_runs_only(mq):
    call = mq.F8GemmCall(_host_rows(mq, 12, 300), [_mat(mq, 40, 300)], torch.zeros(12, 40))
    draw = mq.SampleCall(torch.zeros(3, 50), torch.zeros(3), torch.zeros(3, dtype=torch.int32), workspace=_aligned(1 << 20))
    call(), draw()
    mq.moqe_set_dry_run(False)
    try:
        for c in (call, draw, lambda: mq.moqe_f8_pack(_host_rows(mq, 40, 300), None, _mat(mq, 40, 300).packed)):
            with pytest.raises(ValueError):
                c()
    finally:
        mq.moqe_set_dry_run(True)
