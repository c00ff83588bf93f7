"""On which GPU the marshalled calls run: the current one's stream unless one is given (no GPU: dry-run mode, the current device and the tensors' made up)."""
import pytest
import torch

BF, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def mq():
    from paper_2508_09204_amd import binding
    binding.moqe_set_dry_run(True)
    yield binding
    binding.moqe_set_dry_run(False)


def _aligned(nbytes):
    t = torch.zeros(nbytes + 256, dtype=torch.uint8)
    at = -t.data_ptr() % 256
    return t[at:at + nbytes]


def _calls(mq):
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)  # noqa: E731
    cache = mq.KvCache.empty(3, 2, 32, 64, "cpu")
    batch = mq.KvBatch(z(2, 4, t=I32), z(2, t=I32), 2, 1, 2)
    attn = mq.Attention(4, 0.125)
    rows = lambda M, d: mq.F8Rows(_aligned(M * d).view(M, d), _aligned(M * 4).view(M, 4), M, d)  # noqa: E731
    mat = mq.F8Mat(_aligned(mq.moqe_f8_packed_bytes(32, 256)), 32, 256)
    return [mq.ResidualNormCall(z(2, 256), z(2, 256), z(2, 256, t=BF)), mq.ResidualNormF8Call(None, z(2, 256), rows(2, 256)),
            mq.KvAppendCall(z(2, 512), 4, mq.Rope(None, 0), batch, cache, z(2, 256, t=BF)),
            mq.KvAttentionCall(z(2, 256, t=BF), attn, batch, cache, z(2, 256, t=BF), _aligned(max(256, mq.moqe_kv_attention_workspace_bytes(attn, batch, cache)))),
            mq.F8GemmCall(rows(2, 256), [mat], z(2, 32), workspace=_aligned(256)),
            mq.SampleCall(z(2, 40), z(2), z(2, t=I32), workspace=_aligned(mq.moqe_sample_workspace_bytes(2, 40)))]


@pytest.mark.parametrize("i", range(6))
def test_the_stream_says_which_gpu(mq, monkeypatch, i):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(mq, "_stream", lambda: 0)
    call = _calls(mq)[i]
    call._device = 1                                   # as of tensors on the second GPU
    for stream in (None, 0):                           # the current device's
        with pytest.raises(ValueError, match="GPU 1"):
            call(stream)
    call(0x5000)                                       # a stream of the second GPU, as its caller knows
    call._device = 0
    call()
    call(0)
    call(0x5000)
