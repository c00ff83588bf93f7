"""What the binding of the decoder layer's operators does with its arguments before the library sees them (no GPU; dry-run mode where a call is made)."""
import pytest
import torch

BF, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def mq():
    from paper_2508_09204_amd import binding
    binding.moqe_set_dry_run(True)
    yield binding
    binding.moqe_set_dry_run(False)


def z(*s, t=torch.float32):
    return torch.zeros(s, dtype=t)


@pytest.mark.parametrize("wide", [2 ** 32 + 5, 2 ** 31, -2 ** 31 - 1])
def test_integers_that_do_not_fit_are_refused(mq, wide):
    cache = mq.KvCache.empty(3, 2, 32, 64, "cpu")
    batch = mq.KvBatch(z(2, 4, t=I32), z(2, t=I32), 2, 1, 2)
    q, out = z(2, 256, t=BF), z(2, 256, t=BF)
    with pytest.raises(ValueError, match="window"):
        mq.KvAttentionCall(q, mq.Attention(4, 0.1, window=wide), batch, cache, out)
    with pytest.raises(ValueError, match="window"):
        mq.moqe_kv_attention_workspace_bytes(mq.Attention(4, 0.1, window=wide), batch, cache)
    with pytest.raises(ValueError, match="n_heads"):
        mq.KvAttentionCall(q, mq.Attention(wide, 0.1), batch, cache, out)
    with pytest.raises(ValueError, match="T = "):
        mq.KvBatch(z(2, 4, t=I32), z(2, t=I32), 2, wide, 2).c()
    with pytest.raises(ValueError, match="M = "):
        mq.KvBatch(z(2, 4, t=I32), z(2, t=I32), 2, 1, wide).c()
    with pytest.raises(ValueError, match="rot_dim"):
        mq.Rope(None, wide).c(64)
    with pytest.raises(ValueError, match="gate_rows"):
        mq.ResidualNormCall(z(2, 8), z(2, 8), z(2, 8, t=BF), gate_rows=wide)
    assert mq.Attention(4, 0.1, window=2 ** 31 - 1).c(2).window == 2 ** 31 - 1


def test_calls_without_rows_do_nothing(mq):
    """No rows, or no sequences: accepted, as the library accepts them."""
    cache = mq.KvCache.empty(3, 2, 32, 64, "cpu")
    for S in (0, 2):
        batch = mq.KvBatch(z(S, 4, t=I32), z(S, t=I32), S, 1, 0, z(S + 1, t=I32))
        mq.moqe_kv_append(z(0, 512, t=BF), 4, mq.Rope(z(32, t=torch.float64), 64), batch, cache, z(0, 256, t=BF))
        mq.moqe_kv_attention(z(0, 256, t=BF), mq.Attention(4, 0.1), batch, cache, z(0, 4, 64, t=BF))
    for gate in (None, z(0, 8)):
        mq.moqe_residual_norm(z(0, 8), z(0, 8), z(0, 8, t=BF), z(0, 8), gate, 3 if gate is not None else 0, pre=mq.Norm("rms", 1e-5, z(8)))
    with pytest.raises(ValueError):
        mq.moqe_kv_attention(z(0, 128, t=BF), mq.Attention(4, 0.1), batch, cache, z(0, 256, t=BF))      # rows of another width


def aligned(nbytes):
    t = torch.zeros(nbytes + 256, dtype=torch.uint8)
    at = -t.data_ptr() % 256
    return t[at:at + nbytes]


def test_a_single_row_of_a_wider_buffer(mq):
    """One row has no stride that could be misaligned, whatever the buffer it lies in."""
    cache = mq.KvCache.empty(3, 2, 32, 64, "cpu")
    batch = mq.KvBatch(z(1, 4, t=I32), z(1, t=I32), 1, 1, 1)
    row = lambda n: aligned(2 * 5 * (n + 3)).view(BF).view(5, n + 3)[:1, :n]  # noqa: E731
    mq.moqe_kv_append(row(512), 4, mq.Rope(z(32, t=torch.float64), 64), batch, cache, row(256))
    mq.moqe_kv_attention(row(256), mq.Attention(4, 0.1), batch, cache, row(256))
    r = row(256)
    mq.moqe_residual_norm(None, r, row(256), r)


def _calls(mq, at):
    """One call of each kind, the argument named `at` on another device than the others."""
    def d(name, t):
        return t.to("meta") if name == at else t
    cache = mq.KvCache(d("k", z(3, 2, 2048, t=torch.uint8)), z(3, 2, 2048, t=torch.uint8), z(3, 2), d("v_scale", z(3, 2)), 32, 64)
    batch = mq.KvBatch(d("table", z(2, 4, t=I32)), d("kv_len", z(2, t=I32)), 2, 1, 2, d("cu", z(3, t=I32)))
    rope = mq.Rope(d("inv_freq", z(32, t=torch.float64)), 64, q_gain=d("gain", z(64)))
    attn = mq.Attention(4, 0.1, slopes=d("slopes", z(4)), prefix=d("prefix", z(2, t=I32)))
    return [lambda: mq.KvAppendCall(d("qkv", z(2, 512)), 4, rope, batch, cache, d("q", z(2, 256, t=BF))),
            lambda: mq.KvAttentionCall(d("q", z(2, 256, t=BF)), attn, batch, cache, z(2, 256, t=BF), d("ws", aligned(1 << 20))),
            lambda: mq.ResidualNormCall(d("y", z(2, 8)), z(2, 8), z(2, 8, t=BF), gate=d("gate", z(8)), pre=mq.Norm("layer", 1e-5, z(8), d("offset", z(8))))]


@pytest.mark.parametrize("at,which", [(n, [0, 1]) for n in ("k", "v_scale", "table", "kv_len", "cu", "q")] + [(n, [0]) for n in ("inv_freq", "gain", "qkv")] +
                         [(n, [1]) for n in ("slopes", "prefix", "ws")] + [(n, [2]) for n in ("y", "gate", "offset")])
def test_tensors_on_different_devices_are_refused(mq, at, which):
    for i, make in enumerate(_calls(mq, at)):
        if i in which:
            with pytest.raises(ValueError, match="devices"):
                make()
        else:
            make()


def test_host_memory_is_for_dry_runs_only(mq):
    """Outside a dry run an address on the host would go to a kernel."""
    calls = [make() for make in _calls(mq, None)]
    for call in calls:
        call()
    mq.moqe_set_dry_run(False)
    try:
        for call in calls:
            with pytest.raises(ValueError, match="device memory"):
                call()
    finally:
        mq.moqe_set_dry_run(True)
