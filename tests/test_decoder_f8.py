"""The decoder in 8-bit floating point and its draws without a GPU: all calls with their arguments checked (dry-run mode), and what it refuses."""
import pytest
import torch

from paper_2508_09204_amd import decoder as dec


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


def _model(mq, layers=2, d=256, f=384, heads=4, kv=2, dh=64, K=3, V=500, out_int=False, mlp_int=False):
    f8 = lambda n, k, gated=False: mq.F8Mat(_aligned(mq.moqe_f8_packed_bytes(n, k, gated)), n, k, gated)
    ints = lambda n, k: [mq.QMat(_aligned(mq.moqe_packed_bytes(n, k, 4, 128, False)), None, None, n, k, 4, 128, False, 0, mq.LAYOUT_PACKED) for _ in range(K)]
    router = mq.Router(None, None, torch.zeros(K, d), None, d, 0, K)
    norm = lambda: mq.Norm("rms", 1e-6, torch.ones(d))
    mlp = lambda: (mq.Block(kind=mq.KIND_SILU_MLP, router=router, w0=ints(f, d), w1=ints(f, d), w2=ints(d, f)) if mlp_int else
                   dec.F8Mlp([f8(f, d, True) for _ in range(K)], [f8(d, f) for _ in range(K)]))
    made = [dec.Layer(norm(), [f8((heads + 2 * kv) * dh, d)], ints(d, heads * dh) if out_int else [f8(d, heads * dh) for _ in range(K)], norm(), mlp()) for _ in range(layers)]
    return dec.Decoder(made, norm(), router, mq.Rope(dec.rope_frequencies(dh, device="cpu"), dh), heads, kv, dh, head=f8(V, d) if V else None,
                       embedding=torch.zeros(V, d) if V else None)


@pytest.mark.parametrize("out_int,mlp_int", [(False, False), (True, False), (False, True)])
def test_a_step_and_a_draw_pass_every_check(mq, out_int, mlp_int):
    model = _model(mq, out_int=out_int, mlp_int=mlp_int)
    seqs = dec.Sequences(model, 3, 100, 32, device="cpu")
    for T in (97, 1):
        step = dec.Step(model, seqs, T, _aligned(1 << 24))
        assert step().shape == (3 * T, 256)
        assert step.out8.M == 3 * T and step.out8.d == 256
    assert int(seqs.kv_len[1]) == 98
    with pytest.raises(ValueError):
        dec.Step(model, seqs, 1, _aligned(256))


def test_what_has_no_head_gives_no_tokens(mq):
    model = _model(mq, layers=1, V=0)
    step = dec.Step(model, dec.Sequences(model, 2, 50, 32, device="cpu"), 1, _aligned(1 << 24))
    assert step.out8 is None
    with pytest.raises(ValueError):
        dec.Draw(model, step)
    with pytest.raises(ValueError):
        dec.Generator(model, 2, 10, 10)


def test_a_generator_refuses_tables_and_prompts_that_do_not_fit(mq):
    """Before anything reaches the device: a lookup outside a table ends the process there, and a lookup of another size would move the buffer that the calls point to."""
    model = _model(mq, layers=1, V=50)
    good = model.embedding
    for table in (good[:-1], torch.zeros(50, 255), good.bfloat16()):
        model.embedding = table
        with pytest.raises(ValueError, match="embedding"):
            dec.Generator(model, 2, 10, 10)
    dec.check_tokens(torch.tensor([[0, 49], [3, 4], [5, 6]]), 3, 2, 50)
    dec.check_tokens(torch.tensor([[0], [49]], dtype=torch.int32), 2, 1, 50)
    for tokens in (torch.tensor([[0, 50]]), torch.tensor([[-1, 0]]), torch.zeros(2, 1, dtype=torch.long), torch.zeros(2, dtype=torch.long), torch.zeros(1, 3, dtype=torch.long),
                   torch.zeros(1, 2)):
        with pytest.raises(ValueError, match="tokens"):
            dec.check_tokens(tokens, 1, 2, 50)


def test_a_sequence_without_a_token_goes_on_as_from_token_0():
    table, x = torch.randn(7, 5), torch.empty(3, 5)
    at = x.data_ptr()
    dec.embed(table, torch.tensor([-1, 6, 2], dtype=torch.int32), x)
    assert torch.equal(x, table[[0, 6, 2]]) and x.data_ptr() == at


def test_products_refuse_no_matrix_and_no_rows_a_sample(mq):
    rows = mq.F8Rows(_aligned(2 * 256).view(2, 256), _aligned(8).view(2, 4), 2, 256)
    mat = mq.F8Mat(_aligned(mq.moqe_f8_packed_bytes(32, 256)), 32, 256)
    for mats, T in (([], 1), ([mat], 0), ([mat], -1)):
        with pytest.raises(ValueError):
            mq.F8GemmCall(rows, mats, torch.zeros(2, 32), T=T)
