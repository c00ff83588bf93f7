"""A Generator whose calls are refused between others."""
import pytest
import torch

from tests.test_gpu_f8_decoder import DEV, _how, _model, _uniform
from paper_2508_09204_amd import decoder as dec

pytestmark = pytest.mark.gpu


def test_uniform_numbers_that_do_not_fit_leave_everything_as_it_was():
    S, T, V, n = 3, 12, 600, 5
    model = _model(layers=1, V=V, seed=6)
    prompt = torch.randint(0, V, (S, T), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    u = _uniform(n + 1, S)
    seen = []
    for refused in (False, True):
        g = dec.Generator(model, S, T, n, 32, **_how(S))
        got = [g.start(prompt, u[0]).clone()]
        for i in range(n):
            if refused:
                at = g.seqs.tokens
                for call in (lambda: g.next(u[0, :2]), lambda: g.start(prompt, torch.zeros(S + 1, device=DEV))):
                    with pytest.raises(RuntimeError):
                        call()
                assert g.seqs.tokens == at and int(g.seqs.kv_len[0]) == at
            got.append(g.next(u[1 + i]).clone())
        with pytest.raises(ValueError, match="hold"):
            g.next(u[0])
        torch.cuda.synchronize()
        seen.append(torch.stack(got))
    assert torch.equal(*seen)
