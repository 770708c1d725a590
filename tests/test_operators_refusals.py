"""More refusals of the operators on caller-owned tensors that the host finds by itself, without a GPU."""
import pytest
import torch

from paper_2002_09539_b200 import operators
from paper_2002_09539_b200.build import build

P = 1 << 20   # an aligned address that nothing dereferences
EINVAL = 1


@pytest.fixture(scope="module")
def lib():
    build()
    return operators._ops()


def _gated_backward(lib, T, dx, dwg, dwu):
    m, D, F = 2, 64, 32
    return lib.olsgd_gated_backward(m, T, D, F, 1, 0, P, T * F, F, P, T * D, D, P, F * D, D, P, F * D, D, P, dx, dwg, dwu, P, 1 << 30, None)


@pytest.mark.parametrize("T", [0, 8])
@pytest.mark.parametrize("dx,dwg,dwu,word", [(P, P, None, "both or neither"), (P, None, P, "both or neither"), (None, P + 1, P, "aligned"),
                                             (None, P, P + 1, "aligned"), (P + 1, None, None, "aligned")])
def test_gated_backward_refuses_the_same_outputs_whatever_the_number_of_tokens(lib, T, dx, dwg, dwu, word):
    assert _gated_backward(lib, T, dx, dwg, dwu) == EINVAL
    assert word in lib.olsgd_last_error(None).decode()


# ------------------------------------------------------------------------------ recorded tensors

def _calls_that_would_lose_gradients():
    f, h, i = (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.bfloat16)), (lambda *s: torch.zeros(s, dtype=torch.int32))
    g = lambda t: t.requires_grad_()   # noqa: E731
    o = operators
    return [lambda: o.token_logprobs(g(f(2, 9)), i(2)),
            lambda: o.token_logprobs_backward(g(f(2)), None, f(2, 9), i(2), f(2, 2), f(2)),
            lambda: o.token_logprobs_backward(None, g(f(2)), f(2, 9), i(2), f(2, 2), f(2)),
            lambda: o.token_logprobs_backward(None, None, g(f(2, 9)), i(2), f(2, 2), f(2)),
            lambda: o.clip_grads(g(f(2, 9)), 1.0), lambda: o.clip_grads([g(f(2, 9)), f(2, 3)], 1.0),
            lambda: o.gated_forward(g(h(1, 3, 8)), h(1, 4, 8), h(1, 4, 8)), lambda: o.gated_forward(h(1, 3, 8), g(h(1, 4, 8)), h(1, 4, 8)),
            lambda: o.gated_forward(h(1, 3, 8), h(1, 4, 8), g(h(1, 4, 8))),
            lambda: o.gated_backward(g(h(1, 3, 4)), h(1, 3, 8), h(1, 4, 8), h(1, 4, 8), f(1, 3, 2, 8)),
            lambda: o.gated_backward(h(1, 3, 4), h(1, 3, 8), h(1, 4, 8), h(1, 4, 8), g(f(1, 3, 2, 8))),
            lambda: o.embedding_forward(g(f(1, 5, 8)), i(1, 3)), lambda: o.embedding_backward(g(f(1, 3, 8)), i(1, 3), 5),
            lambda: o.embedding_backward(f(1, 3, 8), i(1, 3), 5, out=g(f(1, 5, 8)))]


@pytest.mark.parametrize("n", range(14))
def test_tensors_that_require_gradients_are_refused_while_torch_records(lib, n):
    call = _calls_that_would_lose_gradients()[n]
    with pytest.raises(ValueError, match="no graph"):
        call()
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):   # the next thing that is wrong with them
        call()
