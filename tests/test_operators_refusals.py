"""More refusals of the operators on caller-owned tensors that the host finds by itself, without a GPU."""
import pytest

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
