"""Products by expert where a group's rows end: along K, where the rows that follow in memory, and what an earlier call left in shared
memory, must not be summed.  Tolerances count roundings, U = 2^-24 being half a step of fp32."""
import math

import pytest
import torch

import paper_2002_09539_b200 as lib

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


# widths that take tiles of 128 and 256 features by 64, 128 and 256 columns; whole panels, 16-byte rows and rows of any alignment
@pytest.mark.parametrize("D,F,scale", [(64, 128, 1), (136, 72, 1), (256, 256, 3), (512, 1024, 1), (333, 201, 2), (1024, 512, 9)])
def test_weights_gradient_of_groups_of_every_length_up_to_two_blocks(D, F, scale):
    """Groups of scale, 2 scale, ... rows, so that their last blocks end everywhere.  The rows of a group are far from its neighbours'
    in size and its products are whole numbers: one row too many, or too few, is no rounding."""
    g = _gen(D + F)
    E, dtype = 129, torch.bfloat16
    sizes = [scale * e for e in range(E)]
    R = sum(sizes)
    ends = torch.tensor([0] + sizes, device="cuda").cumsum(0)
    offsets = ends.to(torch.int32)[None]
    group = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.tensor(sizes, device="cuda"))
    # whole numbers up to 3 times a power of two of the group: every sum is exact in fp32 (at most 1161 * 9 in units of that power)
    unit = 2.0 ** (6 * (group % 3)).double()
    x = (torch.randint(-3, 4, (1, R, D), generator=g, device="cuda") * unit[None, :, None]).to(dtype)
    dy = torch.randint(-3, 4, (1, R, F), generator=g, device="cuda").to(dtype)
    w = torch.zeros((1, E, F, D), dtype=dtype, device="cuda")
    want = torch.zeros((E, F, D), dtype=torch.float64, device="cuda")
    for e in range(E):
        part = slice(int(ends[e]), int(ends[e + 1]))
        want[e] = dy[0, part].double().T @ x[0, part].double()
    want = want.to(dtype)   # (one rounding of an exact sum: the same bits)
    nan = torch.full_like(x, math.nan), torch.full_like(dy, math.nan)
    for _ in range(20):
        lib.expert_product_backward(nan[1], nan[0], w, offsets)   # what is left behind in shared memory
        got = lib.expert_product_backward(dy, x, w, offsets, want_d_x=False)[1]
        beside = lib.expert_product_backward(dy, x, w, offsets)[1]
        assert torch.equal(got[0], want) and torch.equal(beside, got)
    lib.operators_join()
