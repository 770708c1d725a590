"""Distillation through the C calls where the Python functions do not go: the gradient in place of the logits, and in rows that lie apart.
Either way it has the bits of a gradient in a tensor of its own."""
import ctypes as C
import math

import pytest
import torch

import paper_2002_09539_b200 as lib
from paper_2002_09539_b200 import operators

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _call(name, *args):
    fn = getattr(operators._ops(), name)
    assert fn(*args, torch.cuda.current_stream().cuda_stream) == 0, operators._ops().olsgd_last_error(None)


def _together(x, ids, z, t, w, d):
    """olsgd_distill with a gradient in d, a view of rows like x's."""
    N, V = x.shape
    code, need = operators.DTYPES[x.dtype], C.c_size_t()
    assert operators._ops().olsgd_distill_workspace(code, N, V, 1, C.byref(need)) == 0
    ws = torch.empty(max(need.value, 1), dtype=torch.uint8, device="cuda")
    loss, stats = torch.empty(N, device="cuda"), torch.empty((N, 2), device="cuda")
    _call("olsgd_distill", x.data_ptr(), code, N, V, x.stride(0), ids.data_ptr(), z.data_ptr(), 0, ids.shape[1], t, w.data_ptr(), loss.data_ptr(), stats.data_ptr(),
          d.data_ptr(), d.stride(0), ws.data_ptr(), need.value)
    return loss, stats


def _later(x, ids, z, t, w, stats, d):
    N, V = x.shape
    _call("olsgd_distill_backward", w.data_ptr(), x.data_ptr(), operators.DTYPES[x.dtype], N, V, x.stride(0), ids.data_ptr(), z.data_ptr(), 0, ids.shape[1], t,
          stats.data_ptr(), d.data_ptr(), d.stride(0))


# (rows, logits, pairs): rows in a warp, rows that one CTA holds (few and many a CTA), with many pairs, two passes (one segment
# a row and several, one part and several)
SIZES = [(9, 10, 3), (40, 257, 20), (5, 1024, 40), (700, 1500, 8), (1300, 4000, 64), (600, 3000, 100), (500, 8200, 32), (300, 20000, 32), (200, 33000, 50), (3, 4500, 200),
         (2500, 5000, 70), (4, 66000, 32), (300, 50257, 16), (1, 400003, 256)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pitch,offset", [(0, 0), (8, 8), (3, 1), (0, 5)])
@pytest.mark.parametrize("N,V,K", SIZES)
def test_gradient_in_place_and_in_rows_apart(dtype, pitch, offset, N, V, K):
    g = torch.Generator(device="cuda")
    g.manual_seed(N + V)
    ld = V + pitch
    buf = (torch.randn(offset + N * ld + 16, generator=g, device="cuda") * 3).to(dtype)
    rows = lambda b: b[offset:offset + N * ld].view(N, ld)[:, :V]   # noqa: E731
    x = rows(buf)
    x[torch.rand((N, V), generator=g, device="cuda") < 0.1] = -math.inf
    ids = torch.randint(-1, V, (N, K), generator=g, device="cuda", dtype=torch.int32)   # (some are none, some tokens occur several times)
    ids[:, K // 2] = ids[:, 0]
    z, w, t = torch.randn((N, K), generator=g, device="cuda"), torch.randn(N, generator=g, device="cuda"), 1.5
    w[N // 2] = 0.0
    want = lib.distill_loss(x, ids, z, t, d_loss=w)
    stats = lib.distill_loss(x, ids, z, t).stats
    later = lib.distill_backward(w, x, ids, z, stats, t)
    # in place of the logits
    both = buf.clone()
    loss, got = _together(rows(both), ids, z, t, w, rows(both))
    assert torch.equal(loss, want.loss) and torch.equal(got, want.stats) and torch.equal(rows(both), want.d_logits)
    alone = buf.clone()
    _later(rows(alone), ids, z, t, w, stats, rows(alone))
    assert torch.equal(rows(alone), later)
    # in rows further apart than the logits', and not aligned as they are
    far = V + pitch + 5
    apart = torch.full((3 + N * far,), 7.0, dtype=dtype, device="cuda")
    d = apart[3:].view(N, far)
    _together(x, ids, z, t, w, d[:, :V])
    assert torch.equal(d[:, :V], want.d_logits) and bool((d[:, V:] == 7).all()) and bool((apart[:3] == 7).all())
    apart.fill_(7.0)
    _later(x, ids, z, t, w, stats, d[:, :V])
    assert torch.equal(d[:, :V], later) and bool((d[:, V:] == 7).all()) and bool((apart[:3] == 7).all())
    # nothing but the rows was written
    for b in (both, alone):
        rows(b).copy_(x)
        assert torch.equal(b.view(torch.uint8), buf.view(torch.uint8))
    lib.operators_join()
