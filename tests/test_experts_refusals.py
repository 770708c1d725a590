"""Refusals of routing, products by expert, their combination and distillation: found on the host, before anything is launched, so that
they can be driven with made-up pointers and no GPU."""
import ctypes as C

import pytest
import torch

from paper_2002_09539_b200 import operators
from paper_2002_09539_b200.build import build

P = 1 << 20   # an aligned address that nothing dereferences
EINVAL, ENOMEM = 1, 3


@pytest.fixture(scope="module")
def lib():
    build()
    return operators._ops()


def _text(lib):
    return lib.olsgd_last_error(None).decode()


def _expect(lib, got, status, word):
    assert got == status
    assert word in _text(lib)


# ------------------------------------------------------------------------------------ routing

def _route(lib, **kw):
    a = dict(m=2, T=70000, E=64, dtype=0, logits=P, ld=64, k=4, weights=P, ids=P, places=P, tokens=P, offsets=P, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.olsgd_expert_route(a["m"], a["T"], a["E"], a["dtype"], a["logits"], a["ld"], a["k"], 1, a["weights"], a["ids"], a["places"],
                                  a["tokens"], a["offsets"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("bad,status,word", [
    (dict(m=0), EINVAL, "m must"), (dict(m=65536), EINVAL, "m must"), (dict(T=-1), EINVAL, "T must"), (dict(T=(1 << 24) + 1), EINVAL, "T must"),
    (dict(E=0), EINVAL, "E must"), (dict(E=1025), EINVAL, "E must"), (dict(dtype=3), EINVAL, "type"), (dict(k=0), EINVAL, "k must"),
    (dict(k=33), EINVAL, "k must"), (dict(E=3, k=4), EINVAL, "k must"), (dict(ld=63), EINVAL, "row_stride"), (dict(logits=None), EINVAL, "logits"),
    (dict(logits=P + 2), EINVAL, "logits"), (dict(weights=None), EINVAL, "weights"), (dict(ids=P + 1), EINVAL, "ids"),
    (dict(places=None), EINVAL, "places"), (dict(tokens=None), EINVAL, "tokens"), (dict(offsets=None), EINVAL, "offsets"),
    (dict(ws=None), EINVAL, "workspace"), (dict(ws_bytes=16), ENOMEM, "workspace")])
def test_route_refusals(lib, bad, status, word):
    _expect(lib, _route(lib, **bad), status, word)


@pytest.mark.parametrize("bad,word", [(dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(E=0), "E must"), (dict(k=9), "k must"), (dict(dtype=5), "type"),
                                      (dict(dw=None), "d_weights"), (dict(ids=None), "ids"), (dict(w=P + 1), "weights"), (dict(out=None), "d_logits"),
                                      (dict(out=P), "d_logits"), (dict(logits=None), "logits"), (dict(ld=7), "row_stride")])
def test_route_backward_refusals(lib, bad, word):
    a = dict(rows=5, E=8, dtype=0, dw=P, logits=P, ld=8, k=2, ids=P, w=P, out=2 * P)
    a.update(bad)
    _expect(lib, lib.olsgd_expert_route_backward(a["rows"], a["E"], a["dtype"], a["dw"], a["logits"], a["ld"], a["k"], 0, a["ids"], a["w"], a["out"], None),
            EINVAL, word)


# ----------------------------------------------------------------------------------- combining

def _combine(lib, backward=False, **kw):
    a = dict(m=2, T=9, k=2, R=18, D=64, dtype=1, dy=P, rows=P, sw=18 * 64, sr=64, places=P, tokens=P, w=P, y=P, dw=P)
    a.update(kw)
    if backward:
        return lib.olsgd_expert_combine_backward(a["m"], a["T"], a["k"], a["R"], a["D"], a["dtype"], a["dy"], 9 * 64, 64, a["rows"], a["sw"], a["sr"],
                                                 a["places"], a["tokens"], a["w"], a["y"], a["dw"], None)
    return lib.olsgd_expert_combine(a["m"], a["T"], a["k"], a["R"], a["D"], a["dtype"], a["rows"], a["sw"], a["sr"], a["places"], a["w"], a["y"], None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad,word", [(dict(m=0), "m must"), (dict(T=-1), "T k"), (dict(k=0), "k must"), (dict(T=1 << 30, k=2), "T k"), (dict(R=-1), "R at most"),
                                      (dict(D=0), "D must"), (dict(dtype=9), "type"), (dict(rows=None), "rows"), (dict(rows=P + 1), "rows"),
                                      (dict(sr=63), "overlap"), (dict(sw=17 * 64), "overlap"), (dict(places=None), "places"), (dict(w=P + 2), "weights"),
                                      (dict(y=None), "must be non-null")])
def test_combine_refusals(lib, backward, bad, word):
    _expect(lib, _combine(lib, backward, **bad), EINVAL, word)


@pytest.mark.parametrize("bad,word", [(dict(dy=None), "d_y"), (dict(tokens=None), "tokens"), (dict(dw=None), "d_weights"), (dict(w=None), "weights")])
def test_combine_backward_refusals(lib, bad, word):
    _expect(lib, _combine(lib, True, **bad), EINVAL, word)


# ------------------------------------------------------------------------------------ products

def _product(lib, backward=False, **kw):
    m, R, E, D, F = (kw.pop(n, v) for n, v in (("m", 2), ("R", 40), ("E", 3), ("D", 64), ("F", 32)))
    a = dict(dtype=1, dy=P, x=P, xs=(40 * 64, 64), w=P, ws=(3 * 32 * 64, 32 * 64, 64), offsets=P, y=P, dw=P, work=P, bytes=1 << 30)
    a.update(kw)
    if backward:
        return lib.olsgd_expert_product_backward(m, R, E, D, F, a["dtype"], a["dy"], 40 * 32, 32, a["x"], *a["xs"], a["w"], *a["ws"], a["offsets"], a["y"],
                                                 a["dw"], a["work"], a["bytes"], None)
    return lib.olsgd_expert_product(m, R, E, D, F, a["dtype"], a["x"], *a["xs"], a["w"], *a["ws"], a["offsets"], a["y"], a["work"], a["bytes"], None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad,word", [
    (dict(m=0), "m must"), (dict(E=0), "E must"), (dict(E=1025), "E must"), (dict(m=70, E=1000), "m E"), (dict(R=-1), "R must"), (dict(R=1 << 30, m=3), "m R"),
    (dict(D=0), "D and F"), (dict(F=(1 << 24) + 1), "D and F"), (dict(dtype=0), "bf16 and fp16"), (dict(x=None), "x must"), (dict(x=P + 1), "x must"),
    (dict(xs=(40 * 64, 63)), "x: rows"), (dict(xs=(39 * 64, 64)), "x: workers"), (dict(w=None), "w must"), (dict(ws=(3 * 32 * 64, 32 * 64, 60)), "w: rows"),
    (dict(ws=(3 * 32 * 64, 31 * 64, 64)), "w: "), (dict(ws=(2 * 32 * 64, 32 * 64, 64)), "w: workers"), (dict(offsets=None), "offsets"), (dict(offsets=P + 2), "offsets"),
    (dict(y=P + 1), "aligned")])
def test_product_refusals(lib, backward, bad, word):
    _expect(lib, _product(lib, backward, **bad), EINVAL, word)


def test_product_refuses_small_workspaces(lib):
    _expect(lib, _product(lib, x=P + 2, work=None), EINVAL, "workspace")      # copies are needed
    _expect(lib, _product(lib, x=P + 2, bytes=64), ENOMEM, "workspace")
    _expect(lib, _product(lib, True, x=P + 2, bytes=64), ENOMEM, "workspace")
    _expect(lib, _product(lib, True, dy=P + 2, work=P + 8), EINVAL, "workspace")
    _expect(lib, _product(lib, True, dy=None), EINVAL, "d_y must")
    assert _product(lib, True, y=None, dw=None, work=None) == 0               # nothing is wanted
    n = C.c_size_t()
    for backward in (0, 1):
        assert lib.olsgd_expert_product_workspace(2, 40, 3, 64, 32, backward, 1, C.byref(n)) == 0 and n.value == 0
    assert lib.olsgd_expert_product_workspace(2, 0, 3, 64, 32, 1, 0, C.byref(n)) == 0 and n.value == 0
    assert lib.olsgd_expert_product_workspace(2, 40, 3, 64, 32, 1, 1, None) == EINVAL


# -------------------------------------------------------------------------------- distillation

def _distill(lib, backward=False, **kw):
    a = dict(logits=P, dtype=1, rows=4, V=5000, ld=5000, ids=P, teacher=P, tdtype=0, K=8, t=1.0, d_loss=P, loss=P, stats=P, out=2 * P, ldd=5000, ws=P,
             bytes=1 << 30)
    a.update(kw)
    if backward:
        return lib.olsgd_distill_backward(a["d_loss"], a["logits"], a["dtype"], a["rows"], a["V"], a["ld"], a["ids"], a["teacher"], a["tdtype"], a["K"], a["t"],
                                          a["stats"], a["out"], a["ldd"], None)
    return lib.olsgd_distill(a["logits"], a["dtype"], a["rows"], a["V"], a["ld"], a["ids"], a["teacher"], a["tdtype"], a["K"], a["t"], a["d_loss"], a["loss"],
                             a["stats"], a["out"], a["ldd"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad,word", [
    (dict(dtype=3), "type"), (dict(rows=-1), "rows"), (dict(V=0), "V must"), (dict(V=(1 << 27) + 1), "V must"), (dict(ld=4999), "row_stride"),
    (dict(logits=None), "logits"), (dict(logits=P + 1), "logits"), (dict(ids=None), "ids"), (dict(ids=P + 2), "ids"), (dict(teacher=None), "teacher"),
    (dict(teacher=P + 2), "teacher"), (dict(tdtype=4), "type"), (dict(K=0), "K must"), (dict(K=257), "K must"), (dict(t=0.0), "temperature"),
    (dict(t=-1.0), "temperature"), (dict(t=float("nan")), "temperature"), (dict(t=float("inf")), "temperature"), (dict(t=1e-9), "temperature"),
    (dict(stats=None), "stats"), (dict(out=None), "d_logits"), (dict(ldd=4999), "d_row_stride"), (dict(out=P, ld=5008), "in place"), (dict(d_loss=P + 1), "d_loss")])
def test_distill_refusals(lib, backward, bad, word):
    _expect(lib, _distill(lib, backward, **bad), EINVAL, word)


def test_distill_workspaces_and_no_rows(lib):
    _expect(lib, _distill(lib, d_loss=None, out=None, V=200000, ld=200000, ws=None), EINVAL, "workspace")
    _expect(lib, _distill(lib, d_loss=None, out=None, V=200000, ld=200000, bytes=8), ENOMEM, "workspace")
    _expect(lib, _distill(lib, loss=None), EINVAL, "loss")
    _expect(lib, _distill(lib, True, d_loss=None), EINVAL, "d_loss")
    assert _distill(lib, rows=0, logits=None, ids=None, teacher=None, loss=None) == 0 and _distill(lib, True, rows=0, logits=None) == 0


# ------------------------------------------------------------------------------- the Python layer

def _calls_that_would_lose_gradients():
    f, h, i = (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.bfloat16)), (lambda *s: torch.zeros(s, dtype=torch.int32))
    g = lambda t: t.requires_grad_()   # noqa: E731
    o = operators
    return [lambda: o.expert_route(g(f(1, 3, 4)), 2), lambda: o.expert_route_backward(g(f(1, 3, 2)), f(1, 3, 4), i(1, 3, 2), f(1, 3, 2)),
            lambda: o.expert_route_backward(f(1, 3, 2), f(1, 3, 4), i(1, 3, 2), g(f(1, 3, 2))),
            lambda: o.expert_combine(g(h(1, 6, 8)), i(1, 3, 2)), lambda: o.expert_combine(h(1, 6, 8), i(1, 3, 2), g(f(1, 3, 2))),
            lambda: o.expert_combine_backward(g(h(1, 3, 8)), h(1, 6, 8), i(1, 3, 2), i(1, 6), f(1, 3, 2)),
            lambda: o.expert_product(g(h(1, 6, 8)), h(1, 2, 4, 8), i(1, 3)), lambda: o.expert_product(h(1, 6, 8), g(h(1, 2, 4, 8)), i(1, 3)),
            lambda: o.expert_product_backward(g(h(1, 6, 4)), h(1, 6, 8), h(1, 2, 4, 8), i(1, 3)),
            lambda: o.distill_loss(g(f(2, 9)), i(2, 3), f(2, 3)), lambda: o.distill_loss(f(2, 9), i(2, 3), g(f(2, 3))),
            lambda: o.distill_loss(f(2, 9), i(2, 3), f(2, 3), d_loss=g(f(2))), lambda: o.distill_backward(g(f(2)), f(2, 9), i(2, 3), f(2, 3), f(2, 2))]


@pytest.mark.parametrize("n", range(13))
def test_tensors_that_require_gradients_are_refused_while_torch_records(lib, n):
    call = _calls_that_would_lose_gradients()[n]
    with pytest.raises(ValueError, match="no graph"):
        call()
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):   # the next thing that is wrong with them
        call()
