"""Refusals of the operators on caller-owned tensors: they are found on the host, before anything is launched, so
that they can be driven with made-up pointers and no GPU."""
import ctypes as C

import pytest

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


# -------------------------------------------------------------------- token log probabilities
_LP = dict(logits=P, dtype=1, rows=4, V=5000, ld=5000, targets=P, top=3, logp=P, entropy=P, stats=P, top_logp=P, top_ids=P,
           ws=P, ws_bytes=1 << 30)


def _logprobs(lib, **kw):
    a = dict(_LP, **kw)
    return lib.olsgd_token_logprobs(a["logits"], a["dtype"], a["rows"], a["V"], a["ld"], a["targets"], a["top"], a["logp"],
                                    a["entropy"], a["stats"], a["top_logp"], a["top_ids"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("bad,status,word", [
    (dict(logits=None), EINVAL, "logits"), (dict(logits=P + 1), EINVAL, "logits"), (dict(dtype=3), EINVAL, "type"),
    (dict(dtype=-1), EINVAL, "type"), (dict(rows=-1), EINVAL, "rows"), (dict(rows=1 << 31), EINVAL, "rows"),
    (dict(V=0), EINVAL, "V"), (dict(V=(1 << 27) + 1), EINVAL, "V"), (dict(ld=4999), EINVAL, "row_stride"),
    (dict(targets=None), EINVAL, "targets"), (dict(targets=P + 2), EINVAL, "targets"), (dict(top=33), EINVAL, "top"),
    (dict(top=-1), EINVAL, "top"), (dict(V=2, top=3), EINVAL, "top"), (dict(logp=None), EINVAL, "logp"),
    (dict(stats=P + 1), EINVAL, "stats"), (dict(top_ids=None), EINVAL, "top_ids"), (dict(ws=None), EINVAL, "workspace"),
    (dict(ws=P + 16), EINVAL, "workspace"), (dict(ws_bytes=8), ENOMEM, "workspace")])
def test_token_logprobs_refusals(lib, bad, status, word):
    assert _logprobs(lib, **bad) == status
    assert word in _text(lib)


def test_token_logprobs_of_no_rows_is_no_error(lib):
    assert _logprobs(lib, rows=0, logits=None, targets=None) == 0


@pytest.mark.parametrize("bad,word", [
    (dict(logits=None), "logits"), (dict(out=P + 1), "d_logits"), (dict(ldd=4999), "d_row_stride"), (dict(stats=None), "stats"),
    (dict(out=P, logits=P, ld=5008), "in place"), (dict(dlp=P + 1), "d_logp"), (dict(dtype=7), "type")])
def test_token_logprobs_backward_refusals(lib, bad, word):
    a = dict(dlp=P, dh=P, logits=P, dtype=1, rows=4, V=5000, ld=5000, targets=P, stats=P, entropy=P, out=2 * P, ldd=5000)
    a.update(bad)
    assert lib.olsgd_token_logprobs_backward(a["dlp"], a["dh"], a["logits"], a["dtype"], a["rows"], a["V"], a["ld"], a["targets"],
                                             a["stats"], a["entropy"], a["out"], a["ldd"], None) == EINVAL
    assert word in _text(lib)


# -------------------------------------------------------------------------- gradient clipping
def _clip(lib, tensors=((P, 2 * P, 100, 100, 100, 0, 0),), count=None, m=4, max_norm=1.0, norms=P, ws=P, ws_bytes=1 << 30):
    flat = []
    for a, b, n, s, t, i, o in tensors:
        flat += [a, b, n, s, t, (i & 0xFFFFFFFF) | (o << 32)]
    table = (C.c_int64 * max(1, len(flat)))(*flat)
    return lib.olsgd_clip_grads(table, len(tensors) if count is None else count, m, max_norm, norms, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,status,word", [
    (dict(m=0), EINVAL, "m must"), (dict(m=65536), EINVAL, "m must"), (dict(count=-1), EINVAL, "n_tensors"),
    (dict(max_norm=0.0), EINVAL, "max_norm"), (dict(max_norm=-1.0), EINVAL, "max_norm"), (dict(max_norm=float("nan")), EINVAL, "max_norm"),
    (dict(max_norm=float("inf")), EINVAL, "max_norm"), (dict(norms=None), EINVAL, "norms"), (dict(ws=None), EINVAL, "workspace"),
    (dict(ws_bytes=4), ENOMEM, "workspace"),
    (dict(tensors=((0, P, 100, 100, 100, 0, 0),)), EINVAL, "tensor 0"),
    (dict(tensors=((P, 2 * P, 100, 100, 100, 0, 0), (P, 2 * P + 2, 100, 100, 100, 1, 0))), EINVAL, "tensor 1"),
    (dict(tensors=((P, 2 * P, 100, 99, 100, 0, 0),)), EINVAL, "strides"),
    (dict(tensors=((P, 2 * P, 100, 100, 99, 0, 0),)), EINVAL, "strides"),
    (dict(tensors=((P, 2 * P, -1, 100, 100, 0, 0),)), EINVAL, "n must"),
    (dict(tensors=((P, 2 * P, 100, 100, 100, 5, 0),)), EINVAL, "type"),
    (dict(tensors=((P, P, 100, 100, 100, 1, 0),)), EINVAL, "in place"),
    (dict(tensors=((P, P, 100, 100, 128, 0, 0),)), EINVAL, "in place")])
def test_clip_grads_refusals(lib, bad, status, word):
    assert _clip(lib, **bad) == status
    assert word in _text(lib)


def test_clip_grads_of_no_tensors_is_no_error(lib):
    assert _clip(lib, count=0) == 0
