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


# ---------------------------------------------------------------------- gated feed-forward block
_G = dict(m=2, T=8, D=64, F=32, dtype=1, act=0, x=P, xw=512, xr=64, g=P, gw=2048, gr=64, u=P, uw=2048, ur=64, h=P, pre=P, dh=P, dhw=256,
          dhr=32, dx=P, dwg=P, dwu=P, ws=P, ws_bytes=1 << 30)


def _gated(lib, backward, **kw):
    a = dict(_G, **kw)
    head = [a["m"], a["T"], a["D"], a["F"], a["dtype"], a["act"]]
    mats = [a[k] for k in ("x", "xw", "xr", "g", "gw", "gr", "u", "uw", "ur")]
    if not backward:
        return lib.olsgd_gated_forward(*head, *mats, a["h"], a["pre"], a["ws"], a["ws_bytes"], None)
    return lib.olsgd_gated_backward(*head, a["dh"], a["dhw"], a["dhr"], *mats, a["pre"], a["dx"], a["dwg"], a["dwu"], a["ws"], a["ws_bytes"],
                                    None)


_BOTH = [(dict(m=0), EINVAL, "m must"), (dict(T=-1), EINVAL, "T must"), (dict(D=0), EINVAL, "D and F"), (dict(F=(1 << 24) + 1), EINVAL, "D and F"),
         (dict(dtype=0), EINVAL, "bf16 and fp16"), (dict(act=4), EINVAL, "activation"), (dict(act=-1), EINVAL, "activation"),
         (dict(x=None), EINVAL, "x must"), (dict(g=P + 1), EINVAL, "w_gate must"), (dict(u=None), EINVAL, "w_up must"),
         (dict(xr=63), EINVAL, "x: rows"), (dict(xw=511), EINVAL, "x: workers"), (dict(ur=63), EINVAL, "w_up: rows"),
         (dict(gw=2047), EINVAL, "w_gate: workers"), (dict(pre=P + 8), EINVAL, "pre")]


@pytest.mark.parametrize("bad,status,word", _BOTH + [(dict(h=None), EINVAL, "h must"), (dict(xr=65, xw=520, ws=None), EINVAL, "workspace"),
                                                     (dict(x=P + 2, ws_bytes=100), ENOMEM, "workspace")])
def test_gated_forward_refusals(lib, bad, status, word):
    assert _gated(lib, False, **bad) == status
    assert word in _text(lib)


@pytest.mark.parametrize("bad,status,word", _BOTH + [(dict(dh=None), EINVAL, "d_h must"), (dict(dhr=31), EINVAL, "d_h: rows"), (dict(pre=None), EINVAL, "pre"),
                                                     (dict(dwg=None), EINVAL, "both or neither"), (dict(dx=P + 1), EINVAL, "d_x"),
                                                     (dict(ws=None), EINVAL, "workspace"), (dict(ws_bytes=100), ENOMEM, "workspace")])
def test_gated_backward_refusals(lib, bad, status, word):
    assert _gated(lib, True, **bad) == status
    assert word in _text(lib)


def test_gated_calls_that_have_nothing_to_do(lib):
    assert _gated(lib, False, T=0, x=None, h=None) == 0
    assert _gated(lib, True, T=0, x=None, dx=None, dwg=None, dwu=None) == 0
    assert _gated(lib, True, dx=None, dwg=None, dwu=None) == 0


# -------------------------------------------------------------------------- embedding lookup
_E = dict(m=2, T=8, V=100, D=64, dtype=0, table=P, tw=6400, tr=64, ids=P, out=P, dout=P, dw=512, dr=64, odt=0, ow=6400, ws=P, ws_bytes=1 << 30)


def _embedding(lib, backward, **kw):
    a = dict(_E, **kw)
    if not backward:
        return lib.olsgd_embedding_forward(a["m"], a["T"], a["V"], a["D"], a["dtype"], a["table"], a["tw"], a["tr"], a["ids"], 1.0, a["out"], None)
    return lib.olsgd_embedding_backward(a["m"], a["T"], a["V"], a["D"], a["dtype"], a["dout"], a["dw"], a["dr"], a["ids"], 1.0, a["odt"],
                                        a["out"], a["ow"], a["ws"], a["ws_bytes"], None)


_EBOTH = [(dict(m=0), EINVAL, "m must"), (dict(T=-1), EINVAL, "T must"), (dict(T=(1 << 24) + 1), EINVAL, "T must"), (dict(V=0), EINVAL, "V and D"),
          (dict(D=0), EINVAL, "V and D"), (dict(dtype=3), EINVAL, "type"), (dict(ids=None), EINVAL, "ids"), (dict(out=P + 2), EINVAL, "aligned")]


@pytest.mark.parametrize("bad,status,word", _EBOTH + [(dict(table=None), EINVAL, "table"), (dict(tr=63), EINVAL, "table: rows"), (dict(tw=6399), EINVAL, "table: workers")])
def test_embedding_forward_refusals(lib, bad, status, word):
    assert _embedding(lib, False, **bad) == status
    assert word in _text(lib)


@pytest.mark.parametrize("bad,status,word", _EBOTH + [(dict(dout=None), EINVAL, "d_out"), (dict(dr=63), EINVAL, "d_out: rows"), (dict(odt=3), EINVAL, "type"),
                                                      (dict(ow=6399), EINVAL, "d_table: workers"), (dict(ws=P + 8), EINVAL, "workspace"),
                                                      (dict(ws_bytes=64), ENOMEM, "workspace")])
def test_embedding_backward_refusals(lib, bad, status, word):
    assert _embedding(lib, True, **bad) == status
    assert word in _text(lib)


def test_embedding_lookup_of_no_tokens_is_no_error(lib):
    assert _embedding(lib, False, T=0, table=None, ids=None, out=None) == 0
