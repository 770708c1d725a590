"""Operators on caller-owned tensors (the section of that name in include/olsgd.h): argument
checks and marshalling only, like `binding`.

They serve a caller that computes its own gradients for `OverlapLocalSGD("flat", ...)`: tensors
carry the worker dimension first.  Every call runs on the current stream of its tensors'
device, allocates its outputs and workspace with torch (so it may be captured into a CUDA
graph), and returns without waiting.  Tensors that live on another stream are the caller's to
order, as with any torch operation.  Forward and backward are separate calls; nothing is kept
between them but what the caller passes on.
"""
import ctypes as C
import functools
from collections import namedtuple

import torch

from .binding import _check, load_library

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}
MAX_TOP = 32

TokenLogprobs = namedtuple("TokenLogprobs", "logp entropy stats top_logp top_ids")

_vp, _i32, _i64, _sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
_SIGNATURES = {
    "olsgd_token_logprobs_workspace": [_i32, _i64, _i64, _i32, C.POINTER(_sz)],
    "olsgd_token_logprobs": [_vp, _i32, _i64, _i64, _i64, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "olsgd_token_logprobs_backward": [_vp, _vp, _vp, _i32, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _vp],
    "olsgd_clip_grads_workspace": [_i32, _i32, C.POINTER(_sz)],
    "olsgd_gated_workspace": [_i32, _i64, _i64, _i64, _i32, _i32, C.POINTER(_sz)],
    "olsgd_gated_forward": [_i32, _i64, _i64, _i64, _i32, _i32] + 3 * [_vp, _i64, _i64] + [_vp, _vp, _vp, _sz, _vp],
    "olsgd_gated_backward": [_i32, _i64, _i64, _i64, _i32, _i32] + 4 * [_vp, _i64, _i64] + [_vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "olsgd_embedding_forward": [_i32, _i64, _i64, _i64, _i32, _vp, _i64, _i64, _vp, C.c_float, _vp, _vp],
    "olsgd_embedding_workspace": [_i32, _i64, _i64, C.POINTER(_sz)],
    "olsgd_embedding_backward": [_i32, _i64, _i64, _i64, _i32, _vp, _i64, _i64, _vp, C.c_float, _i32, _vp, _i64, _vp, _sz, _vp],
    "olsgd_operators_join": [_vp],
    "olsgd_clip_grads": [_vp, _i32, _i32, C.c_float, _vp, _vp, _sz, _vp],
}
_OPS = None


def _ops():
    global _OPS
    if _OPS is None:
        lib = load_library()
        for name, args in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = _i32, args
        _OPS = lib
    return _OPS


def _need(ok, text, *args):
    if not ok:
        raise ValueError(text % args if args else text)


def _dtype(t, name):
    code = DTYPES.get(t.dtype)
    _need(code is not None, "%s must be float32, bfloat16 or float16", name)
    return code


def _same_device(dev, **tensors):
    for name, t in tensors.items():
        _need(t is None or t.device == dev, "%s must be on %s", name, dev)


def _stream(index):
    return torch.cuda.current_stream(index).cuda_stream


# the same number without the Stream object around it (2 us a call)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream)


def _run(fn, dev, *args):
    """fn(*args, stream) on the tensors' device and its current stream."""
    if torch.cuda.current_device() == dev.index:
        st = fn(*args, _stream(dev.index))
    else:
        with torch.cuda.device(dev):
            st = fn(*args, _stream(dev.index))
    if st:
        _check(_ops(), st)


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(query, *sizes):
    n = _sz()
    _check(_ops(), getattr(_ops(), query)(*sizes, C.byref(n)))
    return n.value


def _workspace(dev, query, *sizes):
    """(tensor, pointer, bytes) of a fresh workspace; torch's allocations are 512-byte aligned."""
    n = _workspace_bytes(query, *sizes)
    if n == 0:
        return None, None, 0
    ws = torch.empty(n, dtype=torch.uint8, device=dev)
    return ws, ws.data_ptr(), n


# ------------------------------------------------------------------ token log probabilities

def _rows_of(t, name):
    """(view [N][V], stride between rows) of a tensor [..., V] whose rows are evenly spaced."""
    _need(t.dim() >= 1 and t.is_cuda, "%s must be a CUDA tensor with at least one dimension", name)
    V = t.shape[-1]
    _need(V >= 1 and (t.stride(-1) == 1 or V == 1), "%s: the last dimension must be contiguous and not empty", name)
    if t.dim() != 2:   # (one launch takes rows at one distance)
        try:
            t = t.view(-1, V)
        except RuntimeError:
            raise ValueError("%s: rows must be evenly spaced" % name) from None
    return t, (t.stride(0) if t.shape[0] > 1 else V)


def _per_row(t, shape, dtype, name):
    _need(t.dtype == dtype and t.shape == shape and t.is_contiguous(), "%s must be contiguous %s of shape %s", name, dtype,
          tuple(shape))
    return t.data_ptr()


def token_logprobs(logits, targets, top=0):
    """olsgd_token_logprobs.  logits [..., V] (rows evenly spaced), targets int32 [...]; a target outside
    [0, V) is a row without a token.  Returns TokenLogprobs(logp, entropy, stats, top_logp, top_ids): float32
    [...], [...], [..., 2], [..., top] and int32 [..., top] (the last two None when top == 0)."""
    lib = _ops()
    rows, ld = _rows_of(logits, "logits")
    code, dev, lead = _dtype(logits, "logits"), logits.device, logits.shape[:-1]
    _same_device(dev, targets=targets)
    tp = _per_row(targets, lead, torch.int32, "targets")
    N, V = rows.shape
    top = int(top)
    _need(0 <= top <= min(V, MAX_TOP), "top must be in [0, min(V, %d)]", MAX_TOP)
    # the float outputs share one allocation: a small call is mostly the time that the host takes
    out = torch.empty(N * (4 + top), dtype=torch.float32, device=dev)
    logp, entropy, stats, top_logp = out.split((N, N, 2 * N, top * N))
    top_ids = torch.empty(lead + (top,), dtype=torch.int32, device=dev) if top else None
    ws, wp, wn = _workspace(dev, "olsgd_token_logprobs_workspace", code, N, V, top)
    p = out.data_ptr()
    _run(lib.olsgd_token_logprobs, dev, rows.data_ptr(), code, N, V, ld, tp, top, p, p + 4 * N, p + 8 * N, p + 16 * N if top else None,
         top_ids.data_ptr() if top else None, wp, wn)
    if len(lead) != 1:
        logp, entropy = logp.view(lead), entropy.view(lead)
    return TokenLogprobs(logp, entropy, stats.view(lead + (2,)), top_logp.view(lead + (top,)) if top else None, top_ids)


def token_logprobs_backward(d_logp, d_entropy, logits, targets, stats, entropy):
    """olsgd_token_logprobs_backward: the gradient of the logits, contiguous, of their type.  d_logp and d_entropy
    are float32 [...] or None (zeros); stats and entropy are token_logprobs' for the same logits."""
    lib = _ops()
    rows, ld = _rows_of(logits, "logits")
    code, dev, lead = _dtype(logits, "logits"), logits.device, logits.shape[:-1]
    _same_device(dev, targets=targets, stats=stats, entropy=entropy, d_logp=d_logp, d_entropy=d_entropy)
    N, V = rows.shape
    d = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
    _run(lib.olsgd_token_logprobs_backward, dev,
         None if d_logp is None else _per_row(d_logp, lead, torch.float32, "d_logp"),
         None if d_entropy is None else _per_row(d_entropy, lead, torch.float32, "d_entropy"),
         rows.data_ptr(), code, N, V, ld, _per_row(targets, lead, torch.int32, "targets"),
         _per_row(stats, lead + (2,), torch.float32, "stats"), _per_row(entropy, lead, torch.float32, "entropy"),
         d.data_ptr(), V)
    return d


# ------------------------------------------------------------------------ gradient clipping

def _worker_rows(t, m, name):
    """Elements between workers of a tensor [m, ...] whose workers' parts are contiguous."""
    _need(t.dim() >= 1 and t.shape[0] == m, "%s must have %s workers", name, m)
    n = t.numel() // m
    if t.is_contiguous():
        return n, n
    _need(t[0].is_contiguous(), "%s: each worker's part must be contiguous", name)
    return n, t.stride(0)


def clip_grads(grads, max_norm, out=None):
    """olsgd_clip_grads.  grads: a tensor or a list of tensors [m, ...], each worker's part contiguous.  Each worker's
    gradients, over all tensors, are scaled by min(1, max_norm / (norm + 1e-6)).  out: tensors of the same shapes, of any
    of the three types, that take the result (the gradients themselves: in place; views of a flat float32 gradient [m][P]:
    widened into it); None: new tensors like the gradients.  Returns (out, norms), norms float32 [m]."""
    lib = _ops()
    single = isinstance(grads, torch.Tensor)
    if single:
        grads, out = [grads], None if out is None else [out]
    _need(len(grads) > 0, "grads is empty")
    if out is None:
        out = [torch.empty(g.shape, dtype=g.dtype, device=g.device) for g in grads]
    _need(len(out) == len(grads), "out must hold one tensor for each gradient")
    m, dev = grads[0].shape[0] if grads[0].dim() else 0, grads[0].device
    _need(dev.type == "cuda" and m >= 1, "grads must be CUDA tensors with the workers first")
    flat = []
    for g, o in zip(grads, out):
        gc, oc = DTYPES.get(g.dtype), DTYPES.get(o.dtype)
        _need(gc is not None and oc is not None, "gradients and out must be float32, bfloat16 or float16")
        _need(g.shape == o.shape and g.device == dev and o.device == dev, "gradients and out must match in shape and device")
        n, gs = _worker_rows(g, m, "a gradient")
        _, os_ = _worker_rows(o, m, "out")
        flat += (g.data_ptr(), o.data_ptr(), n, gs, os_, gc | (oc << 32))
    table = (_i64 * len(flat))(*flat)
    norms = torch.empty(m, dtype=torch.float32, device=dev)
    ws, wp, wn = _workspace(dev, "olsgd_clip_grads_workspace", m, len(grads))
    _run(lib.olsgd_clip_grads, dev, table, len(grads), m, float(max_norm), norms.data_ptr(), wp, wn)
    return (out[0] if single else out), norms


# ---------------------------------------------------------------------- gated feed-forward block

def _matrix(t, name, shape, dtype, dev):
    """(pointer, worker stride, row stride) of a tensor [m][rows][cols] with contiguous rows."""
    _need(t.shape == shape and t.dtype == dtype and t.device == dev, "%s must be %s of shape %s on %s", name, dtype, tuple(shape), dev)
    sw, sr, sc = t.stride()
    _need(sc == 1 or shape[2] == 1, "%s: the last dimension must be contiguous", name)
    return t.data_ptr(), sw, sr


def _aligned(matrix, shape):
    p, sw, sr = matrix
    return p % 16 == 0 and (shape[0] == 1 or sw % 8 == 0) and (shape[1] == 1 or sr % 8 == 0)


def _gated_sizes(x, w_gate, activation):
    _need(x.is_cuda and x.dim() == 3 and w_gate.dim() == 3, "x and w_gate must be CUDA tensors [m][T][D] and [m][F][D]")
    _need(x.dtype in (torch.bfloat16, torch.float16), "x must be bfloat16 or float16")
    _need(activation in ACTIVATIONS, "activation must be one of %s", sorted(ACTIVATIONS))
    m, T, D = x.shape
    return m, T, D, w_gate.shape[1], DTYPES[x.dtype], ACTIVATIONS[activation]


def gated_forward(x, w_gate, w_up, activation="silu", save=False):
    """olsgd_gated_forward: h = act(x w_gate^T) * (x w_up^T) for each worker.  x [m][T][D], w_gate and w_up [m][F][D], bfloat16
    or float16, rows contiguous, any worker and row strides.  Returns h [m][T][F], and with save=True (h, pre), pre being what
    gated_backward takes."""
    lib = _ops()
    m, T, D, F, code, act = _gated_sizes(x, w_gate, activation)
    dtype, dev, ws_shape = x.dtype, x.device, (m, F, D)
    a, b, c = _matrix(x, "x", (m, T, D), dtype, dev), _matrix(w_gate, "w_gate", ws_shape, dtype, dev), _matrix(w_up, "w_up", ws_shape, dtype, dev)
    h = torch.empty((m, T, F), dtype=dtype, device=dev)
    pre = torch.empty((m, T, 2, (F + 7) // 8 * 8), dtype=dtype, device=dev) if save else None
    ok = _aligned(a, (m, T)) and _aligned(b, ws_shape) and _aligned(c, ws_shape)
    ws, wp, wn = _workspace(dev, "olsgd_gated_workspace", m, T, D, F, 0, ok)
    _run(lib.olsgd_gated_forward, dev, m, T, D, F, code, act, *a, *b, *c, h.data_ptr(), pre.data_ptr() if save else None, wp, wn)
    return (h, pre) if save else h


def gated_backward(d_h, x, w_gate, w_up, pre, activation="silu", want_d_x=True, want_d_w=True):
    """olsgd_gated_backward: (d_x, d_w_gate, d_w_up) from d_h [m][T][F] and the forward call's operands and pre; None for
    those not wanted."""
    lib = _ops()
    m, T, D, F, code, act = _gated_sizes(x, w_gate, activation)
    dtype, dev, ws_shape = x.dtype, x.device, (m, F, D)
    d, a = _matrix(d_h, "d_h", (m, T, F), dtype, dev), _matrix(x, "x", (m, T, D), dtype, dev)
    b, c = _matrix(w_gate, "w_gate", ws_shape, dtype, dev), _matrix(w_up, "w_up", ws_shape, dtype, dev)
    _need(pre.shape == (m, T, 2, (F + 7) // 8 * 8) and pre.dtype == dtype and pre.device == dev and pre.is_contiguous(),
          "pre must be the one that gated_forward returned")
    d_x = torch.empty((m, T, D), dtype=dtype, device=dev) if want_d_x else None
    d_wg = d_wu = None
    if want_d_w:
        d_wg, d_wu = torch.empty(ws_shape, dtype=dtype, device=dev), torch.empty(ws_shape, dtype=dtype, device=dev)
    ok = _aligned(a, (m, T)) and _aligned(b, ws_shape) and _aligned(c, ws_shape)
    ws, wp, wn = _workspace(dev, "olsgd_gated_workspace", m, T, D, F, 1, ok)
    _run(lib.olsgd_gated_backward, dev, m, T, D, F, code, act, *d, *a, *b, *c, pre.data_ptr(), d_x.data_ptr() if want_d_x else None,
         d_wg.data_ptr() if want_d_w else None, d_wu.data_ptr() if want_d_w else None, wp, wn)
    return d_x, d_wg, d_wu


# --------------------------------------------------------------------------------- embedding

def embedding_forward(table, ids, scale=1.0):
    """olsgd_embedding_forward: scale * table[i, ids[i]] for each worker i.  table [m][V][D], rows contiguous; ids int32 [m][T],
    those outside [0, V) give rows of zeros.  Returns [m][T][D] of the table's type."""
    lib = _ops()
    _need(table.is_cuda and table.dim() == 3 and ids.dim() == 2, "table must be a CUDA tensor [m][V][D], ids [m][T]")
    code, dev = _dtype(table, "table"), table.device
    m, V, D = table.shape
    T = ids.shape[1]
    _same_device(dev, ids=ids)
    p, sw, sr = _matrix(table, "table", (m, V, D), table.dtype, dev)
    out = torch.empty((m, T, D), dtype=table.dtype, device=dev)
    _run(lib.olsgd_embedding_forward, dev, m, T, V, D, code, p, sw, sr, _per_row(ids, (m, T), torch.int32, "ids"), float(scale),
         out.data_ptr())
    return out


def embedding_backward(d_out, ids, vocab, scale=1.0, dtype=torch.float32, out=None):
    """olsgd_embedding_backward: the gradient of a table [m][vocab][D] from d_out [m][T][D] and the ids of the lookup; new, of
    type `dtype`, or written to `out` (each worker's part contiguous, for example a view of a flat gradient [m][P])."""
    lib = _ops()
    _need(d_out.is_cuda and d_out.dim() == 3, "d_out must be a CUDA tensor [m][T][D]")
    code, dev = _dtype(d_out, "d_out"), d_out.device
    m, T, D = d_out.shape
    V = int(vocab)
    _same_device(dev, ids=ids, out=out)
    p, sw, sr = _matrix(d_out, "d_out", (m, T, D), d_out.dtype, dev)
    if out is None:
        out = torch.empty((m, V, D), dtype=dtype, device=dev)
    _need(out.shape == (m, V, D), "out must be of shape %s", (m, V, D))
    _, ow = _worker_rows(out, m, "out")
    ip = _per_row(ids, (m, T), torch.int32, "ids")
    ws, wp, wn = _workspace(dev, "olsgd_embedding_workspace", m, T, D)
    _run(lib.olsgd_embedding_backward, dev, m, T, V, D, code, p, sw, sr, ip, float(scale), _dtype(out, "out"), out.data_ptr(), ow, wp, wn)
    return out


def operators_join(device="cuda"):
    """olsgd_operators_join on the device's current stream: waits for it, and raises if an operator's bounded wait gave up."""
    dev = torch.device(device)
    if dev.index is None:
        dev = torch.device(dev.type, torch.cuda.current_device())
    _run(_ops().olsgd_operators_join, dev)
