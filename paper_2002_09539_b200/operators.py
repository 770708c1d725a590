"""Operators on caller-owned tensors (the section of that name in include/olsgd.h): argument
checks and marshalling only, like `binding`.

They serve a caller that computes its own gradients for `OverlapLocalSGD("flat", ...)`: tensors
carry the worker dimension first.  Every call runs on the current stream of its tensors'
device, allocates its outputs and workspace with torch (so it may be captured into a CUDA
graph), and returns without waiting.  Tensors that live on another stream are the caller's to
order, as with any torch operation.  Forward and backward are separate calls; nothing is kept
between them but what the caller passes on.  They record no graph: tensors that require
gradients are refused while torch records (detach them, or call under torch.no_grad()).
"""
import ctypes as C
import functools
import operator
from collections import namedtuple

import torch

from .binding import _check, load_library

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}
MAX_TOP = 32
MAX_EXPERTS = 1024
MAX_TEACHER = 256

TokenLogprobs = namedtuple("TokenLogprobs", "logp entropy stats top_logp top_ids")
ExpertRoute = namedtuple("ExpertRoute", "weights ids places tokens offsets")
DistillLoss = namedtuple("DistillLoss", "loss stats d_logits")

_F32, _I32, _U8 = torch.float32, torch.int32, torch.uint8
_strided, _like, _ONE, _TWO = torch.empty_strided, torch.empty_like, (1,), (2, 1)
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
    "olsgd_expert_route_workspace": [_i32, _i64, _i64, C.POINTER(_sz)],
    "olsgd_expert_route": [_i32, _i64, _i64, _i32, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "olsgd_expert_route_backward": [_i64, _i64, _i32, _vp, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _vp],
    "olsgd_expert_combine": [_i32, _i64, _i32, _i64, _i64, _i32, _vp, _i64, _i64, _vp, _vp, _vp, _vp],
    "olsgd_expert_combine_backward": [_i32, _i64, _i32, _i64, _i64, _i32] + 2 * [_vp, _i64, _i64] + [_vp, _vp, _vp, _vp, _vp, _vp],
    "olsgd_expert_product_workspace": [_i32, _i64, _i64, _i64, _i64, _i32, _i32, C.POINTER(_sz)],
    "olsgd_expert_product": [_i32, _i64, _i64, _i64, _i64, _i32] + 2 * [_vp, _i64, _i64] + [_i64, _vp, _vp, _vp, _sz, _vp],
    "olsgd_expert_product_backward": [_i32, _i64, _i64, _i64, _i64, _i32] + 3 * [_vp, _i64, _i64] + [_i64, _vp, _vp, _vp, _vp, _sz, _vp],
    "olsgd_distill_workspace": [_i32, _i64, _i64, _i32, C.POINTER(_sz)],
    "olsgd_distill": [_vp, _i32, _i64, _i64, _i64, _vp, _vp, _i32, _i32, C.c_float, _vp, _vp, _vp, _vp, _i64, _vp, _sz, _vp],
    "olsgd_distill_backward": [_vp, _vp, _i32, _i64, _i64, _i64, _vp, _vp, _i32, _i32, C.c_float, _vp, _vp, _i64, _vp],
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


# Small calls cost what the host takes for them, so the checks below are written to be cheap where
# they pass: one comparison each, no argument packing.

def _refuse(text, *args):
    raise ValueError(text % args if args else text)


def _need(ok, text, *args):
    if not ok:
        _refuse(text, *args)


def _recorded(*tensors):
    """Refuses tensors whose gradients would be lost without a word."""
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            _refuse("the operators record no graph: detach tensors that require gradients, or call under torch.no_grad()")


def _dtype(t, name):
    code = DTYPES.get(t.dtype)
    if code is None:
        _refuse("%s must be float32, bfloat16 or float16", name)
    return code


def _stream(index):
    return torch.cuda.current_stream(index).cuda_stream


# the same numbers without the Stream object and the checks around them (2 us a call)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream)


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _run(fn, dev, *args):
    """fn(*args, stream) on the tensors' device and its current stream."""
    index = dev.index
    if _current_device() == index:
        st = fn(*args, _stream(index))
    else:
        with torch.cuda.device(dev):
            st = fn(*args, _stream(index))
    if st:
        _check(_ops(), st)


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(query, *sizes):
    n = _sz()
    _check(_ops(), getattr(_ops(), query)(*sizes, C.byref(n)))
    return n.value


def _workspace(like, query, *sizes):
    """(tensor, pointer, bytes) of a fresh workspace on like's device; torch's allocations are 512-byte aligned."""
    n = _workspace_bytes(query, *sizes)
    if n == 0:
        return None, None, 0
    ws = _strided((n,), _ONE, dtype=_U8, device=like.device)
    return ws, ws.data_ptr(), n


# ------------------------------------------------------------------ token log probabilities

def _rows_of(t, name):
    """(pointer, type, N, V, stride between rows) of a tensor [..., V] whose rows are evenly spaced."""
    shape = t.shape
    if not t.is_cuda or not shape:
        _refuse("%s must be a CUDA tensor with at least one dimension", name)
    V, stride = shape[-1], t.stride()
    if V < 1 or (V > 1 and stride[-1] != 1):
        _refuse("%s: the last dimension must be contiguous and not empty", name)
    code = DTYPES.get(t.dtype)
    if code is None:
        _refuse("%s must be float32, bfloat16 or float16", name)
    if len(shape) == 2:
        N = shape[0]
        return t.data_ptr(), code, N, V, (stride[0] if N > 1 else V)
    if t.is_contiguous():
        return t.data_ptr(), code, t.numel() // V, V, V
    try:   # (one launch takes rows at one distance)
        rows = t.view(-1, V)
    except RuntimeError:
        raise ValueError("%s: rows must be evenly spaced" % name) from None
    N = rows.shape[0]
    return t.data_ptr(), code, N, V, (rows.stride(0) if N > 1 else V)


def _per_row(t, shape, dtype, dev, name):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.device != dev:
        _refuse("%s must be contiguous %s of shape %s on %s", name, dtype, tuple(shape), dev)
    return t.data_ptr()


def token_logprobs(logits, targets, top=0):
    """olsgd_token_logprobs.  logits [..., V] (rows evenly spaced), targets int32 [...]; a target outside
    [0, V) is a row without a token.  Returns TokenLogprobs(logp, entropy, stats, top_logp, top_ids): float32
    [...], [...], [..., 2], [..., top] and int32 [..., top] (the last two None when top == 0)."""
    if logits.requires_grad:
        _recorded(logits)
    lib = _OPS or _ops()
    xp, code, N, V, ld = _rows_of(logits, "logits")
    dev, lead = logits.device, logits.shape[:-1]
    tp = _per_row(targets, lead, _I32, dev, "targets")
    top = operator.index(top)
    if top < 0 or top > MAX_TOP or top > V:
        _refuse("top must be in [0, min(V, %d)]", MAX_TOP)
    # Tensors of their own: whoever keeps one of them keeps, saves or changes nothing else.  (Allocated the quickest way there
    # is, which is most of what the host does here.)
    top_logp = top_ids = tlp = tip = None
    if len(lead) == 1:
        logp, stats = _strided(lead, _ONE, dtype=_F32, device=dev), _strided((N, 2), _TWO, dtype=_F32, device=dev)
        if top:
            top_logp, top_ids = _strided((N, top), (top, 1), dtype=_F32, device=dev), _strided((N, top), (top, 1), dtype=_I32, device=dev)
    else:
        logp, stats = torch.empty(lead, dtype=_F32, device=dev), torch.empty(lead + (2,), dtype=_F32, device=dev)
        if top:
            top_logp, top_ids = torch.empty(lead + (top,), dtype=_F32, device=dev), torch.empty(lead + (top,), dtype=_I32, device=dev)
    entropy = _like(logp)
    if top:
        tlp, tip = top_logp.data_ptr(), top_ids.data_ptr()
    ws, wp, wn = _workspace(targets, "olsgd_token_logprobs_workspace", code, N, V, top)
    _run(lib.olsgd_token_logprobs, dev, xp, code, N, V, ld, tp, top, logp.data_ptr(), entropy.data_ptr(), stats.data_ptr(), tlp, tip, wp, wn)
    return TokenLogprobs(logp, entropy, stats, top_logp, top_ids)


def token_logprobs_backward(d_logp, d_entropy, logits, targets, stats, entropy):
    """olsgd_token_logprobs_backward: the gradient of the logits, contiguous, of their type.  d_logp and d_entropy
    are float32 [...] or None (zeros); stats and entropy are token_logprobs' for the same logits."""
    _recorded(d_logp, d_entropy, logits, stats, entropy)
    lib = _OPS or _ops()
    xp, code, N, V, ld = _rows_of(logits, "logits")
    dev, lead, f32 = logits.device, logits.shape[:-1], torch.float32
    tp, ep = _per_row(targets, lead, torch.int32, dev, "targets"), _per_row(entropy, lead, f32, dev, "entropy")
    sp = _per_row(stats, lead + (2,), f32, dev, "stats")
    lp = None if d_logp is None else _per_row(d_logp, lead, f32, dev, "d_logp")
    hp = None if d_entropy is None else _per_row(d_entropy, lead, f32, dev, "d_entropy")
    d = logits.new_empty(logits.shape)
    _run(lib.olsgd_token_logprobs_backward, dev, lp, hp, xp, code, N, V, ld, tp, sp, ep, d.data_ptr(), V)
    return d


# ------------------------------------------------------------------------ gradient clipping

def _worker_rows(t, m, name):
    """(elements of a worker, elements between workers) of a tensor [m, ...] whose workers' parts are contiguous."""
    n = t.numel() // m
    if t.is_contiguous():
        return n, n
    if not t[0].is_contiguous():
        _refuse("%s: each worker's part must be contiguous", name)
    return n, (t.stride(0) if m > 1 else n)


def clip_grads(grads, max_norm, out=None):
    """olsgd_clip_grads.  grads: a tensor or a list of tensors [m, ...], each worker's part contiguous.  Each worker's
    gradients, over all tensors, are scaled by min(1, max_norm / (norm + 1e-6)).  out: tensors of the same shapes, of any
    of the three types, that take the result (the gradients themselves: in place; views of a flat float32 gradient [m][P]:
    widened into it); None: new tensors like the gradients; no two of them may overlap, and none twice.  Returns (out, norms),
    norms float32 [m]."""
    lib = _ops()
    single = isinstance(grads, torch.Tensor)
    if single:
        grads, out = [grads], None if out is None else [out]
    _need(len(grads) > 0, "grads is empty")
    if out is None:
        out = [g.new_empty(g.shape) for g in grads]
    _need(len(out) == len(grads), "out must hold one tensor for each gradient")
    first = grads[0]
    if first.requires_grad:
        _recorded(first)
    m, dev = first.shape[0] if first.dim() else 0, first.device
    _need(first.is_cuda and m >= 1, "grads must be CUDA tensors with the workers first")
    index, codes, flat = dev.index, DTYPES, []
    for g, o in zip(grads, out):
        shape = g.shape
        if g.requires_grad or o.requires_grad:
            _recorded(g, o)
        if shape != o.shape or not shape or shape[0] != m or g.get_device() != index or o.get_device() != index:
            _refuse("gradients and out must be on one device, of the same shapes, with %d workers first", m)
        gc, oc = codes.get(g.dtype), codes.get(o.dtype)
        if gc is None or oc is None:
            _refuse("gradients and out must be float32, bfloat16 or float16")
        n = g.numel() // m
        flat += (g.data_ptr(), o.data_ptr(), n, n if g.is_contiguous() else _worker_rows(g, m, "a gradient")[1],
                 n if o.is_contiguous() else _worker_rows(o, m, "out")[1], gc | (oc << 32))
    places = [p for p in flat[1::6] if p]   # (of those that hold anything)
    if len(set(places)) < len(places):
        _refuse("out holds a tensor twice: it would be scaled twice")
    table = (_i64 * len(flat))(*flat)
    norms = first.new_empty(m, dtype=torch.float32)
    ws, wp, wn = _workspace(norms, "olsgd_clip_grads_workspace", m, len(grads))
    _run(lib.olsgd_clip_grads, dev, table, len(grads), m, float(max_norm), norms.data_ptr(), wp, wn)
    return (out[0] if single else out), norms


# ---------------------------------------------------------------------- gated feed-forward block

def _matrix(t, name, shape, dtype, dev):
    """(pointer, worker stride, row stride) of a tensor [m][rows][cols] with contiguous rows."""
    if t.shape != shape or t.dtype != dtype or t.device != dev:
        _refuse("%s must be %s of shape %s on %s", name, dtype, tuple(shape), dev)
    sw, sr, sc = t.stride()
    if sc != 1 and shape[2] != 1:
        _refuse("%s: the last dimension must be contiguous", name)
    return t.data_ptr(), sw, sr


def _aligned(matrix, shape):
    p, sw, sr = matrix
    return p % 16 == 0 and (shape[0] == 1 or sw % 8 == 0) and (shape[1] == 1 or sr % 8 == 0)


def _gated_sizes(x, w_gate, activation):
    if not x.is_cuda or x.dim() != 3 or w_gate.dim() != 3:
        _refuse("x and w_gate must be CUDA tensors [m][T][D] and [m][F][D]")
    code, act = DTYPES.get(x.dtype), ACTIVATIONS.get(activation)
    if not code:
        _refuse("x must be bfloat16 or float16")
    if act is None:
        _refuse("activation must be one of %s", sorted(ACTIVATIONS))
    m, T, D = x.shape
    return m, T, D, w_gate.shape[1], code, act


def gated_forward(x, w_gate, w_up, activation="silu", save=False):
    """olsgd_gated_forward: h = act(x w_gate^T) * (x w_up^T) for each worker.  x [m][T][D], w_gate and w_up [m][F][D], bfloat16
    or float16, rows contiguous, with or without gaps behind rows and workers.  Returns h [m][T][F], and with save=True (h, pre), pre being what
    gated_backward takes."""
    _recorded(x, w_gate, w_up)
    lib = _ops()
    m, T, D, F, code, act = _gated_sizes(x, w_gate, activation)
    dtype, dev, ws_shape = x.dtype, x.device, (m, F, D)
    a, b, c = _matrix(x, "x", (m, T, D), dtype, dev), _matrix(w_gate, "w_gate", ws_shape, dtype, dev), _matrix(w_up, "w_up", ws_shape, dtype, dev)
    h = x.new_empty((m, T, F))
    pre = x.new_empty((m, T, 2, (F + 7) // 8 * 8), dtype=torch.float32) if save else None
    ok = _aligned(a, (m, T)) and _aligned(b, ws_shape) and _aligned(c, ws_shape)
    ws, wp, wn = _workspace(h, "olsgd_gated_workspace", m, T, D, F, 0, ok)
    _run(lib.olsgd_gated_forward, dev, m, T, D, F, code, act, *a, *b, *c, h.data_ptr(), pre.data_ptr() if save else None, wp, wn)
    return (h, pre) if save else h


def gated_backward(d_h, x, w_gate, w_up, pre, activation="silu", want_d_x=True, want_d_w=True):
    """olsgd_gated_backward: (d_x, d_w_gate, d_w_up) from d_h [m][T][F] and the forward call's operands and pre; None for
    those not wanted."""
    _recorded(d_h, x, w_gate, w_up, pre)
    lib = _ops()
    m, T, D, F, code, act = _gated_sizes(x, w_gate, activation)
    dtype, dev, ws_shape = x.dtype, x.device, (m, F, D)
    d, a = _matrix(d_h, "d_h", (m, T, F), dtype, dev), _matrix(x, "x", (m, T, D), dtype, dev)
    b, c = _matrix(w_gate, "w_gate", ws_shape, dtype, dev), _matrix(w_up, "w_up", ws_shape, dtype, dev)
    _need(pre.shape == (m, T, 2, (F + 7) // 8 * 8) and pre.dtype == torch.float32 and pre.device == dev and pre.is_contiguous(),
          "pre must be the one that gated_forward returned")
    d_x = x.new_empty((m, T, D)) if want_d_x else None
    d_wg, d_wu = (x.new_empty(ws_shape), x.new_empty(ws_shape)) if want_d_w else (None, None)
    ok = _aligned(a, (m, T)) and _aligned(b, ws_shape) and _aligned(c, ws_shape)
    ws, wp, wn = _workspace(x, "olsgd_gated_workspace", m, T, D, F, 1, ok)
    _run(lib.olsgd_gated_backward, dev, m, T, D, F, code, act, *d, *a, *b, *c, pre.data_ptr(), d_x.data_ptr() if want_d_x else None,
         d_wg.data_ptr() if want_d_w else None, d_wu.data_ptr() if want_d_w else None, wp, wn)
    return d_x, d_wg, d_wu


# --------------------------------------------------------------------------------- embedding

def embedding_forward(table, ids, scale=1.0):
    """olsgd_embedding_forward: scale * table[i, ids[i]] for each worker i.  table [m][V][D], rows contiguous; ids int32 [m][T],
    those outside [0, V) give rows of zeros.  Returns [m][T][D] of the table's type."""
    _recorded(table)
    lib = _ops()
    if not table.is_cuda or table.dim() != 3 or ids.dim() != 2:
        _refuse("table must be a CUDA tensor [m][V][D], ids [m][T]")
    code, dev = _dtype(table, "table"), table.device
    m, V, D = table.shape
    T = ids.shape[1]
    p, sw, sr = _matrix(table, "table", (m, V, D), table.dtype, dev)
    ip = _per_row(ids, (m, T), torch.int32, dev, "ids")
    out = table.new_empty((m, T, D))
    _run(lib.olsgd_embedding_forward, dev, m, T, V, D, code, p, sw, sr, ip, float(scale), out.data_ptr())
    return out


def embedding_backward(d_out, ids, vocab, scale=1.0, dtype=torch.float32, out=None):
    """olsgd_embedding_backward: the gradient of a table [m][vocab][D] from d_out [m][T][D] and the ids of the lookup; new, of
    type `dtype`, or written to `out` (each worker's part contiguous, for example a view of a flat gradient [m][P])."""
    _recorded(d_out, out)
    lib = _ops()
    if not d_out.is_cuda or d_out.dim() != 3 or d_out.shape[0] < 1:
        _refuse("d_out must be a CUDA tensor [m][T][D] of at least one worker")
    code, dev = _dtype(d_out, "d_out"), d_out.device
    m, T, D = d_out.shape
    V = operator.index(vocab)
    if V < 1:
        _refuse("vocab must be positive")
    p, sw, sr = _matrix(d_out, "d_out", (m, T, D), d_out.dtype, dev)
    if out is None:
        out = d_out.new_empty((m, V, D), dtype=dtype)
    if out.shape != (m, V, D) or out.device != dev:
        _refuse("out must be of shape %s on %s", (m, V, D), dev)
    _, ow = _worker_rows(out, m, "out")
    ip = _per_row(ids, (m, T), torch.int32, dev, "ids")
    ws, wp, wn = _workspace(out, "olsgd_embedding_workspace", m, T, D)
    _run(lib.olsgd_embedding_backward, dev, m, T, V, D, code, p, sw, sr, ip, float(scale), _dtype(out, "out"), out.data_ptr(), ow, wp, wn)
    return out


# ----------------------------------------------------------------------------------- experts

def _route_sizes(logits, k):
    if logits.dim() != 3:
        _refuse("logits must be [m][T][E]")
    xp, code, _, E, ld = _rows_of(logits, "logits")
    k = operator.index(k)
    if E > MAX_EXPERTS:
        _refuse("there may be %d experts at most", MAX_EXPERTS)
    if k < 1 or k > MAX_TOP or k > E:
        _refuse("k must be in [1, min(E, %d)]", MAX_TOP)
    return xp, code, logits.shape[0], logits.shape[1], E, ld, k


def expert_route(logits, k, normalise=True):
    """olsgd_expert_route: the k experts of each token.  logits [m][T][E] (rows evenly spaced); -inf is never chosen.
    normalise: softmax over the chosen, else the chosen ones' share of the softmax over all.  Returns ExpertRoute(weights, ids,
    places, tokens, offsets): float32 [m][T][k], int32 [m][T][k], [m][T][k], [m][T k], [m][E + 1].  The rows' inputs:
    embedding_forward(x, route.tokens); their gradient: expert_combine(d_rows, route.places)."""
    if logits.requires_grad:
        _recorded(logits)
    lib = _OPS or _ops()
    xp, code, m, T, E, ld, k = _route_sizes(logits, k)
    dev = logits.device
    if m < 1:
        _refuse("logits must be of one worker at least")
    lead, by = (m, T, k), (T * k, k, 1)
    weights, ids = _strided(lead, by, dtype=_F32, device=dev), _strided(lead, by, dtype=_I32, device=dev)
    places = _like(ids)
    tokens, offsets = _strided((m, T * k), (T * k, 1), dtype=_I32, device=dev), _strided((m, E + 1), (E + 1, 1), dtype=_I32, device=dev)
    ws, wp, wn = _workspace(offsets, "olsgd_expert_route_workspace", m, T, E)
    _run(lib.olsgd_expert_route, dev, m, T, E, code, xp, ld, k, 1 if normalise else 0, weights.data_ptr(), ids.data_ptr(), places.data_ptr(),
         tokens.data_ptr(), offsets.data_ptr(), wp, wn)
    return ExpertRoute(weights, ids, places, tokens, offsets)


def expert_route_backward(d_weights, logits, ids, weights, normalise=True):
    """olsgd_expert_route_backward: the gradient of the logits, contiguous, of their type.  d_weights float32 [m][T][k]; ids and
    weights are expert_route's for the same logits and `normalise`."""
    _recorded(d_weights, logits, weights)
    lib = _OPS or _ops()
    if ids.dim() != 3:
        _refuse("ids must be [m][T][k]")
    xp, code, m, T, E, ld, k = _route_sizes(logits, ids.shape[2])
    dev, lead = logits.device, (m, T, k)
    gp, ip, wp = _per_row(d_weights, lead, _F32, dev, "d_weights"), _per_row(ids, lead, _I32, dev, "ids"), _per_row(weights, lead, _F32, dev, "weights")
    d = logits.new_empty(logits.shape)
    _run(lib.olsgd_expert_route_backward, dev, m * T, E, code, gp, xp, ld, k, 1 if normalise else 0, ip, wp, d.data_ptr())
    return d


def _combine_sizes(rows, places):
    if not rows.is_cuda or rows.dim() != 3 or places.dim() != 3 or rows.shape[0] < 1 or places.shape[2] < 1:
        _refuse("rows must be a CUDA tensor [m][R][D], places [m][T][k]")
    code = _dtype(rows, "rows")
    m, R, D = rows.shape
    T, k = places.shape[1:]
    return code, m, T, k, R, D


def expert_combine(rows, places, weights=None):
    """olsgd_expert_combine: y[i][t] = sum over j of weights[i][t][j] rows[i][places[i][t][j]].  rows [m][R][D], any of the three
    types, D contiguous; places int32 [m][T][k], those outside [0, R) add nothing; weights float32 [m][T][k], None: all 1.  Returns
    [m][T][D] of the rows' type."""
    _recorded(rows, weights)
    lib = _OPS or _ops()
    code, m, T, k, R, D = _combine_sizes(rows, places)
    dev, lead = rows.device, (m, T, k)
    p, sw, sr = _matrix(rows, "rows", (m, R, D), rows.dtype, dev)
    pp = _per_row(places, lead, _I32, dev, "places")
    wp = None if weights is None else _per_row(weights, lead, _F32, dev, "weights")
    y = rows.new_empty((m, T, D))
    _run(lib.olsgd_expert_combine, dev, m, T, k, R, D, code, p, sw, sr, pp, wp, y.data_ptr())
    return y


def expert_combine_backward(d_y, rows, places, tokens, weights):
    """olsgd_expert_combine_backward: (d_rows, d_weights) from d_y [m][T][D] and the forward call's operands; places and tokens as
    expert_route gives them (each row is named once at most; tokens is negative for the others)."""
    _recorded(d_y, rows, weights)
    lib = _OPS or _ops()
    code, m, T, k, R, D = _combine_sizes(rows, places)
    dev, lead = rows.device, (m, T, k)
    g, r = _matrix(d_y, "d_y", (m, T, D), rows.dtype, dev), _matrix(rows, "rows", (m, R, D), rows.dtype, dev)
    pp, tp = _per_row(places, lead, _I32, dev, "places"), _per_row(tokens, (m, R), _I32, dev, "tokens")
    wp = _per_row(weights, lead, _F32, dev, "weights")
    d_rows, d_weights = rows.new_empty((m, R, D)), _like(weights)
    _run(lib.olsgd_expert_combine_backward, dev, m, T, k, R, D, code, *g, *r, pp, tp, wp, d_rows.data_ptr(), d_weights.data_ptr())
    return d_rows, d_weights


def _product_sizes(x, w, offsets):
    if not x.is_cuda or x.dim() != 3 or w.dim() != 4 or x.shape[0] < 1:
        _refuse("x and w must be CUDA tensors [m][R][D] and [m][E][F][D]")
    code = DTYPES.get(x.dtype)
    if not code:
        _refuse("x must be bfloat16 or float16")
    m, R, D = x.shape
    E, F = w.shape[1:3]
    if w.shape != (m, E, F, D) or w.dtype != x.dtype or w.device != x.device:
        _refuse("w must be %s of shape %s on %s", x.dtype, (m, "E", "F", D), x.device)
    sw, se, sr, sc = w.stride()
    if sc != 1 and D != 1:
        _refuse("w: the last dimension must be contiguous")
    op = _per_row(offsets, (m, E + 1), _I32, x.device, "offsets")
    p = w.data_ptr()
    ok = p % 16 == 0 and (m == 1 or sw % 8 == 0) and (E == 1 or se % 8 == 0) and (F == 1 or sr % 8 == 0)
    return m, R, E, D, F, code, op, (p, sw, se, sr), ok


def expert_product(x, w, offsets):
    """olsgd_expert_product: y[i][r] = w[i][e] x[i][r] for the rows offsets[i][e] <= r < offsets[i][e + 1] of expert e; rows of no
    expert become zeros.  x [m][R][D] and w [m][E][F][D], bfloat16 or float16, the last dimension contiguous, with or without gaps behind
    the others (rows, experts and workers lie one behind another); offsets int32 [m][E + 1], rising.  Returns [m][R][F]."""
    _recorded(x, w)
    lib = _OPS or _ops()
    m, R, E, D, F, code, op, wm, ok = _product_sizes(x, w, offsets)
    a = _matrix(x, "x", (m, R, D), x.dtype, x.device)
    y = x.new_empty((m, R, F))
    ok = ok and _aligned(a, (m, R))
    ws, wp, wn = _workspace(y, "olsgd_expert_product_workspace", m, R, E, D, F, 0, ok)
    _run(lib.olsgd_expert_product, x.device, m, R, E, D, F, code, *a, *wm, op, y.data_ptr(), wp, wn)
    return y


def expert_product_backward(d_y, x, w, offsets, want_d_x=True, want_d_w=True):
    """olsgd_expert_product_backward: (d_x, d_w) from d_y [m][R][F] and the forward call's operands; None for one that is not
    wanted."""
    _recorded(d_y, x, w)
    lib = _OPS or _ops()
    m, R, E, D, F, code, op, wm, ok = _product_sizes(x, w, offsets)
    dtype, dev = x.dtype, x.device
    g, a = _matrix(d_y, "d_y", (m, R, F), dtype, dev), _matrix(x, "x", (m, R, D), dtype, dev)
    d_x = x.new_empty((m, R, D)) if want_d_x else None
    d_w = x.new_empty((m, E, F, D)) if want_d_w else None
    ok = ok and _aligned(g, (m, R)) and _aligned(a, (m, R))
    ws, wp, wn = _workspace(x, "olsgd_expert_product_workspace", m, R, E, D, F, 1, ok)
    _run(lib.olsgd_expert_product_backward, dev, m, R, E, D, F, code, *g, *a, *wm, op, d_x.data_ptr() if want_d_x else None,
         d_w.data_ptr() if want_d_w else None, wp, wn)
    return d_x, d_w


# ------------------------------------------------------------------------------ distillation

def _teacher(logits, ids, teacher, temperature):
    lead, dev = logits.shape[:-1], logits.device
    if ids.dim() != logits.dim() or ids.shape[:-1] != lead or not 1 <= ids.shape[-1] <= MAX_TEACHER:
        _refuse("ids must be [..., K], K in [1, %d], for logits [..., V]", MAX_TEACHER)
    code = _dtype(teacher, "teacher")
    ip, tp = _per_row(ids, ids.shape, _I32, dev, "ids"), _per_row(teacher, ids.shape, teacher.dtype, dev, "teacher")
    t = float(temperature)
    if not 2.0 ** -20 <= t <= 2.0 ** 20:
        _refuse("temperature must be in [2^-20, 2^20]")
    return ip, tp, code, ids.shape[-1], t


def distill_loss(logits, ids, teacher, temperature=1.0, d_loss=None):
    """olsgd_distill: the divergence of a teacher's top logits from the student's distribution, row by row: with
    q = softmax(teacher / temperature) over the K pairs and p = softmax(logits / temperature) over all tokens, sum q (log q -
    log p[ids]).  logits [..., V] (rows evenly spaced), ids int32 [..., K] (outside [0, V): no pair), teacher [..., K] of any of the
    three types.  d_loss float32 [...]: the weight of each row's loss, where it is known by now; the logits' gradient then
    comes with it, from the same read of them where a row fits a multiprocessor and the pairs are few (some 39000 logits of 16 bits or
    24000 of 32, and 64 pairs), else from a second one.  Returns DistillLoss(loss, stats, d_logits): float32 [...] and [..., 2], and the gradient
    (contiguous, of the logits' type) or None."""
    _recorded(logits, teacher, d_loss)
    lib = _OPS or _ops()
    xp, code, N, V, ld = _rows_of(logits, "logits")
    dev, lead = logits.device, logits.shape[:-1]
    ip, tp, tcode, K, t = _teacher(logits, ids, teacher, temperature)
    gp = None if d_loss is None else _per_row(d_loss, lead, _F32, dev, "d_loss")
    if len(lead) == 1:
        loss, stats = _strided(lead, _ONE, dtype=_F32, device=dev), _strided((N, 2), _TWO, dtype=_F32, device=dev)
    else:
        loss, stats = torch.empty(lead, dtype=_F32, device=dev), torch.empty(lead + (2,), dtype=_F32, device=dev)
    d = None if d_loss is None else logits.new_empty(logits.shape)
    ws, wp, wn = _workspace(loss, "olsgd_distill_workspace", code, N, V, 0 if d_loss is None else 1)
    _run(lib.olsgd_distill, dev, xp, code, N, V, ld, ip, tp, tcode, K, t, gp, loss.data_ptr(), stats.data_ptr(),
         None if d is None else d.data_ptr(), V, wp, wn)
    return DistillLoss(loss, stats, d)


def distill_backward(d_loss, logits, ids, teacher, stats, temperature=1.0):
    """olsgd_distill_backward: the logits' gradient alone, contiguous, of their type.  d_loss float32 [...]; stats are
    distill_loss's for the same logits and temperature."""
    _recorded(d_loss, logits, teacher, stats)
    lib = _OPS or _ops()
    xp, code, N, V, ld = _rows_of(logits, "logits")
    dev, lead = logits.device, logits.shape[:-1]
    ip, tp, tcode, K, t = _teacher(logits, ids, teacher, temperature)
    gp, sp = _per_row(d_loss, lead, _F32, dev, "d_loss"), _per_row(stats, lead + (2,), _F32, dev, "stats")
    d = logits.new_empty(logits.shape)
    _run(lib.olsgd_distill_backward, dev, gp, xp, code, N, V, ld, ip, tp, tcode, K, t, sp, d.data_ptr(), V)
    return d


def operators_join(device="cuda"):
    """olsgd_operators_join on the device's current stream: waits for it, and raises if an operator's bounded wait gave up."""
    dev = torch.device(device)
    _need(dev.type == "cuda", "device must be a CUDA device")
    if dev.index is None:
        dev = torch.device(dev.type, torch.cuda.current_device())
    _run(_ops().olsgd_operators_join, dev)
