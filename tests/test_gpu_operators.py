"""The operators on caller-owned tensors against their definitions in 64 bits.

Tolerances count roundings.  u = 2^-24 is half a step of fp32; a sum of n positive terms in fp32, added up in a chain
of length c, is off by at most about c u relative; a result rounded to type t by finfo(t).eps / 2 relative."""
import math

import numpy as np
import pytest
import torch

import paper_2002_09539_b200 as lib

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


# ------------------------------------------------------------------- token log probabilities

def _logprobs_64(x, t):
    """Definition in 64 bits: log p of every token, entropy, log p of the targets."""
    x = x.double()
    empty = torch.isneginf(x).all(dim=-1)
    # relative to the maximum: at the type's lowest value even 64 bits lose log V beside it
    d = x - x.max(dim=-1, keepdim=True).values
    lp = d - torch.logsumexp(d, dim=-1, keepdim=True)
    lp = torch.where(empty[..., None], torch.full_like(lp, -math.inf), lp)
    p = torch.exp(lp)
    h = -torch.xlogy(p, p).sum(dim=-1)
    has = (t >= 0) & (t < x.shape[-1])
    at = torch.where(has, t, torch.zeros_like(t)).long()
    picked = torch.where(has, lp.gather(-1, at[..., None])[..., 0], torch.zeros_like(h))
    return lp, h, picked, has, empty


def _sum_error(V, spread):
    """Relative error of sum exp(x - max) and of its terms: a chain of at most V / 32 + 64 additions in a lane, the
    joins, and terms e^d whose exponent |d| <= spread is rounded three times (difference, constant, product) and whose
    power of two has 2 steps."""
    return (V / 32 + 64 + 3 * spread + 4) * U


def _check_logprobs(x, t, top, r):
    lp, h, picked, has, empty = _logprobs_64(x, t)
    V = x.shape[-1]
    finite = torch.where(torch.isneginf(lp), torch.zeros_like(lp), lp)
    spread = float(min(150.0, (-finite).max() + 1.0))
    rel = _sum_error(V, spread)
    err = (r.logp.double() - picked).abs()
    ok = (r.logp.double() == picked) | (err <= rel + 4 * U * picked.abs())
    assert bool(ok.all()), float(err[torch.isfinite(err)].max())
    mean_d = (torch.exp(lp) * (finite - finite.max(dim=-1, keepdim=True).values).abs()).sum(dim=-1)
    err = (r.entropy.double() - h).abs()
    assert bool((err <= rel * (1 + 2 * mean_d) + 4 * U * (h + mean_d + math.log(V))).all()), float(err.max())
    if top:
        v, i = torch.sort(x.double(), dim=-1, descending=True, stable=True)
        assert torch.equal(r.top_ids.long(), i[..., :top])
        want = lp.gather(-1, i[..., :top])
        got = r.top_logp.double()
        err = (got - want).abs()
        assert bool(((got == want) | (err <= rel + 4 * U * want.abs())).all())
    return lp, h, has, empty, rel


def _check_logprobs_grad(x, t, r, dlp, dh):
    lp, h, has, empty, rel = _check_logprobs(x, t, 0, r)
    d = lib.token_logprobs_backward(dlp, dh, x, t, r.stats, r.entropy)
    p = torch.exp(lp)
    a = torch.zeros_like(h) if dlp is None else torch.where(has, dlp.double(), torch.zeros_like(h))
    b = torch.zeros_like(h) if dh is None else dh.double()
    one = torch.zeros_like(p).scatter_(-1, torch.where(has, t, torch.zeros_like(t)).long()[..., None], 1.0)
    want = a[..., None] * (one - p) - b[..., None] * (torch.xlogy(p, p) + p * h[..., None])
    want = torch.where(empty[..., None], torch.zeros_like(want), want)
    # p is off by `rel` and by the rounding of its own exponent; H by what its own test allows
    lpz = torch.where(p > 0, lp.abs(), torch.zeros_like(p))
    scale = p * (a.abs()[..., None] + b.abs()[..., None] * (lpz + h[..., None] + 1))
    ep = rel + 8 * U * (lpz + 2)
    tol = scale * (4 * ep) + a.abs()[..., None] * one * 2 * U + want.abs() * (torch.finfo(x.dtype).eps / 2 + 4 * U)
    tol = tol + (2.0 ** -25 if x.dtype == torch.float16 else 2.0 ** -126) * 1.01   # below the type's least steps
    err = (d.double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    return d


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,top", [(1, 1, 1), (5, 2, 2), (3, 10, 1), (33, 31, 31), (7, 32, 32), (2, 33, 32), (9, 257, 5), (4, 1000, 20),
                                     (6, 1024, 32), (5, 1025, 7), (3, 1031, 32), (300, 4099, 3), (1, 8191, 20), (2, 50021, 32), (1, 131072, 20),
                                     (700, 2049, 0), (1, 200003, 1)])
def test_token_logprobs(dtype, N, V, top):
    g = _gen(N * 1000 + V)
    x = _randn(g, (N, V), dtype, 3.0)
    t = torch.randint(-1, V + 1, (N,), generator=g, device="cuda", dtype=torch.int32)   # -1 and V: no token
    r = lib.token_logprobs(x, t, top)
    _check_logprobs(x, t, top, r)
    _check_logprobs_grad(x, t, r, _randn(g, (N,)), _randn(g, (N,)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 1500, 20011])
@pytest.mark.parametrize("pattern", ["half masked", "one left", "nothing left", "constant", "lowest", "rising", "falling", "far", "certain"])
def test_token_logprobs_masks_ties_and_extremes(dtype, V, pattern):
    g = _gen(V)
    N, low = 6, torch.finfo(dtype).min
    x = _randn(g, (N, V), dtype, 3.0)
    if pattern == "half masked":
        x.masked_fill_(torch.rand((N, V), generator=g, device="cuda") < 0.5, -math.inf)
        x[:, 3] = 0.5
    elif pattern == "one left":
        keep = x[:, V - 2].clone()
        x.fill_(-math.inf)
        x[:, V - 2] = keep
    elif pattern == "nothing left":
        x.fill_(-math.inf)
        x[0, 5] = 1.0
    elif pattern == "constant":
        x.fill_(1.5)
    elif pattern == "lowest":
        x.fill_(low)          # every token masked with the type's lowest value: uniform
        x[1, 7] = 0.0         # ... and one token left among them
    elif pattern == "rising":
        x = torch.arange(V, device="cuda").float().mul_(8.0 / V).to(dtype).repeat(N, 1).contiguous()
    elif pattern == "falling":
        x = torch.arange(V, 0, -1, device="cuda").float().mul_(8.0 / V).to(dtype).repeat(N, 1).contiguous()
    elif pattern == "far":
        x = (x.float() + 20000.0).to(dtype)
    else:
        x[:, 11] = 300.0
    t = torch.full((N,), 5, dtype=torch.int32, device="cuda")
    r = lib.token_logprobs(x, t, 32)
    _check_logprobs(x, t, 32, r)
    assert bool(torch.isfinite(r.entropy).all()) and bool((r.entropy >= 0).all())
    d = _check_logprobs_grad(x, t, r, _randn(g, (N,)), _randn(g, (N,)))
    if pattern == "nothing left":
        assert bool((d[1:] == 0).all()) and bool((r.entropy[1:] == 0).all())
    if pattern == "lowest":
        assert bool(((r.entropy[0].double() - math.log(V)).abs() <= (V / 32 + 80) * U * (1 + math.log(V))).all())


@pytest.mark.parametrize("V", [100, 5000])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_token_logprobs_nan_and_inf_stay_in_their_row(V, bad):
    g = _gen(V)
    x = _randn(g, (5, V))
    t = torch.tensor([1, 2, -1, 4, 5], dtype=torch.int32, device="cuda")
    want = lib.token_logprobs(x, t, 4)
    x[1, 77], x[2, 30] = bad, bad
    r = lib.token_logprobs(x, t, 4)
    good = torch.tensor([0, 3, 4], device="cuda")
    for a, b in zip(r, want):
        assert torch.equal(a[good], b[good])
    assert bool(torch.isnan(r.logp[1])) and float(r.logp[2]) == 0.0 and bool(torch.isnan(r.entropy[1:3]).all())
    assert int(r.top_ids[1, 0]) == 77 and int(r.top_ids[2, 0]) == 30   # first in their order
    d = lib.token_logprobs_backward(torch.ones(5, device="cuda"), None, x, t, r.stats, r.entropy)
    assert bool(torch.isnan(d[1]).all()) and bool(torch.isfinite(d[good]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,pitch,offset", [(1000, 1003, 1), (4097, 4101, 3), (9000, 9001, 5)])
def test_token_logprobs_of_strided_rows(dtype, V, pitch, offset):
    g = _gen(V)
    buf = _randn(g, (9 * pitch + 16,), dtype, 2.0)
    x = buf[offset:offset + 9 * pitch].view(9, pitch)[:, :V]
    t = torch.randint(0, V, (9,), generator=g, device="cuda", dtype=torch.int32)
    r = lib.token_logprobs(x, t, 6)
    dlp, dh = _randn(g, (9,)), _randn(g, (9,))
    _check_logprobs(x, t, 6, r)
    _check_logprobs_grad(x, t, r, dlp, dh)
    _check_logprobs_grad(x, t, r, None, dh)
    _check_logprobs_grad(x, t, r, dlp, None)
    # the same rows at another alignment: the same alternatives
    assert torch.equal(lib.token_logprobs(x.contiguous(), t, 6).top_ids, r.top_ids)


def test_token_logprobs_gradient_against_differences():
    g = _gen(3)
    N, V, step = 2, 1100, 1e-2
    x = _randn(g, (N, V), torch.float32, 1.0)
    t = torch.tensor([3, 1099], dtype=torch.int32, device="cuda")
    dlp, dh = _randn(g, (N,)), _randn(g, (N,))
    r = lib.token_logprobs(x, t)
    d = lib.token_logprobs_backward(dlp, dh, x, t, r.stats, r.entropy)

    def value(y):   # the function itself in 64 bits
        _, h, picked, _, _ = _logprobs_64(y, t)
        return picked * dlp.double() + h * dh.double()

    for j in (0, 3, 500, 1099):
        e = torch.zeros((N, V), dtype=torch.float64, device="cuda")
        e[:, j] = step
        diff = (value(x.double() + e) - value(x.double() - e)) / (2 * step)
        # central differences: the third derivative is at most about 6 (|dlp| + |dh| (log V + 2)); and the kernel's own error
        scale = dlp.abs().double() + dh.abs().double() * (math.log(V) + 2)
        assert bool(((d[:, j].double() - diff).abs() <= step * step * scale + 1e-5 * scale).all())


def test_token_logprobs_batch_dims_empty_batches_and_refusals():
    g = _gen(5)
    x = _randn(g, (3, 4, 50))
    t = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    r = lib.token_logprobs(x, t, 2)
    assert r.logp.shape == (3, 4) and r.stats.shape == (3, 4, 2) and r.top_ids.shape == (3, 4, 2)
    assert torch.equal(r.logp.view(-1), lib.token_logprobs(x.view(12, 50), t.view(-1), 2).logp)
    e = lib.token_logprobs(x[:0], t[:0], 2)
    assert e.logp.shape == (0, 4)
    assert lib.token_logprobs_backward(None, None, x[:0], t[:0], e.stats, e.entropy).shape == (0, 4, 50)
    for bad in (lambda: lib.token_logprobs(x.transpose(0, 2), t), lambda: lib.token_logprobs(x, t.long()),
                lambda: lib.token_logprobs(x, t, 33), lambda: lib.token_logprobs(x, t, 51), lambda: lib.token_logprobs(x, t[:2]),
                lambda: lib.token_logprobs(x.double(), t), lambda: lib.token_logprobs(x.cpu(), t), lambda: lib.token_logprobs(x, t.cpu()),
                lambda: lib.token_logprobs_backward(t, None, x, t, r.stats, r.entropy),
                lambda: lib.token_logprobs_backward(None, None, x, t, r.entropy, r.entropy)):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------------- gradient clipping

def _check_clip(grads, max_norm, out, norms):
    whole = torch.stack([g.double().flatten(1).square().sum(dim=1) for g in grads]).sum(dim=0).sqrt()
    # sums in 64 bits, of eight exact squares added up in fp32 in four roundings (half of that in the root); the norm is rounded once
    assert bool(((norms.double() - whole).abs() <= whole * 3.01 * U).all())
    c = torch.clamp(max_norm / (whole + 1e-6), max=1.0)
    for g, o in zip(grads, out):
        want = g.double() * c.view(-1, *[1] * (g.dim() - 1))
        # the norm as above; the factor and the product are rounded to fp32, the result to its type
        tol = want.abs() * (4.6 * U + torch.finfo(o.dtype).eps / 2) + torch.finfo(o.dtype).smallest_normal * torch.finfo(o.dtype).eps
        assert bool(((o.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("m", [1, 3, 16])
@pytest.mark.parametrize("tin,tout", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float16, torch.float32),
                                      (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16)])
@pytest.mark.parametrize("sizes", [[1], [7, 4096, 33, 1], [50001, 3], [123457]])
def test_clip_grads(m, tin, tout, sizes):
    g = _gen(m + sum(sizes))
    std = torch.tensor([1.0 if i % 2 == 0 else 1e-5 for i in range(m)], device="cuda")[:, None]
    grads = [(torch.randn((m, n), generator=g, device="cuda") * std).to(tin) for n in sizes]
    keep = [t.clone() for t in grads]
    out = [torch.empty_like(t, dtype=tout) for t in grads]
    got, norms = lib.clip_grads(grads, 0.5, out=out)
    assert got is out
    _check_clip(grads, 0.5, out, norms)
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    again = [torch.empty_like(t) for t in out]
    _, n2 = lib.clip_grads(grads, 0.5, out=again)
    assert torch.equal(n2, norms) and all(torch.equal(a, b) for a, b in zip(again, out))
    if tin == tout:
        _, n3 = lib.clip_grads(grads, 0.5, out=grads)   # in place
        assert torch.equal(n3, norms) and all(torch.equal(a, b) for a, b in zip(grads, out))


def test_clip_grads_into_a_flat_gradient_leaves_the_rest_alone():
    g = _gen(1)
    m, shapes = 3, [(5, 7), (1001,), (4, 3, 11)]
    P = 2000
    flat = torch.full((m, P), -7.0, device="cuda")
    grads = [_randn(g, (m,) + s, torch.bfloat16) for s in shapes]
    out, at = [], 3
    for s in shapes:
        n = int(np.prod(s))
        out.append(flat[:, at:at + n].unflatten(1, s))
        at += n + 5
    _, norms = lib.clip_grads(grads, 1.0, out=out)
    _check_clip(grads, 1.0, out, norms)
    mask = torch.ones(P, dtype=torch.bool, device="cuda")
    at = 3
    for s in shapes:
        n = int(np.prod(s))
        mask[at:at + n] = False
        at += n + 5
    assert bool((flat[:, mask] == -7.0).all())


@pytest.mark.parametrize("count", [8, 9, 48, 49, 256, 257, 601])   # room in one launch for 8, 48 and 256
def test_clip_grads_of_many_tensors(count):
    g = _gen(2)
    grads = [_randn(g, (2, 1 + (i * 37) % 300), torch.float32 if i % 3 else torch.bfloat16) for i in range(count - 1)]
    grads.insert(count // 2, torch.empty((2, 0), device="cuda"))
    out, norms = lib.clip_grads(grads, 2.0)
    _check_clip(grads, 2.0, out, norms)
    _, n2 = lib.clip_grads(grads, 2.0, out=grads)
    assert torch.equal(norms, n2) and all(torch.equal(a, b) for a, b in zip(grads, out))


def test_clip_grads_extremes():
    x = torch.zeros((5, 1000), device="cuda")
    x[0, 3], x[0, 4] = 3e30, 4e30          # squares beyond fp32
    x[1, 5] = math.nan
    x[2, 6], x[2, 7] = math.inf, 1.0
    x[3, 8] = 1e-30                        # squares below fp32
    out, norms = lib.clip_grads(x, 1.0)
    assert abs(float(norms[0]) / 5e30 - 1) < 1e-6 and abs(float(out[0, 3]) - 0.6) < 1e-6
    assert bool(torch.isnan(out[1]).all())
    assert math.isinf(float(norms[2])) and float(out[2, 7]) == 0.0 and bool(torch.isnan(out[2, 6]))
    assert abs(float(norms[3]) / 1e-30 - 1) < 1e-6 and torch.equal(out[3], x[3])
    assert float(norms[4]) == 0.0 and torch.equal(out[4], x[4])


def test_clip_grads_refusals():
    x = torch.ones((2, 10), device="cuda")
    for bad in (lambda: lib.clip_grads([], 1.0), lambda: lib.clip_grads([x, x[:1]], 1.0), lambda: lib.clip_grads(x.cpu(), 1.0),
                lambda: lib.clip_grads(x, 1.0, out=x[:, :5]), lambda: lib.clip_grads(x.double(), 1.0),
                lambda: lib.clip_grads([x], 1.0, out=[]), lambda: lib.clip_grads(torch.ones((10, 2), device="cuda").t(), 1.0)):
        with pytest.raises(ValueError):
            bad()
    for norm in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(lib.OlsgdError):
            lib.clip_grads(x, norm)


# ---------------------------------------------------------------------- gated feed-forward block

ACTS = ["silu", "gelu", "relu", "sigmoid"]


def _act_64(kind, a):
    """act(a), act'(a) in 64 bits."""
    if kind == "relu":
        return a.clamp(min=0.0), (a > 0).double()
    if kind == "gelu":
        k, c = math.sqrt(2 / math.pi), 0.044715
        t = torch.tanh(k * (a + c * a ** 3))
        return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * k * (1 + 3 * c * a * a)
    s = torch.sigmoid(a)
    return (s, s * (1 - s)) if kind == "sigmoid" else (a * s, s * (1 + a * (1 - s)))


def _product_error(K):
    """Relative to sum |x||w|: products of 16-bit values are exact in fp32; 16 of them enter an accumulator at a time,
    which may drop its last bit rather than round it, and so may the alignment of each group of 8."""
    return (K / 8 + 8) * 2 * U


def _check_gated(x, wg, wu, dh, kind):
    dtype = x.dtype
    half, tiny = torch.finfo(dtype).eps / 2, (2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126)
    D, F = x.shape[2], wg.shape[1]
    X, G, Up = x.double(), wg.double(), wu.double()
    a, b = X @ G.mT, X @ Up.mT
    f, df = _act_64(kind, a)
    ea = _product_error(D) * (X.abs() @ G.abs().mT)
    eb = _product_error(D) * (X.abs() @ Up.abs().mT)
    # slopes: |act'| <= 1.13 (gelu's is the steepest), |act''| <= 1.2; the device's exponential and division: 8 steps
    ef = 1.13 * ea + 8 * U * (f.abs() + a.abs())
    h, pre = lib.gated_forward(x, wg, wu, kind, save=True)
    tol = f.abs() * eb + b.abs() * ef + ef * eb + (f * b).abs() * (half + 4 * U) + tiny
    err = (h.double() - f * b).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    assert torch.equal(h, lib.gated_forward(x, wg, wu, kind))
    if dh is None:
        return
    E = dh.double()
    da, db = E * b * df, E * f
    # (a and b are kept as they were accumulated)
    edf = 1.2 * ea + 16 * U * (1 + a.abs())
    if kind == "relu":
        edf = torch.where(a.abs() <= ea, torch.ones_like(a), torch.zeros_like(a))   # the side of 0 is open only there
    eda = E.abs() * (b.abs() * edf + df.abs() * eb + edf * eb) + (half + 4 * U) * da.abs() + tiny
    edb = E.abs() * (1.13 * ea + 8 * U * (f.abs() + a.abs())) + (half + 4 * U) * db.abs() + tiny
    eda, edb = eda * (1 + half), edb * (1 + half)
    dx, dwg, dwu = lib.gated_backward(dh, x, wg, wu, pre, kind)
    A, B = da.abs() + eda, db.abs() + edb
    want = da @ G + db @ Up
    tol = eda @ G.abs() + edb @ Up.abs() + _product_error(2 * F) * (A @ G.abs() + B @ Up.abs()) + half * want.abs() * 1.01 + tiny
    err = (dx.double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    T = x.shape[1]
    for got, d, e, S in ((dwg, da, eda, A), (dwu, db, edb, B)):
        want = d.mT @ X
        tol = e.mT @ X.abs() + _product_error(T) * (S.mT @ X.abs()) + half * want.abs() * 1.01 + tiny
        err = (got.double() - want).abs()
        assert bool((err <= tol).all()), float((err - tol).max())


# tiles of every kind: 64 columns; 256 columns by one CTA and by a pair, in each of the three products; partial rows,
# columns and K blocks; widths with and without 16-byte rows; K in one part and in several, in each product
GATED_SHAPES = [(1, 1, 1, 1), (1, 1, 64, 32), (1, 2, 8, 8), (2, 5, 33, 47), (3, 3, 1001, 37), (2, 4, 2056, 40), (2, 4, 33, 47), (1, 128, 64, 128), (3, 130, 72, 136), (1, 300, 200, 520),
                (2, 257, 1021, 515), (1, 1, 1024, 4096), (1, 17, 4096, 24), (16, 128, 256, 1024), (8, 300, 128, 1024), (8, 600, 1024, 1024),
                (16, 100, 2048, 72), (16, 70, 1024, 100), (5, 401, 1000, 1303),
                (1, 200, 304, 2048), (1, 40, 4096, 64), (1, 5000, 64, 48), (1, 41, 4001, 61), (2, 3000, 67, 45), (1, 512, 1024, 4096),
                (2, 140, 100, 2556), (2, 140, 2556, 98), (1, 35, 67, 129), (1, 35, 129, 67)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", GATED_SHAPES)
def test_gated_block(shape, dtype):
    m, T, D, F = shape
    g = _gen(sum(shape))
    x, dh = _randn(g, (m, T, D), dtype), _randn(g, (m, T, F), dtype)
    wg, wu = _randn(g, (m, F, D), dtype, D ** -0.5), _randn(g, (m, F, D), dtype, D ** -0.5)
    _check_gated(x, wg, wu, dh, ACTS[sum(shape) % 4])
    lib.operators_join()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", ACTS)
def test_gated_block_activations(kind, dtype):
    g = _gen(11)
    x, dh = _randn(g, (2, 70, 96), dtype, 4.0), _randn(g, (2, 70, 80), dtype)
    wg, wu = _randn(g, (2, 80, 96), dtype, 0.2), _randn(g, (2, 80, 96), dtype, 0.1)
    _check_gated(x, wg, wu, dh, kind)


@pytest.mark.parametrize("pad", [8, 3])
def test_gated_block_of_strided_operands(pad):
    """Weights as views of flat rows, tokens as a slice of longer sequences; with 16-byte pitches and without."""
    g = _gen(pad)
    m, T, D, F, dtype = 2, 37, 128, 72, torch.bfloat16
    flat = _randn(g, (m, 2 * F * (D + pad) + 11 * pad), dtype, 0.1)
    wg = flat[:, pad:pad + F * (D + pad)].unflatten(1, (F, D + pad))[:, :, :D]
    wu = flat[:, F * (D + pad) + 2 * pad:2 * F * (D + pad) + 2 * pad].unflatten(1, (F, D + pad))[:, :, :D]
    x = _randn(g, (m, T + 5, D + pad), dtype)[:, 2:T + 2, :D]
    dh = _randn(g, (m, T + 1, F + pad), dtype)[:, 1:, pad:]
    _check_gated(x, wg, wu, dh, "silu")
    h, pre = lib.gated_forward(x, wg, wu, "silu", save=True)
    c = [t.contiguous() for t in (x, wg, wu, dh)]
    assert torch.equal(h, lib.gated_forward(c[0], c[1], c[2]))
    for a, b in zip(lib.gated_backward(dh, x, wg, wu, pre), lib.gated_backward(c[3], c[0], c[1], c[2], pre)):
        assert torch.equal(a, b)


def test_gated_block_extremes_stay_in_their_rows():
    g = _gen(4)
    dtype = torch.bfloat16
    x, dh = _randn(g, (1, 40, 64), dtype), _randn(g, (1, 40, 48), dtype)
    wg, wu = _randn(g, (1, 48, 64), dtype), _randn(g, (1, 48, 64), dtype)
    want = {k: lib.gated_forward(x, wg, wu, k, save=True) for k in ACTS}
    grads = {k: lib.gated_backward(dh, x, wg, wu, want[k][1], k)[0] for k in ACTS}
    x[0, 3, 5] = math.nan
    x[0, 7] = 3e38 * torch.sign(wg[0, 0].float()).to(dtype)   # products beyond fp32
    keep = [i for i in range(40) if i not in (3, 7)]
    for k in ACTS:
        h, pre = lib.gated_forward(x, wg, wu, k, save=True)
        assert bool(torch.isnan(h[0, 3]).all())
        assert torch.equal(h[0, keep], want[k][0][0, keep])
        dx = lib.gated_backward(dh, x, wg, wu, pre, k, want_d_w=False)[0]
        assert torch.equal(dx[0, keep], grads[k][0, keep])


def test_gated_gradients_against_differences():
    g = _gen(6)
    m, T, D, F = 1, 6, 16, 24
    x, wg, wu = _randn(g, (m, T, D), torch.float16), _randn(g, (m, F, D), torch.float16, 0.3), _randn(g, (m, F, D), torch.float16, 0.3)
    dh = _randn(g, (m, T, F), torch.float16)
    _, pre = lib.gated_forward(x, wg, wu, "gelu", save=True)
    dx, dwg, dwu = lib.gated_backward(dh, x, wg, wu, pre, "gelu")
    X, G, Up, E, step = x.double(), wg.double(), wu.double(), dh.double(), 1e-4

    def loss(X, G, Up):
        return float((_act_64("gelu", X @ G.mT)[0] * (X @ Up.mT) * E).sum())

    for got, which in ((dx, 0), (dwg, 1), (dwu, 2)):
        for at in ((0, 0, 0), (0, 3, 7), (0, 5, 15)):
            lo, hi = [X.clone(), G.clone(), Up.clone()], [X.clone(), G.clone(), Up.clone()]
            lo[which][at] -= step
            hi[which][at] += step
            diff = (loss(*hi) - loss(*lo)) / (2 * step)
            # sums of some twenty terms of size one, each of values rounded three times to 11 bits
            assert abs(float(got[at]) - diff) <= 60 * 3 * 2.0 ** -11


def test_gated_parts_empty_batches_and_refusals():
    g = _gen(8)
    x, wg, wu = _randn(g, (2, 9, 40), torch.bfloat16), _randn(g, (2, 16, 40), torch.bfloat16), _randn(g, (2, 16, 40), torch.bfloat16)
    dh = _randn(g, (2, 9, 16), torch.bfloat16)
    h, pre = lib.gated_forward(x, wg, wu, "relu", save=True)
    whole = lib.gated_backward(dh, x, wg, wu, pre, "relu")
    dx, none, _ = lib.gated_backward(dh, x, wg, wu, pre, "relu", want_d_w=False)
    assert none is None and torch.equal(dx, whole[0])
    none, dwg, dwu = lib.gated_backward(dh, x, wg, wu, pre, "relu", want_d_x=False)
    assert none is None and torch.equal(dwg, whole[1]) and torch.equal(dwu, whole[2])
    e, epre = lib.gated_forward(x[:, :0], wg, wu, "relu", save=True)
    assert e.shape == (2, 0, 16)
    dx, dwg, dwu = lib.gated_backward(dh[:, :0], x[:, :0], wg, wu, epre, "relu")
    assert dx.shape == (2, 0, 40) and not bool(dwg.any()) and not bool(dwu.any())
    for bad in (lambda: lib.gated_forward(x, wg, wu, "tanh"), lambda: lib.gated_forward(x.float(), wg, wu), lambda: lib.gated_forward(x, wg, wu[:, :8]),
                lambda: lib.gated_forward(x, wg, wu.half()), lambda: lib.gated_forward(x.cpu(), wg, wu), lambda: lib.gated_forward(x, wg[:1], wu),
                lambda: lib.gated_forward(x.mT, wg, wu), lambda: lib.gated_forward(x, wg.mT.contiguous().mT, wu),
                lambda: lib.gated_backward(dh, x, wg, wu, pre[:, :5], "relu"), lambda: lib.gated_backward(dh[:, :5], x, wg, wu, pre, "relu")):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(lib.OlsgdError):   # workers on top of each other
        lib.gated_forward(x[:1].expand(2, 9, 40), wg, wu)


# -------------------------------------------------------------------------------- embedding

def _check_embedding(table, ids, dout, scale, out_dtype, out=None):
    m, V, D = table.shape
    dtype = table.dtype
    scale32 = float(np.float32(scale))
    has = ((ids >= 0) & (ids < V))[..., None]
    at = torch.where(has[..., 0], ids, torch.zeros_like(ids)).long()
    rows = torch.stack([table[i][at[i]] for i in range(m)]).double() * scale32
    want = torch.where(has, rows, torch.zeros_like(rows))
    got = lib.embedding_forward(table, ids, scale)
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126
    assert bool(((got.double() - want).abs() <= want.abs() * (torch.finfo(dtype).eps / 2 + U) + tiny).all())
    if dout is None:
        return
    d = lib.embedding_backward(dout, ids, V, scale, dtype=out_dtype, out=out)
    E = torch.where(has, dout.double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    want = torch.stack([torch.zeros((V, D), dtype=torch.float64, device="cuda").index_add_(0, at[i], E[i]) for i in range(m)]) * scale32
    size = torch.stack([torch.zeros((V, D), dtype=torch.float64, device="cuda").index_add_(0, at[i], E[i].abs()) for i in range(m)]) * abs(scale32)
    n = torch.stack([torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, at[i], has[i, :, 0].double()) for i in range(m)])
    # a chain of at most 32 additions in a chunk, an eighth of the chunks in a warp, the join, the scale
    chain = torch.clamp(n, max=32) + n / 256 + 12
    tiny = 2.0 ** -24 if out_dtype == torch.float16 else 2.0 ** -126
    tol = size * chain[..., None] * U + want.abs() * (torch.finfo(out_dtype).eps / 2 + 2 * U) + tiny
    err = (d.double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    assert not bool(d[n == 0].any())
    assert torch.equal(d, lib.embedding_backward(dout, ids, V, scale, dtype=out_dtype))   # the same bits again
    return d


@pytest.mark.parametrize("tin,tout", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float16, torch.float32),
                                      (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("m,T,V,D", [(1, 1, 1, 1), (2, 5, 3, 7), (1, 31, 255, 8), (3, 33, 256, 24), (1, 2048, 1000, 16), (2, 2049, 70000, 9),
                                     (1, 4500, 50, 1032), (2, 700, 300, 2050), (1, 64, 5, 4096),
                                     (2, 4096, 257, 8), (3, 4097, 256, 8), (1, 32768, 70000, 8), (2, 32769, 500, 12)])
def test_embedding(m, T, V, D, tin, tout):
    g = _gen(T + V + D)
    table, dout = _randn(g, (m, V, D), tin), _randn(g, (m, T, D), tin)
    ids = torch.randint(-1, V + 1, (m, T), generator=g, device="cuda", dtype=torch.int32)   # -1 and V: no token
    _check_embedding(table, ids, dout, 1.7, tout)


@pytest.mark.parametrize("pattern", ["all one", "all missing", "two", "rising", "zipf", "last", "runs of a chunk"])
@pytest.mark.parametrize("D", [72, 13])
def test_embedding_patterns(pattern, D):
    g = _gen(D)
    m, T, V = 2, 9001, 3000
    if pattern == "all one":
        ids = torch.full((m, T), 17, device="cuda")
    elif pattern == "all missing":
        ids = torch.full((m, T), -5, device="cuda")
    elif pattern == "two":
        ids = torch.randint(0, 2, (m, T), generator=g, device="cuda") * (V - 1)
    elif pattern == "rising":
        ids = torch.arange(T, device="cuda").repeat(m, 1) % V
    elif pattern == "zipf":
        ids = (V ** torch.rand((m, T), generator=g, device="cuda")).long().clamp(max=V - 1)
    elif pattern == "last":
        ids = torch.full((m, T), V - 1, device="cuda")
        ids[:, 5] = 2 ** 31 - 1
    else:   # rows that begin and end on the borders of the chunks of 32
        ids = (torch.arange(T, device="cuda") // 32).repeat(m, 1)
    ids = ids.to(torch.int32).contiguous()
    _check_embedding(_randn(g, (m, V, D), torch.bfloat16), ids, _randn(g, (m, T, D), torch.bfloat16), 0.5, torch.float32)


def test_embedding_sort_is_stable():
    """Sums of a row are formed in the order of its positions: values that only that order adds up to zero."""
    T = 5000
    ids = torch.full((1, T), 9, dtype=torch.int32, device="cuda")
    ids[0, ::7] = 3
    dout = torch.zeros((1, T, 8), device="cuda")
    at = [i for i in range(T) if i % 7][:3]
    dout[0, at[0]], dout[0, at[1]], dout[0, at[2]] = 1e8, 1.0, -1e8
    d = lib.embedding_backward(dout, ids, 10)
    assert bool((d[0, 9] == np.float32(1e8) + np.float32(1.0) - np.float32(1e8)).all())


def test_embedding_of_strided_tensors_into_a_flat_gradient():
    g = _gen(12)
    m, T, V, D = 2, 300, 120, 40
    P = V * D + 100
    for offset, pad in ((4, 8), (3, 1)):
        table = _randn(g, (m, V + 2, D + pad), torch.bfloat16)[:, 1:V + 1, :D]
        dout = _randn(g, (m, T + 3, D + pad), torch.bfloat16)[:, 3:, :D]
        ids = torch.randint(0, V, (m, T), generator=g, device="cuda", dtype=torch.int32)
        flat = torch.full((m, P), -7.0, device="cuda")
        out = flat[:, offset:offset + V * D].unflatten(1, (V, D))
        d = _check_embedding(table, ids, dout, 2.0, torch.float32, out=out)
        assert d is out and bool((flat[:, :offset] == -7).all()) and bool((flat[:, offset + V * D:] == -7).all())


def test_embedding_empty_batches_and_refusals():
    g = _gen(13)
    table, ids = _randn(g, (2, 9, 16)), torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    assert lib.embedding_forward(table, ids[:, :0].contiguous()).shape == (2, 0, 16)
    d = lib.embedding_backward(torch.empty((2, 0, 16), device="cuda"), ids[:, :0].contiguous(), 9)
    assert d.shape == (2, 9, 16) and not bool(d.any())
    for bad in (lambda: lib.embedding_forward(table, ids.long()), lambda: lib.embedding_forward(table, ids[:1]), lambda: lib.embedding_forward(table, ids[:, ::2]),
                lambda: lib.embedding_forward(table.mT, ids), lambda: lib.embedding_forward(table.cpu(), ids),
                lambda: lib.embedding_forward(table, ids.cpu()), lambda: lib.embedding_forward(table.double(), ids),
                lambda: lib.embedding_backward(table, ids, 9), lambda: lib.embedding_backward(table[:, :4], ids, 9, out=table[:, :8])):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------- sizes past 32-bit offsets

def test_token_logprobs_past_32_bit_offsets():
    N, V = 66000, 32800   # 2.16e9 logits
    g = _gen(21)
    x = torch.empty((N, V), dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=g)
    t = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    r = lib.token_logprobs(x, t, 2)
    d = lib.token_logprobs_backward(r.logp, None, x, t, r.stats, r.entropy)
    for rows in (slice(0, 3), slice(N - 3, N), slice(65472, 65476)):
        s = lib.token_logprobs(x[rows].clone(), t[rows].clone(), 2)
        # fewer rows are split over more CTAs: sums in another order
        assert torch.allclose(r.logp[rows], s.logp, rtol=0, atol=3 * _sum_error(V, 12.0)) and torch.equal(r.top_ids[rows], s.top_ids)
        p = torch.softmax(x[rows].double(), dim=1)
        want = r.logp[rows].double()[:, None] * (torch.zeros_like(p).scatter_(1, t[rows].long()[:, None], 1.0) - p)
        assert bool(((d[rows].double() - want).abs() <= want.abs() * 2.0 ** -7).all())


def test_embedding_past_32_bit_offsets():
    V, D, T = 1 << 21, 1040, 300   # 2.18e9 elements of the table
    g = _gen(22)
    table = torch.zeros((1, V, D), dtype=torch.bfloat16, device="cuda")
    ids = torch.randint(V - 50, V, (1, T), generator=g, device="cuda", dtype=torch.int32)
    ids[0, :3] = torch.tensor([0, V - 1, V // 2], dtype=torch.int32, device="cuda")
    table[0, V - 50:].normal_(generator=g)
    out = lib.embedding_forward(table, ids)
    assert torch.equal(out[0], table[0][ids[0].long()])
    d = torch.full_like(table, 3.0)
    lib.embedding_backward(out, ids, V, out=d)
    want = torch.zeros((50, D), dtype=torch.float64, device="cuda")
    late = ids[0] >= V - 50
    want.index_add_(0, ids[0][late].long() - (V - 50), out[0][late].double())
    assert bool(((d[0, V - 50:].double() - want).abs() <= want.abs() * 2.0 ** -8 + 64 * U * 20).all())
    assert not bool(d[0, 1:V // 2].any()) and not bool(d[0, V // 2 + 1:V - 50].any())


def test_gated_block_past_32_bit_offsets():
    T, D, F = 66000, 16, 32800   # 2.16e9 results
    g = _gen(23)
    x, w = _randn(g, (1, T, D), torch.bfloat16), _randn(g, (2, F, D), torch.bfloat16)
    h = lib.gated_forward(x, w[:1], w[1:], "relu")
    for rows in (slice(0, 128), slice(T - 130, T)):
        a, b = x[:, rows].double() @ w[:1].double().mT, x[:, rows].double() @ w[1:].double().mT
        want = a.clamp(min=0) * b
        tol = want.abs() * 2.0 ** -8 + _product_error(D) * (x[:, rows].double().abs() @ w[:1].double().abs().mT) * (b.abs() + 1) \
            + _product_error(D) * (x[:, rows].double().abs() @ w[1:].double().abs().mT) * a.abs()
        assert bool(((h[:, rows].double() - want).abs() <= tol).all())


def test_clip_grads_past_32_bit_offsets_and_of_many_workers():
    x = torch.zeros((2, 2200000000), dtype=torch.bfloat16, device="cuda")
    x[0, -1], x[1, -2], x[1, 5] = 3.0, 4.0, 3.0
    _, norms = lib.clip_grads(x, 1.0, out=x)
    assert norms.tolist() == [3.0, 5.0]
    assert abs(float(x[0, -1]) - 1.0) < 2.0 ** -8 and abs(float(x[1, -2]) - 0.8) < 2.0 ** -8 and abs(float(x[1, 5]) - 0.6) < 2.0 ** -8
    assert int(torch.count_nonzero(x[0])) == 1 and int(torch.count_nonzero(x[1])) == 2
    g = _gen(24)
    grads = [_randn(g, (700, 37)), _randn(g, (700, 1), torch.float16)]
    out, norms = lib.clip_grads(grads, 3.0)
    _check_clip(grads, 3.0, out, norms)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 63])
@pytest.mark.parametrize("parts", ["all", "d_x alone"])
def test_gated_relu_border_is_found_in_64_bits(D, dtype, parts):
    """Pre-activations that fp32 rounds to nothing, of both signs: terms of 2^10, -2^10 and a last one of +-2^-18."""
    g = _gen(D)
    T, F = 4, 40
    x, wg, wu = _randn(g, (1, T, D), dtype), _randn(g, (1, F, D), dtype), _randn(g, (1, F, D), dtype)
    dh = _randn(g, (1, T, F), dtype)
    x[0, 2] = 0.0
    x[0, 2, 0] = x[0, 2, 1] = 32.0
    x[0, 2, 2] = 2.0 ** -9
    x[0, 2, 3:] = 0.0
    wg[0, :, 2] = 1.0
    for f, sign in ((3, 1.0), (17, -1.0), (39, 1.0)):
        wg[0, f, 0], wg[0, f, 1], wg[0, f, 2] = 32.0, -32.0, sign * 2.0 ** -9
    a = x.double() @ wg.double().mT
    assert float(a[0, 2, 3]) == 2.0 ** -18 and float(a[0, 2, 17]) == -2.0 ** -18
    _, pre = lib.gated_forward(x, wg, wu, "relu", save=True)
    db, da = dh.double() * a.clamp(min=0), dh.double() * (x.double() @ wu.double().mT) * (a > 0)
    dx, dwg, _ = lib.gated_backward(dh, x, wg, wu, pre, "relu", want_d_w=parts == "all")
    want = (da @ wg.double() + db @ wu.double())[0, 2]
    size = (da.abs() @ wg.double().abs() + db.abs() @ wu.double().abs())[0, 2]
    assert bool(((dx[0, 2].double() - want).abs() <= size * (2 * torch.finfo(dtype).eps + _product_error(2 * F))).all())
    if dwg is not None:
        want = (da.mT @ x.double())[0]
        size = (da.abs().mT @ x.double().abs())[0]
        for f in (3, 17, 39):
            assert bool(((dwg[0, f].double() - want[f]).abs() <= size[f] * (2 * torch.finfo(dtype).eps + _product_error(T))).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [70, 3000])
def test_token_logprobs_gradient_of_padding_is_zero_whatever_it_holds(V, dtype):
    g = _gen(V)
    x = _randn(g, (6, V), dtype)
    x[1, 3], x[2, 5], x[3, 7] = math.nan, math.inf, -math.inf
    x[4] = math.nan
    t = torch.tensor([0, -1, V, 7, -1, 2], dtype=torch.int32, device="cuda")
    r = lib.token_logprobs(x, t, 2)
    assert r.logp[[1, 2, 4]].tolist() == [0.0, 0.0, 0.0] and float(r.logp[3]) == -math.inf
    dlp = torch.ones(6, device="cuda")
    dlp[5] = 0.0
    for dh in (None, torch.zeros(6, device="cuda")):
        d = lib.token_logprobs_backward(dlp, dh, x, t, r.stats, r.entropy)
        assert not bool(d[[1, 2, 4, 5]].any()) and bool(torch.isfinite(d).all())
        assert bool(d[0].any()) and bool(d[3].any())
    d = lib.token_logprobs_backward(dlp, torch.ones(6, device="cuda"), x, t, r.stats, r.entropy)
    assert bool(torch.isnan(d[[1, 2, 4]]).all()) and bool(torch.isfinite(d[[0, 3, 5]]).all())


def test_operators_of_no_workers_are_refused():
    x = torch.zeros(0, 4, 8, device="cuda")
    ids = torch.zeros(0, 4, dtype=torch.int32, device="cuda")
    for call in (lambda: lib.embedding_forward(x, ids), lambda: lib.embedding_backward(x, ids, 8), lambda: lib.clip_grads(x, 1.0),
                 lambda: lib.gated_forward(x.bfloat16(), x.bfloat16(), x.bfloat16())):
        with pytest.raises((ValueError, lib.OlsgdError)):
            call()
    with pytest.raises(ValueError):
        lib.operators_join("cpu")
