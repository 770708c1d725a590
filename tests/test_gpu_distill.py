"""Distillation from a teacher's top logits against its definition in 64 bits.  Tolerances count roundings, U = 2^-24 being half a
step of fp32."""
import math

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


def _distill_64(x, ids, z, t):
    """(log p, p, q of each pair, log q, terms, rows without a teacher, rows without a distribution)."""
    x, z, V = x.double(), z.double(), x.shape[-1]
    there = (ids >= 0) & (ids < V)
    at = torch.where(there, ids, 0).long()
    z = torch.where(there, z, -math.inf)
    none, empty = torch.isneginf(z).all(dim=-1), torch.isneginf(x).all(dim=-1)
    zt = (z - torch.where(none[..., None], 0.0, z.amax(dim=-1, keepdim=True))) / t
    logq = zt - torch.where(none[..., None], 0.0, torch.logsumexp(zt, dim=-1, keepdim=True))
    q = torch.where(none[..., None], 0.0, torch.exp(logq))
    d = (x - torch.where(empty[..., None], 0.0, x.amax(dim=-1, keepdim=True))) / t
    lp = d - torch.where(empty[..., None], 0.0, torch.logsumexp(d, dim=-1, keepdim=True))
    lpt = lp.gather(-1, at)
    terms = torch.where(q > 0, q * (logq - lpt), 0.0)
    return lp, torch.exp(lp), at, q, logq, lpt, terms, none, empty


def _check(x, ids, z, t, d_loss):
    lp, p, at, q, logq, lpt, terms, none, empty = _distill_64(x, ids, z, t)
    V, K = x.shape[-1], ids.shape[-1]
    finite = torch.where(torch.isneginf(lp), 0.0, lp)
    spread = float(min(150.0, (-finite).max() + 1.0))
    # a sum of exponentials: a chain of V / 32 + 64 additions at most, exponents |d| <= spread of three roundings, 2 steps each
    rel = (V / 32 + 64 + 3 * spread + 4) * U
    lqf = torch.where(q > 0, logq, 0.0)
    rq = (K + 16 + 3 * float(min(150.0, (-lqf).max() + 1.0))) * U
    lptf = torch.where(torch.isneginf(lpt), 0.0, lpt)
    loss = terms.sum(dim=-1)
    tol = (q * (rel + rq + 6 * U * (lqf.abs() + lptf.abs() + 2)) + terms.abs().nan_to_num(posinf=0.0) * (rq + (K + 16) * U)).sum(dim=-1)
    plain = lib.distill_loss(x, ids, z, t)
    both = lib.distill_loss(x, ids, z, t, d_loss=d_loss)
    assert plain.d_logits is None
    for r in (plain, both):
        err = (r.loss.double() - loss).abs()
        ok = (r.loss.double() == loss) | (err <= tol)
        assert bool(ok.all()), float((err - tol)[torch.isfinite(err)].max())
    # the gradient
    G = torch.where(none | empty, 0.0, d_loss.double() / t)[..., None]
    qs = torch.zeros_like(p).scatter_add_(-1, at, q)
    qa = qs
    want = G * (p - qs)
    i = torch.finfo(x.dtype)
    ep = 2 * rel + 8 * U * (torch.where(p > 0, lp.abs(), 0.0) + 2)
    tol = G.abs() * (p * ep + qa * (rq + (K + 4) * U)) + want.abs() * (i.eps / 2 + 4 * U) + i.smallest_normal * i.eps
    for d in (both.d_logits, lib.distill_backward(d_loss, x, ids, z, plain.stats, t), lib.distill_backward(d_loss, x, ids, z, both.stats, t)):
        assert d.dtype == x.dtype and d.is_contiguous()
        err = (d.double() - want).abs()
        assert bool((err <= tol).all()), float((err - tol).max())
        assert bool((d[none | empty] == 0).all())
    return plain, both


def _pairs(g, N, V, K):
    if K <= V:   # distinct tokens
        ids = (torch.randint(0, V, (N, 1), generator=g, device="cuda") + torch.arange(K, device="cuda") * max(1, V // K)) % V
    else:
        ids = torch.randint(0, V, (N, K), generator=g, device="cuda")
    return ids.to(torch.int32)


SHAPES = [(1, 1, 1), (5, 2, 2), (3, 10, 3), (33, 32, 32), (7, 33, 5), (9, 257, 64), (4, 1000, 256), (6, 1024, 8), (5, 1025, 7), (3, 4099, 32), (300, 2049, 4),
          (2, 16384, 20), (3, 16385, 16), (2, 32768, 128), (2, 50021, 32), (1, 131072, 256), (1, 131079, 9), (1, 200003, 64), (700, 1500, 3), (3, 7, 40),
          (900, 2048, 8), (400, 20000, 5), (350, 33000, 2), (330, 1032, 3), (90, 100000, 4)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,K", SHAPES)
def test_distill(dtype, N, V, K):
    g = _gen(N * 1000 + V)
    x, ids = _randn(g, (N, V), dtype, 3.0), _pairs(g, N, V, K)
    _check(x, ids, _randn(g, (N, K), torch.float32, 3.0), 1.0, _randn(g, (N,)))
    _check(x, ids, _randn(g, (N, K), dtype, 3.0), 2.5, _randn(g, (N,)))


# pairs and lengths on either side of every choice between one read and two, and rows enough for a CTA's turn and a segment's
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,K", [(310, 1030, 33), (400, 4096, 64), (7, 4096, 65), (500, 3000, 100), (9, 4097, 128), (5, 2500, 129), (3, 8192, 32), (340, 8193, 32), (6, 8200, 64),
                                   (160, 24313, 33), (12, 24321, 20), (155, 39673, 40), (8, 39681, 32), (6, 65536, 200), (2400, 9000, 256)])
def test_distill_by_one_read_and_by_two(dtype, N, V, K):
    g = _gen(N * 999 + V)
    _check(_randn(g, (N, V), dtype, 3.0), _pairs(g, N, V, K), _randn(g, (N, K), torch.float32, 3.0), 1.5, _randn(g, (N,)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 1500, 20011, 140001])
@pytest.mark.parametrize("pattern", ["no pairs", "some pairs", "one token", "teacher masked", "student masked", "student empty", "constant", "lowest", "far", "learnt", "certain"])
def test_distill_masks_and_extremes(dtype, V, pattern):
    g = _gen(V)
    N, K, t = 5, 12, 1.5
    x, ids, z = _randn(g, (N, V), dtype, 2.0), _pairs(g, N, V, K), _randn(g, (N, K), torch.float32, 2.0)
    if pattern == "no pairs":          # padding: whatever the logits hold
        ids[1:3] = -1
        ids[3] = V
        x[1] = math.nan
        x[2] = -math.inf
    elif pattern == "some pairs":
        ids[:, ::3] = -5
        ids[0, 1:] = V + 7
    elif pattern == "one token":       # the same token in every pair, and in two
        ids[0] = 3
        ids[1, :2] = ids[1, 5]
    elif pattern == "teacher masked":
        z[:, 1::2] = -math.inf
        z[2] = -math.inf
    elif pattern == "student masked":  # a teacher's token among them: the loss is infinite, the gradient is not
        x[torch.rand((N, V), generator=g, device="cuda") < 0.5] = -math.inf
        x[torch.arange(N, device="cuda")[:, None], ids.long()] = 0.5
        x[1, int(ids[1, 4])] = -math.inf
    elif pattern == "student empty":
        x[1] = -math.inf
    elif pattern == "constant":
        x.fill_(1.5)
        z.fill_(-2.0)
    elif pattern == "lowest":
        x.fill_(torch.finfo(dtype).min)
        z.fill_(torch.finfo(torch.float32).min)
        x[1, 7] = 0.0
        ids[1, 0] = 7
        z[1, 0] = 1.0
    elif pattern == "far":
        x, z = (x.float() + 20000.0).to(dtype), z - 30000.0
    elif pattern == "learnt":          # the student is the teacher
        x.fill_(-math.inf)
        x.scatter_(1, ids.long(), z.to(dtype))
        z = z.to(dtype)
    else:
        x[:, 11] = 200.0
        z[:, 0] = 90.0
    if pattern == "no pairs":
        keep = torch.tensor([0, 4], device="cuda")
        _check(x[keep], ids[keep], z[keep], t, _randn(g, (2,)))
        w = _randn(g, (N,))
        r = lib.distill_loss(x, ids, z, t, d_loss=w)
        d = lib.distill_backward(w, x, ids, z, r.stats, t)
        assert bool((r.loss[1:4] == 0).all()) and bool((r.d_logits[1:4] == 0).all()) and bool((d[1:4] == 0).all())
        assert bool((lib.distill_loss(x, ids, z, t).loss[1:4] == 0).all())
        return
    a, b = _check(x, ids, z, t, _randn(g, (N,)))
    if pattern == "student masked":
        assert float(a.loss[1]) == math.inf and bool(torch.isfinite(a.loss[[0, 2, 3, 4]]).all()) and bool(torch.isfinite(b.d_logits).all())
    if pattern == "student empty":
        assert float(a.loss[1]) == math.inf


@pytest.mark.parametrize("V", [100, 5000, 40000])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_distill_nan_and_inf_stay_in_their_row(V, bad):
    g = _gen(V)
    x, ids, z, w = _randn(g, (6, V)), _pairs(g, 6, V, 4), _randn(g, (6, 4)), torch.ones(6, device="cuda")
    w[4] = 0.0
    want = lib.distill_loss(x, ids, z, d_loss=w)
    x[1, 77] = x[4, 30] = bad
    z[2, 3] = bad
    r = lib.distill_loss(x, ids, z, d_loss=w)
    d = lib.distill_backward(w, x, ids, z, r.stats)
    good = torch.tensor([0, 3, 5], device="cuda")
    for a, b in zip(r, want):
        assert torch.equal(a[good], b[good])
    assert bool(torch.isnan(r.loss[[1, 2, 4]]).all())
    for got in (d, r.d_logits):
        assert bool(torch.isnan(got[1]).all()) and bool(torch.isnan(got[2, ids[2].long()]).all()) and bool(torch.isfinite(got[good]).all())
        assert bool((got[4] == 0).all())   # nothing is asked of it


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,pitch,offset", [(1000, 1003, 1), (4097, 4101, 3), (20000, 20008, 5), (33000, 33001, 7)])
def test_distill_of_strided_rows(dtype, V, pitch, offset):
    g = _gen(V)
    buf = _randn(g, (7 * pitch + 16,), dtype, 2.0)
    x = buf[offset:offset + 7 * pitch].view(7, pitch)[:, :V]
    _check(x, _pairs(g, 7, V, 6), _randn(g, (7, 6)), 0.7, _randn(g, (7,)))


@pytest.mark.parametrize("t", [2.0 ** -20, 0.01, 1000.0, 2.0 ** 20])
@pytest.mark.parametrize("V", [50, 3000, 70000])
def test_distill_temperatures(V, t):
    g = _gen(V)
    x = _randn(g, (3, V), torch.float32, min(3.0, 3.0 * t))
    x[0, 5] = -math.inf
    ids = _pairs(g, 3, V, 5)
    ids[ids == 5] = 6
    _check(x, ids, _randn(g, (3, 5), torch.float32, min(3.0, 3.0 * t)), t, _randn(g, (3,)))


def test_distill_gradient_against_differences():
    g = _gen(3)
    N, V, K, t, step = 2, 1100, 6, 1.7, 1e-2
    x, ids, z, w = _randn(g, (N, V)), _pairs(g, N, V, K), _randn(g, (N, K)), _randn(g, (N,))
    d = lib.distill_loss(x, ids, z, t, d_loss=w).d_logits
    for j in (0, 500, int(ids[0, 2]), int(ids[1, 5])):
        e = torch.zeros((N, V), dtype=torch.float64, device="cuda")
        e[:, j] = step
        hi, lo = (_distill_64(x.double() + s * e, ids, z, t)[6].sum(dim=-1) for s in (1, -1))
        diff = w.double() * (hi - lo) / (2 * step)
        # central differences: the third derivative of a log of a sum of exponentials is at most 1 / t^3
        assert bool(((d[:, j].double() - diff).abs() <= w.abs().double() * (step * step + 1e-5)).all())


def test_distill_batch_dims_empty_batches_and_refusals():
    g = _gen(5)
    x, ids, z, w = _randn(g, (3, 4, 50)), _pairs(g, 12, 50, 6).view(3, 4, 6), _randn(g, (3, 4, 6)), _randn(g, (3, 4))
    r = lib.distill_loss(x, ids, z, 2.0, d_loss=w)
    assert r.loss.shape == (3, 4) and r.stats.shape == (3, 4, 2) and r.d_logits.shape == x.shape
    f = lib.distill_loss(x.view(12, 50), ids.view(12, 6), z.view(12, 6), 2.0, d_loss=w.view(12))
    assert torch.equal(f.loss, r.loss.view(12)) and torch.equal(f.d_logits, r.d_logits.view(12, 50))
    e = lib.distill_loss(x[:0], ids[:0], z[:0], d_loss=w[:0])
    assert e.loss.shape == (0, 4) and e.d_logits.shape == (0, 4, 50)
    assert lib.distill_backward(w[:0], x[:0], ids[:0], z[:0], e.stats).shape == (0, 4, 50)
    for bad in (lambda: lib.distill_loss(x.transpose(0, 2), ids, z), lambda: lib.distill_loss(x, ids.long(), z), lambda: lib.distill_loss(x, ids, z[..., :5]),
                lambda: lib.distill_loss(x, ids[:2], z[:2]), lambda: lib.distill_loss(x, ids[..., :0], z[..., :0]), lambda: lib.distill_loss(x, ids, z, 0.0),
                lambda: lib.distill_loss(x, ids, z, math.nan), lambda: lib.distill_loss(x, ids, z.double()), lambda: lib.distill_loss(x.cpu(), ids, z),
                lambda: lib.distill_loss(x, ids, z, d_loss=w.double()), lambda: lib.distill_loss(x, ids, z, d_loss=w[:2]),
                lambda: lib.distill_backward(w, x, ids, z, r.loss), lambda: lib.distill_backward(None, x, ids, z, r.stats),
                lambda: lib.distill_loss(x, ids.expand(50, 3, 4, 6)[0].repeat(1, 1, 50), z.repeat(1, 1, 50))):
        with pytest.raises((ValueError, AttributeError)):
            bad()
