"""Routing to experts, products by expert and their combination against their definitions in 64 bits.

Tolerances count roundings.  U = 2^-24 is half a step of fp32; a result rounded to type t is off by finfo(t).eps / 2
relative, or by half the type's least step."""
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


def _rounding(want, dtype):
    i = torch.finfo(dtype)
    return want.abs() * (i.eps / 2) + i.smallest_normal * i.eps


# ------------------------------------------------------------------------------------ routing

def _route_64(x, k, normalise):
    """(weights, ids, chosen) by the definition: stable sort, -inf never chosen."""
    x = x.double()
    v, i = torch.sort(x, dim=2, descending=True, stable=True)
    v, i = v[..., :k], i[..., :k]
    live = v > -math.inf
    d = v - torch.where(live[..., :1], v[..., :1], 0.0)
    e = torch.where(live, torch.exp(d), 0.0)
    if normalise:
        total = e.sum(dim=2, keepdim=True)
    else:
        total = torch.exp(x - torch.where(live[..., :1], v[..., :1], 0.0)).sum(dim=2, keepdim=True)
    w = torch.where(live, e / torch.where(total > 0, total, 1.0), 0.0)
    return w, torch.where(live, i, -1), live


def _check_tables(ids, r, E):
    m, T, k = ids.shape
    for w in range(m):
        flat = ids[w].reshape(-1)
        slots = torch.nonzero(flat >= 0)[:, 0]
        order = slots[torch.sort(flat[slots], stable=True).indices]
        n = order.numel()
        places = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
        places[order] = torch.arange(n, dtype=torch.int32, device="cuda")
        tokens = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
        tokens[:n] = (order // k).int()
        ends = torch.cumsum(torch.bincount(flat[slots], minlength=E), 0).int()
        assert torch.equal(r.places[w].reshape(-1), places) and torch.equal(r.tokens[w], tokens)
        assert int(r.offsets[w, 0]) == 0 and torch.equal(r.offsets[w, 1:], ends)


def _exp_error(x, E):
    """Relative error of a quotient of exponentials e^d, sum e^d: |d| u for the difference d, 2 steps (4 u) for each exponential and the
    division, a chain of E / 32 + 6 additions."""
    finite = torch.where(torch.isinf(x), 0.0, x.double())
    return (2 * (finite.amax() - finite.amin()) + E / 32 + 6 + 12) * U


def _check_route(x, k, normalise, g=None):
    r = lib.expert_route(x, k, normalise)
    w, ids, live = _route_64(x, k, normalise)
    assert torch.equal(r.ids.long(), ids)
    rel = _exp_error(x, x.shape[2])
    assert bool(((r.weights.double() - w).abs() <= w * rel + 2.0 ** -126).all())
    _check_tables(ids, r, x.shape[2])
    if g is not None:
        dw = _randn(g, r.weights.shape)
        d = lib.expert_route_backward(dw, x, r.ids, r.weights, normalise)
        G = torch.zeros(x.shape, dtype=torch.float64, device="cuda").scatter_add_(2, ids.clamp(min=0), torch.where(live, dw.double(), 0.0))
        chosen = torch.zeros_like(G).scatter_add_(2, ids.clamp(min=0), live.double()) > 0
        top = x.double().amax(dim=2, keepdim=True)
        e = torch.exp(x.double() - torch.where(top > -math.inf, top, 0.0))
        if normalise:
            e = torch.where(chosen, e, 0.0)
        p = e / e.sum(dim=2, keepdim=True).clamp(min=1e-300)
        mean, size = (p * G).sum(dim=2, keepdim=True), (p * G.abs()).sum(dim=2, keepdim=True)
        want = p * (G - mean)
        tol = p * ((G.abs() + size) * (2 * rel + (k + 8) * U)) + _rounding(want, x.dtype)
        assert bool(((d.double() - want).abs() <= tol).all())
        if normalise:
            assert bool((d[~chosen] == 0).all())
    return r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("m,T,E,k", [(1, 1, 1, 1), (1, 1, 2, 2), (2, 7, 5, 3), (1, 8, 64, 8), (3, 33, 32, 2), (1, 1000, 33, 4), (2, 4097, 8, 2), (1, 300, 100, 6),
                                     (1, 65, 128, 32), (2, 129, 257, 5), (1, 70, 1000, 17), (1, 40, 1024, 32), (1, 20000, 16, 1), (160, 40, 9, 2), (40, 500, 6, 3)])
def test_route(dtype, normalise, m, T, E, k):
    g = _gen(m * T + E)
    _check_route(_randn(g, (m, T, E), dtype, 1.5), k, normalise, g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("T", [20, 6000])
@pytest.mark.parametrize("pattern", ["padding", "few left", "ties", "lowest", "one expert", "all padding", "far"])
def test_route_masks_and_ties(dtype, normalise, T, pattern):
    g = _gen(T)
    m, E, k = 2, 24, 4
    x = _randn(g, (m, T, E), dtype)
    if pattern == "padding":
        x[torch.rand((m, T), generator=g, device="cuda") < 0.4] = -math.inf
    elif pattern == "few left":   # fewer experts than k
        x[torch.rand((m, T, E), generator=g, device="cuda") < 0.9] = -math.inf
    elif pattern == "ties":
        x = torch.round(x)
    elif pattern == "lowest":
        x[torch.rand((m, T, E), generator=g, device="cuda") < 0.95] = torch.finfo(dtype).min
    elif pattern == "one expert":
        x[..., 5] = 9.0
        x[..., 7] = 8.0
    elif pattern == "all padding":
        x.fill_(-math.inf)
    else:
        x = x + 30000.0
    if pattern == "lowest":   # differences that overflow to -inf are zeros on both sides
        x64 = x.clone()
        r = lib.expert_route(x, k, normalise)
        w, ids, _ = _route_64(x64, k, normalise)
        assert torch.equal(r.ids.long(), ids)
        assert bool(((r.weights.double() - w).abs() <= w * 60 * U + 2.0 ** -126).all())
        _check_tables(ids, r, E)
    else:
        _check_route(x, k, normalise, g)


def test_route_nan_and_inf_stay_in_their_token():
    g = _gen(3)
    x = _randn(g, (1, 50, 20))
    want = lib.expert_route(x, 3)
    x[0, 4, 7], x[0, 9, 2] = math.nan, math.inf
    keep = [t for t in range(50) if t not in (4, 9)]
    for normalise in (True, False):
        r = lib.expert_route(x, 3, normalise)
        assert int(r.ids[0, 4, 0]) == 7 and int(r.ids[0, 9, 0]) == 2
        assert bool(torch.isnan(r.weights[0, 4]).all()) and bool(torch.isnan(r.weights[0, 9, 0]))
        assert torch.equal(r.ids[0, keep], want.ids[0, keep])
        d = lib.expert_route_backward(torch.ones_like(r.weights), x, r.ids, r.weights, normalise)
        assert bool(torch.isfinite(d[0, keep]).all())


def test_route_of_strided_rows_empty_batches_and_refusals():
    g = _gen(4)
    buf = _randn(g, (2, 30, 41))
    x = buf[:, :, 3:38]
    _check_route(x, 4, False, g)
    a, b = lib.expert_route(x, 4), lib.expert_route(x.contiguous(), 4)
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    e = lib.expert_route(x[:, :0], 4)
    assert e.weights.shape == (2, 0, 4) and e.tokens.shape == (2, 0) and bool((e.offsets == 0).all())
    assert lib.expert_route_backward(e.weights, x[:, :0], e.ids, e.weights).shape == (2, 0, 35)
    for bad in (lambda: lib.expert_route(x[0], 2), lambda: lib.expert_route(x, 0), lambda: lib.expert_route(x, 33), lambda: lib.expert_route(x.double(), 2),
                lambda: lib.expert_route(x.transpose(0, 1), 2), lambda: lib.expert_route(x.transpose(1, 2), 2), lambda: lib.expert_route(buf.new_zeros(1, 2, 1025), 2),
                lambda: lib.expert_route_backward(a.weights.double(), x, a.ids, a.weights), lambda: lib.expert_route_backward(a.weights, x, a.ids.long(), a.weights),
                lambda: lib.expert_route_backward(a.weights[:1], x, a.ids, a.weights)):
        with pytest.raises(ValueError):
            bad()


# ----------------------------------------------------------------------------------- combining

def _slots(g, m, T, k, gone=0.1):
    """places, tokens of a random order of the slots; some tokens have none."""
    R = T * k
    places = torch.full((m, R), -1, dtype=torch.int32, device="cuda")
    tokens = torch.full((m, R), -1, dtype=torch.int32, device="cuda")
    for w in range(m):
        live = torch.nonzero((torch.rand(T, generator=g, device="cuda") >= gone).repeat_interleave(k))[:, 0]
        order = live[torch.randperm(live.numel(), generator=g, device="cuda")]
        places[w, order] = torch.arange(order.numel(), dtype=torch.int32, device="cuda")
        tokens[w, :order.numel()] = (order // k).int()
    return places.view(m, T, k), tokens


def _check_combine(rows, places, tokens, weights, dy):
    m, T, k = places.shape
    D, dtype = rows.shape[2], rows.dtype
    has = (places >= 0)[..., None]
    at = places.clamp(min=0).long()
    picked = torch.stack([rows[w].double()[at[w]] for w in range(m)]) if rows.shape[1] else torch.zeros((m, T, k, D), dtype=torch.float64, device="cuda")
    picked = torch.where(has, picked, 0.0)
    for w in (weights, None):
        W = torch.ones_like(places, dtype=torch.float64) if w is None else w.double()
        y = lib.expert_combine(rows, places, w)
        want, size = (W[..., None] * picked).sum(dim=2), (W.abs()[..., None] * picked.abs()).sum(dim=2)
        assert bool(((y.double() - want).abs() <= size * (k + 1) * U + _rounding(want, dtype)).all())
    d_rows, d_w = lib.expert_combine_backward(dy, rows, places, tokens, weights)
    E = dy.double()[:, :, None]
    want, size = (E * picked).sum(dim=3), (E * picked).abs().sum(dim=3)
    # eight products a piece in a chain, D / 256 pieces a lane (D / 32 where rows are walked one by one), 13 joins
    assert bool(((d_w.double() - want).abs() <= size * (D / 32 + 24) * U + 2.0 ** -126).all())
    want = torch.zeros(rows.shape, dtype=torch.float64, device="cuda")
    for w in range(m):
        live = places[w].reshape(-1) >= 0
        want[w][at[w].reshape(-1)[live]] = (weights[w].double()[..., None] * E[w]).expand(T, k, D).reshape(-1, D)[live]
    assert bool(((d_rows.double() - want).abs() <= want.abs() * U + _rounding(want, dtype)).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,T,k,D", [(1, 1, 1, 1), (1, 1, 8, 64), (2, 5, 3, 7), (1, 8, 8, 1024), (3, 33, 2, 1021), (1, 100, 2, 2048), (2, 40, 5, 4100), (1, 30, 1, 8192),
                                     (2, 64, 9, 72), (1, 1000, 4, 257), (1, 6, 2, 16385)])
def test_combine(dtype, m, T, k, D):
    g = _gen(T * k + D)
    places, tokens = _slots(g, m, T, k)
    _check_combine(_randn(g, (m, T * k, D), dtype), places, tokens, torch.rand((m, T, k), generator=g, device="cuda"), _randn(g, (m, T, D), dtype))


def test_combine_reads_no_rows_that_no_token_has():
    g = _gen(1)
    places, tokens = _slots(g, 2, 40, 3, gone=0.5)
    rows, dy, w = _randn(g, (2, 120, 48)), _randn(g, (2, 40, 48)), torch.rand((2, 40, 3), generator=g, device="cuda")
    want = [lib.expert_combine(rows, places, w), *lib.expert_combine_backward(dy, rows, places, tokens, w)]
    rows[tokens < 0] = math.nan
    gone = (places < 0).all(dim=2)
    assert bool(gone.any())
    dy[gone], w[gone] = math.nan, math.nan
    got = [lib.expert_combine(rows, places, w), *lib.expert_combine_backward(dy, rows, places, tokens, w)]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool((got[0][gone] == 0).all()) and bool((got[1][tokens < 0] == 0).all()) and bool((got[2][gone] == 0).all())
    # places outside the rows, of any value, are no rows
    wild = torch.where(places < 0, torch.tensor([120, -7, 2 ** 31 - 1], dtype=torch.int32, device="cuda").expand_as(places), places)
    assert torch.equal(lib.expert_combine(rows, wild, w), want[0])
    assert all(torch.equal(a, b) for a, b in zip(lib.expert_combine_backward(dy, rows, wild, tokens, w), want[1:]))


def test_combine_shapes_strides_and_refusals():
    g = _gen(2)
    places, tokens = _slots(g, 2, 20, 2)
    buf, gbuf = _randn(g, (2, 45, 67), torch.bfloat16), _randn(g, (2, 25, 70), torch.bfloat16)
    w = torch.rand((2, 20, 2), generator=g, device="cuda")
    for rows, dy in ((buf[:, 3:43, 1:65], gbuf[:, 2:22, 5:69]), (buf[:, :40, :64], gbuf[:, :20, :64])):
        _check_combine(rows, places, tokens, w, dy)
    rows, dy = buf[:, :40, :64].contiguous(), gbuf[:, :20, :64].contiguous()
    # more rows than slots, and fewer (the others are nowhere)
    more = torch.cat([rows, rows], dim=1)
    d_rows, _ = lib.expert_combine_backward(dy, more, places, torch.cat([tokens, torch.full_like(tokens, -1)], dim=1), w)
    assert bool((d_rows[:, 40:] == 0).all())
    fewer = torch.where(places < 11, places, -1)
    _check_combine(rows[:, :11], fewer, tokens[:, :11].contiguous(), w, dy)
    none = torch.full_like(places, -1)
    _check_combine(rows[:, :0], none, tokens[:, :0], w, dy)
    assert lib.expert_combine(rows, places[:, :0]).shape == (2, 0, 64)
    d_rows, d_w = lib.expert_combine_backward(dy[:, :0], rows, places[:, :0], torch.full_like(tokens, -1), w[:, :0])
    assert bool((d_rows == 0).all()) and d_w.shape == (2, 0, 2)
    for bad in (lambda: lib.expert_combine(rows, places.long()), lambda: lib.expert_combine(rows, places, w.double()), lambda: lib.expert_combine(rows[0], places),
                lambda: lib.expert_combine(rows.transpose(1, 2), places), lambda: lib.expert_combine(rows, places[:1]), lambda: lib.expert_combine(rows.double(), places),
                lambda: lib.expert_combine_backward(dy.float(), rows, places, tokens, w), lambda: lib.expert_combine_backward(dy, rows, places, tokens[:, :-1], w),
                lambda: lib.expert_combine_backward(dy, rows, places, tokens, None)):
        with pytest.raises((ValueError, AttributeError)):
            bad()


# ------------------------------------------------------------------------------------ products

def _product_error(K):
    """Relative to sum |x||w|: products of 16-bit values are exact in fp32; the tensor cores add up groups of at least eight in
    one step each, off by at most 2 U (they may cut off instead of rounding), and K / 8 of them in a chain."""
    return (K / 8 + 8) * 2 * U


def _offsets(sizes, lead=0):
    return torch.tensor([[lead + sum(n[:e]) for e in range(len(n) + 1)] for n in sizes], dtype=torch.int32, device="cuda")


def _check_product(x, w, offsets, dy, sizes=None):
    m, R, D = x.shape
    E, F = w.shape[1:3]
    dtype = x.dtype
    y = lib.expert_product(x, w, offsets)
    dx, dw = lib.expert_product_backward(dy, x, w, offsets)
    ends = offsets.tolist()
    for i in range(m):
        inside = torch.zeros(R, dtype=torch.bool, device="cuda")
        for e in range(E):
            part = slice(ends[i][e], ends[i][e + 1])
            inside[part] = True
            X, W, G = x[i, part].double(), w[i, e].double(), dy[i, part].double()
            for got, want, size, K in ((y[i, part], X @ W.T, X.abs() @ W.abs().T, D), (dx[i, part], G @ W, G.abs() @ W.abs(), F),
                                       (dw[i, e], G.T @ X, G.abs().T @ X.abs(), X.shape[0])):
                assert bool(((got.double() - want).abs() <= size * _product_error(K) + _rounding(want, dtype)).all()), (i, e)
        assert bool((y[i, ~inside] == 0).all()) and bool((dx[i, ~inside] == 0).all())
    only_x, only_w = lib.expert_product_backward(dy, x, w, offsets, want_d_w=False), lib.expert_product_backward(dy, x, w, offsets, want_d_x=False)
    assert only_x[1] is None and only_w[0] is None and torch.equal(only_x[0], dx) and torch.equal(only_w[1], dw)
    lib.operators_join()
    return y, dx, dw


SIZES = [(1, [[1]], 0, 8, 8), (1, [[1]], 0, 1, 1), (2, [[3, 0], [0, 5]], 2, 16, 24), (1, [[0, 0, 0]], 7, 64, 64), (1, [[17, 1, 0, 30]], 3, 72, 130),
         (2, [[64, 128, 16], [15, 0, 193]], 5, 64, 128), (1, [[255, 256, 257, 1, 31, 33]], 0, 128, 256), (1, [[1000]], 24, 256, 300),
         (3, [[5] * 12, [0] * 11 + [60], [60] + [0] * 11], 0, 33, 21), (1, [[513, 40]], 1, 1021, 515), (1, [[2, 0, 1] * 40], 0, 520, 1040),
         (1, [[700, 900]], 0, 2048, 40), (1, [[300, 4, 700]], 20, 40, 2048), (4, [[100, 28]] * 4, 0, 256, 256), (1, [[2500, 1800]], 0, 512, 768)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,sizes,behind,D,F", SIZES)
def test_product(dtype, m, sizes, behind, D, F):
    g = _gen(D + F)
    R, E = max(sum(n) for n in sizes) + behind, len(sizes[0])
    _check_product(_randn(g, (m, R, D), dtype), _randn(g, (m, E, F, D), dtype, 0.3), _offsets(sizes), _randn(g, (m, R, F), dtype))


def test_product_of_many_workers_and_experts():
    """More groups than one launch's table holds."""
    g = _gen(9)
    for m, E, n in ((40, 64, 1), (300, 8, 2), (3, 1024, 1), (1500, 1, 3)):
        sizes = [[n] * E for _ in range(m)]
        _check_many(_randn(g, (m, E * n, 24), torch.bfloat16), _randn(g, (m, E, 16, 24), torch.bfloat16), _offsets(sizes), _randn(g, (m, E * n, 16), torch.bfloat16), n)


def _check_many(x, w, offsets, dy, n):
    m, R, D = x.shape
    E, F = w.shape[1:3]
    y = lib.expert_product(x, w, offsets)
    dx, dw = lib.expert_product_backward(dy, x, w, offsets)
    X, G, W = x.double().view(m * E, n, D), dy.double().view(m * E, n, F), w.double().view(m * E, F, D)
    for got, want, size, K in ((y.view(m * E, n, F), X @ W.mT, X.abs() @ W.abs().mT, D), (dx.view(m * E, n, D), G @ W, G.abs() @ W.abs(), F),
                               (dw.view(m * E, F, D), G.mT @ X, G.abs().mT @ X.abs(), n)):
        assert bool(((got.double() - want).abs() <= size * _product_error(K) + _rounding(want, x.dtype)).all())


# few tiles and a long sum: over the features, over a group's rows (one group with nearly all of them, groups with none), or both
PARTS = [(1, [[5, 0, 3]], 4, 4096, 136), (1, [[3000, 0]], 2, 72, 40), (2, [[2000], [7]], 1, 77, 45), (1, [[9000, 70, 0, 1]], 10, 128, 256),
         (1, [[1, 0]], 0, 8192, 4096), (1, [[300]], 50, 4095, 1030), (3, [[2, 700], [1, 1], [0, 0]], 9, 130, 2050), (1, [[40000]], 0, 32, 32)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,sizes,behind,D,F", PARTS)
def test_product_in_parts(dtype, m, sizes, behind, D, F):
    g = _gen(D + F + 1)
    R, E = max(sum(n) for n in sizes) + behind, len(sizes[0])
    offsets = _offsets(sizes, lead=min(behind, 1))
    x, w, dy = _randn(g, (m, R, D), dtype), _randn(g, (m, E, F, D), dtype, 0.1), _randn(g, (m, R, F), dtype, 0.1)
    first = _check_product(x, w, offsets, dy)
    x2 = torch.cat([x.flip(1), x], dim=1)[:, R:]   # (same values, other strides between workers)
    assert all(torch.equal(a, b) for a, b in zip(_check_product(x2, w, offsets, dy), first))


@pytest.mark.parametrize("pad", [0, 1, 8])
def test_product_of_strided_operands(pad):
    """Weights as views of rows that hold all of a worker's parameters, rows as slices; with 16-byte pitches and without."""
    g = _gen(pad)
    m, E, R, D, F, dtype = 3, 4, 90, 128, 72, torch.bfloat16
    per = E * (F + 1) * (D + pad)
    flat = _randn(g, (m, per + 2 * pad + 40 * (pad > 0)), dtype, 0.2)
    w = flat[:, pad:pad + per].unflatten(1, (E, F + 1, D + pad))[:, :, :F, :D]
    x = _randn(g, (m, R + 5, D + pad), dtype)[:, 2:R + 2, :D]
    dy = _randn(g, (m, R + 1, F + pad), dtype)[:, 1:, pad:]
    offsets = _offsets([[20, 0, 33, 30], [90, 0, 0, 0], [1, 2, 3, 4]])
    got = _check_product(x, w, offsets, dy)
    want = lib.expert_product(x.contiguous(), w.contiguous(), offsets), *lib.expert_product_backward(dy.contiguous(), x.contiguous(), w.contiguous(), offsets)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("D,F", [(192, 128), (64, 136), (136, 320)])
def test_product_of_slices_among_nan(D, F):
    """Operands inside larger tensors of NaN, rows of whole panels of 64 columns and others: nothing around a slice is used."""
    g = _gen(D + F)
    m, E, R, dtype = 2, 3, 151, torch.float16
    offsets = _offsets([[70, 0, 61], [1, 129, 3]], lead=9)

    def inside(shape, std=1.0):
        big = torch.full((shape[0], *(n + 16 for n in shape[1:])), math.nan, dtype=dtype, device="cuda")
        part = big[(slice(None),) + tuple(slice(8, 8 + n) for n in shape[1:])]
        part.copy_(_randn(g, shape, dtype, std))
        return part
    x, w, dy = inside((m, R, D)), inside((m, E, F, D), 0.3), inside((m, R, F))
    for i, (a, b) in enumerate(((9, 140), (9, 142))):   # rows of no expert
        x[i, :a], x[i, b:], dy[i, :a], dy[i, b:] = math.nan, math.nan, math.nan, math.nan
    y, dx, dw = lib.expert_product(x, w, offsets), *lib.expert_product_backward(dy, x, w, offsets)
    assert bool(y.isfinite().all()) and bool(dx.isfinite().all()) and bool(dw.isfinite().all())
    x, dy = x.nan_to_num(0.0), dy.nan_to_num(0.0)
    got = _check_product(x, w.contiguous(), offsets, dy)
    assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw)))


def test_product_in_parts_side_by_side_and_replayed():
    """Sums by parts use a workspace: two streams at once, and a captured call whose inputs change, each get their own."""
    g = _gen(4)
    m, R, E, D, F, dtype = 1, 3000, 2, 512, 64, torch.bfloat16
    offsets = [_offsets([[2100, 900]]), _offsets([[0, 2999]])]
    x, w, dy = [_randn(g, (m, R, D), dtype) for _ in range(2)], _randn(g, (m, E, F, D), dtype, 0.2), [_randn(g, (m, R, F), dtype) for _ in range(2)]

    def both(i):
        return (lib.expert_product(x[i], w, offsets[i]), *lib.expert_product_backward(dy[i], x[i], w, offsets[i]))
    want = [both(0), both(1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append(both(i))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for i in range(2) for a, b in zip(got[i], want[i]))
    graph = torch.cuda.CUDAGraph()
    kept = [t.clone() for t in (x[0], dy[0], offsets[0])]
    with torch.cuda.graph(graph):
        out = both(0)
    for i in (1, 0, 1):
        for t, new in zip((x[0], dy[0], offsets[0]), (x[1], dy[1], offsets[1]) if i else kept):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
    lib.operators_join()


@pytest.mark.parametrize("D,F", [(64, 128), (70, 50)])
def test_product_extremes_stay_in_their_rows_and_experts(D, F):
    g = _gen(D)
    sizes = [[37, 0, 64, 90, 3]]
    R = 210
    x, w, dy = _randn(g, (1, R, D), torch.float16), _randn(g, (1, 5, F, D), torch.float16, 0.3), _randn(g, (1, R, F), torch.float16)
    offsets = _offsets(sizes)
    want = lib.expert_product(x, w, offsets), *lib.expert_product_backward(dy, x, w, offsets)
    # rows behind the last group may hold anything; one row of expert 2 is NaN, another of it infinite
    x[:, 194:], dy[:, 194:] = math.nan, math.inf
    x[0, 40], dy[0, 50] = math.nan, math.inf
    y, (dx, dw) = lib.expert_product(x, w, offsets), lib.expert_product_backward(dy, x, w, offsets)
    rows = [r for r in range(R) if r != 40]
    assert torch.equal(y[0, rows], want[0][0, rows]) and bool(torch.isnan(y[0, 40]).all())
    rows = [r for r in range(R) if r != 50]
    assert torch.equal(dx[0, rows], want[1][0, rows]) and not bool(torch.isfinite(dx[0, 50]).any())
    assert torch.equal(dw[0, [0, 1, 3, 4]], want[2][0, [0, 1, 3, 4]]) and bool(torch.isnan(dw[0, 2]).all())
    assert bool((dw[0, 1] == 0).all())


def test_product_offsets_that_do_not_rise_stay_within_bounds():
    """Undefined for the experts concerned, but nothing outside the outputs is touched, rows of the others are right and the call ends."""
    g = _gen(8)
    m, R, E, D, F = 2, 100, 4, 64, 48
    x, w, dy = _randn(g, (m, R, D), torch.bfloat16), _randn(g, (m, E, F, D), torch.bfloat16), _randn(g, (m, R, F), torch.bfloat16)
    wild = torch.tensor([[0, 30, 20, 60, 60], [-5, 40, 40, 2 ** 31 - 1, 90]], dtype=torch.int32, device="cuda")
    y = lib.expert_product(x, w, wild)
    lib.expert_product_backward(dy, x, w, wild)
    lib.operators_join()
    as_taken = torch.tensor([[0, 30, 30, 60, 60], [0, 40, 40, 100, 100]], dtype=torch.int32, device="cuda")
    assert torch.equal(y, lib.expert_product(x, w, as_taken))
    leading = torch.tensor([[10, 30, 50, 60, 60], [99, 99, 100, 100, 100]], dtype=torch.int32, device="cuda")
    _check_product(x, w, leading, dy)


def test_product_shapes_and_refusals():
    g = _gen(7)
    x, w, dy = _randn(g, (2, 9, 16), torch.bfloat16), _randn(g, (2, 3, 8, 16), torch.bfloat16), _randn(g, (2, 9, 8), torch.bfloat16)
    o = _offsets([[4, 5, 0], [0, 0, 1]])
    assert lib.expert_product(x[:, :0], w, o * 0).shape == (2, 0, 8)
    dx, dw = lib.expert_product_backward(dy[:, :0], x[:, :0], w, o * 0)
    assert dx.shape == (2, 0, 16) and bool((dw == 0).all())
    for bad in (lambda: lib.expert_product(x.float(), w.float(), o), lambda: lib.expert_product(x, w.half(), o), lambda: lib.expert_product(x, w, o.long()),
                lambda: lib.expert_product(x, w, o[:, 1:]), lambda: lib.expert_product(x, w[:1], o), lambda: lib.expert_product(x[:, :, :8], w, o),
                lambda: lib.expert_product(x.transpose(1, 2), w, o), lambda: lib.expert_product(x, w.transpose(2, 3), o), lambda: lib.expert_product(x, w.cpu(), o),
                lambda: lib.expert_product_backward(dy[:, :8], x, w, o), lambda: lib.expert_product_backward(dy.half(), x, w, o)):
        with pytest.raises(ValueError):
            bad()


def test_product_gradients_against_differences():
    g = _gen(5)
    x, w, dy = _randn(g, (1, 7, 16), torch.float16), _randn(g, (1, 2, 8, 16), torch.float16, 0.3), _randn(g, (1, 7, 8), torch.float16)
    o = _offsets([[3, 4]])
    dx, dw = lib.expert_product_backward(dy, x, w, o)
    X, W, G, step = x.double(), w.double(), dy.double(), 1e-3

    def loss(X, W):
        return float((X[0, :3] @ W[0, 0].T * G[0, :3]).sum() + (X[0, 3:] @ W[0, 1].T * G[0, 3:]).sum())

    for got, which, at in ((dx, 0, (0, 1, 5)), (dx, 0, (0, 6, 15)), (dw, 1, (0, 0, 2, 3)), (dw, 1, (0, 1, 7, 15))):
        lo, hi = [X.clone(), W.clone()], [X.clone(), W.clone()]
        lo[which][at] -= step
        hi[which][at] += step
        diff = (loss(*hi) - loss(*lo)) / (2 * step)   # linear: exact but for 64-bit rounding
        assert abs(float(got[at]) - diff) <= (abs(diff) + 1e-3) * 2.0 ** -11 + 1e-9 + 30 * 2 * U * 30
