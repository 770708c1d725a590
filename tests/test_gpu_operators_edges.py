"""The operators on caller-owned tensors at the edges of what their documentation allows: values next to a border, at the
ends of a type's range, and data whose cost must not depend on its values.

Tolerances count roundings, as in test_gpu_operators.py."""
import math

import pytest
import torch

import paper_2002_09539_b200 as lib
from paper_2002_09539_b200 import OverlapLocalSGD

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _product_error(K):
    """Relative to sum |x||w|, as in test_gpu_operators.py."""
    return (K / 8 + 8) * 2 * U


def _microseconds(fn, n=15):
    for _ in range(3):
        fn()
    times = []
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        fn()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return sorted(times)[n // 2]


# ------------------------------------------------------------------------ relu's border

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 71])
@pytest.mark.parametrize("F,features", [(1, [0]), (257, [256]), (40, [3, 17]), (520, list(range(520)))])
@pytest.mark.parametrize("how", ["cancelled", "wrong side"])
def test_relu_border_goes_by_the_feature_s_own_size(F, features, how, D, dtype):
    """Gates that fp32 cancels to nothing, or to the wrong sign (a term that is lost beside 2^10, which then goes away): alone, last
    in their block of columns, beside gates that are far smaller, and all at once."""
    g = _gen(F + D)
    T = 4
    x, wg, wu = _randn(g, (1, T, D), dtype), _randn(g, (1, F, D), dtype, 2.0 ** -9), _randn(g, (1, F, D), dtype)
    dh = _randn(g, (1, T, F), dtype)
    at = torch.tensor(features, device="cuda")
    sign = torch.where(at % 3 == 0, 1.0, -1.0).to(dtype)
    x[0, 2] = 0.0
    wg[0, at] = 0.0
    if how == "cancelled":      # 2^10 - 2^10 +- 2^-18
        x[0, 2, 0] = x[0, 2, 1] = 32.0
        x[0, 2, 2] = 2.0 ** -9
        wg[0, at, 0], wg[0, at, 1], wg[0, at, 2] = 32.0, -32.0, sign * 2.0 ** -9
    else:                       # +-(2^10 + 2^-15 - 2^10 - 2^-17), each term in another group of 16
        x[0, 2, 0] = x[0, 2, 32] = 32.0
        x[0, 2, 16], x[0, 2, 48] = 2.0 ** -5, 2.0 ** -8
        wg[0, at, 0], wg[0, at, 32] = sign * 32.0, sign * -32.0
        wg[0, at, 16], wg[0, at, 48] = sign * 2.0 ** -10, sign * -(2.0 ** -9)
    a = x.double() @ wg.double().mT
    assert bool((torch.sign(a[0, 2, at]) == sign.double()).all())
    _, pre = lib.gated_forward(x, wg, wu, "relu", save=True)
    dx, dwg, dwu = lib.gated_backward(dh, x, wg, wu, pre, "relu")
    da, db = dh.double() * (x.double() @ wu.double().mT) * (a > 0), dh.double() * a.clamp(min=0)
    eps = torch.finfo(dtype).eps
    # fp16 steps of 2^-24 below 2^-14: db = dh 2^-18 is rounded there, off by up to 2^-25 before it meets the weights, and so
    # may be da
    step = 2.0 ** -25 if dtype == torch.float16 else 0.0
    want, size = (da.mT @ x.double())[0], (da.abs().mT @ x.double().abs())[0]
    below = step * (1 + x.double().abs().sum(dim=1))[0]
    assert bool(((dwg[0, at].double() - want[at]).abs() <= size[at] * (2 * eps + _product_error(T)) + below).all())
    want = (da @ wg.double() + db @ wu.double())[0, 2]
    size = (da.abs() @ wg.double().abs() + db.abs() @ wu.double().abs())[0, 2]
    below = step * (1 + (wg.double().abs() + wu.double().abs()).sum(dim=1))[0]
    assert bool(((dx[0, 2].double() - want).abs() <= size * (2 * eps + _product_error(2 * F)) + below).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("data", ["zero features", "zero tokens", "integers", "one element", "large", "small"])
def test_relu_gradient_of_exact_zeros(data, dtype):
    """Data whose gates are exactly 0, or whose rows' norms are at the ends of fp32: against the definition in 64 bits."""
    g = _gen(7)
    T, D, F = 70, 133, 75
    x, wg, wu, dh = (_randn(g, s, dtype) for s in ((2, T, D), (2, F, D), (2, F, D), (2, T, F)))
    if data == "zero features":
        wg[:, ::3] = 0
    elif data == "zero tokens":
        x[:, ::2] = 0
    elif data == "integers":
        x, wg = torch.round(x), torch.round(wg)
    elif data == "one element":
        x.zero_()
        x[:, torch.arange(T), torch.arange(T)] = 1.5
        wg *= (torch.rand(wg.shape, generator=g, device="cuda") < 0.2)
    elif dtype == torch.float16:
        x *= 2.0 ** 7 if data == "large" else 2.0 ** -12
    else:
        x *= 2.0 ** 50 if data == "large" else 2.0 ** -70
        dh *= 2.0 ** -50 if data == "large" else 2.0 ** 70
    a, b = x.double() @ wg.double().mT, x.double() @ wu.double().mT
    E, half = dh.double(), torch.finfo(dtype).eps / 2
    _, pre = lib.gated_forward(x, wg, wu, "relu", save=True)
    dx, dwg, _ = lib.gated_backward(dh, x, wg, wu, pre, "relu")
    da, db = E * b * (a > 0), E * a.clamp(min=0)
    ea, eb = (_product_error(D) * (x.double().abs() @ w.double().abs().mT) for w in (wg, wu))
    # fp16's steps below its normal range: 2^-24, or 2^-38 of a worker's largest value where that is beyond 2^15
    step = torch.maximum(da.abs().amax(dim=(1, 2)), db.abs().amax(dim=(1, 2))).mul(2.0 ** -38).clamp(min=2.0 ** -24)[:, None, None]
    step = step if dtype == torch.float16 else 0.0
    eda, edb = E.abs() * eb + da.abs() * (half + 4 * U) + step, E.abs() * ea + db.abs() * (half + 4 * U) + step
    wants = ((dx, da @ wg.double() + db @ wu.double(), eda @ wg.double().abs() + edb @ wu.double().abs(), da.abs() @ wg.double().abs() + db.abs() @ wu.double().abs(), 2 * F),
             (dwg, da.mT @ x.double(), eda.mT @ x.double().abs(), da.abs().mT @ x.double().abs(), T))
    for got, want, err, size, K in wants:
        tol = err * 1.01 + _product_error(K) * (size + err) + want.abs() * half * 1.01 + (2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126)
        there = want.abs() + tol < torch.finfo(dtype).max   # (what comes closer to the largest may be rounded to infinity)
        assert bool((((got.double() - want).abs() <= tol) | ~there).all())


def test_relu_gradient_costs_the_same_whatever_the_zeros():
    """Zero features, zero tokens and integers are ordinary: no more than half again the time of random values (by the sides
    of every zero in 64 bits it was 13 times)."""
    g = _gen(3)
    T, D, F, dtype = 1024, 2048, 2048, torch.bfloat16
    x, dh = _randn(g, (1, T, D), dtype), _randn(g, (1, T, F), dtype)
    wg, wu = _randn(g, (1, F, D), dtype, D ** -0.5), _randn(g, (1, F, D), dtype, D ** -0.5)

    def cost(x, wg):
        _, pre = lib.gated_forward(x, wg, wu, "relu", save=True)
        return _microseconds(lambda: lib.gated_backward(dh, x, wg, wu, pre, "relu"))

    some = lambda t: torch.rand(t.shape, generator=g, device="cuda") < 0.5   # noqa: E731
    zero_w, zero_x = wg.clone(), x.clone()
    zero_w[0, ::2] = 0
    zero_x[0, ::2] = 0
    random = cost(x, wg)
    times = {"zero features": cost(x, zero_w), "zero tokens": cost(zero_x, wg),
             "integers": cost(torch.sign(x) * some(x), torch.sign(wg) * some(wg))}
    assert all(t <= 1.5 * random + 5 for t in times.values()), (random, times)


# ------------------------------------------------------------------- the range of fp16

def _activation_64(kind, a):
    if kind == "sigmoid":
        return torch.sigmoid(a), torch.sigmoid(a) * torch.sigmoid(-a)
    if kind == "relu":
        return a.clamp(min=0.0), (a > 0).double()
    return a * torch.sigmoid(a), torch.sigmoid(a) * (1 + a * torch.sigmoid(-a))


def _check_fp16_gradients(x, wg, wu, dh, kind):
    X, G, Up, E = x.double(), wg.double(), wu.double(), dh.double()
    T, D, F = X.shape[1], X.shape[2], G.shape[1]
    half = 2.0 ** -11
    a, b = X @ G.mT, X @ Up.mT
    f, df = _activation_64(kind, a)
    ea, eb = _product_error(D) * (X.abs() @ G.abs().mT), _product_error(D) * (X.abs() @ Up.abs().mT)
    da, db = E * b * df, E * f
    # act' <= 1.1, act'' <= 0.5; the device's exponential and division: 8 steps
    edf = (a.abs() < ea).double() if kind == "relu" else 0.5 * ea + 16 * U * (1 + a.abs())
    most = torch.maximum(da.abs().amax(dim=(1, 2)), db.abs().amax(dim=(1, 2)))[:, None, None]
    # unscaled, the least step is 2^-24; scaled, the largest is 2^14 or more, so that it is 2^-38 of that (half of it is lost at most)
    step = torch.where((most >= 2.0 ** -4) & (most < 2.0 ** 15), torch.full_like(most, 2.0 ** -25), most * 2.0 ** -39) * 1.01
    eda = E.abs() * (b.abs() * edf + df * eb + edf * eb) + (half + 4 * U) * da.abs() + step
    edb = E.abs() * (1.1 * ea + 8 * U * (f.abs() + a.abs())) + (half + 4 * U) * db.abs() + step
    _, pre = lib.gated_forward(x, wg, wu, kind, save=True)
    got = lib.gated_backward(dh, x, wg, wu, pre, kind)
    sums = ((da @ G + db @ Up, eda @ G.abs() + edb @ Up.abs(), da.abs() @ G.abs() + db.abs() @ Up.abs(), 2 * F),
            (da.mT @ X, eda.mT @ X.abs(), da.abs().mT @ X.abs(), T), (db.mT @ X, edb.mT @ X.abs(), db.abs().mT @ X.abs(), T))
    for g, (want, err, size, K) in zip(got, sums):
        tol = err * 1.01 + _product_error(K) * (size + err) + half * want.abs() * 1.01 + 2.0 ** -25
        there = want.abs() + tol < 65504   # what the result's own type holds
        assert bool((((g.double() - want).abs() <= tol) | ~there).all()) and float(there.double().mean()) > 0.7
    return most.flatten().tolist(), got


@pytest.mark.parametrize("kind", ["silu", "relu", "sigmoid"])
@pytest.mark.parametrize("T,D,F", [(40, 333, 203), (300, 128, 1024), (4096, 64, 64), (130, 2048, 72), (2, 64, 40), (600, 1024, 520)])
def test_fp16_gradients_whose_intermediates_leave_the_type_s_range(T, D, F, kind):
    """Workers whose da and db lie below fp16's normal range, in it, and above it: each is scaled by itself."""
    g = _gen(T + D + F)
    m, dtype = 4, torch.float16
    x, wg, wu, dh = _randn(g, (m, T, D)), _randn(g, (m, F, D), std=D ** -0.5), _randn(g, (m, F, D), std=D ** -0.5), _randn(g, (m, T, F))
    dh[0] *= 2.0 ** -19          # a few of fp16's least steps ...
    wu[0] *= 2.0 ** -6           # ... times a small factor
    wg[0] *= 2.0 ** -6
    x[1], wu[1], wg[1], dh[1] = x[1] * 2.0 ** -9, wu[1] * 2.0 ** 15, wg[1] * 2.0 ** -8, dh[1] * 2.0 ** 12   # above: 2^18
    if kind == "sigmoid":
        wu[1] *= 2.0 ** -8       # (db wu is no larger than da wg)
        x[1] *= 2.0 ** 2
    dh[3] = 0.0
    x, wg, wu, dh = (t.to(dtype) for t in (x, wg, wu, dh))
    most, got = _check_fp16_gradients(x, wg, wu, dh, kind)
    assert most[0] < 2.0 ** -14 and most[3] == 0.0
    if kind != "sigmoid":
        assert most[1] > 65504
    assert all(not bool(t[3].any()) for t in got) and bool(got[1][0].any()) and bool(got[2][0].any())
    # a worker's bits do not depend on the others (the same launches, with every other worker an ordinary one)
    for i in (0, 2):
        rest = [torch.stack([t[i if j == i else 2] for j in range(m)]) for t in (x, wg, wu, dh)]
        _, pre = lib.gated_forward(*rest[:3], kind, save=True)
        for u, v in zip(lib.gated_backward(rest[3], *rest[:3], pre, kind), got):
            assert torch.equal(u[i], v[i])


def test_fp16_weight_gradients_of_many_tokens_of_small_gradients():
    """d_h of 2^-22 times a factor of 2^-8: nothing in fp16, 2^-18 in a sum over 4096 tokens."""
    dtype, (T, D, F) = torch.float16, (4096, 64, 64)
    x, wg = torch.ones((1, T, D), dtype=dtype, device="cuda"), torch.zeros((1, F, D), dtype=dtype, device="cuda")
    wu, dh = torch.full((1, F, D), 2.0 ** -12, dtype=dtype, device="cuda"), torch.full((1, T, F), 2.0 ** -22, dtype=dtype, device="cuda")
    _, pre = lib.gated_forward(x, wg, wu, "sigmoid", save=True)
    dx, dwg, dwu = lib.gated_backward(dh, x, wg, wu, pre, "sigmoid")   # act(0) = 1/2, act'(0) = 1/4, b = 2^-6
    assert bool((dwg == 2.0 ** (12 - 22 - 6 - 2)).all()) and bool((dwu == 2.0 ** (12 - 22 - 1)).all())


def test_fp16_gradients_with_infinities_keep_to_their_rows():
    """A token of infinities does not decide the others' factor."""
    g = _gen(9)
    dtype = torch.float16
    x, wg, wu = _randn(g, (1, 40, 64), dtype), _randn(g, (1, 48, 64), dtype, 0.125), _randn(g, (1, 48, 64), dtype, 0.125)
    for std in (1.0, 2.0 ** -19):
        dh = _randn(g, (1, 40, 48), dtype, std)
        bad = dh.clone()
        bad[0, 5], bad[0, 9, 3] = math.inf, math.nan
        for kind in ("silu", "relu"):
            _, pre = lib.gated_forward(x, wg, wu, kind, save=True)
            want = lib.gated_backward(dh, x, wg, wu, pre, kind)[0]
            got = lib.gated_backward(bad, x, wg, wu, pre, kind)[0]
            keep = [i for i in range(40) if i not in (5, 9)]
            assert torch.allclose(got[0, keep].float(), want[0, keep].float(), rtol=2.0 ** -9, atol=2.0 ** -23)
            assert bool(torch.isnan(got[0, 9]).all()) and not bool(torch.isfinite(got[0, 5]).any())


@pytest.mark.parametrize("m,T,D,F", [(3, 65, 64, 96), (2, 40, 333, 203), (700, 3, 16, 24), (1, 200, 304, 2048)])
@pytest.mark.parametrize("kind", ["silu", "relu"])
def test_captured_fp16_gradients_follow_the_inputs_factor(kind, m, T, D, F):
    """A graph is replayed with gradients of other magnitudes, each with another factor: the bits of eager calls, in plain stream
    order too."""
    g = _gen(m + T + D)
    dtype = torch.float16
    x, wg, wu = _randn(g, (m, T, D), dtype), _randn(g, (m, F, D), dtype, D ** -0.5), _randn(g, (m, F, D), dtype, D ** -0.5)
    dhs = [_randn(g, (m, T, F), dtype, std) for std in (1.0, 2.0 ** -18, 2.0 ** 13, 2.0 ** -12)]
    _, pre = lib.gated_forward(x, wg, wu, kind, save=True)
    before = lib.set_launch_overlap(False)
    try:
        want = [lib.gated_backward(dh, x, wg, wu, pre, kind) for dh in dhs]
        torch.cuda.synchronize()
    finally:
        lib.set_launch_overlap(before)
    dh, stream, graph = dhs[0].clone(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        got = lib.gated_backward(dh, x, wg, wu, pre, kind)
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(10):
        for other, w in zip(dhs, want):
            dh.copy_(other)
            graph.replay()
            eager = lib.gated_backward(other, x, wg, wu, pre, kind)
            for u, v, e in zip(got, w, eager):
                bad += (u != v).sum() + (e != v).sum()
    assert int(bad) == 0 and all(bool(torch.isfinite(t).all()) for t in want[1])
    lib.operators_join()


# ---------------------------------------------------------------------- saturated gates

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens", [1, 3])
def test_sigmoid_gradient_of_saturated_gates(tokens, dtype):
    """act'(a) = e^-|a| / (1 + e^-|a|)^2 keeps its digits on both sides: relative to itself, not to 1."""
    a = torch.cat([torch.arange(-20, 21, device="cuda") * 0.75, torch.tensor([16.0, 17.0], device="cuda")]).to(dtype)
    F = len(a)
    x, wg, wu = torch.zeros((1, tokens, 8), dtype=dtype, device="cuda"), torch.zeros((1, F, 8), dtype=dtype, device="cuda"), torch.zeros((1, F, 8), dtype=dtype, device="cuda")
    x[0, -1, 0], wg[0, :, 0], wu[0, :, 0] = 1.0, a, 1.0
    dh = torch.full((1, tokens, F), 2.0 ** 12, dtype=dtype, device="cuda")
    _, pre = lib.gated_forward(x, wg, wu, "sigmoid", save=True)
    _, dwg, dwu = lib.gated_backward(dh, x, wg, wu, pre, "sigmoid")
    d = a.double()
    want_g, want_u = 2.0 ** 12 * torch.sigmoid(d) * torch.sigmoid(-d), 2.0 ** 12 * torch.sigmoid(d)
    # rounded to the type twice; the exponent |a| log2 e < 32 is rounded twice (32 u ln 2 each), the power of two and the quotient
    # have 2 steps each, three products one
    tol = torch.finfo(dtype).eps * 1.01 + 60 * U
    assert bool(((dwg[0, :, 0].double() - want_g).abs() <= want_g * tol + 2.0 ** -25).all())
    assert bool(((dwu[0, :, 0].double() - want_u).abs() <= want_u * tol + 2.0 ** -25).all())


# --------------------------------------------------------------- clipping in the local step

def test_a_refused_local_step_leaves_the_gradient_as_it_was():
    g = _gen(5)
    m, P = 3, 1003
    grad = _randn(g, (m, P))
    want = grad.double().norm(dim=1)
    opt = OverlapLocalSGD("flat", flat_P=P, m=m, tau=1, gamma=0.1, alpha=0.5, x0=torch.zeros(P, device="cuda"))
    h = grad.clone()
    opt.local_step_with_grads(h)              # the period ends
    params = opt.get_params(0).copy()
    with pytest.raises(lib.OlsgdError, match="period"):
        opt.local_step_with_grads(h, max_norm=0.5)
    for norm in (0.0, math.nan):
        with pytest.raises(lib.OlsgdError):
            opt.local_step_with_grads(h, max_norm=norm)
    torch.cuda.synchronize()
    assert torch.equal(h, grad) and (opt.get_params(0) == params).all()
    opt.period_sync()
    norms = opt.local_step_with_grads(h, max_norm=0.5)
    torch.cuda.synchronize()
    assert bool(((norms.double() - want).abs() <= 4 * U * want).all())   # of the gradient itself, not of a clipped one
    assert bool((h.double().norm(dim=1) <= 0.5 * (1 + 1e-5)).all())
    opt.close()
    # a context that takes no gradients
    X, y = torch.zeros((2, 8, 4), device="cuda"), torch.zeros((2, 8), device="cuda")
    opt = OverlapLocalSGD("linreg", dims=(4,), m=2, batch=2, tau=4, gamma=0.1, alpha=0.5, X=X, y=y, x0=torch.zeros(4, device="cuda"))
    h = _randn(g, (2, opt.P))
    keep = h.clone()
    with pytest.raises(lib.OlsgdError, match="FLAT"):
        opt.local_step_with_grads(h, max_norm=0.1)
    torch.cuda.synchronize()
    assert torch.equal(h, keep)
    opt.close()


def test_norms_are_ready_on_the_caller_s_stream():
    """The context works on its own stream, which is busy; the norms are read on another one at once."""
    g = _gen(6)
    m, P = 3, 1003
    grad = _randn(g, (m, P))
    want = lib.clip_grads(grad, 1.0)[1]
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(main):
        opt = OverlapLocalSGD("flat", flat_P=P, m=m, tau=8, gamma=0.1, alpha=0.5, x0=torch.zeros(P, device="cuda"))
        busy = torch.eye(4096, device="cuda")
        opt.local_step_with_grads(grad.clone(), max_norm=1.0)   # (everything is loaded by now)
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(main):
            h = grad.clone()
            torch.full((m,), math.nan, device="cuda")           # what the norms' memory holds
            for _ in range(20):
                busy = busy @ busy
        with torch.cuda.stream(side):
            norms = opt.local_step_with_grads(h, max_norm=1.0)
            got = norms * 1.0
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    opt.close()


# ------------------------------------------------------------------- torch's own bookkeeping

def test_tensors_that_require_gradients():
    """Refused while torch records, taken under no_grad; also where only a later one of a list does."""
    g = _gen(7)
    x, t = _randn(g, (4, 50)), torch.zeros(4, dtype=torch.int32, device="cuda")
    want = lib.token_logprobs(x, t)
    leaf = x.clone().requires_grad_()
    for bad in (lambda: lib.token_logprobs(leaf, t), lambda: lib.token_logprobs(leaf * 2, t), lambda: lib.clip_grads([x, leaf], 1.0),
                lambda: lib.clip_grads([x], 1.0, out=[leaf])):
        with pytest.raises(ValueError, match="no graph"):
            bad()
    with torch.no_grad():
        assert torch.equal(lib.token_logprobs(leaf, t).logp, want.logp)
    assert torch.equal(lib.token_logprobs(leaf.detach(), t).logp, want.logp)


@pytest.mark.parametrize("N,V,top", [(4, 50, 0), (4, 50, 3), (8, 131072, 20), (3, 5000, 0)])
def test_log_probabilities_are_tensors_of_their_own(N, V, top):
    """Whoever keeps, saves or changes one of them keeps, saves or changes nothing else; autograd takes them like any tensors."""
    g = _gen(8)
    x, t = _randn(g, (N, V)), torch.zeros(N, dtype=torch.int32, device="cuda")
    want = [None if v is None else v.clone() for v in lib.token_logprobs(x, t, top)]
    r = lib.token_logprobs(x, t, top)
    tensors = [v for v in r if v is not None]
    assert all(v.untyped_storage().nbytes() == v.numel() * 4 for v in tensors)
    assert len({v.untyped_storage().data_ptr() for v in tensors}) == len(tensors)
    weights = torch.full((N,), 2.0, device="cuda", requires_grad=True)
    r.logp.mul_(weights)
    r.logp.sum().backward()
    assert torch.equal(weights.grad, want[0])
    assert all(torch.equal(a, b) and a._version == 0 and not a._is_view() for a, b in zip(tensors[1:], want[1:]))


# ------------------------------------------------------------------------- refusals

def test_clip_grads_refuses_to_scale_a_tensor_twice():
    a, b, none = torch.ones((2, 10), device="cuda"), torch.ones((2, 7), device="cuda"), torch.empty((2, 0), device="cuda")
    for grads, out in (([a, b, a], [a, b, a]), ([a, a], [b.new_empty((2, 10))] * 2)):
        with pytest.raises(ValueError, match="twice"):
            lib.clip_grads(grads, 1.0, out=out)
    torch.cuda.synchronize()
    assert bool((a == 1).all()) and bool((b == 1).all())
    # a gradient that counts twice may be read twice, and what is empty may be there as often as it likes
    _, norms = lib.clip_grads([a, none, a, none], 1.0, out=[torch.empty_like(a), none, torch.empty_like(a), none])
    assert bool(((norms.double() - math.sqrt(20)).abs() <= 4 * U * math.sqrt(20)).all())


def test_embedding_gradient_refuses_a_vocabulary_that_is_no_positive_integer():
    d, ids = torch.ones((1, 2, 4), device="cuda"), torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    for vocab in (0, -1):
        with pytest.raises(ValueError, match="vocab"):
            lib.embedding_backward(d, ids, vocab)
    with pytest.raises(TypeError):
        lib.embedding_backward(d, ids, 3.7)
    assert lib.embedding_backward(d, ids, torch.tensor(3)).shape == (1, 3, 4)
