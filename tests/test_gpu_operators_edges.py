"""The operators on caller-owned tensors at the edges of what their documentation allows: values next to a border, at the
ends of a type's range, and data whose cost must not depend on its values.

Tolerances count roundings, as in test_gpu_operators.py."""
import pytest
import torch

import paper_2002_09539_b200 as lib

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


@pytest.mark.parametrize("data,dtype", [(d, t) for d in ("zero features", "zero tokens", "integers", "one element", "large", "small")
                                        for t in (torch.bfloat16, torch.float16) if (d, t) != ("large", torch.float16)])
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
    eda, edb = E.abs() * eb + da.abs() * (half + 4 * U) + 2.0 ** -24, E.abs() * ea + db.abs() * (half + 4 * U) + 2.0 ** -24
    if dtype == torch.bfloat16:
        eda, edb = eda - 2.0 ** -24, edb - 2.0 ** -24
    wants = ((dx, da @ wg.double() + db @ wu.double(), eda @ wg.double().abs() + edb @ wu.double().abs(), da.abs() @ wg.double().abs() + db.abs() @ wu.double().abs(), 2 * F),
             (dwg, da.mT @ x.double(), eda.mT @ x.double().abs(), da.abs().mT @ x.double().abs(), T))
    for got, want, err, size, K in wants:
        tol = err * 1.01 + _product_error(K) * (size + err) + want.abs() * half * 1.01 + (2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126)
        finite = want.abs() < torch.finfo(dtype).max
        assert bool((((got.double() - want).abs() <= tol) | ~finite).all())


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
