"""Operators of sparse language models where one row or element more or less has to show: exact sums in parts of K, tensors of more than
2^31 elements, and the local step that takes their gradients, against the paper's update."""
import math

import numpy as np
import pytest
import torch

import paper_2002_09539_b200 as lib
from oracle.olsgd import OverlapLocalSGD as Oracle
from paper_2002_09539_b200 import OverlapLocalSGD
from test_gpu_experts_together import SparseLanguageModel, _batch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _whole(g, shape, dtype):
    return torch.randint(-3, 4, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


# few tiles and long sums, whose parts end anywhere; a long group beside short and empty ones; sums of one block
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,sizes,behind,D,F", [
    (1, [[5, 0, 3]], 4, 4096, 136), (1, [[3000, 0]], 2, 72, 40), (2, [[2000], [7]], 1, 77, 45), (1, [[9000, 70, 0, 1]], 10, 128, 256), (1, [[1, 0]], 0, 8192, 4096),
    (1, [[300]], 50, 4095, 1030), (3, [[2, 700], [1, 1], [0, 0]], 9, 130, 2050), (1, [[40000]], 0, 32, 32), (1, [[39967, 33]], 0, 64, 128), (1, [[64, 65, 127, 1]], 3, 8200, 64),
    (1, [[1]], 0, 64, 64), (1, [[31, 33, 20000]], 0, 512, 512)])
def test_products_of_whole_numbers_are_exact(m, sizes, behind, D, F, dtype):
    """Whole numbers up to 3: a sum of products is exact in fp32 (at most 40000 * 9), so that each result is the one rounding of the right
    sum, bit for bit, and a row or column left out or taken twice is none.  (fp16: results past its range are infinite on both sides.)"""
    g = _gen(D + F)
    R, E = max(sum(n) for n in sizes) + behind, len(sizes[0])
    lead = min(behind, 1)
    offsets = torch.tensor([[lead + sum(n[:e]) for e in range(E + 1)] for n in sizes], dtype=torch.int32, device="cuda")
    x, w, dy = _whole(g, (m, R, D), dtype), _whole(g, (m, E, F, D), dtype), _whole(g, (m, R, F), dtype)
    y, (dx, dw) = lib.expert_product(x, w, offsets), lib.expert_product_backward(dy, x, w, offsets)
    ends = offsets.tolist()
    for i in range(m):
        for e in range(E):
            part = slice(ends[i][e], ends[i][e + 1])
            X, W, G = x[i, part].double(), w[i, e].double(), dy[i, part].double()
            assert torch.equal(y[i, part], (X @ W.T).to(dtype)) and torch.equal(dx[i, part], (G @ W).to(dtype)) and torch.equal(dw[i, e], (G.T @ X).to(dtype)), (i, e)
    lib.operators_join()


# ------------------------------------------------------------------------ more than 2^31 elements

def test_route_of_more_than_two_to_the_31_logits():
    m, T, E, k = 2, 1_100_000, 1000, 2   # the second worker's last logits lie past 2^31
    g = _gen(1)
    x = torch.empty((m, T, E), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 31
    for i in range(0, T, 100_000):
        x[:, i:i + 100_000] = torch.randn((m, 100_000, E), generator=g, device="cuda", dtype=torch.bfloat16)
    r = lib.expert_route(x, k, False)
    dw = torch.ones_like(r.weights)
    dw[..., 1] = -1.0
    d = lib.expert_route_backward(dw, x, r.ids, r.weights, False)
    for part in (slice(0, 500), slice(T - 500, T)):
        v, at = torch.sort(x[:, part].double(), dim=2, descending=True, stable=True)
        p = torch.softmax(x[:, part].double(), dim=2)
        assert torch.equal(r.ids[:, part].long(), at[..., :k])
        # as in the tests of small ones: differences of at most 12, two exponentials, a chain of E / 32 + 6
        rel = (2 * 12 + E / 32 + 18) * U
        w = p.gather(2, at[..., :k])
        assert bool(((r.weights[:, part].double() - w).abs() <= w * rel).all())
        G = torch.zeros_like(p).scatter_(2, at[..., :k], dw[:, part].double())
        want = p * (G - (p * G).sum(dim=2, keepdim=True))
        tol = p * 2 * (2 * rel + (k + 8) * U) + want.abs() * 2.0 ** -8 + 2.0 ** -130
        assert bool(((d[:, part].double() - want).abs() <= tol).all())
    # rows by expert, tokens rising within one
    assert bool((r.offsets[:, -1] == T * k).all())
    for i in range(m):
        chosen = r.ids[i].flatten().long()
        order = torch.sort(chosen, stable=True).indices
        assert torch.equal(r.tokens[i].long(), order // k)
        assert torch.equal(r.places[i].flatten()[order].long(), torch.arange(T * k, device="cuda"))


@pytest.mark.parametrize("D", [4096, 4095])
def test_combination_of_more_than_two_to_the_31_elements(D):
    T, k, g = 300_000, 2, _gen(2)
    R = T * k
    rows = torch.empty((1, R, D), dtype=torch.bfloat16, device="cuda")
    assert rows.numel() > 2 ** 31
    for i in range(0, R, 50_000):
        rows[:, i:i + 50_000] = torch.randn((1, 50_000, D), generator=g, device="cuda", dtype=torch.bfloat16)
    dy = torch.randn((1, T, D), generator=g, device="cuda", dtype=torch.bfloat16)
    order = torch.randperm(R, generator=g, device="cuda")
    places = torch.empty(R, dtype=torch.int32, device="cuda")
    places[order] = torch.arange(R, dtype=torch.int32, device="cuda")
    tokens, places = (order // k).to(torch.int32)[None], places.view(1, T, k)
    weights = torch.rand((1, T, k), generator=g, device="cuda")
    y = lib.expert_combine(rows, places, weights)
    d_rows, d_w = lib.expert_combine_backward(dy, rows, places, tokens, weights)
    last = torch.arange(R - 1000, R, device="cuda")           # rows past 2^31
    t = torch.cat([order[last] // k, torch.arange(T - 500, T, device="cuda")])
    picked = rows[0][places[0, t].long()].double()            # [.., k, D]
    W, E = weights[0, t].double(), dy[0, t].double()
    want, size = (W[..., None] * picked).sum(dim=1), (W[..., None] * picked.abs()).sum(dim=1)
    assert bool(((y[0, t].double() - want).abs() <= size * (k + 1) * U + want.abs() * 2.0 ** -8 + 2.0 ** -130).all())
    want, size = (E[:, None] * picked).sum(dim=2), (E[:, None] * picked).abs().sum(dim=2)
    assert bool(((d_w[0, t].double() - want).abs() <= size * (D / 32 + 24) * U).all())
    slot = order[last]
    want = weights[0].flatten()[slot].double()[:, None] * dy[0, slot // k].double()
    assert bool(((d_rows[0, last].double() - want).abs() <= want.abs() * (2.0 ** -8 + U) + 2.0 ** -130).all())


def test_products_of_more_than_two_to_the_31_elements():
    """Rows, results and weights each; whole numbers, so that the bits are known."""
    g = _gen(3)
    for m, R, E, D, F in ((1, 540_000, 2, 4096, 64), (1, 540_000, 2, 64, 4096), (4, 128, 65, 4096, 2048)):
        x, dy = _whole(g, (m, R, D), torch.bfloat16), _whole(g, (m, R, F), torch.bfloat16)
        w = _whole(g, (m, E, F, D), torch.bfloat16)
        assert max(x.numel(), dy.numel(), w.numel()) > 2 ** 31
        cuts = torch.sort(torch.randint(0, R + 1, (m, E + 1), generator=g, device="cuda"), dim=1).values.to(torch.int32)
        cuts[:, -1], cuts[:, 0] = R, 0
        y, (dx, dw) = lib.expert_product(x, w, cuts), lib.expert_product_backward(dy, x, w, cuts)
        i, a = m - 1, int(cuts[m - 1, E - 1])
        part = slice(max(a, R - 3000), R)   # the last group's last rows
        X, W, G = x[i, part].double(), w[i, E - 1].double(), dy[i, part].double()
        assert torch.equal(y[i, part], (X @ W.T).to(y.dtype)) and torch.equal(dx[i, part], (G @ W).to(y.dtype))
        total = torch.zeros((F, D), dtype=torch.float64, device="cuda")
        for b in range(a, R, 20_000):
            part = slice(b, min(R, b + 20_000))
            total += dy[i, part].double().T @ x[i, part].double()
        assert torch.equal(dw[i, E - 1], total.to(y.dtype))   # (540000 * 9 < 2^24)
        del x, dy, w, y, dx, dw, X, W, G


def test_distillation_of_more_than_two_to_the_31_logits():
    g = _gen(4)
    for N, V in ((600_000, 4001), (40_000, 60_000), (2_200_000, 1000)):
        x = torch.empty((N, V), dtype=torch.bfloat16, device="cuda")
        assert x.numel() > 2 ** 31
        for i in range(0, N, N // 20):
            x[i:i + N // 20] = torch.randn((N // 20, V), generator=g, device="cuda", dtype=torch.bfloat16)
        ids = torch.randint(0, V, (N, 1), generator=g, device="cuda", dtype=torch.int32)
        z, w = torch.zeros((N, 1), device="cuda"), torch.rand(N, generator=g, device="cuda")
        plain, both = lib.distill_loss(x, ids, z), lib.distill_loss(x, ids, z, d_loss=w)
        later = lib.distill_backward(w, x, ids, z, plain.stats)
        for part in (slice(0, 200), slice(N - 200, N)):
            lp = torch.log_softmax(x[part].double(), dim=1)
            at, p = ids[part].long(), lp.exp()
            loss = -lp.gather(1, at)[:, 0]
            # logits of at most 7 by size: exponents of at most 14 with three roundings, a chain of V / 32 + 64
            rel = (V / 32 + 64 + 42 + 4) * U
            for got in (plain, both):
                assert bool(((got.loss[part].double() - loss).abs() <= rel + 8 * U * loss).all())
            want = w[part].double()[:, None] * p.scatter_add(1, at, torch.full_like(p[:, :1], -1.0))
            for d in (both.d_logits, later):
                tol = w[part].double()[:, None] * p * (2 * rel + 50 * U) + want.abs() * (2.0 ** -8 + 8 * U) + 2.0 ** -130
                assert bool(((d[part].double() - want).abs() <= tol).all())
        del x, plain, both, later


# ------------------------------------------------------------------------------- the local step

def test_each_step_with_a_sparse_model_s_gradient_is_the_paper_s_update():
    """The oracle takes the same gradients: parameters after every local step, and after every synchronisation with the anchor."""
    g = _gen(78)
    m, T, V, D, F, E, k, tau, mu = 3, 40, 90, 24, 40, 5, 2, 2, 0.9
    model = SparseLanguageModel(m, V, D, F, E, k, True)
    x0 = torch.randn(model.P, generator=g, device="cuda") * 0.15
    kw = dict(m=m, tau=tau, gamma=0.1, alpha=0.5, beta=0.5, mu=mu)
    opt, want = OverlapLocalSGD("flat", flat_P=model.P, x0=x0, **kw), Oracle(x0.cpu().numpy(), **kw)
    params, flat = torch.empty((m, model.P), device="cuda"), torch.empty((m, model.P), device="cuda")
    moved = np.zeros(m)
    for step in range(3 * tau):
        for i in range(m):
            opt.get_params(i, out=params[i])
        model.gradient(params, *_batch(g, m, T, V, 8), flat, max_norm=0.5)
        opt.local_step_with_grads(flat)
        if (step + 1) % tau == 0:
            opt.period_sync()
        want.step(flat.cpu().numpy())
        size = max(np.abs(want.x).max(), np.abs(want.u).max(), np.abs(want.z).max())
        # a step rounds five times and a synchronisation m + 5 times, each by U of values of at most `size` (u, which gamma makes smaller,
        # and differences of two such values, among them); what was off before stays off by as much, or less
        tol = (step + 1) * (2 * m + 12) * U * size
        for i in range(m):
            got = opt.get_params(i)
            assert np.abs(got - want.x[i]).max() <= tol
            moved[i] = np.abs(got - params[i].cpu().numpy()).max()
        assert moved.min() > 50 * tol          # (a step that did nothing would show)
        if (step + 1) % tau == 0:
            assert np.abs(opt.get_params(-1) - want.z).max() <= tol
    # the workers' gradients differ, and so do their parameters
    assert min(np.abs(want.x[0] - want.x[i]).max() for i in range(1, m)) > 50 * tol
    lib.operators_join()
    opt.close()
