"""Routing, products by expert, combination and distillation as they are used: a small sparse language model per worker, taught by
another model's top logits and trained through the flat-vector path; and on side streams, captured into graphs, from several threads,
with launches that do not overlap."""
import math
import os
import subprocess
import sys
import threading

import pytest
import torch

import paper_2002_09539_b200 as lib
from paper_2002_09539_b200 import OverlapLocalSGD

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class SparseLanguageModel:
    """Token embedding, a router, experts of two matrices around silu beside a residual, an output matrix; every worker's parameters are one
    flat row."""

    def __init__(self, m, V, D, F, E, k, normalise):
        self.m, self.V, self.D, self.F, self.E, self.k, self.normalise = m, V, D, F, E, k, normalise
        self.shapes = [(V, D), (E, D), (E, F, D), (E, D, F), (V, D)]
        self.P = sum(math.prod(s) for s in self.shapes)

    def views(self, flat):
        out, at = [], 0
        for s in self.shapes:
            n = math.prod(s)
            out.append(flat[:, at:at + n].unflatten(1, s))
            at += n
        return out

    def gradient(self, params, ids, teacher_ids, teacher, d_loss, flat, max_norm=None):
        """Writes the gradient of sum d_loss * loss, rows of `flat`; returns losses, routing, the weights' gradients."""
        scale = math.sqrt(self.D)
        table, Wr, W1, W2, Wo = (w.to(torch.bfloat16) for w in self.views(params))
        x = lib.embedding_forward(table, ids, scale)
        scores = x.float() @ Wr.float().mT
        r = lib.expert_route(scores, self.k, self.normalise)
        rows = lib.embedding_forward(x, r.tokens)
        h1 = lib.expert_product(rows, W1, r.offsets)
        a = (h1.float() * torch.sigmoid(h1.float())).bfloat16()
        h2 = lib.expert_product(a, W2, r.offsets)
        y = lib.expert_combine(h2, r.places, r.weights) + x
        loss = lib.distill_loss(torch.bmm(y, Wo.mT), teacher_ids, teacher, 2.0, d_loss=d_loss)
        d_Wo, dy = torch.bmm(loss.d_logits.mT, y), torch.bmm(loss.d_logits, Wo)
        d_h2, d_w = lib.expert_combine_backward(dy, h2, r.places, r.tokens, r.weights)
        d_a, d_W2 = lib.expert_product_backward(d_h2, a, W2, r.offsets)
        s = torch.sigmoid(h1.float())
        d_h1 = (d_a.float() * s * (1 + h1.float() * (1 - s))).bfloat16()
        d_rows, d_W1 = lib.expert_product_backward(d_h1, rows, W1, r.offsets)
        d_scores = lib.expert_route_backward(d_w, scores, r.ids, r.weights, self.normalise)
        d_Wr = d_scores.mT @ x.float()
        dx = (dy.float() + lib.expert_combine(d_rows, r.places).float() + d_scores @ Wr.float()).bfloat16()
        views = self.views(flat)
        lib.embedding_backward(dx, ids, self.V, scale, out=views[0])
        grads = [views[0], d_Wr, d_W1, d_W2, d_Wo]
        if max_norm is None:
            for v, g in zip(views[1:], grads[1:]):
                v.copy_(g)
        else:
            lib.clip_grads(grads, max_norm, out=views)
        return loss.loss, r, d_w

    def gradient_64(self, params, ids, teacher_ids, teacher, d_loss, chosen):
        """The same function on the same 16-bit parameters with the same choice of experts, in 64 bits, by autograd; and the size of the
        terms that the router's gradient is a difference of."""
        p = params.to(torch.bfloat16).double().requires_grad_()
        table, Wr, W1, W2, Wo = self.views(p)
        x = torch.stack([table[i][ids[i].clamp(min=0).long()] for i in range(self.m)]) * math.sqrt(self.D) * (ids >= 0)[..., None]
        scores = x @ Wr.mT
        at = chosen.long()
        w = torch.softmax(scores.gather(2, at), dim=2) if self.normalise else torch.softmax(scores, dim=2).gather(2, at)
        w.retain_grad()
        worker = torch.arange(self.m, device="cuda")[:, None, None]
        h1 = torch.einsum("mtd,mtkfd->mtkf", x, W1[worker, at])
        y = torch.einsum("mtk,mtkf,mtkdf->mtd", w, h1 * torch.sigmoid(h1), W2[worker, at]) + x
        lp = torch.log_softmax(y @ Wo.mT / 2.0, dim=-1)
        has = teacher_ids >= 0
        q = torch.softmax(torch.where(has, teacher.double() / 2.0, -1e300), dim=-1) * has
        loss = (torch.xlogy(q, q) - q * lp.gather(2, teacher_ids.clamp(min=0).long())).sum(dim=-1)
        (loss * d_loss.double()).sum().backward()
        terms = w.detach() * w.grad.abs()
        terms = torch.zeros_like(scores).scatter_add_(2, at, terms) + torch.softmax(scores.detach(), dim=2) * terms.sum(dim=2, keepdim=True)
        return loss.detach(), p.grad, (terms.mT @ x.detach().abs()).norm()


def _batch(g, m, T, V, K):
    ids = torch.randint(0, V, (m, T), generator=g, device="cuda", dtype=torch.int32)
    teacher_ids = ((torch.randint(0, V, (m, T, 1), generator=g, device="cuda") + 7 * torch.arange(K, device="cuda")) % V).to(torch.int32)
    if T > 2:
        ids[:, T // 2], teacher_ids[:, T // 2] = -1, -1   # a position of padding
    d_loss = torch.rand((m, T), generator=g, device="cuda") / T
    return ids, teacher_ids, torch.randn((m, T, K), generator=g, device="cuda") * 2, d_loss


@pytest.mark.parametrize("m,T,V,D,F,E,k", [(3, 50, 37, 16, 24, 5, 2), (2, 130, 1201, 40, 72, 8, 3), (1, 1, 130, 33, 7, 4, 1), (2, 300, 257, 64, 128, 16, 4)])
@pytest.mark.parametrize("normalise", [True, False])
def test_gradient_of_a_sparse_language_model(m, T, V, D, F, E, k, normalise):
    g = _gen(m + T + V)
    model = SparseLanguageModel(m, V, D, F, E, k, normalise)
    params = torch.randn((m, model.P), generator=g, device="cuda") * 0.15
    batch = _batch(g, m, T, V, min(6, V))
    flat = torch.full((m, model.P), math.nan, device="cuda")
    loss, r, _ = model.gradient(params, *batch, flat)
    want_loss, want, terms = model.gradient_64(params, *batch, r.ids)
    # Values are rounded to 8 bits (2^-9 of them each, at most) some fourteen times on the way (x, h1, a, h2, the combination, y, the logits and
    # their gradient, dy, d_h2, d_a, d_h1, d_rows, dx, the gradient itself): taken as if all had one sign, in norm.  The router's
    # gradient is a difference of terms, each as far off.
    for n, (a, b) in enumerate(zip(model.views(flat), model.views(want))):
        size = float(b.norm()) if n != 1 else float(terms)
        assert float((a.double() - b).norm()) <= 14 * 2.0 ** -8 * size, n
    assert bool(((loss.double() - want_loss).abs() <= 14 * 2.0 ** -8 * (1 + want_loss.abs())).all())
    clipped = torch.full((m, model.P), math.nan, device="cuda")
    model.gradient(params, *batch, clipped, max_norm=0.05)
    norm = flat.double().norm(dim=1)
    c = torch.clamp(0.05 / (norm + 1e-6), max=1.0)[:, None]
    assert bool(((clipped.double() - flat.double() * c).abs() <= 6 * 2.0 ** -24 * flat.double().abs() * c + 2.0 ** -140).all())


def test_training_a_sparse_language_model_through_the_flat_path():
    g = _gen(77)
    m, T, V, D, F, E, k, tau = 4, 48, 100, 32, 64, 6, 2, 2
    model = SparseLanguageModel(m, V, D, F, E, k, True)
    x0 = torch.randn(model.P, generator=g, device="cuda") * 0.15
    opt = OverlapLocalSGD("flat", flat_P=model.P, m=m, tau=tau, gamma=0.1, alpha=0.5, beta=0.5, x0=x0)
    params, flat = torch.empty((m, model.P), device="cuda"), torch.empty((m, model.P), device="cuda")
    for step in range(2 * tau):
        for i in range(m):
            opt.get_params(i, out=params[i])
        loss, r, _ = model.gradient(params, *_batch(g, m, T, V, 8), flat, max_norm=0.5)
        assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(flat).all())
        opt.local_step_with_grads(flat)
        if (step + 1) % tau == 0:
            opt.period_sync()
    assert opt.iteration == 2 * tau
    lib.operators_join()
    opt.close()


# ------------------------------------------------------------------- streams, graphs, launches

def _calls(seed=0, m=2, T=90, V=3000, D=96, F=80, E=7, k=2, K=9):
    """Inputs (to be overwritten in place) and one function over all operators that returns all their outputs."""
    def make(s):
        g = _gen(s)
        ids, teacher_ids, teacher, d_loss = _batch(g, m, T, V, K)
        scores = torch.randn((m, T, E), generator=g, device="cuda")
        scores[:, 5] = -math.inf
        return {"x": torch.randn((m, T, D), generator=g, device="cuda").bfloat16(), "scores": scores,
                "w": torch.randn((m, E, F, D), generator=g, device="cuda").bfloat16() * 0.1, "odd": torch.randn((m, E, F, D + 1), generator=g, device="cuda").bfloat16()[..., 1:],
                "dy": torch.randn((m, T, F), generator=g, device="cuda").bfloat16(), "logits": torch.randn((m, T, V), generator=g, device="cuda").bfloat16() * 2,
                "long": torch.randn((3, 50000), generator=g, device="cuda").bfloat16(), "teacher_ids": teacher_ids, "teacher": teacher, "d_loss": d_loss}

    def run(s):
        r = lib.expert_route(s["scores"], k, False)
        rows = lib.embedding_forward(s["x"], r.tokens)
        h, odd = lib.expert_product(rows, s["w"], r.offsets), lib.expert_product(rows, s["odd"], r.offsets)
        y = lib.expert_combine(h, r.places, r.weights)
        d_h, d_w = lib.expert_combine_backward(s["dy"], h, r.places, r.tokens, r.weights)
        d_rows, d_W = lib.expert_product_backward(d_h, rows, s["w"], r.offsets)
        odd_rows, odd_W = lib.expert_product_backward(d_h, rows, s["odd"], r.offsets)
        d_scores = lib.expert_route_backward(d_w, s["scores"], r.ids, r.weights, False)
        dx = lib.expert_combine(d_rows, r.places)
        one = lib.distill_loss(s["logits"], s["teacher_ids"], s["teacher"], 1.5, d_loss=s["d_loss"])
        two = lib.distill_loss(s["logits"], s["teacher_ids"], s["teacher"], 1.5)
        later = lib.distill_backward(s["d_loss"], s["logits"], s["teacher_ids"], s["teacher"], two.stats, 1.5)
        wide = lib.distill_loss(s["long"], s["teacher_ids"][0, :3], s["teacher"][0, :3], d_loss=s["d_loss"][0, :3])   # a cluster a row
        return [*r, rows, h, odd, y, d_h, d_w, d_rows, d_W, odd_rows, odd_W, d_scores, dx, *one, two.loss, two.stats, later, *wide]

    return make, run


def _same(a, b):
    return all(torch.equal(x.view(torch.uint8) if x.dtype.is_floating_point else x, y.view(torch.uint8) if y.dtype.is_floating_point else y)
               for x, y in zip(a, b))


def test_operators_on_side_streams_and_captured():
    make, run = _calls()
    a, b = make(1), make(2)
    want = [run(a), run(b)]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(s1):
            g1 = run(a)
        with torch.cuda.stream(s2):
            g2 = run(b)
    torch.cuda.synchronize()
    assert _same(g1, want[0]) and _same(g2, want[1])
    # one graph each, replayed at once on both streams, then with the inputs (and with them the groups' sizes) exchanged
    graphs = []
    for s, inputs in ((s1, a), (s2, b)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            with torch.cuda.graph(graph, stream=s):
                outputs = run(inputs)
        graphs.append((graph, s, outputs))
    for exchanged in (False, True):
        if exchanged:
            fresh = (make(2), make(1))
            for inputs, other in ((a, fresh[0]), (b, fresh[1])):
                for k in inputs:
                    inputs[k].copy_(other[k])
            torch.cuda.synchronize()
        for _ in range(3):
            for graph, s, _ in graphs:
                with torch.cuda.stream(s):
                    graph.replay()
        torch.cuda.synchronize()
        for (_, _, outputs), w in zip(graphs, want[::-1] if exchanged else want):
            assert _same(outputs, w)
    lib.operators_join()


def test_operators_give_the_same_bits_in_plain_stream_order_and_over_and_over():
    make, run = _calls()
    inputs = [make(s) for s in (3, 4, 5)]
    before = lib.set_launch_overlap(False)
    try:
        want = [run(a) for a in inputs]
        torch.cuda.synchronize()
    finally:
        lib.set_launch_overlap(before)
    for _ in range(20):
        for a, w in zip(inputs, want):
            assert _same(run(a), w)
    lib.operators_join()


def test_operators_on_the_legacy_stream_of_other_threads():
    make, run = _calls()
    a = make(4)
    want = run(a)
    got, errors = [None] * 4, []

    def work(i):
        try:
            for _ in range(5):
                got[i] = run(a)
        except Exception as e:   # reported below
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for g in got:
        assert _same(g, want)


def test_operators_captured_before_anything_else_ran():
    """The first call a process makes of every operator may be the one that is captured."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import sys, torch
sys.path[:0] = [%r, %r]
from test_gpu_experts_together import _calls, _same
make, run = _calls()
a = make(1)
s = torch.cuda.Stream()
s.wait_stream(torch.cuda.current_stream())
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=s):
    got = run(a)
graph.replay()
torch.cuda.synchronize()
assert _same(got, run(a))
print("captured first: ok")
""" % (root, os.path.join(root, "tests"))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured first: ok" in r.stdout, r.stderr[-2000:]


def test_operators_behind_events_of_other_streams():
    make, run = _calls()
    a = make(5)
    want = run(a)
    busy = torch.eye(4096, device="cuda")
    here, side = torch.cuda.Stream(), torch.cuda.Stream()
    here.wait_stream(torch.cuda.current_stream())

    def forked(busy):
        b = {k: torch.empty_strided(v.shape, v.stride(), dtype=v.dtype, device=v.device).zero_() for k, v in a.items()}
        for _ in range(4):   # what the side stream reads is written here, late
            busy = busy @ busy
        for k in b:
            b[k].copy_(a[k])
        side.wait_stream(here)
        with torch.cuda.stream(side):
            first = run(b)
        here.wait_stream(side)
        return first, run(b), b, busy

    with torch.cuda.stream(here):
        kept = [forked(busy) for _ in range(3)]
    torch.cuda.synchronize()
    for first, second, _, _ in kept:
        assert _same(first, want) and _same(second, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=here):
        first, second, _, _ = forked(busy)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert _same(first, want) and _same(second, want)
    lib.operators_join()


@pytest.mark.parametrize("m,R,E,D,F", [(16, 128, 3, 256, 256), (1, 512, 4, 512, 1024), (2, 65, 9, 1000, 72), (1, 3, 2, 64, 40), (1, 4000, 2, 64, 64), (3, 300, 5, 333, 201)])
def test_product_gradients_side_by_side_keep_the_stream_s_order(m, R, E, D, F):
    """The two products of the backward call overlap, the second also with copies and calls before it: what follows them at once (a torch
    kernel, the next call in the same memory) sees both done, eager and captured."""
    g = _gen(m + R)
    x, w = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, R, D), (m, E, F, D)))
    dys = [torch.randn((m, R, F), generator=g, device="cuda").bfloat16() for _ in range(3)]
    cuts = torch.sort(torch.randint(0, R + 1, (3, m, E + 1), generator=g, device="cuda"), dim=2).values.to(torch.int32)

    def once(i):
        dx, dw = lib.expert_product_backward(dys[i] * 2, x * 2, w * 0.5, cuts[i].clone())
        return dx + 1, dw + 1   # the gradients themselves, the operands and the offsets go back to the allocator at once

    before = lib.set_launch_overlap(False)
    try:
        want = [once(i) for i in range(3)]
        torch.cuda.synchronize()
    finally:
        lib.set_launch_overlap(before)
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(60):
        for i in range(3):
            for a, b in zip(once(i), want[i]):
                bad += (a != b).sum()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        got = [once(i) for i in range(3)]
    for _ in range(20):
        graph.replay()
        for a, b in zip(got, want):
            for u, v in zip(a, b):
                bad += (u != v).sum()
    assert int(bad) == 0
    lib.operators_join()
