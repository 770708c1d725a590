"""The operators on caller-owned tensors as they are used: a small language model per worker, trained through the flat-vector
path; and on side streams, captured into graphs, with launches that do not overlap."""
import math

import pytest
import torch

import paper_2002_09539_b200 as lib
from paper_2002_09539_b200 import OverlapLocalSGD

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class FlatLanguageModel:
    """Token embedding, a gated block and an output matrix; every worker's parameters are one flat row."""

    def __init__(self, m, V, D, F, act="silu"):
        self.m, self.V, self.D, self.F, self.act = m, V, D, F, act
        self.shapes = [(V, D), (F, D), (F, D), (V, F)]
        self.P = sum(a * b for a, b in self.shapes)

    def views(self, flat):
        out, at = [], 0
        for a, b in self.shapes:
            out.append(flat[:, at:at + a * b].unflatten(1, (a, b)))
            at += a * b
        return out

    def gradient(self, params, ids, targets, flat, max_norm=None):
        """Writes the gradient of the mean negative log probability, rows of `flat`, clipped when asked to."""
        E, Wg, Wu, Wo = (w.to(torch.bfloat16) for w in self.views(params))
        x = lib.embedding_forward(E, ids, math.sqrt(self.D))
        h, pre = lib.gated_forward(x, Wg, Wu, self.act, save=True)
        logits = torch.bmm(h, Wo.mT)
        r = lib.token_logprobs(logits, targets)
        has = (targets >= 0).float()
        d_logp = -has / has.sum(dim=1, keepdim=True).clamp(min=1)
        d_logits = lib.token_logprobs_backward(d_logp, None, logits, targets, r.stats, r.entropy)
        d_Wo = torch.bmm(d_logits.mT, h)
        dx, d_Wg, d_Wu = lib.gated_backward(torch.bmm(d_logits, Wo), x, Wg, Wu, pre, self.act)
        views = self.views(flat)
        lib.embedding_backward(dx, ids, self.V, math.sqrt(self.D), out=views[0])
        grads = [views[0], d_Wg, d_Wu, d_Wo]
        if max_norm is None:
            for v, g in zip(views[1:], grads[1:]):
                v.copy_(g)
            return (-r.logp * -d_logp).sum(dim=1), None
        _, norms = lib.clip_grads(grads, max_norm, out=views)
        return (-r.logp * -d_logp).sum(dim=1), norms

    def gradient_64(self, params, ids, targets):
        """The same function on the same 16-bit parameters, in 64 bits, by autograd."""
        p = params.to(torch.bfloat16).double().requires_grad_()
        E, Wg, Wu, Wo = self.views(p)
        x = torch.stack([E[i][ids[i].clamp(min=0).long()] for i in range(self.m)]) * math.sqrt(self.D)
        x = x * (ids >= 0)[..., None]
        a = x @ Wg.mT
        f = a * torch.sigmoid(a) if self.act == "silu" else torch.relu(a)
        lp = torch.log_softmax((f * (x @ Wu.mT)) @ Wo.mT, dim=-1)
        has = (targets >= 0).double()
        picked = lp.gather(-1, targets.clamp(min=0).long()[..., None])[..., 0] * has
        loss = -(picked.sum(dim=1) / has.sum(dim=1).clamp(min=1))
        loss.sum().backward()
        return loss.detach(), p.grad


def _batch(g, m, T, V):
    ids = torch.randint(0, V, (m, T), generator=g, device="cuda", dtype=torch.int32)
    targets = torch.roll(ids, -1, dims=1)
    targets[:, -1] = -1
    ids[:, T // 2], targets[:, T // 2] = -1, -1   # a position of padding
    return ids, targets.contiguous()


@pytest.mark.parametrize("m,T,V,D,F", [(3, 50, 37, 16, 24), (2, 65, 1200, 40, 72), (1, 1, 130, 33, 7)])
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_gradient_of_a_language_model(m, T, V, D, F, act):
    g = _gen(m + T + V)
    model = FlatLanguageModel(m, V, D, F, act)
    params = torch.randn((m, model.P), generator=g, device="cuda") * 0.15
    ids, targets = _batch(g, m, T, V) if T > 1 else (torch.full((m, 1), 5, dtype=torch.int32, device="cuda"),
                                                     torch.full((m, 1), 9, dtype=torch.int32, device="cuda"))
    flat = torch.full((m, model.P), math.nan, device="cuda")
    loss, _ = model.gradient(params, ids, targets, flat)
    want_loss, want = model.gradient_64(params, ids, targets)
    # Values are rounded to 8 bits (2^-9 of them each, at most) eight times on the way (x, h, logits, d_logits, dh, da and db, dx, the
    # gradient), and every matrix product adds up such errors with both signs: taken as if they all had one sign, in norm.
    for a, b in zip(model.views(flat), model.views(want)):
        assert float((a.double() - b).norm()) <= 8 * 2.0 ** -8 * float(b.norm())
    assert bool(((loss.double() - want_loss).abs() <= 8 * 2.0 ** -8 * (1 + want_loss.abs())).all())
    clipped = torch.full((m, model.P), math.nan, device="cuda")
    _, norms = model.gradient(params, ids, targets, clipped, max_norm=0.1)
    # (the embedding's part in flat is fp32, the others are the bf16 gradients themselves)
    want = flat.double().norm(dim=1)
    assert bool(((norms.double() - want).abs() <= 4 * 2.0 ** -24 * want).all())
    c = torch.clamp(0.1 / (want + 1e-6), max=1.0)[:, None]
    assert bool(((clipped.double() - flat.double() * c).abs() <= 5 * 2.0 ** -24 * flat.double().abs() * c + 2.0 ** -140).all())


def test_training_a_language_model_through_the_flat_path():
    g = _gen(77)
    m, T, V, D, F, tau, gamma = 4, 48, 100, 32, 64, 2, 0.1
    model = FlatLanguageModel(m, V, D, F)
    x0 = torch.randn(model.P, generator=g, device="cuda") * 0.15
    opt = OverlapLocalSGD("flat", flat_P=model.P, m=m, tau=tau, gamma=gamma, alpha=0.5, beta=0.5, x0=x0)
    params, flat = torch.empty((m, model.P), device="cuda"), torch.empty((m, model.P), device="cuda")
    for k in range(2 * tau):
        for i in range(m):
            opt.get_params(i, out=params[i])
        ids, targets = _batch(g, m, T, V)
        loss, norms = model.gradient(params, ids, targets, flat, max_norm=0.5)
        assert bool(torch.isfinite(loss).all()) and bool((norms > 0).all())
        before, step = params.clone(), flat.clone()
        opt.local_step_with_grads(flat)
        if k == 0:   # not a sync step: x <- x - gamma g, two roundings
            for i in range(m):
                got = opt.get_params(i, out=torch.empty(model.P, device="cuda")).double()
                want = before[i].double() - float(torch.tensor(gamma)) * step[i].double()
                assert bool(((got - want).abs() <= 2.0 ** -23 * (want.abs() + step[i].double().abs())).all())
        if (k + 1) % tau == 0:
            opt.period_sync()
    assert opt.iteration == 2 * tau
    lib.operators_join()
    opt.close()


def test_local_step_clips_its_gradients():
    g = _gen(5)
    m, P = 3, 1003
    x0 = torch.randn(P, generator=g, device="cuda")
    grad = torch.randn((m, P), generator=g, device="cuda") * torch.tensor([1.0, 1e-3, 4.0], device="cuda")[:, None]
    states = []
    for clip in (False, True):
        opt = OverlapLocalSGD("flat", flat_P=P, m=m, tau=2, gamma=0.1, alpha=0.5, mu=0.9, x0=x0)
        h = grad.clone()
        if clip:
            norms = opt.local_step_with_grads(h, max_norm=1.0)
        else:
            want, wn = lib.clip_grads(grad, 1.0)
            assert opt.local_step_with_grads(want) is None
        opt.join()
        states.append([opt.get_params(i).copy() for i in range(m)])
        opt.close()
    assert torch.equal(norms, wn) and torch.equal(h, want)
    assert all((a == b).all() for a, b in zip(*states))


# ------------------------------------------------------------------- streams, graphs, launches

def _calls(seed, m=2, T=70, V=3000, D=96, F=80):
    """Inputs (to be overwritten in place) and one function over all operators that returns all their outputs."""
    def make(s):
        g = _gen(s)
        ids, targets = _batch(g, m, T, V)
        return {"table": torch.randn((m, V, D), generator=g, device="cuda").bfloat16(), "ids": ids, "targets": targets,
                "wg": torch.randn((m, F, D), generator=g, device="cuda").bfloat16() * 0.1, "wu": torch.randn((m, F, D), generator=g, device="cuda").bfloat16() * 0.1,
                "logits": torch.randn((m, T, V), generator=g, device="cuda") * 2, "dh": torch.randn((m, T, F), generator=g, device="cuda").bfloat16(),
                "odd": torch.randn((m, F, D + 1), generator=g, device="cuda").bfloat16()[:, :, 1:]}

    def run(s):
        x = lib.embedding_forward(s["table"], s["ids"], 3.0)
        h, pre = lib.gated_forward(x, s["wg"], s["wu"], "gelu", save=True)
        dx, dwg, dwu = lib.gated_backward(s["dh"], x, s["wg"], s["wu"], pre, "gelu")
        odd = lib.gated_forward(x, s["odd"], s["wu"])
        dt = lib.embedding_backward(dx, s["ids"], V, 3.0)
        r = lib.token_logprobs(s["logits"], s["targets"], 4)
        dl = lib.token_logprobs_backward(r.logp, r.entropy, s["logits"], s["targets"], r.stats, r.entropy)
        clipped, norms = lib.clip_grads([dt, dwg, dwu], 0.7)
        return [x, h, pre, dx, dwg, dwu, odd, dt, *r, dl, *clipped, norms]

    return make, run


def test_operators_on_a_side_stream_and_captured():
    make, run = _calls(0)
    a, b = make(1), make(2)
    want = [run(a), run(b)]
    torch.cuda.synchronize()
    # two side streams at once
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(s1):
            g1 = run(a)
        with torch.cuda.stream(s2):
            g2 = run(b)
    torch.cuda.synchronize()
    for got, w in ((g1, want[0]), (g2, want[1])):
        assert all(torch.equal(x, y) for x, y in zip(got, w))
    # one graph each, replayed at once on both streams, then with the inputs exchanged
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
            assert all(torch.equal(x, y) for x, y in zip(outputs, w))
    lib.operators_join()


def test_operators_give_the_same_bits_in_plain_stream_order():
    make, run = _calls(0)
    a = make(3)
    want = run(a)
    before = lib.set_launch_overlap(False)
    try:
        got = run(a)
    finally:
        lib.set_launch_overlap(before)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_operators_on_the_legacy_stream_of_another_thread():
    import threading
    make, run = _calls(0)
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
        assert all(torch.equal(x, y) for x, y in zip(g, want))


def test_operators_captured_before_anything_else_ran(tmp_path):
    """The first call a process makes of every operator may be the one that is captured."""
    import subprocess
    import sys
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import sys, torch
sys.path[:0] = [%r, %r]
from test_gpu_operators_together import _calls
make, run = _calls(0)
a = make(1)
s = torch.cuda.Stream()
s.wait_stream(torch.cuda.current_stream())
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=s):
    got = run(a)
graph.replay()
torch.cuda.synchronize()
want = run(a)
assert all(torch.equal(x, y) for x, y in zip(got, want))
print("captured first: ok")
""" % (root, os.path.join(root, "tests"))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured first: ok" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("m,T,D,F", [(16, 128, 256, 256), (1, 512, 512, 1024), (2, 65, 1000, 72), (1, 3, 64, 40), (4, 300, 1024, 512), (1, 4000, 64, 64)])
def test_gated_gradients_side_by_side_keep_the_stream_s_order(m, T, D, F):
    """The two products of the backward pass overlap.  What follows them at once (a torch kernel, the next call in the same
    memory) sees both done: the same bits as with launches in plain order, over and over."""
    g = _gen(m + T)
    x, wg, wu = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, T, D), (m, F, D), (m, F, D)))
    dhs = [torch.randn((m, T, F), generator=g, device="cuda").bfloat16() for _ in range(3)]
    _, pre = lib.gated_forward(x, wg, wu, "gelu", save=True)

    def once(dh):
        dx, dwg, dwu = lib.gated_backward(dh, x, wg, wu, pre, "gelu")
        return dx + 1, dwg + 1, dwu + 1   # the gradients themselves go back to the allocator at once

    before = lib.set_launch_overlap(False)
    try:
        want = [once(dh) for dh in dhs]
        torch.cuda.synchronize()
    finally:
        lib.set_launch_overlap(before)
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(60):
        for dh, w in zip(dhs, want):
            for a, b in zip(once(dh), w):
                bad += (a != b).sum()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        got = [once(dh) for dh in dhs]
    for _ in range(20):
        graph.replay()
        for a, b in zip(got, want):
            for u, v in zip(a, b):
                bad += (u != v).sum()
    assert int(bad) == 0


def _forked(run, inputs, busy, side):
    """One set of calls on the current stream and one on `side`, each behind an event of the other stream: the operators' first
    launches follow event waits, not kernels."""
    here = torch.cuda.current_stream()
    a = {k: torch.empty_strided(v.shape, v.stride(), dtype=v.dtype, device=v.device).zero_() for k, v in inputs.items()}
    # what the side stream reads is written here, late
    for _ in range(4):
        busy = busy @ busy
    for k in a:
        a[k].copy_(inputs[k])
    side.wait_stream(here)
    with torch.cuda.stream(side):
        first = run(a)
    here.wait_stream(side)
    second = run(a)   # and again here, behind the side stream
    return first, second, busy


def test_operators_behind_events_of_other_streams():
    make, run = _calls(0)
    a = make(5)
    want = run(a)
    busy = torch.eye(4096, device="cuda")
    here, side = torch.cuda.Stream(), torch.cuda.Stream()
    here.wait_stream(torch.cuda.current_stream())
    kept = []
    with torch.cuda.stream(here):
        for _ in range(3):
            kept.append(_forked(run, a, busy, side))
    torch.cuda.synchronize()
    for first, second, _ in kept:
        assert all(torch.equal(x, y) for x, y in zip(first, want)) and all(torch.equal(x, y) for x, y in zip(second, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=here):
        first, second, _ = _forked(run, a, busy, side)
    for _ in range(3):
        for t in list(first) + list(second):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(first, want)) and all(torch.equal(x, y) for x, y in zip(second, want))
    lib.operators_join()


@pytest.mark.parametrize("m,T,D,F", [(3, 65, 333, 203), (1, 300, 1021, 77), (2, 130, 67, 640), (2, 4, 9, 3)])
@pytest.mark.parametrize("kind", ["silu", "relu"])
def test_gated_gradients_beside_their_copies_keep_the_stream_s_order(m, T, D, F, kind):
    """With rows that have to be copied the element-wise kernel runs beside the copies, on operands that were written just before
    and in memory that the call before used: the same bits as in plain order, eager and captured."""
    g = _gen(m * T + D)
    x, wg, wu = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, T, D), (m, F, D), (m, F, D)))
    dh = torch.randn((m, T, F), generator=g, device="cuda").bfloat16()

    def once(scale):
        xs, ws = x * scale, wg * scale
        _, pre = lib.gated_forward(xs, ws, wu, kind, save=True)
        both = lib.gated_backward(dh * scale, xs, ws, wu, pre, kind)
        dx = lib.gated_backward(dh, xs, ws, wu, pre, kind, want_d_w=False)[0]
        dw = lib.gated_backward(dh, xs, ws, wu, pre, kind, want_d_x=False)[1:]
        return [t + 1 for t in (*both, dx, *dw)]

    scales = (1.0, -2.0, 0.5)
    before = lib.set_launch_overlap(False)
    try:
        want = [once(s) for s in scales]
        torch.cuda.synchronize()
    finally:
        lib.set_launch_overlap(before)
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(30):
        for s, w in zip(scales, want):
            for a, b in zip(once(s), w):
                bad += (a != b).sum()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        got = [once(s) for s in scales]
    for _ in range(10):
        graph.replay()
        for a, b in zip(got, want):
            for u, v in zip(a, b):
                bad += (u != v).sum()
    assert int(bad) == 0
    lib.operators_join()
